// Attention and its gradients one row at a time: a warp per row, products on the CUDA cores, everything in 32 bits.
// Slots that a row may not see are never read, so whatever they hold (infinities, NaN) stays where it is.
#pragma once
#include <math.h>

#include "bload_layers.cuh"

namespace bload {
namespace rows {

// The slots that row i may see as a query ([lo, hi]), and the queries that may see slot i as a key.  Empty: lo > hi.
struct Span {
    int lo, hi;
};
__device__ __forceinline__ Span keys_of(const AttnParams& p, const int32_t* pos, int i, int lane)
{
    if (pos[i] < 0) return {1, 0};
    Span s{max(i - pos[i], 0), i};
    if (!p.causal) s.hi = warp_seq_end(pos, p.t, i, lane) - 1;
    s.lo = max(s.lo, i - (p.window - 1));
    s.hi = min(s.hi, i + (p.window - 1));
    return s;
}
__device__ __forceinline__ Span queries_of(const AttnParams& p, const int32_t* pos, int j, int lane)
{
    if (pos[j] < 0) return {1, 0};
    Span s{p.causal ? j : max(j - pos[j], 0), warp_seq_end(pos, p.t, j, lane) - 1};
    s.lo = max(s.lo, j - (p.window - 1));
    s.hi = min(s.hi, j + (p.window - 1));
    return s;
}

constexpr int kPer = 4;  // elements of a head per lane: heads of up to 128

template <typename T>
__device__ __forceinline__ void load_row(const T* row, int d, int lane, float (&x)[kPer])
{
#pragma unroll
    for (int e = 0; e < kPer; ++e) x[e] = lane * kPer + e < d ? to_float(row[lane * kPer + e]) : 0.0f;
}
template <typename T>
__device__ __forceinline__ void store_row(T* row, int d, int lane, const float (&x)[kPer])
{
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (lane * kPer + e < d) row[lane * kPer + e] = from_float<T>(x[e]);
}
__device__ __forceinline__ float dot(const float (&x)[kPer], const float (&y)[kPer])
{
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) s = fmaf(x[e], y[e], s);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}
// score from q.k; `inner` receives d score / d (scale q.k)
__device__ __forceinline__ float score_of(const AttnParams& p, float qk, float slope, int apart, float& inner)
{
    float s = qk * p.scale;
    inner = 1.0f;
    if (p.cap > 0.0f) {
        const float th = tanhf(s / p.cap);
        s = p.cap * th;
        inner = 1.0f - th * th;
    }
    return s - slope * (float)abs(apart);
}

template <typename T>
__device__ void forward_row(const AttnParams& p, const AttnTensors<T>& a, int64_t b, int h, int i, int lane)
{
    const Span sp = keys_of(p, p.pos + b * p.t, i, lane);
    const float slope = p.slopes ? p.slopes[h] : 0.0f;
    const int hk = h / p.group;
    float q[kPer], k[kPer], v[kPer], acc[kPer] = {}, m = -INFINITY, l = 0.0f, inner;
    load_row(a.q.at(b, i, h), p.d, lane, q);
    for (int j = sp.lo; j <= sp.hi; ++j) {
        load_row(a.k.at(b, j, hk), p.d, lane, k);
        const float s = score_of(p, dot(q, k), slope, i - j, inner);
        if (s == -INFINITY) continue;
        load_row(a.v.at(b, j, hk), p.d, lane, v);
        const float top = fmaxf(m, s), old = m == -INFINITY ? 0.0f : expf(m - top), w = expf(s - top);
        l = l * old + w;
#pragma unroll
        for (int e = 0; e < kPer; ++e) acc[e] = fmaf(w, v[e], acc[e] * old);
        m = top;
    }
    const float inv = l != 0.0f ? 1.0f / l : 0.0f;  // (NaN stays NaN)
#pragma unroll
    for (int e = 0; e < kPer; ++e) acc[e] *= inv;
    store_row(a.out.at(b, i, h), p.d, lane, acc);
    if (p.lse && lane == 0) p.lse[(b * p.heads + h) * p.t + i] = l != 0.0f ? m + logf(l) : -INFINITY;
}

template <typename T>
__device__ __forceinline__ float weight_of(float s, float lse)
{
    return s == -INFINITY ? 0.0f : expf(s - lse);
}

template <typename T>
__device__ float delta_row(const AttnParams& p, const AttnTensors<T>& a, int64_t b, int h, int i, int lane)
{
    float o[kPer], g[kPer];
    load_row(a.out_in.at(b, i, h), p.d, lane, o);
    load_row(a.dout.at(b, i, h), p.d, lane, g);
    return dot(o, g);
}

template <typename T>
__device__ void dq_row(const AttnParams& p, const AttnTensors<T>& a, int64_t b, int h, int i, int lane)
{
    const Span sp = keys_of(p, p.pos + b * p.t, i, lane);
    const float slope = p.slopes ? p.slopes[h] : 0.0f;
    const int hk = h / p.group;
    float q[kPer], g[kPer], k[kPer], v[kPer], acc[kPer] = {}, inner;
    load_row(a.q.at(b, i, h), p.d, lane, q);
    load_row(a.dout.at(b, i, h), p.d, lane, g);
    const float delta = delta_row(p, a, b, h, i, lane), lse = p.lse[(b * p.heads + h) * p.t + i];
    for (int j = sp.lo; j <= sp.hi; ++j) {
        load_row(a.k.at(b, j, hk), p.d, lane, k);
        load_row(a.v.at(b, j, hk), p.d, lane, v);
        const float s = score_of(p, dot(q, k), slope, i - j, inner);
        const float ds = weight_of<T>(s, lse) * (dot(g, v) - delta) * inner;
#pragma unroll
        for (int e = 0; e < kPer; ++e) acc[e] = fmaf(ds, k[e], acc[e]);
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) acc[e] *= p.scale;
    store_row(a.dq.at(b, i, h), p.d, lane, acc);
    if (lane == 0) p.delta[(b * p.heads + h) * p.t + i] = delta;
}

template <typename T>
__device__ void dkv_row(const AttnParams& p, const AttnTensors<T>& a, int64_t b, int hk, int j, int lane)
{
    const Span sp = queries_of(p, p.pos + b * p.t, j, lane);
    float k[kPer], v[kPer], q[kPer], g[kPer], dk[kPer] = {}, dv[kPer] = {}, inner;
    load_row(a.k.at(b, j, hk), p.d, lane, k);
    load_row(a.v.at(b, j, hk), p.d, lane, v);
    for (int h = hk * p.group; h < (hk + 1) * p.group; ++h) {
        const float slope = p.slopes ? p.slopes[h] : 0.0f;
        for (int i = sp.lo; i <= sp.hi; ++i) {
            load_row(a.q.at(b, i, h), p.d, lane, q);
            load_row(a.dout.at(b, i, h), p.d, lane, g);
            const float s = score_of(p, dot(q, k), slope, i - j, inner);
            const int64_t at = (b * p.heads + h) * p.t + i;
            const float w = weight_of<T>(s, p.lse[at]);
            const float ds = w * (dot(g, v) - p.delta[at]) * inner;
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                dv[e] = fmaf(w, g[e], dv[e]);
                dk[e] = fmaf(ds, q[e], dk[e]);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) dk[e] *= p.scale;
    store_row(a.dk.at(b, j, hk), p.d, lane, dk);
    store_row(a.dv.at(b, j, hk), p.d, lane, dv);
}

}  // namespace rows
}  // namespace bload

// k26_rotary: rotary positions that restart with every sequence of a packed block, and their gradient (the turn by
// minus the same angles).  A frame at position p has each pair (u, w) of its heads turned by p * inv_freq[i].
//
// Bytes only: every element is read and written once.  A thread has one piece of up to 16 bytes of a head (half layout: one of u
// and the one of w that belongs to it) in kHeads heads of a slot: it takes sine and cosine of its angles once for all of them and
// has all its loads under way before the first is used.  At 148 SMs and 6.5 TB/s there are some 340 instructions of time per
// warp and head of 16-bit elements; the turn takes 60, sine and cosine over four heads 45 (with sincosf the interleaved layout
// took 138 us instead of 121 for 16 x 4096 slots of 20 heads of 128, the half layout 116 either way: 5.8 TB/s).  A thread walks
// the slots with its unit and heads fixed: with a thread per slot, unit and group of heads the divisions that place it cost as
// much as the work (166 us).
// Pieces are as wide as alignment and the sizes of the turned part and of the rest allow: 16, 8 or 4 bytes, or one element.
#include "bload_internal.cuh"
#include "bload_layers.cuh"

namespace bload {

namespace {

constexpr int kHeads = 4, kThreads = 256;

template <int BYTES>
struct Word;
template <>
struct Word<16> {
    using type = uint4;
};
template <>
struct Word<8> {
    using type = uint2;
};
template <>
struct Word<4> {
    using type = uint32_t;
};
template <>
struct Word<2> {
    using type = uint16_t;
};

// WIDE: pieces lie on boundaries of their own size
template <typename T, int V, bool WIDE>
struct alignas(V * sizeof(T)) Piece {
    T x[V];
    using W = typename Word<V * sizeof(T)>::type;
    __device__ __forceinline__ void load(const T* p)
    {
        if (WIDE)
            *reinterpret_cast<W*>(x) = *reinterpret_cast<const W*>(p);
        else
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = p[e];
    }
    __device__ __forceinline__ void store(T* p) const
    {
        if (WIDE)
            *reinterpret_cast<W*>(p) = *reinterpret_cast<const W*>(x);
        else
#pragma unroll
            for (int e = 0; e < V; ++e) p[e] = x[e];
    }
};

// Sine and cosine: the angle less the nearest multiple k of pi / 2, in two multiply-adds (pi / 2 in two parts, the first product
// exact as long as k < 2^22), then the Taylor series of both to r^9 and r^8, and the quadrant.  Angles are below 3e5, where the 24 bits
// of 2 / pi place k within 0.01 of a's multiple: |r| <= 0.8, and the series' remainders are below 3e-8 (over 2 million angles the result
// was never off by more than 1e-7; up to 6e6 |r| grew to 1.03 and the error to 4.7e-7).  Larger angles go to sincosf.
__device__ __forceinline__ void sine_cosine(float a, float& sn, float& cs)
{
    if (!(fabsf(a) < 3.0e5f)) {
        sincosf(a, &sn, &cs);
        return;
    }
    constexpr float kRound = 12582912.0f;  // 1.5 * 2^23: adding it rounds to an integer, which then is in the low bits
    const float t = fmaf(a, 0.636619772f, kRound), k = t - kRound;
    const float r = fmaf(k, 4.37113883e-8f, fmaf(k, -1.57079637f, a)), z = r * r;
    float s = fmaf(fmaf(fmaf(fmaf(z, 1.0f / 362880, -1.0f / 5040), z, 1.0f / 120), z, -1.0f / 6), z * r, r);
    float c = fmaf(fmaf(fmaf(fmaf(z, 1.0f / 40320, -1.0f / 720), z, 1.0f / 24), z, -0.5f), z, 1.0f);
    const int quadrant = __float_as_int(t);
    if (quadrant & 1) {
        const float x = s;
        s = c;
        c = x;
    }
    sn = __int_as_float(__float_as_int(s) ^ (quadrant & 2) << 30);
    cs = __int_as_float(__float_as_int(c) ^ ((quadrant + 1) & 2) << 30);
}

// V: elements of a piece.  Units of a head: half layout, (d - n) / V (a turned one is two pieces); interleaved, d / V.
// blockIdx.y and the thread fix a unit and a group of heads; the thread walks the slots with them.
template <typename T, bool INTERLEAVED, int V, bool WIDE>
__global__ void __launch_bounds__(kThreads, 2) k26_rotary(const RotaryParams p, const Heads<const T> x, const Heads<T> y, int units)
{
    constexpr int kPairs = INTERLEAVED ? V / 2 : V;  // of a turned unit
    const int all = units * ((p.heads + kHeads - 1) / kHeads), first = blockIdx.y * kThreads, here = min(all - first, kThreads);
    const int at_once = kThreads / here;  // slots
    const int local = threadIdx.x / here, k = first + threadIdx.x - local * here;
    if (local >= at_once) return;
    const int group = k / units, unit = k - group * units, h0 = group * kHeads;
    const bool turns = unit < p.n / kPairs, two_pieces = !INTERLEAVED && turns;
    const int at = !INTERLEAVED && !turns ? p.n + unit * V : unit * V;
    const bool single = at + V > p.d;  // a last piece of an odd head has one element
    float freq[kPairs];
#pragma unroll
    for (int e = 0; e < kPairs; ++e) freq[e] = turns ? p.inv_freq[unit * kPairs + e] : 0.0f;
    const float factor = p.factor, back = p.gradient ? -p.factor : p.factor;
    const T* const x0 = x.data + h0 * x.head + at;
    T* const y0 = y.data + h0 * y.head + at;
    const int heads = min(p.heads - h0, kHeads);

    const int64_t step = (int64_t)gridDim.x * at_once;
    int64_t slot = (int64_t)blockIdx.x * at_once + local, q = slot / p.t;
    const int64_t step_q = step / p.t;
    int s = (int)(slot - q * p.t);
    const int step_s = (int)(step - step_q * p.t);
    int next = slot < p.slots ? p.pos[slot] : 0;
    for (; slot < p.slots; slot += step) {
        const int pos = next;
        const T* from = x0 + q * x.block + s * x.slot;
        T* to = y0 + q * y.block + s * y.slot;
        Piece<T, V, WIDE> u[kHeads], w[INTERLEAVED ? 1 : kHeads];
#pragma unroll
        for (int j = 0; j < kHeads; ++j)
            if (j < heads) {
                if (!single)
                    u[j].load(from + j * x.head);
                else
                    u[j].x[0] = from[j * x.head];
                if (two_pieces) w[INTERLEAVED ? 0 : j].load(from + j * x.head + p.n);
            }
        if (slot + step < p.slots) next = p.pos[slot + step];
        if (turns && pos >= 0) {
            float cs[kPairs], sn[kPairs];
#pragma unroll
            for (int e = 0; e < kPairs; ++e) {
                sine_cosine((float)pos * freq[e], sn[e], cs[e]);
                sn[e] *= back;
                cs[e] *= factor;
            }
#pragma unroll
            for (int j = 0; j < kHeads; ++j) {
                if (INTERLEAVED) {
#pragma unroll
                    for (int e = 0; e < kPairs; ++e) {
                        T &a = u[j].x[INTERLEAVED ? 2 * e : 0], &b = u[j].x[INTERLEAVED ? 2 * e + 1 : 0];
                        const float fa = to_float(a), fb = to_float(b);
                        a = from_float<T>(fa * cs[e] - fb * sn[e]);
                        b = from_float<T>(fb * cs[e] + fa * sn[e]);
                    }
                } else if (V == 1) {
                    T &a = u[j].x[0], &b = w[INTERLEAVED ? 0 : j].x[0];
                    const float fa = to_float(a), fb = to_float(b);
                    a = from_float<T>(fa * cs[0] - fb * sn[0]);
                    b = from_float<T>(fb * cs[0] + fa * sn[0]);
                } else {
#pragma unroll
                    for (int e = 0; e + 1 < V; e += 2) {
                        T *a = u[j].x + e, *b = w[INTERLEAVED ? 0 : j].x + e;
                        const int f = INTERLEAVED ? 0 : e;
                        const Two fa = two(to_float(a[0]), to_float(a[1])), fb = two(to_float(b[0]), to_float(b[1]));
                        const Two c = two(cs[f], cs[f + 1]), d = two(sn[f], sn[f + 1]), minus_d = two(-sn[f], -sn[f + 1]);
                        const float2 ra = one(fma(fa, c, fb * minus_d)), rb = one(fma(fb, c, fa * d));
                        a[0] = from_float<T>(ra.x);
                        a[1] = from_float<T>(ra.y);
                        b[0] = from_float<T>(rb.x);
                        b[1] = from_float<T>(rb.y);
                    }
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kHeads; ++j)
            if (j < heads) {
                if (!single)
                    u[j].store(to + j * y.head);
                else
                    to[j * y.head] = u[j].x[0];
                if (two_pieces) w[INTERLEAVED ? 0 : j].store(to + j * y.head + p.n);
            }
        q += step_q;
        s += step_s;
        if (s >= p.t) {
            s -= p.t;
            ++q;
        }
    }
}

template <typename T, bool INTERLEAVED, int V, bool WIDE>
cudaError_t launch(const RotaryParams& p, const Heads<const T>& x, const Heads<T>& y, cudaStream_t st)
{
    const int units = INTERLEAVED ? p.d / V + (p.d % V != 0) : (p.d - p.n) / V;
    const int all = units * ((p.heads + kHeads - 1) / kHeads), parts = (all + kThreads - 1) / kThreads;
    const int64_t slots_at_once = all < kThreads ? kThreads / all : 1;
    const int64_t wanted = (p.slots + slots_at_once - 1) / slots_at_once, most = (8 * 148 + parts - 1) / parts;
    k26_rotary<T, INTERLEAVED, V, WIDE><<<dim3((unsigned)(wanted < most ? wanted : most), parts), kThreads, 0, st>>>(p, x, y, units);
    count_launches(1);
    return cudaGetLastError();
}

}  // namespace

template <typename T>
cudaError_t launch_rotary(const RotaryParams& p, const Heads<const T>& x, const Heads<T>& y, cudaStream_t st)
{
    auto fits = [&](int v) {  // pieces of v elements
        auto rows = [&](const auto& h) {
            return reinterpret_cast<uintptr_t>(h.data) % (v * sizeof(T)) == 0 && h.block % v == 0 && h.slot % v == 0 && h.head % v == 0;
        };
        return rows(x) && rows(y) && p.d % v == 0 && (p.interleaved ? 2 * p.n : p.n) % v == 0;
    };
    constexpr int V = 16 / sizeof(T);
    if (p.interleaved) {
        if (fits(V)) return launch<T, true, V, true>(p, x, y, st);
        if (V > 4 && fits(4)) return launch<T, true, 4, true>(p, x, y, st);
        return fits(2) ? launch<T, true, 2, true>(p, x, y, st) : launch<T, true, 2, false>(p, x, y, st);
    }
    if (fits(V)) return launch<T, false, V, true>(p, x, y, st);
    if (V > 4 && fits(4)) return launch<T, false, 4, true>(p, x, y, st);
    return fits(2) ? launch<T, false, 2, true>(p, x, y, st) : launch<T, false, 1, true>(p, x, y, st);
}
template cudaError_t launch_rotary<float>(const RotaryParams&, const Heads<const float>&, const Heads<float>&, cudaStream_t);
template cudaError_t launch_rotary<__half>(const RotaryParams&, const Heads<const __half>&, const Heads<__half>&, cudaStream_t);
template cudaError_t launch_rotary<__nv_bfloat16>(const RotaryParams&, const Heads<const __nv_bfloat16>&,
                                                  const Heads<__nv_bfloat16>&, cudaStream_t);

}  // namespace bload

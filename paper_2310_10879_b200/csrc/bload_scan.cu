// k37_scan: selective state-space scan along the slots of packed blocks, restarted at every sequence start; k39_scan_grad: its
// gradient; k38_scan_join: states between segments; k40_scan_sums: db and dc from the CTAs' sums; k41_scan_step: one new frame each.
//
// Per slot, channel and state one exponential and some four multiply-adds forward: with 16 states that is more than the bytes of
// x, dt, z and y take (16 exponentials a cycle and SM), so the kernels are built around the arithmetic.  A lane has two channels and
// kStates (2 or 4) of their states, packed in pairs; kLanes lanes share a channel.  A CTA of 128 threads has 256 / kLanes channels of a
// block and walks it in runs of 16 slots: delta and delta x of a run are computed once per (slot, channel), by threads that have
// neighbouring channels of a slot as they lie in memory, and go to the lanes through shared memory; sums over the states come back that
// way.  The chain from slot to slot is one multiply-add per state.
//
// Where there are too few walks for the machine, the slots are cut into segments, a CTA each.  k37 and k39 first run over the part
// of a segment that its successor hears of (from the last sequence start on; nothing if a sequence starts there) without output, k38
// joins what they leave, and the walk proper starts from that.
//
// The gradient walks backwards, run by run, from the states that the forward call kept at the start of each run: it rebuilds the
// run's states into shared memory (each thread its own), then goes through them from the last slot to the first.  Sums over
// channels (db, dc) are shared out over the lanes of a warp, then over the CTA's warps, and written once per CTA; k40 adds the CTAs'.
#include <math.h>

#include <type_traits>

#include "bload_internal.cuh"
#include "bload_layers.cuh"

namespace bload {

namespace {

constexpr int kRun = BLOAD_SCAN_RUN, kThreads = 128, kWarps = 4;
constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// LANES share a channel, each with STATES of its states
template <int LANES, int STATES>
struct Split {
    static constexpr int kLanes = LANES, kStates = STATES, kPairs = STATES / 2, kAll = LANES * STATES;
    static constexpr int kChannels = 256 / LANES;   // of a CTA
    static constexpr int kV = kChannels / 8;        // of a thread, where a run lies as in memory: 8 threads per slot
    static constexpr int kPerWarp = 64 / LANES;
    static constexpr int kGroup = LANES < 4 ? LANES : 4;  // slots whose sums over states are taken together
};

// Scratch: per boundary between segments and block what crosses it (0 nothing, 1 a state that nothing before the segment
// enters, 2 one that depends on what entered), the sum of delta over the segment, the state; sums over frames of each CTA; sums
// over the channels of each CTA, [group of channels][block][slot][2 * states].
struct ScanWork {
    int32_t* kind;  // [segments][blocks]
    float* delta;   // [segments][blocks][channels]
    float* state;   // [segments][blocks][channels][states]
    float* frames;  // [segments][blocks][channels * (states + 2)]
    float* across;
    size_t bytes;
};
struct ScanCuts {
    int segments, groups, stride;  // stride: floats of `across` per slot
};

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// exp(delta a) of two states, from delta and a log2(e)
__device__ __forceinline__ Two decay(Two delta, Two a)
{
    const float2 x = one(delta * a);
    return two(ex2(x.x), ex2(x.y));
}

// softplus(v) = max(v, 0) + log1p(e) and sigmoid(v) from e = exp(-|v|), which is in (0, 1].  The product with log2(e) keeps what its
// rounding loses (without: up to 1e-6 of e for v = -10).  log1p(e) = 2 atanh(s), s = e / (2 + e) <= 1/3, by its series to s^15: the
// rest is below 2e-9 of it.
__device__ __forceinline__ void softplus_of(float v, float& value, float& slope)
{
    const float x = fabsf(v) * -kLog2E, rest = fmaf(fabsf(v), -kLog2E, -x) + fabsf(v) * -1.925963033e-8f;
    float e = ex2(x);
    e = e > 0.0f ? fmaf(e, rest * kLn2, e) : e;
    float r, q;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(2.0f + e));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(q) : "f"(1.0f + e));
    const float s = e * r, z = s * s;
    float p = fmaf(z, 1.0f / 15, 1.0f / 13);
    p = fmaf(z, p, 1.0f / 11);
    p = fmaf(z, p, 1.0f / 9);
    p = fmaf(z, p, 1.0f / 7);
    p = fmaf(z, p, 1.0f / 5);
    p = fmaf(z, p, 1.0f / 3);
    const float l = 2.0f * fmaf(s * z, p, s);
    value = v != v ? v : fmaxf(v, 0.0f) + l;
    slope = v < 0.0f ? e * q : q;
}
__device__ __forceinline__ void delta_of(const ScanParams& p, float v, float& value, float& slope)
{
    value = v;
    slope = 1.0f;
    if (p.softplus) softplus_of(v, value, slope);
}

// Where a thread stands: as the lanes hold states, and as a run lies in memory.
template <typename S>
struct Place {
    int lane, warp, part;    // part: which of the states
    int c_lane;              // first of the lane's two channels in the CTA
    int slot, c_mem;         // of the run, first of kV channels in the CTA
    int64_t c0;              // first channel of the CTA
    int there;               // of the kV channels
    int64_t q;               // block
    int segment, first, end; // runs of the segment
    __device__ __forceinline__ Place(const ScanParams& p, const ScanCuts& cuts)
    {
        lane = threadIdx.x & 31;
        warp = threadIdx.x >> 5;
        part = lane % S::kLanes;
        c_lane = warp * S::kPerWarp + lane / S::kLanes * 2;
        slot = threadIdx.x >> 3;
        c_mem = (threadIdx.x & 7) * S::kV;
        const int64_t at = blockIdx.x / cuts.groups;
        c0 = (int64_t)(blockIdx.x - at * cuts.groups) * S::kChannels;
        there = (int)max((int64_t)0, min(p.channels - c0 - c_mem, (int64_t)S::kV));
        segment = (int)(at / p.blocks);
        q = at - segment * p.blocks;
        const int runs = (p.t + kRun - 1) / kRun;
        first = (int)((int64_t)runs * segment / cuts.segments);
        end = (int)((int64_t)runs * (segment + 1) / cuts.segments);
    }
};

// a[channel][state], of the lane's two channels, as pairs of states; 0 where there is none
template <typename S>
__device__ __forceinline__ void load_a(const ScanParams& p, const Place<S>& at, float factor, Two (&a)[2][S::kPairs])
{
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int k = 0; k < S::kPairs; ++k) {
            const int64_t ch = at.c0 + at.c_lane + c;
            const int n = at.part * S::kStates + 2 * k;
            const float* const from = p.a + ch * p.states + n;
            const bool on = ch < p.channels;
            a[c][k] = two(on && n < p.states ? from[0] * factor : 0.0f, on && n + 1 < p.states ? from[1] * factor : 0.0f);
        }
}

// states [channel][state] in memory, from `base` of the CTA's block (or sequence) on
template <typename S>
__device__ __forceinline__ void load_states(const ScanParams& p, const Place<S>& at, const float* base, Two (&h)[2][S::kPairs])
{
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int k = 0; k < S::kPairs; ++k) {
            const int64_t ch = at.c0 + at.c_lane + c;
            const int n = at.part * S::kStates + 2 * k;
            const float* const from = base + ch * p.states + n;
            const bool on = ch < p.channels;
            h[c][k] = two(on && n < p.states ? from[0] : 0.0f, on && n + 1 < p.states ? from[1] : 0.0f);
        }
}
template <typename S>
__device__ __forceinline__ void store_states(const ScanParams& p, const Place<S>& at, float* base, const Two (&h)[2][S::kPairs])
{
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int64_t ch = at.c0 + at.c_lane + c;
        if (ch >= p.channels) continue;
        const int n0 = at.part * S::kStates;
        float* const to = base + ch * p.states + n0;
        if (S::kStates == 4 && p.states % 4 == 0 && reinterpret_cast<uintptr_t>(base) % 16 == 0) {
            if (n0 < p.states) {
                const float2 x = one(h[c][0]), y = one(h[c][S::kPairs - 1]);
                *reinterpret_cast<float4*>(to) = make_float4(x.x, x.y, y.x, y.y);
            }
            continue;
        }
#pragma unroll
        for (int k = 0; k < S::kPairs; ++k) {
            const float2 x = one(h[c][k]);
            if (n0 + 2 * k < p.states) to[2 * k] = x.x;
            if (n0 + 2 * k + 1 < p.states) to[2 * k + 1] = x.y;
        }
    }
}

// b and c of a run, [slot][b, c][kAll] in shared memory; 0 on padding
template <typename T, typename S, bool B, bool C>
struct Rows {
    static constexpr int kEach = kRun * S::kAll / kThreads;
    T b[B ? kEach : 1], c[C ? kEach : 1];
    __device__ __forceinline__ void load(const ScanParams& p, const ScanTensors<T>& a, int64_t q, int s0, unsigned valid)
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int at = threadIdx.x + i * kThreads, slot = at / S::kAll, n = at % S::kAll;
            const bool on = ((valid >> slot) & 1) && n < p.states;
            const int64_t s = s0 + slot;
            if (B) b[i] = on ? a.b.at(q, s)[n] : from_float<T>(0.0f);
            if (C) c[i] = on ? a.c.at(q, s)[n] : from_float<T>(0.0f);
        }
    }
    __device__ __forceinline__ void store(float (*to)[2][S::kAll]) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int at = threadIdx.x + i * kThreads, slot = at / S::kAll, n = at % S::kAll;
            if (B) to[slot][0][n] = to_float(b[i]);
            if (C) to[slot][1][n] = to_float(c[i]);
        }
    }
};
template <typename S>
__device__ __forceinline__ void pairs_of(const float* from, Two (&x)[S::kPairs])
{
    if (S::kStates == 4) {
        const float4 v = *reinterpret_cast<const float4*>(from);
        x[0] = two(v.x, v.y);
        x[S::kPairs - 1] = two(v.z, v.w);
    } else {
        const float2 v = *reinterpret_cast<const float2*>(from);
        x[0] = two(v.x, v.y);
    }
}

// positions of a run: bit s of `valid`: slot s is a frame, of `starts`: it starts a sequence (or is none)
__device__ __forceinline__ void run_masks(const int32_t* pos, int t, int s0, int lane, unsigned& valid, unsigned& starts)
{
    const int here = lane < kRun && s0 + lane < t ? pos[s0 + lane] : -1;
    valid = __ballot_sync(0xffffffffu, here >= 0) & ((1u << kRun) - 1);
    starts = __ballot_sync(0xffffffffu, here <= 0) & ((1u << kRun) - 1);
}

// OUTPUT false: leaves what crosses the segment's end (kind, delta, state of ScanWork).
template <typename T, typename S, bool OUTPUT>
__global__ void __launch_bounds__(kThreads) k37_scan(const ScanParams p, const ScanTensors<T> a, const ScanCuts cuts, const ScanWork work, bool wide)
{
    __shared__ __align__(16) float2 prepared[kRun][S::kChannels];  // delta, delta x
    __shared__ __align__(16) float rows[kRun][2][S::kAll];
    __shared__ __align__(8) float sums[OUTPUT ? kRun : 1][OUTPUT ? S::kChannels : 2];

    const Place<S> at(p, cuts);
    const int32_t* const pos = p.pos + at.q * p.t;
    const int runs = (p.t + kRun - 1) / kRun;
    int run = at.first;
    const int64_t cell = (int64_t)at.segment * p.blocks + at.q, per = p.channels * p.states;
    if (!OUTPUT) {
        const int edge = at.end * kRun;  // of a segment that is not the last: below t
        if (at.segment == cuts.segments - 1 || at.first == at.end || pos[edge] <= 0) {
            if (threadIdx.x == 0) work.kind[cell] = 0;
            return;
        }
        const int start = edge - min(pos[edge], edge);
        run = max(at.first, min(start / kRun, at.end - 1));
        if (threadIdx.x == 0) work.kind[cell] = start < at.first * kRun ? 2 : 1;
    }
    Two A[2][S::kPairs], h[2][S::kPairs];
    load_a(p, at, kLog2E, A);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int k = 0; k < S::kPairs; ++k) h[c][k] = zero();
    if (OUTPUT && at.segment > 0 && at.first < at.end && pos[at.first * kRun] > 0)
        load_states(p, at, work.state + (cell - p.blocks) * per, h);

    float bias[S::kV], skip[S::kV], passed[2] = {0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < S::kV; ++e) {
        const int64_t c = at.c0 + at.c_mem + e;
        bias[e] = p.dt_bias && e < at.there ? p.dt_bias[c] : 0.0f;
        skip[e] = OUTPUT && p.d && e < at.there ? p.d[c] : 0.0f;
    }
    const bool gated = OUTPUT && a.z.data;

    Elements<T, S::kV> x, dt, z;
    Rows<T, S, true, OUTPUT> bc;
    unsigned valid, starts;
    auto fetch = [&](int r) {
        const int s0 = r * kRun;
        run_masks(pos, p.t, s0, at.lane, valid, starts);
        const bool on = (valid >> at.slot) & 1;
        const int64_t s = s0 + at.slot, c = at.c0 + at.c_mem;
        x.clear();
        dt.clear();
        z.clear();
        if (on) {
            x.load(a.x.at(at.q, s) + c, at.there, wide);
            dt.load(a.dt.at(at.q, s) + c, at.there, wide);
            if (gated) z.load(a.z.at(at.q, s) + c, at.there, wide);
        }
        bc.load(p, a, at.q, s0, valid);
    };
    if (run < at.end) fetch(run);
    for (; run < at.end; ++run) {
        const int s0 = run * kRun;
        const unsigned now_valid = valid, now_starts = starts;
        const Elements<T, S::kV> now_x = x, now_z = z;
        {
            const bool on = (valid >> at.slot) & 1;
#pragma unroll
            for (int e = 0; e < S::kV; ++e) {
                float delta, slope;
                delta_of(p, dt.get(e) + bias[e], delta, slope);
                if (!on || e >= at.there) delta = 0.0f;
                prepared[at.slot][at.c_mem + e] = make_float2(delta, delta * x.get(e));
            }
        }
        bc.store(rows);
        if (OUTPUT && p.carry) store_states(p, at, p.carry + (at.q * runs + run) * per, h);
        __syncthreads();
        if (run + 1 < at.end) fetch(run + 1);

#pragma unroll 1
        for (int g = 0; g < kRun; g += S::kGroup) {
            float y[2][S::kGroup];
#pragma unroll
            for (int i = 0; i < S::kGroup; ++i) {
                const int s = g + i;
                const float4 d = *reinterpret_cast<const float4*>(&prepared[s][at.c_lane]);
                Two B[S::kPairs], C[S::kPairs];
                pairs_of<S>(&rows[s][0][at.part * S::kStates], B);
                if (OUTPUT) pairs_of<S>(&rows[s][1][at.part * S::kStates], C);
                const Two delta[2] = {two(d.x, d.x), two(d.z, d.z)}, u[2] = {two(d.y, d.y), two(d.w, d.w)};
                if ((now_starts >> s) & 1) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int k = 0; k < S::kPairs; ++k) h[c][k] = zero();
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    Two sum = zero();
#pragma unroll
                    for (int k = 0; k < S::kPairs; ++k) {
                        h[c][k] = fma(decay(delta[c], A[c][k]), h[c][k], u[c] * B[k]);
                        if (OUTPUT) sum = k ? fma(h[c][k], C[k], sum) : h[c][k] * C[k];
                    }
                    y[c][i] = one(sum).x + one(sum).y;
                }
                if (!OUTPUT) {
                    passed[0] += d.x;
                    passed[1] += d.z;
                }
                if (OUTPUT && p.last && ((now_valid >> s) & 1)) {
                    const int here = s0 + s;
                    if (here + 1 >= p.t || pos[here + 1] <= 0) {  // the sequence ends (uniform)
                        const int64_t id = p.seq_id[at.q * p.t + here];
                        if (id >= 0 && id < p.n_seq) store_states(p, at, p.last + id * per, h);
                    }
                }
            }
            if (OUTPUT) {
                // over the channel's lanes: they end with a slot each (beyond four lanes, with copies of four)
                int which[2] = {0, 0};
#pragma unroll
                for (int c = 0; c < 2; ++c) {
#pragma unroll
                    for (int bit = S::kLanes / 2, n = S::kGroup; bit; bit /= 2) {
                        if (n > 1) {
                            n /= 2;
                            const bool upper = at.lane & bit;
#pragma unroll
                            for (int i = 0; i < n; ++i) {
                                const float send = upper ? y[c][i] : y[c][i + n], keep = upper ? y[c][i + n] : y[c][i];
                                y[c][i] = keep + __shfl_xor_sync(0xffffffffu, send, bit);
                            }
                            if (upper) which[c] += n;
                        } else {
                            y[c][0] += __shfl_xor_sync(0xffffffffu, y[c][0], bit);
                        }
                    }
                }
                if (S::kLanes <= S::kGroup || at.part % (S::kLanes / S::kGroup) == 0)
                    *reinterpret_cast<float2*>(&sums[g + which[0]][at.c_lane]) = make_float2(y[0][0], y[1][0]);
            }
        }
        __syncthreads();
        if (OUTPUT && s0 + at.slot < p.t) {
            const bool on = (now_valid >> at.slot) & 1;
            Elements<T, S::kV> out;
#pragma unroll
            for (int e = 0; e < S::kV; ++e) {
                float v = fmaf(skip[e], now_x.get(e), sums[at.slot][at.c_mem + e]);
                if (gated) v *= now_z.get(e) * sigmoid_of(now_z.get(e));
                out.set(e, on ? v : 0.0f);
            }
            out.store(a.y.at(at.q, s0 + at.slot) + at.c0 + at.c_mem, at.there, wide);
        }
    }
    if (!OUTPUT) {
        store_states(p, at, work.state + cell * per, h);
        if (at.part == 0) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (at.c0 + at.c_lane + c < p.channels) work.delta[cell * p.channels + at.c0 + at.c_lane + c] = passed[c];
        }
    }
}

// What crosses a boundary, in the order of the walk: what a segment leaves by itself and, where nothing starts in it, what
// entered it times the decay over all of its slots.
__global__ void __launch_bounds__(256) k38_scan_join(const ScanParams p, const ScanCuts cuts, const ScanWork work, bool backwards)
{
    const int64_t per = p.channels * p.states, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= p.blocks * per) return;
    const int64_t q = i / per, c = (i - q * per) / p.states;
    const float a = p.a[i - q * per] * kLog2E;
    float state = 0.0f;
    for (int k = 0; k < cuts.segments; ++k) {
        const int64_t cell = (int64_t)(backwards ? cuts.segments - 1 - k : k) * p.blocks + q;
        const int kind = work.kind[cell];
        if (kind == 0) {
            state = 0.0f;
            continue;
        }
        float* const at = work.state + cell * per + (i - q * per);
        state = kind == 2 ? fmaf(ex2(work.delta[cell * p.channels + c] * a), state, *at) : *at;
        *at = state;
    }
}

// dy times the gate, and what the gate's gradient needs
__device__ __forceinline__ float silu_slope(float z, float sig) { return sig * fmaf(z, 1.0f - sig, 1.0f); }

template <typename S>
struct GradShared {
    float4 kept[kRun][S::kPairs][kThreads];     // exp(delta a) h of the slot before, of a thread's states: pair by pair, both channels
    float4 prepared[kRun][S::kChannels];        // delta, delta x, gated dy; then sums over states: g b, g a h, h c (w stays: delta)
    float rows[kRun][2][S::kAll];
    float across[kWarps][kRun][2 * S::kAll];    // db, dc of a warp's channels
};

// OUTPUT false: leaves what crosses the segment's first slot, backwards.
template <typename T, typename S, bool OUTPUT>
__global__ void __launch_bounds__(kThreads) k39_scan_grad(const ScanParams p, const ScanTensors<T> a, const ScanCuts cuts, const ScanWork work, bool wide)
{
    extern __shared__ __align__(16) uint8_t shared_bytes[];
    GradShared<S>& sh = *reinterpret_cast<GradShared<S>*>(shared_bytes);

    const Place<S> at(p, cuts);
    const int32_t* const pos = p.pos + at.q * p.t;
    const int runs = (p.t + kRun - 1) / kRun;
    const int64_t cell = (int64_t)at.segment * p.blocks + at.q, per = p.channels * p.states;
    int run = at.end - 1;
    if (!OUTPUT) {
        const int edge = at.first * kRun;
        if (at.segment == 0 || at.first == at.end || pos[edge] <= 0) {
            if (threadIdx.x == 0) work.kind[cell] = 0;
            return;
        }
        const int stop = warp_seq_end(pos, p.t, edge, at.lane);  // in (edge, t]
        run = min((stop - 1) / kRun, at.end - 1);
        // (the sequence goes on into the next segment: what enters there is handed on)
        if (threadIdx.x == 0) work.kind[cell] = stop > at.end * kRun && at.end < runs ? 2 : 1;
    }
    Two A[2][S::kPairs], e[2][S::kPairs], dA[2][S::kPairs];  // e: exp(delta a) g of the slot behind
    load_a(p, at, kLog2E, A);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int k = 0; k < S::kPairs; ++k) e[c][k] = dA[c][k] = zero();
    if (OUTPUT && at.segment + 1 < cuts.segments && at.first < at.end && pos[at.end * kRun] > 0)
        load_states(p, at, work.state + (cell + p.blocks) * per, e);

    float bias[S::kV], skip[S::kV], d_skip[S::kV], d_bias[S::kV], passed[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < S::kV; ++i) {
        const int64_t c = at.c0 + at.c_mem + i;
        bias[i] = p.dt_bias && i < at.there ? p.dt_bias[c] : 0.0f;
        skip[i] = p.d && i < at.there ? p.d[c] : 0.0f;
        d_skip[i] = d_bias[i] = 0.0f;
    }
    const bool gated = a.z.data != nullptr;

    for (; run >= at.first; --run) {
        const int s0 = run * kRun;
        unsigned valid, starts;
        run_masks(pos, p.t, s0, at.lane, valid, starts);
        const bool on = (valid >> at.slot) & 1;
        const int64_t s_mem = s0 + at.slot, c_mem = at.c0 + at.c_mem;
        Elements<T, S::kV> x, dt, z, dy;
        x.clear();
        dt.clear();
        z.clear();
        dy.clear();
        if (on) {
            if (OUTPUT) x.load(a.x.at(at.q, s_mem) + c_mem, at.there, wide);
            dt.load(a.dt.at(at.q, s_mem) + c_mem, at.there, wide);
            dy.load(a.dy.at(at.q, s_mem) + c_mem, at.there, wide);
            if (gated) z.load(a.z.at(at.q, s_mem) + c_mem, at.there, wide);
        }
        Rows<T, S, OUTPUT, true> bc;
        bc.load(p, a, at.q, s0, valid);
        Two h[2][S::kPairs];
        if (OUTPUT) load_states(p, at, p.carry + (at.q * runs + run) * per, h);
#pragma unroll
        for (int i = 0; i < S::kV; ++i) {
            float delta, slope, g = dy.get(i);
            delta_of(p, dt.get(i) + bias[i], delta, slope);
            if (!on || i >= at.there) delta = 0.0f;
            if (gated) g *= z.get(i) * sigmoid_of(z.get(i));
            sh.prepared[at.slot][at.c_mem + i] = make_float4(delta, delta * x.get(i), g, delta);
        }
        bc.store(sh.rows);
        __syncthreads();

        if (OUTPUT) {
#pragma unroll 4
            for (int s = 0; s < kRun; ++s) {
                const float2 d0 = *reinterpret_cast<const float2*>(&sh.prepared[s][at.c_lane]), d1 = *reinterpret_cast<const float2*>(&sh.prepared[s][at.c_lane + 1]);
                Two B[S::kPairs];
                pairs_of<S>(&sh.rows[s][0][at.part * S::kStates], B);
                const Two delta[2] = {two(d0.x, d0.x), two(d1.x, d1.x)}, u[2] = {two(d0.y, d0.y), two(d1.y, d1.y)};
                const bool start = (starts >> s) & 1;
#pragma unroll
                for (int k = 0; k < S::kPairs; ++k) {
                    float2 w[2];
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const Two v = start ? zero() : decay(delta[c], A[c][k]) * h[c][k];
                        w[c] = one(v);
                        h[c][k] = fma(u[c], B[k], v);
                    }
                    sh.kept[s][k][threadIdx.x] = make_float4(w[0].x, w[0].y, w[1].x, w[1].y);
                }
            }
        }

#pragma unroll 1
        for (int g0 = kRun - S::kGroup; g0 >= 0; g0 -= S::kGroup) {
            float sum[3][2][S::kGroup];  // over states: g b, g a h, h c
#pragma unroll
            for (int i = S::kGroup - 1; i >= 0; --i) {
                const int s = g0 + i;
                const float4 d0 = sh.prepared[s][at.c_lane], d1 = sh.prepared[s][at.c_lane + 1];
                Two B[S::kPairs], C[S::kPairs];
                if (OUTPUT) pairs_of<S>(&sh.rows[s][0][at.part * S::kStates], B);
                pairs_of<S>(&sh.rows[s][1][at.part * S::kStates], C);
                const Two delta[2] = {two(d0.x, d0.x), two(d1.x, d1.x)}, u[2] = {two(d0.y, d0.y), two(d1.y, d1.y)},
                          dv[2] = {two(d0.z, d0.z), two(d1.z, d1.z)};
                const bool start = (starts >> s) & 1;
                Two gb[2], gah[2], hc[2];
                float v[4 * S::kPairs];
#pragma unroll
                for (int k = 0; k < S::kPairs; ++k) {
                    Two w[2], db, dc;
                    if (OUTPUT) {
                        const float4 kept = sh.kept[s][k][threadIdx.x];
                        w[0] = two(kept.x, kept.y);
                        w[1] = two(kept.z, kept.w);
                    }
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const Two g = fma(dv[c], C[k], e[c][k]);
                        if (OUTPUT) {
                            const Two now = fma(u[c], B[k], w[c]), gw = g * w[c];
                            hc[c] = k ? fma(now, C[k], hc[c]) : now * C[k];
                            dc = c ? fma(dv[c], now, dc) : dv[c] * now;
                            db = c ? fma(u[c], g, db) : u[c] * g;
                            gb[c] = k ? fma(g, B[k], gb[c]) : g * B[k];
                            gah[c] = k ? fma(gw, A[c][k], gah[c]) : gw * A[c][k];
                            dA[c][k] = fma(gw, delta[c], dA[c][k]);
                        }
                        e[c][k] = start ? zero() : decay(delta[c], A[c][k]) * g;
                    }
                    if (OUTPUT) {
                        v[2 * k] = one(db).x;
                        v[2 * k + 1] = one(db).y;
                        v[2 * S::kPairs + 2 * k] = one(dc).x;
                        v[2 * S::kPairs + 2 * k + 1] = one(dc).y;
                    }
                }
                if (OUTPUT) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        sum[0][c][i] = one(gb[c]).x + one(gb[c]).y;
                        sum[1][c][i] = one(gah[c]).x + one(gah[c]).y;
                        sum[2][c][i] = one(hc[c]).x + one(hc[c]).y;
                    }
                    int first = 0;
                    share_sums<4 * S::kPairs, 16, S::kLanes>(v, at.lane, first);
                    constexpr int kLeft = Shared<4 * S::kPairs, S::kLanes>::kLeft;
                    // (where the warp has more lanes for a state than values, copies write the same)
#pragma unroll
                    for (int j = 0; j < kLeft; ++j) {
                        const int n = first + j, of_c = n >= 2 * S::kPairs;
                        sh.across[at.warp][s][of_c * S::kAll + at.part * S::kStates + n - of_c * 2 * S::kPairs] = v[j];
                    }
                } else {
                    passed[0] += d0.x;
                    passed[1] += d1.x;
                }
            }
            if (OUTPUT) {
                int which = 0;
#pragma unroll
                for (int m = 0; m < 3; ++m)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        which = 0;
#pragma unroll
                        for (int bit = S::kLanes / 2, n = S::kGroup; bit; bit /= 2) {
                            float* const y = sum[m][c];
                            if (n > 1) {
                                n /= 2;
                                const bool upper = at.lane & bit;
#pragma unroll
                                for (int i = 0; i < n; ++i) {
                                    const float send = upper ? y[i] : y[i + n], keep = upper ? y[i + n] : y[i];
                                    y[i] = keep + __shfl_xor_sync(0xffffffffu, send, bit);
                                }
                                if (upper) which += n;
                            } else {
                                y[0] += __shfl_xor_sync(0xffffffffu, y[0], bit);
                            }
                        }
                    }
                __syncwarp();  // all lanes have read these slots
                if (S::kLanes <= S::kGroup || at.part % (S::kLanes / S::kGroup) == 0) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float4& to = sh.prepared[g0 + which][at.c_lane + c];
                        *reinterpret_cast<float2*>(&to) = make_float2(sum[0][c][0], sum[1][c][0]);
                        to.z = sum[2][c][0];
                    }
                }
            }
        }
        __syncthreads();
        if (OUTPUT && s_mem < p.t) {
            Elements<T, S::kV> dx, ddt, dz;
#pragma unroll
            for (int i = 0; i < S::kV; ++i) {
                const float4 r = sh.prepared[at.slot][at.c_mem + i];
                float value, slope, dv = dy.get(i);
                delta_of(p, dt.get(i) + bias[i], value, slope);
                const float xi = x.get(i);
                if (gated) {
                    const float zi = z.get(i), sig = sigmoid_of(zi);
                    dz.set(i, on ? dv * fmaf(skip[i], xi, r.z) * silu_slope(zi, sig) : 0.0f);
                    dv *= zi * sig;
                }
                const float dd = on ? fmaf(xi, r.x, r.y * kLn2) * slope : 0.0f;
                ddt.set(i, dd);
                dx.set(i, on ? fmaf(r.w, r.x, skip[i] * dv) : 0.0f);
                d_bias[i] += dd;
                if (on) d_skip[i] = fmaf(dv, xi, d_skip[i]);
            }
            dx.store(a.dx.at(at.q, s_mem) + c_mem, at.there, wide);
            ddt.store(a.ddt.at(at.q, s_mem) + c_mem, at.there, wide);
            if (gated) dz.store(a.dz.at(at.q, s_mem) + c_mem, at.there, wide);
        }
        if (OUTPUT) {
            const int n2 = 2 * S::kAll;
            float* const to = work.across + (((blockIdx.x % cuts.groups) * p.blocks + at.q) * (int64_t)p.t + s0) * n2;
            for (int i = threadIdx.x; i < min(kRun, p.t - s0) * n2; i += kThreads) {
                float v = 0.0f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) v += (&sh.across[w][0][0])[i];
                to[i] = v;
            }
        }
        __syncthreads();
    }
    if (!OUTPUT) {
        store_states(p, at, work.state + cell * per, e);
        if (at.part == 0) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (at.c0 + at.c_lane + c < p.channels) work.delta[cell * p.channels + at.c0 + at.c_lane + c] = passed[c];
        }
        return;
    }
    float* const frames = work.frames + cell * (per + 2 * p.channels);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int k = 0; k < S::kPairs; ++k) {
            const int64_t ch = at.c0 + at.c_lane + c;
            const int n = at.part * S::kStates + 2 * k;
            if (ch >= p.channels) continue;
            if (n < p.states) frames[ch * p.states + n] = one(dA[c][k]).x;
            if (n + 1 < p.states) frames[ch * p.states + n + 1] = one(dA[c][k]).y;
        }
    // the sixteen slots' threads of a channel, in their order
    float2* const both = reinterpret_cast<float2*>(&sh.kept[0][0][0]);
#pragma unroll
    for (int i = 0; i < S::kV; ++i) both[at.slot * S::kChannels + at.c_mem + i] = make_float2(d_skip[i], d_bias[i]);
    __syncthreads();
    for (int c = threadIdx.x; c < S::kChannels; c += kThreads) {
        if (at.c0 + c >= p.channels) break;
        float2 v = make_float2(0.0f, 0.0f);
        for (int s = 0; s < kRun; ++s) {
            v.x += both[s * S::kChannels + c].x;
            v.y += both[s * S::kChannels + c].y;
        }
        frames[per + at.c0 + c] = v.x;
        frames[per + p.channels + at.c0 + c] = v.y;
    }
}

// db and dc of a slot and state: the sum over the groups of channels, in their order
template <typename T>
__global__ void __launch_bounds__(256) k40_scan_sums(const ScanParams p, const ScanTensors<T> a, const float* across, int groups, int all)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, slots = p.blocks * p.t;
    const int64_t slot = i / (2 * all);
    if (slot >= slots) return;
    const int n = (int)(i - slot * 2 * all);
    float v = 0.0f;
    for (int g = 0; g < groups; ++g) v += __ldcs(across + g * slots * 2 * all + i);
    const int64_t q = slot / p.t, s = slot - q * p.t;
    if (n < p.states)
        a.db.at(q, s)[n] = from_float<T>(v);
    else if (n >= all && n - all < p.states)
        a.dc.at(q, s)[n - all] = from_float<T>(v);
}

// A lane has four states of a channel, LANES of them the channel, and kRowsAtOnce rows one after the other, all loads under way.
constexpr int kStepRows = 4;
template <typename T, int LANES>
__global__ void __launch_bounds__(kThreads) k41_scan_step(const ScanStepParams p, const ScanStepTensors<T> a, int groups, bool wide)
{
    const int64_t at = blockIdx.x / groups, row0 = at * kStepRows;
    const int part = threadIdx.x % LANES, n0 = part * 4;
    const int64_t c = (blockIdx.x - at * groups) * (kThreads / LANES) + threadIdx.x / LANES;
    const bool on = c < p.channels;
    float h[kStepRows][4], b[kStepRows][4], cc[kStepRows][4], x[kStepRows], dt[kStepRows], z[kStepRows];
    int here[kStepRows];
#pragma unroll
    for (int r = 0; r < kStepRows; ++r) here[r] = row0 + r < p.rows ? p.pos[row0 + r] : -1;
    auto four = [&](const float* from, float (&to)[4]) {
        if (wide) {
            const float4 v = n0 < p.states ? *reinterpret_cast<const float4*>(from) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            to[0] = v.x;
            to[1] = v.y;
            to[2] = v.z;
            to[3] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) to[i] = n0 + i < p.states ? from[i] : 0.0f;
        }
    };
#pragma unroll
    for (int r = 0; r < kStepRows; ++r) {
        const int64_t row = row0 + r;
        const bool state = on && row < p.rows && (here[r] > 0 || (here[r] < 0 && p.next != p.state)), frame = on && here[r] >= 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[r][i] = 0.0f;
            b[r][i] = frame && n0 + i < p.states ? to_float(a.b[row * a.sb + n0 + i]) : 0.0f;
            cc[r][i] = frame && n0 + i < p.states ? to_float(a.c[row * a.sc + n0 + i]) : 0.0f;
        }
        if (state) four(p.state + (row * p.channels + c) * p.states + n0, h[r]);
        x[r] = frame ? to_float(a.x[row * a.sx + c]) : 0.0f;
        dt[r] = frame ? to_float(a.dt[row * a.sdt + c]) : 0.0f;
        z[r] = frame && a.z ? to_float(a.z[row * a.sz + c]) : 0.0f;
    }
    float decays[4] = {0.0f, 0.0f, 0.0f, 0.0f}, bias = 0.0f, skip = 0.0f;
    if (on) {
        four(p.a + c * p.states + n0, decays);
        bias = p.dt_bias ? p.dt_bias[c] : 0.0f;
        skip = p.d ? p.d[c] : 0.0f;
    }
#pragma unroll
    for (int r = 0; r < kStepRows; ++r) {
        const int64_t row = row0 + r;
        if (row >= p.rows) break;
        float delta = dt[r] + bias, slope, y = 0.0f;
        if (p.softplus) softplus_of(delta, delta, slope);
        const float u = delta * x[r];
        if (here[r] >= 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float push = u * b[r][i];
                h[r][i] = here[r] > 0 ? fmaf(ex2(delta * (decays[i] * kLog2E)), h[r][i], push) : push;
                y = fmaf(h[r][i], cc[r][i], y);
            }
        }
#pragma unroll
        for (int bit = LANES / 2; bit; bit /= 2) y += __shfl_xor_sync(0xffffffffu, y, bit);
        if (!on) continue;
        if (here[r] >= 0 || p.next != p.state) {
            float* const to = p.next + (row * p.channels + c) * p.states + n0;
            if (wide) {
                if (n0 < p.states) *reinterpret_cast<float4*>(to) = make_float4(h[r][0], h[r][1], h[r][2], h[r][3]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (n0 + i < p.states) to[i] = h[r][i];
            }
        }
        if (part == 0) {
            y = fmaf(skip, x[r], y);
            if (a.z) y *= z[r] * sigmoid_of(z[r]);
            a.y[row * a.sy + c] = from_float<T>(here[r] >= 0 ? y : 0.0f);
        }
    }
}

// calls go(Split) for the states of a call
template <typename Go>
auto with_split(int states, const Go& go)
{
    if (states <= 8) return go(Split<4, 2>());
    if (states <= 16) return go(Split<4, 4>());
    if (states <= 32) return go(Split<8, 4>());
    return go(Split<16, 4>());
}

// Segments per walk: enough for eight CTAs per SM where there are fewer than two without, of at least 8 runs each.
ScanCuts cuts_of(int64_t blocks, int32_t t, int64_t channels, int states)
{
    return with_split(states, [&](auto s) {
        using S = decltype(s);
        ScanCuts cuts;
        cuts.groups = (int)((channels + S::kChannels - 1) / S::kChannels);
        const int64_t walks = blocks * cuts.groups, runs = (t + kRun - 1) / kRun;
        const int64_t wanted = walks < 2 * 148 ? 8 * 148 / walks : 1, most = runs / 8, n = wanted < most ? wanted : most;
        cuts.segments = (int)(n < 1 ? 1 : n);
        cuts.stride = 2 * S::kAll;
        return cuts;
    });
}

ScanWork work_of(void* base, const ScanCuts& cuts, int64_t blocks, int32_t t, int64_t channels, int states, bool gradient)
{
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t cells = (size_t)cuts.segments * blocks, per = (size_t)channels * states;
    ScanWork w;
    size_t at = 0;
    auto take = [&](size_t floats) {
        char* const here = static_cast<char*>(base) + at;
        at += up(floats * 4);
        return here;
    };
    const bool cut = cuts.segments > 1;
    w.kind = reinterpret_cast<int32_t*>(take(cut ? cells : 0));
    w.delta = reinterpret_cast<float*>(take(cut ? cells * channels : 0));
    w.state = reinterpret_cast<float*>(take(cut ? cells * per : 0));
    w.frames = reinterpret_cast<float*>(take(gradient ? cells * (per + 2 * channels) : 0));
    w.across = reinterpret_cast<float*>(take(gradient ? (size_t)cuts.groups * blocks * t * cuts.stride : 0));
    w.bytes = at;
    return w;
}

template <typename T>
bool on(const Channels<T>& x, size_t n)
{
    return !x.data || (reinterpret_cast<uintptr_t>(x.data) % n == 0 && x.block * sizeof(T) % n == 0 && x.slot * sizeof(T) % n == 0);
}
template <typename T, typename S>
size_t piece()
{
    return S::kV * sizeof(T) < 16 ? S::kV * sizeof(T) : 16;
}

cudaError_t join(const ScanParams& p, const ScanCuts& cuts, const ScanWork& work, bool backwards, cudaStream_t st)
{
    const int64_t n = p.blocks * p.channels * p.states;
    k38_scan_join<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(p, cuts, work, backwards);
    count_launches(1);
    return cudaGetLastError();
}

}  // namespace

size_t scan_work_bytes(int64_t blocks, int32_t t, int64_t channels, int32_t states, bool gradient)
{
    return work_of(nullptr, cuts_of(blocks, t, channels, states), blocks, t, channels, states, gradient).bytes;
}

template <typename T>
cudaError_t launch_scan(const ScanParams& p, const ScanTensors<T>& a, cudaStream_t st)
{
    return with_split(p.states, [&](auto s) {
        using S = decltype(s);
        const ScanCuts cuts = cuts_of(p.blocks, p.t, p.channels, p.states);
        const ScanWork work = work_of(p.work, cuts, p.blocks, p.t, p.channels, p.states, false);
        const size_t n = piece<T, S>();
        const bool wide = on(a.x, n) && on(a.dt, n) && on(a.z, n) && on(a.y, n);
        const unsigned grid = (unsigned)(cuts.segments * p.blocks * cuts.groups);
        if (cuts.segments > 1) {
            k37_scan<T, S, false><<<grid, kThreads, 0, st>>>(p, a, cuts, work, wide);
            count_launches(1);
            cudaError_t e = cudaGetLastError();
            if (e == cudaSuccess) e = join(p, cuts, work, false, st);
            if (e != cudaSuccess) return e;
        }
        k37_scan<T, S, true><<<grid, kThreads, 0, st>>>(p, a, cuts, work, wide);
        count_launches(1);
        return cudaGetLastError();
    });
}

template <typename T>
cudaError_t launch_scan_grad(const ScanParams& p, const ScanTensors<T>& a, cudaStream_t st)
{
    return with_split(p.states, [&](auto s) {
        using S = decltype(s);
        const ScanCuts cuts = cuts_of(p.blocks, p.t, p.channels, p.states);
        const ScanWork work = work_of(p.work, cuts, p.blocks, p.t, p.channels, p.states, true);
        const size_t n = piece<T, S>();
        const bool wide = on(a.x, n) && on(a.dt, n) && on(a.z, n) && on(a.dy, n) && on(a.dx, n) && on(a.ddt, n) && on(a.dz, n);
        const unsigned grid = (unsigned)(cuts.segments * p.blocks * cuts.groups);
        constexpr int kShared = sizeof(GradShared<S>);
        static std::atomic<uint64_t> allowed[2] = {};
        cudaError_t e = allow_shared(k39_scan_grad<T, S, true>, kShared, allowed[0]);
        if (e == cudaSuccess) e = allow_shared(k39_scan_grad<T, S, false>, kShared, allowed[1]);
        if (e != cudaSuccess) return e;
        if (cuts.segments > 1) {
            k39_scan_grad<T, S, false><<<grid, kThreads, kShared, st>>>(p, a, cuts, work, wide);
            count_launches(1);
            e = cudaGetLastError();
            if (e == cudaSuccess) e = join(p, cuts, work, true, st);
            if (e != cudaSuccess) return e;
        }
        k39_scan_grad<T, S, true><<<grid, kThreads, kShared, st>>>(p, a, cuts, work, wide);
        count_launches(1);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
        const int64_t sums = p.blocks * p.t * 2 * S::kAll, per = p.channels * p.states;
        k40_scan_sums<T><<<(unsigned)((sums + 255) / 256), 256, 0, st>>>(p, a, work.across, cuts.groups, S::kAll);
        count_launches(1);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
        return launch_column_sums({work.frames, cuts.segments * p.blocks, per + 2 * p.channels, {p.da, p.dd, p.ddt_bias},
                                   {per, per + p.channels, per + 2 * p.channels}}, st);
    });
}

template <typename T>
cudaError_t launch_scan_step(const ScanStepParams& p, const ScanStepTensors<T>& a, cudaStream_t st)
{
    auto go = [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        const int groups = (int)((p.channels + kThreads / L - 1) / (kThreads / L));
        auto on_16 = [](const float* x) { return reinterpret_cast<uintptr_t>(x) % 16 == 0; };
        const bool wide = p.states % 4 == 0 && on_16(p.state) && on_16(p.next) && on_16(p.a);
        k41_scan_step<T, L><<<(unsigned)((p.rows + kStepRows - 1) / kStepRows * groups), kThreads, 0, st>>>(p, a, groups, wide);
        count_launches(1);
        return cudaGetLastError();
    };
    if (p.states <= 4) return go(std::integral_constant<int, 1>());
    if (p.states <= 8) return go(std::integral_constant<int, 2>());
    if (p.states <= 16) return go(std::integral_constant<int, 4>());
    if (p.states <= 32) return go(std::integral_constant<int, 8>());
    return go(std::integral_constant<int, 16>());
}
#define BLOAD_INSTANTIATE(T)                                                                          \
    template cudaError_t launch_scan<T>(const ScanParams&, const ScanTensors<T>&, cudaStream_t);      \
    template cudaError_t launch_scan_grad<T>(const ScanParams&, const ScanTensors<T>&, cudaStream_t); \
    template cudaError_t launch_scan_step<T>(const ScanStepParams&, const ScanStepTensors<T>&, cudaStream_t);
BLOAD_INSTANTIATE(float)
BLOAD_INSTANTIATE(__half)
BLOAD_INSTANTIATE(__nv_bfloat16)
#undef BLOAD_INSTANTIATE

}  // namespace bload

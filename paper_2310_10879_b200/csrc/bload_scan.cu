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
// Walks that fit on the machine at once, two to an SM, are bound by the latency of a run: there a second half of the CTA prepares and
// finishes runs while the first walks.  Where they leave much of the machine empty, the slots are cut into segments, a CTA each.  k37 and k39 first run over the part
// of a segment that its successor hears of (from the last sequence start on; nothing if a sequence starts there) without output, k38
// joins what they leave, and the walk proper starts from that.
//
// The gradient walks backwards, run by run, from the states that the forward call kept at the start of each run: it rebuilds the states of
// every other slot into shared memory (each thread its own), then goes through them from the last slot to the first.  Sums over
// channels (db, dc) are shared out over the lanes of a warp, then over the CTA's warps, and written once per CTA; k40 adds the CTAs'.
//
// 8 x 4096 x 2048 x 16 bf16, prompts, in halves: 650 us (745 in segments: their parts 228, walk 508); 4 x 10,000 x 1024 x 16 training: 344 +
// 1,020 us for the walks, 1,550 in all.  What bounds them is latency and issue: halves 0.44 instructions a cycle and scheduler, the exponentials at
// 47 % of their rate, shared memory 51 %, 14 warps on an SM (the two halves wait for one another as often as for arithmetic);
// segments 0.5, 40 to 55 %, 53 %, 16 warps.  More states, 8 x 4096 x 2048 bf16, 16 / 32 / 64 of them: forward 630 / 1,000 / 1,855 us,
// training 2,570 / 4,240 / 7,990, of which the sums over CTAs' db and dc 30 / 93 / 344.  Step of 256 x 4096 x 16: 36 us, 4.0 TB/s.
#include <math.h>
#include <stddef.h>

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
    static constexpr int kGroup = 2;                // slots whose sums over states are taken together
    static constexpr int kRow = kChannels + 8;      // of an array by slots and channels, so that slots two apart lie in other banks
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
// exp(delta a) of two states, from delta and a log2(e).  The hardware's exponential is a little too small: for arguments in -[2^-11, 2^-8]
// by 0.09 to 0.14 units of 2^-24 in the mean, up to -2^-4 by 0.3 to 0.5 (measured over 2^20 arguments each).  In a state that 1,000 slots
// contribute to that adds up to more than all roundings, so 0.16 units are added to the argument, which costs nothing.
__device__ __forceinline__ Two decay(Two delta, Two a)
{
    constexpr float kUnits = 0.16f * 5.9604645e-8f * kLog2E;
    const float2 x = one(fma(delta, a, two(kUnits, kUnits)));
    return two(ex2(x.x), ex2(x.y));
}

// softplus(v) = max(v, 0) + log1p(e) of two values, e = exp(-|v|), which is in (0, 1].  The product with log2(e) keeps what its rounding
// loses (without: up to 1e-6 of e for v = -10).  log1p(e) = 2 atanh(s), s = e / (2 + e) <= 1/3, by its series to s^15: the rest is
// below 2e-9 of it.
__device__ __forceinline__ Two softplus_of(Two v)
{
    const float v0 = one(v).x, v1 = one(v).y;
    const Two a = two(fminf(fabsf(v0), 126.0f), fminf(fabsf(v1), 126.0f)), x = a * two(kLog2E, kLog2E);
    const Two rest = fma(a, two(-1.925963033e-8f, -1.925963033e-8f), fma(a, two(-kLog2E, -kLog2E), x));
    Two e = two(ex2(-one(x).x), ex2(-one(x).y));
    e = fma(e, rest * two(kLn2, kLn2), e);
    const float2 d = one(e + two(2.0f, 2.0f));
    float r0, r1;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(d.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(d.y));
    const Two s = e * two(r0, r1), z = s * s;
    auto c = [](float k) { return two(2.0f / k, 2.0f / k); };
    Two p = fma(z, c(15.0f), c(13.0f));
    p = fma(z, p, c(11.0f));
    p = fma(z, p, c(9.0f));
    p = fma(z, p, c(7.0f));
    p = fma(z, p, c(5.0f));
    p = fma(z, p, c(3.0f));
    float m0, m1;  // (NaN stays)
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m0) : "f"(v0), "f"(0.0f));
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m1) : "f"(v1), "f"(0.0f));
    return fma(s * z, p, fma(s, two(2.0f, 2.0f), two(m0, m1)));
}

// The first slot from `from` on, but before `end`, where a sequence starts or padding lies, by a whole warp; `from` if there is none.
__device__ __forceinline__ int warp_start_from(const int32_t* pos, int from, int end, int lane)
{
    for (int s = from; s < end; s += 128) {
        bool starts[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) starts[k] = s + 32 * k + lane < end && pos[s + 32 * k + lane] <= 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const unsigned any = __ballot_sync(0xffffffffu, starts[k]);
            if (any) return s + 32 * k + __ffs(any) - 1;
        }
    }
    return from;
}

// Where a thread stands: as the lanes hold states, and as a run lies in memory.  In shared memory channel e of the kV that a thread
// has in memory order lies at e * 8 + its place among the slot's 8 threads, so that neighbouring threads write side by side.
// A segment ends at a sequence start where there is one in the half segment behind its share of the runs: then nothing crosses.
template <typename S>
struct Place {
    int lane, warp, part;  // part: which of the states
    int ch[2], at[2];      // the lane's two channels, of the CTA and in shared memory; every other lane has them the other way round
    int slot, m;           // of the run, and which 8th of its channels
    int64_t c0;            // first channel of the CTA
    int there;             // of the kV channels
    int64_t q;             // block
    int segment;
    int begin, stop;       // slots of the segment
    bool enters, leaves;   // a sequence crosses its first slot, its last
    __device__ __forceinline__ Place(const ScanParams& p, const ScanCuts& cuts)
    {
        lane = threadIdx.x & 31;
        warp = (threadIdx.x >> 5) % kWarps;
        part = lane % S::kLanes;
        const int pair = warp * (S::kPerWarp / 2) + lane / S::kLanes, e = pair / 8 * 2, odd = part & 1;
        ch[0] = pair % 8 * S::kV + e + odd;
        ch[1] = pair % 8 * S::kV + e + 1 - odd;
        at[0] = (e + odd) * 8 + pair % 8;
        at[1] = (e + 1 - odd) * 8 + pair % 8;
        slot = threadIdx.x % kThreads >> 3;
        m = threadIdx.x & 7;
        const unsigned i = blockIdx.x / (unsigned)cuts.groups, walks = (unsigned)p.blocks;  // (a grid has less than 2^31 CTAs)
        c0 = (int64_t)(blockIdx.x - i * (unsigned)cuts.groups) * S::kChannels;
        there = (int)max((int64_t)0, min(p.channels - c0 - m * S::kV, (int64_t)S::kV));
        segment = (int)(i / walks);
        q = i - segment * walks;
        begin = 0;
        stop = p.t;
        enters = leaves = false;
        if (cuts.segments > 1) {
            const int runs = (p.t + kRun - 1) / kRun, room = runs / cuts.segments * (kRun / 2);
            const int32_t* const pos = p.pos + q * p.t;
            if (segment > 0) {
                const int edge = (int)((int64_t)runs * segment / cuts.segments) * kRun;
                begin = warp_start_from(pos, edge, min(edge + room, p.t), lane);
                enters = pos[begin] > 0;
            }
            if (segment + 1 < cuts.segments) {
                const int edge = (int)((int64_t)runs * (segment + 1) / cuts.segments) * kRun;
                stop = warp_start_from(pos, edge, min(edge + room, p.t), lane);
                leaves = pos[stop] > 0;
            }
        }
    }
    // Position of the run's slot `lane`, up to the first slot behind the run; -1 in front of the segment and behind the block.
    __device__ __forceinline__ int look(const int32_t* pos, int t, int s0) const
    {
        const int s = s0 + lane;
        return lane <= kRun && s >= begin && s < t ? pos[s] : -1;
    }
    // bit s of `valid`: slot s of the run is a frame of the segment, of `starts`: it starts a sequence (or is none), of `ends`:
    // its sequence ends with it
    __device__ __forceinline__ void masks(int here, int s0, unsigned& valid, unsigned& starts, unsigned& ends) const
    {
        const bool mine = lane < kRun && s0 + lane < stop;
        valid = __ballot_sync(0xffffffffu, mine && here >= 0);
        starts = __ballot_sync(0xffffffffu, !mine || here <= 0);
        ends = valid & (__ballot_sync(0xffffffffu, here <= 0) >> 1);
    }
    // whether this thread's slot of the run is the segment's
    __device__ __forceinline__ bool inside(int s0) const { return s0 + slot >= begin && s0 + slot < stop; }
};

// a[channel][state], of the lane's two channels, as pairs of states; 0 where there is none
template <typename S>
__device__ __forceinline__ void load_a(const ScanParams& p, const Place<S>& at, float factor, Two (&a)[2][S::kPairs])
{
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int k = 0; k < S::kPairs; ++k) {
            const int64_t ch = at.c0 + at.ch[c];
            const int n = at.part * S::kStates + 2 * k;
            const float* const from = p.a + ch * p.states + n;
            const bool on = ch < p.channels;
            a[c][k] = two(on && n < p.states ? from[0] * factor : 0.0f, on && n + 1 < p.states ? from[1] * factor : 0.0f);
        }
}

// States [channel][state] in memory, from `base` of the CTA's first channel on
template <typename S>
__device__ __forceinline__ bool states_wide(const ScanParams& p, const float* base)
{
    return S::kStates == 4 && p.states % 4 == 0 && reinterpret_cast<uintptr_t>(base) % 16 == 0;
}
template <typename S>
__device__ __forceinline__ void load_states(const ScanParams& p, const Place<S>& at, const float* base, Two (&h)[2][S::kPairs])
{
    const int n = at.part * S::kStates;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const float* const from = base + ((uint32_t)at.ch[c] * (uint32_t)p.states + (uint32_t)n);
        const int there = at.c0 + at.ch[c] < p.channels ? p.states - n : 0;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (states_wide<S>(p, base)) {
            if (there > 0) *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(from);
        } else {
#pragma unroll
            for (int k = 0; k < S::kStates; ++k) v[k] = k < there ? from[k] : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < S::kPairs; ++k) h[c][k] = two(v[2 * k], v[2 * k + 1]);
    }
}
template <typename S>
__device__ __forceinline__ void prefetch_states(const ScanParams& p, const Place<S>& at, const float* base)
{
#pragma unroll
    for (int c = 0; c < 2; ++c)
        if (at.c0 + at.ch[c] < p.channels && at.part * S::kStates < p.states)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(base + ((uint32_t)at.ch[c] * (uint32_t)p.states + (uint32_t)(at.part * S::kStates))));
}
template <typename S>
__device__ __forceinline__ void store_states(const ScanParams& p, const Place<S>& at, float* base, const Two (&h)[2][S::kPairs])
{
    const int n = at.part * S::kStates;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        float* const to = base + ((uint32_t)at.ch[c] * (uint32_t)p.states + (uint32_t)n);
        const int there = at.c0 + at.ch[c] < p.channels ? p.states - n : 0;
        if (states_wide<S>(p, base)) {
            const float2 x = one(h[c][0]), y = one(h[c][S::kPairs - 1]);
            if (there > 0) *reinterpret_cast<float4*>(to) = make_float4(x.x, x.y, y.x, y.y);
        } else {
#pragma unroll
            for (int k = 0; k < S::kPairs; ++k) {
                if (2 * k < there) to[2 * k] = one(h[c][k]).x;
                if (2 * k + 1 < there) to[2 * k + 1] = one(h[c][k]).y;
            }
        }
    }
}

// Elements of a run in the order of memory.  WIDE: pieces lie on boundaries of their size, channels are a multiple of them, and a
// block of a tensor spans less than 2^32 bytes, so that an address is a base that the CTA shares and a 32-bit offset.
template <typename T, typename S, bool WIDE>
struct Frames {
    using Piece = Elements<T, S::kV>;
    template <typename P>
    static __device__ __forceinline__ P* at_slot(const Channels<P>& x, const Place<S>& at, int s0)
    {
        if constexpr (WIDE) {
            using Byte = std::conditional_t<std::is_const<P>::value, const char, char>;
            Byte* const base = reinterpret_cast<Byte*>(x.data + at.q * x.block + at.c0);
            return reinterpret_cast<P*>(base + ((uint32_t)(s0 + at.slot) * ((uint32_t)x.slot * (uint32_t)sizeof(T)) + (uint32_t)(at.m * S::kV * (int)sizeof(T))));
        } else {
            return x.at(at.q, s0 + at.slot) + at.c0 + at.m * S::kV;
        }
    }
    static __device__ __forceinline__ void load(Piece& v, const Channels<const T>& x, const Place<S>& at, int s0, bool on)
    {
        if constexpr (WIDE) {
            v.load_if(at_slot(x, at, s0), on && at.there);
        } else if (on) {
            v.load(at_slot(x, at, s0), at.there, false);
        } else {
            v.clear();
        }
    }
    static __device__ __forceinline__ void prefetch(const Channels<const T>& x, const Place<S>& at, int s0)
    {
        if (WIDE && at.there && s0 + at.slot >= at.begin) asm volatile("prefetch.global.L2 [%0];" ::"l"(at_slot(x, at, s0)));
    }
    static __device__ __forceinline__ void store(const Piece& v, const Channels<T>& x, const Place<S>& at, int s0)
    {
        if (!WIDE)
            v.store(at_slot(x, at, s0), at.there, false);
        else if (at.there)
            v.store(at_slot(x, at, s0), S::kV, true);
    }
};

// b and c of a run, [slot][b, c][kAll] in shared memory; 0 on padding and where there is no state.  In pieces of 16 bytes where rows
// allow it (p.rows_wide), element by element otherwise.
template <typename T, typename S, bool B, bool C>
struct Rows {
    static constexpr int kV = 16 / sizeof(T) < S::kAll ? 16 / sizeof(T) : S::kAll, kPieces = kRun * S::kAll / kV;
    static constexpr int kEach = (kPieces + kThreads - 1) / kThreads;
    Elements<T, kV> b[B ? kEach : 1], c[C ? kEach : 1];
    // ALL: of the segment's slots, otherwise of those in `wanted`
    template <bool ALL>
    __device__ __forceinline__ void load(const ScanParams& p, const ScanTensors<T>& a, const Place<S>& place, int s0, unsigned wanted = 0)
    {
        const T *const b0 = a.b.data + place.q * a.b.block, *const c0 = a.c.data + place.q * a.c.block;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int at = threadIdx.x % kThreads + i * kThreads, slot = at / (S::kAll / kV), n = at % (S::kAll / kV) * kV;
            const bool here = ALL ? s0 + slot >= place.begin && s0 + slot < place.stop : (wanted >> slot) & 1;
            const int there = slot < kRun && here ? p.states - n : 0;
            if (p.rows_wide) {  // (blocks of less than 2^32 elements, too)
                if (B) b[B ? i : 0].load_if(b0 + ((uint32_t)(s0 + slot) * (uint32_t)a.b.slot + (uint32_t)n), there > 0);
                if (C) c[C ? i : 0].load_if(c0 + ((uint32_t)(s0 + slot) * (uint32_t)a.c.slot + (uint32_t)n), there > 0);
                continue;
            }
            b[B ? i : 0].clear();
            c[C ? i : 0].clear();
            if (there > 0) {
                if (B) b[B ? i : 0].load(b0 + (s0 + slot) * a.b.slot + n, there, false);
                if (C) c[C ? i : 0].load(c0 + (s0 + slot) * a.c.slot + n, there, false);
            }
        }
    }
    // `turn` 2: with the pairs of every four states the other way round
    __device__ __forceinline__ void store(float (*to)[2][S::kAll], unsigned valid, int turn = 0) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int at = threadIdx.x % kThreads + i * kThreads, slot = at / (S::kAll / kV), n = at % (S::kAll / kV) * kV;
            if (slot >= kRun) break;
            const bool on = (valid >> slot) & 1;
#pragma unroll
            for (int e = 0; e < kV; e += 2) {
                const float2 none = make_float2(0.0f, 0.0f);
                if (B) *reinterpret_cast<float2*>(&to[slot][0][n + (e ^ turn)]) = on ? one(b[B ? i : 0].pair(e)) : none;
                if (C) *reinterpret_cast<float2*>(&to[slot][1][n + (e ^ turn)]) = on ? one(c[C ? i : 0].pair(e)) : none;
            }
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

// dt_bias or d of a thread's channels, 0 where there is none
template <int V>
__device__ __forceinline__ Elements<float, V> of_channels(const float* from, int64_t c, int there)
{
    Elements<float, V> v;
    v.clear();
    if (from) v.load(from + c, there, reinterpret_cast<uintptr_t>(from) % 16 == 0);
    return v;
}

// Sums over a channel's lanes of what each has for kGroup slots and its two channels.  The lanes that share a channel have the two in
// turned order, so the first step hands over one channel without choosing; then the slots are shared out.  A lane ends with its first
// channel's sum for slot `first`, in v[0][0] (beyond four lanes, several have the same).
template <typename S>
__device__ __forceinline__ void lane_sums(float (&v)[2][S::kGroup], int lane, int& first)
{
    first = 0;
#pragma unroll
    for (int i = 0; i < S::kGroup; ++i) v[0][i] += __shfl_xor_sync(0xffffffffu, v[1][i], 1);
#pragma unroll
    for (int bit = 2, n = S::kGroup; bit < S::kLanes; bit *= 2) {
        if (n > 1) {
            n /= 2;
            const bool upper = lane & bit;
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const float send = upper ? v[0][i] : v[0][i + n], keep = upper ? v[0][i + n] : v[0][i];
                v[0][i] = keep + __shfl_xor_sync(0xffffffffu, send, bit);
            }
            if (upper) first += n;
        } else {
            v[0][0] += __shfl_xor_sync(0xffffffffu, v[0][0], bit);
        }
    }
}

// Named barriers between the two halves of a CTA: one half arrives, the other waits.
__device__ __forceinline__ void half_arrives(int barrier) { asm volatile("barrier.cta.arrive %0, %1;" ::"r"(barrier), "n"(2 * kThreads) : "memory"); }
__device__ __forceinline__ void half_waits(int barrier) { asm volatile("barrier.cta.sync %0, %1;" ::"r"(barrier), "n"(2 * kThreads) : "memory"); }

// 128 threads prepare, walk and finish a run in turn.  HALVES: of 256 threads half walk, while the other half finish the run in front and
// prepare the one behind, in two buffers: a run takes less time (1.6 us instead of 2.3 alone on an SM), but fewer runs fit.
// OUTPUT false: leaves what crosses the segment's end (kind, delta, state of ScanWork).
template <typename T, typename S, bool WIDE, bool OUTPUT, bool HALVES>
__global__ void __launch_bounds__(HALVES ? 2 * kThreads : kThreads, HALVES ? 2 : 4)
    k37_scan(const ScanParams p, const ScanTensors<T> a, const ScanCuts cuts, const ScanWork work)
{
    constexpr int kBuffers = HALVES ? 2 : 1, kFull = 1, kDone = 3;  // barriers kFull, kDone + buffer
    __shared__ __align__(16) float4 prepared[kBuffers][kRun][S::kChannels];  // delta, delta, delta x, delta x
    __shared__ __align__(16) float rows[kBuffers][kRun][2][S::kAll];
    __shared__ float sums[OUTPUT ? kBuffers : 1][OUTPUT ? kRun : 1][OUTPUT ? S::kRow : 1];
    __shared__ float2 of_channel[S::kChannels / 2][2];  // dt_bias, d, of two channels each

    const Place<S> at(p, cuts);
    const int32_t* const pos = p.pos + at.q * p.t;
    const int runs = (p.t + kRun - 1) / kRun, end = (at.stop + kRun - 1) / kRun;
    int run = at.begin / kRun;
    const int64_t cell = (int64_t)at.segment * p.blocks + at.q, per = p.channels * p.states, first_state = at.c0 * p.states;
    if (!OUTPUT) {
        if (!at.leaves || at.stop <= at.begin) {
            if (threadIdx.x == 0) work.kind[cell] = 0;
            return;
        }
        const int start = at.stop - min(pos[at.stop], at.stop);  // of the sequence
        run = max(run, min(start / kRun, end - 1));
        if (threadIdx.x == 0) work.kind[cell] = start < at.begin ? 2 : 1;
    }
    for (int c = threadIdx.x; c < S::kChannels; c += blockDim.x) {
        const bool there = at.c0 + c < p.channels;
        const int pair = c % S::kV / 2 * 8 + c / S::kV;
        reinterpret_cast<float*>(of_channel[pair])[c & 1] = p.dt_bias && there ? p.dt_bias[at.c0 + c] : 0.0f;
        reinterpret_cast<float*>(of_channel[pair])[2 + (c & 1)] = OUTPUT && p.d && there ? p.d[at.c0 + c] : 0.0f;
    }
    __syncthreads();

    // what prepares and finishes: x, dt, z and y as they lie in memory
    const bool gated = OUTPUT && a.z.data, softplus = p.softplus;
    using F = Frames<T, S, WIDE>;
    Elements<T, S::kV> x, dt, z;
    z.clear();
    Rows<T, S, true, OUTPUT> bc;
    auto of_pair = [&](int which, int e) {
        const float2 v = of_channel[e / 2 * 8 + at.m][which];
        return two(v.x, v.y);
    };
    auto fetch = [&](int s0) {  // (padding as well: whether a slot is a frame is known only when its position has arrived)
        const bool on = at.inside(s0);
        F::load(x, a.x, at, s0, on);
        F::load(dt, a.dt, at, s0, on);
        if (gated) F::load(z, a.z, at, s0, on);
        bc.template load<true>(p, a, at, s0);
    };
    auto prepare = [&](int buffer, unsigned valid) {
        if ((valid >> at.slot) & 1) {
#pragma unroll
            for (int e = 0; e < S::kV; e += 2) {
                Two delta = dt.pair(e) + of_pair(0, e);
                if (softplus) delta = softplus_of(delta);
                if (!WIDE) delta = two(e < at.there ? one(delta).x : 0.0f, e + 1 < at.there ? one(delta).y : 0.0f);
                const float2 d = one(delta), u = one(delta * x.pair(e));
                prepared[buffer][at.slot][e * 8 + at.m] = make_float4(d.x, d.x, u.x, u.x);
                prepared[buffer][at.slot][e * 8 + 8 + at.m] = make_float4(d.y, d.y, u.y, u.y);
            }
        } else {
#pragma unroll
            for (int e = 0; e < S::kV; ++e) prepared[buffer][at.slot][e * 8 + at.m] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
        bc.store(rows[buffer], valid);
    };
    auto finish = [&](int buffer, int s0, unsigned valid, const Elements<T, S::kV>& xs, const Elements<T, S::kV>& zs) {
        if (!at.inside(s0)) return;
        Elements<T, S::kV> out;
        if ((valid >> at.slot) & 1) {
#pragma unroll
            for (int e = 0; e < S::kV; e += 2) {
                Two v = fma(of_pair(1, e), xs.pair(e), two(sums[buffer][at.slot][e * 8 + at.m], sums[buffer][at.slot][e * 8 + 8 + at.m]));
                if (gated) v = v * (zs.pair(e) * sigmoid_of(zs.pair(e)));
                out.set_pair(e, v);
            }
        } else {
            out.clear();
        }
        F::store(out, a.y, at, s0);
    };
    if (HALVES && threadIdx.x >= kThreads) {
        int buffer = 0;
        unsigned before = 0;  // frames of the run in front
        Elements<T, S::kV> before_x, before_z;
        before_x.clear();
        before_z.clear();
        const int first = run;
        int here = -1;
        if (run < end) {
            here = at.look(pos, p.t, run * kRun);
            fetch(run * kRun);
        }
        for (; run < end; ++run) {
            unsigned valid, starts, ends;
            at.masks(here, run * kRun, valid, starts, ends);
            prepare(buffer, valid);  // (the buffer is free: its last run has been finished)
            half_arrives(kFull + buffer);
            const Elements<T, S::kV> now_x = x, now_z = z;
            if (run + 1 < end) {
                here = at.look(pos, p.t, (run + 1) * kRun);
                fetch((run + 1) * kRun);
            }
            buffer ^= 1;
            if (run > first) {
                half_waits(kDone + buffer);
                finish(buffer, (run - 1) * kRun, before, before_x, before_z);
            }
            before = valid;
            before_x = now_x;
            before_z = now_z;
        }
        if (first < end) {
            buffer ^= 1;
            half_waits(kDone + buffer);
            finish(buffer, (end - 1) * kRun, before, before_x, before_z);
        }
        return;
    }

    Two A[2][S::kPairs], h[2][S::kPairs];
    load_a(p, at, kLog2E, A);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int k = 0; k < S::kPairs; ++k) h[c][k] = zero();
    if (OUTPUT && at.enters && at.begin < at.stop) load_states(p, at, work.state + (cell - p.blocks) * per + first_state, h);
    float passed[2] = {0.0f, 0.0f};
    int here = -1, buffer = 0;
    if (run < end) {
        here = at.look(pos, p.t, run * kRun);
        if (!HALVES) fetch(run * kRun);
    }
    for (; run < end; ++run) {
        const int s0 = run * kRun;
        unsigned valid, now_starts, now_ends;
        at.masks(here, s0, valid, now_starts, now_ends);
        if (!OUTPUT || !p.last) now_ends = 0;
        const Elements<T, S::kV> now_x = x, now_z = z;
        if (!HALVES) prepare(buffer, valid);
        if (OUTPUT && p.carry && s0 >= at.begin) store_states(p, at, p.carry + (at.q * runs + run) * per + first_state, h);
        if (HALVES)
            half_waits(kFull + buffer);
        else
            __syncthreads();
        if (run + 1 < end) {
            here = at.look(pos, p.t, s0 + kRun);
            if (!HALVES) fetch(s0 + kRun);
        }

        auto group = [&](int g, auto with_breaks) {
            constexpr bool breaks = decltype(with_breaks)::value;
            float y[2][S::kGroup];
#pragma unroll
            for (int i = 0; i < S::kGroup; ++i) {
                const int s = g + i;
                Two B[S::kPairs], C[S::kPairs];
                pairs_of<S>(&rows[buffer][s][0][at.part * S::kStates], B);
                if (OUTPUT) pairs_of<S>(&rows[buffer][s][1][at.part * S::kStates], C);
                const bool start = breaks && ((now_starts >> s) & 1);
                if (start) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int k = 0; k < S::kPairs; ++k) h[c][k] = zero();
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const float4 d = prepared[buffer][s][at.at[c]];
                    // (no state, no decay: one beyond 32 bits would make NaN of zero)
                    const Two delta = start ? zero() : two(d.x, d.y), u = two(d.z, d.w);
                    Two sum = zero();
#pragma unroll
                    for (int k = 0; k < S::kPairs; ++k) {
                        h[c][k] = fma(decay(delta, A[c][k]), h[c][k], u * B[k]);
                        if (OUTPUT) sum = k ? fma(h[c][k], C[k], sum) : h[c][k] * C[k];
                    }
                    y[c][i] = one(sum).x + one(sum).y;
                    if (!OUTPUT) passed[c] += d.x;
                }
                if (OUTPUT && breaks && ((now_ends >> s) & 1)) {
                    const int64_t id = p.seq_id[at.q * p.t + s0 + s];
                    if (id >= 0 && id < p.n_seq) store_states(p, at, p.last + id * per + first_state, h);
                }
            }
            if (OUTPUT) {
                int first;
                lane_sums<S>(y, at.lane, first);
                sums[buffer][g + first][at.at[0]] = y[0][0];
            }
        };
        if (HALVES && !(now_starts | now_ends)) {  // (in one piece: with two walks on an SM nothing else fills the gaps between groups)
#pragma unroll
            for (int g = 0; g < kRun; g += S::kGroup) group(g, std::false_type());
        } else {
#pragma unroll(HALVES ? 1 : 2)
            for (int g = 0; g < kRun; g += 2 * S::kGroup) {
                if (((now_starts | now_ends) >> g) & ((1 << 2 * S::kGroup) - 1)) {
                    group(g, std::true_type());
                    group(g + S::kGroup, std::true_type());
                } else {
                    group(g, std::false_type());
                    group(g + S::kGroup, std::false_type());
                }
            }
        }
        if (HALVES) {
            half_arrives(kDone + buffer);
            buffer ^= 1;
        } else {
            __syncthreads();
            if (OUTPUT) finish(buffer, s0, valid, now_x, now_z);
        }
    }
    if (!OUTPUT) {
        store_states(p, at, work.state + cell * per + first_state, h);
        if (at.part == 0) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (at.c0 + at.ch[c] < p.channels) work.delta[cell * p.channels + at.c0 + at.ch[c]] = passed[c];
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
    constexpr int kAhead = 8;  // segments whose values are loaded together
    for (int k0 = 0; k0 < cuts.segments; k0 += kAhead) {
        int kind[kAhead];
        float delta[kAhead], own[kAhead];
        auto cell = [&](int j) { return (int64_t)(backwards ? cuts.segments - 1 - k0 - j : k0 + j) * p.blocks + q; };
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            kind[j] = k0 + j < cuts.segments ? work.kind[cell(j)] : 0;
            delta[j] = k0 + j < cuts.segments ? work.delta[cell(j) * p.channels + c] : 0.0f;
            own[j] = k0 + j < cuts.segments ? work.state[cell(j) * per + (i - q * per)] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            // (kind 0: nothing was written)
            if (kind[j] == 2) {
                // Decays are above 0 and finite slot by slot: where their product has left the 32-bit range, nothing still stays
                // nothing, and an infinite state infinite.
                const float left = state == 0.0f || isinf(state) ? state : ex2(delta[j] * a) * state;
                state = left + own[j];
            } else {
                state = kind[j] == 0 ? 0.0f : own[j];
            }
            if (kind[j] == 2) work.state[cell(j) * per + (i - q * per)] = state;
        }
    }
}

template <typename S>
struct GradShared {
    float4 prepared[kRun][S::kChannels];  // delta, delta, delta x, delta x; then sums over states: g b, g a h, h c, and delta
    float dv[kRun][S::kChannels];         // dy times the gate
    float rows[2][kRun][2][S::kAll];      // b, c as they are, and with the pairs of each lane's states the other way round
    // The states that enter every other slot, of a thread, channel by channel.  Where a warp has read those of two slots, it leaves
    // their db and dc, of its channels.
    using States = std::conditional_t<S::kPairs == 2, float4, float2>;
    States kept[kRun / 2][2][kThreads];
    __device__ float* across(int warp, int slot) { return reinterpret_cast<float*>(&kept[slot / 2][slot & 1][warp * 32]); }
};
template <typename S>
constexpr int kPartShared = offsetof(GradShared<S>, kept);  // without output

// OUTPUT false: leaves what crosses the segment's first slot, backwards.
template <typename T, typename S, bool WIDE, bool OUTPUT>
__global__ void __launch_bounds__(kThreads, 4)
    k39_scan_grad(const ScanParams p, const ScanTensors<T> a, const ScanCuts cuts, const ScanWork work)
{
    extern __shared__ __align__(16) uint8_t shared_bytes[];
    GradShared<S>& sh = *reinterpret_cast<GradShared<S>*>(shared_bytes);

    const Place<S> at(p, cuts);
    const int32_t* const pos = p.pos + at.q * p.t;
    const int runs = (p.t + kRun - 1) / kRun, first = at.begin / kRun;
    const int64_t cell = (int64_t)at.segment * p.blocks + at.q, per = p.channels * p.states, first_state = at.c0 * p.states;
    int run = at.begin < at.stop ? (at.stop - 1) / kRun : first - 1;
    if (!OUTPUT) {
        if (!at.enters || at.stop <= at.begin) {
            if (threadIdx.x == 0) work.kind[cell] = 0;
            return;
        }
        const int end = warp_seq_end(pos, p.t, at.begin, at.lane);  // of the sequence
        run = min((end - 1) / kRun, run);
        // (it goes on into the next segment: what enters there is handed on)
        if (threadIdx.x == 0) work.kind[cell] = at.leaves && end > at.stop ? 2 : 1;
    }
    // The state pairs of the lanes of a warp's upper half are the other way round, so that the first step of the sums over channels
    // hands over one of them without choosing.
    const int turned = S::kPairs == 2 && (at.lane & 16) ? 1 : 0;
    const float* const b_rows = &sh.rows[turned][0][0][at.part * S::kStates];
    Two A[2][S::kPairs], e[2][S::kPairs], dA[2][S::kPairs];  // e: exp(delta a) g of the slot behind
    auto turn = [&](Two (&v)[2][S::kPairs]) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const Two x = v[c][0], y = v[c][S::kPairs - 1];
            v[c][0].v = turned ? y.v : x.v;
            v[c][S::kPairs - 1].v = turned ? x.v : y.v;
        }
    };
    load_a(p, at, kLog2E, A);
    turn(A);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int k = 0; k < S::kPairs; ++k) e[c][k] = dA[c][k] = zero();
    if (OUTPUT && at.leaves && at.begin < at.stop) {
        load_states(p, at, work.state + (cell + p.blocks) * per + first_state, e);
        turn(e);
    }

    Two d_skip[S::kV / 2], d_bias[S::kV / 2];
    float passed[2] = {0.0f, 0.0f};
    const int64_t c_mem = at.c0 + at.m * S::kV;
#pragma unroll
    for (int i = 0; i < S::kV / 2; ++i) d_skip[i] = d_bias[i] = zero();
    const bool gated = a.z.data != nullptr, softplus = p.softplus;
    using F = Frames<T, S, WIDE>;

    int here = at.look(pos, p.t, run * kRun);
    for (; run >= first; --run) {
        const int s0 = run * kRun;
        unsigned valid, starts, ends;
        at.masks(here, s0, valid, starts, ends);
        const bool on = (valid >> at.slot) & 1;
        Two h[2][S::kPairs];
        {
            Elements<T, S::kV> x, dt, z, dy;
            x.clear();
            z.clear();
            if (OUTPUT) F::load(x, a.x, at, s0, on);
            F::load(dt, a.dt, at, s0, on);
            F::load(dy, a.dy, at, s0, on);
            if (gated) F::load(z, a.z, at, s0, on);
            Rows<T, S, OUTPUT, true> bc;
            bc.template load<false>(p, a, at, s0, valid);
            here = at.look(pos, p.t, s0 - kRun);  // of the next run
            if (OUTPUT) {
                load_states(p, at, p.carry + (at.q * runs + run) * per + first_state, h);
                turn(h);
            }
            if (on) {
                const auto bias = of_channels<S::kV>(p.dt_bias, c_mem, at.there);
#pragma unroll
                for (int i = 0; i < S::kV; i += 2) {
                    Two delta = dt.pair(i) + bias.pair(i), g = dy.pair(i);
                    if (softplus) delta = softplus_of(delta);
                    if (!WIDE) delta = two(i < at.there ? one(delta).x : 0.0f, i + 1 < at.there ? one(delta).y : 0.0f);
                    if (gated) g = g * (z.pair(i) * sigmoid_of(z.pair(i)));
                    const float2 d = one(delta), u = one(delta * x.pair(i)), dv = one(g);
                    sh.prepared[at.slot][i * 8 + at.m] = make_float4(d.x, d.x, u.x, u.x);
                    sh.prepared[at.slot][i * 8 + 8 + at.m] = make_float4(d.y, d.y, u.y, u.y);
                    sh.dv[at.slot][i * 8 + at.m] = dv.x;
                    sh.dv[at.slot][i * 8 + 8 + at.m] = dv.y;
                }
            } else {
#pragma unroll
                for (int i = 0; i < S::kV; ++i) {
                    sh.prepared[at.slot][i * 8 + at.m] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    sh.dv[at.slot][i * 8 + at.m] = 0.0f;
                }
            }
            bc.store(sh.rows[0], ~0u);
            if (S::kPairs == 2) bc.store(sh.rows[1], ~0u, 2);
        }
        __syncthreads();
        if (run > first) {  // the next run's tensors come as far as the second cache meanwhile
            if (OUTPUT) F::prefetch(a.x, at, s0 - kRun);
            F::prefetch(a.dt, at, s0 - kRun);
            F::prefetch(a.dy, at, s0 - kRun);
            if (gated) F::prefetch(a.z, at, s0 - kRun);
            if (OUTPUT) prefetch_states(p, at, p.carry + (at.q * runs + run - 1) * per + first_state);
        }

        if (OUTPUT) {  // the states that enter the even slots
            auto forward = [&](int g, auto with_breaks) {
                constexpr bool breaks = decltype(with_breaks)::value;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int s = g + i;
                    if (i % 2 == 0)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const float2 x = one(h[c][0]), y = one(h[c][S::kPairs - 1]);
                            if constexpr (S::kPairs == 2)
                                sh.kept[s / 2][c][threadIdx.x] = make_float4(x.x, x.y, y.x, y.y);
                            else
                                sh.kept[s / 2][c][threadIdx.x] = x;
                        }
                    Two B[S::kPairs];
                    pairs_of<S>(b_rows + s * 2 * S::kAll, B);
                    const bool start = breaks && ((starts >> s) & 1);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const float4 d = sh.prepared[s][at.at[c]];
#pragma unroll
                        for (int k = 0; k < S::kPairs; ++k) {
                            const Two push = two(d.z, d.w) * B[k];
                            h[c][k] = start ? push : fma(decay(two(d.x, d.y), A[c][k]), h[c][k], push);
                        }
                    }
                }
            };
#pragma unroll 1
            for (int g = 0; g < kRun; g += 4) {
                if ((starts >> g) & 15)
                    forward(g, std::true_type());
                else
                    forward(g, std::false_type());
            }
        }

        auto backward = [&](int g0, auto with_breaks) {
            constexpr bool breaks = decltype(with_breaks)::value;
            float sum[3][2][S::kGroup];  // over states: g b, g a h, h c
            Two B[2][S::kPairs], C[2][S::kPairs], db[2][S::kPairs], dc[2][S::kPairs];  // of both slots
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (OUTPUT) pairs_of<S>(b_rows + (g0 + i) * 2 * S::kAll, B[i]);
                pairs_of<S>(b_rows + (g0 + i) * 2 * S::kAll + S::kAll, C[i]);
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                Two decays[2][S::kPairs], w[2][S::kPairs], now[2][S::kPairs];  // exp(delta a), exp(delta a) h before, h
                float4 d[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) d[i] = sh.prepared[g0 + i][at.at[c]];
                if (OUTPUT) {
                    float before[4];
                    *reinterpret_cast<typename GradShared<S>::States*>(before) = sh.kept[g0 / 2][c][threadIdx.x];
#pragma unroll
                    for (int k = 0; k < S::kPairs; ++k) now[1][k] = two(before[2 * k], before[2 * k + 1]);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const bool start = breaks && ((starts >> (g0 + i)) & 1);
#pragma unroll
                    for (int k = 0; k < S::kPairs; ++k) {
                        decays[i][k] = decay(two(d[i].x, d[i].y), A[c][k]);
                        if (OUTPUT) {
                            w[i][k] = decays[i][k] * now[1 - i][k];
                            if (start) w[i][k] = zero();
                            now[i][k] = fma(two(d[i].z, d[i].w), B[i][k], w[i][k]);
                        }
                    }
                    if (!OUTPUT) passed[c] += d[i].x;
                }
#pragma unroll
                for (int i = 1; i >= 0; --i) {
                    const bool start = breaks && ((starts >> (g0 + i)) & 1);
                    const float dv1 = sh.dv[g0 + i][at.at[c]];
                    const Two dv = two(dv1, dv1), u = two(d[i].z, d[i].w), delta = two(d[i].x, d[i].y);
                    Two gb, gah, hc;
#pragma unroll
                    for (int k = 0; k < S::kPairs; ++k) {
                        const Two g = fma(dv, C[i][k], e[c][k]);
                        if (OUTPUT) {
                            const Two h1 = now[i][k], gw = g * w[i][k];
                            hc = k ? fma(h1, C[i][k], hc) : h1 * C[i][k];
                            dc[i][k] = c ? fma(dv, h1, dc[i][k]) : dv * h1;
                            db[i][k] = c ? fma(u, g, db[i][k]) : u * g;
                            gb = k ? fma(g, B[i][k], gb) : g * B[i][k];
                            gah = k ? fma(gw, A[c][k], gah) : gw * A[c][k];
                            dA[c][k] = fma(gw, delta, dA[c][k]);
                        }
                        e[c][k] = decays[i][k] * g;
                        if (start) e[c][k] = zero();
                    }
                    if (OUTPUT) {
                        sum[0][c][i] = one(gb).x + one(gb).y;
                        sum[1][c][i] = one(gah).x + one(gah).y;
                        sum[2][c][i] = one(hc).x + one(hc).y;
                    }
                }
            }
            if (OUTPUT) {
                __syncwarp();  // all lanes have read the states of both slots
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float v[4];  // of one pair of states: db, dc
                    if (S::kPairs == 2) {
                        const float2 b1 = one(db[i][S::kPairs - 1]), c1 = one(dc[i][S::kPairs - 1]);
                        const Two b2 = two(__shfl_xor_sync(0xffffffffu, b1.x, 16), __shfl_xor_sync(0xffffffffu, b1.y, 16));
                        const Two c2 = two(__shfl_xor_sync(0xffffffffu, c1.x, 16), __shfl_xor_sync(0xffffffffu, c1.y, 16));
                        const float2 b0 = one(db[i][0] + b2), c0 = one(dc[i][0] + c2);
                        v[0] = b0.x;
                        v[1] = b0.y;
                        v[2] = c0.x;
                        v[3] = c0.y;
                    } else {
                        v[0] = one(db[i][0]).x;
                        v[1] = one(db[i][0]).y;
                        v[2] = one(dc[i][0]).x;
                        v[3] = one(dc[i][0]).y;
                    }
                    constexpr int kTop = S::kPairs == 2 ? 8 : 16;  // the highest lane bit that is left
                    constexpr int kSteps = S::kLanes == 4 ? (kTop == 8 ? 2 : 3) : S::kLanes == 8 ? 1 : 0, kLeft = 4 >> kSteps ? 4 >> kSteps : 1;
                    int from = 0;
                    share_sums<4, kTop, S::kLanes>(v, at.lane, from);
                    // (where the warp has more lanes for a state than values, copies write the same)
#pragma unroll
                    for (int j = 0; j < kLeft; ++j) {
                        const int n = from + j;
                        sh.across(at.warp, g0 + i)[(n >> 1) * S::kAll + at.part * S::kStates + 2 * turned + (n & 1)] = v[j];
                    }
                }
            }
            if (OUTPUT) {
                int slot = 0;
#pragma unroll
                for (int m = 0; m < 3; ++m) lane_sums<S>(sum[m], at.lane, slot);
                __syncwarp();  // all lanes have read these slots
                float4& to = sh.prepared[g0 + slot][at.at[0]];
                const float delta = to.x;
                if (S::kLanes > 4) __syncwarp();  // (lanes with the same)
                to = make_float4(sum[0][0][0], sum[1][0][0], sum[2][0][0], delta);
            }
        };
#pragma unroll 1
        for (int g0 = kRun - S::kGroup; g0 >= 0; g0 -= S::kGroup) {
            if ((starts >> g0) & ((1 << S::kGroup) - 1))
                backward(g0, std::true_type());
            else
                backward(g0, std::false_type());
        }
        __syncthreads();
        if (OUTPUT) {
            if (at.inside(s0)) {
                Elements<T, S::kV> x, dt, z, dy;  // (once more: in registers meanwhile they would cost more)
                x.clear();
                dt.clear();
                z.clear();
                if (on) {
                    F::load(x, a.x, at, s0, true);
                    F::load(dt, a.dt, at, s0, true);
                    F::load(dy, a.dy, at, s0, true);
                    if (gated) F::load(z, a.z, at, s0, true);
                    const auto bias = of_channels<S::kV>(p.dt_bias, c_mem, at.there), skips = of_channels<S::kV>(p.d, c_mem, at.there);
                    const Two ones = two(1.0f, 1.0f), minus = two(-1.0f, -1.0f), ln2 = two(kLn2, kLn2);
#pragma unroll
                    for (int i = 0; i < S::kV; i += 2) {
                        const float4 r0 = sh.prepared[at.slot][i * 8 + at.m], r1 = sh.prepared[at.slot][i * 8 + 8 + at.m];
                        const Two xi = x.pair(i), skip = skips.pair(i), gb = two(r0.x, r1.x), gah = two(r0.y, r1.y);
                        Two dv = dy.pair(i);
                        if (gated) {
                            const Two zi = z.pair(i), sig = sigmoid_of(zi), gate = zi * sig;
                            // d(z sig) = sig (1 + z (1 - sig)) = sig + gate (1 - sig)
                            z.set_pair(i, dv * fma(skip, xi, two(r0.z, r1.z)) * fma(gate, fma(sig, minus, ones), sig));
                            dv = dv * gate;
                        }
                        Two dd = fma(xi, gb, gah * ln2);
                        if (softplus) dd = dd * sigmoid_of(dt.pair(i) + bias.pair(i));
                        const Two dx = fma(two(r0.w, r1.w), gb, skip * dv);
                        d_bias[i / 2] = d_bias[i / 2] + dd;
                        d_skip[i / 2] = fma(dv, xi, d_skip[i / 2]);
                        x.set_pair(i, dx);
                        dt.set_pair(i, dd);
                    }
                }
                F::store(x, a.dx, at, s0);
                F::store(dt, a.ddt, at, s0);
                if (gated) F::store(z, a.dz, at, s0);
            }
            constexpr int n2 = 2 * S::kAll;
            float* const to = work.across + (((blockIdx.x % cuts.groups) * p.blocks + at.q) * (int64_t)p.t + s0) * n2;
#pragma unroll
            for (int i = threadIdx.x; i < kRun * n2 / 4; i += kThreads) {
                const int slot = i / (n2 / 4), n = i % (n2 / 4) * 4;
                float4 v = *reinterpret_cast<const float4*>(sh.across(0, slot) + n);
#pragma unroll
                for (int w = 1; w < kWarps; ++w) {
                    const float4 u = *reinterpret_cast<const float4*>(sh.across(w, slot) + n);
                    v = make_float4(v.x + u.x, v.y + u.y, v.z + u.z, v.w + u.w);
                }
                if (s0 + slot >= at.begin && s0 + slot < at.stop) *reinterpret_cast<float4*>(to + i * 4) = v;
            }
        }
        __syncthreads();
    }
    if (!OUTPUT) {
        turn(e);
        store_states(p, at, work.state + cell * per + first_state, e);
        if (at.part == 0) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (at.c0 + at.ch[c] < p.channels) work.delta[cell * p.channels + at.c0 + at.ch[c]] = passed[c];
        }
        return;
    }
    float* const frames = work.frames + cell * (per + 2 * p.channels);
    turn(dA);
    store_states(p, at, frames + first_state, dA);
    // the sixteen slots' threads of a channel, in their order
    float2* const both = reinterpret_cast<float2*>(&sh.kept[0][0][0]);
#pragma unroll
    for (int i = 0; i < S::kV; i += 2) {
        const float2 d = one(d_skip[i / 2]), b = one(d_bias[i / 2]);
        both[at.slot * S::kChannels + at.m * S::kV + i] = make_float2(d.x, b.x);
        both[at.slot * S::kChannels + at.m * S::kV + i + 1] = make_float2(d.y, b.y);
    }
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

// A lane has four states of a channel, LANES of them the channel, in kStepRows rows, whose loads are all under way before the first is
// used.  Bytes: the states, in and out.  WIDE: states and rows of b and c in pieces of four.
constexpr int kStepRows = 4;
template <typename T, int LANES, bool WIDE>
__global__ void __launch_bounds__(kThreads) k41_scan_step(const ScanStepParams p, const ScanStepTensors<T> a, unsigned groups)
{
    const unsigned at = blockIdx.x / groups;
    const int64_t row0 = (int64_t)at * kStepRows;
    const int part = threadIdx.x % LANES, n0 = part * 4;
    const int64_t c = (int64_t)(blockIdx.x - at * groups) * (kThreads / LANES) + threadIdx.x / LANES;
    const bool on = c < p.channels && n0 < p.states, there = c < p.channels;
    const int rows = (int)min(p.rows - row0, (int64_t)kStepRows);
    const bool in_place = p.next == p.state;
    int here[kStepRows];
#pragma unroll
    for (int r = 0; r < kStepRows; ++r) here[r] = r < rows ? p.pos[row0 + r] : -1;

    const int64_t per = p.channels * p.states, first = row0 * per + c * p.states + n0;
    Elements<float, 4> h[kStepRows], decays;
    Elements<T, 4> b[kStepRows], cc[kStepRows];
    float x[kStepRows], dt[kStepRows], z[kStepRows];
    const int left = p.states - n0;
    {
        const float* from = p.state + first;
        const T *bp = a.b + row0 * a.sb + n0, *cp = a.c + row0 * a.sc + n0, *xp = a.x + row0 * a.sx + c, *dp = a.dt + row0 * a.sdt + c,
                *zp = a.z ? a.z + row0 * a.sz + c : nullptr;
#pragma unroll
        for (int r = 0; r < kStepRows; ++r) {
            h[r].clear();
            b[r].clear();
            cc[r].clear();
            if (on && r < rows) {  // (whether or not they will be used: positions arrive no sooner)
                h[r].load(from, WIDE ? 4 : left, WIDE);
                b[r].load(bp, WIDE ? 4 : left, WIDE);
                cc[r].load(cp, WIDE ? 4 : left, WIDE);
            }
            x[r] = there && r < rows ? to_float(*xp) : 0.0f;
            dt[r] = there && r < rows ? to_float(*dp) : 0.0f;
            z[r] = there && r < rows && a.z ? to_float(*zp) : 0.0f;
            from += per;
            bp += a.sb;
            cp += a.sc;
            xp += a.sx;
            dp += a.sdt;
            if (a.z) zp += a.sz;
        }
    }
    decays.clear();
    float bias = 0.0f, skip = 0.0f;
    if (on) decays.load(p.a + c * p.states + n0, WIDE ? 4 : left, WIDE);
    if (there) {
        bias = p.dt_bias ? p.dt_bias[c] : 0.0f;
        skip = p.d ? p.d[c] : 0.0f;
    }
    Two a2[2] = {decays.pair(0) * two(kLog2E, kLog2E), decays.pair(2) * two(kLog2E, kLog2E)};
    float* to = p.next + first;
    T* yp = a.y + row0 * a.sy + c;
#pragma unroll
    for (int r = 0; r < kStepRows; r += 2) {
        // two rows' delta together
        Two delta = two(dt[r] + bias, dt[r + 1] + bias);
        if (p.softplus) delta = softplus_of(delta);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int k = r + i;
            if (k >= rows) break;
            const float d = i ? one(delta).y : one(delta).x;
            const Two d2 = two(d, d), u = two(d * x[k], d * x[k]);
            Two sum = zero();
            if (here[k] >= 0) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const Two push = u * b[k].pair(2 * j), now = here[k] > 0 ? fma(decay(d2, a2[j]), h[k].pair(2 * j), push) : push;
                    h[k].set_pair(2 * j, now);
                    sum = fma(now, cc[k].pair(2 * j), sum);
                }
            }
            float y = one(sum).x + one(sum).y;
#pragma unroll
            for (int bit = LANES / 2; bit; bit /= 2) y += __shfl_xor_sync(0xffffffffu, y, bit);
            if (on && (here[k] >= 0 || !in_place)) h[k].store(to, WIDE ? 4 : left, WIDE);
            if (there && part == 0) {
                y = fmaf(skip, x[k], y);
                if (a.z) y *= z[k] * sigmoid_of(z[k]);
                *yp = from_float<T>(here[k] >= 0 ? y : 0.0f);
            }
            to += per;
            yp += a.sy;
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

// Segments per walk.  Four CTAs of a walk fit on an SM at once, 592 in all.  What that is for: walks that are too few for it, and a
// second wave that would be almost empty.  Many small segments (two waves or more, up to 14 CTAs per SM) level the SMs out; where the
// runs do not suffice for that, 16 to a segment, one wave.
// Forward, one wave of walks that take half a CTA more (kHalves, two to an SM) does without segments.  It takes as long as an SM with two
// walks, however many SMs have only one; segments take time by the walks, and by how much of each its successor hears of.  So halves from
// three quarters of the wave on; from two thirds on in blocks of less than 128 runs, where few segments fit and the last wave of them is
// part empty; and always where a block makes two segments at most.  Halves / segments, us, 16 states bf16, with last states not wanted:
//     4096 slots, packed tokens      149 walks 623 / 509, 192 635 / 583, 208 630 / 627, 222 635 / 646, 240 635 / 693, 256 634 / 726
//     one sequence a block           149 621 / 525, 192 628 / 634, 208 628 / 697, 222 627 / 720, 256 629 / 826
//     lengths of 30 in the middle    149 632 / 384, 192 639 / 468, 208 638 / 501, 222 643 / 523, 256 641 / 552
//     1024 slots, packed tokens      149 165 / 161, 160 167 / 153, 192 168 / 159, 208 169 / 198, 222 169 / 191, 256 168 / 218
//     640 slots                      149 107 / 107, 192 109 / 110, 208 109 / 134;    512: 149 87 / 103, 192 88 / 118, 222 89 / 120
//     32,768 slots                   149 4,916 / 2,947, 192 4,959 / 3,576, 222 4,957 / 3,921, 256 4,954 / 4,330 (one sequence 6,368)
// (Other walks, prompts of 8 x 4096 x 2048: one segment of whole CTAs 742, 2 775, 4 766, 8 749; training of the same
// 1 segment 3,051, 2 3,057, 4 2,833, 8 2,658; 4 x 10,000 x 1024 training, 64 walks: 9 segments 1,664, 18
// 1,599, 32 1,563; 16 x 4096 x 2048 prompts, 512 walks: one segment 1,103, four 1,407; 20,011 x 509 fp32, 8 walks: 74 segments 470, 78 635;
// 512 walks of 2048 slots, training: one segment 2,372, four 2,626; halves: 4 x 4096 x 2048 440 to 483 instead of 416, 384 walks 1,005
// instead of 911.  Segments that end at a start anywhere in the next share, rather than in
// its first half: 746 instead of 749 and 1,603 instead of 1,555: too unequal.)
constexpr int64_t kHalves = 2 * 148;
ScanCuts cuts_of(int64_t blocks, int32_t t, int64_t channels, int states, bool gradient)
{
    return with_split(states, [&](auto s) {
        using S = decltype(s);
        ScanCuts cuts;
        cuts.groups = (int)((channels + S::kChannels - 1) / S::kChannels);
        const int64_t walks = blocks * cuts.groups, runs = (t + kRun - 1) / kRun, at_once = 4 * 148;
        int64_t n = 1;
        const int64_t from = runs < 48 ? 149 : runs < 128 ? kHalves * 2 / 3 + 1 : kHalves * 3 / 4;
        const bool halves = !gradient && walks >= from && walks <= kHalves;
        if (!halves && (walks < at_once / 2 || (walks > at_once && walks < at_once * 3 / 2))) {
            const int64_t many = 14 * 148 / walks, fit = runs / 16 < many ? runs / 16 : many;
            n = fit * walks >= 2 * at_once ? fit : at_once / walks < fit ? at_once / walks : fit;
        }
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

// Tensors whose pieces of `n` bytes lie on boundaries of their size (at most 16), with blocks of t slots that span less than 2^32 bytes
template <typename T>
bool on(const Channels<T>& x, size_t n, int32_t t)
{
    const size_t m = n < 16 ? n : 16;
    return !x.data || (reinterpret_cast<uintptr_t>(x.data) % m == 0 && x.block * sizeof(T) % m == 0 && x.slot * sizeof(T) % m == 0 &&
                       (uint64_t)x.slot * sizeof(T) < ((uint64_t)1 << 32) / ((uint64_t)t + 2 * kRun));
}
template <typename T>
ScanParams with_rows(ScanParams p, const ScanTensors<T>& a)
{
    p.rows_wide = on(a.b, 16, p.t) && on(a.c, 16, p.t) && p.states * sizeof(T) % 16 == 0;
    return p;
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
    return work_of(nullptr, cuts_of(blocks, t, channels, states, gradient), blocks, t, channels, states, gradient).bytes;
}

template <typename T>
cudaError_t launch_scan(const ScanParams& params, const ScanTensors<T>& a, cudaStream_t st)
{
    const ScanParams p = with_rows(params, a);
    return with_split(p.states, [&](auto s) {
        using S = decltype(s);
        const ScanCuts cuts = cuts_of(p.blocks, p.t, p.channels, p.states, false);
        const ScanWork work = work_of(p.work, cuts, p.blocks, p.t, p.channels, p.states, false);
        constexpr size_t n = S::kV * sizeof(T);
        const bool wide = on(a.x, n, p.t) && on(a.dt, n, p.t) && on(a.z, n, p.t) && on(a.y, n, p.t) && p.channels % S::kV == 0;
        const unsigned grid = (unsigned)(cuts.segments * p.blocks * cuts.groups);
        if (cuts.segments > 1) {
            auto* part = wide ? k37_scan<T, S, true, false, false> : k37_scan<T, S, false, false, false>;
            part<<<grid, kThreads, 0, st>>>(p, a, cuts, work);
            count_launches(1);
            cudaError_t e = cudaGetLastError();
            if (e == cudaSuccess) e = join(p, cuts, work, false, st);
            if (e != cudaSuccess) return e;
        }
        const bool halves = cuts.segments == 1 && grid <= kHalves;
        auto* kernel = halves ? (wide ? k37_scan<T, S, true, true, true> : k37_scan<T, S, false, true, true>)
                              : (wide ? k37_scan<T, S, true, true, false> : k37_scan<T, S, false, true, false>);
        kernel<<<grid, halves ? 2 * kThreads : kThreads, 0, st>>>(p, a, cuts, work);
        count_launches(1);
        return cudaGetLastError();
    });
}

template <typename T>
cudaError_t launch_scan_grad(const ScanParams& params, const ScanTensors<T>& a, cudaStream_t st)
{
    const ScanParams p = with_rows(params, a);
    return with_split(p.states, [&](auto s) {
        using S = decltype(s);
        const ScanCuts cuts = cuts_of(p.blocks, p.t, p.channels, p.states, true);
        const ScanWork work = work_of(p.work, cuts, p.blocks, p.t, p.channels, p.states, true);
        constexpr size_t n = S::kV * sizeof(T);
        const bool wide = on(a.x, n, p.t) && on(a.dt, n, p.t) && on(a.z, n, p.t) && on(a.dy, n, p.t) && on(a.dx, n, p.t) && on(a.ddt, n, p.t) && on(a.dz, n, p.t) &&
                          p.channels % S::kV == 0;
        const unsigned grid = (unsigned)(cuts.segments * p.blocks * cuts.groups);
        constexpr int kShared = sizeof(GradShared<S>);
        static std::atomic<uint64_t> allowed[4] = {};
        auto *part = wide ? k39_scan_grad<T, S, true, false> : k39_scan_grad<T, S, false, false>,
             *kernel = wide ? k39_scan_grad<T, S, true, true> : k39_scan_grad<T, S, false, true>;
        cudaError_t e = allow_shared(kernel, kShared, allowed[wide]);
        if (e == cudaSuccess) e = allow_shared(part, kPartShared<S>, allowed[2 + wide]);
        if (e != cudaSuccess) return e;
        if (cuts.segments > 1) {
            part<<<grid, kThreads, kPartShared<S>, st>>>(p, a, cuts, work);
            count_launches(1);
            e = cudaGetLastError();
            if (e == cudaSuccess) e = join(p, cuts, work, true, st);
            if (e != cudaSuccess) return e;
        }
        kernel<<<grid, kThreads, kShared, st>>>(p, a, cuts, work);
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
        const unsigned groups = (unsigned)((p.channels + kThreads / L - 1) / (kThreads / L));
        auto on_16 = [](const float* x) { return reinterpret_cast<uintptr_t>(x) % 16 == 0; };
        auto on_4 = [&](const T* x, int64_t row) { return reinterpret_cast<uintptr_t>(x) % (4 * sizeof(T)) == 0 && row % 4 == 0; };
        const bool wide = p.states % 4 == 0 && on_16(p.state) && on_16(p.next) && on_16(p.a) && on_4(a.b, a.sb) && on_4(a.c, a.sc);
        auto* kernel = wide ? k41_scan_step<T, L, true> : k41_scan_step<T, L, false>;
        kernel<<<(unsigned)((p.rows + kStepRows - 1) / kStepRows) * groups, kThreads, 0, st>>>(p, a, groups);
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

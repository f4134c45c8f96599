// k27_recurrence: gated linear recurrence along the slots of packed blocks, restarted at every sequence start,
//     f = sigmoid(gate);  h = f h_prev + (1 - f) x
// and its gradient.  The work is bytes only: three tensors move forward, five backward.
//
// A CTA owns 64 channels of a block and walks the slots in runs of 64: 8 warps take 8 slots each, a lane 2 channels.  h_out =
// A h_in + H over any stretch of slots, and stretches compose: a warp reduces its slots to (A, H), every warp then applies those
// of all eight to the state, which gives its own entering state and the next run's.  One barrier per run; the next runs' data
// are under way meanwhile.
//
// Where there are too few such walks for the machine, the slots are cut into segments, a CTA each.  A segment that starts inside
// a sequence needs the state of the one before it, so a segment that ends inside a sequence first reduces itself to (A, H) --
// only from the last sequence start on, which positions tell without a search -- and publishes that, or the state itself if a
// sequence starts inside; its successor looks back over published (A, H) to the nearest state.  Segments are taken by ticket, in
// the order of the walk, so those that one waits for were taken by CTAs that run or have ended, whatever the scheduling.
//
// The gradient walks backwards: E = f g (0 where a sequence starts) is what a slot hands to the one before it, and E_out =
// A E_in + E over a stretch.  It rebuilds h from the states that the forward call kept at the start of each run.
#include <math.h>

#include <type_traits>

#include "bload_internal.cuh"
#include "bload_layers.cuh"

namespace bload {

namespace {

constexpr int kRun = BLOAD_RECURRENCE_RUN;
constexpr int kWarps = 8, kRows = kRun / kWarps, kCh = 64;

__device__ unsigned int g_timeouts;  // bounded waits that gave up (bload_device_timeouts)

// Scratch: a ticket, then per segment (all groups of channels of the first, of the second, ...) a flag, (A, H) and the state.
struct WorkView2 {
    unsigned int* ticket;
    unsigned int* flags;  // 0 nothing, 1 (A, H), 2 the state behind the segment as well
    float4* sums;         // [parts][32]: A, H of a lane's two channels
    float2* states;       // [parts][32]
};
__host__ __device__ inline size_t work_view(int64_t parts, void* base, WorkView2* v)
{
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t flags = 256, sums = flags + up(4 * (size_t)parts), states = sums + 512 * (size_t)parts;
    if (v) {
        char* b = static_cast<char*>(base);
        v->ticket = reinterpret_cast<unsigned int*>(b);
        v->flags = reinterpret_cast<unsigned int*>(b + flags);
        v->sums = reinterpret_cast<float4*>(b + sums);
        v->states = reinterpret_cast<float2*>(b + states);
    }
    return states + 256 * (size_t)parts;
}

// f = sigmoid(g) and 1 - f, each with a small relative error of its own (1 - f must not cancel: it scales the input).  With e =
// exp(-g): f = 1 / (1 + e), 1 - f = e f; g has been held at -87, so that e f does not become inf * 0, and all but 7e-6 of what f is
// then (1.6458e-38) is taken off again: f is above 0 whatever the approximations' last bits (a state that is infinite stays so), and
// down to g = -75 the difference is below 7e-6 of f, below its rounding down to -70.
__device__ __forceinline__ void gate_of(Two g, Two& f, Two& keep)
{
    const float2 y = one(g * two(-1.4426950408889634f, -1.4426950408889634f));
    float2 e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(y.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(y.y));
    const float2 d = one(two(e.x, e.y) + two(1.0f, 1.0f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(d.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(d.y));
    f = two(r.x, r.y);
    keep = two(e.x, e.y) * f;
    f = f + two(-1.6458e-38f, -1.6458e-38f);
}

// A stretch of slots, seen as one: state -> A state + H.  Nothing passes through a stretch in which a sequence starts or that
// holds padding, not even NaN: its A is -0 (gates are above 0, so no product of them is), and what arrives is dropped.  A product of
// small gates may be 0, though: an infinite state passes all the same, as it does slot by slot.  INFINITE: with that test; where it
// costs, chains are followed without, and once more with it if their end is not finite.
constexpr float kShut = -0.0f;
__device__ __forceinline__ bool shut(float A) { return __float_as_int(A) < 0; }
template <bool INFINITE>
__device__ __forceinline__ float open_through(float A, float state, float H)
{
    return INFINITE && A == 0.0f && fabsf(state) == INFINITY ? state + H : fmaf(A, state, H);
}
__device__ __forceinline__ float through(float A, float state, float H) { return shut(A) ? H : open_through<true>(A, state, H); }
// a stretch of two channels: (A, A', H, H')
struct alignas(16) Stretch {
    float2 A, H;
};
__device__ __forceinline__ Two through(const Stretch& s, Two state)
{
    const float2 x = one(state);
    return two(through(s.A.x, x.x, s.H.x), through(s.A.y, x.y, s.H.y));
}
__device__ __forceinline__ bool any_infinite(Two x)  // or NaN, in the warp
{
    return __any_sync(0xffffffffu, !(fabsf(one(x).x) < INFINITY) || !(fabsf(one(x).y) < INFINITY));
}
__device__ __forceinline__ Two open_through(const Stretch& s, Two state)  // neither channel's A is -0
{
    return fma(two(s.A.x, s.A.y), state, two(s.H.x, s.H.y));
}

__device__ __forceinline__ unsigned int flag_of(const unsigned int* p)
{
    unsigned int v;
    asm volatile("ld.acquire.gpu.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
// by one lane, after the warp's writes: they are visible to whoever sees the flag
__device__ __forceinline__ void set_flag(unsigned int* p, unsigned int v, int lane)
{
    __threadfence();
    __syncwarp();
    if (lane == 0) asm volatile("st.release.gpu.u32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}

// The state that enters a segment, for this lane's two channels, by a whole warp: finds the nearest segment before it whose state
// is published, with (A, H) of all between published too, and applies those in the order of the walk.  That is the same chain
// of multiply-adds wherever the state was found, so results do not depend on timing.  Gives up after four seconds, which
// nothing but a hardware failure takes.
__device__ float2 look_back(const WorkView2& w, int64_t part, int64_t step, int lane)
{
    uint64_t since = 0;
    int64_t far = 1;  // how many segments back the lanes begin to look
    for (;;) {
        const int64_t mine = part - (far + lane) * step;
        const unsigned flag = mine >= 0 ? flag_of(w.flags + mine) : 0;
        const unsigned ready = __ballot_sync(0xffffffffu, flag >= 1), state = __ballot_sync(0xffffffffu, flag == 2);
        const int run = ~ready ? __ffs(~ready) - 1 : 32, stop = state ? __ffs(state) - 1 : 32;
        if (stop < run) {
            far += stop;
            break;
        }
        if (run == 32) {
            far += 32;
            continue;
        }
        far = 1;
        uint64_t now;
        asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
        if (since == 0) since = now;
        if (__any_sync(0xffffffffu, now - since > 4000000000ull)) {
            if (lane == 0) atomicAdd(&g_timeouts, 1u);
            return make_float2(0.0f, 0.0f);
        }
        __nanosleep(40);
    }
    __threadfence();
    const float2 from = __ldcg(w.states + (part - far * step) * 32 + lane);
    auto follow = [&](auto infinite) {
        constexpr bool kInfinite = decltype(infinite)::value;
        float2 e = from;
        for (int64_t k = far - 1; k > 0; k -= 16) {  // sixteen loads at a time
            float4 s[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) s[j] = k > j ? __ldcg(w.sums + (part - (k - j) * step) * 32 + lane) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (k > j) e = make_float2(open_through<kInfinite>(s[j].x, e.x, s[j].y), open_through<kInfinite>(s[j].z, e.y, s[j].w));
        }
        return e;
    };
    const float2 e = follow(std::false_type());
    return any_infinite(two(e.x, e.y)) ? follow(std::true_type()) : e;
}

// `bytes` of 16 bytes are copied, the rest are zeros
__device__ __forceinline__ void copy16(void* dst, const void* src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(bytes)
                 : "memory");
}

template <typename T>
struct Pair;  // two neighbouring elements; get_gate holds them at -87 (NaN stays)
template <>
struct Pair<float> {
    using type = float2;
    static __device__ __forceinline__ Two get(float2 x) { return two(x.x, x.y); }
    static __device__ __forceinline__ Two get_gate(float2 x)
    {
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.x) : "f"(-87.0f));
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.y) : "f"(-87.0f));
        return two(x.x, x.y);
    }
    static __device__ __forceinline__ float2 put(float2 x) { return x; }
    static __device__ __forceinline__ float2 join(float a, float b) { return make_float2(a, b); }
};
template <>
struct Pair<__half> {
    using type = __half2;
    static __device__ __forceinline__ Two get(__half2 x) { return two(__low2float(x), __high2float(x)); }
    static __device__ __forceinline__ Two get_gate(__half2 x) { return get(__hmax2_nan(x, __float2half2_rn(-87.0f))); }
    static __device__ __forceinline__ __half2 put(float2 x) { return __floats2half2_rn(x.x, x.y); }
    static __device__ __forceinline__ __half2 join(__half a, __half b) { return __halves2half2(a, b); }
};
template <>
struct Pair<__nv_bfloat16> {
    using type = __nv_bfloat162;
    static __device__ __forceinline__ Two get(__nv_bfloat162 x) { return two(__low2float(x), __high2float(x)); }
    static __device__ __forceinline__ Two get_gate(__nv_bfloat162 x) { return get(__hmax2_nan(x, __float2bfloat162_rn(-87.0f))); }
    static __device__ __forceinline__ __nv_bfloat162 put(float2 x) { return __floats2bfloat162_rn(x.x, x.y); }
    static __device__ __forceinline__ __nv_bfloat162 join(__nv_bfloat16 a, __nv_bfloat16 b) { return __halves2bfloat162(a, b); }
};

// Brings runs to a warp.  STAGED: rows on 16-byte boundaries, copied to shared memory asynchronously, some runs ahead; a lane has
// channels 2l and 2l + 1.  Otherwise elements are loaded one by one into registers, a run ahead, or for three tensors, which would
// not fit beside the run's own values, when the run's turn has come; a lane has channels l and l + 32, so that its loads and stores
// stay side by side with its neighbours'.  (Asynchronous copies of 4 bytes, where rows allow them, were slower: 30,001 x 251 fp32
// 52 us forward and 76 gradient instead of 42 and 59.)
// TENSORS 2: gate and x, or (DH) gate and dh; 3: gate, x, dh.
template <typename T, int TENSORS, bool DH, bool STAGED>
struct Feed {
    static constexpr bool kStaged = STAGED, kEarly = kStaged || TENSORS == 2;
    static constexpr int kRowBytes = kCh * sizeof(T), kTensorBytes = kRows * kRowBytes, kRunBytes = kWarps * TENSORS * kTensorBytes;
    static constexpr int kStages = !kStaged ? 2 : kRunBytes <= 16384 ? 4 : kRunBytes <= 32768 ? 3 : 2;  // of up to 96 KB in all
    static constexpr int kPieces = kStaged ? kRowBytes / 16 : 32, kRowsAtOnce = 32 / kPieces;  // per row; rows that a warp copies at once
    static constexpr int kPer = kStaged ? 16 / (int)sizeof(T) : 1;                             // elements of a piece

    const RecurTensors<T>& a;
    const T* at[TENSORS];  // this lane's first element of the next run to fetch
    const int32_t* pos;
    uint8_t* ring;
    int t, s, lane;          // s: the warp's first slot of the next run to fetch
    int left;                // channels from this lane's first one on (at most 64)
    bool inside;             // (uniform) all 64 channels exist
    int ahead[kStages - 1];  // positions of the runs under way
    T raw[kStaged ? 1 : TENSORS][kStaged ? 1 : kRows][2];

    __device__ __forceinline__ explicit Feed(const RecurTensors<T>& tensors) : a(tensors) {}
    __device__ __forceinline__ const Channels<const T>& tensor(int n) const { return n == 0 ? a.gate : n == 2 || DH ? a.dh : a.x; }
    __device__ __forceinline__ void init(const RecurParams& p, int64_t q, int64_t ch0, int run, uint8_t* shared)
    {
        const int warp = threadIdx.x >> 5;
        lane = threadIdx.x & 31;
        ring = shared + warp * TENSORS * kTensorBytes;
        t = p.t;
        s = run * kRun + warp * kRows;
        pos = p.pos + q * p.t;
        const int c = lane % kPieces * kPer, r = lane / kPieces;
        left = (int)min(p.channels - ch0, (int64_t)kCh) - c;
        inside = ch0 + kCh <= p.channels;
#pragma unroll
        for (int n = 0; n < TENSORS; ++n) at[n] = tensor(n).data + q * tensor(n).block + (int64_t)(s + r) * tensor(n).slot + ch0 + c;
    }
    // begins to fetch the next run into a stage, its positions into ahead[k]; `on`: there is one
    template <int DIR>
    __device__ __forceinline__ void fetch(int stage, int k, bool on)
    {
        if (on) {
            ahead[k] = lane < kRows && s + lane < t ? pos[s + lane] : -1;
            const bool full = s + kRows <= t && inside;  // (uniform)
#pragma unroll
            for (int n = 0; n < TENSORS; ++n) {
                const int64_t slot = tensor(n).slot;
                if (kStaged) {
                    uint8_t* const to = ring + stage * kRunBytes + n * kTensorBytes + lane * 16;
                    const T* from = at[n];
                    if (full) {
#pragma unroll
                        for (int j = 0; j < kRows / kRowsAtOnce; ++j, from += kRowsAtOnce * slot) copy16(to + j * 512, from, 16);
                    } else {
#pragma unroll
                        for (int j = 0; j < kRows / kRowsAtOnce; ++j, from += kRowsAtOnce * slot) {
                            const int bytes = s + lane / kPieces + j * kRowsAtOnce >= t ? 0 : min(max(left * (int)sizeof(T), 0), 16);
                            copy16(to + j * 512, bytes ? from : tensor(n).data, bytes);
                        }
                    }
                } else {
#pragma unroll
                    for (int r = 0; r < kRows; ++r)
#pragma unroll
                        for (int c = 0; c < 2; ++c)
                            raw[kStaged ? 0 : n][kStaged ? 0 : r][c] = full || (left > 32 * c && s + r < t) ? at[n][r * slot + 32 * c] : from_float<T>(0.0f);
                }
                at[n] += DIR * kRun * slot;
            }
            s += DIR * kRun;
        }
        if (kStaged) asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ __forceinline__ typename Pair<T>::type get(int stage, int n, int r) const
    {
        const uint8_t* const row = ring + stage * kRunBytes + n * kTensorBytes + r * kRowBytes;
        if (!kStaged) return Pair<T>::join(raw[kStaged ? 0 : n][kStaged ? 0 : r][0], raw[kStaged ? 0 : n][kStaged ? 0 : r][1]);
        return reinterpret_cast<const typename Pair<T>::type*>(row)[lane];
    }
};

// OUTPUT false: only reduces `count` runs from `run` on (direction of the walk) to (A, state).
// before(state): called when the first runs are under way, brings the state that enters.
template <typename T, bool GRAD, bool STAGED, bool OUTPUT, typename Before>
__device__ __forceinline__ void walk(const RecurParams& p, const RecurTensors<T>& a, int64_t q, int64_t ch0, int run, int count,
                                     uint8_t* ring, Stretch (&sums)[2][GRAD ? 2 : 1][kWarps][32], Two (&entering)[2][32], Two& state, float2& A,
                                     const Before& before)
{
    constexpr int kTensors = GRAD && OUTPUT ? 3 : 2;
    constexpr int kDir = GRAD ? -1 : 1;
    constexpr bool kForward = !GRAD || OUTPUT;  // h is needed
    using F = Feed<T, kTensors, GRAD && !OUTPUT, STAGED>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int runs = (p.t + kRun - 1) / kRun;
    constexpr bool kApart = !STAGED;
    const int64_t c0 = ch0 + (kApart ? lane : 2 * lane), c1 = kApart ? c0 + 32 : c0 + 1;
    const bool on0 = c0 < p.channels, on1 = c1 < p.channels;

    F feed(a);
    feed.init(p, q, ch0, run, ring);
#pragma unroll
    for (int k = 0; k < F::kStages - 1 && F::kEarly; ++k) feed.template fetch<kDir>(k, k, k < count);
    before(state);
    if (warp == 0) entering[0][lane] = state;

    T *out0 = nullptr, *out1 = nullptr;  // this lane's first element of the warp's first slot
    if (OUTPUT) {
        const Channels<T>& o = GRAD ? a.dgate : a.h;
        out0 = o.data + q * o.block + (int64_t)(run * kRun + warp * kRows) * o.slot + c0;
        if (GRAD) out1 = a.dx.data + q * a.dx.block + (int64_t)(run * kRun + warp * kRows) * a.dx.slot + c0;
    }
    float* carry_at = OUTPUT && p.carry ? p.carry + (q * runs + run) * p.channels : nullptr;

    int stage = 0;
    for (int i = 0; i < count; ++i, run += kDir) {
        const int s_warp = run * kRun + warp * kRows;
        if (!F::kEarly) feed.template fetch<kDir>(0, 0, true);
        Two h_in = zero();  // (gradient) the state that entered this run forward
        if (GRAD && OUTPUT) h_in = two(on0 ? carry_at[c0] : 0.0f, on1 ? carry_at[c1] : 0.0f);
        if (STAGED) {
            asm volatile("cp.async.wait_group %0;" ::"n"(F::kStages - 2) : "memory");
            __syncwarp();
        }
        constexpr unsigned kAll = (1u << kRows) - 1;
        const unsigned cont = __ballot_sync(0xffffffffu, feed.ahead[0] > 0) & kAll;   // bit r: slot r continues a sequence
        const unsigned valid = __ballot_sync(0xffffffffu, feed.ahead[0] >= 0) & kAll;  // is a frame

        Two f[kRows], keep[kRows], x[kRows], dh[GRAD ? kRows : 1];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            gate_of(Pair<T>::get_gate(feed.get(stage, 0, r)), f[r], keep[r]);
            if (kForward) x[r] = Pair<T>::get(feed.get(stage, 1, r));
            if (GRAD) dh[GRAD ? r : 0] = Pair<T>::get(feed.get(stage, kTensors - 1, r));
        }
        if (valid != kAll) {
#pragma unroll
            for (int r = 0; r < kRows; ++r)
                if (!((valid >> r) & 1)) {
                    f[r] = keep[r] = x[r] = zero();
                    if (GRAD) dh[GRAD ? r : 0] = zero();
                }
        }
        const int buffer = i & 1;
        Stretch own;
        own.A = make_float2(kShut, kShut);
        if (cont == kAll) {
            Two through_all = f[0];
#pragma unroll
            for (int r = 1; r < kRows; ++r) through_all = through_all * f[r];
            own.A = one(through_all);
        }
        if (kForward && !GRAD) {
#pragma unroll
            for (int r = 0; r < kRows; ++r) x[r] = keep[r] * x[r];
        }
        // (a warp without a break, the usual case, takes loops without tests)
        auto reduce = [&](auto with_breaks) {
            constexpr bool breaks = decltype(with_breaks)::value;
            if (kForward) {
                Two H = zero();
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    if (breaks && !((cont >> r) & 1)) H = zero();
                    H = fma(f[r], H, GRAD ? keep[r] * x[r] : x[r]);
                }
                own.H = one(H);
                sums[buffer][0][warp][lane] = own;
            }
            if (GRAD) {
                Two E = zero();
#pragma unroll
                for (int r = kRows - 1; r >= 0; --r) {
                    E = f[r] * (dh[GRAD ? r : 0] + E);
                    if (breaks && !((cont >> r) & 1)) E = zero();
                }
                own.H = one(E);
                sums[buffer][GRAD ? 1 : 0][warp][lane] = own;
            }
        };
        if (cont == kAll)
            reduce(std::false_type());
        else
            reduce(std::true_type());
        // the next run to fetch takes the stage of the run before this one (in registers: this one's)
        __syncwarp();
#pragma unroll
        for (int k = 0; k + 1 < F::kStages - 1; ++k) feed.ahead[k] = feed.ahead[k + 1];
        if (F::kEarly) feed.template fetch<kDir>(stage == 0 ? F::kStages - 1 : stage - 1, F::kStages - 2, i + F::kStages - 1 < count);
        stage = stage + 1 == F::kStages ? 0 : stage + 1;
        __syncthreads();

        if (OUTPUT && !GRAD && carry_at && warp == 0) {
            const float2 e = one(entering[buffer][lane]);
            if (on0) carry_at[c0] = e.x;
            if (on1) carry_at[c1] = e.y;
        }
        // The state that enters this warp: through the warps in front of it.  The last of them goes on to the next run's state and
        // leaves it for all, read behind the next barrier.  A shut stretch has A = -0, so a multiply-add drops what arrives --
        // unless that is infinite or NaN, which then shows in the end; only in that case are the stretches gone through again
        // with a test on each.
        const int in_front = GRAD ? kWarps - 1 - warp : warp;
        const Two entered = entering[buffer][lane];
        Two mine = entered;
#pragma unroll
        for (int k = 0; k < kWarps - 1; ++k)
            if (k < in_front) mine = open_through(sums[buffer][GRAD ? 1 : 0][GRAD ? kWarps - 1 - k : k][lane], mine);
        if (any_infinite(mine)) {
            mine = entered;
            for (int k = 0; k < in_front; ++k) mine = through(sums[buffer][GRAD ? 1 : 0][GRAD ? kWarps - 1 - k : k][lane], mine);
        }
        if (in_front == kWarps - 1) {
            entering[buffer ^ 1][lane] = through(sums[buffer][GRAD ? 1 : 0][warp][lane], mine);
        }
        if (!OUTPUT) {
#pragma unroll
            for (int k = 0; k < kWarps; ++k) {
                const Stretch s = sums[buffer][GRAD ? 1 : 0][k][lane];
                A = make_float2(shut(A.x) || shut(s.A.x) ? kShut : A.x * s.A.x, shut(A.y) || shut(s.A.y) ? kShut : A.y * s.A.y);
            }
        }
        if (!OUTPUT) continue;

        const bool full = s_warp + kRows <= p.t;  // (uniform)
        auto put = [&](T* at, Two v) {
            if (!kApart && on1) {
                *reinterpret_cast<typename Pair<T>::type*>(at) = Pair<T>::put(one(v));
            } else {
                if (on0) at[0] = from_float<T>(one(v).x);
                if (on1) at[kApart ? 32 : 1] = from_float<T>(one(v).y);
            }
        };
        auto finish = [&](auto with_breaks, auto with_edges) {
            constexpr bool breaks = decltype(with_breaks)::value, edges = decltype(with_edges)::value;
            auto store = [&](T* at, int r, Two v) {
                if (!edges && !kApart) {
                    *reinterpret_cast<typename Pair<T>::type*>(at) = Pair<T>::put(one(v));
                } else if (!edges) {
                    at[0] = from_float<T>(one(v).x);
                    at[32] = from_float<T>(one(v).y);
                } else if (full || s_warp + r < p.t) {
                    put(at, v);
                }
            };
            if (!GRAD) {
                T* at = out0;
#pragma unroll
                for (int r = 0; r < kRows; ++r, at += a.h.slot) {
                    if (breaks && !((cont >> r) & 1)) mine = zero();
                    mine = fma(f[r], mine, x[r]);
                    store(at, r, mine);
                }
            } else {
                const Two minus = two(-1.0f, -1.0f);
#pragma unroll
                for (int r = 0; r < kRows; ++r) {  // h in front of every slot, less x
                    if (breaks && !((cont >> r) & 1)) h_in = zero();
                    const Two before = h_in;
                    h_in = fma(f[r], before, keep[r] * x[r]);
                    x[r] = fma(x[r], minus, before);
                }
                T *at0 = out0 + (kRows - 1) * a.dgate.slot, *at1 = out1 + (kRows - 1) * a.dx.slot;
#pragma unroll
                for (int r = kRows - 1; r >= 0; --r, at0 -= a.dgate.slot, at1 -= a.dx.slot) {  // then g, from the last slot to the first
                    if (breaks && !((valid >> r) & 1)) mine = zero();
                    const Two g = dh[GRAD ? r : 0] + mine, dx = keep[r] * g;
                    mine = f[r] * g;
                    if (breaks && !((cont >> r) & 1)) mine = zero();
                    store(at0, r, dx * f[r] * x[r]);
                    store(at1, r, dx);
                }
            }
        };
        if (GRAD) {
            for (int k = 0; k < warp; ++k) h_in = through(sums[buffer][0][k][lane], h_in);
        }
        if (!(full && feed.inside))
            finish(std::true_type(), std::true_type());
        else if (cont == kAll)
            finish(std::false_type(), std::false_type());
        else
            finish(std::true_type(), std::false_type());
        if (!GRAD) {
            out0 += kRun * a.h.slot;
            if (carry_at) carry_at += p.channels;
        } else {
            out0 -= kRun * a.dgate.slot;
            out1 -= kRun * a.dx.slot;
            carry_at -= p.channels;
        }
    }
    if (STAGED) asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();  // the ring and the sums may be used again
    state = entering[count & 1][lane];
    __syncthreads();
}

template <typename T, bool GRAD, bool STAGED>
__global__ void __launch_bounds__(256, 2)
    k27_recurrence(const RecurParams p, const RecurTensors<T> a, int groups_per_block, int segments)
{
    extern __shared__ __align__(16) uint8_t ring[];  // [stages][8 warps][tensors][8 rows][64]
    __shared__ Stretch sums[2][GRAD ? 2 : 1][kWarps][32];
    __shared__ Two entering[2][32];
    __shared__ float2 from_before[32];
    __shared__ unsigned int drawn;

    const int lane = threadIdx.x & 31;
    const int runs = (p.t + kRun - 1) / kRun;
    const int64_t groups = p.blocks * groups_per_block;
    WorkView2 work;
    work_view(groups * segments, p.work, &work);
    int64_t part = blockIdx.x;
    if (segments > 1) {
        if (threadIdx.x == 0) drawn = atomicAdd(work.ticket, 1u);
        __syncthreads();
        part = drawn;
    }
    const int turn = (int)(part / groups);
    const int64_t group = part - turn * groups, q = group / groups_per_block, ch0 = (group - q * groups_per_block) * kCh;
    const int segment = GRAD ? segments - 1 - turn : turn;
    const int first = (int)((int64_t)runs * segment / segments), end = (int)((int64_t)runs * (segment + 1) / segments);
    Two state = zero();
    float2 A = make_float2(1.0f, 1.0f);
    if (segments > 1) {
        const int32_t* const pos = p.pos + q * p.t;
        const bool left = segment > 0 && pos[first * kRun] > 0;                  // a sequence crosses that edge
        const bool right = segment < segments - 1 && pos[end * kRun] > 0;
        const bool need = GRAD ? right : left, give = GRAD ? left : right;
        bool open = false;
        if (give) {  // the part of the segment that its successor in the walk hears of
            int from, count;
            if (GRAD) {
                const int stop = min(warp_seq_end(pos, p.t, first * kRun, lane), end * kRun);
                count = (stop - 1) / kRun - first + 1;
                from = first + count - 1;
                open = stop == end * kRun && need;
            } else {
                const int start = min(max(end * kRun - pos[end * kRun], 0), end * kRun - 1);
                from = max(start / kRun, first);
                count = end - from;
                open = start < first * kRun && need;
            }
            walk<T, GRAD, STAGED, false>(p, a, q, ch0, from, count, ring, sums, entering, state, A, [](Two&) {});
        }
        walk<T, GRAD, STAGED, true>(p, a, q, ch0, GRAD ? end - 1 : first, end - first, ring, sums, entering, state, A, [&](Two& enters) {
            if (threadIdx.x < 32) {
                const float2 own = one(enters);
                if (give && !open) {
                    work.states[part * 32 + lane] = own;
                    set_flag(work.flags + part, 2, lane);
                } else if (give) {
                    work.sums[part * 32 + lane] = make_float4(A.x, own.x, A.y, own.y);
                    set_flag(work.flags + part, 1, lane);
                }
                float2 e = make_float2(0.0f, 0.0f);
                if (need) e = look_back(work, part, groups, lane);
                if (open) {
                    work.states[part * 32 + lane] = make_float2(through(A.x, e.x, own.x), through(A.y, e.y, own.y));
                    set_flag(work.flags + part, 2, lane);
                }
                from_before[lane] = e;
            }
            __syncthreads();
            enters = two(from_before[lane].x, from_before[lane].y);
        });
    } else {
        walk<T, GRAD, STAGED, true>(p, a, q, ch0, GRAD ? end - 1 : first, end - first, ring, sums, entering, state, A, [](Two&) {});
    }
}

int64_t groups_of(int64_t blocks, int64_t channels) { return blocks * ((channels + kCh - 1) / kCh); }

// Segments per walk: as many as give each of the 148 SMs two CTAs, of at least 4 runs each; from 149 walks on, one.  8 x 2048 bf16 channels (256 walks) of
// 10,000 slots take 212 us in one segment each and 253 in two on heavy-tailed lengths (320 on one sequence, whose first segments
// are read twice); 144 walks of 20,000 slots 305 us in one segment, 222 in two (434 on one sequence).
int segments_of(int64_t blocks, int32_t t, int64_t channels)
{
    const int64_t runs = (t + kRun - 1) / kRun, groups = groups_of(blocks, channels);
    const int64_t wanted = (2 * 148) / groups, most = runs / 4, segments = wanted < most ? wanted : most;
    return (int)(segments < 1 ? 1 : segments);
}

template <typename T, bool GRAD, bool STAGED>
cudaError_t launch(const RecurParams& p, const RecurTensors<T>& a, cudaStream_t st)
{
    using F = Feed<T, GRAD ? 3 : 2, false, STAGED>;
    constexpr int kShared = STAGED ? F::kStages * F::kRunBytes : 0;
    static_assert(!GRAD || !STAGED || kShared >= Feed<T, 2, true, STAGED>::kStages * Feed<T, 2, true, STAGED>::kRunBytes, "both walks fit");
    const int64_t groups = groups_of(p.blocks, p.channels);
    const int segments = segments_of(p.blocks, p.t, p.channels);
    auto* kernel = k27_recurrence<T, GRAD, STAGED>;
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t shared = allow_shared(kernel, kShared, allowed);
    if (shared != cudaSuccess) return shared;
    if (segments > 1) {  // ticket and flags
        const cudaError_t e = cudaMemsetAsync(p.work, 0, 256 + 4 * (size_t)(groups * segments), st);
        if (e != cudaSuccess) return e;
    }
    kernel<<<(unsigned)(groups * segments), 256, kShared, st>>>(p, a, (int)((p.channels + kCh - 1) / kCh), segments);
    count_launches(1);
    return cudaGetLastError();
}

template <typename T>
bool on_16(const Channels<T>& x)
{
    return reinterpret_cast<uintptr_t>(x.data) % 16 == 0 && x.block * sizeof(T) % 16 == 0 && x.slot * sizeof(T) % 16 == 0;
}
template <typename T, bool GRAD>
cudaError_t launch_on(const RecurParams& p, const RecurTensors<T>& a, cudaStream_t st)
{
    const bool staged = on_16(a.gate) && on_16(a.x) && (GRAD ? on_16(a.dh) && on_16(a.dgate) && on_16(a.dx) : on_16(a.h));
    return staged ? launch<T, GRAD, true>(p, a, st) : launch<T, GRAD, false>(p, a, st);
}

}  // namespace

size_t recurrence_work_bytes(int64_t blocks, int32_t t, int64_t channels)
{
    const int segments = segments_of(blocks, t, channels);
    return segments > 1 ? work_view(groups_of(blocks, channels) * segments, nullptr, nullptr) : 0;
}

template <typename T>
cudaError_t launch_recurrence(const RecurParams& p, const RecurTensors<T>& a, cudaStream_t st)
{
    return launch_on<T, false>(p, a, st);
}
template <typename T>
cudaError_t launch_recurrence_grad(const RecurParams& p, const RecurTensors<T>& a, cudaStream_t st)
{
    return launch_on<T, true>(p, a, st);
}
#define BLOAD_INSTANTIATE(T)                                                                            \
    template cudaError_t launch_recurrence<T>(const RecurParams&, const RecurTensors<T>&, cudaStream_t); \
    template cudaError_t launch_recurrence_grad<T>(const RecurParams&, const RecurTensors<T>&, cudaStream_t);
BLOAD_INSTANTIATE(float)
BLOAD_INSTANTIATE(__half)
BLOAD_INSTANTIATE(__nv_bfloat16)
#undef BLOAD_INSTANTIATE

int64_t recurrence_timeouts()
{
    unsigned int v = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&v, g_timeouts, sizeof v) != cudaSuccess) {
        (void)cudaGetLastError();
        return -1;
    }
    return (int64_t)v;
}

}  // namespace bload

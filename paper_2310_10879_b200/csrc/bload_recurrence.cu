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
// exp(-g): f = 1 / (1 + e), 1 - f = e f; e is held at 2^126 (f at 2^-126) so that e f does not become inf * 0.
__device__ __forceinline__ void gate_of(float g, float& f, float& keep)
{
    float y = -1.4426950408889634f * g, e;
    asm("min.NaN.f32 %0, %1, 0f42FC0000;" : "=f"(y) : "f"(y));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(y));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(f) : "f"(1.0f + e));
    keep = e * f;
    f -= 1.1754943508222875e-38f;  // 2^-126: a gate held there is 0, others do not change
}

// A stretch of slots, seen as one: state -> A state + H.  Nothing passes through a stretch in which a sequence starts or that
// holds padding, not even NaN: its A is -0 (gates are not negative, so no product of them is), and what arrives is dropped.
constexpr float kShut = -0.0f;
__device__ __forceinline__ bool shut(float A) { return __float_as_int(A) < 0; }
__device__ __forceinline__ float through(float A, float state, float H) { return shut(A) ? H : fmaf(A, state, H); }
__device__ __forceinline__ float both(float A1, float A2) { return shut(A1) || shut(A2) ? kShut : A1 * A2; }

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
    float2 e = __ldcg(w.states + (part - far * step) * 32 + lane);
    for (int64_t k = far - 1; k > 0; k -= 8) {  // eight loads at a time
        float4 s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = k > j ? __ldcg(w.sums + (part - (k - j) * step) * 32 + lane) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (k > j) e = make_float2(fmaf(s[j].x, e.x, s[j].y), fmaf(s[j].z, e.y, s[j].w));
    }
    return e;
}

__device__ __forceinline__ void copy16(void* dst, const void* src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(bytes)
                 : "memory");
}

template <typename T>
struct Pair;  // two neighbouring elements
template <>
struct Pair<float> {
    using type = float2;
    static __device__ __forceinline__ float2 get(float2 x) { return x; }
    static __device__ __forceinline__ float2 put(float a, float b) { return make_float2(a, b); }
};
template <>
struct Pair<__half> {
    using type = __half2;
    static __device__ __forceinline__ float2 get(__half2 x) { return __half22float2(x); }
    static __device__ __forceinline__ __half2 put(float a, float b) { return __floats2half2_rn(a, b); }
};
template <>
struct Pair<__nv_bfloat16> {
    using type = __nv_bfloat162;
    static __device__ __forceinline__ float2 get(__nv_bfloat162 x) { return __bfloat1622float2(x); }
    static __device__ __forceinline__ __nv_bfloat162 put(float a, float b) { return __floats2bfloat162_rn(a, b); }
};

// One run as a warp and lane see it: 8 slots of 2 channels.
template <bool GRAD>
struct Run {
    float f[kRows][2], x[kRows][2], keep[GRAD ? kRows : 1][2], dh[GRAD ? kRows : 1][2];
    unsigned cont, valid;  // bit r: slot r continues a sequence, is a frame
};

// Brings runs to a warp, some ahead of their use.  STAGED: rows on 16-byte boundaries, copied to shared memory
// asynchronously, lane l has channels 2l and 2l + 1.  Otherwise elements are loaded one by one into registers, a run
// ahead, and lane l has channels l and l + 32.  TENSORS 2: gate and x, or (DH) gate and dh; 3: gate, x, dh.
template <typename T, int TENSORS, bool DH, bool STAGED>
struct Feed {
    static constexpr int kRowBytes = kCh * sizeof(T), kTensorBytes = kRows * kRowBytes, kRunBytes = kWarps * TENSORS * kTensorBytes;
    static constexpr int kStages = !STAGED ? 2 : kRunBytes <= 16384 ? 4 : kRunBytes <= 32768 ? 3 : 2;  // of up to 96 KB in all
    static constexpr int kPieces = kRowBytes / 16, kRowsAtOnce = 32 / kPieces;

    const RecurTensors<T>& a;
    const T* at[TENSORS];  // this lane's first element of the next run to fetch
    const int32_t* pos;
    uint8_t* ring;
    int t, s, bytes, lane;  // s: the warp's first slot of the next run to fetch; bytes: of a row that this lane copies at once
    int64_t left;           // channels from this lane's first one on
    int ahead[kStages - 1]; // positions of the runs under way
    T raw[STAGED ? 1 : TENSORS][STAGED ? 1 : kRows][2];

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
        const int c = STAGED ? lane % kPieces * (16 / (int)sizeof(T)) : lane, r = STAGED ? lane / kPieces : 0;
        left = p.channels - ch0 - c;
        bytes = left <= 0 ? 0 : left * (int64_t)sizeof(T) < 16 ? (int)left * (int)sizeof(T) : 16;
#pragma unroll
        for (int n = 0; n < TENSORS; ++n) at[n] = tensor(n).data + q * tensor(n).block + (int64_t)(s + r) * tensor(n).slot + ch0 + c;
    }
    // begins to fetch the next run into a stage, its positions into ahead[k]; `on`: there is one
    template <int DIR>
    __device__ __forceinline__ void fetch(int stage, int k, bool on)
    {
        if (on) {
            ahead[k] = lane < kRows && s + lane < t ? pos[s + lane] : -1;
#pragma unroll
            for (int n = 0; n < TENSORS; ++n) {
                const int64_t slot = tensor(n).slot;
                if (STAGED) {
                    uint8_t* const to = ring + stage * kRunBytes + n * kTensorBytes + lane * 16;
#pragma unroll
                    for (int j = 0; j < kRows / kRowsAtOnce; ++j) {
                        const bool in = s + lane / kPieces + j * kRowsAtOnce < t && bytes > 0;
                        copy16(to + j * 512, in ? at[n] + j * kRowsAtOnce * slot : tensor(n).data, in ? bytes : 0);
                    }
                } else {
#pragma unroll
                    for (int r = 0; r < kRows; ++r)
#pragma unroll
                        for (int c = 0; c < 2; ++c)
                            raw[STAGED ? 0 : n][STAGED ? 0 : r][c] = s + r < t && left > 32 * c ? at[n][r * slot + 32 * c] : from_float<T>(0.0f);
                }
                at[n] += DIR * kRun * slot;
            }
            s += DIR * kRun;
        }
        if (STAGED) asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ __forceinline__ float2 get(int stage, int n, int r) const
    {
        if (STAGED)
            return Pair<T>::get(reinterpret_cast<const typename Pair<T>::type*>(ring + stage * kRunBytes + n * kTensorBytes + r * kRowBytes)[lane]);
        return make_float2(to_float(raw[STAGED ? 0 : n][STAGED ? 0 : r][0]), to_float(raw[STAGED ? 0 : n][STAGED ? 0 : r][1]));
    }
};

// OUTPUT false: only reduces `count` runs from `run` on (direction of the walk) to (A, state).
template <typename T, bool GRAD, bool STAGED, bool OUTPUT>
__device__ __forceinline__ void walk(const RecurParams& p, const RecurTensors<T>& a, int64_t q, int64_t ch0, int run, int count,
                                     uint8_t* ring, float4 (&sums)[2][GRAD ? 2 : 1][kWarps][32], float2& state, float2& A)
{
    constexpr int kTensors = GRAD && OUTPUT ? 3 : 2;
    constexpr int kDir = GRAD ? -1 : 1;
    using F = Feed<T, kTensors, GRAD && !OUTPUT, STAGED>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int runs = (p.t + kRun - 1) / kRun;
    const int64_t c0 = ch0 + (STAGED ? 2 * lane : lane), c1 = STAGED ? c0 + 1 : c0 + 32;
    const bool on0 = c0 < p.channels, on1 = c1 < p.channels;

    F feed(a);
    feed.init(p, q, ch0, run, ring);
#pragma unroll
    for (int k = 0; k < F::kStages - 1; ++k) feed.template fetch<kDir>(k, k, k < count);

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
        float2 h_in = make_float2(0.0f, 0.0f);  // (gradient) the state that entered this run forward
        if (GRAD && OUTPUT) {
            if (on0) h_in.x = carry_at[c0];
            if (on1) h_in.y = carry_at[c1];
        }
        if (STAGED) {
            asm volatile("cp.async.wait_group %0;" ::"n"(F::kStages - 2) : "memory");
            __syncwarp();
        }
        const int pos = feed.ahead[0];
        Run<GRAD> w;
        w.cont = __ballot_sync(0xffffffffu, pos > 0) & ((1u << kRows) - 1);
        w.valid = __ballot_sync(0xffffffffu, pos >= 0) & ((1u << kRows) - 1);
        const bool whole = w.cont == (1u << kRows) - 1;  // (uniform) a stretch without a break, the usual case in long sequences

        float fA[2] = {1.0f, 1.0f}, H[2] = {0.0f, 0.0f}, E[2] = {0.0f, 0.0f};
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const float2 g = feed.get(stage, 0, r), v = feed.get(stage, 1, r);
            const float2 d = kTensors == 3 ? feed.get(stage, kTensors - 1, r) : v;
            const bool on = (w.cont >> r) & 1, is = (w.valid >> r) & 1;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float f, keep;
                gate_of(k ? g.y : g.x, f, keep);
                float x = k ? v.y : v.x, dh = k ? d.y : d.x;
                if (!whole && !is) f = keep = x = dh = 0.0f;
                w.f[r][k] = f;
                if (GRAD) {
                    w.keep[GRAD ? r : 0][k] = keep;
                    w.dh[GRAD ? r : 0][k] = dh;
                    w.x[r][k] = x;
                } else {
                    w.x[r][k] = keep * x;
                }
                if (!GRAD || OUTPUT) {
                    const float add = GRAD ? keep * x : w.x[r][k];
                    H[k] = whole || on ? fmaf(f, H[k], add) : add;
                }
                fA[k] *= f;
            }
        }
        if (!whole) fA[0] = fA[1] = kShut;
        const int buffer = i & 1;
        if (GRAD) {
#pragma unroll
            for (int r = kRows - 1; r >= 0; --r)
#pragma unroll
                for (int k = 0; k < 2; ++k) E[k] = whole || (w.cont >> r) & 1 ? w.f[r][k] * (w.dh[GRAD ? r : 0][k] + E[k]) : 0.0f;
            sums[buffer][GRAD ? 1 : 0][warp][lane] = make_float4(fA[0], E[0], fA[1], E[1]);
        }
        if (!GRAD || OUTPUT) sums[buffer][0][warp][lane] = make_float4(fA[0], H[0], fA[1], H[1]);
        // the next run to fetch takes the stage of the run before this one (in registers: this one's)
        __syncwarp();
#pragma unroll
        for (int k = 0; k + 1 < F::kStages - 1; ++k) feed.ahead[k] = feed.ahead[k + 1];
        feed.template fetch<kDir>(stage == 0 ? F::kStages - 1 : stage - 1, F::kStages - 2, i + F::kStages - 1 < count);
        stage = stage + 1 == F::kStages ? 0 : stage + 1;
        __syncthreads();

        if (OUTPUT && !GRAD && carry_at && warp == 0) {
            if (on0) carry_at[c0] = state.x;
            if (on1) carry_at[c1] = state.y;
        }
        float2 in = state, mine = state;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) {
            const int n = GRAD ? kWarps - 1 - k : k;
            const float4 s = sums[buffer][GRAD ? 1 : 0][n][lane];
            if (n == warp) mine = in;
            in.x = through(s.x, in.x, s.y);
            in.y = through(s.z, in.y, s.w);
            if (!OUTPUT) {
                A.x = both(A.x, s.x);
                A.y = both(A.y, s.z);
            }
        }
        state = in;
        if (!OUTPUT) continue;

        auto put = [&](T* at, float v0, float v1) {
            if (STAGED && on1) {
                *reinterpret_cast<typename Pair<T>::type*>(at) = Pair<T>::put(v0, v1);
            } else {
                if (on0) at[0] = from_float<T>(v0);
                if (on1) at[STAGED ? 1 : 32] = from_float<T>(v1);
            }
        };
        if (!GRAD) {
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const bool on = whole || (w.cont >> r) & 1;
                mine.x = on ? fmaf(w.f[r][0], mine.x, w.x[r][0]) : w.x[r][0];
                mine.y = on ? fmaf(w.f[r][1], mine.y, w.x[r][1]) : w.x[r][1];
                if (s_warp + r < p.t) put(out0 + r * a.h.slot, mine.x, mine.y);
            }
            out0 += kRun * a.h.slot;
            if (carry_at) carry_at += p.channels;
        } else {
            for (int k = 0; k < warp; ++k) {
                const float4 s = sums[buffer][0][k][lane];
                h_in.x = through(s.x, h_in.x, s.y);
                h_in.y = through(s.z, h_in.y, s.w);
            }
            float h[2] = {h_in.x, h_in.y};  // h in front of every slot, less x
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float before = whole || (w.cont >> r) & 1 ? h[k] : 0.0f;
                    h[k] = fmaf(w.f[r][k], before, w.keep[GRAD ? r : 0][k] * w.x[r][k]);
                    w.x[r][k] = before - w.x[r][k];
                }
            float e[2] = {mine.x, mine.y};  // then g from the last slot to the first
#pragma unroll
            for (int r = kRows - 1; r >= 0; --r) {
                float dg[2], dx[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float g = whole || (w.valid >> r) & 1 ? w.dh[GRAD ? r : 0][k] + e[k] : 0.0f;
                    dx[k] = w.keep[GRAD ? r : 0][k] * g;
                    dg[k] = dx[k] * w.f[r][k] * w.x[r][k];
                    e[k] = whole || (w.cont >> r) & 1 ? w.f[r][k] * g : 0.0f;
                }
                if (s_warp + r < p.t) {
                    put(out0 + r * a.dgate.slot, dg[0], dg[1]);
                    put(out1 + r * a.dx.slot, dx[0], dx[1]);
                }
            }
            out0 -= kRun * a.dgate.slot;
            out1 -= kRun * a.dx.slot;
            carry_at -= p.channels;
        }
    }
    if (STAGED) asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();  // the ring and the sums may be used again
}

template <typename T, bool GRAD, bool STAGED>
__global__ void __launch_bounds__(256, GRAD || !STAGED ? 2 : 3)
    k27_recurrence(const RecurParams p, const RecurTensors<T> a, int groups_per_block, int segments)
{
    extern __shared__ __align__(16) uint8_t ring[];  // [stages][8 warps][tensors][8 rows][64]
    __shared__ float4 sums[2][GRAD ? 2 : 1][kWarps][32];
    __shared__ float2 entering[32];
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
    float2 state = make_float2(0.0f, 0.0f), A = make_float2(1.0f, 1.0f);
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
            walk<T, GRAD, STAGED, false>(p, a, q, ch0, from, count, ring, sums, state, A);
        }
        if (threadIdx.x < 32) {
            const float2 own = state;
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
            entering[lane] = e;
        }
        __syncthreads();
        state = entering[lane];
    }
    walk<T, GRAD, STAGED, true>(p, a, q, ch0, GRAD ? end - 1 : first, end - first, ring, sums, state, A);
}

int64_t groups_of(int64_t blocks, int64_t channels) { return blocks * ((channels + kCh - 1) / kCh); }

// Segments per walk: as many as keep two CTAs on each of the 148 SMs busy, of at least 4 runs each.
int segments_of(int64_t blocks, int32_t t, int64_t channels)
{
    const int64_t runs = (t + kRun - 1) / kRun, groups = groups_of(blocks, channels);
    const int64_t wanted = groups >= 200 ? 1 : (2 * 148) / groups, most = runs / 4;
    return (int)(wanted < most ? (wanted < 1 ? 1 : wanted) : (most < 1 ? 1 : most));
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
    static const cudaError_t set = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared);
    if (set != cudaSuccess) return set;
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

}  // namespace

size_t recurrence_work_bytes(int64_t blocks, int32_t t, int64_t channels)
{
    const int segments = segments_of(blocks, t, channels);
    return segments > 1 ? work_view(groups_of(blocks, channels) * segments, nullptr, nullptr) : 0;
}

template <typename T>
cudaError_t launch_recurrence(const RecurParams& p, const RecurTensors<T>& a, cudaStream_t st)
{
    return on_16(a.gate) && on_16(a.x) && on_16(a.h) ? launch<T, false, true>(p, a, st) : launch<T, false, false>(p, a, st);
}
template <typename T>
cudaError_t launch_recurrence_grad(const RecurParams& p, const RecurTensors<T>& a, cudaStream_t st)
{
    return on_16(a.gate) && on_16(a.x) && on_16(a.dh) && on_16(a.dgate) && on_16(a.dx) ? launch<T, true, true>(p, a, st)
                                                                                  : launch<T, true, false>(p, a, st);
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

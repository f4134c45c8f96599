// k27_recurrence: gated linear recurrence along the slots of packed blocks, restarted at every sequence start,
//     f = sigmoid(gate);  h = f h_prev + (1 - f) x
// and its gradient, each in one pass over the data.  The work is bytes only: three tensors move forward, five backward.
//
// A run of 64 slots by 64 channels is a tile: 8 warps own 8 slots each, a lane 2 channels.  h_out = A h_in + H over any stretch
// of slots, and stretches compose, so a warp reduces its slots to (A, H), the warps combine theirs through shared memory, and
// a tile needs only the state that enters it.  That state comes from the tiles before it by looking back: a tile publishes
// (A, H) as soon as it has them, and the state behind it as soon as it has that; its successor reads back over published (A, H)
// to the nearest published state.  Positions tell where nothing is needed: no tile looks back that starts with a sequence
// start or padding, none publishes whose successor does, and a tile with a start inside publishes at once.  A position p > 0
// in slot s also says that slot s - p starts the sequence, so every look back ends.
//
// Tiles are taken by ticket, in order of time, so those that a tile waits for were taken before it by CTAs that run or have
// ended; within a CTA tickets are processed in order.  So the earliest unfinished tile never waits, whatever the scheduling.
//
// The gradient walks the time backwards: E = f g (0 where a sequence starts) is what a slot hands to the one before it, and
// E_out = A E_in + E over a stretch.  It rebuilds h from the states the forward call kept at the start of each run.
#include "bload_internal.cuh"
#include "bload_layers.cuh"

namespace bload {

namespace {

constexpr int kRun = BLOAD_RECURRENCE_RUN;
constexpr int kWarps = 8, kRows = kRun / kWarps, kCh = 64;

__device__ unsigned int g_timeouts;  // bounded waits that gave up (bload_device_timeouts)

// Scratch: a ticket, then per tile (group-major within a step of time) a flag, (A, H) and the state.
struct WorkView2 {
    unsigned int* ticket;
    unsigned int* flags;  // 0 nothing, 1 (A, H), 2 the state behind the tile as well
    float4* sums;         // [tiles][32]: A, H of a lane's two channels
    float2* states;       // [tiles][32]
};
__host__ __device__ inline size_t work_view(int64_t tiles, void* base, WorkView2* v)
{
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t flags = 256, sums = flags + up(4 * (size_t)tiles), states = sums + 512 * (size_t)tiles;
    if (v) {
        char* b = static_cast<char*>(base);
        v->ticket = reinterpret_cast<unsigned int*>(b);
        v->flags = reinterpret_cast<unsigned int*>(b + flags);
        v->sums = reinterpret_cast<float4*>(b + sums);
        v->states = reinterpret_cast<float2*>(b + states);
    }
    return states + 256 * (size_t)tiles;
}

// f = sigmoid(g) and 1 - f, each with a small relative error of its own (1 - f must not cancel: it scales the input)
__device__ __forceinline__ void gate_of(float g, float& f, float& keep)
{
    float e, big;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-1.4426950408889634f * fabsf(g)));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(big) : "f"(1.0f + e));
    const float small = e * big;
    f = g >= 0.0f ? big : small;
    keep = g >= 0.0f ? small : big;
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

// The state that enters a tile, for this lane's two channels, by a whole warp: finds the nearest tile before it whose state
// is published, with (A, H) of all between published too, and applies those in the order of the walk.  That is the same chain
// of multiply-adds wherever the state was found, so results do not depend on timing.  Gives up after four seconds, which
// nothing but a hardware failure takes.
__device__ float2 look_back(const WorkView2& w, int64_t tile, int64_t step, int lane)
{
    uint64_t since = 0;
    int64_t far = 1;  // how many tiles back the lanes begin to look
    for (;;) {
        const int64_t mine = tile - (far + lane) * step;
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
    float2 e = __ldcg(w.states + (tile - far * step) * 32 + lane);
    for (int64_t k = far - 1; k > 0; k -= 8) {  // eight loads at a time
        float4 s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = k > j ? __ldcg(w.sums + (tile - (k - j) * step) * 32 + lane) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
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

// STAGED: rows on 16-byte boundaries; tiles are copied to shared memory asynchronously, one ahead, lane l has channels 2l and
// 2l + 1.  Otherwise elements are loaded one by one, lane l has channels l and l + 32.
template <typename T, bool GRAD, bool STAGED>
__global__ void __launch_bounds__(256, GRAD ? 2 : 3) k27_recurrence(const RecurParams p, const RecurTensors<T> a, int64_t tiles, int groups_per_block)
{
    constexpr int kTensors = GRAD ? 3 : 2;
    constexpr int kRowBytes = kCh * sizeof(T), kTensorBytes = kRows * kRowBytes;  // of a warp
    extern __shared__ __align__(16) uint8_t staged[];  // [2 stages][8 warps][tensors][8 rows][64]
    __shared__ float4 sums[2][GRAD ? 2 : 1][kWarps][32];
    __shared__ float2 entering[2][32];
    __shared__ int64_t tickets[2];

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int runs = (p.t + kRun - 1) / kRun;
    const int64_t groups = p.blocks * groups_per_block;
    WorkView2 work;
    work_view(tiles, p.work, &work);
    const bool by_ticket = runs > 1;

    // where a tile is
    int64_t q = 0, ch0 = 0;
    int run = 0, s0 = 0;
    auto place = [&](int64_t tile) {
        const int64_t step = tile / groups, g = tile - step * groups;
        run = (int)(GRAD ? runs - 1 - step : step);
        q = g / groups_per_block;
        ch0 = (g - q * groups_per_block) * kCh;
        s0 = run * kRun;
    };
    // positions of the warp's rows (lanes 0 to 7), the tile's first slot (9), the slot behind the tile (10), its last (11)
    auto positions = [&]() {
        const int s = lane < 9 ? s0 + warp * kRows + lane : lane == 9 ? s0 : lane == 10 ? s0 + kRun : s0 + kRun - 1;
        return s < p.t && lane < 12 ? p.pos[q * p.t + s] : -1;
    };
    auto copy_in = [&](int stage) {
        uint8_t* const to = staged + (stage * kWarps + warp) * kTensors * kTensorBytes;
        constexpr int kPieces = kRowBytes / 16;
#pragma unroll
        for (int n = 0; n < kTensors; ++n) {
            const Channels<const T>& x = n == 0 ? a.gate : n == 1 ? a.x : a.dh;
#pragma unroll
            for (int k = lane; k < kRows * kPieces; k += 32) {
                const int r = k / kPieces, piece = k % kPieces;
                const int s = s0 + warp * kRows + r;
                const int64_t c = ch0 + piece * (16 / (int)sizeof(T));
                const int64_t left = s < p.t ? (p.channels - c) * (int64_t)sizeof(T) : 0;
                const int bytes = left <= 0 ? 0 : left < 16 ? (int)left : 16;
                copy16(to + n * kTensorBytes + r * kRowBytes + piece * 16, bytes ? x.at(q, s) + c : x.data, bytes);
            }
        }
    };

    int64_t tile, next, after = 0;
    if (by_ticket) {
        if (tid == 0) {
            tickets[0] = atomicAdd(work.ticket, 1u);
            tickets[1] = atomicAdd(work.ticket, 1u);
        }
        __syncthreads();
        tile = tickets[0];
        next = tickets[1];
        __syncthreads();
    } else {
        tile = blockIdx.x;
        next = tile + gridDim.x;
    }
    int pos_next = -1;
    if (tile < tiles) {
        place(tile);
        pos_next = positions();
        if (STAGED) copy_in(0);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");

    for (int turn = 0; tile < tiles; ++turn) {
        place(tile);
        const int pos = pos_next;
        const int64_t q_here = q, ch_here = ch0;
        const int run_here = run, s_here = s0;
        const int buffer = turn & 1;
        if (by_ticket && tid == 0) after = atomicAdd(work.ticket, 1u);  // two tiles ahead: its latency is hidden
        if (next < tiles) {
            place(next);
            pos_next = positions();
            if (STAGED) copy_in(buffer ^ 1);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");

        const unsigned cont = __ballot_sync(0xffffffffu, pos > 0), valid = __ballot_sync(0xffffffffu, pos >= 0);
        const int last_pos = __shfl_sync(0xffffffffu, pos, 11);
        const bool left = run_here > 0 && (cont >> 9) & 1, right = (cont >> 10) & 1;  // a sequence crosses that edge
        const bool closed = last_pos < kRun;                                         // one starts inside (or padding): nothing passes through
        const bool need = GRAD ? right : left, give = GRAD ? left : right;
        const int64_t c0 = ch_here + (STAGED ? 2 * lane : lane), c1 = STAGED ? c0 + 1 : c0 + 32;

        float f[kRows][2], keep[GRAD ? kRows : 1][2], x[kRows][2], dh[GRAD ? kRows : 1][2];
        float2 carry = make_float2(0.0f, 0.0f);
        if (GRAD && left) {
            const float* at = p.carry + (q_here * runs + run_here) * p.channels;
            if (c0 < p.channels) carry.x = at[c0];
            if (c1 < p.channels) carry.y = at[c1];
        }
        if (STAGED) {
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            __syncwarp();
        }
        // gates and inputs (forward: x is (1 - f) x); zeros on padding
        {
            const uint8_t* const from = staged + (buffer * kWarps + warp) * kTensors * kTensorBytes;
            float raw[kTensors][kRows][2];
#pragma unroll
            for (int n = 0; n < kTensors; ++n) {
                const Channels<const T>& src = n == 0 ? a.gate : n == 1 ? a.x : a.dh;
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    if (STAGED) {
                        const float2 v = Pair<T>::get(reinterpret_cast<const typename Pair<T>::type*>(from + n * kTensorBytes + r * kRowBytes)[lane]);
                        raw[n][r][0] = v.x;
                        raw[n][r][1] = v.y;
                    } else {
                        const int s = s_here + warp * kRows + r;
                        const T* at = s < p.t ? src.at(q_here, s) : nullptr;
                        raw[n][r][0] = at && c0 < p.channels ? to_float(at[c0]) : 0.0f;
                        raw[n][r][1] = at && c1 < p.channels ? to_float(at[c1]) : 0.0f;
                    }
                }
            }
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float kp;
                    gate_of(raw[0][r][k], f[r][k], kp);
                    const bool is = (valid >> r) & 1;
                    if (GRAD) {
                        keep[r][k] = is ? kp : 0.0f;
                        f[r][k] = is ? f[r][k] : 0.0f;
                        x[r][k] = is ? raw[1][r][k] : 0.0f;
                        dh[r][k] = is ? raw[kTensors - 1][r][k] : 0.0f;
                    } else {
                        x[r][k] = is ? kp * raw[1][r][k] : 0.0f;
                    }
                }
        }
        // the warp's slots as one step, forward and (gradient) backward
        {
            float A[2] = {1.0f, 1.0f}, H[2] = {0.0f, 0.0f}, E[2] = {0.0f, 0.0f};
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float add = GRAD ? keep[r][k] * x[r][k] : x[r][k];
                    H[k] = (cont >> r) & 1 ? fmaf(f[r][k], H[k], add) : add;
                    A[k] *= f[r][k];
                }
            if (~cont & ((1u << kRows) - 1)) A[0] = A[1] = kShut;
            sums[buffer][0][warp][lane] = make_float4(A[0], H[0], A[1], H[1]);
            if (GRAD) {
#pragma unroll
                for (int r = kRows - 1; r >= 0; --r)
#pragma unroll
                    for (int k = 0; k < 2; ++k) E[k] = (cont >> r) & 1 ? f[r][k] * (dh[r][k] + E[k]) : 0.0f;
                sums[buffer][GRAD ? 1 : 0][warp][lane] = make_float4(A[0], E[0], A[1], E[1]);
            }
        }
        if (by_ticket && tid == 0) tickets[buffer] = after;
        __syncthreads();
        if (by_ticket) after = tickets[buffer];

        // the stretch between the tile's edge and this warp, and (last warp of the walk) the whole tile
        float2 in = make_float2(0.0f, 0.0f);
        float a0 = 1.0f, a1 = 1.0f;
        {
            const int first = GRAD ? kWarps - 1 : 0, dir = GRAD ? -1 : 1;
            const int steps = GRAD ? kWarps - 1 - warp : warp;
            for (int k = 0; k < steps; ++k) {
                const float4 s = sums[buffer][GRAD ? 1 : 0][first + dir * k][lane];
                in.x = through(s.x, in.x, s.y);
                in.y = through(s.z, in.y, s.w);
                a0 = both(a0, s.x);
                a1 = both(a1, s.z);
            }
        }
        if (warp == (GRAD ? 0 : kWarps - 1) && (need || give || (!GRAD && p.carry))) {
            const float4 s = sums[buffer][GRAD ? 1 : 0][warp][lane];
            const float A0 = both(a0, s.x), A1 = both(a1, s.z), H0 = through(s.x, in.x, s.y), H1 = through(s.z, in.y, s.w);
            float2 e = make_float2(0.0f, 0.0f);
            if (give && (!need || closed)) {
                work.states[tile * 32 + lane] = make_float2(H0, H1);
                set_flag(work.flags + tile, 2, lane);
            }
            if (need) {
                const bool open = give && !closed;
                if (open && !__all_sync(0xffffffffu, flag_of(work.flags + tile - groups) == 2)) {
                    work.sums[tile * 32 + lane] = make_float4(A0, H0, A1, H1);
                    set_flag(work.flags + tile, 1, lane);
                }
                e = look_back(work, tile, groups, lane);
                if (open) {
                    work.states[tile * 32 + lane] = make_float2(fmaf(A0, e.x, H0), fmaf(A1, e.y, H1));
                    set_flag(work.flags + tile, 2, lane);
                }
                entering[buffer][lane] = e;
            }
            if (!GRAD && p.carry) {
                float* at = p.carry + (q_here * runs + run_here) * p.channels;
                if (c0 < p.channels) at[c0] = e.x;
                if (c1 < p.channels) at[c1] = e.y;
            }
        }
        if (need) {
            __syncthreads();
            const float2 e = entering[buffer][lane];
            in.x = through(a0, e.x, in.x);
            in.y = through(a1, e.y, in.y);
        }

        auto put = [&](const Channels<T>& to, int r, float v0, float v1) {
            const int s = s_here + warp * kRows + r;
            if (s >= p.t) return;
            T* at = to.at(q_here, s);
            if (STAGED && c1 < p.channels) {
                *reinterpret_cast<typename Pair<T>::type*>(at + c0) = Pair<T>::put(v0, v1);
            } else {
                if (c0 < p.channels) at[c0] = from_float<T>(v0);
                if (c1 < p.channels) at[c1] = from_float<T>(v1);
            }
        };
        if (!GRAD) {
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const bool on = (cont >> r) & 1;
                in.x = on ? fmaf(f[r][0], in.x, x[r][0]) : x[r][0];
                in.y = on ? fmaf(f[r][1], in.y, x[r][1]) : x[r][1];
                put(a.h, r, in.x, in.y);
            }
        } else {
            // h in front of every slot, less x; then g from the last slot to the first
            for (int k = 0; k < warp; ++k) {
                const float4 s = sums[buffer][0][k][lane];
                carry.x = through(s.x, carry.x, s.y);
                carry.y = through(s.z, carry.y, s.w);
            }
            float h[2] = {carry.x, carry.y};
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float before = (cont >> r) & 1 ? h[k] : 0.0f;
                    h[k] = fmaf(f[r][k], before, keep[r][k] * x[r][k]);
                    x[r][k] = before - x[r][k];
                }
            float e[2] = {in.x, in.y};
#pragma unroll
            for (int r = kRows - 1; r >= 0; --r) {
                float dg[2], dx[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float g = (valid >> r) & 1 ? dh[r][k] + e[k] : 0.0f;
                    dx[k] = keep[r][k] * g;
                    dg[k] = dx[k] * f[r][k] * x[r][k];
                    e[k] = (cont >> r) & 1 ? f[r][k] * g : 0.0f;
                }
                put(a.dgate, r, dg[0], dg[1]);
                put(a.dx, r, dx[0], dx[1]);
            }
        }
        tile = next;
        next = by_ticket ? after : next + gridDim.x;
    }
}

int64_t tiles_of(int64_t blocks, int64_t t, int64_t channels)
{
    return blocks * ((channels + kCh - 1) / kCh) * ((t + kRun - 1) / kRun);
}

template <typename T, bool GRAD, bool STAGED>
cudaError_t launch(const RecurParams& p, const RecurTensors<T>& a, cudaStream_t st)
{
    const int64_t tiles = tiles_of(p.blocks, p.t, p.channels);
    const int shared = STAGED ? 2 * kRun * kCh * (int)sizeof(T) * (GRAD ? 3 : 2) : 0;
    auto* kernel = k27_recurrence<T, GRAD, STAGED>;
    struct Fit {
        cudaError_t error;
        int ctas;
    };
    static const Fit fit = [&] {
        Fit f{cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, shared), 0};
        int device = 0, sms = 0, per = 0;
        if (f.error == cudaSuccess) f.error = cudaGetDevice(&device);
        if (f.error == cudaSuccess) f.error = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
        if (f.error == cudaSuccess) f.error = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, 256, shared);
        f.ctas = sms * per;
        return f;
    }();
    if (fit.error != cudaSuccess) return fit.error;
    if (p.t > kRun) {  // ticket and flags
        const cudaError_t e = cudaMemsetAsync(p.work, 0, 256 + 4 * (size_t)tiles, st);
        if (e != cudaSuccess) return e;
    }
    kernel<<<(unsigned)(tiles < fit.ctas ? tiles : fit.ctas), 256, shared, st>>>(p, a, tiles, (int)((p.channels + kCh - 1) / kCh));
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
    return t > kRun ? work_view(tiles_of(blocks, t, channels), nullptr, nullptr) : 0;
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

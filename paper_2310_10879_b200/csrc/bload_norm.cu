// k31_norm: layer norm over the channels of every frame of a packed batch; k32_norm_grad: its gradient; k33_column_sums: sums of
// partial sums, for the gradients of weights.
//
// Bytes only: x in, y out; x and dy in, dx out -- as long as there are few instructions to an element (10 of them take as long as the
// bytes of a 16-bit element, forward).  So a team of threads has a frame, with as many channels to a thread as its registers hold: up
// to 2,048 channels that is one warp forward (64 each), whose sums need no barrier.  x stays in registers as 32-bit numbers: first the
// mean, then the squares around it (in one pass their difference would lose what a large mean has in common), then y.  In the gradient a
// thread has the same 16 channels of every frame, and their sums over frames stay in its registers until the CTA has done its last
// frame; each CTA then writes them once, and k33 adds the CTAs' in their order.  x and dy are read from shared memory twice, before and
// behind the sums over channels.
// 16 x 4096 x 2048 bf16: 105 us forward (5.1 TB/s), 162 gradient (5.0 TB/s); rows off 16-byte boundaries, 4 x 5003 x 1027 fp32: 53 us (3.1
// TB/s) and 73 (3.4 TB/s).
#include <type_traits>

#include "bload_internal.cuh"
#include "bload_layers.cuh"

namespace bload {

namespace {

constexpr int kMaxShared = 216 * 1024;

// Frame `row` of a tensor; rows of blocks that lie one behind the other (p.flat) need no division.
template <typename C>
__device__ __forceinline__ auto frame(const NormParams& p, const C& x, int64_t row)
{
    if (p.flat) return x.data + row * x.slot;
    const int64_t q = row / p.t;
    return x.at(q, row - q * p.t);
}

// 1 / sqrt(v): the approximation and one Newton step
__device__ __forceinline__ float inverse_root(float v)
{
    float r;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return v > 1e-37f && r > 0.0f ? r * fmaf(-0.5f * v * r, r, 1.5f) : 1.0f / sqrtf(v);
}

// Who has a frame: a warp (ONE; kTeams of them in a CTA), or all warps of the CTA.
template <bool ONE>
struct Team {
    static constexpr int kTeams = ONE ? 4 : 1;
    int lane, warp, warps, rank, size;  // warps: of the team; rank, size: of the thread in the team
    __device__ __forceinline__ Team()
    {
        lane = threadIdx.x & 31;
        warp = threadIdx.x >> 5;
        warps = ONE ? 1 : blockDim.x >> 5;
        rank = ONE ? lane : threadIdx.x;
        size = ONE ? 32 : blockDim.x;
    }
    __device__ __forceinline__ void sync() const
    {
        if (ONE)
            __syncwarp();
        else
            __syncthreads();
    }
    // sums over the team of N values each; `red`: [warps][N], the caller alternates between two of them
    template <int N>
    __device__ __forceinline__ void sums(float (&v)[N], float* red) const
    {
        if (ONE) {
#pragma unroll
            for (int bit = 16; bit; bit /= 2)
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], bit);
            return;
        }
        int first = 0;
        float w[N];
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = v[i];
        share_sums<N, 16, 1>(w, lane, first);
        if (lane % (32 / N) == 0) red[warp * N + first] = w[0];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = 0.0f;
        for (int k = 0; k < warps; ++k) {
            Elements<float, N> sums;
            sums.load(red + k * N, N, true);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += sums.x[i];
        }
    }
};

// Brings groups of R frames to a team through shared memory, up to two groups under way while one is worked on.
// V > 1: rows on 16-byte boundaries; each thread copies its own P pieces (no barrier).  V == 1: rows on any boundary, of a tensor that
// itself begins on such a one; they are copied by the granules of 16 bytes that hold them (a granule at a row's edge has elements of
// its neighbours; behind the tensor's last element nothing is read), which takes a barrier of the team per group.  Where that does not
// fit (p.stages 0) elements are read from global memory each time.
// Padding is copied, too, and not used: whether a frame is padding is known only when its position has arrived.
template <typename T, int V, int P, int R, int TENSORS, bool ONE>
struct Feed {
    static constexpr int kStageBytes = R * TENSORS * P * 16;  // V > 1: of a thread
    const NormParams& p;
    const Team<ONE>& team;
    const Channels<const T>* tensors[TENSORS];
    uint8_t* ring;  // of the team, in shared memory
    static constexpr int step = 32 * V;  // channels c0 + j * step + 0 .. V - 1 are the thread's
    int c0, pitch, left, stage;          // left: channels from c0 on
    int64_t row0, stride;
    int pos;        // of the next group, frame `lane`
    float2 stat;    // and its mean and deviation
    bool stats;

    static __host__ __device__ int pitch_of(int64_t channels) { return (int)((channels * sizeof(T) + 15) / 16 * 16 + 16); }
    // bytes of a stage of a team
    static __host__ __device__ int stage_bytes(int64_t channels, int threads) { return V > 1 ? kStageBytes * threads : R * TENSORS * pitch_of(channels); }

    __device__ __forceinline__ Feed(const NormParams& params, const Team<ONE>& t, uint8_t* shared, bool with_stats) : p(params), team(t), stats(with_stats)
    {
        c0 = (ONE ? 0 : team.warp * 32 * V * P) + team.lane * V;
        left = (int)p.channels - c0;
        pitch = pitch_of(p.channels);
        const int mine = ONE ? team.warp : 0;
        ring = shared + mine * p.stages * stage_bytes(p.channels, team.size);
        row0 = ((int64_t)blockIdx.x * Team<ONE>::kTeams + mine) * R;
        stride = (int64_t)gridDim.x * Team<ONE>::kTeams * R;
        stage = 0;
    }
    __device__ __forceinline__ void look(int64_t row)
    {
        const bool on = team.lane < R && row + team.lane < p.rows;
        pos = on ? p.pos[row + team.lane] : -1;
        if (stats) stat = on && pos >= 0 ? p.stats[row + team.lane] : make_float2(0.0f, 0.0f);
    }
    __device__ __forceinline__ uint8_t* piece(int in, int r, int n) const  // the first; the others 512 bytes apart
    {
        return ring + (((in * R + r) * TENSORS + n) * P * team.size + (ONE ? 0 : team.warp * 32 * P) + team.lane) * 16;
    }
    __device__ __forceinline__ uint8_t* row_at(int in, int r, int n) const { return ring + ((in * R + r) * TENSORS + n) * pitch; }
    __device__ __forceinline__ void fetch(int64_t row, int to)
    {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (row + r >= p.rows) break;
#pragma unroll
            for (int n = 0; n < TENSORS; ++n) {
                const T* const from = frame(p, *tensors[n], row + r);
                if (V > 1) {
                    const uint32_t at = (uint32_t)__cvta_generic_to_shared(piece(to, r, n));
#pragma unroll
                    for (int j = 0; j < P; ++j)
                        if (j * step < left)
                            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + (uint32_t)(j * 512)), "l"(from + c0 + j * step)
                                         : "memory");
                } else {
                    const int shift = (int)(reinterpret_cast<uintptr_t>(from) & 15), bytes = shift + (int)(p.channels * sizeof(T));
                    const uint8_t* const at = reinterpret_cast<const uint8_t*>(from) - shift;
                    const int64_t there = p.end[n] - reinterpret_cast<uintptr_t>(at);  // bytes up to the tensor's end
                    const uint32_t to_row = (uint32_t)__cvta_generic_to_shared(row_at(to, r, n));
                    for (int k = team.rank * 16; k < bytes; k += team.size * 16)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to_row + (uint32_t)k), "l"(at + k),
                                     "r"((int)min(there - k, (int64_t)16))
                                     : "memory");
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ __forceinline__ void start()
    {
        look(row0);
        if (V == 1 && !p.stages) return;
        for (int k = 0; k < p.stages; ++k) fetch(row0 + k * stride, k);
    }
    // the group of row0 is there; returns which of its frames are frames, and looks at the next ones' positions
    __device__ __forceinline__ unsigned arrive(bool first, float2 (&st)[R])
    {
        if (V > 1) {
            if (p.stages == 3)
                asm volatile("cp.async.wait_group 2;" ::: "memory");
            else if (p.stages == 2)
                asm volatile("cp.async.wait_group 1;" ::: "memory");
            else
                asm volatile("cp.async.wait_group 0;" ::: "memory");
        } else if (p.stages) {
            if (p.stages == 3)
                asm volatile("cp.async.wait_group 1;" ::: "memory");
            else
                asm volatile("cp.async.wait_group 0;" ::: "memory");
            team.sync();  // and all are done with the group before this one
            if (first)
                asm volatile("cp.async.commit_group;" ::: "memory");
            else
                fetch(row0 + (p.stages - 1) * stride, stage ? stage - 1 : p.stages - 1);
        }
        const unsigned live = __ballot_sync(0xffffffffu, pos >= 0);
        if (stats)
#pragma unroll
            for (int r = 0; r < R; ++r) st[r] = make_float2(__shfl_sync(0xffffffffu, stat.x, r), __shfl_sync(0xffffffffu, stat.y, r));
        look(row0 + stride);
        return live;
    }
    __device__ __forceinline__ void leave()
    {
        if (V > 1) fetch(row0 + p.stages * stride, stage);
        stage = stage + 1 >= p.stages ? 0 : stage + 1;
        row0 += stride;
    }
    __device__ __forceinline__ void finish() const { asm volatile("cp.async.wait_group 0;" ::: "memory"); }
    // this thread's channels of a frame as 32-bit numbers, in pairs; 0 where there is none
    __device__ __forceinline__ void take(int r, int n, Two (&x)[V * P / 2]) const
    {
        if constexpr (V > 1) {
            const uint4* const at = reinterpret_cast<const uint4*>(piece(stage, r, n));
#pragma unroll
            for (int j = 0; j < P; ++j) {
                Elements<T, V> e;
                *reinterpret_cast<uint4*>(e.x) = j * step < left ? at[j * 32] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int k = 0; k < V; k += 2) x[(j * V + k) / 2] = e.pair(k);
            }
        } else {
            const T* const from = frame(p, *tensors[n], row0 + r);
            auto read = [&](const T* row) {
#pragma unroll
                for (int k = 0; k < P; k += 2)
                    x[k / 2] = two(k * step < left ? to_float(row[k * step]) : 0.0f, (k + 1) * step < left ? to_float(row[(k + 1) * step]) : 0.0f);
            };
            if (p.stages)
                read(reinterpret_cast<const T*>(row_at(stage, r, n) + (reinterpret_cast<uintptr_t>(from) & 15)) + c0);
            else
                read(from + c0);
        }
    }
    // writes this thread's channels of a frame; value(k): those of pair k
    template <typename Value>
    __device__ __forceinline__ void put(T* to, const Value& value) const
    {
        if constexpr (V > 1) {
#pragma unroll
            for (int j = 0; j < P; ++j) {
                if (j * step >= left) break;
                Elements<T, V> e;
#pragma unroll
                for (int k = 0; k < V; k += 2) e.set_pair(k, value((j * V + k) / 2));
                e.store(to + c0 + j * step, V, true);
            }
        } else {
#pragma unroll
            for (int k = 0; k < P / 2; ++k) {
                if (2 * k * step >= left) break;
                const float2 v = one(value(k));
                to[c0 + 2 * k * step] = from_float<T>(v.x);
                if ((2 * k + 1) * step < left) to[c0 + (2 * k + 1) * step] = from_float<T>(v.y);
            }
        }
    }
};

// A weight's values for pair k of a thread's channels
template <int V>
__device__ __forceinline__ Two weight_of(const float* from, float otherwise, int k, int c0, int left)
{
    constexpr int step = 32 * V;
    if (!from) return two(otherwise, otherwise);
    if constexpr (V > 1) {
        const int c = 2 * k / V * step;
        if (c >= left) return two(otherwise, otherwise);
        const float* const at = from + c0 + c + 2 * k % V;
        if (reinterpret_cast<uintptr_t>(from) % 8) return two(at[0], at[1]);
        const float2 v = *reinterpret_cast<const float2*>(at);
        return two(v.x, v.y);
    } else {
        const int c = 2 * k * step;
        return two(c < left ? from[c0 + c] : otherwise, c + step < left ? from[c0 + c + step] : otherwise);
    }
}

template <typename T, int V, int P, bool ONE>
__global__ void __launch_bounds__(ONE ? 128 : 256) k31_norm(const NormParams p, const NormTensors<T> a)
{
    constexpr int K = V * P / 2;
    extern __shared__ __align__(16) uint8_t shared_bytes[];
    __shared__ __align__(16) float red[2][16];
    const Team<ONE> team;
    const float inv = 1.0f / (float)p.channels;
    Feed<T, V, P, 1, 1, ONE> feed(p, team, shared_bytes, false);
    feed.tensors[0] = &a.x;
    // weight and bias as pairs, where a thread finds its own side by side with its neighbours'
    constexpr int kVector = V > 1 ? 2 : 1;  // pairs that are read together
    Two* const params = reinterpret_cast<Two*>(shared_bytes + p.params_at);
    const int mine = (ONE ? 0 : team.warp * 32 * K) + team.lane * kVector;
    if (!ONE || team.warp == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int at = mine + k / kVector * 32 * kVector + k % kVector;
            params[at] = weight_of<V>(p.weight, 1.0f, k, feed.c0, feed.left);
            params[team.size * K + at] = weight_of<V>(p.bias, 0.0f, k, feed.c0, feed.left);
        }
    }
    if (ONE) __syncthreads();
    auto param = [&](int which, int k) {
        const Two* const at = params + which * team.size * K + mine + k / kVector * 32 * kVector;
        if constexpr (kVector == 2) {
            const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(at);
            return Two{k % 2 ? v.y : v.x};
        } else {
            return at[0];
        }
    };
    feed.start();
    for (bool first = true; feed.row0 < p.rows; first = false) {
        float2 none[1];
        const bool live = feed.arrive(first, none) & 1;
        Two x[K];
        float mean[1] = {0.0f}, square[1] = {0.0f};
        if (live) {  // (all of the team)
            feed.take(0, 0, x);
            Two sum[2] = {zero(), zero()};
#pragma unroll
            for (int k = 0; k < K; ++k) sum[k & 1] = sum[k & 1] + x[k];
            mean[0] = one(sum[0] + sum[1]).x + one(sum[0] + sum[1]).y;
            team.template sums<1>(mean, red[0]);
            mean[0] *= inv;
            const Two minus = two(-mean[0], -mean[0]);
            sum[0] = sum[1] = zero();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                x[k] = x[k] + minus;
                if (V > 1 ? 2 * k / V * feed.step < feed.left : (2 * k + 1) * feed.step < feed.left) {
                    sum[k & 1] = fma(x[k], x[k], sum[k & 1]);
                } else if (V == 1 && 2 * k * feed.step < feed.left) {
                    sum[k & 1] = fma(two(one(x[k]).x, 0.0f), two(one(x[k]).x, 0.0f), sum[k & 1]);
                }
            }
            square[0] = one(sum[0] + sum[1]).x + one(sum[0] + sum[1]).y;
            team.template sums<1>(square, red[1]);
            square[0] = inverse_root(fmaf(square[0], inv, p.eps));
            const Two scale = two(square[0], square[0]);
            feed.put(frame(p, a.y, feed.row0), [&](int k) {
                return fma(x[k] * scale, param(0, k), param(1, k));
            });
        } else {
            feed.put(frame(p, a.y, feed.row0), [](int) { return zero(); });
        }
        if (p.stats && team.rank == 0) p.stats[feed.row0] = make_float2(mean[0], square[0]);
        feed.leave();
    }
    feed.finish();
}

// ROWS: frames at once
template <typename T, int V, int P, int ROWS, bool ONE>
__global__ void __launch_bounds__(ONE ? 128 : 512, ONE ? 4 : 1) k32_norm_grad(const NormParams p, const NormTensors<T> a)
{
    constexpr int R = ROWS, K = V * P / 2;
    extern __shared__ __align__(16) uint8_t shared_bytes[];
    __shared__ __align__(16) float red[2][16 * 2 * R];
    const Team<ONE> team;
    const int channels = (int)p.channels;
    const float inv = 1.0f / (float)channels;
    Feed<T, V, P, R, 2, ONE> feed(p, team, shared_bytes, true);
    feed.tensors[0] = &a.x;
    feed.tensors[1] = &a.dy;
    constexpr int step = decltype(feed)::step;
    const int c0 = feed.c0, left = feed.left;
    Two w[K], dw[K], db[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        w[k] = weight_of<V>(p.weight, 1.0f, k, c0, left);
        dw[k] = db[k] = zero();
    }
    feed.start();
    int turn = 0;
    for (bool first = true; feed.row0 < p.rows; first = false) {
        float2 st[R];
        const unsigned live = feed.arrive(first, st);
        float sums[2 * R];  // of g, of g n
#pragma unroll
        for (int r = 0; r < R; ++r) {
            Two of_g = zero(), of_gn = zero();
            if ((live >> r) & 1) {
                Two x[K], dy[K];
                feed.take(r, 0, x);
                feed.take(r, 1, dy);
                const Two minus = two(-st[r].x, -st[r].x), scale = two(st[r].y, st[r].y);
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const Two n = (x[k] + minus) * scale, g = dy[k] * w[k];
                    of_g = of_g + g;
                    of_gn = fma(g, n, of_gn);
                    dw[k] = fma(dy[k], n, dw[k]);
                    db[k] = db[k] + dy[k];
                }
            }
            sums[2 * r] = one(of_g).x + one(of_g).y;
            sums[2 * r + 1] = one(of_gn).x + one(of_gn).y;
        }
        team.template sums<2 * R>(sums, red[turn]);
        turn ^= 1;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (feed.row0 + r >= p.rows) continue;
            if ((live >> r) & 1) {
                Two x[K], dy[K];
                feed.take(r, 0, x);
                feed.take(r, 1, dy);
                const float m1 = sums[2 * r] * inv, m2 = sums[2 * r + 1] * inv;
                const Two minus = two(-st[r].x, -st[r].x), scale = two(st[r].y, st[r].y), minus1 = two(-m1, -m1), minus2 = two(-m2, -m2);
                feed.put(frame(p, a.dx, feed.row0 + r), [&](int k) { return scale * fma((x[k] + minus) * scale, minus2, fma(dy[k], w[k], minus1)); });
            } else {
                feed.put(frame(p, a.dx, feed.row0 + r), [](int) { return zero(); });
            }
        }
        feed.leave();
    }
    feed.finish();
    if (!p.work) return;
    auto channel = [&](int k, int h) { return V > 1 ? c0 + 2 * k / V * step + 2 * k % V + h : c0 + (2 * k + h) * step; };
    float* const to = p.work + (int64_t)blockIdx.x * 2 * channels;
    if (ONE) {  // the CTA's warps, in their order
        __syncthreads();
        float* const all = reinterpret_cast<float*>(shared_bytes);  // [2][channels] per team
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (channel(k, h) < channels) {
                    all[(2 * team.warp) * channels + channel(k, h)] = h ? one(dw[k]).y : one(dw[k]).x;
                    all[(2 * team.warp + 1) * channels + channel(k, h)] = h ? one(db[k]).y : one(db[k]).x;
                }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * channels; i += blockDim.x) {
            float v = 0.0f;
#pragma unroll
            for (int m = 0; m < Team<ONE>::kTeams; ++m) v += all[2 * m * channels + i];
            to[i] = v;
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (channel(k, h) < channels) {
                to[channel(k, h)] = h ? one(dw[k]).y : one(dw[k]).x;
                to[channels + channel(k, h)] = h ? one(db[k]).y : one(db[k]).x;
            }
}

// A CTA has 32 columns; its 16 warps take every sixteenth row each, and their sums are added in order.
__global__ void __launch_bounds__(512) k33_column_sums(const ColumnSums s)
{
    constexpr int W = 16, U = 4;
    __shared__ float sums[W][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t column = (int64_t)blockIdx.x * 32 + lane;
    float v[U] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (column < s.columns) {
        const float* from = s.part + column;
        int64_t row = warp;
        for (; row + (U - 1) * W < s.rows; row += U * W)
#pragma unroll
            for (int k = 0; k < U; ++k) v[k] += __ldcs(from + (row + k * W) * s.columns);
        for (; row < s.rows; row += W) v[0] += __ldcs(from + row * s.columns);
    }
    sums[warp][lane] = (v[0] + v[1]) + (v[2] + v[3]);
    __syncthreads();
    if (warp || column >= s.columns) return;
    float total = 0.0f;
#pragma unroll
    for (int k = 0; k < W; ++k) total += sums[k][lane];
    float* const out = column < s.end[0] ? s.out[0] : column < s.end[1] ? s.out[1] : s.out[2];
    const int64_t first = column < s.end[0] ? 0 : column < s.end[1] ? s.end[0] : s.end[1];
    if (out) out[column - first] = total;
}

// Channels of a thread: forward 16, 32 or 64, the least with which a warp has the frame; gradient 16, above 8,192 channels 32.
int per_thread(int64_t channels, bool gradient)
{
    if (gradient) return channels <= 8192 ? 16 : 32;
    return channels <= 512 ? 16 : channels <= 1024 ? 32 : 64;
}
struct Launch {
    int warps, rows, grid;  // of a team (one warp: four teams in a CTA); frames at once; CTAs
};
Launch launch_of(int64_t rows, int64_t channels, bool gradient)
{
    const int per = per_thread(channels, gradient), at_once = gradient && per <= 16 ? 2 : 1;
    const int warps = (int)((channels + per * 32 - 1) / (per * 32)), teams = warps == 1 ? 4 : 1;
    const int64_t wanted = (rows + at_once * teams - 1) / (at_once * teams), most = 148 * (16 / (warps * teams) > 1 ? 16 / (warps * teams) : 1);
    return {warps, at_once, (int)(wanted < most ? wanted : most)};  // 512 threads per SM
}

template <typename T>
bool on_16(const Channels<T>& x)
{
    return reinterpret_cast<uintptr_t>(x.data) % 16 == 0 && x.block * sizeof(T) % 16 == 0 && x.slot * sizeof(T) % 16 == 0;
}
// the address behind a tensor's last element
template <typename T>
uintptr_t end_of(const NormParams& p, const Channels<T>& x)
{
    return reinterpret_cast<uintptr_t>(x.data + (p.rows / p.t - 1) * x.block + (p.t - 1) * x.slot + p.channels);
}
template <typename T>
bool begins_on_16(const Channels<T>& x)
{
    return reinterpret_cast<uintptr_t>(x.data) % 16 == 0;
}
template <typename T>
bool flat(const NormParams& p, const Channels<T>& x) { return p.rows == p.t || x.block == p.t * x.slot; }

// calls go(V, P, one warp to a frame) for a call
template <typename T, bool GRADIENT, typename Go>
cudaError_t with_shape(int64_t channels, bool wide, int warps, const Go& go)
{
    constexpr int V = 16 / sizeof(T);
    auto per = [&](auto n, auto one) {
        constexpr int N = decltype(n)::value;
        return wide ? go(std::integral_constant<int, V>(), std::integral_constant<int, N / V>(), one)
                    : go(std::integral_constant<int, 1>(), std::integral_constant<int, N>(), one);
    };
    const int n = per_thread(channels, GRADIENT);
    using std::integral_constant;
    if constexpr (GRADIENT) {
        if (n == 32) return per(integral_constant<int, 32>(), std::false_type());
        return warps == 1 ? per(integral_constant<int, 16>(), std::true_type()) : per(integral_constant<int, 16>(), std::false_type());
    } else {
        if (n == 16) return per(integral_constant<int, 16>(), std::true_type());
        if (n == 32) return per(integral_constant<int, 32>(), std::true_type());
        return warps == 1 ? per(integral_constant<int, 64>(), std::true_type()) : per(integral_constant<int, 64>(), std::false_type());
    }
}

// Stages of `F` that fit where up to `ctas` CTAs share an SM's memory, beside `params` bytes of weights: fewer CTAs rather than less than
// two.  Returns the bytes of a CTA; `ctas`: how many share.
template <typename F, int V>
int shared_of(NormParams& p, const Launch& l, bool granules, int params, int& ctas)
{
    const int teams = l.warps == 1 ? 4 : 1, stage = F::stage_bytes(p.channels, l.warps * 32) * teams;
    ctas = 16 / (l.warps * teams) > 1 ? 16 / (l.warps * teams) : 1;
    while (ctas > 1 && (kMaxShared / ctas - params) / stage < 2) --ctas;
    const int fit = (kMaxShared / ctas - params) / stage;
    p.stages = fit > 3 ? 3 : fit < 1 ? 1 : fit;
    if (V == 1 && (!granules || p.stages < 2)) p.stages = 0;
    p.params_at = (p.stages * stage + 15) / 16 * 16;
    return p.params_at + params;
}

}  // namespace

cudaError_t launch_column_sums(const ColumnSums& s, cudaStream_t st)
{
    k33_column_sums<<<(unsigned)((s.columns + 31) / 32), 512, 0, st>>>(s);
    count_launches(1);
    return cudaGetLastError();
}

size_t norm_work_bytes(int64_t rows, int64_t channels)
{
    return (size_t)launch_of(rows, channels, true).grid * 2 * channels * sizeof(float);
}

template <typename T>
cudaError_t launch_norm(const NormParams& params, const NormTensors<T>& a, cudaStream_t st)
{
    NormParams p = params;
    p.flat = flat(p, a.x) && flat(p, a.y);
    p.end[0] = end_of(p, a.x);
    const bool wide = on_16(a.x) && on_16(a.y) && p.channels % (16 / sizeof(T)) == 0, granules = begins_on_16(a.x);
    const Launch l = launch_of(p.rows, p.channels, false);
    return with_shape<T, false>(p.channels, wide, l.warps, [&](auto v, auto n, auto one_warp) {
        constexpr int V = decltype(v)::value, P = decltype(n)::value;
        constexpr bool kOne = decltype(one_warp)::value;
        auto* kernel = k31_norm<T, V, P, kOne>;
        int ctas;
        const int shared = shared_of<Feed<T, V, P, 1, 1, kOne>, V>(p, l, granules, 2 * V * P * 32 * l.warps * 4, ctas);
        static std::atomic<uint64_t> allowed{0};
        const cudaError_t e = allow_shared(kernel, kMaxShared, allowed);
        if (e != cudaSuccess) return e;
        kernel<<<l.grid < 148 * ctas ? l.grid : 148 * ctas, kOne ? 128 : l.warps * 32, shared, st>>>(p, a);
        count_launches(1);
        return cudaGetLastError();
    });
}

template <typename T>
cudaError_t launch_norm_grad(const NormParams& params, const NormTensors<T>& a, cudaStream_t st)
{
    NormParams p = params;
    p.flat = flat(p, a.x) && flat(p, a.dy) && flat(p, a.dx);
    p.end[0] = end_of(p, a.x);
    p.end[1] = end_of(p, a.dy);
    const bool wide = on_16(a.x) && on_16(a.dy) && on_16(a.dx) && p.channels % (16 / sizeof(T)) == 0, granules = begins_on_16(a.x) && begins_on_16(a.dy);
    const Launch l = launch_of(p.rows, p.channels, true);
    const cudaError_t e = with_shape<T, true>(p.channels, wide, l.warps, [&](auto v, auto n, auto one_warp) {
        constexpr int V = decltype(v)::value, P = decltype(n)::value, R = V * P <= 16 ? 2 : 1;
        constexpr bool kOne = decltype(one_warp)::value;
        auto* kernel = k32_norm_grad<T, V, P, R, kOne>;
        int ctas;
        int shared = shared_of<Feed<T, V, P, R, 2, kOne>, V>(p, l, granules, 0, ctas);
        const int sums = kOne ? 4 * 2 * (int)p.channels * 4 : 0;
        if (shared < sums) shared = sums;
        static std::atomic<uint64_t> allowed{0};
        const cudaError_t f = allow_shared(kernel, kMaxShared, allowed);
        if (f != cudaSuccess) return f;
        kernel<<<l.grid, kOne ? 128 : l.warps * 32, shared, st>>>(p, a);
        count_launches(1);
        return cudaGetLastError();
    });
    if (e != cudaSuccess || !p.work) return e;
    const int64_t c = p.channels;
    return launch_column_sums({p.work, l.grid, 2 * c, {p.dweight, p.dbias, nullptr}, {c, 2 * c, 2 * c}}, st);
}
#define BLOAD_INSTANTIATE(T)                                                                     \
    template cudaError_t launch_norm<T>(const NormParams&, const NormTensors<T>&, cudaStream_t); \
    template cudaError_t launch_norm_grad<T>(const NormParams&, const NormTensors<T>&, cudaStream_t);
BLOAD_INSTANTIATE(float)
BLOAD_INSTANTIATE(__half)
BLOAD_INSTANTIATE(__nv_bfloat16)
#undef BLOAD_INSTANTIATE

}  // namespace bload

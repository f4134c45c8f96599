// k31_norm: layer norm over the channels of every frame of a packed batch; k32_norm_grad: its gradient; k33_column_sums: sums of
// partial sums, for the gradients of weights.
//
// Bytes only: x in, y out; x and dy in, dx out.  A CTA takes kRows frames at once and keeps them in registers: the mean, then the
// squares around it (in one pass their difference would lose what a large mean has in common), then y.  A thread has the same
// channels of every frame, so the gradient's sums over frames stay in its registers until the CTA has done its last frame; each CTA
// then writes them once, and k33 adds the CTAs' in their order.
#include <type_traits>

#include "bload_internal.cuh"
#include "bload_layers.cuh"

namespace bload {

namespace {

// V: elements of a piece (16 bytes, or one where rows do not allow it), P: pieces of a thread
template <int V, int P>
struct Shape {
    static constexpr int kPer = V * P;         // channels of a thread: 8, above 2,048 channels 16, above 8,192 32
    static constexpr int kRows = 32 / kPer;    // frames at once
    static constexpr int kMaxWarps = kPer > 8 ? 16 : 8;
};

// Frame `row` of a tensor; rows of blocks that lie one behind the other (p.flat) need no division.
template <typename C>
__device__ __forceinline__ auto frame(const NormParams& p, const C& x, int64_t row)
{
    if (p.flat) return x.data + row * x.slot;
    const int64_t q = row / p.t;
    return x.at(q, row - q * p.t);
}

// sums over the CTA's threads of N values each; `red`: [warps][N], the caller alternates between two of them
template <int N>
__device__ __forceinline__ void block_sums(float (&v)[N], float* red, int warps)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int first = 0;
    float w[N];
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = v[i];
    share_sums<N, 16, 1>(w, lane, first);
    if (lane % (32 / N) == 0) red[warp * N + first] = w[0];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.0f;
    for (int k = 0; k < warps; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += red[k * N + i];
}

template <typename T, int V, int P>
__global__ void __launch_bounds__(Shape<V, P>::kMaxWarps * 32) k31_norm(const NormParams p, const NormTensors<T> a)
{
    using S = Shape<V, P>;
    constexpr int R = S::kRows;
    __shared__ float red[2][S::kMaxWarps * R];
    const int warps = blockDim.x >> 5, c0 = threadIdx.x * V, step = blockDim.x * V, channels = (int)p.channels;
    const float inv = 1.0f / (float)channels;
    for (int64_t row0 = (int64_t)blockIdx.x * R; row0 < p.rows; row0 += (int64_t)gridDim.x * R) {
        Elements<T, V> x[R][P];
        bool live[R];
        float sum[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = row0 + r;
            live[r] = row < p.rows && p.pos[row] >= 0;
            const T* from = frame(p, a.x, row);
#pragma unroll
            for (int j = 0; j < P; ++j)
                if (live[r] && c0 + j * step < channels)
                    x[r][j].load(from + c0 + j * step, V, true);
                else
                    x[r][j].clear();
            sum[r] = 0.0f;
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < P; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) sum[r] += x[r][j].get(e);
        block_sums<R>(sum, red[0], warps);
        float square[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            sum[r] *= inv;
            square[r] = 0.0f;
#pragma unroll
            for (int j = 0; j < P; ++j)
                if (c0 + j * step < channels)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float d = x[r][j].get(e) - sum[r];
                        square[r] = fmaf(d, d, square[r]);
                    }
        }
        block_sums<R>(square, red[1], warps);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            square[r] = live[r] ? 1.0f / sqrtf(fmaf(square[r], inv, p.eps)) : 0.0f;
            if (p.stats && threadIdx.x == 0 && row0 + r < p.rows) p.stats[row0 + r] = make_float2(sum[r], square[r]);
        }
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const int c = c0 + j * step;
            if (c >= channels) continue;
            float w[V], b[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                w[e] = p.weight ? p.weight[c + e] : 1.0f;
                b[e] = p.bias ? p.bias[c + e] : 0.0f;
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int64_t row = row0 + r;
                if (row >= p.rows) continue;
#pragma unroll
                for (int e = 0; e < V; ++e) x[r][j].set(e, live[r] ? fmaf((x[r][j].get(e) - sum[r]) * square[r], w[e], b[e]) : 0.0f);
                x[r][j].store(frame(p, a.y, row) + c, V, true);
            }
        }
    }
}

template <typename T, int V, int P>
__global__ void __launch_bounds__(Shape<V, P>::kMaxWarps * 32) k32_norm_grad(const NormParams p, const NormTensors<T> a)
{
    using S = Shape<V, P>;
    constexpr int R = S::kRows;
    __shared__ float red[2][S::kMaxWarps * 2 * R];
    const int warps = blockDim.x >> 5, c0 = threadIdx.x * V, step = blockDim.x * V, channels = (int)p.channels;
    const float inv = 1.0f / (float)channels;
    float w[P][V], dw[P][V], db[P][V];
#pragma unroll
    for (int j = 0; j < P; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = c0 + j * step + e;
            w[j][e] = p.weight && c < channels ? p.weight[c] : 1.0f;
            dw[j][e] = db[j][e] = 0.0f;
        }
    int turn = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * R; row0 < p.rows; row0 += (int64_t)gridDim.x * R, turn ^= 1) {
        Elements<T, V> x[R][P], dy[R][P];
        bool live[R];
        float2 st[R];
        float sums[2 * R];  // of g, of g n
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = row0 + r;
            live[r] = row < p.rows && p.pos[row] >= 0;
            st[r] = live[r] ? p.stats[row] : make_float2(0.0f, 0.0f);
            const T *fx = frame(p, a.x, row), *fdy = frame(p, a.dy, row);
#pragma unroll
            for (int j = 0; j < P; ++j)
                if (live[r] && c0 + j * step < channels) {
                    x[r][j].load(fx + c0 + j * step, V, true);
                    dy[r][j].load(fdy + c0 + j * step, V, true);
                } else {
                    x[r][j].clear();
                    dy[r][j].clear();
                }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            sums[2 * r] = sums[2 * r + 1] = 0.0f;
#pragma unroll
            for (int j = 0; j < P; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float d = dy[r][j].get(e), n = (x[r][j].get(e) - st[r].x) * st[r].y, g = d * w[j][e];
                    sums[2 * r] += g;
                    sums[2 * r + 1] = fmaf(g, n, sums[2 * r + 1]);
                    dw[j][e] = fmaf(d, n, dw[j][e]);
                    db[j][e] += d;
                }
        }
        block_sums<2 * R>(sums, red[turn], warps);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = row0 + r;
            if (row >= p.rows) continue;
            const float m1 = sums[2 * r] * inv, m2 = sums[2 * r + 1] * inv;
            T* to = frame(p, a.dx, row);
#pragma unroll
            for (int j = 0; j < P; ++j) {
                if (c0 + j * step >= channels) continue;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float n = (x[r][j].get(e) - st[r].x) * st[r].y;
                    x[r][j].set(e, live[r] ? st[r].y * (fmaf(dy[r][j].get(e), w[j][e], -m1) - n * m2) : 0.0f);
                }
                x[r][j].store(to + c0 + j * step, V, true);
            }
        }
    }
    if (p.work) {
        float* const to = p.work + (int64_t)blockIdx.x * 2 * channels;
#pragma unroll
        for (int j = 0; j < P; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int c = c0 + j * step + e;
                if (c < channels) {
                    to[c] = dw[j][e];
                    to[channels + c] = db[j][e];
                }
            }
    }
}

// A CTA has 32 columns; its 8 warps take every eighth row each, and their sums are added in order.
__global__ void __launch_bounds__(256) k33_column_sums(const ColumnSums s)
{
    __shared__ float sums[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t column = (int64_t)blockIdx.x * 32 + lane;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (column < s.columns) {
        const float* from = s.part + column;
        int64_t row = warp;
        for (; row + 24 < s.rows; row += 32)
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += __ldcs(from + (row + 8 * k) * s.columns);
        for (; row < s.rows; row += 8) v[0] += __ldcs(from + row * s.columns);
    }
    sums[warp][lane] = (v[0] + v[1]) + (v[2] + v[3]);
    __syncthreads();
    if (warp || column >= s.columns) return;
    float total = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) total += sums[k][lane];
    const int which = column < s.end[0] ? 0 : column < s.end[1] ? 1 : 2;
    if (s.out[which]) s.out[which][column - (which ? s.end[which - 1] : 0)] = total;
}

int per_thread(int64_t channels) { return channels <= 2048 ? 8 : channels <= 8192 ? 16 : 32; }

// warps of a CTA, and how many CTAs
struct Launch {
    int warps, grid;
};
Launch launch_of(int64_t rows, int64_t channels)
{
    const int per = per_thread(channels), at_once = 32 / per;
    const int warps = (int)((channels + per * 32 - 1) / (per * 32));
    const int64_t wanted = (rows + at_once - 1) / at_once, most = 148 * (32 / warps);  // 1,024 threads per SM
    return {warps, (int)(wanted < most ? wanted : most)};
}

template <typename T>
bool on_16(const Channels<T>& x)
{
    return reinterpret_cast<uintptr_t>(x.data) % 16 == 0 && x.block * sizeof(T) % 16 == 0 && x.slot * sizeof(T) % 16 == 0;
}

}  // namespace

cudaError_t launch_column_sums(const ColumnSums& s, cudaStream_t st)
{
    k33_column_sums<<<(unsigned)((s.columns + 31) / 32), 256, 0, st>>>(s);
    count_launches(1);
    return cudaGetLastError();
}

size_t norm_work_bytes(int64_t rows, int64_t channels)
{
    return (size_t)launch_of(rows, channels).grid * 2 * channels * sizeof(float);
}

// calls go(kernel's V, P) for the sizes of a call
template <typename T, typename Go>
cudaError_t with_shape(int64_t channels, bool wide, const Go& go)
{
    constexpr int V = 16 / sizeof(T);
    auto per = [&](auto n) {
        constexpr int N = decltype(n)::value;
        return wide ? go(std::integral_constant<int, V>(), std::integral_constant<int, N / V>())
                    : go(std::integral_constant<int, 1>(), std::integral_constant<int, N>());
    };
    const int n = per_thread(channels);
    return n == 8 ? per(std::integral_constant<int, 8>()) : n == 16 ? per(std::integral_constant<int, 16>()) : per(std::integral_constant<int, 32>());
}
template <typename T>
bool flat(const NormParams& p, const Channels<T>& x) { return p.rows == p.t || x.block == p.t * x.slot; }

template <typename T>
cudaError_t launch_norm(const NormParams& params, const NormTensors<T>& a, cudaStream_t st)
{
    NormParams p = params;
    p.flat = flat(p, a.x) && flat(p, a.y);
    const Launch l = launch_of(p.rows, p.channels);
    return with_shape<T>(p.channels, on_16(a.x) && on_16(a.y) && p.channels % (16 / sizeof(T)) == 0, [&](auto v, auto n) {
        k31_norm<T, decltype(v)::value, decltype(n)::value><<<l.grid, l.warps * 32, 0, st>>>(p, a);
        count_launches(1);
        return cudaGetLastError();
    });
}

template <typename T>
cudaError_t launch_norm_grad(const NormParams& params, const NormTensors<T>& a, cudaStream_t st)
{
    NormParams p = params;
    p.flat = flat(p, a.x) && flat(p, a.dy) && flat(p, a.dx);
    const Launch l = launch_of(p.rows, p.channels);
    const bool wide = on_16(a.x) && on_16(a.dy) && on_16(a.dx) && p.channels % (16 / sizeof(T)) == 0;
    const cudaError_t e = with_shape<T>(p.channels, wide, [&](auto v, auto n) {
        k32_norm_grad<T, decltype(v)::value, decltype(n)::value><<<l.grid, l.warps * 32, 0, st>>>(p, a);
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

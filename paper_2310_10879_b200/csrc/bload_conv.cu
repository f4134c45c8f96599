// k34_conv: short causal convolution per channel inside the sequences of packed blocks, u_s = bias + sum_j w_j x_{s-j}, with or
// without u sigmoid(u) behind it; k35_conv_grad: its gradient; k36_conv_step: one new frame of each of many sequences.
//
// Bytes only: x in, y out (gradient: x, dy in, dx out).  A thread has V channels and walks a tile of slots; the inputs of the last
// taps - 1 slots stay in its registers, so every element is read once (and a tile's first taps - 1 slots by the tile before, too).  A
// tap counts where it does not reach in front of the sequence, j <= pos[s]: the test is the same for the whole CTA, and taken only
// where a sequence has just begun.
//
// The gradient walks the same way.  du_s goes to dx of the slots s - j, whose sums are in registers until slot s - (taps - 1) has
// all of its own; the taps - 1 slots behind the tile are computed once more for it.  Sums over the frames (weights, bias) stay in
// registers; a tile writes them once and k33 adds the tiles' in their order.
#include <type_traits>

#include "bload_internal.cuh"
#include "bload_layers.cuh"

namespace bload {

namespace {

constexpr int kThreads = 128, kAhead = 4;  // slots that are loaded together

// What a tile of a call is: CTAs are [block][tile][group of channels].
struct ConvTiles {
    int slots, tiles, groups, threads;
};

// weights by the distance back; channels of a thread are neighbours (WIDE) or blockDim.x apart
template <typename T, int V, int K, bool WIDE>
struct Columns {
    int64_t c0, step;
    int there;  // of the V channels
    __device__ __forceinline__ Columns(int64_t channels, int group)
    {
        const int64_t first = (int64_t)group * blockDim.x * V;
        c0 = first + (WIDE ? (int64_t)threadIdx.x * V : threadIdx.x);
        step = WIDE ? 1 : blockDim.x;
        const int64_t left = channels - c0;
        there = left <= 0 ? 0 : WIDE ? (int)min(left, (int64_t)V) : (int)min((left + step - 1) / step, (int64_t)V);
    }
    __device__ __forceinline__ void load(Elements<T, V>& x, const T* row) const
    {
        if (WIDE)
            x.load(row + c0, there, true);
        else
            x.load_apart(row + c0, step, there);
    }
    __device__ __forceinline__ void store(const Elements<T, V>& x, T* row) const
    {
        if (WIDE)
            x.store(row + c0, there, true);
        else
            x.store_apart(row + c0, step, there);
    }
    __device__ __forceinline__ void weights(const ConvParams& p, float (&w)[K][V], float (&bias)[V]) const
    {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            bias[e] = p.bias && e < there ? p.bias[c0 + e * step] : 0.0f;
#pragma unroll
            for (int j = 0; j < K; ++j) w[j][e] = j < p.taps && e < there ? p.weight[(c0 + e * step) * p.taps + p.taps - 1 - j] : 0.0f;
        }
    }
};

// taps of slot with position pos; K <= 4: there are K of them
template <int K>
__device__ __forceinline__ int taps_of(const ConvParams& p, int pos)
{
    return min(pos + 1, K <= 4 ? K : p.taps);
}

// u = bias + sum of the first `taps` (x is that of the slot itself, win[j - 1] of j slots back)
template <int V, int K>
__device__ __forceinline__ void convolve(float (&u)[V], const float (&bias)[V], const float (&w)[K][V], const float (&x)[V],
                                         const float (&win)[K - 1][V], int taps)
{
#pragma unroll
    for (int e = 0; e < V; ++e) u[e] = fmaf(w[0][e], x[e], bias[e]);
    if (taps == K) {
#pragma unroll
        for (int j = 1; j < K; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) u[e] = fmaf(w[j][e], win[j - 1][e], u[e]);
    } else {
#pragma unroll
        for (int j = 1; j < K; ++j)
            if (j < taps)
#pragma unroll
                for (int e = 0; e < V; ++e) u[e] = fmaf(w[j][e], win[j - 1][e], u[e]);
    }
}

template <typename T, int V, int K, bool WIDE>
__global__ void __launch_bounds__(kThreads) k34_conv(const ConvParams p, const ConvTensors<T> a, const ConvTiles tiles)
{
    const int64_t at = blockIdx.x / tiles.groups, q = at / tiles.tiles;
    const Columns<T, V, K, WIDE> col(p.channels, (int)(blockIdx.x - at * tiles.groups));
    const int s0 = (int)(at - q * tiles.tiles) * tiles.slots, s1 = min(s0 + tiles.slots, p.t);
    if (s0 >= p.t) return;
    float w[K][V], bias[V], win[K - 1][V];
    col.weights(p, w, bias);
    const int32_t* const pos = p.pos + q * p.t;
    const T* const x0 = a.x.data + q * a.x.block;
    T* const y0 = a.y.data + q * a.y.block;
    const int back = taps_of<K>(p, pos[s0]) - 1;  // inputs in front of the tile that its first slot sees (garbage positions: of this block)
#pragma unroll
    for (int j = 1; j < K; ++j) {
        Elements<T, V> x;
        x.clear();
        if (j <= back && j <= s0) col.load(x, x0 + (s0 - j) * a.x.slot);
#pragma unroll
        for (int e = 0; e < V; ++e) win[j - 1][e] = x.get(e);
    }
    const int64_t keep = p.taps - 1;
    for (int s = s0; s < s1; s += kAhead) {
        Elements<T, V> x[kAhead];
        int here[kAhead + 1];
#pragma unroll
        for (int i = 0; i <= kAhead; ++i) here[i] = s + i < p.t ? pos[s + i] : -1;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            x[i].clear();
            if (s + i < s1 && here[i] >= 0) col.load(x[i], x0 + (int64_t)(s + i) * a.x.slot);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (s + i >= s1) break;
            float v[V], u[V];
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = x[i].get(e);
            convolve<V, K>(u, bias, w, v, win, taps_of<K>(p, here[i]));
            if (p.tails && here[i] >= 0 && here[i + 1] != here[i] + 1) {  // the sequence ends
                const int64_t id = p.seq_id[q * p.t + s + i];
                if (id >= 0 && id < p.n_seq) {
                    T* const to = static_cast<T*>(p.tails) + id * keep * p.channels;
#pragma unroll
                    for (int j = 0; j < K - 1; ++j)
                        if (j < keep) {
                            Elements<T, V> old;
#pragma unroll
                            for (int e = 0; e < V; ++e) old.set(e, j > here[i] ? 0.0f : j == 0 ? v[e] : win[j > 0 ? j - 1 : 0][e]);
#pragma unroll
                            for (int e = 0; e < V; ++e)
                                if (e < col.there) to[(keep - 1 - j) * p.channels + col.c0 + e * col.step] = old.x[e];
                        }
                }
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float y = p.silu ? u[e] * sigmoid_of(u[e]) : u[e];
                x[i].set(e, here[i] >= 0 ? y : 0.0f);
            }
            col.store(x[i], y0 + (int64_t)(s + i) * a.y.slot);
#pragma unroll
            for (int e = 0; e < V; ++e) {
#pragma unroll
                for (int j = K - 2; j > 0; --j) win[j][e] = win[j - 1][e];
                win[0][e] = v[e];
            }
        }
    }
}

template <typename T, int V, int K, bool WIDE>
__global__ void __launch_bounds__(kThreads) k35_conv_grad(const ConvParams p, const ConvTensors<T> a, const ConvTiles tiles)
{
    const int64_t at = blockIdx.x / tiles.groups, q = at / tiles.tiles;
    const Columns<T, V, K, WIDE> col(p.channels, (int)(blockIdx.x - at * tiles.groups));
    const int s0 = (int)(at - q * tiles.tiles) * tiles.slots, s1 = min(s0 + tiles.slots, p.t);
    const int taps = K <= 4 ? K : p.taps;
    float w[K][V], bias[V], win[K - 1][V], dw[K][V], db[V], dx[K][V];  // dx[j]: of j slots back, so far
    col.weights(p, w, bias);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        db[e] = 0.0f;
#pragma unroll
        for (int j = 0; j < K; ++j) dw[j][e] = dx[j][e] = 0.0f;
    }
    if (s0 < p.t) {
        const int32_t* const pos = p.pos + q * p.t;
        const T *const x0 = a.x.data + q * a.x.block, *const dy0 = a.dy.data + q * a.dy.block;
        T* const dx0 = a.dx.data + q * a.dx.block;
        const int back = taps_of<K>(p, pos[s0]) - 1;
#pragma unroll
        for (int j = 1; j < K; ++j) {
            Elements<T, V> x;
            x.clear();
            if (j <= back && j <= s0) col.load(x, x0 + (s0 - j) * a.x.slot);
#pragma unroll
            for (int e = 0; e < V; ++e) win[j - 1][e] = x.get(e);
        }
        const int end = s1 + taps - 1;
        for (int s = s0; s < end; s += kAhead) {
            Elements<T, V> x[kAhead], dy[kAhead];
            int here[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {  // a slot behind the tile counts where it reaches into it
                here[i] = s + i < p.t ? pos[s + i] : -1;
                if (s + i >= s1 && here[i] < s + i - s1 + 1) here[i] = -1;
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                x[i].clear();
                dy[i].clear();
                if (here[i] >= 0 && s + i < end) {
                    col.load(x[i], x0 + (int64_t)(s + i) * a.x.slot);
                    col.load(dy[i], dy0 + (int64_t)(s + i) * a.dy.slot);
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (s + i >= end) break;
                float v[V], du[V];
                const int n = taps_of<K>(p, here[i]);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    v[e] = x[i].get(e);
                    du[e] = dy[i].get(e);
                }
                if (p.silu) {
                    float u[V];
                    convolve<V, K>(u, bias, w, v, win, n);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float g = sigmoid_of(u[e]);
                        du[e] = here[i] >= 0 ? du[e] * fmaf(u[e] * g, 1.0f - g, g) : 0.0f;
                    }
                }
                const bool mine = s + i < s1;
#pragma unroll
                for (int j = 0; j < K; ++j)
                    if (j < n) {
#pragma unroll
                        for (int e = 0; e < V; ++e) dx[j][e] = fmaf(w[j][e], du[e], dx[j][e]);
                        if (mine)
#pragma unroll
                            for (int e = 0; e < V; ++e) dw[j][e] = fmaf(du[e], j == 0 ? v[e] : win[j > 0 ? j - 1 : 0][e], dw[j][e]);
                    }
                if (mine)
#pragma unroll
                    for (int e = 0; e < V; ++e) db[e] += du[e];
                // slot s + i - (taps - 1) has all of its own
                const int done = s + i - (taps - 1);
                if (done >= s0) {
                    Elements<T, V> out;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        float last = dx[K - 1][e];
                        if (K > 4) {
#pragma unroll
                            for (int j = 0; j < K; ++j) last = j == taps - 1 ? dx[j][e] : last;
                        }
                        out.set(e, last);
                    }
                    col.store(out, dx0 + (int64_t)done * a.dx.slot);
                }
#pragma unroll
                for (int e = 0; e < V; ++e) {
#pragma unroll
                    for (int j = K - 1; j > 0; --j) dx[j][e] = dx[j - 1][e];
                    dx[0][e] = 0.0f;
#pragma unroll
                    for (int j = K - 2; j > 0; --j) win[j][e] = win[j - 1][e];
                    win[0][e] = v[e];
                }
            }
        }
    }
    if (p.work) {
        float* const to = p.work + at * p.channels * (taps + 1);
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e < col.there) {
                const int64_t c = col.c0 + e * col.step;
#pragma unroll
                for (int j = 0; j < K; ++j)
                    if (j < taps) to[c * taps + taps - 1 - j] = dw[j][e];
                to[p.channels * taps + c] = db[e];
            }
    }
}

// A thread has V channels of kRowsAtOnce rows: its weights serve all of them, and the rows' loads are under way together.
constexpr int kRowsAtOnce = 4;
template <typename T, int V, int K, bool WIDE>
__global__ void __launch_bounds__(kThreads) k36_conv_step(const ConvParams p, int64_t rows, const T* state, T* next, const T* x, int64_t sx,
                                                         T* y, int64_t sy, int groups)
{
    const int64_t at = blockIdx.x / groups, row0 = at * kRowsAtOnce;
    const Columns<T, V, K, WIDE> col(p.channels, (int)(blockIdx.x - at * groups));
    const int64_t keep = p.taps - 1, size = keep * p.channels;
    Elements<T, V> now[kRowsAtOnce], old[kRowsAtOnce][K - 1];  // old[j - 1]: j frames back
    int here[kRowsAtOnce];
#pragma unroll
    for (int r = 0; r < kRowsAtOnce; ++r) here[r] = row0 + r < rows ? p.pos[row0 + r] : -1;
#pragma unroll
    for (int r = 0; r < kRowsAtOnce; ++r) {
        const bool on = row0 + r < rows;
        now[r].clear();
        if (on && here[r] >= 0) col.load(now[r], x + (row0 + r) * sx);
#pragma unroll
        for (int j = 1; j < K; ++j) {
            old[r][j - 1].clear();
            if (on && j <= keep && (here[r] < 0 || j <= here[r])) col.load(old[r][j - 1], state + (row0 + r) * size + (keep - j) * p.channels);
        }
    }
    float w[K][V], bias[V];
    col.weights(p, w, bias);
#pragma unroll
    for (int r = 0; r < kRowsAtOnce; ++r) {
        if (row0 + r >= rows) break;
        float v[V], u[V], win[K - 1][V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            v[e] = now[r].get(e);
#pragma unroll
            for (int j = 1; j < K; ++j) win[j - 1][e] = old[r][j - 1].get(e);
        }
        convolve<V, K>(u, bias, w, v, win, taps_of<K>(p, here[r]));
        Elements<T, V> out;
#pragma unroll
        for (int e = 0; e < V; ++e) out.set(e, here[r] < 0 ? 0.0f : p.silu ? u[e] * sigmoid_of(u[e]) : u[e]);
        col.store(out, y + (row0 + r) * sy);
        T* const to = next + (row0 + r) * size;
        if (here[r] >= 0) {
#pragma unroll
            for (int j = 0; j < K - 1; ++j)
                if (j < keep) col.store(j == 0 ? now[r] : old[r][j > 0 ? j - 1 : 0], to + (keep - 1 - j) * p.channels);
        } else if (next != state) {
#pragma unroll
            for (int j = 0; j < K - 1; ++j)
                if (j < keep) col.store(old[r][j], to + (keep - 1 - j) * p.channels);
        }
    }
}

// Channels of a thread: 8 forward (4 for 32-bit elements), 4 in the gradient, whose sums take a register each; 2 for more than 4 taps.
int channels_per_thread(size_t size, int taps, bool gradient) { return taps > 4 ? 2 : gradient || size == 4 ? 4 : 8; }

ConvTiles tiles_of(int64_t blocks, int32_t t, int64_t channels, int v)
{
    ConvTiles x;
    const int64_t units = (channels + v - 1) / v;
    x.threads = units >= kThreads ? kThreads : (int)((units + 31) / 32 * 32);
    x.groups = (int)((units + x.threads - 1) / x.threads);
    // eight CTAs per SM, of at least 32 slots each
    const int64_t wanted = 148 * 8 * kThreads / x.threads / x.groups, slots = wanted ? (blocks * t + wanted - 1) / wanted : t;
    x.slots = (int)(slots < 32 ? 32 : slots > t ? t : slots);
    x.tiles = (t + x.slots - 1) / x.slots;
    return x;
}

template <typename T, int V>
bool on(const Channels<T>& x)
{
    constexpr size_t n = V * sizeof(T) < 16 ? V * sizeof(T) : 16;
    return reinterpret_cast<uintptr_t>(x.data) % n == 0 && x.block * sizeof(T) % n == 0 && x.slot * sizeof(T) % n == 0;
}

// calls go(K) for the taps of a call: exactly 2, 3 or 4, or up to 8
template <typename Go>
cudaError_t with_taps(int taps, const Go& go)
{
    switch (taps) {
        case 2: return go(std::integral_constant<int, 2>());
        case 3: return go(std::integral_constant<int, 3>());
        case 4: return go(std::integral_constant<int, 4>());
        default: return go(std::integral_constant<int, 8>());
    }
}
template <int K, bool GRADIENT, typename T>
constexpr int kChannels = K > 4 ? 2 : GRADIENT || sizeof(T) == 4 ? 4 : 8;
// one tap has no place in an exact instance
int taps_class(int taps) { return taps == 1 ? BLOAD_CONV_MAX_TAPS : taps; }

}  // namespace

size_t conv_work_bytes(int64_t blocks, int32_t t, int64_t channels, int32_t taps, int32_t dtype)
{
    const ConvTiles x = tiles_of(blocks, t, channels, channels_per_thread(dtype == BLOAD_F32 ? 4 : 2, taps_class(taps), true));
    return (size_t)blocks * x.tiles * channels * (taps + 1) * sizeof(float);
}

template <typename T>
cudaError_t launch_conv(const ConvParams& p, const ConvTensors<T>& a, cudaStream_t st)
{
    return with_taps(p.taps, [&](auto k) {
        constexpr int K = decltype(k)::value, V = kChannels<K, false, T>;
        const ConvTiles x = tiles_of(p.blocks, p.t, p.channels, V);
        const bool wide = on<const T, V>(a.x) && on<T, V>(a.y) && p.channels % V == 0;
        auto* kernel = wide ? k34_conv<T, V, K, true> : k34_conv<T, V, K, false>;
        kernel<<<(unsigned)(p.blocks * x.tiles * x.groups), x.threads, 0, st>>>(p, a, x);
        count_launches(1);
        return cudaGetLastError();
    });
}

template <typename T>
cudaError_t launch_conv_grad(const ConvParams& p, const ConvTensors<T>& a, cudaStream_t st)
{
    ConvTiles x{};
    const cudaError_t e = with_taps(p.taps, [&](auto k) {
        constexpr int K = decltype(k)::value, V = kChannels<K, true, T>;
        x = tiles_of(p.blocks, p.t, p.channels, V);
        const bool wide = on<const T, V>(a.x) && on<const T, V>(a.dy) && on<T, V>(a.dx) && p.channels % V == 0;
        auto* kernel = wide ? k35_conv_grad<T, V, K, true> : k35_conv_grad<T, V, K, false>;
        kernel<<<(unsigned)(p.blocks * x.tiles * x.groups), x.threads, 0, st>>>(p, a, x);
        count_launches(1);
        return cudaGetLastError();
    });
    if (e != cudaSuccess || !p.work) return e;
    const int64_t n = p.channels * p.taps, all = n + p.channels;
    return launch_column_sums({p.work, p.blocks * x.tiles, all, {p.dweight, p.dbias, nullptr}, {n, all, all}}, st);
}

template <typename T>
cudaError_t launch_conv_step(const ConvParams& p, int64_t rows, const T* state, T* next, const T* x, int64_t sx, T* y, int64_t sy,
                             cudaStream_t st)
{
    return with_taps(p.taps, [&](auto k) {
        constexpr int K = decltype(k)::value, V = kChannels<K, true, T>;
        const int64_t units = (p.channels + V - 1) / V;
        const int threads = units >= kThreads ? kThreads : (int)((units + 31) / 32 * 32), groups = (int)((units + threads - 1) / threads);
        auto fits = [&](const T* data, int64_t row) { return on<const T, V>(Channels<const T>{data, row, 0}); };
        const bool wide = fits(state, p.channels) && fits(next, p.channels) && fits(x, sx) && fits(y, sy) && p.channels % V == 0;
        auto* kernel = wide ? k36_conv_step<T, V, K, true> : k36_conv_step<T, V, K, false>;
        kernel<<<(unsigned)((rows + kRowsAtOnce - 1) / kRowsAtOnce * groups), threads, 0, st>>>(p, rows, state, next, x, sx, y, sy, groups);
        count_launches(1);
        return cudaGetLastError();
    });
}
#define BLOAD_INSTANTIATE(T)                                                                     \
    template cudaError_t launch_conv<T>(const ConvParams&, const ConvTensors<T>&, cudaStream_t); \
    template cudaError_t launch_conv_grad<T>(const ConvParams&, const ConvTensors<T>&, cudaStream_t); \
    template cudaError_t launch_conv_step<T>(const ConvParams&, int64_t, const T*, T*, const T*, int64_t, T*, int64_t, cudaStream_t);
BLOAD_INSTANTIATE(float)
BLOAD_INSTANTIATE(__half)
BLOAD_INSTANTIATE(__nv_bfloat16)
#undef BLOAD_INSTANTIATE

}  // namespace bload

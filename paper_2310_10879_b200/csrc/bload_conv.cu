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
//
// 8 x 4096 x 2048 bf16, 4 taps, with the gate: 62 us forward (4.3 TB/s), 104 gradient (3.9 TB/s; 576 CTAs with all their registers); step of
// 256 x 4096 fp16 7.9 us; last inputs of 219 prompts kept as well: 3 us more; 2047 channels, rows off any boundary: 193 and 326 us, by
// element loads when a slot's turn has come, nothing ahead.  Bound by latency and issue: 30 instructions an element in the
// gradient, 0.55 of the issue slots, half of what the multiply-adds allow.
#include <type_traits>

#include "bload_internal.cuh"
#include "bload_layers.cuh"

namespace bload {

namespace {

constexpr int kThreads = 128;

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
    // slot s of the block that begins at `first` (WIDE: a block spans less than 2^32 bytes)
    __device__ __forceinline__ void store_slot(const Elements<T, V>& x, T* first, int64_t slot, int s) const
    {
        if (WIDE)
            x.store(reinterpret_cast<T*>(reinterpret_cast<char*>(first) + ((uint32_t)s * ((uint32_t)slot * (uint32_t)sizeof(T)) + (uint32_t)c0 * (uint32_t)sizeof(T))), there, true);
        else
            store(x, first + s * slot);
    }
    __device__ __forceinline__ void weights(const ConvParams& p, Two (&w)[K][V / 2], Two (&bias)[V / 2]) const
    {
        auto of = [&](const float* from, int64_t each, int e) { return e < there ? from[(c0 + e * step) * each] : 0.0f; };
#pragma unroll
        for (int e = 0; e < V; e += 2) {
            bias[e / 2] = p.bias ? two(of(p.bias, 1, e), of(p.bias, 1, e + 1)) : zero();
#pragma unroll
            for (int j = 0; j < K; ++j) {
                const float* const from = p.weight + p.taps - 1 - j;
                w[j][e / 2] = j < p.taps ? two(of(from, p.taps, e), of(from, p.taps, e + 1)) : zero();
            }
        }
    }
};

// taps of slot with position pos; K <= 4: there are K of them
template <int K>
__device__ __forceinline__ int taps_of(const ConvParams& p, int pos)
{
    return min(pos + 1, K <= 4 ? K : p.taps);
}

// Slots that are worked on together: a multiple of the taps, so that the window of the last K inputs turns in place.
template <int K>
constexpr int kChunk = K <= 3 ? 2 * K : K;

// Brings chunks of slots to a thread, its channels of TENSORS tensors.  WIDE: by asynchronous copies into shared memory, each thread's
// own (no barrier), three chunks ahead; otherwise into registers when their turn has come.
template <typename T, int V, int K, bool WIDE, int TENSORS>
struct Slots {
    static constexpr int U = kChunk<K>, kStages = 4, kBytes = V * sizeof(T);
    static constexpr int kShared = WIDE ? kStages * U * TENSORS * kBytes * kThreads : 0;
    const Columns<T, V, K, WIDE>& col;
    const Channels<const T>* tensors[TENSORS];
    const T* at[TENSORS];  // the block's first slot (WIDE: the CTA's; a block spans less than 2^32 bytes)
    uint32_t mine;         // WIDE: bytes from there to the thread's channels
    const int32_t* pos;
    uint32_t ring;
    int t, stage;
    int next[U + 1];  // positions of the next chunk, and the slot behind
    Elements<T, V> raw[WIDE ? 1 : U][TENSORS];

    __device__ __forceinline__ Slots(const Columns<T, V, K, WIDE>& c) : col(c) {}
    __device__ __forceinline__ void init(const ConvParams& p, int64_t q, uint8_t* shared)
    {
        pos = p.pos + q * p.t;
        t = p.t;
        stage = 0;
        ring = (uint32_t)__cvta_generic_to_shared(shared) + threadIdx.x * kBytes;
#pragma unroll
        for (int n = 0; n < TENSORS; ++n) at[n] = tensors[n]->data + q * tensors[n]->block + (WIDE ? 0 : col.c0);
        mine = (uint32_t)col.c0 * (uint32_t)sizeof(T);
    }
    // WIDE: slot s of a tensor of this block
    __device__ __forceinline__ const T* slot_of(int n, int s) const
    {
        return reinterpret_cast<const T*>(reinterpret_cast<const char*>(at[n]) + ((uint32_t)s * ((uint32_t)tensors[n]->slot * (uint32_t)sizeof(T)) + mine));
    }
    __device__ __forceinline__ void look(int s)
    {
#pragma unroll
        for (int i = 0; i <= U; ++i) next[i] = s + i < t ? pos[s + i] : -1;
    }
    // begins to copy a chunk; slots from `end` on are not touched
    __device__ __forceinline__ void fetch(int s, int end, int to)
    {
        if constexpr (WIDE) {
            if (col.there) {
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    if (s + i >= end) break;
#pragma unroll
                    for (int n = 0; n < TENSORS; ++n) {
                        const uint32_t dst = ring + (uint32_t)(((to * U + i) * TENSORS + n) * kBytes * kThreads);
                        const T* const src = slot_of(n, s + i);
                        if constexpr (kBytes == 16)
                            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
                        else
                            asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(kBytes) : "memory");
                    }
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    }
    __device__ __forceinline__ void start(int s, int end)
    {
        look(s);
#pragma unroll
        for (int k = 0; k < kStages - 1; ++k) fetch(s + k * U, end, k);
    }
    // The chunk of slot s has come: here[i] are its positions, changed by `which` (those below 0 are not loaded).
    template <typename Which>
    __device__ __forceinline__ void arrive(int s, int end, int (&here)[U + 1], const Which& which)
    {
#pragma unroll
        for (int i = 0; i <= U; ++i) here[i] = which(s + i, next[i]);
        fetch(s + (kStages - 1) * U, end, stage ? stage - 1 : kStages - 1);
        look(s + U);
        if constexpr (WIDE) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
        } else {
#pragma unroll
            for (int i = 0; i < U; ++i)
#pragma unroll
                for (int n = 0; n < TENSORS; ++n) {
                    raw[WIDE ? 0 : i][n].clear();
                    if (here[i] >= 0 && s + i < end) raw[WIDE ? 0 : i][n].load_apart(at[n] + (int64_t)(s + i) * tensors[n]->slot, col.step, col.there);
                }
        }
    }
    // slot i of the chunk, 0 where it is not `on`
    __device__ __forceinline__ void get(int i, int n, bool on, Two (&x)[V / 2]) const
    {
        Elements<T, V> e;
        e.clear();
        if constexpr (WIDE) {
            if (on && col.there) {
                const uint32_t src = ring + (uint32_t)(((stage * U + i) * TENSORS + n) * kBytes * kThreads);
                if constexpr (kBytes == 16) {
                    uint4 w;
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(src) : "memory");
                    *reinterpret_cast<uint4*>(e.x) = w;
                } else if constexpr (kBytes == 8) {
                    uint2 w;
                    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w.x), "=r"(w.y) : "r"(src) : "memory");
                    *reinterpret_cast<uint2*>(e.x) = w;
                } else {
                    uint32_t w;
                    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(src) : "memory");
                    *reinterpret_cast<uint32_t*>(e.x) = w;
                }
            }
        } else {
            e = raw[WIDE ? 0 : i][n];
        }
#pragma unroll
        for (int k = 0; k < V; k += 2) x[k / 2] = e.pair(k);
    }
    __device__ __forceinline__ void leave() { stage = stage + 1 == kStages ? 0 : stage + 1; }
    __device__ __forceinline__ void finish() const
    {
        if (WIDE) asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
    // the inputs in front of slot s0 that it sees, into the window: slot s lies at s % K, counted from s0
    __device__ __forceinline__ void behind(const ConvParams& p, int s0, Two (&win)[K][V / 2])
    {
        const int back = taps_of<K>(p, pos[s0]) - 1;  // (whatever positions hold: inside the block)
#pragma unroll
        for (int j = 1; j < K; ++j) {
            Elements<T, V> x;
            x.clear();
            if (j <= back && j <= s0) {
                if (WIDE)
                    x.load(slot_of(0, s0 - j), col.there, true);
                else
                    x.load_apart(at[0] + (int64_t)(s0 - j) * tensors[0]->slot, col.step, col.there);
            }
#pragma unroll
            for (int k = 0; k < V; k += 2) win[K - j][k / 2] = x.pair(k);
        }
#pragma unroll
        for (int k = 0; k < V / 2; ++k) win[0][k] = zero();
    }
};

// calls go(j) for the first n taps; where n is K, without a test on each
template <int K, typename Go>
__device__ __forceinline__ void for_taps(int n, const Go& go)
{
    if (n == K) {
#pragma unroll
        for (int j = 0; j < K; ++j) go(j);
    } else {
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (j < n) go(j);
    }
}

template <typename T, int V, int K, bool WIDE>
__global__ void __launch_bounds__(kThreads) k34_conv(const ConvParams p, const ConvTensors<T> a, const ConvTiles tiles)
{
    extern __shared__ __align__(16) uint8_t shared_bytes[];
    using S = Slots<T, V, K, WIDE, 1>;
    constexpr int U = S::U, H = V / 2;
    const unsigned at = blockIdx.x / (unsigned)tiles.groups, q = at / (unsigned)tiles.tiles;
    const Columns<T, V, K, WIDE> col(p.channels, (int)(blockIdx.x - at * (unsigned)tiles.groups));
    const int s0 = (int)(at - q * (unsigned)tiles.tiles) * tiles.slots, s1 = min(s0 + tiles.slots, p.t);
    if (s0 >= p.t) return;
    S slots(col);
    slots.tensors[0] = &a.x;
    slots.init(p, q, shared_bytes);
    slots.start(s0, s1);
    Two w[K][H], bias[H], win[K][H];  // win: the last K inputs, slot s0 + i at i % K
    col.weights(p, w, bias);
    slots.behind(p, s0, win);
    T* const y0 = a.y.data + q * a.y.block;
    const int64_t keep = p.taps - 1;
    const int full = K <= 4 ? K - 1 : p.taps - 1;
    for (int s = s0; s < s1; s += U) {
        int here[U + 1];
        slots.arrive(s, s1, here, [](int, int pos) { return pos; });
        auto chunk = [&](auto with_tests) {
            constexpr bool tests = decltype(with_tests)::value;
#pragma unroll
            for (int i = 0; i < U; ++i) {
                if (tests && s + i >= s1) break;
                const bool on = !tests || here[i] >= 0;
                Two(&now)[H] = win[i % K];
                slots.get(i, 0, on, now);
                Elements<T, V> out;
                if (on) {
                    Two u[H];
#pragma unroll
                    for (int k = 0; k < H; ++k) u[k] = bias[k];
                    for_taps<K>(!tests && K <= 4 ? K : taps_of<K>(p, here[i]), [&](int j) {
#pragma unroll
                        for (int k = 0; k < H; ++k) u[k] = fma(w[j][k], win[(i + K - j) % K][k], u[k]);
                    });
#pragma unroll
                    for (int k = 0; k < H; ++k) out.set_pair(2 * k, p.silu ? u[k] * sigmoid_of(u[k]) : u[k]);
                    if (tests && p.tails && here[i + 1] != here[i] + 1) {  // the sequence ends
                        const int64_t id = p.seq_id[(int64_t)q * p.t + s + i];
                        if (id >= 0 && id < p.n_seq) {
                            T* const to = static_cast<T*>(p.tails) + id * keep * p.channels + col.c0;
#pragma unroll
                            for (int j = 0; j < K - 1; ++j)
                                if (j < keep) {
#pragma unroll
                                    for (int e = 0; e < V; ++e) {
                                        const float2 x = one(win[(i + K - j) % K][e / 2]);
                                        if (e < col.there) to[(keep - 1 - j) * p.channels + e * col.step] = from_float<T>(j > here[i] ? 0.0f : e & 1 ? x.y : x.x);
                                    }
                                }
                        }
                    }
                } else {
                    out.clear();
                }
                col.store_slot(out, y0, a.y.slot, s + i);
            }
        };
        // whole chunks in which no sequence begins or ends need no tests
        bool plain = s + U <= s1;
#pragma unroll
        for (int i = 0; i < U; ++i) plain = plain && here[i] >= full && (i + 1 < U || !p.tails || here[U] > 0);
        if (plain)
            chunk(std::false_type());
        else
            chunk(std::true_type());
        slots.leave();
    }
    slots.finish();
}

template <typename T, int V, int K, bool WIDE>
__global__ void __launch_bounds__(kThreads) k35_conv_grad(const ConvParams p, const ConvTensors<T> a, const ConvTiles tiles)
{
    extern __shared__ __align__(16) uint8_t shared_bytes[];
    using S = Slots<T, V, K, WIDE, 2>;
    constexpr int U = S::U, H = V / 2;
    const unsigned at = blockIdx.x / (unsigned)tiles.groups, q = at / (unsigned)tiles.tiles;
    const Columns<T, V, K, WIDE> col(p.channels, (int)(blockIdx.x - at * (unsigned)tiles.groups));
    const int s0 = (int)(at - q * (unsigned)tiles.tiles) * tiles.slots, s1 = min(s0 + tiles.slots, p.t);
    const int taps = K <= 4 ? K : p.taps;
    Two w[K][H], bias[H], win[K][H], dw[K][H], db[H], dx[K][H];  // dx: of the last K slots, so far; slot s0 + i at i % K
#pragma unroll
    for (int k = 0; k < H; ++k) {
        db[k] = zero();
#pragma unroll
        for (int j = 0; j < K; ++j) dw[j][k] = dx[j][k] = zero();
    }
    if (s0 < p.t) {
        const int end = min(s1 + taps - 1, p.t);
        S slots(col);
        slots.tensors[0] = &a.x;
        slots.tensors[1] = &a.dy;
        slots.init(p, q, shared_bytes);
        slots.start(s0, end);
        col.weights(p, w, bias);
        slots.behind(p, s0, win);
        T* const dx0 = a.dx.data + q * a.dx.block;
        for (int s = s0; s < s1 + taps - 1; s += U) {
            int here[U + 1];
            // a slot behind the tile counts where it reaches into it
            slots.arrive(s, end, here, [&](int slot, int pos) { return slot >= s1 && pos < slot - s1 + 1 ? -1 : pos; });
            auto chunk = [&](auto with_tests) {
                constexpr bool tests = decltype(with_tests)::value;
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    if (tests && s + i >= s1 + taps - 1) break;
                    const bool on = !tests || (here[i] >= 0 && s + i < end), mine = !tests || s + i < s1;
                    Two(&now)[H] = win[i % K];
                    Two du[H];
                    slots.get(i, 0, on, now);
                    slots.get(i, 1, on, du);
#pragma unroll
                    for (int k = 0; k < H; ++k) dx[i % K][k] = zero();
                    if (on) {
                        const int n = !tests && K <= 4 ? K : taps_of<K>(p, here[i]);
                        if (p.silu) {
                            Two u[H];
#pragma unroll
                            for (int k = 0; k < H; ++k) u[k] = bias[k];
                            for_taps<K>(n, [&](int j) {
#pragma unroll
                                for (int k = 0; k < H; ++k) u[k] = fma(w[j][k], win[(i + K - j) % K][k], u[k]);
                            });
                            // d(u sig) = sig + u sig (1 - sig)
#pragma unroll
                            for (int k = 0; k < H; ++k) {
                                const Two sig = sigmoid_of(u[k]);
                                du[k] = du[k] * fma(u[k] * sig, fma(sig, two(-1.0f, -1.0f), two(1.0f, 1.0f)), sig);
                            }
                        }
                        for_taps<K>(n, [&](int j) {
#pragma unroll
                            for (int k = 0; k < H; ++k) dx[(i + K - j) % K][k] = fma(w[j][k], du[k], dx[(i + K - j) % K][k]);
                        });
                        if (mine) {
                            for_taps<K>(n, [&](int j) {
#pragma unroll
                                for (int k = 0; k < H; ++k) dw[j][k] = fma(du[k], win[(i + K - j) % K][k], dw[j][k]);
                            });
#pragma unroll
                            for (int k = 0; k < H; ++k) db[k] = db[k] + du[k];
                        }
                    }
                    // slot s + i - (taps - 1) has all of its own
                    const int done = s + i - (taps - 1);
                    if (!tests || done >= s0) {
                        Elements<T, V> out;
#pragma unroll
                        for (int k = 0; k < H; ++k) {
                            Two v = dx[(i + 1) % K][k];
                            if (K > 4) {
#pragma unroll
                                for (int j = 0; j < K; ++j) v.v = j == taps - 1 ? dx[(i + K - j) % K][k].v : v.v;
                            }
                            out.set_pair(2 * k, v);
                        }
                        col.store_slot(out, dx0, a.dx.slot, done);
                    }
                }
            };
            bool plain = s > s0 && s + U <= s1;
#pragma unroll
            for (int i = 0; i < U; ++i) plain = plain && here[i] >= taps - 1;
            if (plain)
                chunk(std::false_type());
            else
                chunk(std::true_type());
            slots.leave();
        }
        slots.finish();
    }
    if (p.work) {
        float* const to = p.work + (int64_t)at * p.channels * (taps + 1);
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e < col.there) {
                const int64_t c = col.c0 + e * col.step;
                auto half = [&](Two x) { return e & 1 ? one(x).y : one(x).x; };
#pragma unroll
                for (int j = 0; j < K; ++j)
                    if (j < taps) to[c * taps + taps - 1 - j] = half(dw[j][e / 2]);
                to[p.channels * taps + c] = half(db[e / 2]);
            }
    }
}

// A thread has V channels of kRowsAtOnce rows: its weights serve all of them, and the rows' loads are under way together.
constexpr int kRowsAtOnce = 4;
template <typename T, int V, int K, bool WIDE>
__global__ void __launch_bounds__(kThreads) k36_conv_step(const ConvParams p, int64_t rows, const T* state, T* next, const T* x, int64_t sx,
                                                         T* y, int64_t sy, int groups)
{
    const unsigned at = blockIdx.x / (unsigned)groups;
    const int64_t row0 = (int64_t)at * kRowsAtOnce;
    const Columns<T, V, K, WIDE> col(p.channels, (int)(blockIdx.x - at * (unsigned)groups));
    const int64_t keep = p.taps - 1, size = keep * p.channels;
    Elements<T, V> now[kRowsAtOnce], old[kRowsAtOnce][K - 1];  // old[j - 1]: j frames back
    int here[kRowsAtOnce];
#pragma unroll
    for (int r = 0; r < kRowsAtOnce; ++r) here[r] = row0 + r < rows ? p.pos[row0 + r] : -1;
#pragma unroll
    for (int r = 0; r < kRowsAtOnce; ++r) {
        const bool on = row0 + r < rows;
        now[r].clear();
        if (on) col.load(now[r], x + (row0 + r) * sx);  // (whether or not it will be used: positions arrive no sooner)
#pragma unroll
        for (int j = 1; j < K; ++j) {
            old[r][j - 1].clear();
            if (on && j <= keep) col.load(old[r][j - 1], state + (row0 + r) * size + (keep - j) * p.channels);
        }
    }
    Two w[K][V / 2], bias[V / 2];
    col.weights(p, w, bias);
#pragma unroll
    for (int r = 0; r < kRowsAtOnce; ++r) {
        if (row0 + r >= rows) break;
        if (here[r] >= 0 && here[r] < K - 1) {  // in front of the sequence there is nothing
#pragma unroll
            for (int j = 1; j < K; ++j)
                if (j > here[r]) old[r][j - 1].clear();
        }
        Two u[V / 2];
#pragma unroll
        for (int k = 0; k < V / 2; ++k) u[k] = bias[k];
        for_taps<K>(taps_of<K>(p, here[r]), [&](int j) {
#pragma unroll
            for (int k = 0; k < V / 2; ++k) u[k] = fma(w[j][k], (j ? old[r][j > 0 ? j - 1 : 0] : now[r]).pair(2 * k), u[k]);
        });
        Elements<T, V> out;
        out.clear();
        if (here[r] >= 0)
#pragma unroll
            for (int k = 0; k < V / 2; ++k) out.set_pair(2 * k, p.silu ? u[k] * sigmoid_of(u[k]) : u[k]);
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
    // four CTAs per SM, as many as registers allow, in one wave; tiles of at least 32 slots
    const int64_t wanted = (int64_t)148 * 4 * kThreads / x.threads / x.groups / blocks, slots = wanted > 1 ? (t + wanted - 1) / wanted : t;
    x.slots = (int)(slots < 32 ? 32 : slots);
    x.tiles = (t + x.slots - 1) / x.slots;
    return x;
}

// pieces of V elements lie on boundaries of their size, and t slots span less than 2^32 bytes
template <typename T, int V>
bool on(const Channels<T>& x, int32_t t)
{
    constexpr size_t n = V * sizeof(T) < 16 ? V * sizeof(T) : 16;
    if ((uint64_t)x.slot * sizeof(T) >= ((uint64_t)1 << 31) / (uint64_t)t) return false;
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
        const bool wide = on<const T, V>(a.x, p.t) && on<T, V>(a.y, p.t) && p.channels % V == 0 && p.channels * (int64_t)sizeof(T) < ((int64_t)1 << 31);
        auto* kernel = wide ? k34_conv<T, V, K, true> : k34_conv<T, V, K, false>;
        constexpr int kShared = Slots<T, V, K, true, 1>::kShared;
        static std::atomic<uint64_t> allowed{0};
        const cudaError_t e = allow_shared(k34_conv<T, V, K, true>, kShared, allowed);
        if (e != cudaSuccess) return e;
        kernel<<<(unsigned)(p.blocks * x.tiles * x.groups), x.threads, wide ? kShared : 0, st>>>(p, a, x);
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
        const bool wide = on<const T, V>(a.x, p.t) && on<const T, V>(a.dy, p.t) && on<T, V>(a.dx, p.t) && p.channels % V == 0 && p.channels * (int64_t)sizeof(T) < ((int64_t)1 << 31);
        auto* kernel = wide ? k35_conv_grad<T, V, K, true> : k35_conv_grad<T, V, K, false>;
        constexpr int kShared = Slots<T, V, K, true, 2>::kShared;
        static std::atomic<uint64_t> allowed{0};
        const cudaError_t e = allow_shared(k35_conv_grad<T, V, K, true>, kShared, allowed);
        if (e != cudaSuccess) return e;
        kernel<<<(unsigned)(p.blocks * x.tiles * x.groups), x.threads, wide ? kShared : 0, st>>>(p, a, x);
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
        auto fits = [&](const T* data, int64_t row) { return on<const T, V>(Channels<const T>{data, row, 0}, 1); };
        const bool wide = fits(state, p.channels) && fits(next, p.channels) && fits(x, sx) && fits(y, sy) && p.channels % V == 0 && p.channels * (int64_t)sizeof(T) < ((int64_t)1 << 31);
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

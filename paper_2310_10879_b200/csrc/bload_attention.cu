// Attention inside the sequences of packed blocks, and its gradients, on the fifth-generation tensor cores.
//
//   k29_attention       128 queries per CTA: scores S = Q K^T and out += P V per tile of 128 keys
//   k30_attention_grad  <queries>: 128 queries per CTA, dq;  <keys>: 128 keys per CTA, dk and dv
//
// Every row (a query, or a key of the second gradient kernel) may see one interval of slots [lo, hi] -- its sequence, cut by
// causality and by the window -- so a CTA walks the tiles from the smallest lo of its rows to their largest hi, and a tile's
// mask is a range of columns per row.  Products run in 16 bits with sums in 32; scores, statistics, probabilities and
// accumulators are held in 32 bits, and P and dS are rounded to the inputs' type as operands of the second product.  For
// fp16 they are scaled by powers of two first, since its smallest step, 2^-24, is one of 16 million keys' even share, and dS is that
// times whatever dout is: P by a constant, dS row by row by what the row's largest needs (see k30_attention_grad).
//
// Hidden slots must have no influence, but a product multiplies them by zero, and 0 * NaN is not 0.  So a tile that is hidden
// from any row of the CTA is scanned (one multiply-add by zero per pair of elements), and infinities and NaN in it are cleared in
// shared memory before a product reads across it.  Rows that may see a frame that held some have them added in the end, read
// from memory once more (add_junk): a clean row's bits do not depend on what a hidden slot holds.  With v and dout infinite
// everywhere, 8,192 slots of 4 heads on 2 of 128 take 254 us forward and 600 gradient (fp16 1,120; clean: 155 and 360), 4 x 4096 slots of
// heavy-tailed lengths 250 and 610 (fp16 750; clean: 46 and 125).
#include <cuda.h>
#include <math.h>

#include <type_traits>

#include "bload_internal.cuh"
#include "bload_layers.cuh"
#include "bload_tc.cuh"

namespace bload {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kNever = 1 << 30;

__device__ unsigned int g_timeouts;  // bounded waits that gave up (bload_device_timeouts)

template <bool BF16>
struct Element {
    using type = __half;
};
template <>
struct Element<true> {
    using type = __nv_bfloat16;
};

// The interval of the other side that a row may see: the keys of a query, the queries of a key.  Empty: lo > hi.
struct Span {
    int lo, hi;
};
// That of row `row`, of this warp's rows row0 .. row0 + 31.
__device__ __forceinline__ Span span_of(const AttnParams& p, const int32_t* pos, int row, bool keys, int lane)
{
    const int row0 = row - lane;
    const int here = row < p.t ? pos[row] : -1;
    int end = row + 1;
    if (keys || !p.causal) {  // (uniform) the sequence of a row ends at the next start or padding in the warp, or behind it
        const unsigned stops = __ballot_sync(0xffffffffu, here <= 0) & ~((2u << lane) - 1);
        const int last = __shfl_sync(0xffffffffu, here, 31);
        int behind = row0 + 32;
        if (last >= 0) behind = warp_seq_end(pos, p.t, row0 + 31, lane);
        end = stops ? row0 + __ffs(stops) - 1 : behind;
    }
    if (here < 0) return {kNever, -1};
    Span s;
    if (keys) {
        s.lo = p.causal ? row : max(row - here, 0);
        s.hi = end - 1;
    } else {
        s.lo = max(row - here, 0);
        s.hi = p.causal ? row : end - 1;
    }
    s.lo = max(s.lo, row - (p.window - 1));
    s.hi = min(s.hi, row + (p.window - 1));
    return s;
}

// Meeting point of the two warps that share 32 rows.
__device__ __forceinline__ void pair_barrier(int pair) { asm volatile("bar.sync %0, 64;" ::"r"(1 + pair) : "memory"); }

// columns [lo, hi] of 32
__device__ __forceinline__ uint32_t column_mask(int lo, int hi)
{
    lo = max(lo, 0);
    hi = min(hi, 31);
    return lo > hi ? 0u : (0xffffffffu << lo) & (0xffffffffu >> (31 - hi));
}

// The intervals of a CTA's rows together.
struct Reach {
    int lo, hi;         // smallest lo, largest hi
    int all_lo, all_hi; // [all_lo, all_hi] is seen by every row that sees anything
    int least;          // columns that the row sees that sees the fewest
};
template <int WARPS>
struct ReachShared {
    int lo[WARPS], hi[WARPS], all_lo[WARPS], all_hi[WARPS], least[WARPS];
};
template <int WARPS>
__device__ __forceinline__ void put_reach(ReachShared<WARPS>& sh, int warp, int lane, const Span& s)
{
    const bool some = s.lo <= s.hi;
    const int lo = __reduce_min_sync(0xffffffffu, some ? s.lo : kNever), hi = __reduce_max_sync(0xffffffffu, some ? s.hi : -1);
    const int all_lo = __reduce_max_sync(0xffffffffu, some ? s.lo : -1), all_hi = __reduce_min_sync(0xffffffffu, some ? s.hi : kNever);
    const int least = __reduce_min_sync(0xffffffffu, some ? s.hi - s.lo + 1 : kNever);
    if (lane == 0) {
        sh.lo[warp] = lo;
        sh.hi[warp] = hi;
        sh.all_lo[warp] = all_lo;
        sh.all_hi[warp] = all_hi;
        sh.least[warp] = least;
    }
}
template <int WARPS>
__device__ __forceinline__ Reach get_reach(const ReachShared<WARPS>& sh)
{
    Reach r{sh.lo[0], sh.hi[0], sh.all_lo[0], sh.all_hi[0], sh.least[0]};
#pragma unroll
    for (int w = 1; w < WARPS; ++w) {
        r.lo = min(r.lo, sh.lo[w]);
        r.hi = max(r.hi, sh.hi[w]);
        r.all_lo = max(r.all_lo, sh.all_lo[w]);
        r.all_hi = min(r.all_hi, sh.all_hi[w]);
        r.least = min(r.least, sh.least[w]);
    }
    return r;
}

// A CTA's tiles of COLUMNS columns: tile i starts at first + i * step.  Causal walks start at the CTA's own rows, from where queries go
// down and keys go up, so that the first tile can be copied in before the positions are known; others at the smallest lo.
template <int COLUMNS>
struct Walk {
    int first, step;
    static __device__ __forceinline__ int causal_first(const AttnParams& p, int row0, bool keys)
    {
        return keys ? row0 : row0 + (min(p.t - row0, 128) - 1) / COLUMNS * COLUMNS;
    }
    __device__ __forceinline__ Walk(const AttnParams& p, const Reach& r, int row0, bool keys)
    {
        first = p.causal ? causal_first(p, row0, keys) : r.lo;
        step = p.causal && !keys ? -COLUMNS : COLUMNS;
    }
    __device__ __forceinline__ int count(const Reach& r) const
    {
        return r.hi < 0 ? 0 : step > 0 ? (r.hi - first) / COLUMNS + 1 : (max(first - r.lo, 0) + COLUMNS - 1) / COLUMNS + 1;
    }
    __device__ __forceinline__ int operator()(int i) const { return first + i * step; }
};

// score in units of log2 from q.k, with the cap and the distance bias; `inner` = d score / d (scale q.k)
struct Modifier {
    enum { kPlain, kNear, kAny };  // no cap; capped and every |scale q.k / cap| of the warp's columns below 1/2; capped
    float by, unit, cap2, slope2;  // scale * log2e; scale / cap; cap * log2e; slope * log2e
    __device__ __forceinline__ Modifier(const AttnParams& p, int h)
    {
        by = p.scale * kLog2e;
        unit = p.cap > 0.0f ? p.scale / p.cap : 0.0f;
        cap2 = p.cap * kLog2e;
        slope2 = p.slopes ? p.slopes[h] * kLog2e : 0.0f;
    }
    // which of the three a warp's scores take, so that the usual small ones cost no special functions
    __device__ __forceinline__ int kind(const uint32_t (&qk)[32]) const
    {
        if (!(cap2 > 0.0f)) return kPlain;
        float top[2] = {};
#pragma unroll
        for (int e = 0; e < 32; ++e) top[e & 1] = fmaxf(top[e & 1], fabsf(__uint_as_float(qk[e])));
        return __all_sync(0xffffffffu, fmaxf(top[0], top[1]) * fabsf(unit) < 0.5f) ? kNear : kAny;
    }
    // Of two neighbouring columns, the first `apart` slots behind (a whole number, exact as float: conversions of integers run at
    // a quarter of the rate of additions).
    // tanh(y), |y| < 1/2: y (1 + c1 y^2 + ... + c4 y^8), the coefficients of smallest largest relative error (2.8e-8, found by
    // iteratively reweighted least squares).  Else 1 - 2 / (1 + exp(2 y)), whose absolute error of some 2^-23 is small against
    // values from 0.46 on, but not against a score much smaller than its cap.
    template <int KIND>
    __device__ __forceinline__ Two apply(Two qk, float apart, Two& inner) const
    {
        auto both = [](float c) { return two(c, c); };
        Two x;
        if (KIND == kPlain) {
            x = qk * both(by);
            inner = both(1.0f);
        } else {
            const Two y = qk * both(unit), z = y * y;
            Two th = fma(z, both(0.0171350036f), both(-0.0529860742f));
            th = fma(th, z, both(0.133247793f));
            th = fma(th, z, both(-0.333330691f));
            th = fma(th * z, y, y);
            if (KIND == kAny) {
                const float2 y1 = one(y), t1 = one(th);
                auto far = [](float v) { return fmaf(-2.0f, tc::inverse_fast(1.0f + tc::exp2_fast(v * (2.0f * kLog2e))), 1.0f); };
                th = two(fabsf(y1.x) < 0.5f ? t1.x : far(y1.x), fabsf(y1.y) < 0.5f ? t1.y : far(y1.y));  // (NaN goes to far, and stays)
            }
            x = both(cap2) * th;
            inner = fma(th * both(-1.0f), th, both(1.0f));
        }
        const float2 v = one(x);
        return two(fmaf(-slope2, fabsf(apart), v.x), fmaf(-slope2, fabsf(apart - 1.0f), v.y));
    }
    // f(kind) with the kind as a constant
    template <typename F>
    static __device__ __forceinline__ void with(int kind, F f)
    {
        if (kind == kNear)
            f(std::integral_constant<int, kNear>());
        else if (kind == kAny)
            f(std::integral_constant<int, kAny>());
        else
            f(std::integral_constant<int, kPlain>());
    }
};

// -lse in units of log2; a row without any weight keeps none
__device__ __forceinline__ float minus_lse(float lse) { return lse == -INFINITY ? -INFINITY : -lse * kLog2e; }

// Junk: which tiles of a CTA's walk held infinities or NaN in a frame, and what its rows may see.
template <int COLUMNS>
struct Junk {
    uint32_t tiles[BLOAD_MAX_T_BLOCK / COLUMNS / 32 + 1];
    Span spans[128];
    int any;
};

// Scans a tile [ROWS][DP] in shared memory, number `turn` of its walk, with THREADS threads for infinities and NaN, and clears them;
// ready(): called before anything is cleared.  (Behind the block's last slot copies fill in zeros.)
template <bool BF16, int ROWS, int DP, int THREADS, typename Ready>
__device__ __forceinline__ void scan_tile(const AttnParams& p, const int32_t* pos, uint8_t* tile, int row0, int tid, Junk<ROWS>& junk, int turn,
                                          const Ready& ready)
{
    uint32_t acc = 0;
    constexpr int kChunks = ROWS * DP / 8 / THREADS;
#pragma unroll
    for (int k = 0; k < kChunks; ++k) {
        const uint4 x = *reinterpret_cast<const uint4*>(tile + (k * THREADS + tid) * 16);
        acc = tc::probe<BF16>(tc::probe<BF16>(acc, x.x), x.y);
        acc = tc::probe<BF16>(tc::probe<BF16>(acc, x.z), x.w);
    }
    if (!(acc & 0x7fff7fffu)) return;
    ready();
    for (int k = 0; k < kChunks; ++k) {
        uint32_t* const at = reinterpret_cast<uint32_t*>(tile + (k * THREADS + tid) * 16);
        bool some = false;
        for (int e = 0; e < 4; ++e) {
            const uint32_t x = at[e], odd = tc::probe<BF16>(0u, x);
            if (!(odd & 0x7fff7fffu)) continue;
            some = true;
            at[e] = x & ((odd & 0x7fff ? 0u : 0xffffu) | (odd & 0x7fff0000u ? 0u : 0xffff0000u));
        }
        const int row = row0 + (k * THREADS + tid) / 8 % ROWS;
        if (some && row < p.t && pos[row] >= 0) {
            atomicOr(&junk.tiles[turn / 32], 1u << turn % 32);
            junk.any = 1;
        }
    }
}

template <bool BF16, int ROWS, int DP, int THREADS>
__device__ __noinline__ void scan_tile_apart(const AttnParams& p, const int32_t* pos, uint8_t* tile, int row0, int tid, Junk<ROWS>& junk, int turn,
                                             uint32_t after, uint32_t parity, int& dead)
{
    scan_tile<BF16, ROWS, DP, THREADS>(p, pos, tile, row0, tid, junk, turn, [&] {
        if (after && !tc::bar_wait(after, parity)) dead = 1;
    });
}

// What the cleared elements of x add to the CTA's 128 rows, to add[128][DP]: infinities and NaN of every frame that a row may see
// in a tile where some were cleared; POISON: NaN for each of them.  A warp has ROWS rows, a lane DP / 32 elements; of a tile that a row
// sees as far as any row does, the sum is formed once for the warp's rows.
template <bool POISON, int ROWS, int DP, int COLUMNS, typename T, typename Walk>
__device__ __noinline__ void add_junk(const AttnParams& p, const Junk<COLUMNS>& junk, const Reach reach, const Walk walk, int tiles, const Heads<const T> x, int b, int head,
                                      int heads, float* add, int warp, int lane)
{
    constexpr int kPer = DP / 32;
    const bool on = lane * kPer < p.d;
    for (int r = warp * ROWS; r < (warp + 1) * ROWS; ++r)
        for (int e = 0; e < kPer; ++e) add[r * DP + lane * kPer + e] = 0.0f;
    for (int i = 0; i < tiles; ++i) {
        if (!((junk.tiles[i / 32] >> i % 32) & 1)) continue;
        const int first = max(walk(i), reach.lo), last = min(walk(i) + COLUMNS - 1, reach.hi);
        for (int hs = head; hs < head + heads; ++hs) {
            auto sum = [&](int lo, int hi, float (&s)[kPer]) {
                for (int e = 0; e < kPer; ++e) s[e] = 0.0f;
                if (!on) return;
#pragma unroll 8
                for (int j = lo; j <= hi; ++j) {
                    using W = typename std::conditional<kPer == 4, uint2, uint32_t>::type;
                    const W w = *reinterpret_cast<const W*>(x.at(b, j, hs) + lane * kPer);
#pragma unroll
                    for (int e = 0; e < kPer; ++e) {
                        const float v = to_float(reinterpret_cast<const T*>(&w)[e]);
                        s[e] += POISON ? v * 0.0f : isfinite(v) ? 0.0f : v;
                    }
                }
            };
            float whole[kPer];
            bool have = false;
            for (int r = warp * ROWS; r < (warp + 1) * ROWS; ++r) {
                const int lo = max(junk.spans[r].lo, first), hi = min(junk.spans[r].hi, last);
                if (lo > hi) continue;
                float own[kPer];
                const bool all = lo == first && hi == last;
                if (!all) sum(lo, hi, own);
                if (all && !have) sum(lo, hi, whole);
                have |= all;
                for (int e = 0; e < kPer; ++e) add[r * DP + lane * kPer + e] += all ? whole[e] : own[e];
            }
        }
    }
}

// 32 columns of a row to 64 bytes of a staged output tile (128-byte rows, swizzled)
template <bool BF16>
__device__ __forceinline__ void stage_columns(uint8_t* tile, int row, int column, const float (&x)[32])
{
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        uint4 w;
        w.x = tc::pack<BF16>(x[8 * c], x[8 * c + 1]);
        w.y = tc::pack<BF16>(x[8 * c + 2], x[8 * c + 3]);
        w.z = tc::pack<BF16>(x[8 * c + 4], x[8 * c + 5]);
        w.w = tc::pack<BF16>(x[8 * c + 6], x[8 * c + 7]);
        *reinterpret_cast<uint4*>(tile + row * 128 + (((column / 8 + c) ^ (row & 7)) * 16)) = w;
    }
}

// ---- forward ------------------------------------------------------------------------------------------------------

struct ForwardMaps {
    CUtensorMap q, k, v, out;  // boxes of 128, kKeys, kKeys, 32 rows by 64 elements
};

template <int DP>
struct ForwardTile {
    static constexpr int kHalves = DP / 64;  // warps that share 32 rows, with 64 columns each
    static constexpr int kKeys = 64 * kHalves, kWarps = 4 * kHalves, kThreads = 32 * kWarps + 64;
    static constexpr int kStages = DP == 64 ? 2 : 1;
    static constexpr int kQueries = 128 * DP * 2, kTile = kKeys * DP * 2;  // bytes
    static constexpr int kShared = kQueries + 2 * kStages * kTile + 1024;
    static constexpr int kTmem = DP + kKeys, kCtas = 512 / kTmem;  // per SM
};

// Heads of up to 128 elements: tiles of 128 keys, two CTAs per SM.  Warps 0 to 7 have the queries' arithmetic: warp w and warp w + 4
// the same 32 rows, a row per lane, each half of the columns (with one warp per row the tensor cores were busy 31 % of the time:
// too few warps to hide the latency of their own steps).  The two halves of a row agree on its maximum through shared memory,
// each keeps its own sum.  Heads of up to 64: tiles of 64 keys, four warps, four CTAs per SM (short sequences leave a CTA with
// two or three tiles between its first copies and its last store, so it pays to have more of them: 16 x 1000 frames of features 64 us,
// in the instance for 128, half zeros, 89; one sequence of 16,384 takes 372 us here and 316 there).
// Scores come from tensor memory, P goes back over them.  Two more warps copy tiles in and issue the products.  The CTAs of an SM
// share its tensor memory evenly, so one's products run under the others' exponentials.
template <bool BF16, int DP, bool MOD>
__global__ void __launch_bounds__(ForwardTile<DP>::kThreads, ForwardTile<DP>::kCtas)
    k29_attention(const AttnParams p, const AttnTensors<typename Element<BF16>::type> a, const __grid_constant__ ForwardMaps maps)
{
    using Tile = ForwardTile<DP>;
    constexpr int kHalves = Tile::kHalves, kKeys = Tile::kKeys, kWarps = Tile::kWarps;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t bars[5 + 4 * Tile::kStages];
    __shared__ uint32_t tmem_base;
    __shared__ int dead;
    __shared__ Junk<kKeys> junk;
    __shared__ ReachShared<4> reach_shared;
    __shared__ float halves[2][kHalves][128];  // [turn][half][row]: maxima, and in the end sums

    uint8_t* const tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* const q_tile = tiles;
    uint8_t* const k_tiles = tiles + Tile::kQueries;
    uint8_t* const v_tiles = k_tiles + Tile::kStages * Tile::kTile;
    const uint32_t bar0 = tc::smem_of(bars);
    const uint32_t q_full = bar0, s_full = bar0 + 8, p_full = bar0 + 16, o_done = bar0 + 24, k_full = bar0 + 32,
                   k_free = k_full + 8 * Tile::kStages, v_full = k_free + 8 * Tile::kStages, v_free = v_full + 8 * Tile::kStages,
                   given_up = v_free + 8 * Tile::kStages;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int q_tiles = (p.t + 127) / 128;
    const int64_t bh = blockIdx.x % (p.blocks * p.heads);
    const int i0 = (q_tiles - 1 - (int)(blockIdx.x / (p.blocks * p.heads))) * 128;  // the longest rows of a long sequence first
    const int h = (int)(bh % p.heads), hk = h / p.group, b = (int)(bh / p.heads);
    const int32_t* const pos = p.pos + (int64_t)b * p.t;
    const int half = warp >> 2, quarter = warp & 3;  // of the arithmetic's warps
    const int own_row = quarter * 32 + lane, row = i0 + own_row;

    auto load = [&](bool keys, int s, int j0) {  // the tile of keys (or of values) from slot j0 on, to stage s
        const uint32_t bar = (keys ? k_full : v_full) + 8 * s, to = tc::smem_of(keys ? k_tiles : v_tiles) + s * Tile::kTile;
        tc::bar_expect(bar, Tile::kTile);
        for (int x = 0; x < DP; x += 64) tc::tensor_load(to + x * (2 * kKeys), keys ? &maps.k : &maps.v, x, j0, hk, b, bar);
    };
    Span span{kNever, -1};
    if (warp < kWarps) {
        span = span_of(p, pos, row, false, lane);
        if (half == 0) {
            put_reach(reach_shared, quarter, lane, span);
            junk.spans[own_row] = span;
            if (tid < (int)(sizeof junk.tiles / 4)) junk.tiles[tid] = 0;
        }
        if (tid == 0) dead = junk.any = 0;
    } else if (warp == kWarps) {
        if (lane == 0) {
            tc::bar_init(q_full, 1);
            tc::bar_init(s_full, 1);
            tc::bar_init(p_full, 32 * kWarps);
            tc::bar_init(o_done, 1);
            for (int s = 0; s < 4 * Tile::kStages; ++s) tc::bar_init(k_full + 8 * s, 1);
            tc::bar_init(given_up, 1);
            tc::bar_init_done();
            tc::bar_expect(q_full, Tile::kQueries);  // under way while the rows look for their keys
            for (int x = 0; x < DP; x += 64) tc::tensor_load(tc::smem_of(q_tile) + x * 256, &maps.q, x, i0, h, b, q_full);
            if (p.causal) {
                const int j0 = Walk<kKeys>::causal_first(p, i0, false);
                load(true, 0, j0);
                load(false, 0, j0);
            }
        }
    } else {
        tc::tmem_alloc<Tile::kTmem>(tc::smem_of(&tmem_base));
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = tmem_base, o_at = tmem, s_at = tmem + DP;
    const Reach reach = get_reach(reach_shared);
    const Walk<kKeys> walk(p, reach, i0, false);
    const int n = walk.count(reach);
    float m = -INFINITY, l = 0.0f;  // running maximum (log2 units; may lag by kLag) and sum
    // fp16 holds up to 2^16: exponentials of up to 2^kLag are kept 2^kLift times as large, sum and accumulator with them
    constexpr float kLag = 8.0f, kLift = BF16 ? 0.0f : 7.0f;
    int issued_k = p.causal, issued_v = p.causal;  // (warp of the copies)
    bool ended = false;                            // (warp of the products) none are under way

    if (warp == kWarps) {
        if (lane == 0) {
            bool ok = true;
            if (n == 0) ok = tc::bar_wait(q_full, 0) && (!p.causal || (tc::bar_wait(k_full, 0) && tc::bar_wait(v_full, 0)));  // (copies end)
            for (int i = p.causal; i < n; ++i) {
                const int s = i % Tile::kStages;
                const uint32_t parity = (i / Tile::kStages + 1) & 1;
                if (!(ok = tc::bar_wait(k_free + 8 * s, parity))) break;
                load(true, s, walk(i));
                issued_k = i + 1;
                if (!(ok = tc::bar_wait(v_free + 8 * s, parity))) break;
                load(false, s, walk(i));
                issued_v = i + 1;
            }
            if (!ok) dead = 1;
        }
    } else if (warp == kWarps + 1) {
        ended = true;
        if (n > 0) {
            const uint32_t leader = tc::elect();
            bool ok = __all_sync(0xffffffffu, tc::bar_wait(q_full, 0));
            ended = false;
            for (int i = 0; i < n && ok; ++i) {
                const int s = i % Tile::kStages;
                const uint32_t parity = (i / Tile::kStages) & 1;
                // the scores take the place of the last tile's P: the product that reads it has to be over
                ok = __all_sync(0xffffffffu, tc::bar_wait(k_full + 8 * s, parity) && (i == 0 || tc::bar_wait(o_done, (i - 1) & 1)));
                if (!ok) break;
                tc::fence_after();
                tc::product_rows<BF16, kKeys, DP>(leader, s_at, tc::smem_of(q_tile), tc::smem_of(k_tiles) + s * Tile::kTile);
                if (i + Tile::kStages < n) tc::products_arrive(leader, k_free + 8 * s);  // (nothing arrives that nobody waits for)
                tc::products_arrive(leader, s_full);
                ok = __all_sync(0xffffffffu, tc::bar_wait(v_full + 8 * s, parity) && tc::bar_wait(p_full, i & 1));
                if (!ok) break;
                tc::fence_after();
                tc::product_across<BF16, kKeys, DP, 64>(leader, o_at, s_at, tc::smem_of(v_tiles) + s * Tile::kTile, i > 0);
                if (i + Tile::kStages < n) tc::products_arrive(leader, v_free + 8 * s);
                tc::products_arrive(leader, o_done);
            }
            if (!ok) {
                dead = 1;
                tc::products_arrive(leader, given_up);
                tc::bar_wait(given_up, 0);
                ended = true;
            }
        }
    } else {
        const Modifier modify(p, h);
        const uint32_t lanes = (uint32_t)quarter << 21;  // this warp's 32 lanes of tensor memory
        const float by = modify.by;
        bool ok = true;
        for (int i = 0; i < n; ++i) {
            const int st = i % Tile::kStages;
            const int j0 = walk(i), mine0 = j0 + 64 * half;  // the tile's and this warp's first key
            // (a warp that gives up goes on without waiting: its partner meets it at a barrier in every turn)
            if (ok && !(ok = __all_sync(0xffffffffu, tc::bar_wait(s_full, i & 1)))) dead = 1;
            tc::fence_after();
            // The scores in units of log2 are x by (MOD: x itself); hidden ones are -inf.  They are read twice, for the maximum and
            // for the exponentials: 64 of them would not stay in this thread's registers.  What changes them is written back.
            const uint32_t own_at = s_at + lanes + 64 * half;
            const float apart = (float)(row - mine0);
            // All seen by all of the warp's rows, none by any: per 64 columns, or for heads of at most 64 elements, where short walks
            // are what counts, per 32 (16 x 1000 frames of features 69 -> 65 us, but one sequence of 16,384 304 -> 321 us).
            constexpr int kFine = kHalves == 1 ? 2 : 1;
            bool clear[2], blind[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int c0 = mine0 + 32 * c, c1 = c0 + 64 / kFine - 1;
                clear[c] = c < kFine ? (bool)__all_sync(0xffffffffu, span.lo <= c0 && span.hi >= c1) : clear[0];
                blind[c] = c < kFine ? (bool)__all_sync(0xffffffffu, span.lo > c1 || span.hi < c0) : blind[0];
            }
            float top = -INFINITY;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                if (blind[c]) continue;
                uint32_t s[32];
                tc::tmem_load(s, own_at + 32 * c);
                tc::tmem_loaded();
                tc::settle(s);
                if (MOD)
                    Modifier::with(modify.kind(s), [&](auto kind) {
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            Two inner;
                            const float2 x = one(modify.apply<decltype(kind)::value>(two(__uint_as_float(s[e]), __uint_as_float(s[e + 1])),
                                                                                     apart - (float)(32 * c + e), inner));
                            s[e] = __float_as_uint(x.x);
                            s[e + 1] = __float_as_uint(x.y);
                        }
                    });
                if (!clear[c]) {
                    const uint32_t mask = column_mask(span.lo - mine0 - 32 * c, span.hi - mine0 - 32 * c);
#pragma unroll
                    for (int e = 0; e < 32; ++e) s[e] = (mask >> e) & 1 ? s[e] : 0xff800000u;
                }
                if (MOD || !clear[c]) tc::tmem_store(own_at + 32 * c, s);
                float t4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int e = 0; e < 32; e += 2)
                    t4[(e / 2) & 3] = fmaxf(t4[(e / 2) & 3], fmaxf(__uint_as_float(s[e]), __uint_as_float(s[e + 1])));
                top = fmaxf(top, fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])));
            }
            if (MOD || !clear[0] || !clear[1]) tc::tmem_stored();
            if (kHalves == 2) {
                halves[i & 1][half][own_row] = top;
                pair_barrier(quarter);
                top = fmaxf(top, halves[i & 1][kHalves - 1 - half][own_row]);
            }
            if (!MOD) top *= by;
            // The maximum that scales the exponentials may lag behind by a factor of 2^8: the result is the same, and the
            // accumulator in tensor memory is rescaled only when a row has moved further than that.  (The second half's warp
            // sees the same maxima and moves with the first's.)
            const bool move = top > m + kLag || (m == -INFINITY && top > m);
            if (__any_sync(0xffffffffu, move)) {
                const float now = move ? top : m;
                const float down = m == now ? 1.0f : m == -INFINITY ? 0.0f : tc::exp2_fast(m - now);
                l *= down;
                m = now;
                if (i > 0) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const uint32_t at = o_at + lanes + half * 64 + 32 * c;
                        uint32_t o[32];
                        tc::tmem_load(o, at);
                        tc::tmem_loaded();
                        tc::settle(o);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * down);
                        tc::tmem_store(at, o);
                    }
                }
            }
            const float off = m == -INFINITY ? 0.0f : kLift - m;
            const Two by2 = two(by, by), off2 = two(off, off);
            Two sum[2] = {zero(), zero()};
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                if (blind[c]) {
                    const uint32_t none[16] = {};
                    tc::tmem_store16(own_at + 16 * c, none);
                    continue;
                }
                uint32_t s[32], w[16];
                tc::tmem_load(s, own_at + 32 * c);
                tc::tmem_loaded();
                tc::settle(s);
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    const Two raw = two(__uint_as_float(s[e]), __uint_as_float(s[e + 1]));
                    const float2 x = one(MOD ? raw + off2 : fma(raw, by2, off2));
                    const float p0 = tc::exp2_fast(x.x), p1 = tc::exp2_fast(x.y);
                    sum[(e / 2) & 1] = sum[(e / 2) & 1] + two(p0, p1);
                    w[e / 2] = tc::pack<BF16>(p0, p1);
                }
                tc::tmem_store16(own_at + 16 * c, w);  // over scores that this thread is done with
            }
            const float2 sums = one(sum[0] + sum[1]);
            l += sums.x + sums.y;
            if (j0 < reach.all_lo || j0 + kKeys - 1 > reach.all_hi) {  // hidden from some row: no junk may reach the product
                if (ok && !tc::bar_wait(v_full + 8 * st, (i / Tile::kStages) & 1)) dead = 1;
                scan_tile<BF16, kKeys, DP, 32 * kWarps>(p, pos, v_tiles + st * Tile::kTile, j0, tid, junk, i, [] {});
                __syncwarp();
                tc::writes_to_async();
            }
            tc::tmem_stored();
            tc::fence_before();
            tc::bar_arrive(p_full);
        }
        if (kHalves == 2) halves[n & 1][half][own_row] = l;
    }
    __syncthreads();
    // Products and copies under way end before the CTA gives up its memory.  Where no wait gave up, products have waited for all copies,
    // and whoever reads the accumulators waits for the last product.
    if (dead && warp == kWarps + 1 && !ended) tc::bar_wait(o_done, (n - 1) & 1);
    if (dead && warp == kWarps && lane == 0) {
        tc::bar_wait(q_full, 0);
        for (int i = max(0, issued_k - Tile::kStages); i < issued_k; ++i) tc::bar_wait(k_full + 8 * (i % Tile::kStages), (i / Tile::kStages) & 1);
        for (int i = max(0, issued_v - Tile::kStages); i < issued_v; ++i) tc::bar_wait(v_full + 8 * (i % Tile::kStages), (i / Tile::kStages) & 1);
    }
    float* const extra = reinterpret_cast<float*>(k_tiles);  // [128][DP], over the tiles of keys and values
    static_assert(128 * DP * 4 <= 2 * Tile::kStages * Tile::kTile, "fits");
    const bool add = junk.any && !dead;
    if (add) {
        if (warp < kWarps) {
            if (!tc::bar_wait(o_done, (n - 1) & 1)) atomicAdd(&g_timeouts, 1u);
            add_junk<false, 128 / kWarps, DP, kKeys>(p, junk, reach, walk, n, a.v, b, hk, 1, extra, warp, lane);
        }
        __syncthreads();
    }
    if (dead) {
        if (tid == 0) atomicAdd(&g_timeouts, 1u);
    } else if (warp < kWarps) {
        const uint32_t lanes = (uint32_t)quarter << 21;
        if (kHalves == 2) l += halves[n & 1][kHalves - 1 - half][own_row];
        const bool empty = l == 0.0f;
        const float inv = 1.0f / l;
        if (n > 0 && !tc::bar_wait(o_done, (n - 1) & 1)) atomicAdd(&g_timeouts, 1u);
        tc::fence_after();
#pragma unroll
        for (int k = 0; k < 2; ++k) {  // each half has 64 of the columns
            const int c = half * 2 + k;
            uint32_t o[32];
            if (n > 0) {
                tc::tmem_load(o, o_at + lanes + 32 * c);
                tc::tmem_loaded();
                tc::settle(o);
            }
            float x[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = empty || n == 0 ? 0.0f : __uint_as_float(o[e]) * inv;
            if (add && !empty)
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] += extra[own_row * DP + 32 * c + e];
            stage_columns<BF16>(q_tile + (c / 2) * (128 * 128), own_row, (c % 2) * 32, x);
        }
        tc::writes_to_async();
        __syncwarp();
        if (lane == 0 && half * 64 < p.d && i0 + quarter * 32 < p.t) {  // the 32 rows by 64 columns that this warp has staged
            tc::tensor_store(&maps.out, half * 64, i0 + quarter * 32, h, b, tc::smem_of(q_tile) + half * (128 * 128) + quarter * 32 * 128);
            tc::stores_read();
        }
        if (half == 0 && p.lse && row < p.t)
            p.lse[((int64_t)b * p.heads + h) * p.t + row] = empty ? -INFINITY : (m + (log2f(l) - kLift)) * kLn2;
    }
    tc::fence_before();
    __syncthreads();
    if (warp == kWarps + 1) tc::tmem_free<Tile::kTmem>(tmem);
}

// ---- gradients ----------------------------------------------------------------------------------------------------

struct GradMaps {
    CUtensorMap a1, a2;  // the CTA's own rows: boxes of 128 rows.  q, dout | k, v
    CUtensorMap b1, b2;  // what streams by: boxes of kColumns.     k, v    | q, dout
    CUtensorMap b2_first;  // fp16: b2 in boxes of 128 rows by 8 elements
};

// Tiles of 128 columns and all of the tensor memory; for heads of at most 64 elements, tiles of 64 and half of it: then two CTAs
// share an SM, and one's first copies and last stores run under the other's products (16 x 1000 frames of features in fp16 232 us,
// in the instance for 128, half zeros, 333; one sequence of 16,384 in bf16 1,045 here and 806 there).
template <int DP>
struct GradTile {
    static constexpr int kColumns = DP;                             // of a tile: rows of B1 and B2
    static constexpr int kWarps = kColumns / 8;                     // with the arithmetic: 32 rows by 32 columns each
    static constexpr int kThreads = 32 * kWarps + 64;               // then a warp for copies, a warp for products
    static constexpr int kTmem = 2 * DP + 2 * kColumns;             // two accumulators, S, dP
    static constexpr int kStages = DP == 64 ? 4 : 2;
    static constexpr int kOwn = 128 * DP * 2, kStream = kColumns * DP * 2;
    static constexpr int kShared = 2 * kOwn + kStages * 2 * kStream + 1024;
    static_assert(kTmem == 256 || kTmem == 512, "a power of two");
};

// Both gradient kernels keep two tiles of 128 rows (A1, A2) and let pairs of tiles (B1, B2) stream by:
//     S = A1 B1^T, dP = A2 B2^T,   P = exp(score(S) - lse),   dS = P (dP - delta) inner,
//     acc1 += dS B1,               acc2 += P B2 (KEYS) or (P inner) B1 (queries)
// KEYS: rows are keys, acc1 = dk, acc2 = dv, streamed over the query heads that share them; lse and delta belong to columns.
// Queries: acc1 = dq; lse and delta belong to rows.  delta = sum_j P_ij dP_ij is first taken as dout . out with the rounded out
// of the forward call; the row sum eps of P (dP - delta) over the walk is exactly what that is off by, so delta + eps goes to
// the second kernel, and for rows that see at most kExact columns, few of which share the error, dq is corrected by
// -eps * sum_j P_ij inner k_j.  acc2 holds that sum, over the tiles that such a row of the CTA may reach (a row sees itself, so they
// lie within kExact of the CTA's rows), if it has one: what a row gets does not depend on what else is in its CTA.  With a distance
// bias few keys have the weight however many a row sees, and all rows are corrected.  (All rows always: 4 x 4096 tokens 503 -> 521 us,
// one sequence of 16,384 822 -> 894.)
//
// P lies over S and dS over dP, and the products take turns: ..., acc2(n), S(n + 1), acc1(n), dP(n + 1), acc2(n + 1), ...  While
// acc1(n) and dP(n + 1) run, P(n + 1) is made from S(n + 1); while acc2 and the next S run, dS from dP.  (Two groups of warps with
// tiles of 64 columns each, taking turns, kept the tensor cores at 41 %: with 64 columns a product reads 192 bytes of shared
// memory per cycle where there are 128, and what it reads of A serves half as many columns.)
constexpr int kExact = 1024;

// fp16: P is made 2^14 times as large (its rows' sums are 1, so none is much above 1), and each row of dS is multiplied by 2^14 and a
// power of two of its own, `lift`, so that 2^14 lift max|dout| max|v| is between 2^9 and 2^10 over the first eight elements of both at the row's
// own slot (for a key: dout of the first head that shares it): every row sees itself, and vectors of like elements have no dS above
// 2^15 then.  Terms are off by 2^-34 of that product where they do not have fp16's 11 bits; without a scale a row of 4,000 keys and
// dout of 1e-2 has dS of 2e-6, which is 32 steps of fp16, and one above 65,504 was infinite.  Where a row's dS do not fit all the
// same, its acc1 comes out infinite or NaN, and the CTA walks AGAIN, twice: to find such rows' largest dS, and with a lift
// from that (rows that fit keep theirs, and their bits): so do keys whose own slot has no dout at all.  The gradient of 4 x 4096 tokens takes 519 us (without lifts 505), of 16 x 1000
// frames of features 232 (214); to agree on a row's lift among its warps in every tile took 574 and 257.
constexpr float kLiftP = 16384.0f;
constexpr int kOneWalk = 0, kMeasure = 1, kLastWalk = 2;
__device__ __forceinline__ float power_of_two(int exponent) { return __int_as_float((exponent + 127) << 23); }
__device__ __forceinline__ int exponent_of(float x) { return (__float_as_int(x) >> 23) - 127; }  // x >= 0; 128 for infinities and NaN

// The 32 rows by 32 columns (from `first` on, `column` in the tile) that a warp has staged, to memory: 16 bytes per lane, side by side.
// At one CTA per SM that is 400 to 600 cycles less than a tensor store, whose reads the CTA has to see the end of; the forward
// kernel, whose CTAs hide each other's ends, is slower for it (features 65 -> 70 us).
template <typename T>
__device__ __forceinline__ void store_staged(const uint8_t* tile, int own_row0, int column, const AttnParams& p, const Heads<T>& out, int b, int h,
                                             int row0, int first, int lane)
{
    const int c = lane % 4;
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int r = k * 8 + lane / 4;
        if (first + c * 8 < p.d && row0 + r < p.t)
            *reinterpret_cast<uint4*>(out.at(b, row0 + r, h) + first + c * 8) =
                *reinterpret_cast<const uint4*>(tile + (own_row0 + r) * 128 + (((column / 8 + c) ^ (r & 7)) * 16));
    }
    __syncwarp();
}

template <bool BF16, int DP, bool KEYS>
struct GradShared {
    static constexpr int kColumns = GradTile<DP>::kColumns;
    alignas(128) uint4 b2_first[BF16 ? 1 : 128];  // eight elements of B2's tensor at each row's own slot
    float4 column_stats[KEYS ? GradTile<DP>::kWarps : 1][KEYS ? 16 : 1];  // per warp: -lse (log2 units) and -delta of 16 pairs of columns
    uint64_t bars[8 + 4 * GradTile<DP>::kStages];
    uint32_t tmem_base;
    int dead, again, stuck;
    Junk<kColumns> junk;
    ReachShared<4> reach;
    float eps[kColumns / 32][128], delta[KEYS ? 1 : 128];
    float tops[BF16 ? 1 : kColumns / 32][BF16 ? 1 : 128];  // per 32 columns and row: the largest of dS * lift
};

// All of k30_attention_grad; true if the CTA has to walk AGAIN (fp16: see kLiftP).
template <bool BF16, int DP, bool MOD, bool KEYS, bool AGAIN>
__device__ __forceinline__ bool attention_grad(const AttnParams& p, const AttnTensors<typename Element<BF16>::type>& a, const GradMaps& maps,
                                               GradShared<BF16, DP, KEYS>& sh)
{
    using Tile = GradTile<DP>;
    constexpr int kColumns = Tile::kColumns, kWarps = Tile::kWarps, kStages = Tile::kStages;
    extern __shared__ uint8_t raw[];
    int &dead = sh.dead, &again = sh.again, &stuck = sh.stuck;
    auto& junk = sh.junk;
    auto& column_stats = sh.column_stats;
    auto& eps_shared = sh.eps;
    auto& delta_shared = sh.delta;
    auto& tops = sh.tops;

    uint8_t* const tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* const a1 = tiles;
    uint8_t* const a2 = tiles + Tile::kOwn;
    uint8_t* const stream = tiles + 2 * Tile::kOwn;  // per stage: B1, B2
    const uint32_t bar0 = tc::smem_of(sh.bars);
    const uint32_t a_full = bar0, s_full = bar0 + 8, dp_full = bar0 + 16, p_full = bar0 + 24, ds_full = bar0 + 32, acc1_done = bar0 + 40,
                   acc2_done = bar0 + 48, b1_full = bar0 + 56, b2_full = b1_full + 8 * kStages, b1_free = b2_full + 8 * kStages,
                   b2_free = b1_free + 8 * kStages, given_up = b2_free + 8 * kStages;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int own_heads = KEYS ? p.kv_heads : p.heads;
    const int own_tiles = (p.t + 127) / 128;
    const int64_t bh = blockIdx.x % (p.blocks * own_heads);
    const int turn = (int)(blockIdx.x / (p.blocks * own_heads));
    const int r0 = (KEYS ? turn : own_tiles - 1 - turn) * 128;  // the longest walks of a long sequence first
    const int h = (int)(bh % own_heads), b = (int)(bh / own_heads);
    const int32_t* const pos = p.pos + (int64_t)b * p.t;
    const int part = warp >> 2, quarter = warp & 3;  // of the arithmetic's warps: which 32 columns, which 32 rows
    const int own_row = quarter * 32 + lane, row = r0 + own_row;

    // the tile B1 or B2 of head hs from slot j0 on, to stage s
    auto load = [&](bool one, int s, int j0, int hs) {
        const uint32_t bar = (one ? b1_full : b2_full) + 8 * s, to = tc::smem_of(stream) + (2 * s + (one ? 0 : 1)) * Tile::kStream;
        tc::bar_expect(bar, Tile::kStream);
        for (int x = 0; x < DP; x += 64) tc::tensor_load(to + x * (2 * kColumns), one ? &maps.b1 : &maps.b2, x, j0, hs, b, bar);
    };
    const int first_head = KEYS ? h * p.group : h / p.group;  // of the other side
    auto begin = [&] {  // by one thread: barriers, and the copies that need no positions
        if (AGAIN)
            for (int k = 0; k < 8 + 4 * kStages; ++k) tc::bar_inval(bar0 + 8 * k);
        tc::bar_init(a_full, 1);
        tc::bar_init(s_full, 1);
        tc::bar_init(dp_full, 1);
        tc::bar_init(p_full, 32 * kWarps);
        tc::bar_init(ds_full, 32 * kWarps);
        tc::bar_init(acc1_done, 1);
        tc::bar_init(acc2_done, 1);
        for (int s = 0; s < 4 * kStages; ++s) tc::bar_init(b1_full + 8 * s, 1);
        tc::bar_init(given_up, 1);
        tc::bar_init_done();
        tc::bar_expect(a_full, 2 * Tile::kOwn + (BF16 ? 0 : 128 * 16));
        if (!BF16) tc::tensor_load(tc::smem_of(sh.b2_first), &maps.b2_first, 0, r0, first_head, b, a_full);
        for (int x = 0; x < DP; x += 64) {
            tc::tensor_load(tc::smem_of(a1) + x * 256, &maps.a1, x, r0, h, b, a_full);
            tc::tensor_load(tc::smem_of(a2) + x * 256, &maps.a2, x, r0, h, b, a_full);
        }
        if (p.causal) {
            const int j0 = Walk<kColumns>::causal_first(p, r0, KEYS);
            load(true, 0, j0, first_head);
            load(false, 0, j0, first_head);
        }
    };
    Span span{kNever, -1};
    float own_lse = 0.0f;  // queries: of this row
    // dout . out of the queries: DP / 8 lanes share a row, 16 bytes each, so that a load of a warp touches few lines (with a row per
    // lane it was 32 each, and the rows were known after 4 us instead of 1.4)
    using E = typename Element<BF16>::type;
    constexpr int kSumLanes = DP / 8, kSumRows = kWarps * 32 / kSumLanes, kPasses = KEYS ? 1 : 128 / kSumRows;
    const int sum_row = warp * (32 / kSumLanes) + lane / kSumLanes, sum_chunk = lane % kSumLanes;
    uint4 out_part[kPasses] = {};
    if (warp < kWarps) {
        if (!KEYS) {  // under way while the rows look for their columns
            if (row < p.t) own_lse = p.lse[((int64_t)b * p.heads + h) * p.t + row];
#pragma unroll
            for (int k = 0; k < kPasses; ++k) {
                const int r = r0 + sum_row + k * kSumRows;
                if (r < p.t && sum_chunk * 8 < p.d) out_part[k] = *reinterpret_cast<const uint4*>(a.out_in.at(b, r, h) + sum_chunk * 8);
            }
        }
        span = span_of(p, pos, row, KEYS, lane);
        if (part == 0) {
            put_reach(sh.reach, quarter, lane, span);
            junk.spans[own_row] = span;
            if (tid < (int)(sizeof junk.tiles / 4)) junk.tiles[tid] = 0;
        }
        if (tid == 0) {
            dead = junk.any = stuck = 0;
            again = AGAIN;
        }
    } else if (warp == kWarps) {
        if (lane == 0) begin();  // under way while the rows look for their columns
    } else if (!AGAIN) {
        tc::tmem_alloc<Tile::kTmem>(tc::smem_of(&sh.tmem_base));
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = sh.tmem_base, acc1_at = tmem, acc2_at = tmem + DP, s_at = tmem + 2 * DP, dp_at = s_at + kColumns;
    const Reach reach = get_reach(sh.reach);
    const Walk<kColumns> walk(p, reach, r0, KEYS);
    const int per_head = walk.count(reach);
    const int n = KEYS ? per_head * p.group : per_head;
    const int exact = MOD && p.slopes ? p.t : kExact;
    const bool second = KEYS || reach.least <= exact;  // acc2 is kept
    auto kept = [&](int j0) {  // for the tile from column j0 on
        return KEYS || second && j0 + kColumns > r0 - (exact - 1) && j0 <= r0 + 127 + (exact - 1);
    };
    float delta = 0.0f, lift = 1.0f;
    int issued1, issued2;  // (warp of the copies)
    bool ended;            // (warp of the products) none are under way

    for (int pass = AGAIN ? kMeasure : kOneWalk;; ++pass) {
        issued1 = issued2 = p.causal;
        ended = false;
        if (warp == kWarps) {
            if (lane == 0) {
                bool ok = true;
                if (n == 0) ok = tc::bar_wait(a_full, 0) && (!p.causal || (tc::bar_wait(b1_full, 0) && tc::bar_wait(b2_full, 0)));  // (copies end)
                for (int i = p.causal; i < n; ++i) {
                    const int s = i % kStages;
                    const uint32_t parity = (i / kStages + 1) & 1;
                    const int j0 = walk(KEYS ? i % per_head : i), hs = KEYS ? first_head + i / per_head : first_head;
                    if (!(ok = tc::bar_wait(b1_free + 8 * s, parity))) break;
                    load(true, s, j0, hs);
                    issued1 = i + 1;
                    if (!(ok = tc::bar_wait(b2_free + 8 * s, parity))) break;
                    load(false, s, j0, hs);
                    issued2 = i + 1;
                }
                if (!ok) dead = 1;
            }
        } else if (warp == kWarps + 1) {
            ended = true;
            if (n > 0) {
                ended = false;
                const uint32_t leader = tc::elect();
                auto all = [](bool x) { return (bool)__all_sync(0xffffffffu, x); };
                bool ok = all(tc::bar_wait(a_full, 0));
                uint32_t turns2 = 0;  // tiles kept so far
                for (int i = 0; i <= n && ok; ++i) {  // acc2(i - 1), S(i), acc1(i - 1), dP(i)
                    const int s = i % kStages, sl = (i + kStages - 1) % kStages;
                    const uint32_t at = tc::smem_of(stream) + s * 2 * Tile::kStream, last = tc::smem_of(stream) + sl * 2 * Tile::kStream;
                    const bool last_kept = i > 0 && kept(walk(i - 1));
                    if (last_kept) {
                        if (!(ok = all(tc::bar_wait(p_full, (i - 1) & 1)))) break;
                        tc::fence_after();
                        tc::product_across<BF16, kColumns, DP, 32>(leader, acc2_at, s_at, KEYS ? last + Tile::kStream : last, KEYS ? i > 1 : turns2 > 0);
                        ++turns2;
                        // (nothing arrives that nobody waits for: here and below, stages that no copy takes again, ends that no product needs)
                        if (KEYS && i - 1 + kStages < n) tc::products_arrive(leader, b2_free + 8 * sl);
                        if (i < n) tc::products_arrive(leader, acc2_done);
                    }
                    if (i < n) {
                        // S's place is free when the product is over that reads the last P there, or when the last S has been read
                        if (!(ok = all(tc::bar_wait(b1_full + 8 * s, (i / kStages) & 1) &&
                                       (i == 0 || tc::bar_wait(last_kept ? acc2_done : p_full, (last_kept && !KEYS ? turns2 - 1 : i - 1) & 1)))))
                            break;
                        tc::fence_after();
                        tc::product_rows<BF16, kColumns, DP>(leader, s_at, tc::smem_of(a1), at);
                        tc::products_arrive(leader, s_full);
                    }
                    if (i > 0) {
                        if (!(ok = all(tc::bar_wait(ds_full, (i - 1) & 1)))) break;
                        tc::fence_after();
                        tc::product_across<BF16, kColumns, DP, 32>(leader, acc1_at, dp_at, last, i > 1);
                        if (i - 1 + kStages < n) tc::products_arrive(leader, b1_free + 8 * sl);
                        tc::products_arrive(leader, acc1_done);
                    }
                    if (i < n) {
                        if (!(ok = all(tc::bar_wait(b2_full + 8 * s, (i / kStages) & 1) && (i == 0 || tc::bar_wait(acc1_done, (i - 1) & 1))))) break;
                        tc::fence_after();
                        tc::product_rows<BF16, kColumns, DP>(leader, dp_at, tc::smem_of(a2), at + Tile::kStream);
                        if (!KEYS && i + kStages < n) tc::products_arrive(leader, b2_free + 8 * s);
                        tc::products_arrive(leader, dp_full);
                    }
                }
                if (!ok) {
                    dead = 1;
                    tc::products_arrive(leader, given_up);
                    tc::bar_wait(given_up, 0);
                    ended = true;
                }
            }
        } else {
            const uint32_t lanes = (uint32_t)quarter << 21;
            Two lse2 = zero(), eps2 = zero();  // lse and delta of this row, negative
            constexpr float kUp = BF16 ? 0.0f : 14.0f;  // log2 kLiftP
            if (!KEYS && row < p.t) {          // this row's statistics
                const float lse = minus_lse(own_lse) + kUp;
                lse2 = two(lse, lse);
            }
            if ((!KEYS || !BF16) && pass != kLastWalk) {
                if (!tc::bar_wait(a_full, 0)) dead = 1;
                if (!BF16) {
                    const uint4 own = *reinterpret_cast<const uint4*>(a2 + own_row * 128 + (own_row & 7) * 16);  // dout, or v
                    lift = power_of_two(-5 - min(max(exponent_of(tc::largest_of_halves(own) * tc::largest_of_halves(sh.b2_first[BF16 ? 0 : own_row])), -64), 64));
                }
            }
            if (!KEYS && pass != kLastWalk) {
#pragma unroll
                for (int k = 0; k < kPasses; ++k) {
                    const int r = sum_row + k * kSumRows;
                    const uint4 dout = *reinterpret_cast<const uint4*>(a2 + sum_chunk / 8 * (128 * 128) + r * 128 + ((sum_chunk % 8) ^ (r & 7)) * 16);
                    float sum = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        sum = fmaf(to_float(reinterpret_cast<const E*>(&out_part[k])[e]), to_float(reinterpret_cast<const E*>(&dout)[e]), sum);
#pragma unroll
                    for (int o = 1; o < kSumLanes; o *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    if (sum_chunk == 0) delta_shared[KEYS ? 0 : r] = sum;
                }
                asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory");  // of the warps with the arithmetic
                delta = delta_shared[KEYS ? 0 : own_row];
            }
            const Two delta2 = two(-delta, -delta);
            // Junk in a tile that is hidden from some row must not reach the products across it.  (B1 is scanned when S is done, which reads
            // it; B2 while dP may still read it, so whoever has something to clear waits for dP's end, which waits for nothing of this turn.
            // A query with junk in dout has NaN for its delta, so its dS are NaN whatever dP reads.)
            auto scan = [&](uint32_t full, int i, int which, int j0) {
                if (j0 >= reach.all_lo && j0 + kColumns - 1 <= reach.all_hi) return;
                if (!tc::bar_wait(full + 8 * (i % kStages), (i / kStages) & 1)) dead = 1;
                scan_tile_apart<BF16, kColumns, DP, 32 * kWarps>(p, pos, stream + ((i % kStages) * 2 + which) * Tile::kStream, j0, tid, junk,
                                                                 KEYS ? i % per_head : i, which ? dp_full : 0, i & 1, dead);
                __syncwarp();
                tc::writes_to_async();
            };
            // KEYS: statistics of this warp's 32 columns of tile i, a tile ahead
            float next_lse = 0.0f, next_delta = 0.0f;
            auto fetch = [&](int i) {
                const int column = walk(i % per_head) + 32 * part + lane;
                const int64_t at = ((int64_t)b * p.heads + first_head + i / per_head) * p.t + column;
                next_lse = column < p.t ? p.lse[at] : 0.0f;
                next_delta = column < p.t ? p.delta[at] : 0.0f;
            };
            if (KEYS && n > 0) fetch(0);
            float top = 0.0f;  // kMeasure
            for (int i = 0; i < n; ++i) {
                const int j0 = walk(KEYS ? i % per_head : i), mine0 = j0 + 32 * part;  // the tile's and this warp's first column
                const Modifier modify(p, KEYS ? first_head + i / per_head : h);
                if (KEYS) {
                    __syncwarp();
                    float* const st = reinterpret_cast<float*>(&column_stats[KEYS ? warp : 0][KEYS ? lane / 2 : 0]) + (lane & 1);
                    st[0] = minus_lse(next_lse) + kUp;
                    st[2] = -next_delta;
                    __syncwarp();
                    if (i + 1 < n) fetch(i + 1);
                }
                const bool keep = kept(j0), clear = __all_sync(0xffffffffu, span.lo <= mine0 && span.hi >= mine0 + 31);
                const uint32_t mask = clear ? 0xffffffffu : column_mask(span.lo - mine0, span.hi - mine0);
                if (!__all_sync(0xffffffffu, tc::bar_wait(s_full, i & 1))) {
                    dead = 1;
                    break;
                }
                tc::fence_after();
                if (__all_sync(0xffffffffu, mask == 0)) {  // nothing of this block of 32 x 32 is seen
                    const uint32_t none[16] = {};
                    if (keep) {
                        tc::tmem_store16(s_at + lanes + 32 * part, none);
                        scan(KEYS ? b2_full : b1_full, i, KEYS ? 1 : 0, j0);
                        tc::tmem_stored();
                        tc::fence_before();
                    }
                    tc::bar_arrive(p_full);
                    if (!__all_sync(0xffffffffu, tc::bar_wait(dp_full, i & 1))) {
                        dead = 1;
                        break;
                    }
                    tc::fence_after();
                    tc::tmem_store16(dp_at + lanes + 32 * part, none);
                    if (KEYS || !keep) scan(b1_full, i, 0, j0);
                    tc::tmem_stored();
                    tc::fence_before();
                    tc::bar_arrive(ds_full);
                    continue;
                }
                float w[32], in[MOD ? 32 : 1];  // P, inner
                {
                    uint32_t s[32];
                    tc::tmem_load(s, s_at + lanes + 32 * part);
                    tc::tmem_loaded();
                    tc::settle(s);
                    if (!keep) {  // S has been read
                        tc::fence_before();
                        tc::bar_arrive(p_full);
                    }
                    const Two by2 = two(modify.by, modify.by);
                    const float apart = (float)(row - mine0);
                    if (MOD)
                        Modifier::with(modify.kind(s), [&](auto kind) {
#pragma unroll
                            for (int e = 0; e < 32; e += 2) {
                                Two inner;
                                const float2 x = one(modify.apply<decltype(kind)::value>(two(__uint_as_float(s[e]), __uint_as_float(s[e + 1])),
                                                                                         apart - (float)e, inner));
                                s[e] = __float_as_uint(x.x);
                                s[e + 1] = __float_as_uint(x.y);
                                in[MOD ? e : 0] = one(inner).x;
                                in[MOD ? e + 1 : 0] = one(inner).y;
                            }
                        });
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        Two lse_here = lse2;
                        if (KEYS) {
                            const float2 l = *reinterpret_cast<const float2*>(&column_stats[KEYS ? warp : 0][KEYS ? e / 2 : 0]);
                            lse_here = two(l.x, l.y);
                        }
                        const Two raw = two(__uint_as_float(s[e]), __uint_as_float(s[e + 1]));
                        const float2 x = one(MOD ? raw + lse_here : fma(raw, by2, lse_here));
                        w[e] = tc::exp2_fast(x.x);
                        w[e + 1] = tc::exp2_fast(x.y);
                    }
                }
                if (!clear) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        w[e] = (mask >> e) & 1 ? w[e] : 0.0f;
                        if (MOD) in[MOD ? e : 0] = (mask >> e) & 1 ? in[MOD ? e : 0] : 0.0f;
                    }
                }
                if (keep) {
                    uint32_t pw[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 2)
                        pw[e / 2] = MOD && !KEYS ? tc::pack<BF16>(w[e] * in[MOD ? e : 0], w[e + 1] * in[MOD ? e + 1 : 0]) : tc::pack<BF16>(w[e], w[e + 1]);
                    tc::tmem_store16(s_at + lanes + 32 * part, pw);  // over the scores they were made from
                    if (MOD && KEYS)
#pragma unroll
                        for (int e = 0; e < 32; ++e) w[e] *= in[MOD ? e : 0];  // (only together from here on)
                    scan(KEYS ? b2_full : b1_full, i, KEYS ? 1 : 0, j0);
                    tc::tmem_stored();
                    tc::fence_before();
                    tc::bar_arrive(p_full);
                }
                if (!BF16) {  // (while dP is made)
                    const Two lift2 = two(lift, lift);
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        const float2 x = one(two(w[e], w[e + 1]) * lift2);
                        w[e] = x.x;
                        w[e + 1] = x.y;
                    }
                }
                if (!__all_sync(0xffffffffu, tc::bar_wait(dp_full, i & 1))) {
                    dead = 1;
                    break;
                }
                tc::fence_after();
                // f(e, dS of columns e and e + 1, before `inner` if that is kept apart)
                // (with a cap and rows of queries, two numbers per column wait for dP already: it is read in halves then, for registers)
                constexpr int kAtOnce = MOD && !KEYS ? 16 : 32;
                auto score_gradients = [&](const auto& f) {
#pragma unroll
                    for (int c = 0; c < 32; c += kAtOnce) {
                        uint32_t d[kAtOnce];
                        tc::tmem_load(d, dp_at + lanes + 32 * part + c);
                        tc::tmem_loaded();
                        tc::settle(d);
#pragma unroll
                        for (int k = 0; k < kAtOnce; k += 2) {
                            const int e = c + k;
                            Two delta_here = delta2;
                            if (KEYS) {
                                const float2 l = *(reinterpret_cast<const float2*>(&column_stats[KEYS ? warp : 0][KEYS ? e / 2 : 0]) + 1);
                                delta_here = two(l.x, l.y);
                            }
                            Two g = two(__uint_as_float(d[k]), __uint_as_float(d[k + 1])) + delta_here;
                            if (!clear) g = two((mask >> e) & 1 ? one(g).x : 0.0f, (mask >> (e + 1)) & 1 ? one(g).y : 0.0f);  // (may be NaN)
                            f(e, two(w[e], w[e + 1]) * g);
                        }
                    }
                };
                if (!BF16 && __builtin_expect(pass == kMeasure, 0))
                    score_gradients([&](int e, Two g) {
                        if (MOD && !KEYS) g = g * two(in[MOD ? e : 0], in[MOD ? e + 1 : 0]);
                        const float most = tc::largest(0.0f, one(g).x, one(g).y);
                        top = most <= 3.0e38f ? fmaxf(top, most) : top;
                    });
                uint32_t dw[16];
                score_gradients([&](int e, Two g) {
                    if (!KEYS) {
                        eps2 = eps2 + g;
                        if (MOD) g = g * two(in[MOD ? e : 0], in[MOD ? e + 1 : 0]);
                    }
                    dw[e / 2] = tc::pack<BF16>(one(g).x, one(g).y);
                });
                tc::tmem_store16(dp_at + lanes + 32 * part, dw);
                if (KEYS || !keep) scan(b1_full, i, 0, j0);
                tc::tmem_stored();
                tc::fence_before();
                tc::bar_arrive(ds_full);
            }
            if (!KEYS) eps_shared[part][own_row] = (one(eps2).x + one(eps2).y) * (1.0f / lift);
            if (!BF16) tops[BF16 ? 0 : part][BF16 ? 0 : own_row] = top;
            if (!BF16 && !AGAIN && part == 0 && n > 0) {  // one column tells: infinity times anything is not finite
                if (!tc::bar_wait(acc1_done, (n - 1) & 1)) stuck = 1;  // (the end counts it)
                tc::fence_after();
                uint32_t x = tc::tmem_load1(acc1_at + lanes);
                tc::tmem_loaded();
                tc::settle(x);
                if (span.lo <= span.hi && (x & 0x7f800000u) == 0x7f800000u && (KEYS || isfinite(delta))) again = 1;
                tc::fence_before();
            }
        }
        __syncthreads();
        if (BF16 || dead || (!AGAIN && stuck) || !again || pass == kLastWalk) break;
        if (!AGAIN) return true;
        if (warp < kWarps) {
            if (!tc::bar_wait(acc1_done, (n - 1) & 1)) stuck = 1;
            float most = 0.0f;
            for (int k = 0; k < kColumns / 32; ++k) most = fmaxf(most, tops[BF16 ? 0 : k][BF16 ? 0 : own_row]);
            if (most > 65000.0f) lift *= power_of_two(14 - exponent_of(most));
        }
        __syncthreads();
        if (stuck) break;
        if (warp == kWarps && lane == 0) begin();
        __syncthreads();
        tc::fence_after();
    }
    // (as in the forward kernel: what is under way ends before the CTA gives up its memory)
    if (dead && warp == kWarps + 1 && !ended) tc::bar_wait(acc1_done, (n - 1) & 1);
    if (dead && warp == kWarps && lane == 0) {
        tc::bar_wait(a_full, 0);
        for (int i = max(0, issued1 - kStages); i < issued1; ++i) tc::bar_wait(b1_full + 8 * (i % kStages), (i / kStages) & 1);
        for (int i = max(0, issued2 - kStages); i < issued2; ++i) tc::bar_wait(b2_full + 8 * (i % kStages), (i / kStages) & 1);
    }
    float* const extra = reinterpret_cast<float*>(stream);  // [128][DP], KEYS: of dk, then of dv; over the stream's tiles
    static_assert((KEYS ? 2 : 1) * 128 * DP * 4 <= kStages * 2 * Tile::kStream, "fits");
    const bool add = junk.any && !dead;
    if (add) {  // dS times an infinite element: its sign would be that of dS, and q.k is not finite either; NaN
        if (warp < kWarps) {
            if (!tc::bar_wait(acc1_done, (n - 1) & 1)) atomicAdd(&g_timeouts, 1u);
            add_junk<true, 128 / kWarps, DP, kColumns>(p, junk, reach, walk, per_head, KEYS ? a.q : a.k, b, first_head, KEYS ? p.group : 1, extra, warp, lane);
            if (KEYS)
                add_junk<false, 128 / kWarps, DP, kColumns>(p, junk, reach, walk, per_head, a.dout, b, first_head, p.group, extra + 128 * DP, warp, lane);
        }
        __syncthreads();
    }
    if (dead) {
        if (tid == 0) atomicAdd(&g_timeouts, 1u);
    } else if (warp < kWarps) {
        const uint32_t lanes = (uint32_t)quarter << 21;
        const bool empty = span.lo > span.hi, few = !KEYS && second && span.hi - span.lo < exact;
        if (n > 0 && !tc::bar_wait(acc1_done, (n - 1) & 1)) atomicAdd(&g_timeouts, 1u);
        tc::fence_after();
        const float undo_p = BF16 ? 1.0f : 1.0f / kLiftP, undo = BF16 ? 1.0f : undo_p / lift;  // powers of two
        float off = 0.0f;
        if (!KEYS) {
            for (int k = 0; k < kColumns / 32; ++k) off += eps_shared[k][own_row];
            off *= undo_p;
            if (part == 0 && row < p.t) p.delta[((int64_t)b * p.heads + h) * p.t + row] = empty ? 0.0f : delta + off;
        }
        // chunks of 32 columns of dq, or of dk and then dv, are shared out among the warps of a row
#pragma unroll
        for (int k = part; k < (KEYS ? 2 : 1) * DP / 32; k += kColumns / 32) {
            const bool dv = KEYS && k >= DP / 32;
            const int c = dv ? k - DP / 32 : k;
            uint32_t o[32], o2[32] = {};
            if (n > 0) {
                tc::tmem_load(o, (dv ? acc2_at : acc1_at) + lanes + 32 * c);
                if (!KEYS && second) tc::tmem_load(o2, acc2_at + lanes + 32 * c);
                tc::tmem_loaded();
                tc::settle(o);
                tc::settle(o2);
            }
            float x[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                float y = __uint_as_float(o[e]) * (dv ? undo_p : undo);
                if (few) y = fmaf(-off, __uint_as_float(o2[e]) * undo_p, y);
                x[e] = empty || n == 0 ? 0.0f : y * (dv ? 1.0f : p.scale);
            }
            if (add && !empty)
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] += extra[(dv ? 128 * DP : 0) + own_row * DP + 32 * c + e];
            uint8_t* const tile = (dv ? a2 : a1) + (c / 2) * (128 * 128);
            stage_columns<BF16>(tile, own_row, (c % 2) * 32, x);
            store_staged(tile, quarter * 32, (c % 2) * 32, p, !KEYS ? a.dq : dv ? a.dv : a.dk, b, h, r0 + quarter * 32, 32 * c, lane);
        }
    }
    tc::fence_before();
    __syncthreads();
    if (warp == kWarps + 1) tc::tmem_free<Tile::kTmem>(tmem);
    return false;
}

template <bool BF16, int DP, bool MOD, bool KEYS>
__global__ void __launch_bounds__(GradTile<DP>::kThreads, DP == 64 ? 2 : 1)
    k30_attention_grad(const __grid_constant__ AttnParams p, const __grid_constant__ AttnTensors<typename Element<BF16>::type> a,
                       const __grid_constant__ GradMaps maps)
{
    __shared__ GradShared<BF16, DP, KEYS> sh;
    const bool again = attention_grad<BF16, DP, MOD, KEYS, false>(p, a, maps, sh);
    if constexpr (!BF16)  // (in line: a call here, taken or not, cost every CTA 2 us)
        if (__builtin_expect(again, 0)) (void)attention_grad<BF16, DP, MOD, KEYS, true>(p, a, maps, sh);
}

// ---- launches -----------------------------------------------------------------------------------------------------

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled()
{
    static const EncodeTiled fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<EncodeTiled>(f);
    }();
    return fn;
}

// The tensor [block, head, slot, element] with boxes of `box` slots by 64 elements: elements from d on read as zeros and are
// not written, nor are slots from t on.
template <typename P>
bool make_map(CUtensorMap* map, const AttnParams& p, bool bf16, const Heads<P>& x, int heads, int box, int elements = 64)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)p.d, (cuuint64_t)p.t, (cuuint64_t)heads, (cuuint64_t)p.blocks};
    auto bytes = [](int64_t stride) { return (cuuint64_t)(stride ? stride * 2 : 16); };  // (0: a dimension of length one)
    const cuuint64_t strides[3] = {bytes(x.slot), bytes(x.head), bytes(x.block)};
    const cuuint32_t boxes[4] = {(cuuint32_t)elements, (cuuint32_t)box, 1, 1}, steps[4] = {1, 1, 1, 1};
    return encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
                  const_cast<void*>(static_cast<const void*>(x.data)), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  elements == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool BF16, int DP, bool MOD>
cudaError_t forward(const AttnParams& p, const AttnTensors<typename Element<BF16>::type>& a, cudaStream_t st)
{
    ForwardMaps m;
    if (!make_map(&m.q, p, BF16, a.q, p.heads, 128) || !make_map(&m.k, p, BF16, a.k, p.kv_heads, ForwardTile<DP>::kKeys) ||
        !make_map(&m.v, p, BF16, a.v, p.kv_heads, ForwardTile<DP>::kKeys) || !make_map(&m.out, p, BF16, a.out, p.heads, 32))
        return cudaErrorInvalidValue;
    const int64_t grid = p.blocks * p.heads * ((p.t + 127) / 128);
    if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
    auto* kernel = k29_attention<BF16, DP, MOD>;
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t e = allow_shared(kernel, ForwardTile<DP>::kShared, allowed);
    if (e != cudaSuccess) return e;
    kernel<<<(unsigned)grid, ForwardTile<DP>::kThreads, ForwardTile<DP>::kShared, st>>>(p, a, m);
    count_launches(1);
    return cudaGetLastError();
}

template <bool BF16, int DP, bool MOD, bool KEYS>
cudaError_t gradient(const AttnParams& p, const AttnTensors<typename Element<BF16>::type>& a, cudaStream_t st)
{
    GradMaps m;
    const int own = KEYS ? p.kv_heads : p.heads, other = KEYS ? p.heads : p.kv_heads;
    const bool ok = make_map(&m.a1, p, BF16, KEYS ? a.k : a.q, own, 128) && make_map(&m.a2, p, BF16, KEYS ? a.v : a.dout, own, 128) &&
              make_map(&m.b1, p, BF16, KEYS ? a.q : a.k, other, GradTile<DP>::kColumns) &&
              make_map(&m.b2, p, BF16, KEYS ? a.dout : a.v, other, GradTile<DP>::kColumns) &&
              (BF16 || make_map(&m.b2_first, p, BF16, KEYS ? a.dout : a.v, other, 128, 8));
    const int64_t grid = p.blocks * own * ((p.t + 127) / 128);
    if (!ok || grid > 0x7fffffffLL) return cudaErrorInvalidValue;
    auto* kernel = k30_attention_grad<BF16, DP, MOD, KEYS>;
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t e = allow_shared(kernel, GradTile<DP>::kShared, allowed);
    if (e != cudaSuccess) return e;
    kernel<<<(unsigned)grid, GradTile<DP>::kThreads, GradTile<DP>::kShared, st>>>(p, a, m);
    count_launches(1);
    return cudaGetLastError();
}

template <bool BF16, int DP, bool MOD>
cudaError_t both(const AttnParams& p, const AttnTensors<typename Element<BF16>::type>& a, cudaStream_t st)
{
    const cudaError_t e = gradient<BF16, DP, MOD, false>(p, a, st);
    return e != cudaSuccess ? e : gradient<BF16, DP, MOD, true>(p, a, st);
}

}  // namespace

template <typename T>
cudaError_t launch_attention(const AttnParams& p, const AttnTensors<T>& a, cudaStream_t st)
{
    constexpr bool kBf16 = sizeof(T) == 2 && !std::is_same<T, __half>::value;
    const bool mod = p.cap > 0.0f || p.slopes || p.scale <= 0.0f;  // (without, the largest product has the largest score)
    if (p.d <= 64) return mod ? forward<kBf16, 64, true>(p, a, st) : forward<kBf16, 64, false>(p, a, st);
    return mod ? forward<kBf16, 128, true>(p, a, st) : forward<kBf16, 128, false>(p, a, st);
}
template <typename T>
cudaError_t launch_attention_grad(const AttnParams& p, const AttnTensors<T>& a, cudaStream_t st)
{
    constexpr bool kBf16 = sizeof(T) == 2 && !std::is_same<T, __half>::value;
    const bool mod = p.cap > 0.0f || p.slopes || p.scale <= 0.0f;  // (without, the largest product has the largest score)
    if (p.d <= 64) return mod ? both<kBf16, 64, true>(p, a, st) : both<kBf16, 64, false>(p, a, st);
    return mod ? both<kBf16, 128, true>(p, a, st) : both<kBf16, 128, false>(p, a, st);
}
#define BLOAD_INSTANTIATE(T)                                                                          \
    template cudaError_t launch_attention<T>(const AttnParams&, const AttnTensors<T>&, cudaStream_t); \
    template cudaError_t launch_attention_grad<T>(const AttnParams&, const AttnTensors<T>&, cudaStream_t);
BLOAD_INSTANTIATE(__half)
BLOAD_INSTANTIATE(__nv_bfloat16)
#undef BLOAD_INSTANTIATE

int64_t attention_timeouts()
{
    unsigned int v = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&v, g_timeouts, sizeof v) != cudaSuccess) {
        (void)cudaGetLastError();
        return -1;
    }
    return (int64_t)v;
}

}  // namespace bload

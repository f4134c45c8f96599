// Shared by the layers on packed batches (rotary positions, attention, recurrence): element types, the extent of a
// sequence around a slot, and the launch parameters.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "bload.h"

namespace bload {

// A tensor [block, slot, head, element] by strides in elements.
template <typename P>
struct Heads {
    P* data;
    int64_t block, slot, head;
    __host__ __device__ P* at(int64_t q, int64_t s, int64_t h) const { return data + q * block + s * slot + h * head; }
};

struct AttnParams {
    const int32_t* pos;   // [blocks, t]
    const float* slopes;  // [heads] or NULL
    float* lse;           // [blocks, heads, t] or NULL (forward only)
    float* delta;         // [blocks, heads, t] (gradient only)
    int64_t blocks;
    int32_t t, heads, kv_heads, group, d;
    int32_t causal, window;  // window = t where none was asked for
    float scale, cap;        // cap = 0: scores are not capped
};

template <typename T>
struct AttnTensors {
    Heads<const T> q, k, v, out_in, dout;
    Heads<T> out, dq, dk, dv;
};

struct RotaryParams {
    const int32_t* pos;
    const float* inv_freq;
    int64_t slots;  // blocks * t
    int32_t t, heads, d, n;  // n: pairs that turn
    int32_t interleaved, gradient;
    float factor;
    // several axes: the coordinate of axis k and slot s is coords[k * slots + s]; NULL: positions, one axis
    const int32_t *coords, *axis;
    int32_t axes;
};

struct RecurParams {
    const int32_t* pos;
    float* carry;  // [blocks, runs, channels] or NULL
    void* work;
    int64_t blocks, channels;
    int32_t t;
};
template <typename T>
struct Channels {
    T* data;
    int64_t block, slot;
    __host__ __device__ T* at(int64_t q, int64_t s) const { return data + q * block + s * slot; }
};
template <typename T>
struct RecurTensors {
    Channels<const T> gate, x, dh;
    Channels<T> h, dgate, dx;
};

struct NormParams {
    const int32_t* pos;
    const float *weight, *bias;
    float2* stats;
    float *dweight, *dbias;
    float* work;  // [CTAs][2][channels]
    int64_t rows, channels;
    int32_t t;
    float eps;
    bool flat;    // blocks of every tensor lie one behind the other
    int32_t stages, params_at;  // groups of frames in shared memory, and where weight and bias begin there
    uintptr_t end[2];  // where x and dy end
};
template <typename T>
struct NormTensors {
    Channels<const T> x, dy;
    Channels<T> y, dx;
};

struct ConvParams {
    const int32_t* pos;
    const float *weight, *bias;
    const int32_t* seq_id;
    int64_t n_seq;
    void* tails;
    float *dweight, *dbias;
    float* work;  // [tiles of all blocks][channels * (taps + 1)]
    int64_t blocks, channels;
    int32_t t, taps, silu;
};
template <typename T>
struct ConvTensors {
    Channels<const T> x, dy;
    Channels<T> y, dx;
};

struct ScanParams {
    const int32_t* pos;
    const float *a, *d, *dt_bias;
    float* carry;
    void* work;
    const int32_t* seq_id;
    int64_t n_seq;
    float* last;
    float *da, *dd, *ddt_bias;
    int64_t blocks, channels;
    int32_t t, states, softplus;
    bool rows_wide;  // rows of b and c are whole pieces of 16 bytes
};
template <typename T>
struct ScanTensors {
    Channels<const T> x, dt, b, c, z, dy;
    Channels<T> y, dx, ddt, db, dc, dz;
};
struct ScanStepParams {
    const int32_t* pos;
    const float *a, *d, *dt_bias, *state;
    float* next;
    int64_t rows, channels;
    int32_t states, softplus;
};
template <typename T>
struct ScanStepTensors {  // by rows
    const T *x, *dt, *b, *c, *z;
    T* y;
    int64_t sx, sdt, sb, sc, sz, sy;
};

// Lets a kernel have `bytes` of dynamic shared memory, once per device (`done`: one bit each, of the kernel).
template <typename F>
cudaError_t allow_shared(F* kernel, int bytes, std::atomic<uint64_t>& done)
{
    int device = 0;
    const cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const uint64_t bit = device < 64 ? (uint64_t)1 << device : 0;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    const cudaError_t f = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (f == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return f;
}

template <typename T>
cudaError_t launch_rotary(const RotaryParams& p, const Heads<const T>& x, const Heads<T>& y, cudaStream_t st);
template <typename T>
cudaError_t launch_attention(const AttnParams& p, const AttnTensors<T>& a, cudaStream_t st);
template <typename T>
cudaError_t launch_attention_grad(const AttnParams& p, const AttnTensors<T>& a, cudaStream_t st);
template <typename T>
cudaError_t launch_recurrence(const RecurParams& p, const RecurTensors<T>& a, cudaStream_t st);
template <typename T>
cudaError_t launch_recurrence_grad(const RecurParams& p, const RecurTensors<T>& a, cudaStream_t st);

template <typename T>
cudaError_t launch_norm(const NormParams& p, const NormTensors<T>& a, cudaStream_t st);
template <typename T>
cudaError_t launch_norm_grad(const NormParams& p, const NormTensors<T>& a, cudaStream_t st);
template <typename T>
cudaError_t launch_conv(const ConvParams& p, const ConvTensors<T>& a, cudaStream_t st);
template <typename T>
cudaError_t launch_conv_grad(const ConvParams& p, const ConvTensors<T>& a, cudaStream_t st);
template <typename T>
cudaError_t launch_conv_step(const ConvParams& p, int64_t rows, const T* state, T* next, const T* x, int64_t sx, T* y, int64_t sy,
                             cudaStream_t st);
template <typename T>
cudaError_t launch_scan(const ScanParams& p, const ScanTensors<T>& a, cudaStream_t st);
template <typename T>
cudaError_t launch_scan_grad(const ScanParams& p, const ScanTensors<T>& a, cudaStream_t st);
template <typename T>
cudaError_t launch_scan_step(const ScanStepParams& p, const ScanStepTensors<T>& a, cudaStream_t st);

// Up to three arrays side by side in the columns of `part`: out[k][i] = sum over rows of part[row][column], rows in a fixed order.
struct ColumnSums {
    const float* part;
    int64_t rows, columns;
    float* out[3];       // NULL: not wanted
    int64_t end[3];      // columns below end[k] and not below end[k - 1] go to out[k]
};
cudaError_t launch_column_sums(const ColumnSums& s, cudaStream_t st);

size_t norm_work_bytes(int64_t rows, int64_t channels);
size_t conv_work_bytes(int64_t blocks, int32_t t, int64_t channels, int32_t taps, int32_t dtype);
size_t scan_work_bytes(int64_t blocks, int32_t t, int64_t channels, int32_t states, bool gradient);
size_t recurrence_work_bytes(int64_t blocks, int32_t t, int64_t channels);
int64_t attention_timeouts(), recurrence_timeouts();  // see bload_device_timeouts

#ifdef __CUDACC__
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Two numbers in one 64-bit register: multiplies and adds of both are one instruction, which matters where a kernel runs close
// to the instruction rate.
struct Two {
    unsigned long long v;
};
__device__ __forceinline__ Two two(float a, float b)
{
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 one(Two x)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x.v));
    return r;
}
__device__ __forceinline__ Two operator*(Two a, Two b)
{
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Two operator+(Two a, Two b)
{
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Two fma(Two a, Two b, Two c)
{
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ Two zero() { return {0ull}; }

// V neighbouring elements in registers.  WIDE: they lie on a boundary of their size (at most 16 bytes) and all exist; otherwise
// the first `there` of them are moved one by one, and the rest read as zeros.
template <typename T, int V>
struct alignas(V * sizeof(T) < 16 ? V * sizeof(T) : 16) Elements {
    T x[V];
    static constexpr int kBytes = V * sizeof(T), kWord = kBytes < 16 ? kBytes : 16;
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = from_float<T>(0.0f);
    }
    __device__ __forceinline__ void load(const T* p, int there, bool wide)
    {
        if (wide && there >= V) {
            if constexpr (kWord == 16) {
#pragma unroll
                for (int k = 0; k < kBytes / 16; ++k) reinterpret_cast<uint4*>(x)[k] = reinterpret_cast<const uint4*>(p)[k];
            } else if constexpr (kWord == 8) {
                *reinterpret_cast<uint2*>(x) = *reinterpret_cast<const uint2*>(p);
            } else if constexpr (kWord == 4) {
                *reinterpret_cast<uint32_t*>(x) = *reinterpret_cast<const uint32_t*>(p);
            } else {
                x[0] = p[0];
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = e < there ? p[e] : from_float<T>(0.0f);
        }
    }
    __device__ __forceinline__ void store(T* p, int there, bool wide) const
    {
        if (wide && there >= V) {
            if constexpr (kWord == 16) {
#pragma unroll
                for (int k = 0; k < kBytes / 16; ++k) reinterpret_cast<uint4*>(p)[k] = reinterpret_cast<const uint4*>(x)[k];
            } else if constexpr (kWord == 8) {
                *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(x);
            } else if constexpr (kWord == 4) {
                *reinterpret_cast<uint32_t*>(p) = *reinterpret_cast<const uint32_t*>(x);
            } else {
                p[0] = x[0];
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < there) p[e] = x[e];
        }
    }
    // WIDE loads that are predicated rather than branched around: a branch's two values meet in registers, and waiting for them there
    // would keep a load that is issued early from overlapping with what follows.
    __device__ __forceinline__ void load_if(const T* p, bool on)
    {
        if constexpr (kBytes % 16 == 0) {
#pragma unroll
            for (int k = 0; k < kBytes / 16; ++k) {
                uint32_t w[4] = {0u, 0u, 0u, 0u};
                asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\t@p ld.global.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
                             : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3])
                             : "l"(reinterpret_cast<const char*>(p) + 16 * k), "r"((uint32_t)on));
#pragma unroll
                for (int i = 0; i < 4; ++i) reinterpret_cast<uint32_t*>(x)[4 * k + i] = w[i];
            }
        } else if constexpr (kBytes == 8) {
            uint32_t w[2] = {0u, 0u};
            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %3, 0;\n\t@p ld.global.v2.u32 {%0, %1}, [%2];\n\t}" : "+r"(w[0]), "+r"(w[1]) : "l"(p), "r"((uint32_t)on));
            reinterpret_cast<uint32_t*>(x)[0] = w[0];
            reinterpret_cast<uint32_t*>(x)[1] = w[1];
        } else {
            static_assert(kBytes == 4, "4, 8 or whole pieces of 16 bytes");
            uint32_t w = 0u;
            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p ld.global.u32 %0, [%1];\n\t}" : "+r"(w) : "l"(p), "r"((uint32_t)on));
            reinterpret_cast<uint32_t*>(x)[0] = w;
        }
    }
    // elements `step` apart
    __device__ __forceinline__ void load_apart(const T* p, int64_t step, int there)
    {
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = e < there ? p[e * step] : from_float<T>(0.0f);
    }
    __device__ __forceinline__ void store_apart(T* p, int64_t step, int there) const
    {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e < there) p[e * step] = x[e];
    }
    __device__ __forceinline__ float get(int e) const { return to_float(x[e]); }
    __device__ __forceinline__ void set(int e, float v) { x[e] = from_float<T>(v); }
    // elements e and e + 1, e even
    __device__ __forceinline__ Two pair(int e) const
    {
        if constexpr (sizeof(T) == 4) {
            return two(x[e], x[e + 1]);
        } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(x + e);  // (its halves are the upper halves of 32-bit numbers)
            return two(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
        } else {
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(x + e));
            return two(v.x, v.y);
        }
    }
    __device__ __forceinline__ void set_pair(int e, Two v)
    {
        const float2 f = one(v);
        if constexpr (sizeof(T) == 4) {
            x[e] = f.x;
            x[e + 1] = f.y;
        } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
            *reinterpret_cast<__nv_bfloat162*>(x + e) = __floats2bfloat162_rn(f.x, f.y);
        } else {
            *reinterpret_cast<__half2*>(x + e) = __floats2half2_rn(f.x, f.y);
        }
    }
};

// sigmoid(v) = 1 / (1 + exp(-v)), to a few 2^-23 of itself for |v| up to some tens (where exp(-v) passes 2^128 it is 0)
__device__ __forceinline__ float sigmoid_of(float v)
{
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    return r;
}

__device__ __forceinline__ Two sigmoid_of(Two v)
{
    const float2 x = one(v * two(-1.4426950408889634f, -1.4426950408889634f));
    float2 e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(x.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(x.y));
    e = one(two(e.x, e.y) + two(1.0f, 1.0f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(e.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(e.y));
    return two(r.x, r.y);
}

// Sums of N values (a power of two, at most 32) over the lanes that differ in the bits from 16 down to LOW: the values are shared
// out on the way, so that each step exchanges half as many.  A lane ends with `left` sums, v[0..left-1], of the values from index
// `first` on: N - 1 exchanges instead of 5 N for a whole warp.
template <int N, int LOW>
struct Shared {
    static constexpr int kSteps = LOW == 1 ? 5 : LOW == 2 ? 4 : LOW == 4 ? 3 : LOW == 8 ? 2 : LOW == 16 ? 1 : 0;
    static constexpr int kLeft = (N >> kSteps) > 1 ? N >> kSteps : 1;
};
template <int N, int BIT, int LOW>
__device__ __forceinline__ void share_sums(float* v, int lane, int& first)
{
    if constexpr (BIT >= LOW) {
        if constexpr (N > 1) {
            constexpr int H = N / 2;
            const bool upper = lane & BIT;
#pragma unroll
            for (int i = 0; i < H; ++i) {
                const float send = upper ? v[i] : v[i + H], keep = upper ? v[i + H] : v[i];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, send, BIT);
            }
            if (upper) first += H;
            share_sums<H, BIT / 2, LOW>(v, lane, first);
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], BIT);
            share_sums<1, BIT / 2, LOW>(v, lane, first);
        }
    }
}

// First slot behind the sequence that holds slot i (pos[i] >= 0), by a whole warp: pos[s] == s - start holds up to the
// end of the sequence and nowhere behind it.  The next 128 slots are looked at together, which ends it for short sequences; then 32
// probes cut the range by 32 (three rounds for 32,768 slots).  Whatever pos holds, the result is in (i, t].
__device__ __forceinline__ int warp_seq_end(const int32_t* pos, int t, int i, int lane)
{
    const int start = i - pos[i];
    int lo = i, hi = t;
    bool near[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int s = i + 1 + 32 * k + lane;
        near[k] = s < t && pos[s] == s - start;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const unsigned out = ~__ballot_sync(0xffffffffu, near[k]);
        if (out) return i + 32 * k + __ffs(out);
    }
    lo = i + 128;
    while (hi - lo > 1) {
        const int step = (hi - lo - 1 + 31) / 32;
        const int s = lo + step * (lane + 1);
        const bool in = s < hi && pos[s] == s - start;
        const unsigned m = ~__ballot_sync(0xffffffffu, in);
        const int n = m ? __ffs(m) - 1 : 32;
        lo += step * n;
        hi = min(hi, lo + step);
    }
    return hi;
}
#endif

}  // namespace bload

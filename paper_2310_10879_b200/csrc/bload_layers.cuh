// Shared by the layers on packed batches (rotary positions, attention, recurrence): element types, the extent of a
// sequence around a slot, and the launch parameters.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

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

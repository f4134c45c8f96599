// Gated linear recurrence along the slots of packed blocks, restarted at every sequence start:
//     f = sigmoid(gate);  h = f h_prev + (1 - f) x
// and its gradient.  A thread per channel walks the slots.
#include "bload_internal.cuh"
#include "bload_layers.cuh"

namespace bload {

namespace {

constexpr int kRun = BLOAD_RECURRENCE_RUN;

// f = sigmoid(g) and 1 - f, each with a small relative error of its own (1 - f must not cancel: it scales the input).
__device__ __forceinline__ void gate_of(float g, float& f, float& keep)
{
    const float e = expf(-fabsf(g));
    const float big = 1.0f / (1.0f + e), small = e * big;
    f = g >= 0.0f ? big : small;
    keep = g >= 0.0f ? small : big;
}

template <typename T>
__global__ void k27_recurrence(RecurParams p, RecurTensors<T> a)
{
    const int64_t item = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, q = item / p.channels, c = item % p.channels;
    if (q >= p.blocks) return;
    const int runs = (p.t + kRun - 1) / kRun;
    float h = 0.0f;
    for (int s = 0; s < p.t; ++s) {
        if (p.carry && s % kRun == 0) p.carry[(q * runs + s / kRun) * p.channels + c] = h;
        const int pos = p.pos[q * p.t + s];
        if (pos <= 0) h = 0.0f;
        if (pos >= 0) {
            float f, keep;
            gate_of(to_float(a.gate.at(q, s)[c]), f, keep);
            h = f * h + keep * to_float(a.x.at(q, s)[c]);
        }
        a.h.at(q, s)[c] = from_float<T>(h);
    }
}

template <typename T>
__global__ void k28_recurrence_grad(RecurParams p, RecurTensors<T> a)
{
    const int64_t item = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, q = item / p.channels, c = item % p.channels;
    if (q >= p.blocks) return;
    const int runs = (p.t + kRun - 1) / kRun;
    float from_right = 0.0f;  // f_{s+1} g_{s+1} where the sequence continues
    for (int r = runs - 1; r >= 0; --r) {
        float before[kRun];  // h_{s-1}
        float h = p.carry[(q * runs + r) * p.channels + c];
        const int s0 = r * kRun, s1 = min(s0 + kRun, p.t);
        for (int s = s0; s < s1; ++s) {
            const int pos = p.pos[q * p.t + s];
            if (pos <= 0) h = 0.0f;
            before[s - s0] = h;
            if (pos >= 0) {
                float f, keep;
                gate_of(to_float(a.gate.at(q, s)[c]), f, keep);
                h = f * h + keep * to_float(a.x.at(q, s)[c]);
            }
        }
        for (int s = s1 - 1; s >= s0; --s) {
            const int pos = p.pos[q * p.t + s];
            float dg = 0.0f, dx = 0.0f;
            if (pos >= 0) {
                float f, keep;
                gate_of(to_float(a.gate.at(q, s)[c]), f, keep);
                const float g = to_float(a.dh.at(q, s)[c]) + from_right;
                dx = keep * g;
                dg = g * (before[s - s0] - to_float(a.x.at(q, s)[c])) * f * keep;
                from_right = pos > 0 ? f * g : 0.0f;
            } else {
                from_right = 0.0f;
            }
            a.dgate.at(q, s)[c] = from_float<T>(dg);
            a.dx.at(q, s)[c] = from_float<T>(dx);
        }
    }
}

}  // namespace

template <typename T>
cudaError_t launch_recurrence(const RecurParams& p, const RecurTensors<T>& a, cudaStream_t st)
{
    k27_recurrence<T><<<(unsigned)((p.blocks * p.channels + 127) / 128), 128, 0, st>>>(p, a);
    count_launches(1);
    return cudaGetLastError();
}
template <typename T>
cudaError_t launch_recurrence_grad(const RecurParams& p, const RecurTensors<T>& a, cudaStream_t st)
{
    k28_recurrence_grad<T><<<(unsigned)((p.blocks * p.channels + 127) / 128), 128, 0, st>>>(p, a);
    count_launches(1);
    return cudaGetLastError();
}
#define BLOAD_INSTANTIATE(T)                                                                            \
    template cudaError_t launch_recurrence<T>(const RecurParams&, const RecurTensors<T>&, cudaStream_t); \
    template cudaError_t launch_recurrence_grad<T>(const RecurParams&, const RecurTensors<T>&, cudaStream_t);
BLOAD_INSTANTIATE(float)
BLOAD_INSTANTIATE(__half)
BLOAD_INSTANTIATE(__nv_bfloat16)
#undef BLOAD_INSTANTIATE

}  // namespace bload

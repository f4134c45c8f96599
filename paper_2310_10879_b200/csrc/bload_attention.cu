// Attention inside the sequences of packed blocks and its gradients.
#include "bload_attention_rows.cuh"
#include "bload_internal.cuh"

namespace bload {

namespace {

enum { kForward, kDq, kDkv };

// A warp per row: the simplest form that is right for every case.
template <typename T, int WHAT>
__global__ void __launch_bounds__(256) k29_attention_rows(AttnParams p, AttnTensors<T> a)
{
    const int lane = threadIdx.x & 31;
    const int heads = WHAT == kDkv ? p.kv_heads : p.heads;
    const int64_t items = p.blocks * heads * p.t, warps = ((int64_t)gridDim.x * blockDim.x) >> 5;
    for (int64_t item = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5; item < items; item += warps) {
        const int i = (int)(item % p.t);
        const int h = (int)(item / p.t % heads);
        const int64_t b = item / p.t / heads;
        if (WHAT == kForward) rows::forward_row(p, a, b, h, i, lane);
        if (WHAT == kDq) rows::dq_row(p, a, b, h, i, lane);
        if (WHAT == kDkv) rows::dkv_row(p, a, b, h, i, lane);
    }
}

template <typename T, int WHAT>
cudaError_t launch(const AttnParams& p, const AttnTensors<T>& a, cudaStream_t st)
{
    const int64_t items = p.blocks * (WHAT == kDkv ? p.kv_heads : p.heads) * p.t, grid = (items + 7) / 8;
    k29_attention_rows<T, WHAT><<<(unsigned)(grid < 148 * 64 ? grid : 148 * 64), 256, 0, st>>>(p, a);
    count_launches(1);
    return cudaGetLastError();
}

}  // namespace

template <typename T>
cudaError_t launch_attention(const AttnParams& p, const AttnTensors<T>& a, cudaStream_t st)
{
    return launch<T, kForward>(p, a, st);
}
template <typename T>
cudaError_t launch_attention_grad(const AttnParams& p, const AttnTensors<T>& a, cudaStream_t st)
{
    cudaError_t e = launch<T, kDq>(p, a, st);
    return e != cudaSuccess ? e : launch<T, kDkv>(p, a, st);
}
#define BLOAD_INSTANTIATE(T)                                                                          \
    template cudaError_t launch_attention<T>(const AttnParams&, const AttnTensors<T>&, cudaStream_t); \
    template cudaError_t launch_attention_grad<T>(const AttnParams&, const AttnTensors<T>&, cudaStream_t);
BLOAD_INSTANTIATE(__half)
BLOAD_INSTANTIATE(__nv_bfloat16)
#undef BLOAD_INSTANTIATE

}  // namespace bload

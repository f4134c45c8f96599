// k26_rotary: rotary positions that restart with every sequence of a packed block, and their gradient (the turn by
// minus the same angles).  A frame at position p has each pair (u, w) of its heads turned by p * inv_freq[i].
#include "bload_internal.cuh"
#include "bload_layers.cuh"

namespace bload {

namespace {

// A thread per (slot, pair or copied element), over all heads: the angle is computed once for all of them.
template <typename T>
__global__ void __launch_bounds__(256) k26_rotary(RotaryParams p, Heads<const T> x, Heads<T> y)
{
    const int units = p.n + (p.d - 2 * p.n);
    const int64_t items = p.slots * units;
    for (int64_t item = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; item < items; item += (int64_t)gridDim.x * blockDim.x) {
        const int64_t slot = item / units;
        const int unit = (int)(item - slot * units);
        const int64_t q = slot / p.t;
        const int64_t s = slot - q * p.t;
        const int pos = p.pos[slot];
        const T* xs = x.at(q, s, 0);
        T* ys = y.at(q, s, 0);
        if (unit >= p.n) {
            const int e = p.n + unit;
            for (int h = 0; h < p.heads; ++h) ys[h * y.head + e] = xs[h * x.head + e];
            continue;
        }
        float sn, cs;
        sincosf((float)pos * p.inv_freq[unit], &sn, &cs);
        sn *= p.gradient ? -p.factor : p.factor;
        cs *= p.factor;
        const int iu = p.interleaved ? 2 * unit : unit, iw = p.interleaved ? 2 * unit + 1 : p.n + unit;
        for (int h = 0; h < p.heads; ++h) {
            const T tu = xs[h * x.head + iu], tw = xs[h * x.head + iw];
            const float u = to_float(tu), w = to_float(tw);
            ys[h * y.head + iu] = pos >= 0 ? from_float<T>(u * cs - w * sn) : tu;
            ys[h * y.head + iw] = pos >= 0 ? from_float<T>(w * cs + u * sn) : tw;
        }
    }
}

}  // namespace

template <typename T>
cudaError_t launch_rotary(const RotaryParams& p, const Heads<const T>& x, const Heads<T>& y, cudaStream_t st)
{
    const int64_t items = p.slots * (p.d - p.n);
    const int64_t grid = (items + 255) / 256;
    k26_rotary<T><<<(unsigned)(grid < 148 * 64 ? grid : 148 * 64), 256, 0, st>>>(p, x, y);
    count_launches(1);
    return cudaGetLastError();
}
template cudaError_t launch_rotary<float>(const RotaryParams&, const Heads<const float>&, const Heads<float>&, cudaStream_t);
template cudaError_t launch_rotary<__half>(const RotaryParams&, const Heads<const __half>&, const Heads<__half>&, cudaStream_t);
template cudaError_t launch_rotary<__nv_bfloat16>(const RotaryParams&, const Heads<const __nv_bfloat16>&,
                                                  const Heads<__nv_bfloat16>&, cudaStream_t);

}  // namespace bload

// C ABI of the layers on packed batches: argument checks and dispatch on the element type.  See include/bload.h.
#include <math.h>

#include "bload_internal.cuh"
#include "bload_layers.cuh"

namespace bload {
namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int check_common(int64_t block_count, int32_t t_block, int32_t dtype, const int32_t* d_pos)
{
    if (block_count < 0 || block_count > 0x7fffffffLL || t_block < 1) return BLOAD_ERR_ARG;
    if (t_block > BLOAD_MAX_T_BLOCK || dtype < BLOAD_F32 || dtype > BLOAD_BF16) return BLOAD_ERR_UNSUPPORTED;
    if (block_count == 0) return BLOAD_OK;
    if (!d_pos) return BLOAD_ERR_NULL;
    if (!aligned(d_pos, 4)) return BLOAD_ERR_ALIGN;
    return BLOAD_OK;
}
size_t size_of(int32_t dtype) { return dtype == BLOAD_F32 ? 4 : 2; }

constexpr int64_t kMaxStride = (int64_t)1 << 39;  // bytes fit the 40 bits of a tensor map, products of a call 63 bits

// strides of dimensions longer than one; an output may not be broadcast (stride 0), an input of the rotary or the
// recurrence may
int check_stride(int64_t n, int64_t stride, bool zero_ok)
{
    if (n <= 1) return BLOAD_OK;
    return (stride > 0 || (zero_ok && stride == 0)) && stride < kMaxStride ? BLOAD_OK : BLOAD_ERR_ARG;
}
int check_heads(const bload_heads_t& x, int64_t blocks, int64_t t, int64_t heads, size_t align, bool zero_ok)
{
    if (!x.data) return BLOAD_ERR_NULL;
    int rc;
    if ((rc = check_stride(blocks, x.block_stride, zero_ok))) return rc;
    if ((rc = check_stride(t, x.slot_stride, zero_ok))) return rc;
    if ((rc = check_stride(heads, x.head_stride, zero_ok))) return rc;
    return aligned(x.data, align) ? BLOAD_OK : BLOAD_ERR_ALIGN;
}
// Strides of dimensions of length one are not used: 0 in their place keeps every address in range.
template <typename P>
Heads<P> heads_of(const bload_heads_t& x, int64_t blocks, int64_t t, int64_t heads)
{
    return {static_cast<P*>(x.data), blocks > 1 ? x.block_stride : 0, t > 1 ? x.slot_stride : 0, heads > 1 ? x.head_stride : 0};
}

int done(cudaError_t ce)
{
    if (ce == cudaSuccess) return BLOAD_OK;
    (void)cudaGetLastError();
    return BLOAD_ERR_CUDA;
}

int rotary(const int32_t* d_pos, int64_t block_count, int32_t t_block, int32_t heads, int32_t head_dim, int32_t dtype,
           const bload_heads_t* x, const bload_heads_t* y, const float* d_inv_freq, int32_t rot_dim, int32_t interleaved,
           float factor, int gradient, void* stream)
{
    if (!x || !y) return BLOAD_ERR_NULL;
    int rc = check_common(block_count, t_block, dtype, d_pos);
    if (rc) return rc;
    if (heads < 1 || heads > 4096 || head_dim < 1 || head_dim > 4096 || rot_dim < 0 || rot_dim > head_dim || (rot_dim & 1) || !isfinite(factor))
        return BLOAD_ERR_ARG;
    if (block_count == 0) return BLOAD_OK;
    if (rot_dim && !d_inv_freq) return BLOAD_ERR_NULL;
    if (!aligned(d_inv_freq, 4)) return BLOAD_ERR_ALIGN;
    if ((rc = check_heads(*x, block_count, t_block, heads, size_of(dtype), true))) return rc;
    if ((rc = check_heads(*y, block_count, t_block, heads, size_of(dtype), false))) return rc;
    RotaryParams p{d_pos, d_inv_freq, block_count * t_block, t_block, heads, head_dim, rot_dim / 2, interleaved != 0, gradient,
                   factor};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto go = [&](auto zero) {
        using T = decltype(zero);
        return launch_rotary<T>(p, heads_of<const T>(*x, block_count, t_block, heads),
                                heads_of<T>(*y, block_count, t_block, heads), st);
    };
    return done(dtype == BLOAD_F32 ? go(float()) : dtype == BLOAD_F16 ? go(__half()) : go(__nv_bfloat16()));
}

int check_attention(const bload_attention_t* a, bool gradient)
{
    if (!a) return BLOAD_ERR_NULL;
    int rc = check_common(a->block_count, a->t_block, a->dtype, a->d_pos);
    if (rc) return rc;
    if (a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads || a->head_dim < 1 || a->window < 0) return BLOAD_ERR_ARG;
    if (!isfinite(a->scale) || !isfinite(a->softcap) || a->softcap < 0.0f) return BLOAD_ERR_ARG;
    if (a->block_count * a->heads > 0x7fffffffLL || a->block_count * a->heads * ((a->t_block + 127) / 128) > 0x7fffffffLL)
        return BLOAD_ERR_ARG;
    if (a->dtype == BLOAD_F32 || a->head_dim % 8 || a->head_dim > 128) return BLOAD_ERR_UNSUPPORTED;
    if (a->block_count == 0) return BLOAD_OK;
    auto tensor = [&](const bload_heads_t& x, int heads) {
        int e = check_heads(x, a->block_count, a->t_block, heads, 16, false);
        if (e) return e;
        const bool whole = (a->block_count == 1 || x.block_stride % 8 == 0) && (a->t_block == 1 || x.slot_stride % 8 == 0) &&
                           (heads == 1 || x.head_stride % 8 == 0);
        return whole ? BLOAD_OK : BLOAD_ERR_ALIGN;
    };
    if ((rc = tensor(a->q, a->heads)) || (rc = tensor(a->k, a->kv_heads)) || (rc = tensor(a->v, a->kv_heads)) ||
        (rc = tensor(a->out, a->heads)))
        return rc;
    if (gradient) {
        if (!a->d_lse || !a->d_delta) return BLOAD_ERR_NULL;
        if ((rc = tensor(a->dout, a->heads)) || (rc = tensor(a->dq, a->heads)) || (rc = tensor(a->dk, a->kv_heads)) ||
            (rc = tensor(a->dv, a->kv_heads)))
            return rc;
        if (!aligned(a->d_delta, 4)) return BLOAD_ERR_ALIGN;
    }
    if (!aligned(a->d_lse, 4) || !aligned(a->d_slopes, 4)) return BLOAD_ERR_ALIGN;
    return BLOAD_OK;
}

// The forward call reads the fields up to d_lse only: its caller's block may end there.
template <typename T>
AttnTensors<T> attention_tensors(const bload_attention_t* a, bool gradient)
{
    const int64_t b = a->block_count, t = a->t_block;
    AttnTensors<T> x{};
    x.q = heads_of<const T>(a->q, b, t, a->heads);
    x.k = heads_of<const T>(a->k, b, t, a->kv_heads);
    x.v = heads_of<const T>(a->v, b, t, a->kv_heads);
    x.out = heads_of<T>(a->out, b, t, a->heads);
    x.out_in = heads_of<const T>(a->out, b, t, a->heads);
    if (gradient) {
        x.dout = heads_of<const T>(a->dout, b, t, a->heads);
        x.dq = heads_of<T>(a->dq, b, t, a->heads);
        x.dk = heads_of<T>(a->dk, b, t, a->kv_heads);
        x.dv = heads_of<T>(a->dv, b, t, a->kv_heads);
    }
    return x;
}
AttnParams attention_params(const bload_attention_t* a, bool gradient)
{
    AttnParams p;
    p.pos = a->d_pos;
    p.slopes = a->d_slopes;
    p.lse = a->d_lse;
    p.delta = gradient ? a->d_delta : nullptr;
    p.blocks = a->block_count;
    p.t = a->t_block;
    p.heads = a->heads;
    p.kv_heads = a->kv_heads;
    p.group = a->heads / a->kv_heads;
    p.d = a->head_dim;
    p.causal = a->causal != 0;
    p.window = a->window > 0 && a->window < a->t_block ? a->window : a->t_block;
    p.scale = a->scale;
    p.cap = a->softcap;
    return p;
}

// at most 2^31 - 1 pieces of 64 slots by 64 channels (a grid holds that many)
bool recurrence_fits(int64_t blocks, int32_t t, int64_t channels)
{
    if (channels < 1 || channels > 0x7fffffffLL) return false;
    return blocks <= 0x7fffffffLL / (((channels + 63) / 64) * ((t + 63) / 64));
}
int check_recurrence(const bload_recurrence_t* a, bool gradient)
{
    if (!a) return BLOAD_ERR_NULL;
    int rc = check_common(a->block_count, a->t_block, a->dtype, a->d_pos);
    if (rc) return rc;
    if (!recurrence_fits(a->block_count, a->t_block, a->channels)) return BLOAD_ERR_ARG;
    if (a->block_count == 0) return BLOAD_OK;
    auto tensor = [&](const bload_channels_t& x, bool zero_ok) {
        if (!x.data) return BLOAD_ERR_NULL;
        int e;
        if ((e = check_stride(a->block_count, x.block_stride, zero_ok))) return e;
        if ((e = check_stride(a->t_block, x.slot_stride, zero_ok))) return e;
        return aligned(x.data, size_of(a->dtype)) ? BLOAD_OK : BLOAD_ERR_ALIGN;
    };
    if ((rc = tensor(a->gate, true)) || (rc = tensor(a->x, true))) return rc;
    if (!gradient && (rc = tensor(a->h, false))) return rc;
    if (gradient) {
        if (!a->d_carry) return BLOAD_ERR_NULL;
        if ((rc = tensor(a->dh, true)) || (rc = tensor(a->dgate, false)) || (rc = tensor(a->dx, false))) return rc;
    }
    if (!aligned(a->d_carry, 16)) return BLOAD_ERR_ALIGN;
    const size_t need = bload_recurrence_work_bytes(a->block_count, a->t_block, a->channels);
    if (need) {
        if (!a->d_work) return BLOAD_ERR_NULL;
        if (!aligned(a->d_work, 256)) return BLOAD_ERR_ALIGN;
        if (a->work_bytes < need) return BLOAD_ERR_WORKSPACE;
    }
    return BLOAD_OK;
}
template <typename P>
Channels<P> channels_of(const bload_channels_t& x, int64_t blocks, int64_t t)
{
    return {static_cast<P*>(x.data), blocks > 1 ? x.block_stride : 0, t > 1 ? x.slot_stride : 0};
}
template <typename T>
RecurTensors<T> recurrence_tensors(const bload_recurrence_t* a)
{
    const int64_t b = a->block_count, t = a->t_block;
    return {channels_of<const T>(a->gate, b, t), channels_of<const T>(a->x, b, t), channels_of<const T>(a->dh, b, t),
            channels_of<T>(a->h, b, t), channels_of<T>(a->dgate, b, t), channels_of<T>(a->dx, b, t)};
}

}  // namespace
}  // namespace bload

using namespace bload;

extern "C" {

int bload_rotary(const int32_t* d_pos, int64_t block_count, int32_t t_block, int32_t heads, int32_t head_dim, int32_t dtype,
                 const bload_heads_t* x, const bload_heads_t* y, const float* d_inv_freq, int32_t rot_dim,
                 int32_t interleaved, float factor, void* stream)
{
    return rotary(d_pos, block_count, t_block, heads, head_dim, dtype, x, y, d_inv_freq, rot_dim, interleaved, factor, 0, stream);
}

int bload_rotary_grad(const int32_t* d_pos, int64_t block_count, int32_t t_block, int32_t heads, int32_t head_dim,
                      int32_t dtype, const bload_heads_t* dy, const bload_heads_t* dx, const float* d_inv_freq,
                      int32_t rot_dim, int32_t interleaved, float factor, void* stream)
{
    return rotary(d_pos, block_count, t_block, heads, head_dim, dtype, dy, dx, d_inv_freq, rot_dim, interleaved, factor, 1, stream);
}

int bload_attention(const bload_attention_t* a, void* stream)
{
    int rc = check_attention(a, false);
    if (rc || a->block_count == 0) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const AttnParams p = attention_params(a, false);
    return done(a->dtype == BLOAD_F16 ? launch_attention<__half>(p, attention_tensors<__half>(a, false), st)
                                      : launch_attention<__nv_bfloat16>(p, attention_tensors<__nv_bfloat16>(a, false), st));
}

int bload_attention_grad(const bload_attention_t* a, void* stream)
{
    int rc = check_attention(a, true);
    if (rc || a->block_count == 0) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const AttnParams p = attention_params(a, true);
    return done(a->dtype == BLOAD_F16 ? launch_attention_grad<__half>(p, attention_tensors<__half>(a, true), st)
                                      : launch_attention_grad<__nv_bfloat16>(p, attention_tensors<__nv_bfloat16>(a, true), st));
}

size_t bload_recurrence_work_bytes(int64_t block_count, int32_t t_block, int64_t channels)
{
    if (block_count < 1 || t_block < 1 || t_block > BLOAD_MAX_T_BLOCK || !recurrence_fits(block_count, t_block, channels)) return 0;
    return recurrence_work_bytes(block_count, t_block, channels);
}

int bload_recurrence(const bload_recurrence_t* a, void* stream)
{
    int rc = check_recurrence(a, false);
    if (rc || a->block_count == 0) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const RecurParams p{a->d_pos, a->d_carry, a->d_work, a->block_count, a->channels, a->t_block};
    return done(a->dtype == BLOAD_F32   ? launch_recurrence<float>(p, recurrence_tensors<float>(a), st)
                : a->dtype == BLOAD_F16 ? launch_recurrence<__half>(p, recurrence_tensors<__half>(a), st)
                                        : launch_recurrence<__nv_bfloat16>(p, recurrence_tensors<__nv_bfloat16>(a), st));
}

int bload_recurrence_grad(const bload_recurrence_t* a, void* stream)
{
    int rc = check_recurrence(a, true);
    if (rc || a->block_count == 0) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const RecurParams p{a->d_pos, a->d_carry, a->d_work, a->block_count, a->channels, a->t_block};
    return done(a->dtype == BLOAD_F32   ? launch_recurrence_grad<float>(p, recurrence_tensors<float>(a), st)
                : a->dtype == BLOAD_F16 ? launch_recurrence_grad<__half>(p, recurrence_tensors<__half>(a), st)
                                        : launch_recurrence_grad<__nv_bfloat16>(p, recurrence_tensors<__nv_bfloat16>(a), st));
}

int64_t bload_device_timeouts(void) 
{
    const int64_t a = attention_timeouts(), r = recurrence_timeouts();
    return a < 0 || r < 0 ? -1 : a + r;
}

}  // extern "C"

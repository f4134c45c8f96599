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

struct AxesOf {
    const int32_t *coords, *axis;
    int32_t axes;
};

int rotary(const AxesOf* axes, const int32_t* d_pos, int64_t block_count, int32_t t_block, int32_t heads, int32_t head_dim, int32_t dtype,
           const bload_heads_t* x, const bload_heads_t* y, const float* d_inv_freq, int32_t rot_dim, int32_t interleaved,
           float factor, int gradient, void* stream)
{
    if (!x || !y) return BLOAD_ERR_NULL;
    int rc = check_common(block_count, t_block, dtype, d_pos);
    if (rc) return rc;
    if (heads < 1 || heads > 4096 || head_dim < 1 || head_dim > 4096 || rot_dim < 0 || rot_dim > head_dim || (rot_dim & 1) || !isfinite(factor))
        return BLOAD_ERR_ARG;
    if (axes && (axes->axes < 1 || axes->axes > BLOAD_MAX_AXES)) return BLOAD_ERR_ARG;
    if (block_count == 0) return BLOAD_OK;
    if (rot_dim && !d_inv_freq) return BLOAD_ERR_NULL;
    if (!aligned(d_inv_freq, 4)) return BLOAD_ERR_ALIGN;
    if (axes && (!axes->coords || (rot_dim && !axes->axis))) return BLOAD_ERR_NULL;
    if (axes && !(aligned(axes->coords, 4) && aligned(axes->axis, 4))) return BLOAD_ERR_ALIGN;
    if ((rc = check_heads(*x, block_count, t_block, heads, size_of(dtype), true))) return rc;
    if ((rc = check_heads(*y, block_count, t_block, heads, size_of(dtype), false))) return rc;
    RotaryParams p{d_pos, d_inv_freq, block_count * t_block, t_block, heads, head_dim, rot_dim / 2, interleaved != 0, gradient,
                   factor, axes ? axes->coords : nullptr, axes ? axes->axis : nullptr, axes ? axes->axes : 0};
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

// strides and address of a [block, slot, channel] tensor
int check_channels(const bload_channels_t& x, int64_t blocks, int64_t t, size_t size, bool zero_ok)
{
    if (!x.data) return BLOAD_ERR_NULL;
    int e;
    if ((e = check_stride(blocks, x.block_stride, zero_ok)) || (e = check_stride(t, x.slot_stride, zero_ok))) return e;
    return aligned(x.data, size) ? BLOAD_OK : BLOAD_ERR_ALIGN;
}
template <typename... P>
bool on_4(const P*... p)
{
    return (aligned(p, 4) && ...);
}
int check_work(const void* work, size_t bytes, size_t need)
{
    if (!need) return BLOAD_OK;
    if (!work) return BLOAD_ERR_NULL;
    if (!aligned(work, 256)) return BLOAD_ERR_ALIGN;
    return bytes < need ? BLOAD_ERR_WORKSPACE : BLOAD_OK;
}

int check_norm(const bload_norm_t* a, bool gradient)
{
    if (!a) return BLOAD_ERR_NULL;
    int rc = check_common(a->block_count, a->t_block, a->dtype, a->d_pos);
    if (rc) return rc;
    if (a->channels < 1 || !isfinite(a->eps) || a->eps < 0.0f) return BLOAD_ERR_ARG;
    if (a->channels > BLOAD_NORM_MAX_CHANNELS) return BLOAD_ERR_UNSUPPORTED;
    if (a->block_count == 0) return BLOAD_OK;
    auto tensor = [&](const bload_channels_t& x, bool zero_ok) {
        return check_channels(x, a->block_count, a->t_block, size_of(a->dtype), zero_ok);
    };
    if (!on_4(a->d_weight, a->d_bias) || !aligned(a->d_stats, 8)) return BLOAD_ERR_ALIGN;
    if ((rc = tensor(a->x, true))) return rc;
    if (!gradient) return tensor(a->y, false);
    if (!a->d_stats) return BLOAD_ERR_NULL;
    if ((rc = tensor(a->dy, true)) || (rc = tensor(a->dx, false))) return rc;
    if (!on_4(a->d_dweight, a->d_dbias)) return BLOAD_ERR_ALIGN;
    return check_work(a->d_work, a->work_bytes,
                      a->d_dweight || a->d_dbias ? bload_norm_work_bytes(a->block_count, a->t_block, a->channels, a->dtype) : 0);
}
template <typename T>
NormTensors<T> norm_tensors(const bload_norm_t* a, bool gradient)
{
    const int64_t b = a->block_count, t = a->t_block;
    NormTensors<T> x{};
    x.x = channels_of<const T>(a->x, b, t);
    if (gradient) {
        x.dy = channels_of<const T>(a->dy, b, t);
        x.dx = channels_of<T>(a->dx, b, t);
    } else {
        x.y = channels_of<T>(a->y, b, t);
    }
    return x;
}
NormParams norm_params(const bload_norm_t* a, bool gradient)
{
    NormParams p{};
    p.pos = a->d_pos;
    p.weight = a->d_weight;
    p.bias = a->d_bias;
    p.stats = reinterpret_cast<float2*>(a->d_stats);
    if (gradient && (a->d_dweight || a->d_dbias)) {
        p.dweight = a->d_dweight;
        p.dbias = a->d_dbias;
        p.work = static_cast<float*>(a->d_work);
    }
    p.rows = a->block_count * a->t_block;
    p.channels = a->channels;
    p.t = a->t_block;
    p.eps = a->eps;
    return p;
}

bool fits_31(int64_t a, int64_t b) { return b == 0 || a <= 0x7fffffffLL / b; }  // a, b >= 0: a * b < 2^31

bool conv_fits(int64_t blocks, int32_t t, int64_t channels)
{
    return channels >= 1 && channels <= 0x7fffffffLL && fits_31(blocks, (int64_t)((t + 31) / 32)) &&
           fits_31(blocks * ((t + 31) / 32), channels / 256 + 1);
}
int check_conv(const bload_conv_t* a, bool gradient)
{
    if (!a) return BLOAD_ERR_NULL;
    int rc = check_common(a->block_count, a->t_block, a->dtype, a->d_pos);
    if (rc) return rc;
    if (!conv_fits(a->block_count, a->t_block, a->channels) || a->taps < 1) return BLOAD_ERR_ARG;
    if (a->taps > BLOAD_CONV_MAX_TAPS) return BLOAD_ERR_UNSUPPORTED;
    if (a->block_count == 0) return BLOAD_OK;
    const size_t size = size_of(a->dtype);
    auto tensor = [&](const bload_channels_t& x, bool zero_ok) { return check_channels(x, a->block_count, a->t_block, size, zero_ok); };
    if (!a->d_weight) return BLOAD_ERR_NULL;
    if (!on_4(a->d_weight, a->d_bias)) return BLOAD_ERR_ALIGN;
    if ((rc = tensor(a->x, true))) return rc;
    if (!gradient) {
        if (a->d_tails) {
            if (!a->d_seq_id) return BLOAD_ERR_NULL;
            if (a->n_seq < 0) return BLOAD_ERR_ARG;
            if (!aligned(a->d_tails, size) || !aligned(a->d_seq_id, 4)) return BLOAD_ERR_ALIGN;
        }
        return tensor(a->y, false);
    }
    if ((rc = tensor(a->dy, true)) || (rc = tensor(a->dx, false))) return rc;
    if (!on_4(a->d_dweight, a->d_dbias)) return BLOAD_ERR_ALIGN;
    return check_work(a->d_work, a->work_bytes,
                      a->d_dweight || a->d_dbias ? bload_conv_work_bytes(a->block_count, a->t_block, a->channels, a->taps, a->dtype) : 0);
}
template <typename T>
ConvTensors<T> conv_tensors(const bload_conv_t* a, bool gradient)
{
    const int64_t b = a->block_count, t = a->t_block;
    ConvTensors<T> x{};
    x.x = channels_of<const T>(a->x, b, t);
    if (gradient) {
        x.dy = channels_of<const T>(a->dy, b, t);
        x.dx = channels_of<T>(a->dx, b, t);
    } else {
        x.y = channels_of<T>(a->y, b, t);
    }
    return x;
}
ConvParams conv_params(const bload_conv_t* a, bool gradient)
{
    ConvParams p{};
    p.pos = a->d_pos;
    p.weight = a->d_weight;
    p.bias = a->d_bias;
    if (!gradient && a->d_tails && a->taps > 1) {
        p.seq_id = a->d_seq_id;
        p.n_seq = a->n_seq;
        p.tails = a->d_tails;
    }
    if (gradient && (a->d_dweight || a->d_dbias)) {
        p.dweight = a->d_dweight;
        p.dbias = a->d_dbias;
        p.work = static_cast<float*>(a->d_work);
    }
    p.blocks = a->block_count;
    p.channels = a->channels;
    p.t = a->t_block;
    p.taps = a->taps;
    p.silu = a->silu != 0;
    return p;
}

bool scan_fits(int64_t blocks, int64_t t, int64_t channels, int64_t states)
{
    if (channels < 1 || channels > 0x7fffffffLL || blocks > 0x7fffffffLL || states < 1 || states > BLOAD_SCAN_MAX_STATES) return false;
    return fits_31(blocks, channels / 16 + 1) && (blocks == 0 || t <= (1LL << 31) / blocks) &&
           (blocks == 0 || channels * (states + 2) <= (1LL << 35) / blocks);
}
int check_scan(const bload_scan_t* a, bool gradient)
{
    if (!a) return BLOAD_ERR_NULL;
    int rc = check_common(a->block_count, a->t_block, a->dtype, a->d_pos);
    if (rc) return rc;
    if (a->states < 1) return BLOAD_ERR_ARG;
    if (a->states > BLOAD_SCAN_MAX_STATES) return BLOAD_ERR_UNSUPPORTED;
    if (!scan_fits(a->block_count, a->t_block, a->channels, a->states)) return BLOAD_ERR_ARG;
    if (a->block_count == 0) return BLOAD_OK;
    const size_t size = size_of(a->dtype);
    auto tensor = [&](const bload_channels_t& x, bool zero_ok) { return check_channels(x, a->block_count, a->t_block, size, zero_ok); };
    if (!a->d_a) return BLOAD_ERR_NULL;
    if (!on_4(a->d_a, a->d_d, a->d_dt_bias)) return BLOAD_ERR_ALIGN;
    if ((rc = tensor(a->x, true)) || (rc = tensor(a->dt, true)) || (rc = tensor(a->b, true)) || (rc = tensor(a->c, true))) return rc;
    if (a->z.data && (rc = tensor(a->z, true))) return rc;
    if (!aligned(a->d_carry, 16)) return BLOAD_ERR_ALIGN;
    if (!gradient) {
        if ((rc = tensor(a->y, false))) return rc;
        if (a->d_last) {
            if (!a->d_seq_id) return BLOAD_ERR_NULL;
            if (a->n_seq < 0) return BLOAD_ERR_ARG;
            if (!on_4(a->d_last, a->d_seq_id)) return BLOAD_ERR_ALIGN;
        }
    } else {
        if (!a->d_carry || !a->d_da) return BLOAD_ERR_NULL;
        if ((rc = tensor(a->dy, true)) || (rc = tensor(a->dx, false)) || (rc = tensor(a->ddt, false)) || (rc = tensor(a->db, false)) ||
            (rc = tensor(a->dc, false)))
            return rc;
        if (a->z.data && (rc = tensor(a->dz, false))) return rc;
        if (!on_4(a->d_da, a->d_dd, a->d_ddt_bias)) return BLOAD_ERR_ALIGN;
    }
    return check_work(a->d_work, a->work_bytes, bload_scan_work_bytes(a->block_count, a->t_block, a->channels, a->states, gradient));
}
template <typename T>
ScanTensors<T> scan_tensors(const bload_scan_t* a, bool gradient)
{
    const int64_t b = a->block_count, t = a->t_block;
    ScanTensors<T> x{};
    x.x = channels_of<const T>(a->x, b, t);
    x.dt = channels_of<const T>(a->dt, b, t);
    x.b = channels_of<const T>(a->b, b, t);
    x.c = channels_of<const T>(a->c, b, t);
    x.z = channels_of<const T>(a->z, b, t);
    if (gradient) {
        x.dy = channels_of<const T>(a->dy, b, t);
        x.dx = channels_of<T>(a->dx, b, t);
        x.ddt = channels_of<T>(a->ddt, b, t);
        x.db = channels_of<T>(a->db, b, t);
        x.dc = channels_of<T>(a->dc, b, t);
        if (a->z.data) x.dz = channels_of<T>(a->dz, b, t);
    } else {
        x.y = channels_of<T>(a->y, b, t);
    }
    return x;
}
ScanParams scan_params(const bload_scan_t* a, bool gradient)
{
    ScanParams p{};
    p.pos = a->d_pos;
    p.a = a->d_a;
    p.d = a->d_d;
    p.dt_bias = a->d_dt_bias;
    p.carry = a->d_carry;
    p.work = a->d_work;
    if (gradient) {
        p.da = a->d_da;
        p.dd = a->d_dd;
        p.ddt_bias = a->d_ddt_bias;
    } else if (a->d_last) {
        p.seq_id = a->d_seq_id;
        p.n_seq = a->n_seq;
        p.last = a->d_last;
    }
    p.blocks = a->block_count;
    p.channels = a->channels;
    p.t = a->t_block;
    p.states = a->states;
    p.softplus = a->softplus != 0;
    return p;
}

// calls go(element) for an element type
template <typename Go>
int with_type(int32_t dtype, const Go& go)
{
    return done(dtype == BLOAD_F32 ? go(float()) : dtype == BLOAD_F16 ? go(__half()) : go(__nv_bfloat16()));
}

// what the calls for single frames have in common; BLOAD_OK with rows == 0: nothing to do
int check_step(int64_t rows, int64_t channels, int32_t dtype, const int32_t* d_pos, const void* state, const void* next, size_t state_align)
{
    if (rows < 0 || channels < 1 || channels > 0x7fffffffLL || !fits_31(rows, channels / 256 + 1)) return BLOAD_ERR_ARG;
    if (dtype < BLOAD_F32 || dtype > BLOAD_BF16) return BLOAD_ERR_UNSUPPORTED;
    if (rows == 0) return BLOAD_OK;
    if (!d_pos || !state || !next) return BLOAD_ERR_NULL;
    return aligned(d_pos, 4) && aligned(state, state_align) && aligned(next, state_align) ? BLOAD_OK : BLOAD_ERR_ALIGN;
}
int64_t row_stride(const bload_channels_t& x, int64_t rows) { return rows > 1 ? x.block_stride : 0; }

}  // namespace
}  // namespace bload

using namespace bload;

extern "C" {

int bload_rotary(const int32_t* d_pos, int64_t block_count, int32_t t_block, int32_t heads, int32_t head_dim, int32_t dtype,
                 const bload_heads_t* x, const bload_heads_t* y, const float* d_inv_freq, int32_t rot_dim,
                 int32_t interleaved, float factor, void* stream)
{
    return rotary(nullptr, d_pos, block_count, t_block, heads, head_dim, dtype, x, y, d_inv_freq, rot_dim, interleaved, factor, 0, stream);
}

int bload_rotary_grad(const int32_t* d_pos, int64_t block_count, int32_t t_block, int32_t heads, int32_t head_dim,
                      int32_t dtype, const bload_heads_t* dy, const bload_heads_t* dx, const float* d_inv_freq,
                      int32_t rot_dim, int32_t interleaved, float factor, void* stream)
{
    return rotary(nullptr, d_pos, block_count, t_block, heads, head_dim, dtype, dy, dx, d_inv_freq, rot_dim, interleaved, factor, 1, stream);
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

int bload_rotary_axes(const int32_t* d_pos, const int32_t* d_coords, int32_t axes, const int32_t* d_axis, int64_t block_count,
                      int32_t t_block, int32_t heads, int32_t head_dim, int32_t dtype, const bload_heads_t* x, const bload_heads_t* y,
                      const float* d_inv_freq, int32_t rot_dim, int32_t interleaved, float factor, void* stream)
{
    const AxesOf of{d_coords, d_axis, axes};
    return rotary(&of, d_pos, block_count, t_block, heads, head_dim, dtype, x, y, d_inv_freq, rot_dim, interleaved, factor, 0, stream);
}

int bload_rotary_axes_grad(const int32_t* d_pos, const int32_t* d_coords, int32_t axes, const int32_t* d_axis, int64_t block_count,
                           int32_t t_block, int32_t heads, int32_t head_dim, int32_t dtype, const bload_heads_t* dy,
                           const bload_heads_t* dx, const float* d_inv_freq, int32_t rot_dim, int32_t interleaved, float factor, void* stream)
{
    const AxesOf of{d_coords, d_axis, axes};
    return rotary(&of, d_pos, block_count, t_block, heads, head_dim, dtype, dy, dx, d_inv_freq, rot_dim, interleaved, factor, 1, stream);
}

size_t bload_norm_work_bytes(int64_t block_count, int32_t t_block, int64_t channels, int32_t)
{
    if (block_count < 1 || block_count > 0x7fffffffLL || t_block < 1 || t_block > BLOAD_MAX_T_BLOCK || channels < 1 ||
        channels > BLOAD_NORM_MAX_CHANNELS)
        return 0;
    return norm_work_bytes(block_count * t_block, channels);
}

int bload_norm(const bload_norm_t* a, void* stream)
{
    int rc = check_norm(a, false);
    if (rc || a->block_count == 0) return rc;
    return with_type(a->dtype, [&](auto zero) {
        using T = decltype(zero);
        return launch_norm<T>(norm_params(a, false), norm_tensors<T>(a, false), static_cast<cudaStream_t>(stream));
    });
}

int bload_norm_grad(const bload_norm_t* a, void* stream)
{
    int rc = check_norm(a, true);
    if (rc || a->block_count == 0) return rc;
    return with_type(a->dtype, [&](auto zero) {
        using T = decltype(zero);
        return launch_norm_grad<T>(norm_params(a, true), norm_tensors<T>(a, true), static_cast<cudaStream_t>(stream));
    });
}

size_t bload_conv_work_bytes(int64_t block_count, int32_t t_block, int64_t channels, int32_t taps, int32_t dtype)
{
    if (block_count < 1 || block_count > 0x7fffffffLL || t_block < 1 || t_block > BLOAD_MAX_T_BLOCK || taps < 1 ||
        taps > BLOAD_CONV_MAX_TAPS || dtype < BLOAD_F32 || dtype > BLOAD_BF16 || !conv_fits(block_count, t_block, channels))
        return 0;
    return conv_work_bytes(block_count, t_block, channels, taps, dtype);
}

int bload_conv(const bload_conv_t* a, void* stream)
{
    int rc = check_conv(a, false);
    if (rc || a->block_count == 0) return rc;
    return with_type(a->dtype, [&](auto zero) {
        using T = decltype(zero);
        return launch_conv<T>(conv_params(a, false), conv_tensors<T>(a, false), static_cast<cudaStream_t>(stream));
    });
}

int bload_conv_grad(const bload_conv_t* a, void* stream)
{
    int rc = check_conv(a, true);
    if (rc || a->block_count == 0) return rc;
    return with_type(a->dtype, [&](auto zero) {
        using T = decltype(zero);
        return launch_conv_grad<T>(conv_params(a, true), conv_tensors<T>(a, true), static_cast<cudaStream_t>(stream));
    });
}

int bload_conv_step(int64_t rows, int64_t channels, int32_t dtype, int32_t taps, int32_t silu, const int32_t* d_pos, const void* state,
                    void* next, const bload_channels_t* x, const bload_channels_t* y, const float* d_weight, const float* d_bias,
                    void* stream)
{
    if (!x || !y) return BLOAD_ERR_NULL;
    if (taps < 1) return BLOAD_ERR_ARG;
    if (taps > BLOAD_CONV_MAX_TAPS || dtype < BLOAD_F32 || dtype > BLOAD_BF16) return BLOAD_ERR_UNSUPPORTED;
    const char one_tap = 0;  // has no state
    const size_t size = size_of(dtype);
    int rc = check_step(rows, channels, dtype, d_pos, taps > 1 ? state : &one_tap, taps > 1 ? next : &one_tap, taps > 1 ? size : 1);
    if (rc || rows == 0) return rc;
    if (!d_weight) return BLOAD_ERR_NULL;
    if (!on_4(d_weight, d_bias)) return BLOAD_ERR_ALIGN;
    if ((rc = check_channels(*x, rows, 1, size, true)) || (rc = check_channels(*y, rows, 1, size, false))) return rc;
    ConvParams p{};
    p.pos = d_pos;
    p.weight = d_weight;
    p.bias = d_bias;
    p.channels = channels;
    p.taps = taps;
    p.silu = silu != 0;
    return with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        return launch_conv_step<T>(p, rows, static_cast<const T*>(state), static_cast<T*>(next), static_cast<const T*>(x->data),
                                   row_stride(*x, rows), static_cast<T*>(y->data), row_stride(*y, rows), static_cast<cudaStream_t>(stream));
    });
}

size_t bload_scan_work_bytes(int64_t block_count, int32_t t_block, int64_t channels, int32_t states, int32_t gradient)
{
    if (block_count < 1 || t_block < 1 || t_block > BLOAD_MAX_T_BLOCK || !scan_fits(block_count, t_block, channels, states)) return 0;
    return scan_work_bytes(block_count, t_block, channels, states, gradient != 0);
}

int bload_scan(const bload_scan_t* a, void* stream)
{
    int rc = check_scan(a, false);
    if (rc || a->block_count == 0) return rc;
    return with_type(a->dtype, [&](auto zero) {
        using T = decltype(zero);
        return launch_scan<T>(scan_params(a, false), scan_tensors<T>(a, false), static_cast<cudaStream_t>(stream));
    });
}

int bload_scan_grad(const bload_scan_t* a, void* stream)
{
    int rc = check_scan(a, true);
    if (rc || a->block_count == 0) return rc;
    return with_type(a->dtype, [&](auto zero) {
        using T = decltype(zero);
        return launch_scan_grad<T>(scan_params(a, true), scan_tensors<T>(a, true), static_cast<cudaStream_t>(stream));
    });
}

int bload_scan_step(const bload_scan_step_t* a, void* stream)
{
    if (!a) return BLOAD_ERR_NULL;
    if (a->states < 1) return BLOAD_ERR_ARG;
    if (a->states > BLOAD_SCAN_MAX_STATES) return BLOAD_ERR_UNSUPPORTED;
    int rc = check_step(a->rows, a->channels, a->dtype, a->d_pos, a->state, a->next, 4);
    if (!rc && !fits_31(a->rows, a->channels / 8 + 1)) rc = BLOAD_ERR_ARG;
    if (rc || a->rows == 0) return rc;
    if (!a->d_a) return BLOAD_ERR_NULL;
    if (!on_4(a->d_a, a->d_d, a->d_dt_bias)) return BLOAD_ERR_ALIGN;
    const size_t size = size_of(a->dtype);
    auto tensor = [&](const bload_channels_t& x, bool zero_ok) { return check_channels(x, a->rows, 1, size, zero_ok); };
    if ((rc = tensor(a->x, true)) || (rc = tensor(a->dt, true)) || (rc = tensor(a->b, true)) || (rc = tensor(a->c, true)) ||
        (rc = tensor(a->y, false)))
        return rc;
    if (a->z.data && (rc = tensor(a->z, true))) return rc;
    const ScanStepParams p{a->d_pos, a->d_a, a->d_d, a->d_dt_bias, a->state, a->next, a->rows, a->channels, a->states, a->softplus != 0};
    return with_type(a->dtype, [&](auto zero) {
        using T = decltype(zero);
        const int64_t n = a->rows;
        auto in = [](const bload_channels_t& x) { return static_cast<const T*>(x.data); };
        const ScanStepTensors<T> t{in(a->x), in(a->dt), in(a->b), in(a->c), in(a->z), static_cast<T*>(a->y.data), row_stride(a->x, n),
                                   row_stride(a->dt, n), row_stride(a->b, n), row_stride(a->c, n), row_stride(a->z, n), row_stride(a->y, n)};
        return launch_scan_step<T>(p, t, static_cast<cudaStream_t>(stream));
    });
}

int64_t bload_device_timeouts(void) 
{
    const int64_t a = attention_timeouts(), r = recurrence_timeouts();
    return a < 0 || r < 0 ? -1 : a + r;
}

}  // extern "C"

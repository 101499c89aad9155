// Entry points of the layer products: checks, operands off the 16-byte grid, the layer path.
#include <algorithm>

#include "harp_internal.h"
#include "harp_linear.h"

namespace {

using namespace harp_linear;

constexpr int64_t kMostRows = 1ll << 30, kMostDim = 1ll << 20;
constexpr int64_t kMostDepthI8 = 131071;         // 128 * 128 * d_in stays below 2^31

bool aligned(const void *p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// One 16-byte piece of the padded copy a thread; the source is read by the aligned words that hold the bytes of the piece, which
// two neighbours make up a word of the result.  Weights (offsets given) are copied for the groups that have rows; offsets that fall
// make an empty group whatever they are clamped to.
__global__ void pad_rows_kernel(const uint8_t *__restrict__ src, int64_t pitch, int64_t rows, int64_t bytes, uint4 *__restrict__ dst, int64_t pieces,
                                const int32_t *__restrict__ offsets, int64_t group_rows) {
    const int64_t piece = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, at = piece * 16;
    if (piece >= pieces) return;
    for (int64_t r = (int64_t)blockIdx.y * blockDim.y + threadIdx.y; r < rows; r += (int64_t)gridDim.y * blockDim.y) {
        if (offsets) {
            const int64_t e = r / group_rows;
            if (offsets[e + 1] <= offsets[e]) continue;
        }
        const int64_t left = bytes - at;                             // bytes of the row from here on, 1 at least
        const uintptr_t p = reinterpret_cast<uintptr_t>(src + r * pitch + at);
        const uint32_t shift = (uint32_t)(p & 3) * 8;
        const uint32_t *const w = reinterpret_cast<const uint32_t *>(p & ~(uintptr_t)3);
        uint32_t v[5];
#pragma unroll
        for (int k = 0; k < 5; ++k) v[k] = 4 * k < (int64_t)(p & 3) + (left < 16 ? left : 16) ? w[k] : 0u;
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            o[k] = __funnelshift_r(v[k], v[k + 1], shift);
            const int64_t keep = left - 4 * k;                       // bytes of this word that belong to the row
            if (keep <= 0) o[k] = 0;
            else if (keep < 4) o[k] &= (1u << (8 * keep)) - 1u;
        }
        dst[r * pieces + piece] = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// An operand that the copy engine cannot address is copied to rows of whole 16-byte pieces first.
struct Operand {
    const void **ptr;
    int64_t *ld;
    int64_t rows, d;
    bool bad(int es) const { return !aligned(*ptr, 16) || *ld * es % 16 != 0; }
    int64_t pieces(int es) const { return (d * es + 15) / 16; }
};

// What a first call on a device asks for (attributes, a symbol's address, the pool) is no work of the stream: it may be asked for while
// this thread captures.
struct OutsideCapture {
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    OutsideCapture() { cudaThreadExchangeStreamCaptureMode(&mode); }
    ~OutsideCapture() { cudaThreadExchangeStreamCaptureMode(&mode); }
};

// for a CUDA call that failed: nothing of it stays behind for the next one, and an earlier failure is the one to tell
harp_status_t refused(harp_status_t earlier = HARP_OK) {
    cudaGetLastError();
    return earlier == HARP_OK ? HARP_ERR_CUDA : earlier;
}

harp_status_t run(Call c, cudaStream_t s) {
    const OutsideCapture outside;
    const Device *dev = device();
    if (!dev) return HARP_ERR_UNSUPPORTED;
    const int es = c.i8 ? 1 : 2;
    Operand ops[2] = {{&c.rows, &c.ld_rows, c.n_rows, c.d_rows},
                      {&c.other, &c.ld_other, c.product == GRAD_WEIGHTS ? c.n_rows : c.n_groups * c.d_out,
                       c.product == GRAD_WEIGHTS ? c.d_out : c.d_in}};
    int64_t bytes = 0;
    for (const Operand &o : ops)
        if (o.bad(es)) bytes += o.rows * o.pieces(es) * 16;
    if (bytes == 0) return gemm(c, *dev, s);
    int id = 0;
    if (cudaGetDevice(&id) != cudaSuccess) return refused();
    cudaMemPool_t pool = harp_scratch_pool(id);
    void *scratch = nullptr;
    if ((pool ? cudaMallocFromPoolAsync(&scratch, (size_t)bytes, pool, s) : cudaMallocAsync(&scratch, (size_t)bytes, s)) != cudaSuccess) {
        cudaGetLastError();
        return HARP_ERR_ALLOC;
    }
    uint8_t *to = static_cast<uint8_t *>(scratch);
    harp_status_t st = HARP_OK;
    for (const Operand &o : ops) {
        if (!o.bad(es)) continue;
        const bool weight = o.ptr == &c.other && c.product != GRAD_WEIGHTS;
        // 64 pieces of four rows a CTA, and as many CTAs as are resident at once
        const int64_t pieces = o.pieces(es), across = (pieces + 63) / 64;
        const int64_t down = std::max<int64_t>(1, std::min<int64_t>((o.rows + 3) / 4, (int64_t)dev->sms * 8 / across));
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)across, (unsigned)down);
        cfg.blockDim = dim3(64, 4);
        cfg.stream = s;
        // (its own status: cudaGetLastError would tell what an earlier call of this thread left)
        const cudaError_t err = cudaLaunchKernelEx(&cfg, pad_rows_kernel, static_cast<const uint8_t *>(*o.ptr), *o.ld * es, o.rows, o.d * es,
                                                   reinterpret_cast<uint4 *>(to), pieces, weight ? c.offsets : nullptr, c.d_out);
        g_harp_launches.fetch_add(1, std::memory_order_relaxed);
        if (err != cudaSuccess) {
            st = refused();
            break;
        }
        *o.ptr = to;
        *o.ld = pieces * 16 / es;
        to += o.rows * pieces * 16;
    }
    if (st == HARP_OK) st = gemm(c, *dev, s);
    if (cudaFreeAsync(scratch, s) != cudaSuccess) st = refused(st);
    return st;
}


harp_status_t check_sizes(int64_t n_rows, int64_t d_in, int64_t d_out, int64_t n_groups) {
    if (n_rows < 0 || d_in < 1 || d_out < 1 || n_groups < 1) return HARP_ERR_BAD_DIM;
    if (n_rows > kMostRows || d_in > kMostDim || d_out > kMostDim || n_groups > kMaxGroups) return HARP_ERR_TOO_LARGE;
    return HARP_OK;
}
harp_status_t check_ld(int64_t a, int64_t d_a, int64_t b, int64_t d_b, int64_t c, int64_t d_c) {
    if (a < d_a || b < d_b || c < d_c) return HARP_ERR_BAD_DIM;
    return a > kMostLd || b > kMostLd || c > kMostLd ? HARP_ERR_TOO_LARGE : HARP_OK;
}
harp_status_t check_out(const void *out, harp_dtype_t dtype) {
    return aligned(out, harp_dtype_size(dtype)) ? HARP_OK : HARP_ERR_BAD_DIM;
}

harp_status_t linear_i8(const int8_t *x, int64_t ld_x, const float *x_scale, const int8_t *w, int64_t ld_w, const float *w_scale,
                        const int32_t *offsets, bool grouped, int32_t n_groups, int64_t n_rows, int64_t d_in, int64_t d_out, void *y,
                        int64_t ld_y, harp_dtype_t y_dtype, void *stream) {
    if (y_dtype != HARP_F32 && y_dtype != HARP_BF16) return HARP_ERR_BAD_DTYPE;
    harp_status_t st = check_sizes(n_rows, d_in, d_out, n_groups);
    if (st != HARP_OK) return st;
    if (d_in > kMostDepthI8) return HARP_ERR_TOO_LARGE;
    if ((st = check_ld(ld_x, d_in, ld_w, d_in, ld_y, d_out)) != HARP_OK) return st;
    if (n_rows == 0) return HARP_OK;
    if (!x || !x_scale || !w || !w_scale || !y || (grouped && !offsets)) return HARP_ERR_NULL;
    if (!aligned(x_scale, 4) || !aligned(w_scale, 4) || !aligned(offsets, 4)) return HARP_ERR_BAD_DIM;
    if ((st = check_out(y, y_dtype)) != HARP_OK) return st;
    Call c;
    c.i8 = true;
    c.out_dtype = y_dtype;
    c.rows = x; c.ld_rows = ld_x; c.d_rows = d_in;
    c.other = w; c.ld_other = ld_w;
    c.n_rows = n_rows; c.d_in = d_in; c.d_out = d_out; c.n_groups = n_groups; c.offsets = offsets;
    c.row_scale = x_scale; c.channel_scale = w_scale;
    c.out = y; c.ld_out = ld_y;
    return run(c, static_cast<cudaStream_t>(stream));
}

}  // namespace

extern "C" {

harp_status_t harp_linear_i8(const int8_t *x, int64_t ld_x, const float *x_scale, const int8_t *w, int64_t ld_w, const float *w_scale,
                             int64_t n_rows, int64_t d_in, int64_t d_out, void *y, int64_t ld_y, harp_dtype_t y_dtype, void *stream) {
    return linear_i8(x, ld_x, x_scale, w, ld_w, w_scale, nullptr, false, 1, n_rows, d_in, d_out, y, ld_y, y_dtype, stream);
}

harp_status_t harp_grouped_linear_i8(const int8_t *x, int64_t ld_x, const float *x_scale, const int8_t *w, int64_t ld_w,
                                     const float *w_scale, const int32_t *offsets, int32_t n_groups, int64_t n_rows, int64_t d_in,
                                     int64_t d_out, void *y, int64_t ld_y, harp_dtype_t y_dtype, void *stream) {
    return linear_i8(x, ld_x, x_scale, w, ld_w, w_scale, offsets, true, n_groups, n_rows, d_in, d_out, y, ld_y, y_dtype, stream);
}

harp_status_t harp_grouped_linear(const void *x, int64_t ld_x, const void *w, int64_t ld_w, const int32_t *offsets, int32_t n_groups,
                                  int64_t n_rows, int64_t d_in, int64_t d_out, void *y, int64_t ld_y, harp_dtype_t y_dtype, void *stream) {
    if (y_dtype != HARP_F32 && y_dtype != HARP_BF16) return HARP_ERR_BAD_DTYPE;
    harp_status_t st = check_sizes(n_rows, d_in, d_out, n_groups);
    if (st != HARP_OK) return st;
    if ((st = check_ld(ld_x, d_in, ld_w, d_in, ld_y, d_out)) != HARP_OK) return st;
    if (n_rows == 0) return HARP_OK;
    if (!x || !w || !y || !offsets) return HARP_ERR_NULL;
    if (!aligned(x, 2) || !aligned(w, 2) || !aligned(offsets, 4)) return HARP_ERR_BAD_DIM;
    if ((st = check_out(y, y_dtype)) != HARP_OK) return st;
    Call c;
    c.out_dtype = y_dtype;
    c.rows = x; c.ld_rows = ld_x; c.d_rows = d_in;
    c.other = w; c.ld_other = ld_w;
    c.n_rows = n_rows; c.d_in = d_in; c.d_out = d_out; c.n_groups = n_groups; c.offsets = offsets;
    c.out = y; c.ld_out = ld_y;
    return run(c, static_cast<cudaStream_t>(stream));
}

harp_status_t harp_grouped_grad_rows(const void *gy, int64_t ld_gy, const void *w, int64_t ld_w, const int32_t *offsets, int32_t n_groups,
                                     int64_t n_rows, int64_t d_in, int64_t d_out, void *gx, int64_t ld_gx, harp_dtype_t gx_dtype,
                                     void *stream) {
    if (gx_dtype != HARP_F32 && gx_dtype != HARP_BF16) return HARP_ERR_BAD_DTYPE;
    harp_status_t st = check_sizes(n_rows, d_in, d_out, n_groups);
    if (st != HARP_OK) return st;
    if ((st = check_ld(ld_gy, d_out, ld_w, d_in, ld_gx, d_in)) != HARP_OK) return st;
    if (n_rows == 0) return HARP_OK;
    if (!gy || !w || !gx || !offsets) return HARP_ERR_NULL;
    if (!aligned(gy, 2) || !aligned(w, 2) || !aligned(offsets, 4)) return HARP_ERR_BAD_DIM;
    if ((st = check_out(gx, gx_dtype)) != HARP_OK) return st;
    Call c;
    c.product = GRAD_ROWS;
    c.out_dtype = gx_dtype;
    c.rows = gy; c.ld_rows = ld_gy; c.d_rows = d_out;
    c.other = w; c.ld_other = ld_w;
    c.n_rows = n_rows; c.d_in = d_in; c.d_out = d_out; c.n_groups = n_groups; c.offsets = offsets;
    c.out = gx; c.ld_out = ld_gx;
    return run(c, static_cast<cudaStream_t>(stream));
}

harp_status_t harp_grouped_grad_weights(const void *gy, int64_t ld_gy, const void *x, int64_t ld_x, const int32_t *offsets,
                                        int32_t n_groups, int64_t n_rows, int64_t d_in, int64_t d_out, void *gw, int64_t ld_gw,
                                        harp_dtype_t gw_dtype, int accumulate, void *stream) {
    if (gw_dtype != HARP_F32 && gw_dtype != HARP_BF16) return HARP_ERR_BAD_DTYPE;
    harp_status_t st = check_sizes(n_rows, d_in, d_out, n_groups);
    if (st != HARP_OK) return st;
    if ((st = check_ld(ld_gy, d_out, ld_x, d_in, ld_gw, d_in)) != HARP_OK) return st;
    if (!gw || (n_rows > 0 && (!gy || !x || !offsets))) return HARP_ERR_NULL;
    if (!aligned(gy, 2) || !aligned(x, 2) || !aligned(offsets, 4)) return HARP_ERR_BAD_DIM;
    if ((st = check_out(gw, gw_dtype)) != HARP_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (n_rows == 0) {
        const size_t es = harp_dtype_size(gw_dtype);
        if (accumulate) return HARP_OK;
        return cudaMemset2DAsync(gw, (size_t)ld_gw * es, 0, (size_t)d_in * es, (size_t)n_groups * (size_t)d_out, s) == cudaSuccess ? HARP_OK : refused();
    }
    Call c;
    c.product = GRAD_WEIGHTS;
    c.out_dtype = gw_dtype;
    c.rows = x; c.ld_rows = ld_x; c.d_rows = d_in;
    c.other = gy; c.ld_other = ld_gy;
    c.n_rows = n_rows; c.d_in = d_in; c.d_out = d_out; c.n_groups = n_groups; c.offsets = offsets;
    c.out = gw; c.ld_out = ld_gw;
    c.accumulate = accumulate ? 1 : 0;
    return run(c, s);
}

int64_t harp_processed_linear_scratch_bytes(const harp_plan_t *plan_in, int64_t n_rows) {
    if (!plan_in || n_rows < 0 || n_rows > kMostRows) return 0;
    return n_rows * ((plan_in->d + 15) / 16 * 16 + 4);
}

harp_status_t harp_processed_linear_i8(const harp_plan_t *plan_in, const harp_plan_t *plan_out, void *x, int64_t n_rows, harp_dtype_t dtype,
                                       const int8_t *w, int64_t ld_w, const float *w_scale, void *y, void *scratch, void *stream) {
    if (!plan_in || !plan_out) return HARP_ERR_NULL;
    if (dtype != HARP_F32 && dtype != HARP_BF16) return HARP_ERR_BAD_DTYPE;
    const int64_t d_in = plan_in->d, d_out = plan_out->d;
    harp_status_t st = check_sizes(n_rows, d_in, d_out, 1);
    if (st != HARP_OK) return st;
    if (d_in > kMostDepthI8) return HARP_ERR_TOO_LARGE;
    if (ld_w < d_in) return HARP_ERR_BAD_DIM;
    if (n_rows == 0) return HARP_OK;
    if (!x || !w || !w_scale || !y) return HARP_ERR_NULL;
    if ((st = check_out(x, dtype)) != HARP_OK || (st = check_out(y, dtype)) != HARP_OK) return st;
    if (!aligned(w_scale, 4) || !aligned(scratch, 16)) return HARP_ERR_BAD_DIM;
    int id = -1;
    if (cudaGetDevice(&id) != cudaSuccess) return refused();
    if (id != plan_in->device || id != plan_out->device) return HARP_ERR_DIM_MISMATCH;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    void *own = nullptr;
    if (!scratch) {
        const OutsideCapture outside;
        const size_t bytes = (size_t)harp_processed_linear_scratch_bytes(plan_in, n_rows);
        cudaMemPool_t pool = harp_scratch_pool(id);
        if ((pool ? cudaMallocFromPoolAsync(&own, bytes, pool, s) : cudaMallocAsync(&own, bytes, s)) != cudaSuccess) {
            cudaGetLastError();
            return HARP_ERR_ALLOC;
        }
    }
    const int64_t ld_q = (d_in + 15) / 16 * 16;
    int8_t *const q = static_cast<int8_t *>(own ? own : scratch);
    float *const scale = reinterpret_cast<float *>(q + n_rows * ld_q);
    st = harp_apply(plan_in, x, n_rows, dtype, 0, stream);
    if (st == HARP_OK) st = harp_quantize_rows(x, d_in, n_rows, d_in, dtype, q, ld_q, scale, stream);
    if (st == HARP_OK) st = harp_linear_i8(q, ld_q, scale, w, ld_w, w_scale, n_rows, d_in, d_out, y, d_out, dtype, stream);
    if (st == HARP_OK) st = harp_apply(plan_out, y, n_rows, dtype, 1, stream);
    if (own && cudaFreeAsync(own, s) != cudaSuccess) st = refused(st);
    return st;
}

int32_t harp_linear_error_word(void) {
    const Device *dev = device();
    int32_t word = 0;
    if (!dev || cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&word, dev->err, sizeof word, cudaMemcpyDeviceToHost) != cudaSuccess) {
        cudaGetLastError();
        return -1;
    }
    return word;
}

}  // extern "C"

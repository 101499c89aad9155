// Rows to 8 bits with one scale per row (harp_quantize_rows):
//
//   a = max_j |x_j|,  scale = a / 127,  q_j = the whole number nearest to 127 x_j / a (ties to even).
//
// Bound by memory: n d (element + 1) bytes.  A row is read once: its threads keep it in registers between the maximum
// and the quotients (eight 16-byte pieces a thread at most; rows beyond that are read again, from L2 as a rule).
//
// The quotient is rounded as if it were exact, so that the result depends on the definition alone and not on the order of its
// operations: x = a / 2 lies exactly between 63 and 64 in every row that holds it.  For bf16, 127 x has at most 15 significant bits and the
// correctly rounded fp32 quotient decides like the exact one; it takes a product with the correctly rounded reciprocal and one correction
// by the remainder (Markstein: Computation of elementary functions on the IBM RISC System/6000 processor, 1990).  For fp32 a quotient next to a tie is
// taken again in 64 bits.  Rows whose largest value is below 2^-60 or above 2^100 are first brought to the middle of the range by a power of two.
#include <algorithm>

#include "harp_internal.h"
#include "harp_linear.h"

namespace {

constexpr float kSmall = 0x1p-60f, kLarge = 0x1p100f;

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

struct RowScale {
    float up, most, inverse;        // power of two that the row is multiplied by; the largest value after it and its reciprocal
    bool valid;                     // false: the row is zero or not finite, its q are zero
};
__device__ __forceinline__ RowScale row_scale(uint32_t bits, float *scale) {
    RowScale s;
    const float most = __uint_as_float(bits);
    const bool finite = bits < 0x7f800000u;
    *scale = finite ? __fdiv_rn(most, 127.0f) : __uint_as_float(0x7fffffffu);
    s.valid = finite && bits != 0;
    s.up = most < kSmall ? 0x1p89f : most > kLarge ? 0x1p-100f : 1.0f;
    s.most = most * s.up;           // 2^-149 * 2^89 = 2^-60 at least, unless it is zero
    s.inverse = __frcp_rn(s.most);
    return s;
}
// bf16 values
__device__ __forceinline__ int quotient_bf16(float x, const RowScale &s) {
    const float a = x * s.up * 127.0f;
    float y = a * s.inverse;
    y = fmaf(fmaf(-y, s.most, a), s.inverse, y);
    return __float2int_rn(y);
}
__device__ __forceinline__ int quotient_f32(float x, const RowScale &s) {
    x *= s.up;
    const float y = x * s.inverse * 127.0f;
    const float r = rintf(y);
    if (fabsf(fabsf(y - r) - 0.5f) < 1e-4f) return __double2int_rn(127.0 * (double)x / (double)s.most);
    return (int)r;
}
template <typename T> __device__ __forceinline__ int quotient(T x, const RowScale &s);
template <> __device__ __forceinline__ int quotient<float>(float x, const RowScale &s) { return quotient_f32(x, s); }
template <> __device__ __forceinline__ int quotient<__nv_bfloat16>(__nv_bfloat16 x, const RowScale &s) { return quotient_bf16(__bfloat162float(x), s); }

__device__ __forceinline__ uint32_t largest(uint32_t m, const uint4 &v, float) {
    return max(max(max(m, v.x & 0x7fffffffu), v.y & 0x7fffffffu), max(v.z & 0x7fffffffu, v.w & 0x7fffffffu));
}
// the larger of either half, as two 16-bit maxima in one register
__device__ __forceinline__ uint32_t largest(uint32_t m, const uint4 &v, __nv_bfloat16) {
    m = __vmaxu2(m, __vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu));
    return __vmaxu2(m, __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
}
__device__ __forceinline__ uint32_t as_f32_bits(uint32_t m, float) { return m; }
__device__ __forceinline__ uint32_t as_f32_bits(uint32_t m, __nv_bfloat16) { return max(m & 0xffffu, m >> 16) << 16; }

__device__ __forceinline__ uint32_t pack(int a, int b, int c, int d) {
    return __byte_perm(__byte_perm((uint32_t)a, (uint32_t)b, 0x0040), __byte_perm((uint32_t)c, (uint32_t)d, 0x0040), 0x5410);
}
__device__ __forceinline__ void put(int8_t *q, const uint4 &v, const RowScale &s, float) {
    uint32_t r = 0;
    if (s.valid) r = pack(quotient_f32(__uint_as_float(v.x), s), quotient_f32(__uint_as_float(v.y), s),
                          quotient_f32(__uint_as_float(v.z), s), quotient_f32(__uint_as_float(v.w), s));
    *reinterpret_cast<uint32_t *>(q) = r;
}
__device__ __forceinline__ void put(int8_t *q, const uint4 &v, const RowScale &s, __nv_bfloat16) {
    uint2 r = make_uint2(0, 0);
    if (s.valid) {
        auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
        auto hi = [](uint32_t w) { return __uint_as_float(w & 0xffff0000u); };
        r.x = pack(quotient_bf16(lo(v.x), s), quotient_bf16(hi(v.x), s), quotient_bf16(lo(v.y), s), quotient_bf16(hi(v.y), s));
        r.y = pack(quotient_bf16(lo(v.z), s), quotient_bf16(hi(v.z), s), quotient_bf16(lo(v.w), s), quotient_bf16(hi(v.w), s));
    }
    *reinterpret_cast<uint2 *>(q) = r;
}

// the largest of a row's threads: threadIdx.x within the row, threadIdx.y the row of the CTA
__device__ __forceinline__ uint32_t row_max(uint32_t m) {
    __shared__ uint32_t part[32];
    m = __reduce_max_sync(~0u, m);
    const int warps = blockDim.x >> 5;
    if (warps == 1) return m;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) part[threadIdx.y * warps + warp] = m;
    __syncthreads();
    return __reduce_max_sync(~0u, lane < warps ? part[threadIdx.y * warps + lane] : 0u);
}

// PIECES 16-byte pieces a thread in registers; 0: any row, element by element, read twice
template <typename T, int PIECES>
__global__ void __launch_bounds__(1024) quantize_kernel(const T *__restrict__ x, int64_t ld_x, int64_t n_rows, int64_t d, int8_t *__restrict__ q, int64_t ld_q,
                                float *__restrict__ scale) {
    constexpr int V = 16 / (int)sizeof(T);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const bool inside = row < n_rows;
    const T *const xr = x + row * ld_x;
    int8_t *const qr = q + row * ld_q;
    uint32_t m = 0;
    if constexpr (PIECES > 0) {
        uint4 v[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int64_t at = ((int64_t)i * blockDim.x + threadIdx.x) * V;
            v[i] = make_uint4(0, 0, 0, 0);
            if (inside && at < d) v[i] = *reinterpret_cast<const uint4 *>(xr + at);
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) m = largest(m, v[i], T());
        m = as_f32_bits(m, T());
        m = row_max(m);
        float sc;
        const RowScale s = row_scale(m, &sc);
        if (!inside) return;
        if (threadIdx.x == 0) scale[row] = sc;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int64_t at = ((int64_t)i * blockDim.x + threadIdx.x) * V;
            if (at < d) put(qr + at, v[i], s, T());
        }
    } else {
        if (inside)
            for (int64_t j = threadIdx.x; j < d; j += blockDim.x) m = max(m, magnitude((float)xr[j]));
        m = row_max(m);
        float sc;
        const RowScale s = row_scale(m, &sc);
        if (!inside) return;
        if (threadIdx.x == 0) scale[row] = sc;
        for (int64_t j = threadIdx.x; j < d; j += blockDim.x) qr[j] = (int8_t)(s.valid ? quotient<T>(xr[j], s) : 0);
    }
}

template <typename T, int PIECES>
cudaError_t launch(const T *x, int64_t ld_x, int64_t n_rows, int64_t d, int8_t *q, int64_t ld_q, float *scale, int threads, cudaStream_t s) {
    const int rows = threads >= 128 ? 1 : 128 / threads;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((n_rows + rows - 1) / rows));
    cfg.blockDim = dim3((unsigned)threads, (unsigned)rows);
    cfg.stream = s;
    cudaLaunchAttribute la;
    la.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    la.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &la;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, quantize_kernel<T, PIECES>, x, ld_x, n_rows, d, q, ld_q, scale);
}

template <typename T>
harp_status_t quantize(const T *x, int64_t ld_x, int64_t n_rows, int64_t d, int8_t *q, int64_t ld_q, float *scale, cudaStream_t s) {
    constexpr int V = 16 / (int)sizeof(T);
    const bool wide = reinterpret_cast<uintptr_t>(x) % 16 == 0 && ld_x % V == 0 && d % V == 0 &&
                      reinterpret_cast<uintptr_t>(q) % V == 0 && ld_q % V == 0;
    const int64_t pieces = (d + V - 1) / V;
    cudaError_t err;
    auto threads = [&](int each) { return (int)((pieces + 32 * each - 1) / (32 * each) * 32); };
    if (!wide || pieces > 8 * 1024) err = launch<T, 0>(x, ld_x, n_rows, d, q, ld_q, scale, (int)std::min<int64_t>(1024, (d + 127) / 128 * 32), s);
    else if (pieces <= 1024 && n_rows <= 296) err = launch<T, 1>(x, ld_x, n_rows, d, q, ld_q, scale, threads(1), s);
    else if (pieces <= 2048 && n_rows <= 296) err = launch<T, 2>(x, ld_x, n_rows, d, q, ld_q, scale, threads(2), s);
    else if (pieces <= 4096) err = launch<T, 4>(x, ld_x, n_rows, d, q, ld_q, scale, threads(4), s);
    else err = launch<T, 8>(x, ld_x, n_rows, d, q, ld_q, scale, threads(8), s);
    g_harp_launches.fetch_add(1, std::memory_order_relaxed);
    if (err != cudaSuccess) {
        cudaGetLastError();
        return HARP_ERR_CUDA;
    }
    return HARP_OK;
}

}  // namespace

extern "C" harp_status_t harp_quantize_rows(const void *x, int64_t ld_x, int64_t n_rows, int64_t d, harp_dtype_t dtype,
                                            int8_t *q, int64_t ld_q, float *scale, void *stream) {
    if (dtype != HARP_F32 && dtype != HARP_BF16) return HARP_ERR_BAD_DTYPE;
    if (n_rows < 0 || n_rows > INT32_MAX || d < 1 || d > (1ll << 20) || ld_x < d || ld_q < d) return HARP_ERR_BAD_DIM;
    if (n_rows == 0) return HARP_OK;
    if (!x || !q || !scale) return HARP_ERR_NULL;
    const uintptr_t es = dtype == HARP_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(x) % es || reinterpret_cast<uintptr_t>(scale) % 4) return HARP_ERR_BAD_DIM;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return dtype == HARP_F32 ? quantize(static_cast<const float *>(x), ld_x, n_rows, d, q, ld_q, scale, s)
                             : quantize(static_cast<const __nv_bfloat16 *>(x), ld_x, n_rows, d, q, ld_q, scale, s);
}

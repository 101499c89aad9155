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
// settled by the remainder.  Rows whose largest value is below 2^-60 or above 2^100 are first brought to the middle of the range by a power of two.
#include <algorithm>

#include "harp_internal.h"
#include "harp_linear.h"

namespace {

constexpr float kSmall = 0x1p-60f, kLarge = 0x1p100f;

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

struct RowScale {
    float up, most;                 // power of two that the row is multiplied by; the largest value after it
    float factor, inverse;          // bf16: 127 up and 1 / most; fp32: up and 127 / most
    bool valid;                     // false: the row is zero or not finite, its q are zero
};
template <typename T>
__device__ __forceinline__ RowScale row_scale(uint32_t bits, float *scale) {
    RowScale s;
    const float most = __uint_as_float(bits);
    const bool finite = bits < 0x7f800000u;
    *scale = finite ? __fdiv_rn(most, 127.0f) : __uint_as_float(0x7fffffffu);
    s.valid = finite && bits != 0;
    s.up = most < kSmall ? 0x1p89f : most > kLarge ? 0x1p-100f : 1.0f;
    s.most = most * s.up;           // 2^-149 * 2^89 = 2^-60 at least, unless it is zero
    s.factor = sizeof(T) == 2 ? 127.0f * s.up : s.up;
    s.inverse = sizeof(T) == 2 ? __frcp_rn(s.most) : __fdiv_rn(127.0f, s.most);
    return s;
}

// A value of magnitude up to 127 plus 1.5 * 2^23 is rounded to the nearest whole number, ties to even, and has it in its low byte.
constexpr float kRound = 12582912.0f;

// bf16: the sum that holds q in its low byte
__device__ __forceinline__ uint32_t quotient(float x, const RowScale &s, __nv_bfloat16) {
    const float a = x * s.factor;
    float y = a * s.inverse;
    y = fmaf(fmaf(-y, s.most, a), s.inverse, y);
    return __float_as_uint(y + kRound);
}
// fp32: the same, and whether the quotient, which two roundings put off by 2^-16 at most, is next to a tie
__device__ __forceinline__ uint32_t quotient(float x, const RowScale &s, bool &near) {
    const float y = x * s.factor * s.inverse, r = y + kRound;
    near |= fabsf(y - (r - kRound)) > 0.49995f;
    return __float_as_uint(r);
}
// Next to the tie c / 2 (c odd) the sign of 254 |x| - c most decides.  Either product is a rounded value and its error, which fma gives
// exactly; the rounded ones are within a factor of two, so their difference is exact, and that of the errors, of eight bits each, is too.
__device__ __forceinline__ uint32_t exact_quotient(float x, const RowScale &s) {
    const float v = fabsf(x * s.up), c = rintf(2.0f * v * s.inverse);
    const float p = 254.0f * v, t = c * s.most, d = (p - t) + (fmaf(254.0f, v, -p) - fmaf(c, s.most, -t));
    const int odd = __float2int_rn(c), low = odd >> 1;
    const int q = d > 0.0f ? low + 1 : d < 0.0f ? low : low + (low & 1);
    return (uint32_t)(x < 0.0f ? -q : q);
}

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

__device__ __forceinline__ uint32_t pack(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t settled(float x, const RowScale &s) {
    bool near = false;
    const uint32_t r = quotient(x, s, near);
    return near ? exact_quotient(x, s) : r;
}
__device__ __forceinline__ void put(int8_t *q, const uint4 &v, const RowScale &s, float) {
    const float x = __uint_as_float(v.x), y = __uint_as_float(v.y), z = __uint_as_float(v.z), w = __uint_as_float(v.w);
    bool near = false;
    uint32_t r = pack(quotient(x, s, near), quotient(y, s, near), quotient(z, s, near), quotient(w, s, near));
    if (near) r = pack(settled(x, s), settled(y, s), settled(z, s), settled(w, s));
    *reinterpret_cast<uint32_t *>(q) = s.valid ? r : 0u;
}
__device__ __forceinline__ void put(int8_t *q, const uint4 &v, const RowScale &s, __nv_bfloat16 b) {
    auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
    auto hi = [](uint32_t w) { return __uint_as_float(w & 0xffff0000u); };
    const uint32_t x = pack(quotient(lo(v.x), s, b), quotient(hi(v.x), s, b), quotient(lo(v.y), s, b), quotient(hi(v.y), s, b));
    const uint32_t y = pack(quotient(lo(v.z), s, b), quotient(hi(v.z), s, b), quotient(lo(v.w), s, b), quotient(hi(v.w), s, b));
    *reinterpret_cast<uint2 *>(q) = s.valid ? make_uint2(x, y) : make_uint2(0, 0);
}
__device__ __forceinline__ int8_t one(float x, const RowScale &s) { return (int8_t)(s.valid ? settled(x, s) : 0u); }
__device__ __forceinline__ int8_t one(__nv_bfloat16 x, const RowScale &s) { return (int8_t)(s.valid ? quotient(__bfloat162float(x), s, x) : 0u); }

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

// Rows off the 16-byte grid: element by element, ELEMS of them a thread in registers; 0: read twice
template <typename T, int ELEMS>
__global__ void __launch_bounds__(1024) quantize_any_kernel(const T *__restrict__ x, int64_t ld_x, int64_t n_rows, int64_t d, int8_t *__restrict__ q,
                                                            int64_t ld_q, float *__restrict__ scale) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const bool inside = row < n_rows;
    const T *const xr = x + row * ld_x;
    int8_t *const qr = q + row * ld_q;
    uint32_t m = 0;
    T v[ELEMS ? ELEMS : 1];
    if constexpr (ELEMS > 0) {
#pragma unroll
        for (int i = 0; i < ELEMS; ++i) {
            const int64_t j = (int64_t)i * blockDim.x + threadIdx.x;
            v[i] = inside && j < d ? xr[j] : T(0.0f);
        }
#pragma unroll
        for (int i = 0; i < ELEMS; ++i) m = max(m, magnitude((float)v[i]));
    } else if (inside) {
        for (int64_t j = threadIdx.x; j < d; j += blockDim.x) m = max(m, magnitude((float)xr[j]));
    }
    m = row_max(m);
    float sc;
    const RowScale s = row_scale<T>(m, &sc);
    if (!inside) return;
    if (threadIdx.x == 0) scale[row] = sc;
    if constexpr (ELEMS > 0) {
#pragma unroll
        for (int i = 0; i < ELEMS; ++i) {
            const int64_t j = (int64_t)i * blockDim.x + threadIdx.x;
            if (j < d) qr[j] = one(v[i], s);
        }
    } else {
        for (int64_t j = threadIdx.x; j < d; j += blockDim.x) qr[j] = one(xr[j], s);
    }
}

// PIECES 16-byte pieces a thread in registers.  THREADS: most threads a CTA
template <typename T, int PIECES, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? PIECES == 8 ? 4 : 6 : THREADS == 512 ? 2 : 1) quantize_kernel(const T *__restrict__ x, int64_t ld_x, int64_t n_rows, int64_t d, int8_t *__restrict__ q, int64_t ld_q,
                                float *__restrict__ scale) {
    constexpr int V = 16 / (int)sizeof(T);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const bool inside = row < n_rows;
    const T *const xr = x + row * ld_x;
    int8_t *const qr = q + row * ld_q;
    uint32_t m = 0;
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
    const RowScale s = row_scale<T>(m, &sc);
    if (!inside) return;
    if (threadIdx.x == 0) scale[row] = sc;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int64_t at = ((int64_t)i * blockDim.x + threadIdx.x) * V;
        if (at < d) put(qr + at, v[i], s, T());
    }
}

template <typename T>
cudaError_t launch(void (*kernel)(const T *, int64_t, int64_t, int64_t, int8_t *, int64_t, float *), const T *x, int64_t ld_x, int64_t n_rows,
                   int64_t d, int8_t *q, int64_t ld_q, float *scale, int64_t threads, cudaStream_t s) {
    const int64_t rows = threads >= 128 ? 1 : 128 / threads;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((n_rows + rows - 1) / rows));
    cfg.blockDim = dim3((unsigned)threads, (unsigned)rows);
    cfg.stream = s;
    cudaLaunchAttribute la;
    la.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    la.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &la;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, x, ld_x, n_rows, d, q, ld_q, scale);
}

template <typename T>
harp_status_t quantize(const T *x, int64_t ld_x, int64_t n_rows, int64_t d, int8_t *q, int64_t ld_q, float *scale, cudaStream_t s) {
    constexpr int V = 16 / (int)sizeof(T);
    const bool wide = reinterpret_cast<uintptr_t>(x) % 16 == 0 && ld_x % V == 0 && d % V == 0 &&
                      reinterpret_cast<uintptr_t>(q) % V == 0 && ld_q % V == 0;
    const int64_t pieces = (d + V - 1) / V;
    // pieces a thread: one or two where few rows leave the machine to latency; four, or eight in wide rows, so that several CTAs of a row share an SM
    auto run = [&](auto kernel, int64_t units, int each) {
        return launch<T>(kernel, x, ld_x, n_rows, d, q, ld_q, scale, (units + 32 * each - 1) / (32 * each) * 32, s);
    };
    cudaError_t err;
    if (!wide && d <= 16 * 1024) err = run(quantize_any_kernel<T, 16>, d, 16);
    else if (!wide || pieces > 8 * 1024) err = run(quantize_any_kernel<T, 0>, 1024, 1);
    else if (pieces <= 1024 && n_rows <= 296) err = run(quantize_kernel<T, 1, 1024>, pieces, 1);
    else if (pieces <= 2048 && n_rows <= 296) err = run(quantize_kernel<T, 2, 1024>, pieces, 2);
    else if (pieces <= 4 * 256) err = run(quantize_kernel<T, 4, 256>, pieces, 4);
    else if (pieces <= 8 * 256) err = run(quantize_kernel<T, 8, 256>, pieces, 8);
    else if (pieces <= 8 * 512) err = run(quantize_kernel<T, 8, 512>, pieces, 8);
    else err = run(quantize_kernel<T, 8, 1024>, pieces, 8);
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
    if (ld_x > harp_linear::kMostLd || ld_q > harp_linear::kMostLd) return HARP_ERR_TOO_LARGE;
    if (n_rows == 0) return HARP_OK;
    if (!x || !q || !scale) return HARP_ERR_NULL;
    const uintptr_t es = dtype == HARP_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(x) % es || reinterpret_cast<uintptr_t>(scale) % 4) return HARP_ERR_BAD_DIM;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return dtype == HARP_F32 ? quantize(static_cast<const float *>(x), ld_x, n_rows, d, q, ld_q, scale, s)
                             : quantize(static_cast<const __nv_bfloat16 *>(x), ld_x, n_rows, d, q, ld_q, scale, s);
}

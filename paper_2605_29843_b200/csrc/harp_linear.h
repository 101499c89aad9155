// Declarations shared by the translation units of the layer products (harp_linear.cu: entry points, harp_gemm.cu: the
// kernel, harp_quantize.cu: rows to 8 bits).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "harp.h"

namespace harp_linear {

// Which of the three products of a layer: y = x W^T, dx = dy W, dW = dy^T x (per group).
enum Product { FORWARD = 0, GRAD_ROWS = 1, GRAD_WEIGHTS = 2 };

constexpr int64_t kMostLd = 1ll << 37;   // leading dimensions: the copy engine's rows lie less than 2^40 bytes apart
constexpr int kMaxGroups = 1024;         // offsets and tile counts of all groups stay in shared memory

// One call, after its checks.  `lanes` is the dimension that lies along the lanes of tensor memory and contiguous in the
// output (d_out, d_in, d_in), `cols` the other output dimension (rows of the batch, rows, d_out), `depth` the contracted one
// (d_in, d_out, rows of the group).
struct Call {
    Product product = FORWARD;
    bool i8 = false;                     // 8-bit operands with scales; bf16 otherwise
    harp_dtype_t out_dtype = HARP_BF16;
    const void *rows = nullptr;          // x (FORWARD, GRAD_WEIGHTS) or dy (GRAD_ROWS): n_rows x d_rows
    int64_t ld_rows = 0, d_rows = 0;
    const void *other = nullptr;         // w: n_groups x d_out x d_in; dy: n_rows x d_out for GRAD_WEIGHTS
    int64_t ld_other = 0;
    int64_t n_rows = 0, d_in = 0, d_out = 0;
    int32_t n_groups = 1;
    const int32_t *offsets = nullptr;    // device, n_groups + 1; null: one group of all rows
    const float *row_scale = nullptr, *channel_scale = nullptr;
    void *out = nullptr;
    int64_t ld_out = 0;
    int accumulate = 0;
};

struct Device {
    int sms = 0, pairs = 0;              // SMs; CTA pairs of the product kernel that are resident at once
    int clusters[3] = {};                // ... clusters of 1, 2 and 4 CTAs that divide the contracted dimension, two CTAs an SM
    int32_t *err = nullptr;              // device word: a wait gave up
};
// of the current device; null where the driver or the device cannot run these kernels
const Device *device();

harp_status_t gemm(const Call &c, const Device &dev, cudaStream_t stream);          // operands on 16-byte boundaries

}  // namespace harp_linear

// Products of a 4-bit matrix with several rows of activations (mx_batch.cu), as mx.cu calls them.
#pragma once
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "ctx.h"

namespace llvq {

size_t mx_batch_bytes(const llvq_ctx* ctx, int64_t n_out, int64_t k_in, int batch);
int mx_batch_product(const llvq_ctx* ctx, const uint8_t* d_codes, const uint8_t* d_scales, int64_t n_out, int64_t k_in, const uint16_t* d_x, int batch,
                     uint16_t* d_y, uint8_t* work, cudaStream_t st);

}  // namespace llvq

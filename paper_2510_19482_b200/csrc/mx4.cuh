// Microscaled 4-bit floating point: what the quantiser and the products share.
//
//   codes    uint8 [rows][K/2], two E2M1 values to a byte, the even column in the low half
//   scales   uint8 [rows][K/B]: MXFP4 B = 32, E8M0 (2^(byte - 127), 255 = NaN); NVFP4 B = 16, E4M3 (sign bit clear, 127 = NaN)
#pragma once

#include "common.cuh"

namespace elutq {

inline int mx4_block(int format) { return format == ELUTQ_MX4_MXFP4 ? 32 : 16; }

// The arguments of every entry that are the same: a format, and a K that fills whole blocks and 16-byte pieces of codes.
inline int mx4_check(int format, int rows, int K) {
    if (rows <= 0 || K <= 0) return ELUTQ_ERR_INVALID_ARG;
    if (format != ELUTQ_MX4_MXFP4 && format != ELUTQ_MX4_NVFP4) return ELUTQ_ERR_INVALID_ARG;
    return K % 32 != 0 ? ELUTQ_ERR_SHAPE : ELUTQ_OK;
}
inline bool mx4_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// The status words of the 4-bit products, one a device (mx4_gemm.cu); a cudaError_t value each.  The current device's, copied in `stream` (which is waited for): no CUDA
// call but the device's number where no product has been launched on it.  Clearing: of every device that one has been launched on, which is waited for.
int mx4_status(unsigned* word, cudaStream_t stream);
int mx4_clear_status();

}  // namespace elutq

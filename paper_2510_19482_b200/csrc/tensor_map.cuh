// The driver's encoder of TMA descriptors, found at run time (the library is not linked against the driver).
#pragma once

#include <cuda.h>

namespace elutq {

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                   const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled_fn();       // hlq_tmem.cu; null: the driver has none

}  // namespace elutq

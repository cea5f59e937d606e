// Host-side services that the library's translation units share (not exported).
#pragma once

#include <cuda.h>
#include <stddef.h>

namespace csd {
namespace host {

#define CSD_LOCAL __attribute__((visibility("hidden")))

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

CSD_LOCAL EncodeTiledFn encode_tiled();   // the driver's tensor-map encoder, or nullptr
CSD_LOCAL int multiprocessors();          // of the current device; 148 where none can be asked
CSD_LOCAL void other_work_enqueued();     // voids the record of which step preceded which (csd_set_overlap)

}  // namespace host
}  // namespace csd

// The decode kernel's instantiations with modified scores and masks, and those over chosen pages, live in translation units of their
// own (scored_api.cu, selected_api.cu).
#pragma once

#include "common.cuh"
#include "host_common.h"

namespace pdattn {

// Launches decode_kernel<.., MOD> (chained merge) for the given head size, page size, row tiles (8 or 16) and cache type.
PDATTN_HIDDEN pdattn_status launch_scored_decode(const CUtensorMap& mk, const CUtensorMap& mv, const DecodeParams& P,
                                                 int head_dim, int block_size, bool nt2, bool fp8, int grid,
                                                 cudaStream_t stream, bool dependent);
// ... decode_kernel<.., SEL>
PDATTN_HIDDEN pdattn_status launch_selected_decode(const CUtensorMap& mk, const CUtensorMap& mv, const DecodeParams& P,
                                                   int head_dim, int block_size, bool nt2, bool fp8, int grid,
                                                   cudaStream_t stream, bool dependent);

}  // namespace pdattn

// Instantiations and launch of the decode kernel over chosen pages (see scored.h).
#include "scored.h"
#include "variant_launch.cuh"

namespace pdattn {

pdattn_status launch_selected_decode(const CUtensorMap& mk, const CUtensorMap& mv, const DecodeParams& P, int head_dim,
                                     int block_size, bool nt2, bool fp8, int grid, cudaStream_t stream, bool dependent) {
  return launch_variant<false, true>(mk, mv, P, head_dim, block_size, nt2, fp8, grid, stream, dependent);
}

}  // namespace pdattn

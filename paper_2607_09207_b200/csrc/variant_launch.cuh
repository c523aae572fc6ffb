// Launch of the decode kernel's chained-merge instantiations with modified scores (MOD) or chosen pages (SEL).  Each of the two
// is instantiated in a translation unit of its own (scored_api.cu, selected_api.cu): they take the compiler a while.
#pragma once

#include "decode.cuh"
#include "host_common.h"

namespace pdattn {

namespace {

template <bool MOD, bool SEL, int D, int NT, int BS, int EB>
pdattn_status launch_one(const CUtensorMap& mk, const CUtensorMap& mv, const DecodeParams& P, int grid, cudaStream_t stream,
                         bool dependent) {
  using C = Cfg<D, NT, BS, EB>;
  auto kern = decode_kernel<D, NT, BS, false, true, EB, false, MOD, SEL>;
  static bool attr_set[kMaxDevices] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail("cudaGetDevice", e);
  if (dev < 0 || dev >= kMaxDevices) return PDATTN_UNSUPPORTED;
  if (!attr_set[dev]) {
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::CHAIN_DYN_BYTES);
    if (e != cudaSuccess) return cuda_fail("cudaFuncSetAttribute", e);
    attr_set[dev] = true;
  }
  e = launch_dependent(kern, grid, C::NTHREADS, C::CHAIN_DYN_BYTES, stream, dependent, mk, mv, P);
  if (e != cudaSuccess) return cuda_fail("decode_kernel launch", e);
  return PDATTN_OK;
}

template <bool MOD, bool SEL, int D, int NT, int BS>
pdattn_status launch_eb(const CUtensorMap& mk, const CUtensorMap& mv, const DecodeParams& P, bool fp8, int grid,
                        cudaStream_t stream, bool dependent) {
  return fp8 ? launch_one<MOD, SEL, D, NT, BS, 1>(mk, mv, P, grid, stream, dependent)
             : launch_one<MOD, SEL, D, NT, BS, 2>(mk, mv, P, grid, stream, dependent);
}

template <bool MOD, bool SEL, int D, int NT>
pdattn_status launch_bs(const CUtensorMap& mk, const CUtensorMap& mv, const DecodeParams& P, int block_size, bool fp8,
                        int grid, cudaStream_t stream, bool dependent) {
  return block_size == 64   ? launch_eb<MOD, SEL, D, NT, 64>(mk, mv, P, fp8, grid, stream, dependent)
         : block_size == 32 ? launch_eb<MOD, SEL, D, NT, 32>(mk, mv, P, fp8, grid, stream, dependent)
                            : launch_eb<MOD, SEL, D, NT, 16>(mk, mv, P, fp8, grid, stream, dependent);
}

template <bool MOD, bool SEL>
pdattn_status launch_variant(const CUtensorMap& mk, const CUtensorMap& mv, const DecodeParams& P, int head_dim, int block_size,
                             bool nt2, bool fp8, int grid, cudaStream_t stream, bool dependent) {
  if (head_dim == 128)
    return nt2 ? launch_bs<MOD, SEL, 128, 2>(mk, mv, P, block_size, fp8, grid, stream, dependent)
               : launch_bs<MOD, SEL, 128, 1>(mk, mv, P, block_size, fp8, grid, stream, dependent);
  return nt2 ? launch_bs<MOD, SEL, 64, 2>(mk, mv, P, block_size, fp8, grid, stream, dependent)
             : launch_bs<MOD, SEL, 64, 1>(mk, mv, P, block_size, fp8, grid, stream, dependent);
}

}  // namespace

}  // namespace pdattn

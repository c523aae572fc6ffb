// Device code of libpdattn (sm_100a only), one header per part:
//   common.cuh       constants, kernel parameters, PTX wrappers, shared-memory plan, span walk and sequencing
//   tile_bf16.cuh    one 64-token tile on one warp, bf16 cache
//   tile_fp8.cuh     the same over an fp8 (e4m3) cache
//   decode.cuh       decode_kernel: persistent split-KV flash decoding (chained or barrier merge at piece end)
//   prefix_mma.cuh   prefix_kernel: shared prompt tiles of a GRPO group, warp-level MMAs
//   prefix_umma.cuh  prefix_umma_kernel: the same on tcgen05 with tensor-memory operands (included by the API file)
//   aux_kernels.cuh  append_kernel, append_fp8_kernel, stream_read_kernel, combine_kernel, plan_kernel
// and, in translation units of their own:
//   rope.cuh, pages.cuh   rope_append_kernel; the page bookkeeping (ops_api.cu)
//   prefill_umma.cuh      prefill_kernel, prefill_join_kernel: prompt attention on tcgen05 (prefill_api.cu)
//   tree_umma.cuh         tree_kernel, tree_join_kernel: trees of drafted tokens on tcgen05 (tree_api.cu)
//   summary.cuh, accept.cuh   summarize_kernel, select_kernel: pages chosen by their keys' bounds; accept_kernel (sparse_api.cu)
//   scored_api.cu         decode_kernel with modified scores and masks (scored.h)
//   selected_api.cu       decode_kernel over chosen pages (scored.h); both by variant_launch.cuh
// umma.cuh holds the tcgen05 wrappers that the tensor-memory kernels use, host_common.h what the host sides share.
#pragma once

#include "common.cuh"
#include "tile_bf16.cuh"
#include "tile_fp8.cuh"
#include "decode.cuh"
#include "prefix_mma.cuh"
#include "aux_kernels.cuh"

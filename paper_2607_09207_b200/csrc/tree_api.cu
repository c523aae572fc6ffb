// Host side of pdattn_decode_tree: argument checks, tensor maps, launch.
#include <cstdio>
#include <type_traits>

#include "../../include/pdattn.h"
#include "host_common.h"
#include "tree_umma.cuh"

namespace {

using namespace pdattn;

constexpr size_t kTreeRec = WS_CLEARED_BYTES;                                                   // [TR_CTAS][2][2] int4
constexpr size_t kTreePartials = (kTreeRec + TR_CTAS * 4 * sizeof(int4) + 255) / 256 * 256;
size_t part_bytes(int head_dim) { return static_cast<size_t>(2) * (head_dim + 2) * 128 * 4; }   // of one piece: two row tiles

template <int D, bool PAIR, int EB>
pdattn_status launch_tree(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const TreeParams& P, int dev, int grid,
                          cudaStream_t stream) {
  using C = TreeCfg<D, PAIR, EB>;
  auto kern = tree_kernel<D, PAIR, EB>;
  static bool attr_set[kMaxDevices] = {};
  if (!attr_set[dev]) {
    // the kernel re-deals its launch registers (see there): a build that launches with fewer would wait for good
    cudaFuncAttributes fa;
    cudaError_t e = cudaFuncGetAttributes(&fa, kern);
    if (e != cudaSuccess) return cuda_fail("cudaFuncGetAttributes", e);
    if (fa.numRegs != TR_LAUNCH_REGS) {
      snprintf(cuda_error_text(), kCudaErrorTextBytes, "tree_kernel was built with %d registers a thread, %d are wanted", fa.numRegs,
               TR_LAUNCH_REGS);
      return PDATTN_CUDA_ERROR;
    }
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::DYN_BYTES);
    if (e != cudaSuccess) return cuda_fail("cudaFuncSetAttribute", e);
    attr_set[dev] = true;
  }
  cudaError_t e = launch_dependent(kern, grid, TR_NTHREADS, C::DYN_BYTES, stream, true, mq, mk, mv, P);
  if (e != cudaSuccess) return cuda_fail("tree_kernel launch", e);
  // no unit that a row of the table can describe is long enough to be cut: nothing to join
  if ((static_cast<int64_t>(P.MB) << P.bs_log2) <= (2 * kTreeMinCut - 1) * kTreeKeys) return PDATTN_OK;
  e = launch_dependent(tree_join_kernel<D, PAIR>, dim3(grid, PAIR ? 2 : 1, D / TR_JOIN_COLS), 128, 0, stream, true, P, grid);
  if (e != cudaSuccess) return cuda_fail("tree_join_kernel launch", e);
  return PDATTN_OK;
}

pdattn_status tree_common(const pdattn_args* a, const int32_t* cu_tokens, int num_tokens, const uint64_t* tree_mask,
                          int max_tree_tokens, bool fp8, const float* k_scale, const float* v_scale, pdattn_stream_t stream) {
  if (!a || num_tokens < 0) return PDATTN_INVALID_ARG;
  pdattn_status s = check_shape(a->num_seqs, a->num_q_heads, a->num_kv_heads, a->head_dim, a->block_size);
  if (s != PDATTN_OK) return s;
  if (max_tree_tokens < 1) return PDATTN_INVALID_ARG;
  if (max_tree_tokens > 64 || a->num_seqs > TR_MAX_SEQS) return PDATTN_UNSUPPORTED;
  if (a->num_seqs == 0 || num_tokens == 0) return PDATTN_OK;
  if (!a->q || !a->k_cache || !a->v_cache || !a->out || !a->block_table || !a->context_lens || !a->workspace || !cu_tokens || !tree_mask)
    return PDATTN_INVALID_ARG;
  if (fp8 && (!k_scale || !v_scale)) return PDATTN_INVALID_ARG;
  if (a->max_blocks_per_seq <= 0 || a->num_blocks <= 0) return PDATTN_INVALID_ARG;
  const int G = a->num_q_heads / a->num_kv_heads, d = a->head_dim, bs = a->block_size;
  // dense pools of one-byte codes: the stride fields are not used
  const int64_t st = fp8 ? d : a->kv_token_stride, sh = fp8 ? static_cast<int64_t>(bs) * d : a->kv_head_stride;
  const int64_t sb = fp8 ? sh * a->num_kv_heads : a->kv_block_stride;
  if (sb <= 0 || sh <= 0 || st < d) return PDATTN_INVALID_ARG;
  if ((sb | sh | st) % 8 != 0) return PDATTN_UNSUPPORTED;
  auto mis = [](const void* p, size_t al) { return (reinterpret_cast<uintptr_t>(p) & (al - 1)) != 0; };
  if (mis(a->q, 16) || mis(a->k_cache, 16) || mis(a->v_cache, 16) || mis(a->out, 16) || mis(a->workspace, 256) || mis(tree_mask, 8))
    return PDATTN_MISALIGNED;
  if (a->workspace_bytes < kTreePartials + TR_CTAS * 2 * part_bytes(d)) return PDATTN_WORKSPACE_TOO_SMALL;
  const int TQ = 128 / G;
  const bool pair = max_tree_tokens > TQ;
  int dev = 0;
  DevInfo* di = nullptr;
  s = device_info(&dev, &di);
  if (s != PDATTN_OK) return s;

  CUtensorMap mq, mk, mv;
  s = make_map(a->q, d, TQ, a->num_kv_heads, num_tokens, 0, G, 0, kMapQ, &mq);
  if (s != PDATTN_OK) return s;
  s = make_map(a->k_cache, d, bs, a->num_kv_heads, a->num_blocks, sb, sh, st, fp8 ? kMapK8 : 4, &mk);
  if (s != PDATTN_OK) return s;
  s = make_map(a->v_cache, d, bs, a->num_kv_heads, a->num_blocks, sb, sh, st, fp8 ? kMapV8 : 4, &mv);
  if (s != PDATTN_OK) return s;

  uint8_t* ws = static_cast<uint8_t*>(a->workspace);
  TreeParams P{};
  P.out = static_cast<__nv_bfloat16*>(a->out);
  P.block_table = a->block_table;
  P.context_lens = a->context_lens;
  P.cu_tokens = cu_tokens;
  P.mask = tree_mask;
  P.v_cache = a->v_cache;
  P.sb = sb;
  P.sh = sh;
  P.st = st;
  P.k_scale = k_scale;
  P.v_scale = v_scale;
  P.hdr = reinterpret_cast<WsHeader*>(ws);
  P.rec = reinterpret_cast<int4*>(ws + kTreeRec);
  P.partials = reinterpret_cast<float*>(ws + kTreePartials);
  P.N = num_tokens;
  P.S = a->num_seqs;
  P.Hq = a->num_q_heads;
  P.Hkv = a->num_kv_heads;
  P.G = G;
  P.MB = a->max_blocks_per_seq;
  P.NB = a->num_blocks;
  P.bs_log2 = bs == 64 ? 6 : bs == 32 ? 5 : 4;
  P.TQ = TQ;
  P.max_n = max_tree_tokens;
  P.scale_log2 = a->scale * 1.4426950408889634f;
  const int grid = di->sm_count < TR_CTAS ? di->sm_count : TR_CTAS;
  cudaStream_t cs = reinterpret_cast<cudaStream_t>(stream);
  auto go = [&](auto dd, auto pp) {
    constexpr int D = decltype(dd)::value;
    constexpr bool PAIR = decltype(pp)::value;
    return fp8 ? launch_tree<D, PAIR, 1>(mq, mk, mv, P, dev, grid, cs) : launch_tree<D, PAIR, 2>(mq, mk, mv, P, dev, grid, cs);
  };
  if (d == 128)
    return pair ? go(std::integral_constant<int, 128>{}, std::true_type{}) : go(std::integral_constant<int, 128>{}, std::false_type{});
  return pair ? go(std::integral_constant<int, 64>{}, std::true_type{}) : go(std::integral_constant<int, 64>{}, std::false_type{});
}

}  // namespace

extern "C" {

pdattn_status pdattn_tree_workspace_size(int num_q_heads, int num_kv_heads, int head_dim, int block_size, int max_tree_tokens,
                                         size_t* device_bytes) {
  if (!device_bytes) return PDATTN_INVALID_ARG;
  const pdattn_status s = check_shape(0, num_q_heads, num_kv_heads, head_dim, block_size);
  if (s != PDATTN_OK) return s;
  if (max_tree_tokens < 1) return PDATTN_INVALID_ARG;
  if (max_tree_tokens > 64) return PDATTN_UNSUPPORTED;
  *device_bytes = kTreePartials + TR_CTAS * 2 * part_bytes(head_dim);
  return PDATTN_OK;
}

pdattn_status pdattn_decode_tree(const pdattn_args* args, const int32_t* cu_tokens, int num_tokens, const uint64_t* tree_mask,
                                 int max_tree_tokens, pdattn_stream_t stream) {
  return tree_common(args, cu_tokens, num_tokens, tree_mask, max_tree_tokens, false, nullptr, nullptr, stream);
}

pdattn_status pdattn_decode_tree_fp8(const pdattn_args* args, const int32_t* cu_tokens, int num_tokens, const uint64_t* tree_mask,
                                     int max_tree_tokens, const float* k_scale, const float* v_scale, pdattn_stream_t stream) {
  return tree_common(args, cu_tokens, num_tokens, tree_mask, max_tree_tokens, true, k_scale, v_scale, stream);
}

}  // extern "C"

// Host side of the operators for draft trees and sparse attention that are not attention themselves: page summaries, the choice of
// pages, the accepted path of a tree.  Argument checks (all before any CUDA call) and launches; no allocation, no synchronisation.
#include "../../include/pdattn.h"
#include "accept.cuh"
#include "host_common.h"
#include "summary.cuh"

namespace {

using namespace pdattn;

bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// What every call over a cache checks; element_bytes 1: dense code pools, whose strides are filled in here.
pdattn_status check_cache(int num_kv_heads, int head_dim, int block_size, int num_blocks, int element_bytes, int64_t* sb,
                          int64_t* sh, int64_t* st) {
  if (num_kv_heads <= 0 || num_blocks <= 0) return PDATTN_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return PDATTN_UNSUPPORTED;
  if (block_size != 16 && block_size != 32 && block_size != 64) return PDATTN_UNSUPPORTED;
  if (element_bytes != 1 && element_bytes != 2) return PDATTN_UNSUPPORTED;
  if (element_bytes == 1) {
    *st = head_dim;
    *sh = static_cast<int64_t>(block_size) * head_dim;
    *sb = *sh * num_kv_heads;
  }
  if (*sb <= 0 || *sh <= 0 || *st < head_dim) return PDATTN_INVALID_ARG;
  if ((*sb | *sh | *st) % 8 != 0) return PDATTN_UNSUPPORTED;
  return PDATTN_OK;
}

pdattn_status summarize(SummaryParams& P, int head_dim, bool fp8, int64_t grid, cudaStream_t stream) {
  if (misaligned(P.k, 16) || misaligned(P.codes, 16) || misaligned(P.err, 4)) return PDATTN_MISALIGNED;
  if (grid > INT32_MAX) return PDATTN_UNSUPPORTED;
  auto kern = head_dim == 128 ? (fp8 ? summarize_kernel<128, true> : summarize_kernel<128, false>)
                              : (fp8 ? summarize_kernel<64, true> : summarize_kernel<64, false>);
  const int warps = P.Hkv < 8 ? P.Hkv : 8;
  const cudaError_t e = launch_dependent(kern, static_cast<unsigned>(grid), 32 * warps, 0, stream, true, P);
  if (e != cudaSuccess) return cuda_fail("summarize_kernel launch", e);
  return PDATTN_OK;
}

// Pages that a block of select_kernel scores: as many, from 256 to 2048, as leave four blocks an SM (48 sequences to 32,768 tokens, 64/8
// heads: 25 us with 1024, 29 with 512, 36 with 2048).  More units than the workspace's zeroed words can number are enough by themselves: a block takes a
// whole one.
int select_chunk(int64_t units, int pages, int sms) {
  int chunk = 2048;
  while (chunk > 256 && units * ((pages + chunk - 1) / chunk) < 4ll * sms) chunk /= 2;
  return chunk;
}
constexpr size_t kSelectKeys = WS_CLEARED_BYTES;
static_assert(WS_CLEARED_BYTES == 8448 && (WS_CLEARED_BYTES % 256) == 0, "workspace layout");

}  // namespace

extern "C" {

pdattn_status pdattn_summarize_append(const pdattn_summary_args* a, const int32_t* block_table, const int32_t* context_lens,
                                      const int32_t* cu_tokens, int num_tokens, int num_seqs, int max_blocks_per_seq,
                                      pdattn_stream_t stream) {
  if (!a || num_tokens < 0 || num_seqs < 0) return PDATTN_INVALID_ARG;
  int64_t sb = a->kv_block_stride, sh = a->kv_head_stride, st = a->kv_token_stride;
  const pdattn_status s = check_cache(a->num_kv_heads, a->head_dim, a->block_size, a->num_blocks, a->element_bytes, &sb, &sh, &st);
  if (s != PDATTN_OK) return s;
  if (num_seqs == 0 || num_tokens == 0) return PDATTN_OK;
  if (!a->k_cache || !a->codes || !a->exponents || !block_table || !context_lens || max_blocks_per_seq <= 0) return PDATTN_INVALID_ARG;
  if (a->element_bytes == 1 && !a->k_scale) return PDATTN_INVALID_ARG;
  if (!cu_tokens && num_tokens != num_seqs) return PDATTN_INVALID_ARG;
  SummaryParams P{a->k_cache, sb, sh, st, a->k_scale, a->codes, a->exponents, block_table, context_lens, cu_tokens, nullptr,
                  static_cast<int32_t*>(a->workspace), num_seqs, a->num_kv_heads, max_blocks_per_seq, a->num_blocks, a->block_size,
                  num_tokens};
  const int64_t grid = cu_tokens ? static_cast<int64_t>(num_tokens) / a->block_size + num_seqs : num_seqs;
  return summarize(P, a->head_dim, a->element_bytes == 1, grid, reinterpret_cast<cudaStream_t>(stream));
}

pdattn_status pdattn_summarize_pages(const pdattn_summary_args* a, const int32_t* pages, int num_pages, pdattn_stream_t stream) {
  if (!a || num_pages < 0) return PDATTN_INVALID_ARG;
  int64_t sb = a->kv_block_stride, sh = a->kv_head_stride, st = a->kv_token_stride;
  const pdattn_status s = check_cache(a->num_kv_heads, a->head_dim, a->block_size, a->num_blocks, a->element_bytes, &sb, &sh, &st);
  if (s != PDATTN_OK) return s;
  if (num_pages == 0) return PDATTN_OK;
  if (!a->k_cache || !a->codes || !a->exponents || !pages) return PDATTN_INVALID_ARG;
  if (a->element_bytes == 1 && !a->k_scale) return PDATTN_INVALID_ARG;
  SummaryParams P{a->k_cache, sb, sh, st, a->k_scale, a->codes, a->exponents, nullptr, nullptr, nullptr, pages,
                  static_cast<int32_t*>(a->workspace), 0, a->num_kv_heads, 0, a->num_blocks, a->block_size, num_pages};
  return summarize(P, a->head_dim, a->element_bytes == 1, num_pages, reinterpret_cast<cudaStream_t>(stream));
}

pdattn_status pdattn_select_workspace_size(int num_seqs, int num_kv_heads, int max_blocks_per_seq, size_t* device_bytes) {
  if (num_seqs < 0 || num_kv_heads <= 0 || max_blocks_per_seq <= 0 || !device_bytes) return PDATTN_INVALID_ARG;
  *device_bytes = kSelectKeys + static_cast<size_t>(num_seqs) * num_kv_heads * max_blocks_per_seq * 4;
  return PDATTN_OK;
}

pdattn_status pdattn_select_pages(const pdattn_select_args* a, pdattn_stream_t stream) {
  if (!a) return PDATTN_INVALID_ARG;
  const pdattn_status s = check_shape(a->num_seqs, a->num_q_heads, a->num_kv_heads, a->head_dim, a->block_size);
  if (s != PDATTN_OK) return s;
  if (a->num_first < 0 || a->num_recent < 1 || static_cast<int64_t>(a->num_first) + a->num_recent > a->num_selected)
    return PDATTN_INVALID_ARG;
  if (a->num_seqs == 0) return PDATTN_OK;
  if (!a->q || !a->codes || !a->exponents || !a->block_table || !a->context_lens || !a->selected || !a->workspace)
    return PDATTN_INVALID_ARG;
  if (a->max_blocks_per_seq <= 0 || a->num_blocks <= 0) return PDATTN_INVALID_ARG;
  if (misaligned(a->q, 16) || misaligned(a->codes, 16) || misaligned(a->workspace, 256)) return PDATTN_MISALIGNED;
  size_t need = 0;
  pdattn_select_workspace_size(a->num_seqs, a->num_kv_heads, a->max_blocks_per_seq, &need);
  if (a->workspace_bytes < need) return PDATTN_WORKSPACE_TOO_SMALL;
  const int64_t units = static_cast<int64_t>(a->num_seqs) * a->num_kv_heads;
  uint8_t* ws = static_cast<uint8_t*>(a->workspace);
  SelectParams P{};
  P.q = static_cast<const __nv_bfloat16*>(a->q);
  P.codes = a->codes;
  P.exps = a->exponents;
  P.table = a->block_table;
  P.lens = a->context_lens;
  P.selected = a->selected;
  P.keys = reinterpret_cast<uint32_t*>(ws + kSelectKeys);
  P.tickets = reinterpret_cast<int32_t*>(ws + WS_TICKETS_OFFSET);
  P.err = &reinterpret_cast<WsHeader*>(ws)->err;
  P.S = a->num_seqs;
  P.Hq = a->num_q_heads;
  P.Hkv = a->num_kv_heads;
  P.G = a->num_q_heads / a->num_kv_heads;
  P.MB = a->max_blocks_per_seq;
  P.NB = a->num_blocks;
  P.bs = a->block_size;
  P.K = a->num_selected;
  P.first = a->num_first;
  P.recent = a->num_recent;
  const int most = a->max_blocks_per_seq - a->num_first - a->num_recent;      // pages that a unit may have to score
  int dev = 0;
  DevInfo* di = nullptr;
  const pdattn_status ds = device_info(&dev, &di);
  if (ds != PDATTN_OK) return ds;
  P.chunk = units <= MAX_SPANS ? select_chunk(units, most > 1 ? most : 1, di->sm_count) : a->max_blocks_per_seq;
  P.chunks = most > P.chunk ? (most + P.chunk - 1) / P.chunk : 1;
  const int64_t grid = units * P.chunks;
  if (grid > INT32_MAX) return PDATTN_UNSUPPORTED;
  auto kern = a->head_dim == 128 ? (P.G > 8 ? select_kernel<128, 2> : select_kernel<128, 1>)
                                 : (P.G > 8 ? select_kernel<64, 2> : select_kernel<64, 1>);
  const cudaError_t e = launch_dependent(kern, static_cast<unsigned>(grid), SEL_THREADS, 0, reinterpret_cast<cudaStream_t>(stream), true, P);
  if (e != cudaSuccess) return cuda_fail("select_kernel launch", e);
  return PDATTN_OK;
}

pdattn_status pdattn_tree_accept(void* k_cache, void* v_cache, const int32_t* block_table, const int32_t* context_lens,
                                 const int32_t* cu_tokens, const int32_t* accepted, const int32_t* accepted_counts,
                                 int max_accepted, int num_seqs, int num_kv_heads, int head_dim, int block_size,
                                 int max_blocks_per_seq, int num_blocks, int element_bytes, int64_t kv_block_stride,
                                 int64_t kv_head_stride, int64_t kv_token_stride, void* workspace, pdattn_stream_t stream) {
  if (num_seqs < 0 || max_accepted < 0) return PDATTN_INVALID_ARG;
  const pdattn_status s = check_cache(num_kv_heads, head_dim, block_size, num_blocks, element_bytes, &kv_block_stride,
                                      &kv_head_stride, &kv_token_stride);
  if (s != PDATTN_OK) return s;
  if (max_accepted > ACCEPT_MAX || num_kv_heads > 65535) return PDATTN_UNSUPPORTED;
  if (num_seqs == 0 || max_accepted == 0) return PDATTN_OK;
  if (!k_cache || !v_cache || !block_table || !context_lens || !cu_tokens || !accepted || !accepted_counts || max_blocks_per_seq <= 0)
    return PDATTN_INVALID_ARG;
  if (misaligned(k_cache, 16) || misaligned(v_cache, 16) || misaligned(workspace, 4)) return PDATTN_MISALIGNED;
  AcceptParams P{static_cast<uint8_t*>(k_cache), static_cast<uint8_t*>(v_cache), kv_block_stride * element_bytes,
                 kv_head_stride * element_bytes, kv_token_stride * element_bytes, block_table, context_lens, cu_tokens, accepted,
                 accepted_counts, static_cast<int32_t*>(workspace), num_seqs, num_kv_heads, max_blocks_per_seq, num_blocks,
                 block_size, max_accepted};
  auto kern = head_dim == 128 ? (element_bytes == 1 ? accept_kernel<128, true> : accept_kernel<128, false>)
                              : (element_bytes == 1 ? accept_kernel<64, true> : accept_kernel<64, false>);
  const cudaError_t e = launch_dependent(kern, dim3(num_seqs, num_kv_heads), ACCEPT_THREADS, 0, reinterpret_cast<cudaStream_t>(stream),
                                         true, P);
  if (e != cudaSuccess) return cuda_fail("accept_kernel launch", e);
  return PDATTN_OK;
}

}  // extern "C"

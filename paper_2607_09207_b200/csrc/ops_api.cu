// Host side of the operators around the decode step: rotary positions with the KV append, and the page bookkeeping.
// Argument checks (all before any CUDA call) and launches; no allocation, no synchronisation.
#include "../../include/pdattn.h"
#include "common.cuh"
#include "host_common.h"
#include "pages.cuh"
#include "rope.cuh"

namespace {

using namespace pdattn;

bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// ---- rotary positions with the append ------------------------------------------------------------
pdattn_status rope_common(const pdattn_rope_args* a, const int32_t* positions, bool fp8, const float* k_scale,
                          const float* v_scale, pdattn_stream_t stream) {
  if (!a) return PDATTN_INVALID_ARG;
  if (a->num_tokens < 0 || a->num_seqs < 0 || a->num_q_heads < 0 || a->num_kv_heads <= 0) return PDATTN_INVALID_ARG;
  if (a->head_dim != 64 && a->head_dim != 128) return PDATTN_UNSUPPORTED;
  if (a->block_size != 16 && a->block_size != 32 && a->block_size != 64) return PDATTN_UNSUPPORTED;
  if (a->rotary_dim <= 0 || a->rotary_dim > a->head_dim) return PDATTN_INVALID_ARG;
  if (a->rotary_dim % 16 != 0) return PDATTN_UNSUPPORTED;
  if (a->interleaved != 0 && a->interleaved != 1) return PDATTN_INVALID_ARG;
  if (a->num_tokens == 0) return PDATTN_OK;
  if (!a->k_new || !a->v_new || !a->k_cache || !a->v_cache || !a->block_table || !a->context_lens || !a->inv_freq)
    return PDATTN_INVALID_ARG;
  if (a->num_q_heads > 0 && (!a->q || !a->q_out)) return PDATTN_INVALID_ARG;
  if (a->num_seqs == 0 || (!a->cu_tokens && a->num_tokens != a->num_seqs)) return PDATTN_INVALID_ARG;
  if (a->max_blocks_per_seq <= 0 || a->num_blocks <= 0) return PDATTN_INVALID_ARG;
  const int64_t q_row = static_cast<int64_t>(a->num_q_heads) * a->head_dim;
  const int64_t kv_row = static_cast<int64_t>(a->num_kv_heads) * a->head_dim;
  if (a->num_q_heads > 0 && a->q_token_stride < q_row) return PDATTN_INVALID_ARG;
  if (a->k_token_stride < kv_row || a->v_token_stride < kv_row) return PDATTN_INVALID_ARG;
  if ((a->k_token_stride | a->v_token_stride) % 8 != 0 || (a->num_q_heads > 0 && a->q_token_stride % 8 != 0))
    return PDATTN_UNSUPPORTED;
  if (!fp8) {
    if (a->kv_block_stride <= 0 || a->kv_head_stride <= 0 || a->kv_token_stride < a->head_dim) return PDATTN_INVALID_ARG;
    if ((a->kv_block_stride | a->kv_head_stride | a->kv_token_stride) % 8 != 0) return PDATTN_UNSUPPORTED;
  } else if (!k_scale || !v_scale) {
    return PDATTN_INVALID_ARG;
  }
  if (misaligned(a->k_new, 16) || misaligned(a->v_new, 16) || misaligned(a->k_cache, 16) || misaligned(a->v_cache, 16) ||
      misaligned(a->q, 16) || misaligned(a->q_out, 16) || misaligned(a->workspace, 4))
    return PDATTN_MISALIGNED;
  // in place only row for row: a dense output over a strided input would overwrite rows that are still to be read
  if (a->num_q_heads > 0 && a->q_out == a->q && a->q_token_stride != q_row) return PDATTN_INVALID_ARG;
  int dev = 0;
  DevInfo* di = nullptr;
  const pdattn_status s = device_info(&dev, &di);
  if (s != PDATTN_OK) return s;
  RopeParams P{};
  P.q = static_cast<const __nv_bfloat16*>(a->q);
  P.k_new = static_cast<const __nv_bfloat16*>(a->k_new);
  P.v_new = static_cast<const __nv_bfloat16*>(a->v_new);
  P.q_out = static_cast<__nv_bfloat16*>(a->q_out);
  P.k_cache = a->k_cache;
  P.v_cache = a->v_cache;
  P.block_table = a->block_table;
  P.context_lens = a->context_lens;
  P.cu_tokens = a->cu_tokens;
  P.positions = positions;
  P.inv_freq = a->inv_freq;
  P.k_scale = k_scale;
  P.v_scale = v_scale;
  P.q_ts = a->q_token_stride;
  P.k_ts = a->k_token_stride;
  P.v_ts = a->v_token_stride;
  P.sb = a->kv_block_stride;
  P.sh = a->kv_head_stride;
  P.st = a->kv_token_stride;
  P.err = static_cast<int32_t*>(a->workspace);
  P.magnitude = a->magnitude;
  P.N = a->num_tokens;
  P.S = a->num_seqs;
  P.Hq = a->num_q_heads;
  P.Hkv = a->num_kv_heads;
  P.bs = a->block_size;
  P.MB = a->max_blocks_per_seq;
  P.NB = a->num_blocks;
  P.R = a->rotary_dim;
  P.interleaved = a->interleaved;
  // One token per block while that leaves SMs without four blocks (latency: a block's rows in one or two rounds);
  // more tokens per block beyond, so that a thread's angle work is spread over more rows.
  int tpb = 1;
  while (tpb < kRopeMaxTokens && a->num_tokens > static_cast<int64_t>(tpb) * 8 * di->sm_count) tpb *= 2;
  P.tokens_per_block = tpb;
  const int grid = (a->num_tokens + tpb - 1) / tpb;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  auto kern = a->head_dim == 128 ? (fp8 ? rope_append_kernel<128, true> : rope_append_kernel<128, false>)
                                 : (fp8 ? rope_append_kernel<64, true> : rope_append_kernel<64, false>);
  const cudaError_t e = launch_dependent(kern, grid, kRopeThreads, 0, st, true, P);
  if (e != cudaSuccess) return cuda_fail("rope_append_kernel launch", e);
  return PDATTN_OK;
}

// ---- pages ---------------------------------------------------------------------------------------
struct PagesLayout {
  size_t head, lens, tails, map, total;
};
PagesLayout pages_layout(int num_blocks, int num_seqs) {
  PagesLayout w;
  w.head = WS_CLEARED_BYTES;
  w.lens = w.head + 256;
  w.tails = w.lens + align_up(static_cast<size_t>(num_seqs) * 4, 256);
  w.map = w.tails + align_up(static_cast<size_t>(num_seqs) * 4, 256);
  w.total = w.map + align_up(static_cast<size_t>(num_blocks) * 4, 256);
  return w;
}

// What every page operation checks, and the scratch it works in.
pdattn_status pages_check(const pdattn_page_pool* pool, const void* table, const void* lens, int num_seqs,
                          int max_blocks_per_seq, int block_size, void* workspace, size_t workspace_bytes, PagePool* p,
                          PagesScratch* x) {
  if (!pool || pool->num_blocks <= 0 || num_seqs < 0 || max_blocks_per_seq <= 0 || block_size <= 0) return PDATTN_INVALID_ARG;
  if (block_size != 16 && block_size != 32 && block_size != 64) return PDATTN_UNSUPPORTED;
  if (!pool->ref_counts || !pool->free_list || !pool->free_count || !workspace) return PDATTN_INVALID_ARG;
  if (num_seqs > 0 && (!table || !lens)) return PDATTN_INVALID_ARG;
  if (misaligned(workspace, 256)) return PDATTN_MISALIGNED;
  const PagesLayout w = pages_layout(pool->num_blocks, num_seqs);
  if (workspace_bytes < w.total) return PDATTN_WORKSPACE_TOO_SMALL;
  *p = PagePool{pool->ref_counts, pool->free_list, pool->free_count, pool->num_blocks};
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  x->err = reinterpret_cast<int32_t*>(ws);
  x->head = reinterpret_cast<int32_t*>(ws + w.head);
  x->lens = reinterpret_cast<int32_t*>(ws + w.lens);
  x->tails = reinterpret_cast<int32_t*>(ws + w.tails);
  x->map = reinterpret_cast<int32_t*>(ws + w.map);
  return PDATTN_OK;
}

}  // namespace

extern "C" {

pdattn_status pdattn_rope_append(const pdattn_rope_args* args, pdattn_stream_t stream) {
  return rope_common(args, nullptr, false, nullptr, nullptr, stream);
}
pdattn_status pdattn_rope_append_fp8(const pdattn_rope_args* args, const float* k_scale, const float* v_scale,
                                     pdattn_stream_t stream) {
  return rope_common(args, nullptr, true, k_scale, v_scale, stream);
}
pdattn_status pdattn_rope_append_at(const pdattn_rope_args* args, const int32_t* positions, pdattn_stream_t stream) {
  if (!positions) return PDATTN_INVALID_ARG;
  return rope_common(args, positions, false, nullptr, nullptr, stream);
}
pdattn_status pdattn_rope_append_at_fp8(const pdattn_rope_args* args, const int32_t* positions, const float* k_scale,
                                        const float* v_scale, pdattn_stream_t stream) {
  if (!positions) return PDATTN_INVALID_ARG;
  return rope_common(args, positions, true, k_scale, v_scale, stream);
}

pdattn_status pdattn_pages_workspace_size(int num_blocks, int num_seqs, size_t* device_bytes) {
  if (num_blocks <= 0 || num_seqs < 0 || !device_bytes) return PDATTN_INVALID_ARG;
  *device_bytes = pages_layout(num_blocks, num_seqs).total;
  return PDATTN_OK;
}

pdattn_status pdattn_pages_init(const pdattn_page_pool* pool, pdattn_stream_t stream) {
  if (!pool || pool->num_blocks <= 0 || !pool->ref_counts || !pool->free_list || !pool->free_count) return PDATTN_INVALID_ARG;
  const PagePool p{pool->ref_counts, pool->free_list, pool->free_count, pool->num_blocks};
  const cudaError_t e = launch_dependent(pages_init_kernel, (p.NB + 255) / 256, 256, 0, reinterpret_cast<cudaStream_t>(stream), true, p);
  if (e != cudaSuccess) return cuda_fail("pages_init_kernel launch", e);
  return PDATTN_OK;
}

pdattn_status pdattn_pages_reserve(const pdattn_page_pool* pool, int32_t* block_table, int32_t* context_lens,
                                   const int32_t* new_tokens, int num_seqs, int max_blocks_per_seq, int block_size,
                                   void* workspace, size_t workspace_bytes, pdattn_stream_t stream) {
  PagePool p;
  PagesScratch x;
  const pdattn_status s = pages_check(pool, block_table, context_lens, num_seqs, max_blocks_per_seq, block_size, workspace,
                                      workspace_bytes, &p, &x);
  if (s != PDATTN_OK) return s;
  if (num_seqs == 0) return PDATTN_OK;
  if (!new_tokens) return PDATTN_INVALID_ARG;
  const cudaError_t e = launch_dependent(pages_reserve_kernel, 1, kPagesThreads, 0, reinterpret_cast<cudaStream_t>(stream), true,
                                         p, block_table, context_lens, new_tokens, num_seqs, max_blocks_per_seq, block_size, x.err);
  if (e != cudaSuccess) return cuda_fail("pages_reserve_kernel launch", e);
  return PDATTN_OK;
}

pdattn_status pdattn_pages_fork(const pdattn_page_pool* pool, int32_t* block_table, int32_t* context_lens,
                                const int32_t* parents, const int32_t* children, int num_forks, int num_seqs,
                                int max_blocks_per_seq, int block_size, int32_t* copy_src, int32_t* copy_dst,
                                void* workspace, size_t workspace_bytes, pdattn_stream_t stream) {
  PagePool p;
  PagesScratch x;
  const pdattn_status s = pages_check(pool, block_table, context_lens, num_seqs, max_blocks_per_seq, block_size, workspace,
                                      workspace_bytes, &p, &x);
  if (s != PDATTN_OK) return s;
  if (num_forks < 0 || num_forks > num_seqs) return PDATTN_INVALID_ARG;   // every child is a row of its own
  if (num_forks == 0) return PDATTN_OK;
  if (!parents || !children || !copy_src || !copy_dst) return PDATTN_INVALID_ARG;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e = launch_dependent(pages_fork_kernel, 1, kPagesThreads, 0, st, true, p, block_table, context_lens, parents, children,
                                   num_forks, num_seqs, max_blocks_per_seq, block_size, copy_src, copy_dst, x);
  if (e != cudaSuccess) return cuda_fail("pages_fork_kernel launch", e);
  e = launch_dependent(pages_fork_rows_kernel, num_forks, 128, 0, st, true, p, block_table, parents, children, max_blocks_per_seq,
                       block_size, x);
  if (e != cudaSuccess) return cuda_fail("pages_fork_rows_kernel launch", e);
  return PDATTN_OK;
}

pdattn_status pdattn_pages_free(const pdattn_page_pool* pool, int32_t* block_table, int32_t* context_lens,
                                const int32_t* seqs, int num_freed, int num_seqs, int max_blocks_per_seq, int block_size,
                                void* workspace, size_t workspace_bytes, pdattn_stream_t stream) {
  PagePool p;
  PagesScratch x;
  const pdattn_status s = pages_check(pool, block_table, context_lens, num_seqs, max_blocks_per_seq, block_size, workspace,
                                      workspace_bytes, &p, &x);
  if (s != PDATTN_OK) return s;
  if (num_freed < 0) return PDATTN_INVALID_ARG;
  if (num_freed == 0 || num_seqs == 0) return PDATTN_OK;
  if (!seqs) return PDATTN_INVALID_ARG;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e = launch_dependent(pages_free_kernel, num_freed, 128, 0, st, true, p, block_table, context_lens, seqs, num_seqs,
                                   max_blocks_per_seq, block_size, x.err);
  if (e != cudaSuccess) return cuda_fail("pages_free_kernel launch", e);
  e = launch_dependent(pages_books_kernel<false>, kPagesCluster, kPagesThreads, 0, st, true, p, static_cast<int32_t*>(nullptr),
                       static_cast<int32_t*>(nullptr), 0, x);
  if (e != cudaSuccess) return cuda_fail("pages_books_kernel launch", e);
  return PDATTN_OK;
}

pdattn_status pdattn_pages_trim(const pdattn_page_pool* pool, int32_t* block_table, int32_t* context_lens,
                                const int32_t* new_lens, int num_seqs, int max_blocks_per_seq, int block_size,
                                void* workspace, size_t workspace_bytes, pdattn_stream_t stream) {
  PagePool p;
  PagesScratch x;
  const pdattn_status s = pages_check(pool, block_table, context_lens, num_seqs, max_blocks_per_seq, block_size, workspace,
                                      workspace_bytes, &p, &x);
  if (s != PDATTN_OK) return s;
  if (num_seqs == 0) return PDATTN_OK;
  if (!new_lens) return PDATTN_INVALID_ARG;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e = launch_dependent(pages_trim_kernel, num_seqs, 128, 0, st, true, p, block_table, context_lens, new_lens,
                                   max_blocks_per_seq, block_size, x.err);
  if (e != cudaSuccess) return cuda_fail("pages_trim_kernel launch", e);
  e = launch_dependent(pages_books_kernel<false>, kPagesCluster, kPagesThreads, 0, st, true, p, static_cast<int32_t*>(nullptr),
                       static_cast<int32_t*>(nullptr), 0, x);
  if (e != cudaSuccess) return cuda_fail("pages_books_kernel launch", e);
  return PDATTN_OK;
}

pdattn_status pdattn_pages_compact(const pdattn_page_pool* pool, int32_t* block_table, const int32_t* context_lens,
                                   int num_seqs, int max_blocks_per_seq, int block_size, int32_t* copy_src,
                                   int32_t* copy_dst, int max_copies, void* workspace, size_t workspace_bytes,
                                   pdattn_stream_t stream) {
  PagePool p;
  PagesScratch x;
  const pdattn_status s = pages_check(pool, block_table, context_lens, num_seqs, max_blocks_per_seq, block_size, workspace,
                                      workspace_bytes, &p, &x);
  if (s != PDATTN_OK) return s;
  if (max_copies < p.NB / 2) return PDATTN_INVALID_ARG;    // there are never more moves than that
  if (max_copies > 0 && (!copy_src || !copy_dst)) return PDATTN_INVALID_ARG;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e = launch_dependent(pages_books_kernel<true>, kPagesCluster, kPagesThreads, 0, st, true, p, copy_src, copy_dst, max_copies, x);
  if (e != cudaSuccess) return cuda_fail("pages_books_kernel launch", e);
  if (num_seqs == 0) return PDATTN_OK;
  e = launch_dependent(pages_remap_kernel, num_seqs, 128, 0, st, true, p, block_table, context_lens, max_blocks_per_seq, block_size, x);
  if (e != cudaSuccess) return cuda_fail("pages_remap_kernel launch", e);
  return PDATTN_OK;
}

pdattn_status pdattn_pages_copy(void* k_cache, void* v_cache, const int32_t* copy_src, const int32_t* copy_dst,
                                int num_copies, int num_kv_heads, int head_dim, int block_size, int num_blocks,
                                int element_bytes, int64_t kv_block_stride, int64_t kv_head_stride,
                                int64_t kv_token_stride, void* workspace, pdattn_stream_t stream) {
  if (num_copies < 0 || num_kv_heads <= 0 || num_blocks <= 0) return PDATTN_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return PDATTN_UNSUPPORTED;
  if (block_size != 16 && block_size != 32 && block_size != 64) return PDATTN_UNSUPPORTED;
  if (element_bytes != 1 && element_bytes != 2) return PDATTN_UNSUPPORTED;
  if (num_copies > (1 << 29)) return PDATTN_INVALID_ARG;
  if (num_copies == 0) return PDATTN_OK;
  if (!k_cache || !v_cache || !copy_src || !copy_dst) return PDATTN_INVALID_ARG;
  const int64_t row = head_dim, head = static_cast<int64_t>(block_size) * head_dim;
  if (element_bytes == 1) {                 // dense pools of one-byte codes, as for pdattn_decode_fp8
    kv_token_stride = row;
    kv_head_stride = head;
    kv_block_stride = num_kv_heads * head;
  }
  if (kv_block_stride <= 0 || kv_head_stride <= 0 || kv_token_stride < head_dim) return PDATTN_INVALID_ARG;
  if ((kv_block_stride | kv_head_stride | kv_token_stride) % 8 != 0) return PDATTN_UNSUPPORTED;
  if (misaligned(k_cache, 16) || misaligned(v_cache, 16) || misaligned(workspace, 4)) return PDATTN_MISALIGNED;
  int dev = 0;
  DevInfo* di = nullptr;
  const pdattn_status s = device_info(&dev, &di);
  if (s != PDATTN_OK) return s;
  CopyParams P{};
  P.k = static_cast<uint8_t*>(k_cache);
  P.v = static_cast<uint8_t*>(v_cache);
  P.src = copy_src;
  P.dst = copy_dst;
  P.sb = kv_block_stride * element_bytes;
  P.sh = kv_head_stride * element_bytes;
  P.st = kv_token_stride * element_bytes;
  P.n = num_copies;
  P.NB = num_blocks;
  P.heads = num_kv_heads;
  P.rows = block_size;
  P.row_chunks = head_dim * element_bytes / 16;
  P.dense = (kv_token_stride == row && kv_head_stride == head) ||                                   // [head][token][dim]
            (kv_head_stride == row && kv_token_stride == static_cast<int64_t>(num_kv_heads) * row);   // [token][head][dim]
  P.err = static_cast<int32_t*>(workspace);
  const int64_t units = 2ll * num_copies;
  const int grid = static_cast<int>(units < 8ll * di->sm_count ? units : 8ll * di->sm_count);
  const cudaError_t e = launch_dependent(pages_copy_kernel, grid, kCopyThreads, 0, reinterpret_cast<cudaStream_t>(stream), true, P);
  if (e != cudaSuccess) return cuda_fail("pages_copy_kernel launch", e);
  return PDATTN_OK;
}

}  // extern "C"

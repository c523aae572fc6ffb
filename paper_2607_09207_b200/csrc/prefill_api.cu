// Host side of pdattn_prefill: argument checks, tensor maps, launch.
#include <cstdio>
#include <type_traits>

#include "../../include/pdattn.h"
#include "host_common.h"
#include "prefill_umma.cuh"

namespace {

using namespace pdattn;

template <int D, bool CAP, bool GEN>
pdattn_status launch_prefill_kernel(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv,
                                    const PrefillParams& P, int dev, int sms, cudaStream_t stream) {
  using C = PrefillCfg<D>;
  auto kern = prefill_kernel<D, CAP, GEN>;
  static bool attr_set[kMaxDevices] = {};
  if (!attr_set[dev]) {
    // the kernel re-deals its launch registers (see there): a build that launches with fewer would wait for good
    cudaFuncAttributes fa;
    cudaError_t e = cudaFuncGetAttributes(&fa, kern);
    if (e != cudaSuccess) return cuda_fail("cudaFuncGetAttributes", e);
    if (fa.numRegs != PF_LAUNCH_REGS) {
      snprintf(cuda_error_text(), kCudaErrorTextBytes, "prefill_kernel was built with %d registers a thread, %d are wanted",
               fa.numRegs, PF_LAUNCH_REGS);
      return PDATTN_CUDA_ERROR;
    }
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::DYN_BYTES);
    if (e != cudaSuccess) return cuda_fail("cudaFuncSetAttribute", e);
    attr_set[dev] = true;
  }
  const int units = P.n_items * P.splits;
  const int grid = units < sms ? units : sms;
  const cudaError_t e = launch_dependent(kern, grid, PF_NTHREADS, C::DYN_BYTES, stream, true, mq, mk, mv, P);
  if (e != cudaSuccess) return cuda_fail("prefill_kernel launch", e);
  if (P.splits > 1) {
    const cudaError_t j = launch_dependent(prefill_join_kernel<D>, dim3(P.n_items, 2, D / 8), 128, 0, stream, true, P);
    if (j != cudaSuccess) return cuda_fail("prefill_join_kernel launch", j);
  }
  return PDATTN_OK;
}

// Items of a call (pair slots x KV heads), and the parts each may be cut into along the keys: as many as fill PF_UNITS CTAs; up
// to 2/3 of PF_UNITS items in three parts, two rounds of a third each in place of a whole one (28/4 heads, whole and in three: 16 x
// 8 tokens over 16,000 keys 232 and 168 us, over 4000 66 and 56, over 1000 24 and 23; 850 tokens without a history 25 and 28).
constexpr int PF_UNITS = 148;
int64_t prefill_items(int num_seqs, int num_tokens, int Hq, int Hkv) {
  return (static_cast<int64_t>(num_tokens) / (2 * (128 / (Hq / Hkv))) + num_seqs) * Hkv;
}
int prefill_splits(int64_t items) {
  if (items <= 0 || items > PF_UNITS * 2 / 3) return 1;
  return items <= PF_UNITS / 2 ? static_cast<int>(PF_UNITS / items) : 3;
}
size_t prefill_part_bytes(int head_dim) { return static_cast<size_t>(2) * (head_dim + 2) * 128 * 4; }
constexpr size_t kPrefillParts = WS_CLEARED_BYTES;             // [items] int32
constexpr size_t kPrefillPartials = WS_CLEARED_BYTES + 1024;   // 256-byte aligned
static_assert(kPrefillPartials % 256 == 0 && PF_UNITS * 2 / 3 * 4 <= 1024, "workspace layout");

}  // namespace

extern "C" {

pdattn_status pdattn_prefill_workspace_size(int num_seqs, int num_tokens, int num_q_heads, int num_kv_heads, int head_dim,
                                            int block_size, size_t* device_bytes) {
  if (!device_bytes || num_tokens < 0) return PDATTN_INVALID_ARG;
  const pdattn_status s = check_shape(num_seqs, num_q_heads, num_kv_heads, head_dim, block_size);
  if (s != PDATTN_OK) return s;
  const int64_t items = prefill_items(num_seqs, num_tokens, num_q_heads, num_kv_heads);
  const int splits = prefill_splits(items);
  *device_bytes = splits > 1 ? kPrefillPartials + static_cast<size_t>(items) * splits * prefill_part_bytes(head_dim) : WS_CLEARED_BYTES;
  return PDATTN_OK;
}

pdattn_status pdattn_prefill(const pdattn_args* a, const int32_t* cu_tokens, int num_tokens,
                             const pdattn_score_args* score, pdattn_stream_t stream) {
  if (!a || num_tokens < 0) return PDATTN_INVALID_ARG;
  pdattn_status s = check_shape(a->num_seqs, a->num_q_heads, a->num_kv_heads, a->head_dim, a->block_size);
  if (s != PDATTN_OK) return s;
  if (a->num_seqs == 0 || num_tokens == 0) return PDATTN_OK;
  if (!a->q || !a->k_cache || !a->v_cache || !a->out || !a->block_table || !a->context_lens || !a->workspace || !cu_tokens)
    return PDATTN_INVALID_ARG;
  if (a->max_blocks_per_seq <= 0 || a->num_blocks <= 0) return PDATTN_INVALID_ARG;
  if (a->kv_block_stride <= 0 || a->kv_head_stride <= 0 || a->kv_token_stride < a->head_dim) return PDATTN_INVALID_ARG;
  if ((a->kv_block_stride | a->kv_head_stride | a->kv_token_stride) % 8 != 0) return PDATTN_UNSUPPORTED;
  if (score && (!valid_cap(score->logit_cap) || score->window < 0)) return PDATTN_INVALID_ARG;
  auto mis = [](const void* p, size_t al) { return (reinterpret_cast<uintptr_t>(p) & (al - 1)) != 0; };
  if (mis(a->q, 16) || mis(a->k_cache, 16) || mis(a->v_cache, 16) || mis(a->out, 16) || mis(a->workspace, 256))
    return PDATTN_MISALIGNED;
  if (a->workspace_bytes < WS_CLEARED_BYTES) return PDATTN_WORKSPACE_TOO_SMALL;
  const int G = a->num_q_heads / a->num_kv_heads;
  const int TQ = 128 / G;
  const int64_t items = prefill_items(a->num_seqs, num_tokens, a->num_q_heads, a->num_kv_heads);
  if (items > INT32_MAX / 2) return PDATTN_UNSUPPORTED;
  // a workspace without room for the parts' results is taken too: the items then stay whole
  int splits = prefill_splits(items);
  if (splits > 1) {
    const int64_t room = a->workspace_bytes > kPrefillPartials
                             ? static_cast<int64_t>((a->workspace_bytes - kPrefillPartials) / prefill_part_bytes(a->head_dim)) / items : 0;
    if (splits > room) splits = room > 1 ? static_cast<int>(room) : 1;
  }
  int dev = 0;
  DevInfo* di = nullptr;
  s = device_info(&dev, &di);
  if (s != PDATTN_OK) return s;

  CUtensorMap mq, mk, mv;
  s = make_map(a->q, a->head_dim, TQ, a->num_kv_heads, num_tokens, 0, G, 0, kMapQ, &mq);
  if (s != PDATTN_OK) return s;
  s = make_map(a->k_cache, a->head_dim, a->block_size, a->num_kv_heads, a->num_blocks, a->kv_block_stride, a->kv_head_stride,
               a->kv_token_stride, 4, &mk);
  if (s != PDATTN_OK) return s;
  s = make_map(a->v_cache, a->head_dim, a->block_size, a->num_kv_heads, a->num_blocks, a->kv_block_stride, a->kv_head_stride,
               a->kv_token_stride, 4, &mv);
  if (s != PDATTN_OK) return s;

  constexpr float kLog2e = 1.4426950408889634f;
  PrefillParams P{};
  P.out = static_cast<__nv_bfloat16*>(a->out);
  P.block_table = a->block_table;
  P.context_lens = a->context_lens;
  P.cu_tokens = cu_tokens;
  P.v_cache = static_cast<const __nv_bfloat16*>(a->v_cache);
  P.sb = a->kv_block_stride;
  P.sh = a->kv_head_stride;
  P.st = a->kv_token_stride;
  P.hdr = static_cast<WsHeader*>(a->workspace);
  P.N = num_tokens;
  P.S = a->num_seqs;
  P.Hq = a->num_q_heads;
  P.Hkv = a->num_kv_heads;
  P.G = G;
  P.MB = a->max_blocks_per_seq;
  P.NB = a->num_blocks;
  P.bs_log2 = a->block_size == 64 ? 6 : a->block_size == 32 ? 5 : 4;
  P.TQ = TQ;
  P.n_items = static_cast<int>(items);
  P.splits = splits;
  P.parts = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(a->workspace) + kPrefillParts);
  P.partials = reinterpret_cast<float*>(static_cast<uint8_t*>(a->workspace) + kPrefillPartials);
  P.scale_log2 = a->scale * kLog2e;
  const bool cap = score && score->logit_cap > 0.f;
  if (score) {
    P.slopes = score->bias_slopes;
    P.key_begin = score->key_begin;
    P.prefix_lens = score->prefix_lens;
    P.window = score->window;
    if (cap) {
      P.cap2 = score->logit_cap * kLog2e;
      P.cap_x = a->scale / score->logit_cap;
    }
  }
  // scores are brought to base-2 units one by one for a bias, and for a scale that is not positive (the other form takes the
  // maximum of the raw scores)
  const bool gen = P.slopes != nullptr || (!cap && !(a->scale > 0.f));
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  auto go = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (cap) return gen ? launch_prefill_kernel<D, true, true>(mq, mk, mv, P, dev, di->sm_count, st)
                        : launch_prefill_kernel<D, true, false>(mq, mk, mv, P, dev, di->sm_count, st);
    return gen ? launch_prefill_kernel<D, false, true>(mq, mk, mv, P, dev, di->sm_count, st)
               : launch_prefill_kernel<D, false, false>(mq, mk, mv, P, dev, di->sm_count, st);
  };
  return a->head_dim == 128 ? go(std::integral_constant<int, 128>{}) : go(std::integral_constant<int, 64>{});
}

}  // extern "C"

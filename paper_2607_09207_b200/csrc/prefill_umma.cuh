// Prompt attention over the paged cache on the 5th-generation tensor cores: prefill_kernel.
//
//   x_t = scale q.k_t, capped by a tanh and biased by distance if asked;  out = softmax_t(x_t) . V over lo <= t < hi
//
// Work.  The query rows of one KV head are packed: row r of a 128-row tile is head r % G of token r / G, so a tile holds
// floor(128 / G) whole tokens and K/V tiles are read once for all G heads.  An item is (sequence, pair of tiles, KV head); a
// persistent CTA walks the 128-key tiles that any row of its pair sees and takes the next item from a counter, sequences from the
// last to the first and in each the late (long) pairs first.  Sequence s owns the pair slots from cu[s] / (2 tokens-per-tile) + s on: enough of them without a prefix
// sum, so the launch needs no host copy of the lengths (slots without tokens are stepped over).
//
//   S_t[128, 128 keys]  = Q_t . K^T         both from shared memory               t = 0, 1: the two tiles of the pair
//   O_t[128, d]        += P_t . V           P from tensor memory (over S_t's columns), V from shared memory
//
// The pair is what keeps the tensor cores busy: while the softmax warps of one tile work on S_t the products of the other
// run.  Roles: warps 0-3 and 4-7 softmax of tile 0 and 1 (a thread owns a row: no shuffles), warp 8 issues the MMAs, warp 10
// loads Q and K, warp 11 V (TMA), warp 12 prepares items ahead, warps 14 and 15 guard V (9 and 13 only complete the groups
// that registers are dealt to).  S_t of the next key tile is issued right behind the P_t . V of the present one by the same
// thread, in order, so the buffer that P_t occupies needs no further wait, and scores that have arrived say that the product
// before them is done.
//
// Few rows over long contexts.  Items that would leave most SMs idle are cut along the keys into up to P.splits parts of at
// least PF_MIN_TILES key tiles; each writes its (m, l, O) and prefill_join_kernel puts them together in order.
//
// Masks are intervals per row.  A key tile that every row of a tile sees whole takes no mask at all; the others ("edge" tiles)
// are masked by select.  A masked weight is 0, and 0 * inf or 0 * NaN would still poison the row, so in edge tiles the guards set
// the non-finite elements of V to 0 before the product and note the keys; a row that does see such a key adds those elements
// to its output at the end, whatever their weight.  In a tile that is seen whole the product takes them as they are: infinite, or
// NaN where a weight is 0 in 32 bits.  (Guards on every tile would make that infinite too, and cost 11 % of 8191 causal tokens.)
//
// Numbers: scores, maxima, sums and O in fp32; the weights are rounded to bf16 for the second product (at most 2^-8 of each,
// independent: the same size as the final rounding of the output; two terms, as in the decode kernel, would cost half as much
// tensor work again).  The reference of the online softmax follows the running maximum only when that grew by more than 2^8,
// so O is rarely rescaled.
//
// Bound: the chain of a tile, about 4000 cycles a pair and key tile (clock stamps of an instrumented build) against the 2048 that
// its 32 MMAs take -- scores to weights 2500 (128 exponentials a thread, two warps to a quadrant), weights to the next scores
// 1300 (barrier, half of P.V, Q.K^T, barrier).  Tried and not faster: two threads a row (16 softmax warps), the scores in registers
// throughout (the code then outgrows the instruction caches), a share of the exponentials on the FMA pipe, one MMA warp per tile
// (the tiles fall into step and their phases no longer overlap).  8191 causal tokens, 28/4 heads of 128: 445-510 us, 0.94-1.08
// PFLOP/s (the spread is the clock under the power cap); with a cap 665-690 (1055 where every score lies past it), with a distance
// bias 615-640.  Also tried for those two: the bias as packed multiply-adds (no gain), worked out again in the second pass in place
// of the write-back (+13 %), tanh in unpacked operations (+10 %).
//
// Every wait is bounded; on expiry the CTA raises ERR_TIMEOUT, the waits fall through, the MMA thread drains, tensor memory
// is freed and the CTA returns.
#pragma once

#include <climits>
#include <type_traits>

#include "umma.cuh"

namespace pdattn {

struct PrefillParams {
  __nv_bfloat16* out;
  const int32_t *block_table, *context_lens, *cu_tokens;
  const float* slopes;           // per query head, or null
  const int32_t *key_begin, *prefix_lens;
  const __nv_bfloat16* v_cache;  // for the guarded elements only: element strides as in pdattn_args
  int64_t sb, sh, st;
  WsHeader* hdr;
  int N, S, Hq, Hkv, G, MB, NB, bs_log2;
  int TQ;                        // tokens of a tile: 128 / G
  int n_items;                   // pair slots x KV heads
  int splits;                    // parts an item may be cut into
  int32_t* parts;                // [n_items] parts it was cut into (splits > 1 only)
  float* partials;               // [n_items * splits][2 tiles][O columns, m, l][128 rows]
  int window;
  float scale_log2;              // scale * log2(e)
  float cap2;                    // cap * log2(e)
  float cap_x;                   // scale / cap
};

constexpr int PF_KEYS = 128;     // keys of a tile
constexpr int PF_MIN_TILES = 4;  // key tiles of a part, at least
constexpr int PF_ITEMS = 3;      // items in flight between the warps
constexpr int PF_AHEAD = 2;      // a CTA draws its next item when the loads of the present one come to its last two key tiles
constexpr int PF_GUARDS = 2;     // warps that guard V
constexpr int PF_TAIL = 4;       // key tiles at the end of an item among which each of its two row tiles ends
constexpr int PF_NTHREADS = 512;
constexpr int PF_LAUNCH_REGS = 128, PF_SOFTMAX_REGS = 184, PF_OTHER_REGS = 72;   // a thread
static_assert(256 * PF_SOFTMAX_REGS + 256 * PF_OTHER_REGS <= PF_NTHREADS * PF_LAUNCH_REGS, "register split");

template <int D>
struct PrefillCfg {
  static constexpr int HALVES = D / 64;
  static constexpr int HALF_BYTES = 128 * 128;              // 128 rows of one 64-column block
  static constexpr int TILE_BYTES = HALVES * HALF_BYTES;    // a Q, K or V tile
  static constexpr int NK = D == 128 ? 3 : 6;               // rings of K tiles and of V tiles
  static constexpr int NV = D == 128 ? 2 : 4;
  static constexpr int CTRL_BYTES = 1024;
  static constexpr int DYN_BYTES = 1024 + (2 + NK + NV) * TILE_BYTES + CTRL_BYTES;
  static constexpr int COL_S = 0, COL_O = 256, TMEM_COLS = 512;
  static_assert(DYN_BYTES <= 232448, "shared memory");
};

struct PrefillItem {
  int s, g, tok0, n;             // sequence, KV head, first token of the pair within the sequence, new tokens of the sequence
  int L, row0;                   // context length; cu_tokens[s]
  int keys;                      // tokens of the context that the table row can describe
  int part;                      // slot of its partial result, or -1: the item is whole
  int begin[2], end[2];          // key tiles [begin, end) of each tile; begin == end: none
  int plain, edges;              // key tiles [plain, edges) are seen whole by every row of both tiles
  int rows[2];                   // tokens of each tile
};

struct PrefillCtrl {
  // per key tile c of the CTA (mod 8): K has landed; V has landed; V has passed the guard; step c is done, i.e. the products of
  // K(c) and of V(c - 1) for both tiles of the pair
  uint64_t k_full[8], v_full[8], v_ok[8], step[8];
  uint64_t q_full[2], q_free[2], s_full[2];
  uint64_t p_part[2][2];                         // per tile: the weights of its first, of its second 64 keys are stored
  uint64_t o_full[2];                            // the item's last product into O is done
  uint64_t item_full[PF_ITEMS], item_free[PF_ITEMS], item_ask;
  uint64_t drained;
  PrefillItem item[PF_ITEMS];
  uint32_t page_bad[8];                          // per key tile (mod 8): bit j set = its page j had a bad id
  uint32_t v_bad[8][4];                          // per key tile: keys whose V held something non-finite
  uint32_t abort, tmem_base;
};
static_assert(sizeof(PrefillCtrl) <= 1024, "control block");

// The tokens of a pair slot: sequence s (whose rows begin at row0, row1 - row0 of them), first token tok0.  false: none.  One
// warp; 32 probes per round.
__device__ __forceinline__ bool prefill_slot(const PrefillParams& P, int slot, int lane, int& s, int& row0, int& row1, int& tok0) {
  const int TP = 2 * P.TQ;
  int lo = 0, len = P.S;                                // the last sequence whose first slot is at or before this one
  while (len > 1) {
    const int step = (len + 31) / 32, i = lane * step;
    const bool below = i < len && __ldg(P.cu_tokens + lo + i) / TP + lo + i <= slot;
    const uint32_t m = __ballot_sync(0xffffffffu, below);
    const int b = m ? 31 - __clz(m) : 0;
    lo += b * step;
    len = min(step, len - b * step);
  }
  s = lo;
  row0 = __ldg(P.cu_tokens + lo);
  row1 = __ldg(P.cu_tokens + lo + 1);
  tok0 = (slot - (row0 / TP + lo)) * TP;
  return row0 >= 0 && row1 <= P.N && tok0 >= 0 && tok0 < row1 - row0;
}

// first and one-past-last key that token j of a sequence sees
__device__ __forceinline__ int2 prefill_interval(const PrefillParams& P, int L, int keys, int n, int row0, int prefix, int j) {
  const int pos = L - n + j;
  int lo = 0;
  if (P.window > 0) lo = max(lo, pos - P.window + 1);
  if (P.key_begin) lo = max(lo, __ldg(P.key_begin + row0 + j));
  const int hi = pos < 0 ? 0 : min(keys, max(pos + 1, prefix));
  return lo < hi ? make_int2(lo, hi) : make_int2(0, 0);
}

// Bounded wait that also gives up when the CTA's abort flag is up.  A poll suspends the thread in hardware for a while: most
// waits end in the first few, and the clock, whose reading costs more than a tile's barrier, comes into it after those.
__device__ __forceinline__ bool prefill_wait(uint32_t bar, uint32_t parity, const uint32_t* abort_flag) {
  if (mbar_try_wait(bar, parity)) return true;
  unsigned long long t0 = 0ull;
#pragma unroll 1
  for (uint32_t i = 1;; ++i) {
    if (mbar_try_wait_hint(bar, parity, PDATTN_WAIT_HINT_NS)) return true;
    if ((i & 63u) == 0u) {
      const unsigned long long now = globaltimer_ns();
      if (t0 == 0ull) t0 = now;
      if (*reinterpret_cast<const volatile uint32_t*>(abort_flag) || now - t0 > kWaitLimitNs) return false;
    }
  }
}

__device__ __forceinline__ uint64_t pack_f32x2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack_f32x2(uint64_t v, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// x <- tanh(x k), 32 values, to 2^-21 of each.  Capped scores mostly lie well inside the cap: up to 0.6 of it an odd polynomial (see
// kTanh) does it on the FMA pipe; the exponential unit, which the softmax needs, would be asked three times per score
// otherwise.  A warp that holds a larger one works out both forms and chooses value by value, as tanh_any does: a score's tanh has
// the same bits whatever else its warp holds.  Rows that no token owns (`valid`; they hold what an earlier kernel left) do not count.
__device__ __forceinline__ void tanh_columns(uint32_t (&x)[32], float k, bool valid) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 32; i += 2) top = max3(top, fabsf(__uint_as_float(x[i])), fabsf(__uint_as_float(x[i + 1])));
  const uint64_t kk = pack_f32x2(k, k);
  auto pair = [&](int i, auto far_) {
    const uint64_t t = mul_f32x2(pack_f32x2(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), kk);
    const uint64_t u = mul_f32x2(t, t);
    uint64_t p = fma_f32x2(pack_f32x2(kTanh[0], kTanh[0]), u, pack_f32x2(kTanh[1], kTanh[1]));
    p = fma_f32x2(p, u, pack_f32x2(kTanh[2], kTanh[2]));
    p = fma_f32x2(p, u, pack_f32x2(kTanh[3], kTanh[3]));
    p = fma_f32x2(p, u, pack_f32x2(1.f, 1.f));
    float y[2];
    unpack_f32x2(mul_f32x2(p, t), y[0], y[1]);
    if constexpr (decltype(far_)::value) {
      float tt[2];
      unpack_f32x2(t, tt[0], tt[1]);
#pragma unroll
      for (int e = 0; e < 2; ++e) y[e] = fabsf(tt[e]) <= kTanhNear ? y[e] : tanh_far(tt[e]);
    }
    x[i] = __float_as_uint(y[0]);
    x[i + 1] = __float_as_uint(y[1]);
  };
  if (__any_sync(0xffffffffu, valid && top * fabsf(k) > kTanhNear)) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) pair(i, std::true_type{});
  } else {
#pragma unroll
    for (int i = 0; i < 32; i += 2) pair(i, std::false_type{});
  }
}

// The non-finite elements of V that the guard set to 0, for columns 32 q .. + 31 of a row that sees keys [lo, hi): rare, kept
// small rather than fast.
template <int D>
__device__ __forceinline__ void add_guarded(const PrefillParams& P, int s, int g, int lo, int hi, int q, float (&v)[32]) {
#pragma unroll 1
  for (int key = lo; key < hi; ++key) {
    const int b = key >> P.bs_log2;
    const int id = b < P.MB ? __ldg(P.block_table + static_cast<int64_t>(s) * P.MB + b) : -1;
    if (id < 0 || id >= P.NB) continue;
    const __nv_bfloat16* row = P.v_cache + id * P.sb + g * P.sh + (key & ((1 << P.bs_log2) - 1)) * P.st + q * 32;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 w = *reinterpret_cast<const uint4*>(row + i * 8);
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if ((u[e] & 0x7f80u) == 0x7f80u) v[i * 8 + 2 * e] += __uint_as_float(u[e] << 16);
        if ((u[e] & 0x7f800000u) == 0x7f800000u) v[i * 8 + 2 * e + 1] += __uint_as_float(u[e] & 0xffff0000u);
      }
    }
  }
}

__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }   // known to be the same in every lane

// CAP: scores capped by a tanh.  GEN: scores brought to base-2 units one by one (distance bias, or a scale that is not
// positive); without it the scale rides in the exponent's multiply-add.
template <int D, bool CAP, bool GEN>
__global__ void __launch_bounds__(PF_NTHREADS, 1)
prefill_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
               const __grid_constant__ CUtensorMap tmV, const __grid_constant__ PrefillParams P) {
  using C = PrefillCfg<D>;
  constexpr int NK = C::NK, NV = C::NV;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t pad = (1024u - (raw & 1023u)) & 1023u;
  uint8_t* smem = smem_raw + pad;
  const uint32_t sQ = raw + pad, sK = sQ + 2 * C::TILE_BYTES, sV = sK + NK * C::TILE_BYTES;
  PrefillCtrl* ctrl = reinterpret_cast<PrefillCtrl*>(smem + (2 + NK + NV) * C::TILE_BYTES);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float NEG_INF = __int_as_float(0xff800000);

  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&ctrl->drained), 1);
    mbar_init(smem_u32(&ctrl->item_ask), 1);
    for (int i = 0; i < 8; ++i) {
      mbar_init(smem_u32(&ctrl->k_full[i]), 1);
      mbar_init(smem_u32(&ctrl->v_full[i]), 1);
      mbar_init(smem_u32(&ctrl->v_ok[i]), PF_GUARDS);
      mbar_init(smem_u32(&ctrl->step[i]), 1);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&ctrl->q_full[t]), 1);
      mbar_init(smem_u32(&ctrl->q_free[t]), 1);
      mbar_init(smem_u32(&ctrl->s_full[t]), 1);
      mbar_init(smem_u32(&ctrl->p_part[t][0]), 4);
      mbar_init(smem_u32(&ctrl->p_part[t][1]), 4);
      mbar_init(smem_u32(&ctrl->o_full[t]), 1);
    }
    for (int i = 0; i < PF_ITEMS; ++i) {
      mbar_init(smem_u32(&ctrl->item_full[i]), 1);
      mbar_init(smem_u32(&ctrl->item_free[i]), 8 + 1 + 2 + PF_GUARDS);   // softmax, MMA, loads, guards
    }
    ctrl->abort = 0;
    fence_mbar_init();
  }
  if (warp == 8) {
    tmem_alloc(smem_u32(&ctrl->tmem_base), C::TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = uniform(static_cast<int>(*reinterpret_cast<volatile uint32_t*>(&ctrl->tmem_base)));
  asm volatile("griddepcontrol.wait;" ::: "memory");   // a programmatic dependent of the kernel before it on the stream
  const uint32_t* abort_flag = &ctrl->abort;
  auto fail = [&]() {
    atomicOr(&P.hdr->err, ERR_TIMEOUT);
    atomicExch(&ctrl->abort, 1u);
  };
  // the k-th item of this CTA (false: no more, or a wait ran out); uniform over the warp
  auto get_item = [&](int k, const PrefillItem*& it) -> bool {
    const int e = k % PF_ITEMS;
    if (!__all_sync(0xffffffffu, prefill_wait(smem_u32(&ctrl->item_full[e]), (k / PF_ITEMS) & 1, abort_flag))) {
      if (lane == 0) fail();
      return false;
    }
    it = &ctrl->item[e];
    return it->s >= 0;
  };
  auto done_item = [&](int k) {      // the warp reads nothing of the k-th item any more
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&ctrl->item_free[k % PF_ITEMS]));
  };
  auto active = [](const PrefillItem& it, int t, int kt) { return kt >= it.begin[t] && kt < it.end[t]; };
  auto tiles_from = [](const PrefillItem& it) {
    return it.begin[0] == it.end[0] ? it.begin[1] : it.begin[1] == it.end[1] ? it.begin[0] : min(it.begin[0], it.begin[1]);
  };
  auto tiles_to = [](const PrefillItem& it) { return max(it.begin[0] == it.end[0] ? 0 : it.end[0], it.begin[1] == it.end[1] ? 0 : it.end[1]); };
  // whether key tile kt may be masked for some row of the pair
  auto edge = [](int plain, int edges, int kt) { return kt < plain || kt >= edges; };

  // The softmax threads hold many scores each; they take the registers that the others leave.
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PF_OTHER_REGS));
    if (warp == 12) {
      // ================= items.  Each is drawn no earlier than its loads can begin: what a CTA draws ahead, one that is
      // idle cannot have (37 sequences of 36 tokens over 2048 keys, 28/4 heads, an item per SM: 82 us drawn three ahead, 51 so)
      int next = blockIdx.x;
      const int n_units = P.n_items * P.splits;
      for (int k = 0;; ++k) {
        PrefillItem it;
        it.s = -1;
        auto draw = [&]() {
          int drawn = 0;
          if (lane == 0) drawn = atomicAdd(&P.hdr->counter, 1);
          next = static_cast<int>(gridDim.x) + __shfl_sync(0xffffffffu, drawn, 0);
        };
        if (k > 0) {
          if (!__all_sync(0xffffffffu, prefill_wait(smem_u32(&ctrl->item_ask), (k - 1) & 1, abort_flag))) {
            if (lane == 0) fail();
            break;
          }
          draw();
        }
        for (; static_cast<unsigned>(next) < static_cast<unsigned>(n_units); draw()) {   // (slots without tokens are passed over)
          const int slots = P.n_items / P.Hkv;
          const int unit = next, item = unit / P.splits, split = unit - item * P.splits;
          const int slot = slots - 1 - item / P.Hkv;      // the late pairs of a sequence, which see most keys, first
          it.g = item % P.Hkv;
          int s, row1;
          if (!prefill_slot(P, slot, lane, s, it.row0, row1, it.tok0)) {
            if (P.splits > 1 && split == 0 && lane == 0) P.parts[item] = 0;
            continue;
          }
          it.n = row1 - it.row0;
          it.L = max(0, __ldg(P.context_lens + s));
          // tokens past the end of the table row are left out like those of a bad page
          it.keys = static_cast<int>(min(static_cast<int64_t>(it.L), static_cast<int64_t>(P.MB) << P.bs_log2));
          if (it.keys < it.L && lane == 0) atomicOr(&P.hdr->err, ERR_BAD_PAGE);
          it.plain = 0;
          it.edges = INT_MAX;
          const int prefix = P.prefix_lens ? __ldg(P.prefix_lens + s) : 0;
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            it.rows[t] = min(P.TQ, max(0, it.n - it.tok0 - t * P.TQ));
            int lo_min = INT_MAX, lo_max = 0, hi_min = INT_MAX, hi_max = 0;
            for (int j = lane; j < it.rows[t]; j += 32) {
              const int2 v = prefill_interval(P, it.L, it.keys, it.n, it.row0, prefix, it.tok0 + t * P.TQ + j);
              if (v.y > 0) lo_min = min(lo_min, v.x);
              lo_max = max(lo_max, v.x);
              hi_max = max(hi_max, v.y);
              hi_min = min(hi_min, v.y);                  // a row that sees nothing: every tile is an edge tile
            }
            lo_min = __reduce_min_sync(0xffffffffu, lo_min);
            lo_max = __reduce_max_sync(0xffffffffu, lo_max);
            hi_min = __reduce_min_sync(0xffffffffu, hi_min);
            hi_max = __reduce_max_sync(0xffffffffu, hi_max);
            it.begin[t] = hi_max > 0 ? lo_min / PF_KEYS : 0;
            it.end[t] = hi_max > 0 ? (hi_max - 1) / PF_KEYS + 1 : 0;
            if (hi_max > 0) {
              it.plain = max(it.plain, (lo_max + PF_KEYS - 1) / PF_KEYS);
              it.edges = min(it.edges, hi_min / PF_KEYS);
            }
          }
          it.part = -1;
          if (P.splits > 1) {
            // this unit's share of the item's key tiles
            const int k0 = tiles_from(it), n = max(0, tiles_to(it) - k0);
            const int parts = max(1, min(P.splits, n / PF_MIN_TILES));
            if (split == 0 && lane == 0) P.parts[item] = parts;
            if (split >= parts) continue;
            if (parts > 1) it.part = unit;
            const int a = k0 + static_cast<int>(static_cast<int64_t>(n) * split / parts);
            const int b = k0 + static_cast<int>(static_cast<int64_t>(n) * (split + 1) / parts);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              it.begin[t] = max(it.begin[t], a);
              it.end[t] = min(it.end[t], b);
              if (it.begin[t] >= it.end[t]) it.begin[t] = it.end[t] = 0;
            }
          }
          it.s = s;
          break;
        }
        const int e = k % PF_ITEMS;
        if (!__all_sync(0xffffffffu, prefill_wait(smem_u32(&ctrl->item_free[e]), ((k / PF_ITEMS) & 1) ^ 1, abort_flag))) {
          if (lane == 0) fail();
          break;
        }
        if (lane == 0) {
          ctrl->item[e] = it;
          mbar_arrive(smem_u32(&ctrl->item_full[e]));     // (release: the item is visible to whoever sees the phase)
        }
        __syncwarp();
        if (it.s < 0) break;
      }
      // this CTA draws no more items; the last CTA to say so rearms the counter for the next call
      if (lane == 0 && atomicAdd(&P.hdr->done, 1) == static_cast<int>(gridDim.x) - 1) {
        P.hdr->done = 0;
        P.hdr->counter = 0;
      }
    } else if (warp == 10 || warp == 11) {
      // ================= loads: Q and K (warp 10), V (warp 11)
      const bool isV = warp == 11;
      const int ppt = PF_KEYS >> P.bs_log2;               // pages of a key tile
      const int j = lane & (ppt - 1), h = lane / ppt;
      const int ring = isV ? NV : NK;
      const CUtensorMap* tm = isV ? &tmV : &tmK;
      const uint32_t dst0 = (isV ? sV : sK) + h * C::HALF_BYTES + (j << P.bs_log2) * 128;
      uint64_t* full = isV ? ctrl->v_full : ctrl->k_full;
      bool any_bad = false, ok = true;
      int c = 0, slot = 0, nq[2] = {0, 0};
      int start = 0, start1 = 0, read = -1;               // first tiles of this item and the one before; items known to be released
      const PrefillItem* ip;
      for (int k = 0; ok && get_item(k, ip); ++k) {
        const PrefillItem& it = *ip;
        start1 = start;
        start = c;
        const int32_t* row = P.block_table + static_cast<int64_t>(it.s) * P.MB;
        const int npages = static_cast<int>((static_cast<int64_t>(it.keys) + (1 << P.bs_log2) - 1) >> P.bs_log2);
        auto page_id = [&](int kt) {
          const int i = kt * ppt + j;
          return i < npages ? __ldg(row + i) : -2;             // -2: past the end, filled with zeros
        };
        const int k0 = tiles_from(it), k1 = tiles_to(it);
        int id_next = k0 < k1 ? page_id(k0) : 0;
        bool asked = isV;                                 // for the next item; the K loads ask
        if (!isV) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (!ok || it.begin[t] == it.end[t]) continue;
            ok = __all_sync(0xffffffffu, prefill_wait(smem_u32(&ctrl->q_free[t]), (nq[t] & 1) ^ 1, abort_flag));
            if (ok) ++nq[t];
            if (ok && lane == 0) {
              const uint32_t bar = smem_u32(&ctrl->q_full[t]);
              mbar_arrive_expect_tx(bar, static_cast<uint32_t>(C::HALVES * P.TQ * P.G * 128));
#pragma unroll
              for (int hh = 0; hh < C::HALVES; ++hh)
                tma_load_4d(sQ + t * C::TILE_BYTES + hh * C::HALF_BYTES, &tmQ, hh * 64, 0, it.g, it.row0 + it.tok0 + t * P.TQ, bar);
            }
            __syncwarp();
          }
        }
        for (int kt = k0; kt < k1 && ok; ++kt) {
          int id = id_next;
          if (kt + 1 < k1) id_next = page_id(kt + 1);
          if (!asked && kt >= k1 - PF_AHEAD) {
            if (lane == 0) mbar_arrive(smem_u32(&ctrl->item_ask));
            asked = true;
          }
          if (!active(it, 0, kt) && !active(it, 1, kt)) continue;
          const bool bad = id != -2 && (id < 0 || id >= P.NB);
          const uint32_t badmask = __ballot_sync(0xffffffffu, bad && h == 0);
          any_bad |= badmask != 0;
          if (id < 0 || id >= P.NB) id = P.NB;            // out-of-bounds coordinate: TMA fills zeros, nothing is read
          // the slot's previous tile: K(c - NK) is done with step c - NK, V(c - NV) with step c - NV + 1
          const int need = isV ? c - NV + 1 : c - NK;
          // V(c) brings a new v_bad[c & 7], and the softmax warps read the old one only after they handed that tile's weights over:
          // the products do not hold it for them.  Within an item a row tile's next weights do.  That leaves the last key tile of
          // each of the two; they end at most 2 apart (hi grows by at most one a token, and a pair has at most 256 tokens), so
          // among the item's last PF_TAIL.  Where c - 8 is one of those, the release of its item says that it was read.  (Items
          // three back are released, or this one could not have been published.)
          const int last = c - 8;
          const int owner = last < start && last >= start - PF_TAIL ? k - 1 : last < start1 && last >= start1 - PF_TAIL ? k - 2 : -1;
          const bool owed = isV && last >= 0 && owner > read;
          if (owed) read = owner;
          // (one copy of the wait: a second one here, or the read of v_bad before the weights go, moves code and costs 1-5 %)
#pragma unroll 1
          for (int i = owed ? 0 : c >= ring ? 1 : 2; i < 2 && ok; ++i)
            ok = __all_sync(0xffffffffu, prefill_wait(smem_u32(i ? &ctrl->step[need & 7] : &ctrl->item_free[owner % PF_ITEMS]),
                                                      (i ? need >> 3 : owner / PF_ITEMS) & 1, abort_flag));
          if (!ok) break;
          const uint32_t bar = smem_u32(&full[c & 7]);
          if (lane == 0) {
            if (!isV) ctrl->page_bad[c & 7] = badmask;
            mbar_arrive_expect_tx(bar, static_cast<uint32_t>(C::TILE_BYTES));
          }
          __syncwarp();
          if (h < C::HALVES) tma_load_4d(dst0 + slot * C::TILE_BYTES, tm, h * 64, 0, it.g, id, bar);
          if (++slot == ring) slot = 0;
          ++c;
        }
        if (!asked && lane == 0) mbar_arrive(smem_u32(&ctrl->item_ask));
        done_item(k);
      }
      if (lane == 0) {
        if (any_bad) atomicOr(&P.hdr->err, ERR_BAD_PAGE);
        if (!ok) fail();
      }
      if (*reinterpret_cast<const volatile uint32_t*>(abort_flag)) {
        // given up: no copy may still be on its way into this CTA's shared memory when it ends
        for (int i = max(0, c - ring); i < c; ++i) mbar_wait(smem_u32(&full[i & 7]), (i >> 3) & 1);
#pragma unroll
        for (int t = 0; t < 2; ++t)
          if (nq[t] > 0) mbar_wait(smem_u32(&ctrl->q_full[t]), (nq[t] - 1) & 1);
      }
    } else if (warp == 8) {
      // ================= MMA issue: the warp runs the loop as one, one elected lane issues.  The two tiles take strict turns:
      // that keeps their softmax phases apart, so that one tile's exponentials run while the other's products do.
      uint32_t elected;
      asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(elected));
      const PrefillItem* ip;
      int c = 0, kslot = 0, vslot = 0;   // key tiles of this CTA so far; ring slots of K(c) and of V(c - 1)
      uint32_t nq = 0, np = 0;           // bit t: parity of q_full, p_part of tile t
      bool ok = true;
      constexpr uint32_t ID_S = umma_idesc(128, PF_KEYS, 0, 0);   // Q (K-major) x K tile (K-major)
      constexpr uint32_t ID_O = umma_idesc(128, D, 0, 1);         // P (tensor memory) x V tile (MN-major)
      const uint64_t q_desc = umma_desc(sQ, 16, 1024), k_desc = umma_desc(sK, 16, 1024), v_desc = umma_desc(sV, C::HALF_BYTES, 1024);
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        ok = ok && __all_sync(0xffffffffu, prefill_wait(smem_u32(bar), parity, abort_flag));
      };
      for (int k = 0; ok && get_item(k, ip); ++k) {
        const int b0 = uniform(ip->begin[0]), e0 = uniform(ip->end[0]), b1 = uniform(ip->begin[1]), e1 = uniform(ip->end[1]);
        const int k0 = uniform(tiles_from(*ip)), k1 = uniform(tiles_to(*ip));
        done_item(k);
        // bit t: O_t starts anew; scores of tile c - 1 whose product is to come
        uint32_t fresh = 3u, pending = 0u;
        for (int kt = k0; kt <= k1 && ok; ++kt) {
          const uint32_t mine = (kt >= b0 && kt < e0 ? 1u : 0u) | (kt >= b1 && kt < e1 ? 2u : 0u);
          if (!mine && kt < k1) continue;
          if (pending) wait(&ctrl->v_ok[(c - 1) & 7], ((c - 1) >> 3) & 1);
          if (mine) wait(&ctrl->k_full[c & 7], (c >> 3) & 1);
          // (loops, not straight-line code: see prefill_wait)
#pragma unroll 1
          for (int t = 0; t < 2 && ok; ++t) {
            const uint32_t tS = tbase + C::COL_S + t * 128, tO = tbase + C::COL_O + t * D;
            if ((pending >> t) & 1) {
              // O_t (+)= P_t . V of key tile c - 1; the first half runs while the second is still being made
              uint64_t vd = v_desc + static_cast<uint64_t>(uniform(vslot) * (C::TILE_BYTES >> 4));
              uint32_t accum = ((fresh >> t) & 1) ^ 1, a = tS;
#pragma unroll 1
              for (int h = 0; h < 2; ++h) {
                wait(&ctrl->p_part[t][h], (np >> t) & 1);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  umma_ts_elected(tO, a, vd, ID_O, accum, elected);
                  accum = 1u;
                  a += 8;
                  vd += 2048 >> 4;
                }
              }
              np ^= 1u << t;
              fresh &= ~(1u << t);
              if (!((mine >> t) & 1)) tc_commit_elected(smem_u32(&ctrl->o_full[t]), elected);   // that was this tile's last
            }
            if ((mine >> t) & 1) {
              if (kt == (t ? b1 : b0)) {
                wait(&ctrl->q_full[t], (nq >> t) & 1);
                nq ^= 1u << t;
              }
              if (!ok) break;
              tc_fence_after();
              uint64_t kd = k_desc + static_cast<uint64_t>(uniform(kslot) * (C::TILE_BYTES >> 4));
              uint64_t qd = q_desc + static_cast<uint64_t>(t * (C::TILE_BYTES >> 4));
              uint32_t accum = 0u;
#pragma unroll 1
              for (int hh = 0; hh < C::HALVES; ++hh) {
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) {
                  umma_ss_elected(tS, qd + kk * 2, kd + kk * 2, ID_S, accum, elected);
                  accum = 1u;
                }
                qd += C::HALF_BYTES >> 4;
                kd += C::HALF_BYTES >> 4;
              }
              tc_commit_elected(smem_u32(&ctrl->s_full[t]), elected);
              if (kt == (t ? e1 : e0) - 1) tc_commit_elected(smem_u32(&ctrl->q_free[t]), elected);
            }
          }
          pending = mine;
          if (kt == k1) break;                            // those were the item's last products
          // K(c) and V(c - 1) have been used (an earlier item's last V included)
          tc_commit_elected(smem_u32(&ctrl->step[c & 7]), elected);
          ++c;
          if (++kslot == NK) kslot = 0;
          if (c > 1 && ++vslot == NV) vslot = 0;
        }
      }
      if (lane == 0 && !ok) fail();
      // nothing that was issued may still be running on the tensor cores when the tensor memory goes back
      tc_commit_elected(smem_u32(&ctrl->drained), elected);
      mbar_wait(smem_u32(&ctrl->drained), 0);
      __syncwarp();
    } else if (warp >= 16 - PF_GUARDS) {
      // ================= guards of V: each takes its share of every 64 keys
      const int w = warp - (16 - PF_GUARDS);
      constexpr int WORDS = 4 / PF_GUARDS;                // 32 keys each
      const PrefillItem* ip;
      int c = 0, slot = 0;
      bool ok = true;
      for (int k = 0; ok && get_item(k, ip); ++k) {
        const PrefillItem& it = *ip;
        const int k1 = tiles_to(it);
        for (int kt = tiles_from(it); kt < k1; ++kt) {
          if (!active(it, 0, kt) && !active(it, 1, kt)) continue;
          if (!__all_sync(0xffffffffu, prefill_wait(smem_u32(&ctrl->v_full[c & 7]), (c >> 3) & 1, abort_flag))) {
            ok = false;
            break;
          }
          if (edge(it.plain, it.edges, kt)) {
            const uint32_t base = sV + slot * C::TILE_BYTES;
#pragma unroll 1
            for (int e = 0; e < WORDS; ++e) {
              // 32 keys: a key's row of a 64-column block is 128 bytes = 8 chunks, four keys per warp-wide load.  A bf16 is not
              // finite when its eight exponent bits are all set: adding one to them then carries into the sign's place.
              const uint32_t rows = base + (w * WORDS + e) * 32 * 128;
              uint32_t bad = 0u;
#pragma unroll 1
              for (int hh = 0; hh < C::HALVES; ++hh) {
                uint32_t v[8][4], hit[8];
#pragma unroll
                for (int q = 0; q < 8; ++q)
                  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v[q][0]), "=r"(v[q][1]), "=r"(v[q][2]), "=r"(v[q][3])
                               : "r"(rows + hh * C::HALF_BYTES + (q * 32 + lane) * 16));
                uint32_t any = 0u;
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                  hit[q] = 0u;
#pragma unroll
                  for (int i = 0; i < 4; ++i) hit[q] |= (v[q][i] & 0x7f807f80u) + 0x00800080u;
                  any |= hit[q];
                }
                if (any & 0x80008000u) {
#pragma unroll
                  for (int q = 0; q < 8; ++q) {
                    if (!(hit[q] & 0x80008000u)) continue;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                      if ((v[q][i] & 0x7f80u) == 0x7f80u) v[q][i] &= 0xffff0000u;
                      if ((v[q][i] & 0x7f800000u) == 0x7f800000u) v[q][i] &= 0x0000ffffu;
                    }
                    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(rows + hh * C::HALF_BYTES + (q * 32 + lane) * 16),
                                 "r"(v[q][0]), "r"(v[q][1]), "r"(v[q][2]), "r"(v[q][3]) : "memory");
                    bad |= 1u << (q * 4 + (lane >> 3));
                  }
                }
              }
              bad = __reduce_or_sync(0xffffffffu, bad);
              if (lane == 0) ctrl->v_bad[c & 7][w * WORDS + e] = bad;
            }
            fence_proxy_async();         // the stores above before the tensor cores' reads
            __syncwarp();
          }
          if (lane == 0) mbar_arrive(smem_u32(&ctrl->v_ok[c & 7]));
          if (++slot == NV) slot = 0;
          ++c;
        }
        done_item(k);
      }
      if (!ok && lane == 0) fail();
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(PF_SOFTMAX_REGS));
    // ================= softmax: a thread owns row r of tile t
    const int t = warp >> 2;
    const int r = threadIdx.x & 127;
    const uint32_t lane_addr = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tbase + C::COL_S + t * 128 + lane_addr, tO = tbase + C::COL_O + t * D + lane_addr;
    const int rj = r / P.G, rh = r - rj * P.G;          // token in the tile, head in the KV group
    const float sc = CAP ? P.cap2 : P.scale_log2;       // brings scores (with CAP: their tanh) to base-2 units
    // warp-uniform: tensor-memory accesses need the whole warp.  No thread leaves this path early: after a failed wait it
    // carries on, and its further waits return at once.
    auto wait_all = [&](uint64_t* bar, uint32_t parity) {
      if (!__all_sync(0xffffffffu, prefill_wait(smem_u32(bar), parity, abort_flag)) && lane == 0) fail();
    };
    const PrefillItem* ip;
    int c = 0, nt = 0, no = 0;         // key tiles of the CTA, of this tile; items of this tile that had keys
    for (int k = 0; get_item(k, ip); ++k) {
      const PrefillItem& it = *ip;
      const int my_begin = it.begin[t], my_end = it.end[t], my_rows = it.rows[t], other_begin = it.begin[t ^ 1], other_end = it.end[t ^ 1], plain = it.plain, edges = it.edges;
      const int j = it.tok0 + t * P.TQ + rj;            // token within the sequence
      const bool valid = rj < my_rows;
      int lo = 0, hi = 0;
      const int pos = it.L - it.n + j;
      if (valid) {
        const int2 v = prefill_interval(P, it.L, it.keys, it.n, it.row0, P.prefix_lens ? __ldg(P.prefix_lens + it.s) : 0, j);
        lo = v.x;
        hi = v.y;
      }
      const float slope2 = (GEN && valid && P.slopes) ? -1.4426950408889634f * __ldg(P.slopes + it.g * P.G + rh) : 0.f;
      float m = NEG_INF, l = 0.f;
      int poison_from = INT_MAX, poison_to = -1;        // key tiles with a non-finite V that this row sees
      const int k1 = tiles_to(it);
      for (int kt = tiles_from(it); kt < k1; ++kt) {
        if (kt < my_begin || kt >= my_end) {
          if (kt >= other_begin && kt < other_end) ++c;
          continue;
        }
        wait_all(&ctrl->s_full[t], nt & 1);
        tc_fence_after();
        const bool first = kt == my_begin;
        // Two passes over the scores, 32 columns at a time, so that the loops stay small: a tile's worth of straight-line code
        // would not fit the instruction caches that all the roles share.  The next columns are on their way while these are
        // worked on.  The first pass takes the maximum, and where scores are modified or masked it writes them back; the
        // second makes the weights, whose columns 16 q .. + 15 lie over scores that have been read.
        uint32_t x0[32], x1[32];
        auto first_pass = [&](auto masked_) {
          constexpr bool MASKED = decltype(masked_)::value;
          const uint32_t pb = MASKED ? ctrl->page_bad[c & 7] : 0u;
          float m4[4] = {NEG_INF, NEG_INF, NEG_INF, NEG_INF};
          auto columns = [&](uint32_t (&x)[32], int q) {
            const int k0 = kt * PF_KEYS + q * 32;
            if (CAP) tanh_columns(x, P.cap_x, valid);
            if (GEN) {
              const float d0 = static_cast<float>(k0 - pos);
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                const float v = __uint_as_float(x[i]) * sc;
                x[i] = __float_as_uint(fmaf(slope2, fabsf(d0 + static_cast<float>(i)), v));
              }
            }
            if (MASKED) {
              const int a = lo - k0, b = hi - k0;
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (i < a || i >= b) x[i] = __float_as_uint(NEG_INF);
              if (pb) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if ((pb >> ((q * 32 + i) >> P.bs_log2)) & 1u) x[i] = __float_as_uint(NEG_INF);
              }
            }
            if (CAP || GEN || MASKED) tmem_st32(tS + q * 32, x);
#pragma unroll
            for (int i = 0; i < 32; i += 2) m4[(i >> 1) & 3] = max3(m4[(i >> 1) & 3], __uint_as_float(x[i]), __uint_as_float(x[i + 1]));
          };
          tmem_ld32(tS, x0);
#pragma unroll 1
          for (int q = 0; q < 4; q += 2) {
            tc_wait_ld();
            tmem_ld32(tS + q * 32 + 32, x1);
            columns(x0, q);
            tc_wait_ld();
            if (q == 0) tmem_ld32(tS + 64, x0);
            columns(x1, q + 1);
          }
          if (CAP || GEN || MASKED) tc_wait_st();
          return fmaxf(max3(m4[0], m4[1], m4[2]), m4[3]);
        };
        const bool masked = edge(plain, edges, kt) || ctrl->page_bad[c & 7] != 0;
        float mx = masked ? first_pass(std::true_type{}) : first_pass(std::false_type{});
        tmem_ld32(tS, x0);                              // (for the second pass)
        if (!GEN) mx = mx == NEG_INF ? NEG_INF : mx * sc;
        const bool grow = first || mx > m + 8.f;
        const float m_new = grow ? fmaxf(m, mx) : m;
        const float mu = m_new == NEG_INF ? 0.f : m_new;
        const float alpha = grow ? fast_exp2(m - mu) : 1.f;
        m = m_new;
        if (__any_sync(0xffffffffu, valid && !first && alpha != 1.f)) {
          // new reference: scale this row of O (the product before this one was done when the scores came)
#pragma unroll 1
          for (int q = 0; q < D / 16; ++q) {
            uint32_t o[16];
            tmem_ld16(tO + q * 16, o);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
            tmem_st16(tO + q * 16, o);
          }
        }
        uint64_t sum0 = 0ull, sum1 = 0ull;
        const uint64_t sc2 = pack_f32x2(sc, sc), mu2 = pack_f32x2(-mu, -mu);
        auto weights = [&](const uint32_t (&x)[32], int q) {
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint64_t xx = pack_f32x2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1]));
            float p0, p1;
            unpack_f32x2(GEN ? add_f32x2(xx, mu2) : fma_f32x2(xx, sc2, mu2), p0, p1);
            p0 = fast_exp2(p0);
            p1 = fast_exp2(p1);
            const uint64_t pp = pack_f32x2(p0, p1);
            if (i & 1) sum1 = add_f32x2(sum1, pp);
            else sum0 = add_f32x2(sum0, pp);
            pk[i] = pack_bf16x2(p0, p1);
          }
          tmem_st16(tS + q * 16, pk);
        };
#pragma unroll 1
        for (int q = 0; q < 4; q += 2) {
          tc_wait_ld();
          tmem_ld32(tS + q * 32 + 32, x1);
          weights(x0, q);
          tc_wait_ld();
          if (q == 0) tmem_ld32(tS + 64, x0);
          weights(x1, q + 1);
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&ctrl->p_part[t][q >> 1]));
        }
        {
          float a0, a1, b0, b1;
          unpack_f32x2(sum0, a0, a1);
          unpack_f32x2(sum1, b0, b1);
          l = l * alpha + ((a0 + a1) + (b0 + b1));
        }
        if (masked) {
          wait_all(&ctrl->v_ok[c & 7], (c >> 3) & 1);
          uint32_t seen = 0;
          if (edge(plain, edges, kt)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int a = max(0, min(32, lo - kt * PF_KEYS - 32 * e)), b = max(0, min(32, hi - kt * PF_KEYS - 32 * e));
              const uint32_t vis = (b >= 32 ? 0xffffffffu : (1u << b) - 1u) & ~(a >= 32 ? 0xffffffffu : (1u << a) - 1u);
              seen |= *reinterpret_cast<volatile uint32_t*>(&ctrl->v_bad[c & 7][e]) & vis;
            }
          }
          if (seen) {
            poison_from = min(poison_from, kt);
            poison_to = kt;
          }
        }
        ++nt;
        ++c;
      }
      // ---- the item's rows
      if (my_rows > 0) {
        const bool any = my_begin != my_end;
        if (any) {
          wait_all(&ctrl->o_full[t], no & 1);
          ++no;
          tc_fence_after();
        }
        // a part of an item leaves its sums as they are
        float* part = it.part >= 0 ? P.partials + (static_cast<int64_t>(it.part) * 2 + t) * ((D + 2) * 128) + r : nullptr;
        const float inv = part ? 1.f : l > 0.f ? 1.f / l : (l != l ? l : 0.f);
        if (part) {
          part[D * 128] = m;
          part[(D + 1) * 128] = l;
        }
        // A thread holds a row; written like that, every store of a warp would touch 32 lines.  Groups of four lanes transpose
        // 4 x 4 chunks of 16 bytes among themselves, so that a store writes 64 bytes of each of eight rows.
        __nv_bfloat16* out0 = P.out + (static_cast<int64_t>(it.row0 + it.tok0 + t * P.TQ) * P.Hq + it.g * P.G) * D;
        const int offset = valid ? (rj * P.Hq + rh) * D : -1;     // of this thread's row
#pragma unroll 1
        for (int q = 0; q < D / 32; ++q) {
          uint32_t o[32];
          if (any) {
            tmem_ld32(tO + q * 32, o);
            tc_wait_ld();
          }
          float v[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = any && inv != 0.f ? __uint_as_float(o[i]) * inv : 0.f;
          if (poison_to >= 0) add_guarded<D>(P, it.s, it.g, max(lo, poison_from * PF_KEYS), min(hi, (poison_to + 1) * PF_KEYS), q, v);
          if (part) {
#pragma unroll
            for (int i = 0; i < 32; ++i) part[(q * 32 + i) * 128] = v[i];
            continue;
          }
          uint4 w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            w[i] = make_uint4(pack_bf16x2(v[8 * i], v[8 * i + 1]), pack_bf16x2(v[8 * i + 2], v[8 * i + 3]),
                              pack_bf16x2(v[8 * i + 4], v[8 * i + 5]), pack_bf16x2(v[8 * i + 6], v[8 * i + 7]));
          __syncwarp();
          // afterwards chunk (lane & 3) of the rows of lanes 4 (lane / 4) + 0 .. 3 lies in w[0 .. 3]
          auto swap = [&](uint4& a, uint4& b, int mask) {          // lanes with the bit hand out a and keep b, the others the other way round
            const bool up = lane & mask;
            const uint4 give = up ? a : b;
            const uint4 got = make_uint4(__shfl_xor_sync(0xffffffffu, give.x, mask), __shfl_xor_sync(0xffffffffu, give.y, mask),
                                         __shfl_xor_sync(0xffffffffu, give.z, mask), __shfl_xor_sync(0xffffffffu, give.w, mask));
            if (up) a = got;
            else b = got;
          };
          swap(w[0], w[1], 1);
          swap(w[2], w[3], 1);
          swap(w[0], w[2], 2);
          swap(w[1], w[3], 2);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int at = __shfl_sync(0xffffffffu, offset, (lane & ~3) + i);
            if (at >= 0) *reinterpret_cast<uint4*>(out0 + at + q * 32 + (lane & 3) * 8) = w[i];
          }
        }
        tc_fence_before();
      }
      done_item(k);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 8) tmem_dealloc(tbase, C::TMEM_COLS);
}

// The parts of the items that were cut along the keys, put together in order: block (item, tile, 8 columns), a thread per row.
//   M = max m_j;  out = sum O_j 2^(m_j - M) / sum l_j 2^(m_j - M)
// Bound by the latency of its loads (neighbouring rows are neighbours in memory): four parts are fetched at a time.
template <int D>
__global__ void __launch_bounds__(128)
prefill_join_kernel(const __grid_constant__ PrefillParams P) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int item = blockIdx.x, t = blockIdx.y, q = blockIdx.z, r = threadIdx.x;
  const int parts = join_parts(P.parts[item], P.splits);
  if (parts <= 1) return;
  int s, row0, row1, tok0;
  prefill_slot(P, P.n_items / P.Hkv - 1 - item / P.Hkv, r & 31, s, row0, row1, tok0);
  const int g = item % P.Hkv, rj = r / P.G, rh = r - rj * P.G, j = tok0 + t * P.TQ + rj;
  if (rj >= P.TQ || j >= row1 - row0) return;
  const float* first = P.partials + (static_cast<int64_t>(item) * P.splits * 2 + t) * ((D + 2) * 128) + r;
  constexpr int64_t STEP = 2 * (D + 2) * 128;
  const float NEG_INF = __int_as_float(0xff800000);
  float M = NEG_INF, L = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int p = 0; p < parts; ++p) M = fmaxf(M, first[p * STEP + D * 128]);
#pragma unroll 4
  for (int p = 0; p < parts; ++p) {
    const float* part = first + p * STEP;
    const float m = part[D * 128], l = part[(D + 1) * 128];
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = part[(q * 8 + i) * 128];
    const float f = m == NEG_INF ? 0.f : fast_exp2(m - M);        // 0: saw nothing
    L += l * f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // infinities and NaN of V stand whatever the weight
      const bool odd = (__float_as_uint(x[i]) & 0x7f800000u) == 0x7f800000u;
      o[i] += odd ? x[i] : x[i] * f;
    }
  }
  const float inv = L > 0.f ? 1.f / L : (L != L ? L : 0.f);
  *reinterpret_cast<uint4*>(P.out + (static_cast<int64_t>(row0 + j) * P.Hq + g * P.G + rh) * D + q * 8) =
      make_uint4(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv), pack_bf16x2(o[4] * inv, o[5] * inv),
                 pack_bf16x2(o[6] * inv, o[7] * inv));
}

}  // namespace pdattn

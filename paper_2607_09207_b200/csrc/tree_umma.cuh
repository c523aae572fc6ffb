// Attention for a tree of drafted tokens over the paged cache, on the 5th-generation tensor cores: tree_kernel, tree_join_kernel.
//
//   out = softmax_t(scale q.k_t) . V over the keys before the tree and those of the tree that the token's mask names
//
// Rows.  The query rows of one KV head are packed: row r of a 128-row tile is head r % G of token r / G, so a tile holds
// floor(128 / G) whole tokens and every K/V tile is read once for all of them.
//
//   S_t[128, 128 keys] = Q_t . K^T     both from shared memory            t = 0, 1
//   O_t[128, d]       += P_t . V       P from tensor memory (over S_t's columns), V from shared memory
//
// Two softmax groups of four warps (a thread owns a row: no shuffles) keep the memory system busy, in one of two ways:
//   PAIR   trees of more than 128 rows: t are two row tiles, every key tile serves both;
//   split  at most 128 rows: both groups have the same rows and take turns with the key tiles, so two chains of scores -> weights ->
//          product run at a time and meet at the end, where each group stores half of the columns of
//          (O_0 2^(m_0 - m) + O_1 2^(m_1 - m)) / l.  The groups' tensor-memory lanes are the same: no copies for that.
//
// Work.  The key tiles of all units (sequence, KV head, pair of row tiles) form one stream that is cut into equal shares, one per
// CTA (partition.h): long contexts are spread over all SMs whatever the batch looks like, and nothing depends on the host knowing
// the lengths.  A CTA works out its share from the lengths by itself (every warp sums its part of the batch, then one warp walks).  A unit
// that a share's end cuts leaves (m, l, O) per piece, at most two a CTA; tree_join_kernel puts them together in order.
//
// Roles: warps 0-7 softmax, 8 issues the MMAs, 9 walks the units and loads Q, 10 loads K, 11 V (TMA), 12-15: over the bf16 cache two
// of them guard V (see prefill_umma.cuh: non-finite elements of V at keys that some row does not see are set to 0 and added
// again for the rows that see them); over the fp8 cache they widen the codes of K and V to fp16 (exact), which is the guard as well.
// fp8: V's pages are transposed, so its tile is K-major in the second product.
//
// Numbers: scores, maxima, sums and O in fp32.  The weights are rounded to bf16 for the second product (at most 2^-8 of each,
// independent; the fp8 form to fp16, 2^-11): the size of the final rounding.  The reference of the online softmax follows the
// running maximum when that grew by more than 2^8, so O is rarely rescaled.
//
// Every wait is bounded; on expiry the CTA raises ERR_TIMEOUT, the waits fall through, the MMA warp drains, tensor memory is
// freed and the CTA returns.
#pragma once

#include <climits>
#include <type_traits>

#include "partition.h"
#include "umma.cuh"

namespace pdattn {

constexpr int TR_CTAS = 148;                       // shares of a call, at most
constexpr int TR_MAX_SEQS = 65536;
constexpr int TR_ITEMS = 4;                        // items in flight between the warps
constexpr int TR_NTHREADS = 512;
constexpr int TR_LAUNCH_REGS = 128, TR_SOFTMAX_REGS = 184, TR_OTHER_REGS = 72;   // a thread
static_assert(256 * TR_SOFTMAX_REGS + 256 * TR_OTHER_REGS <= TR_NTHREADS * TR_LAUNCH_REGS, "register split");

struct TreeParams {
  __nv_bfloat16* out;
  const int32_t *block_table, *context_lens, *cu_tokens;
  const uint64_t* mask;
  const void* v_cache;           // for the guarded elements only: element strides, or dense code pages [d][slot]
  int64_t sb, sh, st;
  const float *k_scale, *v_scale;
  WsHeader* hdr;
  int4* rec;                     // [gridDim][2] pieces of cut units: (sequence or -1, KV head, row pair, 1: it ends the unit)
  float* partials;               // [gridDim][2][2 tiles][O columns, m, l][128 rows]
  int N, S, Hq, Hkv, G, MB, NB, bs_log2;
  int TQ;                        // tokens of a row tile: 128 / G
  int max_n;                     // tokens of a tree
  float scale_log2;              // scale * log2(e)
};

template <int D, bool PAIR, int EB>
struct TreeCfg {
  static constexpr int HALVES = D / 64;
  static constexpr int HALF_BYTES = 128 * 128;              // 128 rows of one 64-column block
  static constexpr int TILE_BYTES = HALVES * HALF_BYTES;    // a Q, K or V tile of 16-bit elements
  static constexpr int RAW_BYTES = 128 * D;                 // a K or V tile of codes
  static constexpr int QT = PAIR ? 2 : 1;
  static constexpr int LAG = PAIR ? 1 : 2;                  // the product of key tile c is issued with the scores of c + LAG
  // rings of K tiles, of V tiles, of code tiles (each of K and of V)
  static constexpr int NK = EB == 1 ? 2 : D == 128 ? 3 : 6;
  static constexpr int NV = EB == 1 ? 2 : D == 128 ? (PAIR ? 2 : 3) : (PAIR ? 4 : 6);
  static constexpr int NR = EB == 2 ? 0 : D == 128 ? (PAIR ? 1 : 2) : 4;   // (at most 4: see page_bad)
  static constexpr int RING_BYTES = (QT + NK + NV) * TILE_BYTES + 2 * NR * RAW_BYTES;
  static constexpr int CTRL_BYTES = 2048;
  static constexpr int DYN_BYTES = 1024 + RING_BYTES + CTRL_BYTES;
  static constexpr int COL_S = 0, COL_O = 256, TMEM_COLS = 512;
  static_assert(DYN_BYTES <= 232448, "shared memory");
  static_assert(NV >= LAG && NK >= 2 && (EB == 2 || NR >= 1), "rings");
};

struct TreeItem {
  int s, g, tok0, n;             // sequence (-1: no more), KV head, first token of the pair within the tree, tokens of the tree
  int row0, L;                   // cu_tokens[s]; context length
  int keys;                      // tokens of the context that the table row can describe
  int tb, te;                    // key tiles
  int edge;                      // key tiles from this one on may be masked
  int part;                      // slot of its partial result, or -1: the unit is whole
  int rows[2];                   // tokens of each row tile (split: of the one tile, twice)
};

struct TreeCtrl {
  // per key tile c of the CTA (mod 8): K, V have landed; V has passed the guard (fp8: K, V are widened); step c is done, i.e. the scores
  // of key tile c and the product of c - LAG
  uint64_t k_full[8], v_full[8], k_ok[8], v_ok[8], step[8];
  uint64_t q_full, q_ok, q_free;
  uint64_t s_full[2], p_part[2][2];              // per group: scores are there; the weights of the first, the second 64 keys are stored
  uint64_t o_full[2];                            // the item's last product into O is done
  uint64_t item_full[TR_ITEMS], item_free[TR_ITEMS];
  uint64_t drained, meet, meet_widen;            // all softmax warps are here; all widening warps are
  TreeItem item[TR_ITEMS];
  // Per key tile (mod 8): bit j set = its page j had a bad id; keys whose V held something non-finite.  Both are read before the last
  // weights of key tile c are handed over, and written anew for c + 8 only when the product of c is done (K(c + 8) is loaded after
  // step c + 8 - NK >= c + 2, or codes after those of c + 8 - NR were widened, which waits for step c + 8 - NR - NK >= c + 2).
  uint32_t page_bad[8];
  uint32_t v_bad[8][4];
  uint32_t odd[TR_ITEMS];                        // split: some row sees such a key
  uint32_t abort, tmem_base;
  float2 ml[64 * 2];                             // split: (m, l) of group 1's rows, then the factors of both groups
};
static_assert(sizeof(TreeCtrl) <= 2048, "control block");

// Bounded wait that also gives up when the CTA's abort flag is up; the clock comes into it after 64 polls.
__device__ __forceinline__ bool tree_wait(uint32_t bar, uint32_t parity, const uint32_t* abort_flag) {
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
__device__ __forceinline__ int tree_uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }   // known to be the same in every lane
__device__ __forceinline__ uint64_t tree_pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void tree_unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t tree_fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t tree_add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// Instruction descriptor as umma_idesc's, for fp16 operands.
__host__ __device__ constexpr uint32_t umma_idesc_f16(int M, int N) {
  return (1u << 4) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}

// What the batch asks of one sequence.
struct TreeSeq {
  int n, row0, L, keys, tiles, units;
};
template <bool PAIR>
__device__ __forceinline__ TreeSeq tree_seq(const TreeParams& P, int s) {
  TreeSeq q;
  q.units = q.tiles = q.n = q.row0 = q.L = q.keys = 0;
  if (s >= P.S) return q;
  q.row0 = __ldg(P.cu_tokens + s);
  q.n = __ldg(P.cu_tokens + s + 1) - q.row0;
  q.L = max(0, __ldg(P.context_lens + s));
  // tokens past the end of the table row are left out like those of a bad page
  q.keys = static_cast<int>(min(static_cast<int64_t>(q.L), static_cast<int64_t>(P.MB) << P.bs_log2));
  q.tiles = static_cast<int>((static_cast<int64_t>(q.keys) + kTreeKeys - 1) / kTreeKeys);
  const int tokens = PAIR ? 2 * P.TQ : P.TQ;
  if (q.row0 >= 0 && q.n > 0 && q.n <= P.max_n && static_cast<int64_t>(q.row0) + q.n <= P.N) q.units = (q.n + tokens - 1) / tokens * P.Hkv;
  return q;
}

// The keys k0 .. k0 + 31 that a row sees, as bits: all before the tree (which begins at `at`, below 0 where the context is
// shorter than the tree), and the tree's own by its mask.
__device__ __forceinline__ uint32_t tree_visible(int k0, int at, int keys, uint64_t mask) {
  const int hist = max(0, min(32, at - k0)), end = max(0, min(32, keys - k0));
  const int i = k0 - at;
  const uint32_t tree = static_cast<uint32_t>(i >= 64 || i <= -32 ? 0ull : i >= 0 ? mask >> i : mask << -i);
  const uint32_t before = hist >= 32 ? 0xffffffffu : (1u << hist) - 1u;
  return (before | tree) & (end >= 32 ? 0xffffffffu : (1u << end) - 1u);
}

// The non-finite elements of V that the guard set to 0, for columns c0 .. c0 + 31 of a row: rare, kept small rather than fast.
template <int D, int EB>
__device__ __noinline__ void tree_add_guarded(const TreeParams& P, const TreeItem& it, uint64_t mask, int c0, float* v) {
  const int at = it.L - it.n;
  const int from = max(it.edge, it.tb) * kTreeKeys, to = min(it.te * kTreeKeys, it.keys);
#pragma unroll 1
  for (int key = from; key < to; ++key) {
    if (!(tree_visible(key & ~31, at, it.keys, mask) >> (key & 31) & 1u)) continue;
    const int id = __ldg(P.block_table + static_cast<int64_t>(it.s) * P.MB + (key >> P.bs_log2));
    if (id < 0 || id >= P.NB) continue;
    const int slot = key & ((1 << P.bs_log2) - 1);
#pragma unroll 1
    for (int i = 0; i < 32; ++i) {
      if constexpr (EB == 2) {
        const uint32_t u = static_cast<const uint16_t*>(P.v_cache)[id * P.sb + it.g * P.sh + slot * P.st + c0 + i];
        if ((u & 0x7f80u) == 0x7f80u) v[i] += __uint_as_float(u << 16);
      } else {
        const uint32_t u = static_cast<const uint8_t*>(P.v_cache)[((static_cast<int64_t>(id) * P.Hkv + it.g) * D + c0 + i) << P.bs_log2 | slot];
        if ((u & 0x7fu) == 0x7fu) v[i] += __uint_as_float(0x7fc00000u);
      }
    }
  }
}

template <int D, bool PAIR, int EB>
__global__ void __launch_bounds__(TR_NTHREADS, 1)
tree_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
            const __grid_constant__ CUtensorMap tmV, const __grid_constant__ TreeParams P) {
  using C = TreeCfg<D, PAIR, EB>;
  constexpr int NK = C::NK, NV = C::NV, NR = C::NR, QT = C::QT, LAG = C::LAG;
  constexpr bool F8 = EB == 1;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t pad = (1024u - (raw & 1023u)) & 1023u;
  uint8_t* smem = smem_raw + pad;
  const uint32_t sQ = raw + pad, sK = sQ + QT * C::TILE_BYTES, sV = sK + NK * C::TILE_BYTES;
  const uint32_t rK = sV + NV * C::TILE_BYTES, rV = rK + NR * C::RAW_BYTES;
  TreeCtrl* ctrl = reinterpret_cast<TreeCtrl*>(smem + C::RING_BYTES);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float NEG_INF = __int_as_float(0xff800000);

  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&ctrl->drained), 1);
    mbar_init(smem_u32(&ctrl->meet), 8);
    mbar_init(smem_u32(&ctrl->meet_widen), 4);
    for (int i = 0; i < 8; ++i) {
      mbar_init(smem_u32(&ctrl->k_full[i]), 1);
      mbar_init(smem_u32(&ctrl->v_full[i]), 1);
      mbar_init(smem_u32(&ctrl->k_ok[i]), 4);
      mbar_init(smem_u32(&ctrl->v_ok[i]), F8 ? 4 : 2);
      mbar_init(smem_u32(&ctrl->step[i]), 1);
    }
    mbar_init(smem_u32(&ctrl->q_full), 1);
    mbar_init(smem_u32(&ctrl->q_ok), 4);
    mbar_init(smem_u32(&ctrl->q_free), 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&ctrl->s_full[t]), 1);
      mbar_init(smem_u32(&ctrl->p_part[t][0]), 4);
      mbar_init(smem_u32(&ctrl->p_part[t][1]), 4);
      mbar_init(smem_u32(&ctrl->o_full[t]), 1);
    }
    for (int i = 0; i < TR_ITEMS; ++i) {
      mbar_init(smem_u32(&ctrl->item_full[i]), 1);
      mbar_init(smem_u32(&ctrl->item_free[i]), 8 + 1 + 2 + (F8 ? 4 : 2));   // softmax, MMA, loads, guards
    }
    ctrl->abort = 0;
    fence_mbar_init();
  }
  if (warp == 8) {
    tmem_alloc(smem_u32(&ctrl->tmem_base), C::TMEM_COLS);
    tmem_relinquish();
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");   // a programmatic dependent of the kernel before it on the stream
  // ---- cost of every 32 sequences (over the rings, which hold nothing yet)
  int64_t* chunk_cost = reinterpret_cast<int64_t*>(smem);
  int64_t* chunk_units = chunk_cost + TR_MAX_SEQS / 32;
  const int chunks = (P.S + 31) / 32;
  for (int c = warp; c < chunks; c += TR_NTHREADS / 32) {
    const TreeSeq q = tree_seq<PAIR>(P, c * 32 + lane);
    int64_t cost = static_cast<int64_t>(q.units) * (q.tiles + kTreeStart), units = q.units;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      cost += __shfl_xor_sync(0xffffffffu, cost, o);
      units += __shfl_xor_sync(0xffffffffu, units, o);
    }
    if (lane == 0) {
      chunk_cost[c] = cost;
      chunk_units[c] = units;
    }
    if (q.n > P.max_n && blockIdx.x == 0) atomicOr(&P.hdr->err, ERR_TOO_LARGE);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = tree_uniform(static_cast<int>(*reinterpret_cast<volatile uint32_t*>(&ctrl->tmem_base)));
  const uint32_t* abort_flag = &ctrl->abort;

  // ---- this CTA's share: from (s0, u0, t0) to (s1, u1, t1); warp 9 walks it
  int s0 = 0, u0 = 0, t0 = 0, s1 = 0, u1 = 0, t1 = 0;
  if (warp == 9) {
    int64_t total = 0, all_units = 0;
    for (int c = lane; c < chunks; c += 32) {
      total += chunk_cost[c];
      all_units += chunk_units[c];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      total += __shfl_xor_sync(0xffffffffu, total, o);
      all_units += __shfl_xor_sync(0xffffffffu, all_units, o);
    }
    auto locate = [&](int64_t x, int& s, int& u, int& t) {
      s = P.S;
      u = t = 0;
      if (x >= total) return;
      int64_t before = 0;
      int chunk = 0;
      for (int base = 0; base < chunks; base += 32) {      // the chunk that holds x
        const int64_t own = base + lane < chunks ? chunk_cost[base + lane] : 0;
        int64_t incl = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int64_t y = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += y;
        }
        const uint32_t m = __ballot_sync(0xffffffffu, before + incl > x);
        if (m) {
          const int l = __ffs(m) - 1;
          chunk = base + l;
          before += __shfl_sync(0xffffffffu, incl - own, l);
          break;
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
      }
      const TreeSeq q = tree_seq<PAIR>(P, chunk * 32 + lane);
      const int64_t own = static_cast<int64_t>(q.units) * (q.tiles + kTreeStart);
      int64_t incl = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
      }
      const uint32_t m = __ballot_sync(0xffffffffu, before + incl > x);
      const int l = m ? __ffs(m) - 1 : 31;
      s = chunk * 32 + l;
      tree_cut(x - before - __shfl_sync(0xffffffffu, incl - own, l), __shfl_sync(0xffffffffu, q.tiles, l), &u, &t);
      if (u >= __shfl_sync(0xffffffffu, q.units, l)) {      // (a cut that moved to the end of the sequence's last unit)
        ++s;
        u = 0;
      }
    };
    const int shares = tree_shares(total, all_units, gridDim.x), me = blockIdx.x;
    locate(me < shares ? total * me / shares : total, s0, u0, t0);
    locate(me < shares ? total * (me + 1) / shares : total, s1, u1, t1);
  }
  fence_proxy_async();                                      // (the sums were written before the copies that overwrite them)
  __syncthreads();                                          // the sums have been read: the rings may be filled

  auto fail = [&]() {
    atomicOr(&P.hdr->err, ERR_TIMEOUT);
    atomicExch(&ctrl->abort, 1u);
  };
  // warp-uniform bounded wait
  auto wait = [&](uint64_t* bar, uint32_t parity) -> bool {
    return __all_sync(0xffffffffu, tree_wait(smem_u32(bar), parity & 1, abort_flag));
  };
  // the k-th item of this CTA (false: no more, or a wait ran out); uniform over the warp
  auto get_item = [&](int k, const TreeItem*& it) -> bool {
    if (!wait(&ctrl->item_full[k % TR_ITEMS], k / TR_ITEMS)) {
      if (lane == 0) fail();
      return false;
    }
    it = &ctrl->item[k % TR_ITEMS];
    return it->s >= 0;
  };
  auto done_item = [&](int k) {      // the warp reads nothing of the k-th item any more
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&ctrl->item_free[k % TR_ITEMS]));
  };

  // The softmax threads hold many scores each; they take the registers that the others leave.
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TR_OTHER_REGS));
    if (warp == 9) {
      // ================= items, and Q of the one before: its buffer is free only when the item before that has all its scores
      int4 rec[2] = {make_int4(-1, 0, 0, 0), make_int4(-1, 0, 0, 0)};
      int base = s0 & ~31;
      TreeSeq win = tree_seq<PAIR>(P, base + lane);
      int s = s0, u = u0, t = t0;
      bool ok = true, more = true, ran_out = false;
      int pend_k = -1, pend_g = 0, pend_row = 0;           // item whose Q is to be loaded
      int nq = 0;
      for (int k = 0; ok && more; ++k) {                   // (the last round publishes that there are no more)
        {
          TreeItem it;
          it.s = -1;
          while (s < P.S && (s < s1 || (s == s1 && (u < u1 || (u == u1 && t < t1))))) {
            if (s >= base + 32) {
              base = s & ~31;
              win = tree_seq<PAIR>(P, base + lane);
            }
            const int l = s - base, units = __shfl_sync(0xffffffffu, win.units, l), tiles = __shfl_sync(0xffffffffu, win.tiles, l);
            if (u >= units) {
              ++s;
              u = t = 0;
              continue;
            }
            const int n = __shfl_sync(0xffffffffu, win.n, l);
            const int per_head = units / P.Hkv, pair = u % per_head;
            it.s = s;
            it.g = u / per_head;
            it.tok0 = PAIR ? pair * 2 * P.TQ : 0;
            it.n = n;
            it.row0 = __shfl_sync(0xffffffffu, win.row0, l);
            it.L = __shfl_sync(0xffffffffu, win.L, l);
            it.keys = __shfl_sync(0xffffffffu, win.keys, l);
            if (it.keys < it.L) ran_out = true;
            it.tb = t;
            it.te = s == s1 && u == u1 ? t1 : tiles;
            it.edge = min(max(0, it.L - n), it.keys) / kTreeKeys;
            it.part = -1;
            if (it.te - it.tb < tiles) {
              const int which = it.tb > 0 ? 0 : 1;
              it.part = 2 * blockIdx.x + which;
              rec[which] = make_int4(s, it.g, pair, it.te == tiles ? 1 : 0);
            }
            it.rows[0] = min(P.TQ, n - it.tok0);
            it.rows[1] = PAIR ? min(P.TQ, max(0, n - it.tok0 - P.TQ)) : it.rows[0];
            if (it.te == tiles) {
              ++u;
              t = 0;
            } else {
              t = it.te;
            }
            break;
          }
          more = it.s >= 0;
          ok = wait(&ctrl->item_free[k % TR_ITEMS], (k / TR_ITEMS) ^ 1);
          if (!ok) break;
          if (lane == 0) {
            ctrl->item[k % TR_ITEMS] = it;
            ctrl->odd[k % TR_ITEMS] = 0u;
            mbar_arrive(smem_u32(&ctrl->item_full[k % TR_ITEMS]));     // (release: the item is visible to whoever sees the phase)
          }
          __syncwarp();
          const int now_k = more && it.te > it.tb ? k : -1, now_g = it.g, now_row = it.row0 + it.tok0;
          // Q of the item before
          if (pend_k >= 0) {
            ok = wait(&ctrl->q_free, nq ^ 1);
            if (ok && lane == 0) {
              const uint32_t bar = smem_u32(&ctrl->q_full);
              mbar_arrive_expect_tx(bar, static_cast<uint32_t>(QT * C::HALVES * P.TQ * P.G * 128));
#pragma unroll
              for (int i = 0; i < QT; ++i)
#pragma unroll
                for (int hh = 0; hh < C::HALVES; ++hh)
                  tma_load_4d(sQ + i * C::TILE_BYTES + hh * C::HALF_BYTES, &tmQ, hh * 64, 0, pend_g, pend_row + i * P.TQ, bar);
            }
            __syncwarp();
            if (ok) ++nq;
          }
          pend_k = now_k;
          pend_g = now_g;
          pend_row = now_row;
        }
      }
      if (lane == 0) {
        P.rec[2 * blockIdx.x] = rec[0];
        P.rec[2 * blockIdx.x + 1] = rec[1];
        if (ran_out) atomicOr(&P.hdr->err, ERR_BAD_PAGE);
        if (!ok) fail();
      }
      // given up: no copy may still be on its way into this CTA's shared memory when it ends
      if (*reinterpret_cast<const volatile uint32_t*>(abort_flag) && nq > 0) mbar_wait(smem_u32(&ctrl->q_full), (nq - 1) & 1);
    } else if (warp == 10 || warp == 11) {
      // ================= loads: K (warp 10), V (warp 11)
      const bool isV = warp == 11;
      const int ppt = kTreeKeys >> P.bs_log2;              // pages of a key tile
      const int j = lane & (ppt - 1), h = lane / ppt;
      const int ring = F8 ? NR : isV ? NV : NK;
      const CUtensorMap* tm = isV ? &tmV : &tmK;
      const uint32_t dst0 = F8 ? (isV ? rV : rK) + (j << P.bs_log2) * D
                               : (isV ? sV : sK) + h * C::HALF_BYTES + (j << P.bs_log2) * 128;
      const int slot_bytes = F8 ? C::RAW_BYTES : C::TILE_BYTES;
      uint64_t* full = isV ? ctrl->v_full : ctrl->k_full;
      bool any_bad = false, ok = true;
      int c = 0, slot = 0;
      const TreeItem* ip;
      for (int k = 0; ok && get_item(k, ip); ++k) {
        const TreeItem& it = *ip;
        const int32_t* row = P.block_table + static_cast<int64_t>(it.s) * P.MB;
        const int npages = static_cast<int>((static_cast<int64_t>(it.keys) + (1 << P.bs_log2) - 1) >> P.bs_log2);
        auto page_id = [&](int kt) {
          const int i = kt * ppt + j;
          return i < npages ? __ldg(row + i) : -2;          // -2: past the end, filled with zeros
        };
        const int te = it.te, g = it.g;
        int id_next = it.tb < te ? page_id(it.tb) : 0;
        for (int kt = it.tb; kt < te; ++kt) {
          int id = id_next;
          if (kt + 1 < te) id_next = page_id(kt + 1);
          const bool bad = id != -2 && (id < 0 || id >= P.NB);
          const uint32_t badmask = __ballot_sync(0xffffffffu, bad && h == 0);
          any_bad |= badmask != 0;
          if (id < 0 || id >= P.NB) id = P.NB;              // out-of-bounds coordinate: TMA fills zeros, nothing is read
          // the slot's previous tile: codes are free when they have been widened; K(c - NK) with step c - NK, V(c - NV) with
          // step c - NV + LAG
          if (c >= ring) {
            if (F8) ok = wait(isV ? &ctrl->v_ok[(c - ring) & 7] : &ctrl->k_ok[(c - ring) & 7], (c - ring) >> 3);
            else ok = wait(&ctrl->step[(isV ? c - NV + LAG : c - NK) & 7], (isV ? c - NV + LAG : c - NK) >> 3);
            if (!ok) break;
          }
          const uint32_t bar = smem_u32(&full[c & 7]);
          if (lane == 0) {
            if (!isV) ctrl->page_bad[c & 7] = badmask;
            mbar_arrive_expect_tx(bar, static_cast<uint32_t>(slot_bytes));
          }
          __syncwarp();
          if constexpr (F8) {
            if (h == 0) tma_load_4d(dst0 + slot * C::RAW_BYTES, tm, 0, 0, g, id, bar);
          } else {
            if (h < C::HALVES) tma_load_4d(dst0 + slot * C::TILE_BYTES, tm, h * 64, 0, g, id, bar);
          }
          if (++slot == ring) slot = 0;
          ++c;
        }
        done_item(k);
      }
      if (lane == 0) {
        if (any_bad) atomicOr(&P.hdr->err, ERR_BAD_PAGE);
        if (!ok) fail();
      }
      // given up: see above
      if (*reinterpret_cast<const volatile uint32_t*>(abort_flag))
        for (int i = max(0, c - ring); i < c; ++i) mbar_wait(smem_u32(&full[i & 7]), (i >> 3) & 1);
    } else if (warp == 8) {
      // ================= MMA issue: the warp runs the loop as one, one elected lane issues
      uint32_t elected;
      asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(elected));
      const TreeItem* ip;
      int c = 0, kslot = 0, vslot = 0;   // key tiles of this CTA so far; ring slots of K(c) and of the next V
      uint32_t nq = 0, np = 0;           // parity of q; bit t: parity of p_part of group t
      int nv = 0;                        // products so far
      bool ok = true;
      constexpr uint32_t ID_S = F8 ? umma_idesc_f16(128, kTreeKeys) : umma_idesc(128, kTreeKeys, 0, 0);   // Q x K tile, both K-major
      constexpr uint32_t ID_O = F8 ? umma_idesc_f16(128, D) : umma_idesc(128, D, 0, 1);   // P (tensor memory) x V (MN-major; fp8: K-major)
      const uint64_t q_desc = umma_desc(sQ, 16, 1024), k_desc = umma_desc(sK, 16, 1024);
      const uint64_t v_desc = F8 ? umma_desc(sV, 16, 1024) : umma_desc(sV, C::HALF_BYTES, 1024);
      for (int k = 0; ok && get_item(k, ip); ++k) {
        const int n = tree_uniform(ip->te - ip->tb);
        const uint32_t active = PAIR ? 1u | (tree_uniform(ip->rows[1]) > 0 ? 2u : 0u) : 3u;
        done_item(k);
        if (n <= 0) continue;
        for (int j = 0; j < n + LAG && ok; ++j) {
          const uint32_t turn = PAIR ? active : 1u << (j & 1);        // groups that key tiles j and j - LAG belong to
          if (j >= LAG) ok = wait(&ctrl->v_ok[nv & 7], nv >> 3);
          if (ok && j < n) ok = wait(F8 ? &ctrl->k_ok[c & 7] : &ctrl->k_full[c & 7], c >> 3);
          if (ok && j == 0) {
            ok = wait(F8 ? &ctrl->q_ok : &ctrl->q_full, nq);
            nq ^= 1;
          }
#pragma unroll 1
          for (int t = 0; t < 2 && ok; ++t) {
            if (!((turn >> t) & 1)) continue;
            const uint32_t tS = tbase + C::COL_S + t * 128, tO = tbase + C::COL_O + t * D;
            if (j >= LAG) {
              // O_t (+)= P_t . V of key tile j - LAG; the first half runs while the second is still being made
              uint64_t vd = v_desc + static_cast<uint64_t>(tree_uniform(vslot) * (C::TILE_BYTES >> 4));
              uint32_t accum = j >= 2 * LAG ? 1u : 0u, a = tS;
#pragma unroll 1
              for (int h = 0; h < 2; ++h) {
                ok = wait(&ctrl->p_part[t][h], np >> t);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  umma_ts_elected(tO, a, vd + (F8 ? i * 2 : i * (2048 >> 4)), ID_O, accum, elected);
                  accum = 1u;
                  a += 8;
                }
                vd += F8 ? (D * 128) >> 4 : 4 * (2048 >> 4);
              }
              if (!ok) break;
              np ^= 1u << t;
              if (j >= n) tc_commit_elected(smem_u32(&ctrl->o_full[t]), elected);   // that was this group's last
            }
            if (j < n) {
              tc_fence_after();
              uint64_t kd = k_desc + static_cast<uint64_t>(tree_uniform(kslot) * (C::TILE_BYTES >> 4));
              uint64_t qd = q_desc + static_cast<uint64_t>(PAIR ? t * (C::TILE_BYTES >> 4) : 0);
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
            }
          }
          if (!ok) break;
          if (j >= LAG) {
            ++nv;
            if (++vslot == NV) vslot = 0;
          }
          if (j < n) {
            if (j == n - 1) tc_commit_elected(smem_u32(&ctrl->q_free), elected);
            // the scores of c and the product of c - LAG (an earlier item's last ones included)
            tc_commit_elected(smem_u32(&ctrl->step[c & 7]), elected);
            ++c;
            if (++kslot == NK) kslot = 0;
          }
        }
      }
      if (lane == 0 && !ok) fail();
      // nothing that was issued may still be running on the tensor cores when the tensor memory goes back
      tc_commit_elected(smem_u32(&ctrl->drained), elected);
      mbar_wait(smem_u32(&ctrl->drained), 0);
      __syncwarp();
    } else if (F8) {
      // ================= widening, warps 12-15: a thread moves 16 codes at a time.  K of the next key tile comes before V of this one.
      const int w = warp - 12, id = w * 32 + lane;
      const TreeItem* ip;
      int c = 0, nq = 0;
      int rk = 0, rv = 0, ok_ = 0, ov = 0;                 // ring slots: codes of K, of V; K, V
      int nv = 0, meets = 0;
      bool ok = true;
      auto widen = [&](uint32_t src, uint32_t d0, uint32_t d1) {     // 16 codes to two 16-byte chunks; returns whether one is NaN
        uint32_t x[4];
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(src) : "memory");
        uint32_t y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = cvt_e4m3x2_f16x2(x[i >> 1] >> (16 * (i & 1)));
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(d0), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(d1), "r"(y[4]), "r"(y[5]), "r"(y[6]), "r"(y[7]) : "memory");
      };
      auto publish = [&](uint64_t* bar) {
        fence_proxy_async();                               // the stores above before the tensor cores' reads
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(bar));
      };
      auto do_v = [&](int edge_tile, int v) {
        // V(v): codes [page][d][slot], linear; tile [64-key block][d][64 keys]
        ok = ok && wait(&ctrl->v_full[v & 7], v >> 3);
        if (ok && v >= NV) ok = wait(&ctrl->step[(v - NV + LAG) & 7], (v - NV + LAG) >> 3);
        if (!ok) return;
        const uint32_t src = rV + rv * C::RAW_BYTES, dst = sV + ov * C::TILE_BYTES;
        if (edge_tile) {
          // the guard: which keys hold a NaN code
          // warp w looks at keys 32 w .. + 31, all of d
          uint32_t bad = 0u;
#pragma unroll 1
          for (int i = lane; i < 2 * D; i += 32) {         // 16 keys of one d
            const int key = w * 32 + (i / D) * 16, dd = i % D;
            const int page = key >> P.bs_log2, in = key & ((1 << P.bs_log2) - 1);
            uint32_t x[4];
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                         : "r"(src + ((page * D + dd) << P.bs_log2) + in) : "memory");
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              // a byte is NaN when its low seven bits are all set: adding one carries into the eighth
              const uint32_t hit = ((x[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
              if (hit) {
#pragma unroll
                for (int b = 0; b < 4; ++b)
                  if (hit >> (8 * b + 7) & 1u) bad |= 1u << ((i / D) * 16 + e * 4 + b);
                x[e] &= ~((hit >> 7) * 0xffu);
              }
            }
            // (written back: the widening below reads it, by other warps too)
            if (bad)
              asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(src + ((page * D + dd) << P.bs_log2) + in), "r"(x[0]), "r"(x[1]),
                           "r"(x[2]), "r"(x[3]) : "memory");
          }
          bad = __reduce_or_sync(0xffffffffu, bad);
          if (lane == 0) ctrl->v_bad[v & 7][w] = bad;
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&ctrl->meet_widen));
          ok = wait(&ctrl->meet_widen, meets++);           // (bounded, unlike a named barrier)
          if (!ok) return;
        }
#pragma unroll 4
        for (int i = id; i < D * 8; i += 128) {            // chunk i of 16 codes, as they lie
          const int page = (i << 4) / (D << P.bs_log2), in_page = (i << 4) - page * (D << P.bs_log2);
          const int dd = in_page >> P.bs_log2, key = (page << P.bs_log2) + (in_page & ((1 << P.bs_log2) - 1));
          const uint32_t row = dst + (key >> 6) * (D * 128) + dd * 128;
          const int ch = (key & 63) >> 3;
          widen(src + (i << 4), row + ((ch ^ (dd & 7)) << 4), row + (((ch + 1) ^ (dd & 7)) << 4));
        }
        publish(&ctrl->v_ok[v & 7]);
        if (++rv == NR) rv = 0;
        if (++ov == NV) ov = 0;
      };
      for (int k = 0; ok && get_item(k, ip); ++k) {
        const TreeItem& it = *ip;
        const int tb = it.tb, te = it.te, edge = it.edge;
        for (int kt = tb; kt < te && ok; ++kt) {
          // K(c): codes [key][d], rows swizzled by the copy; tile [64-element block][key][64]
          ok = wait(&ctrl->k_full[c & 7], c >> 3);
          if (ok && c >= NK) ok = wait(&ctrl->step[(c - NK) & 7], (c - NK) >> 3);
          if (!ok) break;
          {
            const uint32_t src = rK + rk * C::RAW_BYTES + id * D, dst = sK + ok_ * C::TILE_BYTES + id * 128;   // key `id`
#pragma unroll 4
            for (int i = 0; i < D / 16; ++i) {
              const int from = D == 128 ? i ^ (id & 7) : i ^ ((id >> 1) & 3);
              const uint32_t row = dst + (i >> 2) * C::HALF_BYTES;
              const int ch = (i & 3) * 2;
              widen(src + (from << 4), row + ((ch ^ (id & 7)) << 4), row + (((ch + 1) ^ (id & 7)) << 4));
            }
          }
          publish(&ctrl->k_ok[c & 7]);
          if (++rk == NR) rk = 0;
          if (++ok_ == NK) ok_ = 0;
          if (kt == tb) {
            // Q in place, bf16 to fp16
            ok = wait(&ctrl->q_full, nq);
            nq ^= 1;
            if (!ok) break;
#pragma unroll 1
            for (int i = id; i < QT * C::TILE_BYTES / 16; i += 128) {
              uint32_t x[4];
              asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(sQ + i * 16) : "memory");
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = pack_f16x2(__uint_as_float(x[e] << 16), __uint_as_float(x[e] & 0xffff0000u));
              asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(sQ + i * 16), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
            }
            publish(&ctrl->q_ok);
          } else {
            do_v(kt - 1 >= edge, nv++);
          }
          ++c;
        }
        if (te > tb && ok) do_v(te - 1 >= edge, nv++);
        done_item(k);
      }
      if (!ok && lane == 0) fail();
    } else if (warp >= 14) {
      // ================= guards of V: each takes its share of every 64 keys
      const int w = warp - 14;
      const TreeItem* ip;
      int c = 0, slot = 0;
      bool ok = true;
      for (int k = 0; ok && get_item(k, ip); ++k) {
        const TreeItem& it = *ip;
        const int te = it.te, edge = it.edge;
        for (int kt = it.tb; kt < te; ++kt) {
          ok = wait(&ctrl->v_full[c & 7], c >> 3);
          if (!ok) break;
          if (kt >= edge) {
            const uint32_t base = sV + slot * C::TILE_BYTES;
#pragma unroll 1
            for (int e = 0; e < 2; ++e) {
              // 32 keys: a key's row of a 64-column block is 128 bytes = 8 chunks, four keys per warp-wide load.  A bf16 is not
              // finite when its eight exponent bits are all set: adding one to them then carries into the sign's place.
              const uint32_t rows = base + (w * 2 + e) * 32 * 128;
              uint32_t bad = 0u;
#pragma unroll 1
              for (int hq = 0; hq < C::HALVES * 8; ++hq) {
                const int hh = hq >> 3, q = hq & 7;
                const uint32_t at = rows + hh * C::HALF_BYTES + (q * 32 + lane) * 16;
                uint32_t v[4], hit = 0u;
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at) : "memory");
#pragma unroll
                for (int i = 0; i < 4; ++i) hit |= (v[i] & 0x7f807f80u) + 0x00800080u;
                if (hit & 0x80008000u) {
#pragma unroll
                  for (int i = 0; i < 4; ++i) {
                    if ((v[i] & 0x7f80u) == 0x7f80u) v[i] &= 0xffff0000u;
                    if ((v[i] & 0x7f800000u) == 0x7f800000u) v[i] &= 0x0000ffffu;
                  }
                  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
                  bad |= 1u << (q * 4 + (lane >> 3));
                }
              }
              bad = __reduce_or_sync(0xffffffffu, bad);
              if (lane == 0) ctrl->v_bad[c & 7][w * 2 + e] = bad;
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
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(TR_SOFTMAX_REGS));
    // ================= softmax: a thread owns row r; group t has row tile t (PAIR) or every second key tile
    const int t = warp >> 2;
    const int r = threadIdx.x & 127;
    const uint32_t lane_addr = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tbase + C::COL_S + t * 128 + lane_addr, tO = tbase + C::COL_O + t * D + lane_addr;
    const int rj = r / P.G, rh = r - rj * P.G;          // token in the tile, head in the KV group
    // warp-uniform: tensor-memory accesses need the whole warp.  No thread leaves this path early: after a failed wait it
    // carries on, and its further waits return at once.
    auto wait_all = [&](uint64_t* bar, uint32_t parity) {
      if (!wait(bar, parity) && lane == 0) fail();
    };
    int meets = 0;
    auto meet = [&]() {                // all eight warps (bounded, unlike a named barrier)
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ctrl->meet));
      wait_all(&ctrl->meet, meets++);
    };
    const TreeItem* ip;
    int c0 = 0, nt = 0, no = 0;        // key tiles of the CTA before this item; of this group; items of this group that had keys
    for (int k = 0; get_item(k, ip); ++k) {
      const TreeItem& it = *ip;
      const int tb = it.tb, te = it.te, edge = it.edge, rows = it.rows[t], keys = it.keys;
      const int at = it.L - it.n;                       // where the tree begins
      const int j = it.tok0 + (PAIR ? t * P.TQ : 0) + rj;   // token within the tree
      const bool valid = rj < rows;
      const bool sees = valid && at + j >= 0;           // a token before position 0 sees nothing
      const bool mine = PAIR ? rows > 0 : true;
      const bool busy = __any_sync(0xffffffffu, valid); // some row of this warp belongs to a token
      uint64_t mask = 0ull;
      if (sees) mask = __ldg(P.mask + it.row0 + j) & (it.n >= 64 ? ~0ull : (1ull << it.n) - 1ull);
      // scores to base-2 units; the maximum is taken of raw scores, so a negative factor flips their signs first
      float sc = P.scale_log2 * (F8 ? __ldg(P.k_scale + it.g) : 1.f);
      const bool flip = sc < 0.f;
      sc = fabsf(sc);
      if (sc == 0.f) sc = 1.1754944e-38f;               // (all weights alike; 0 * inf would be NaN)
      float m = NEG_INF, l = 0.f;
      bool odd = false;                                 // this row sees a key with a non-finite V
      for (int kt = PAIR ? tb : tb + t; mine && kt < te; kt += PAIR ? 1 : 2) {
        const int c = c0 + (kt - tb);
        wait_all(&ctrl->s_full[t], nt);
        tc_fence_after();
        const bool first = kt == (PAIR ? tb : tb + t);
        ++nt;
        if (!busy) {
          if (lane < 2) mbar_arrive(smem_u32(&ctrl->p_part[t][lane]));
          continue;
        }
        // Two passes over the scores, 32 columns at a time, so that the loops stay small; the next columns are on their way while
        // these are worked on.  The first pass takes the maximum, and where scores are masked it writes them back; the second makes
        // the weights, whose columns 16 q .. + 15 lie over scores that have been read.
        uint32_t x0[32], x1[32];
        auto first_pass = [&](auto masked_) {
          constexpr bool MASKED = decltype(masked_)::value;
          const uint32_t pb = MASKED ? ctrl->page_bad[c & 7] : 0u;
          float m4[4] = {NEG_INF, NEG_INF, NEG_INF, NEG_INF};
          auto columns = [&](uint32_t (&x)[32], int q) {
            if (MASKED) {
              const int k0 = kt * kTreeKeys + q * 32;
              uint32_t vis = sees ? tree_visible(k0, at, keys, mask) : 0u;
              if (pb) {
                if (P.bs_log2 == 4) vis &= ~(((pb >> (2 * q)) & 1u ? 0xffffu : 0u) | ((pb >> (2 * q + 1)) & 1u ? 0xffff0000u : 0u));
                else if ((pb >> (q >> (P.bs_log2 - 5))) & 1u) vis = 0u;
              }
              if (flip) {
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] ^= 0x80000000u;
              }
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!((vis >> i) & 1u)) x[i] = __float_as_uint(NEG_INF);
              tmem_st32(tS + q * 32, x);
            }
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
          if (MASKED) tc_wait_st();
          return fmaxf(max3(m4[0], m4[1], m4[2]), m4[3]);
        };
        const bool masked = kt >= edge || flip || ctrl->page_bad[c & 7] != 0;
        float mx = masked ? first_pass(std::true_type{}) : first_pass(std::false_type{});
        tmem_ld32(tS, x0);                              // (for the second pass)
        mx = mx == NEG_INF ? NEG_INF : mx * sc;
        const bool grow = first || mx > m + 8.f;
        const float m_new = grow ? fmaxf(m, mx) : m;
        const float mu = m_new == NEG_INF ? 0.f : m_new;
        const float alpha = grow ? fast_exp2(m - mu) : 1.f;
        m = m_new;
        if (__any_sync(0xffffffffu, valid && !first && alpha != 1.f)) {
          // new reference: scale this row of O.  PAIR: the product before this one was done when the scores came; split: so it
          // was, the scores of this tile were issued behind it.
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
        const uint64_t sc2 = tree_pack2(sc, sc), mu2 = tree_pack2(-mu, -mu);
        auto weights = [&](const uint32_t (&x)[32], int q) {
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float p0, p1;
            tree_unpack2(tree_fma2(tree_pack2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), sc2, mu2), p0, p1);
            p0 = fast_exp2(p0);
            p1 = fast_exp2(p1);
            const uint64_t pp = tree_pack2(p0, p1);
            if (i & 1) sum1 = tree_add2(sum1, pp);
            else sum0 = tree_add2(sum0, pp);
            pk[i] = F8 ? pack_f16x2(p0, p1) : pack_bf16x2(p0, p1);
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
          if (q == 2 && kt >= edge) {
            // before the last weights go, for they let the guard's word be written anew: does this row see a guarded key?
            wait_all(&ctrl->v_ok[c & 7], c >> 3);
            if (sees) {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                odd |= (*reinterpret_cast<volatile uint32_t*>(&ctrl->v_bad[c & 7][e]) &
                        tree_visible(kt * kTreeKeys + 32 * e, at, keys, mask)) != 0u;
            }
          }
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&ctrl->p_part[t][q >> 1]));
        }
        {
          float a0, a1, b0, b1;
          tree_unpack2(sum0, a0, a1);
          tree_unpack2(sum1, b0, b1);
          l = l * alpha + ((a0 + a1) + (b0 + b1));
        }
      }
      c0 += te - tb;
      // ---- the item's rows
      const bool any = mine && (PAIR ? te > tb : te > tb + t);   // this group had key tiles
      const float vs = F8 ? __ldg(P.v_scale + it.g) : 1.f;
      if (any) {
        wait_all(&ctrl->o_full[t], no);
        ++no;
        tc_fence_after();
      }
      float f[2] = {0.f, 0.f};                          // factors of O_0 and O_1 in this row's output
      bool have[2];
      const bool whole = it.part < 0;
      if (PAIR) {
        have[0] = any && t == 0;
        have[1] = any && t == 1;
        f[t] = whole ? (l > 0.f ? 1.f / l : (l != l ? l : 0.f)) : 1.f;
      } else {
        have[0] = te > tb;
        have[1] = te > tb + 1;
        if (odd) atomicOr(&ctrl->odd[k % TR_ITEMS], 1u);
        if (t == 1) ctrl->ml[r] = make_float2(m, l);
        meet();
        odd = *reinterpret_cast<volatile uint32_t*>(&ctrl->odd[k % TR_ITEMS]) != 0u;
        if (whole) {
          if (t == 0) {
            const float2 other = ctrl->ml[r];
            const float M = fmaxf(m, other.x);
            f[0] = m == NEG_INF ? 0.f : fast_exp2(m - M);
            f[1] = other.x == NEG_INF ? 0.f : fast_exp2(other.x - M);
            const float sum = l * f[0] + other.y * f[1];
            const float inv = sum > 0.f ? 1.f / sum : (sum != sum ? sum : 0.f);
            f[0] *= inv;
            f[1] *= inv;
            ctrl->ml[r] = make_float2(f[0], f[1]);
          }
          meet();
          if (t == 1) {
            const float2 both = ctrl->ml[r];
            f[0] = both.x;
            f[1] = both.y;
          }
          tc_fence_after();                             // (the other group's O: its product was seen to be done before the barrier)
        } else {
          f[t] = 1.f;
          have[t ^ 1] = false;
        }
      }
      f[0] *= vs;
      f[1] *= vs;
      if (mine && busy) {
        // a part of a unit leaves its sums as they are
        float* part = whole ? nullptr : P.partials + (static_cast<int64_t>(it.part) * 2 + t) * ((D + 2) * 128) + r;
        if (part && valid) {
          part[D * 128] = m;
          part[(D + 1) * 128] = l;
        }
        __nv_bfloat16* out0 = P.out + (static_cast<int64_t>(it.row0 + it.tok0 + (PAIR ? t * P.TQ : 0)) * P.Hq + it.g * P.G) * D;
        const int offset = valid ? (rj * P.Hq + rh) * D : -1;     // of this thread's row
        const int q0 = PAIR || part ? 0 : t * (D / 64), q1 = PAIR || part ? D / 32 : q0 + D / 64;
#pragma unroll 1
        for (int q = q0; q < q1; ++q) {
          float v[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = 0.f;
#pragma unroll
          for (int tt = 0; tt < 2; ++tt) {
            if (!have[tt]) continue;                    // (uniform over the warp)
            uint32_t o[32];
            tmem_ld32(tbase + C::COL_O + tt * D + lane_addr + q * 32, o);
            tc_wait_ld();
            // (a factor of 0: the row saw nothing in those tiles, and what O holds may be anything)
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = f[tt] != 0.f ? fmaf(__uint_as_float(o[i]), f[tt], v[i]) : v[i];
          }
          if (odd && sees && (PAIR || !part || t == 0)) {
            float add[32];                              // (a copy: v stays in registers)
#pragma unroll
            for (int i = 0; i < 32; ++i) add[i] = v[i];
            tree_add_guarded<D, EB>(P, it, mask, q * 32, add);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = add[i];
          }
          if (part) {
            if (valid) {
#pragma unroll
              for (int i = 0; i < 32; ++i) part[(q * 32 + i) * 128] = v[i];
            }
            continue;
          }
          // A thread holds a row; written like that, every store of a warp would touch 32 lines.  Groups of four lanes transpose
          // 4 x 4 chunks of 16 bytes among themselves, so that a store writes 64 bytes of each of eight rows.
          uint4 w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            w[i] = make_uint4(pack_bf16x2(v[8 * i], v[8 * i + 1]), pack_bf16x2(v[8 * i + 2], v[8 * i + 3]),
                              pack_bf16x2(v[8 * i + 4], v[8 * i + 5]), pack_bf16x2(v[8 * i + 6], v[8 * i + 7]));
          __syncwarp();
          auto swap = [&](uint4& a, uint4& b, int mask_) {         // lanes with the bit hand out a and keep b, the others the other way round
            const bool up = lane & mask_;
            const uint4 give = up ? a : b;
            const uint4 got = make_uint4(__shfl_xor_sync(0xffffffffu, give.x, mask_), __shfl_xor_sync(0xffffffffu, give.y, mask_),
                                         __shfl_xor_sync(0xffffffffu, give.z, mask_), __shfl_xor_sync(0xffffffffu, give.w, mask_));
            if (up) a = got;
            else b = got;
          };
          swap(w[0], w[1], 1);
          swap(w[2], w[3], 1);
          swap(w[0], w[2], 2);
          swap(w[1], w[3], 2);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int at_ = __shfl_sync(0xffffffffu, offset, (lane & ~3) + i);
            if (at_ >= 0) *reinterpret_cast<uint4*>(out0 + at_ + q * 32 + (lane & 3) * 8) = w[i];
          }
        }
        tc_fence_before();
      }
      // split: neither group may hand weights of the next item over while the other still reads O
      if (!PAIR) meet();
      done_item(k);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 8) tmem_dealloc(tbase, C::TMEM_COLS);
}

// The pieces of the units that shares' ends cut, put together in order: block (share in which the unit begins, row tile, 8 columns),
// a thread per row.     M = max m_j;  out = sum O_j 2^(m_j - M) / sum l_j 2^(m_j - M)
// Bound by the latency of its loads (neighbouring rows are neighbours in memory): four pieces are fetched at a time.
template <int D, bool PAIR>
__global__ void __launch_bounds__(128)
tree_join_kernel(const __grid_constant__ TreeParams P, int ctas) {
  __shared__ int list[2 * TR_CTAS], last[4], count[4];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int c = blockIdx.x, t = blockIdx.y, q = blockIdx.z, r = threadIdx.x, warp = r >> 5, lane = r & 31;
  const int4 head = P.rec[2 * c + 1];
  if (head.x < 0) return;
  // the unit's other pieces: first pieces of the shares that follow, up to the one that ends the unit (shares may be empty)
  int n = 1;
  if (r == 0) list[0] = 2 * c + 1;
  for (int base = c + 1; base < ctas; base += 128) {
    const int cc = base + r;
    const int4 x = cc < ctas ? P.rec[2 * cc] : make_int4(-1, 0, 0, 0);
    const bool own = x.x == head.x && x.y == head.y && x.z == head.z;
    const uint32_t ends = __ballot_sync(0xffffffffu, own && x.w == 1), owns = __ballot_sync(0xffffffffu, own);
    const uint32_t upto = ends ? (ends & (0u - ends)) * 2u - 1u : 0xffffffffu;      // lanes up to the one that ends the unit
    if (lane == 0) {
      last[warp] = ends != 0u;
      count[warp] = __popc(owns & upto);
    }
    __syncthreads();
    int before = n;
    bool over = false;
    for (int w = 0; w < warp; ++w) {
      over |= last[w] != 0;
      before += count[w];
    }
    if (!over && own && (upto >> lane & 1u)) list[before + __popc(owns & upto & ((1u << lane) - 1u))] = 2 * cc;
    bool ended = false;
    for (int w = 0; w < 4 && !ended; ++w) {
      n += count[w];
      ended = last[w] != 0;
    }
    __syncthreads();
    if (ended) break;
  }
  __syncthreads();
  const int row0 = __ldg(P.cu_tokens + head.x), tree = __ldg(P.cu_tokens + head.x + 1) - row0;
  const int rj = r / P.G, rh = r - rj * P.G;
  const int j = (PAIR ? (2 * head.z + t) * P.TQ : 0) + rj;
  if (rj >= P.TQ || j >= tree) return;
  // PAIR: a piece has one part per row tile; split: both groups' parts belong to the one row tile
  const int parts = PAIR ? n : 2 * n;
  constexpr int64_t TILE_FLOATS = (D + 2) * 128;
  auto part = [&](int p) {
    const int slot = PAIR ? list[p] : list[p >> 1];
    return P.partials + (static_cast<int64_t>(slot) * 2 + (PAIR ? t : p & 1)) * TILE_FLOATS + r;
  };
  const float NEG_INF = __int_as_float(0xff800000);
  float M = NEG_INF, L = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int p = 0; p < parts; ++p) M = fmaxf(M, part(p)[D * 128]);
#pragma unroll 4
  for (int p = 0; p < parts; ++p) {
    const float* x = part(p);
    const float m = x[D * 128], l = x[(D + 1) * 128];
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[(q * 8 + i) * 128];
    if (m == NEG_INF) continue;                          // saw nothing: what it holds may be anything
    const float f = fast_exp2(m - M);
    L += l * f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // infinities and NaN of V stand whatever the weight
      const bool odd = (__float_as_uint(y[i]) & 0x7f800000u) == 0x7f800000u;
      o[i] += odd ? y[i] : y[i] * f;
    }
  }
  const float inv = L > 0.f ? 1.f / L : (L != L ? L : 0.f);
  *reinterpret_cast<uint4*>(P.out + (static_cast<int64_t>(row0 + j) * P.Hq + head.y * P.G + rh) * D + q * 8) =
      make_uint4(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv), pack_bf16x2(o[4] * inv, o[5] * inv),
                 pack_bf16x2(o[6] * inv, o[7] * inv));
}

}  // namespace pdattn

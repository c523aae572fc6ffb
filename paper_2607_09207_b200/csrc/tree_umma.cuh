// Attention for a tree of drafted tokens over the paged cache, on the 5th-generation tensor cores: tree_kernel, tree_join_kernel.
//
//   out = softmax_t(scale q.k_t) . V over the keys before the tree and those of the tree that the token's mask names
//
// Rows.  The query rows of one KV head are packed: row r of a 128-row tile is head r % G of token r / G, so a tile holds
// floor(128 / G) whole tokens and every K/V tile is read once for all of them.
//
//   S_t[128, 64 keys] = Q_t . K^T     both from shared memory            t = 0, 1
//   O_t[128, d]      += P_t . V       P from tensor memory (over S_t's columns), V from shared memory
//
// A group's scores have two buffers of 64 columns: those of its next key tile are there when it has handed over the weights of the
// present one, so no product waits in the chain of a group, and 64 scores stay in a thread's registers: read once, no second pass.
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
// Roles: warps 0-7 softmax, 8 walks the units and loads Q and K, 9 loads V (TMA), 10 and 11 issue the MMAs of a group each, 12-15: over the
// bf16 cache two of them guard V (see prefill_umma.cuh: non-finite elements of V at keys that some row does not see are set to 0 and added
// again for the rows that see them); over the fp8 cache they widen V's codes to fp16 (exact), which is the guard as well, and split Q.
//
// fp8.  The codes of K are an operand as they come: Q is split into two e4m3 terms per element, with a power of two per row, and
// both run against the same K tile (twice the multiplications at twice the rate).  V's pages are transposed, so its tile is K-major
// in the second product.
//
// Numbers: scores, maxima, sums and O in fp32.  The weights are rounded to bf16 for the second product (at most 2^-8 of each,
// independent): the size of the final rounding.  (Two terms, as the single-token steps have them, would cost half as much tensor work
// again, where the products are a third to two thirds of a key tile's time.)  In the paired form a quarter of the exponentials is a
// polynomial good to 2^-18.5, the others to 2^-22.  The reference of the online softmax follows the running maximum when that grew by
// more than 2^8, so O is rarely rescaled.  The fp8 form rounds them to fp16 (2^-11 of each), whose range is short: all carry a factor
// 2^11, which l and O have alike within a piece, and the reference, a whole number at or above the maximum when it moves, lags by 2^4 at most.
// So weights end at 2^15 and have all bits down to 2^-24 of the row's largest; smaller ones are off by at most 2^-35 of it.  (With plain
// weights what lies 2^-25 below vanished, and with it what thousands of keys 17 below the largest score add up to.)  All rows of a warp
// move their references when one must: the factors are powers of two, so that changes no bit of normal weights, and there are fewer moves (each
// row by itself, with a lag of 2^2: 304 -> 342 us for 32 x 16 tokens).
//
// Bound and times (replays of a graph; in brackets under the power cap, which long runs of this kernel reach):
//   256 sequences x up to 8 tokens over up to 4600 keys, 28/4 heads of 128    248 us [290]   bytes, 5.6 TB/s; 4 us a unit at the change from one
//       to the next (the groups meet, results), 0.65 a key tile
//   8 x 64 over up to 32,000, 64/8 heads    324 us [385]   0.94 PFLOP/s: the chain of a group, scores -> weights -> product; a
//       key tile takes a pair of row tiles 1950 cycles, 1280 of them MMAs (48 cycles one of scores: 128 x 16 x 64, Q from shared memory)
//   32 x 16 over up to 32,767, e4m3 codes, 64/8 heads    307 us [360]   the same; 1190 cycles a key tile, 640 of them MMAs
// Built and not faster: key tiles of 128 read twice (8 x 64 417 instead of 385 under the cap), two warps a row (324 -> 372, codes
// 306 -> 355: the chain's latencies stay and its halves have to meet), the maximum of the tile before, turns at the exponential unit,
// four loading warps instead of two (256 x 8: the same).  Rows of small trees twice in the row tile, each with half of a tile's keys, so
// that all softmax warps work (at most 64 rows): 249 -> 246, not worth a form of its own.
//
// Every wait is bounded; on expiry the CTA raises ERR_TIMEOUT, the waits fall through, the MMA warp drains, tensor memory is
// freed and the CTA returns.
#pragma once

#include <cuda_fp16.h>

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
  int4* rec;                     // [gridDim][2][2] pieces of cut units: (sequence or -1, KV head, row pair, 1: it ends the unit),
                                 // (cu_tokens of the sequence, tokens of the tree, 0, 0)
  float* partials;               // [gridDim][2][2 tiles][O columns, m, l][128 rows]
  int N, S, Hq, Hkv, G, MB, NB, bs_log2;
  int TQ;                        // tokens of a row tile: 128 / G
  int max_n;                     // tokens of a tree
  float scale_log2;              // scale * log2(e)
};

template <int D, bool PAIR, int EB>
struct TreeCfg {
  static constexpr int HALVES = D / 64;
  static constexpr int Q_HALF = 128 * 128;                  // 128 rows of one 64-column block
  static constexpr int Q_BYTES = HALVES * Q_HALF;           // a row tile of Q
  static constexpr int HALF_BYTES = kTreeKeys * 128;        // 64 keys of one 64-column block
  static constexpr int TILE_BYTES = HALVES * HALF_BYTES;    // a K or V tile of 16-bit elements
  static constexpr int RAW_BYTES = kTreeKeys * D;           // a K or V tile of codes
  static constexpr int QT = PAIR ? 2 : 1;
  static constexpr int NQ = PAIR ? 1 : 2;                   // buffers of an item's Q
  static constexpr int LAG = PAIR ? 2 : 4;                  // the product of key tile c is issued with the scores of c + LAG
  // bytes of a K tile (codes as they come, or bf16) and of the two e4m3 tiles that Q becomes over codes (head_dim 128: in Q's place)
  static constexpr int K_BYTES = EB == 1 ? RAW_BYTES : TILE_BYTES;
  static constexpr int QP_BYTES = EB == 1 && D == 64 ? 2 * 128 * D : 0;
  // rings of K tiles, of V tiles, of V's code tiles
  static constexpr int NK = EB == 2 && D == 128 ? 5 : 6;
  static constexpr int NV = EB == 1 ? 4 : D == 128 ? 5 : 6;
  static constexpr int NR = EB == 1 ? 4 : 0;
  static constexpr int RING_BYTES = NQ * QT * (Q_BYTES + QP_BYTES) + NK * K_BYTES + NV * TILE_BYTES + NR * RAW_BYTES;
  static constexpr int CTRL_BYTES = 2048 + (EB == 1 ? TR_ITEMS * QT * 512 : 0);
  static constexpr int DYN_BYTES = 1024 + RING_BYTES + CTRL_BYTES;
  static constexpr int COL_S = 0, COL_O = 256, TMEM_COLS = 512;
  static_assert(DYN_BYTES <= 232448, "shared memory");
  static_assert(NV >= LAG && NK >= 2 && NK <= 6 && (EB == 2 || NR >= 1), "rings");
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
  // per key tile c of the CTA (mod 8): K, V have landed; V has passed the guard (fp8: is widened); step c is done, i.e. the scores
  // of key tile c and the product of c - LAG
  uint64_t k_full[8], v_full[8], v_ok[8], step[8];
  uint64_t q_full[2], q_ok[2], q_free[2];        // per buffer of Q: it has landed; fp8: is split; its scores are done
  // fp8: the factors of an item's rows are there.  Per item in flight, not per buffer of Q: the scores run ahead of the softmax, so a
  // buffer may have its next users before the softmax has come to the first.
  uint64_t scale_ok[TR_ITEMS];
  uint64_t s_full[2][2], p_full[2][2], pv_done[2][2];   // per group and buffer: scores are there; weights are stored; their product is done
  uint64_t item_full[TR_ITEMS], item_free[TR_ITEMS];
  uint64_t drained[2], meet, meet_widen;         // all softmax warps are here; all widening warps are
  TreeItem item[TR_ITEMS];
  // Per key tile: bit j set = its page j had a bad id; keys whose V held something non-finite.  Both are read before the weights of
  // key tile c are handed over.  They are written anew with K(c + 16), loaded after step c + 16 - NK >= c + 10, which is issued behind
  // the product of c + 6 or a later one, and with V(c + 8), which waits for step c + 8 - NV + LAG >= c + LAG, the one behind the product of c.
  uint32_t page_bad[16];
  uint32_t v_bad[8][2];
  uint32_t odd[TR_ITEMS];                        // split: some row sees such a key
  uint32_t abort, tmem_base;
  float2 ml[64 * 2];                             // split: (m, l) of group 1's rows, then the factors of both groups
};
static_assert(sizeof(TreeCtrl) <= 2048, "control block");
// Behind it over codes: per item in flight and row of its Q, the factor that belongs to the e4m3 terms.
constexpr int TR_QSCALE_AT = 2048;

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
// A look that does not suspend the thread.
__device__ __forceinline__ bool mbar_test_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n"
      "selp.u32 %0, 1, 0, p;\n"
      "}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ int tree_uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }   // known to be the same in every lane
// 2^x of two values on the FMA pipe, x <= 127: x = n + f with n the nearest whole number, and 2^f by the polynomial of degree 4 with the
// smallest largest relative error on [-1/2, 1/2] (2^-18.5).  0 from x = -126.5 down, NaN for NaN.
__device__ __forceinline__ void tree_exp2_pair(float& a, float& b) {
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(-127.f));
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(b) : "f"(-127.f));
  const uint64_t x = pack_f32x2(a, b);
  constexpr float kMagic = 12582912.f;               // 1.5 * 2^23: the sum's last bits are n
  const uint64_t t = add_f32x2(x, pack_f32x2(kMagic, kMagic));
  const uint64_t n = add_f32x2(t, pack_f32x2(-kMagic, -kMagic));
  const uint64_t f = fma_f32x2(n, pack_f32x2(-1.f, -1.f), x);
  uint64_t p = fma_f32x2(pack_f32x2(0.009570089168846607f, 0.009570089168846607f), f, pack_f32x2(0.05591785907745361f, 0.05591785907745361f));
  p = fma_f32x2(p, f, pack_f32x2(0.2402474582195282f, 0.2402474582195282f));
  p = fma_f32x2(p, f, pack_f32x2(0.6931217908859253f, 0.6931217908859253f));
  p = fma_f32x2(p, f, pack_f32x2(0.9999992847442627f, 0.9999992847442627f));
  float ta, tb;
  unpack_f32x2(t, ta, tb);
  p = mul_f32x2(p, pack_f32x2(__uint_as_float((__float_as_uint(ta) << 23) + 0x3f800000u),
                              __uint_as_float((__float_as_uint(tb) << 23) + 0x3f800000u)));
  unpack_f32x2(p, a, b);
}
// D[tmem] (+)= A[smem] . B[smem], e4m3 operands
__device__ __forceinline__ void umma_ss_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p; }" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accum)
      : "memory");
}
// Matrix descriptor of K-major rows of D bytes: 128-byte swizzle for 128, 64-byte swizzle for 64.
template <int D>
__device__ __forceinline__ uint64_t umma_desc_rows(uint32_t saddr) {
  static_assert(D == 128 || D == 64, "row size");
  return static_cast<uint64_t>((saddr >> 4) & 0x3fffu) | (1ull << 16) | (static_cast<uint64_t>((8 * D) >> 4) << 32) | (1ull << 46) |
         ((D == 128 ? 2ull : 4ull) << 61);
}
// Instruction descriptor as umma_idesc's, for fp16 operands (kind::f16) or e4m3 ones (kind::f8f6f4): both are format 0.
__host__ __device__ constexpr uint32_t umma_idesc_f16(int M, int N) {
  return (1u << 4) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}

// What the batch asks of one sequence.
struct TreeSeq {
  int n, row0, L, keys, tiles, units;
  int wrong;                     // why it is left out (an error bit), or 0
};
template <bool PAIR>
__device__ __forceinline__ TreeSeq tree_seq(const TreeParams& P, int s) {
  TreeSeq q;
  q.units = q.tiles = q.n = q.row0 = q.L = q.keys = q.wrong = 0;
  if (s >= P.S) return q;
  q.row0 = __ldg(P.cu_tokens + s);
  const int row1 = __ldg(P.cu_tokens + s + 1);
  if (row1 != q.row0) {
    if (q.row0 < 0 || row1 < q.row0 || row1 > P.N) q.wrong = ERR_BAD_SEQUENCE;     // not a range of the call's tokens
    else if (row1 - q.row0 > P.max_n) q.wrong = ERR_TOO_LARGE;
    else q.n = row1 - q.row0;
  }
  q.L = max(0, __ldg(P.context_lens + s));
  // tokens past the end of the table row are left out like those of a bad page
  q.keys = static_cast<int>(min(static_cast<int64_t>(q.L), static_cast<int64_t>(P.MB) << P.bs_log2));
  q.tiles = static_cast<int>((static_cast<int64_t>(q.keys) + kTreeKeys - 1) / kTreeKeys);
  const int tokens = PAIR ? 2 * P.TQ : P.TQ;
  q.units = (q.n + tokens - 1) / tokens * P.Hkv;
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
  const uint32_t sQ = raw + pad, sQP = sQ + (D == 64 ? C::NQ * QT * C::Q_BYTES : 0);   // (codes) Q's terms
  const uint32_t sK = sQ + C::NQ * QT * (C::Q_BYTES + C::QP_BYTES), sV = sK + NK * C::K_BYTES, rV = sV + NV * C::TILE_BYTES;
  TreeCtrl* ctrl = reinterpret_cast<TreeCtrl*>(smem + C::RING_BYTES);
  float* q_scale = reinterpret_cast<float*>(smem + C::RING_BYTES + TR_QSCALE_AT);   // [TR_ITEMS][QT][128]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float NEG_INF = __int_as_float(0xff800000);

  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&ctrl->drained[0]), 1);
    mbar_init(smem_u32(&ctrl->drained[1]), 1);
    mbar_init(smem_u32(&ctrl->meet), 8);
    mbar_init(smem_u32(&ctrl->meet_widen), 4);
    for (int i = 0; i < 8; ++i) {
      mbar_init(smem_u32(&ctrl->k_full[i]), 1);
      mbar_init(smem_u32(&ctrl->v_full[i]), 1);
      mbar_init(smem_u32(&ctrl->v_ok[i]), F8 ? 4 : 2);
      mbar_init(smem_u32(&ctrl->step[i]), PAIR ? 2 : 1);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&ctrl->q_full[t]), 1);
      mbar_init(smem_u32(&ctrl->q_ok[t]), 4);
      mbar_init(smem_u32(&ctrl->q_free[t]), 2);
      for (int b = 0; b < 2; ++b) {
        mbar_init(smem_u32(&ctrl->s_full[t][b]), 1);
        mbar_init(smem_u32(&ctrl->p_full[t][b]), 4);
        mbar_init(smem_u32(&ctrl->pv_done[t][b]), 1);
      }
    }
    for (int i = 0; i < TR_ITEMS; ++i) {
      mbar_init(smem_u32(&ctrl->scale_ok[i]), 4);
      mbar_init(smem_u32(&ctrl->item_full[i]), 1);
      mbar_init(smem_u32(&ctrl->item_free[i]), 8 + 2 + 1 + (F8 ? 4 : 2));   // softmax, MMA, V, guards
    }
    ctrl->abort = 0;
    fence_mbar_init();
  }
  if (warp == 10) {
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
    if (q.wrong && blockIdx.x == 0) atomicOr(&P.hdr->err, q.wrong);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = tree_uniform(static_cast<int>(*reinterpret_cast<volatile uint32_t*>(&ctrl->tmem_base)));
  const uint32_t* abort_flag = &ctrl->abort;

  // ---- this CTA's share: from (s0, u0, t0) to (s1, u1, t1); warp 8 walks it
  int s0 = 0, u0 = 0, t0 = 0, s1 = 0, u1 = 0, t1 = 0;
  if (warp == 8) {
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
    if (warp == 8 || warp == 9) {
      // ================= loads: warp 8 walks the share, publishes its items and loads Q and K; warp 9 loads V
      const bool isV = warp == 9;
      const int ppt = kTreeKeys >> P.bs_log2;              // pages of a key tile
      const int pj = lane & (ppt - 1), h = lane / ppt;
      const bool codes = F8 && isV;                        // to be widened: a ring of their own
      const int ring = codes ? NR : isV ? NV : NK;
      const CUtensorMap* tm = isV ? &tmV : &tmK;
      const uint32_t dst0 = F8 ? (isV ? rV : sK) + (pj << P.bs_log2) * D
                               : (isV ? sV : sK) + h * C::HALF_BYTES + (pj << P.bs_log2) * 128;
      uint64_t* full = isV ? ctrl->v_full : ctrl->k_full;
      bool any_bad = false, ok = true;
      int c = 0, slot = 0;
      auto load_tiles = [&](const TreeItem& it) {
        const int32_t* row = P.block_table + static_cast<int64_t>(it.s) * P.MB;
        const int npages = static_cast<int>((static_cast<int64_t>(it.keys) + (1 << P.bs_log2) - 1) >> P.bs_log2);
        auto page_id = [&](int kt) {
          const int i = kt * ppt + pj;
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
            if (codes) ok = wait(&ctrl->v_ok[(c - NR) & 7], (c - NR) >> 3);
            else ok = wait(&ctrl->step[(isV ? c - NV + LAG : c - NK) & 7], (isV ? c - NV + LAG : c - NK) >> 3);
            if (!ok) return;
          }
          const uint32_t bar = smem_u32(&full[c & 7]);
          if (lane == 0) {
            if (!isV) ctrl->page_bad[c & 15] = badmask;
            mbar_arrive_expect_tx(bar, static_cast<uint32_t>(F8 ? C::RAW_BYTES : C::TILE_BYTES));
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
      };
      if (isV) {
        const TreeItem* ip;
        for (int k = 0; ok && get_item(k, ip); ++k) {
          load_tiles(*ip);
          done_item(k);
        }
      } else {
        int4 rec[4] = {make_int4(-1, 0, 0, 0), make_int4(0, 0, 0, 0), make_int4(-1, 0, 0, 0), make_int4(0, 0, 0, 0)};
        int base = s0 & ~31;
        TreeSeq win = tree_seq<PAIR>(P, base + lane);
        int s = s0, u = u0, t = t0;
        bool more = true, ran_out = false;
        int nq = 0;
        for (int k = 0; ok && more; ++k) {                   // (the last round publishes that there are no more)
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
              rec[2 * which] = make_int4(s, it.g, pair, it.te == tiles ? 1 : 0);
              rec[2 * which + 1] = make_int4(it.row0, n, 0, 0);
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
          if (more && it.te > it.tb) {
            // Q first: an MMA warp that finds nothing to do in an item is done with its Q at once, and must not be so for the
            // buffer's next user before this wait has seen the last one
            const int qb = nq % C::NQ;
            ok = wait(&ctrl->q_free[qb], (nq / C::NQ) ^ 1);
            if (!ok) break;
            if (lane == 0) {
              const uint32_t bar = smem_u32(&ctrl->q_full[qb]);
              mbar_arrive_expect_tx(bar, static_cast<uint32_t>(QT * C::HALVES * P.TQ * P.G * 128));
#pragma unroll
              for (int i = 0; i < QT; ++i)
#pragma unroll
                for (int hh = 0; hh < C::HALVES; ++hh)
                  tma_load_4d(sQ + (qb * QT + i) * C::Q_BYTES + hh * C::Q_HALF, &tmQ, hh * 64, 0, it.g, it.row0 + it.tok0 + i * P.TQ, bar);
            }
            __syncwarp();
            ++nq;
          }
          ok = wait(&ctrl->item_free[k % TR_ITEMS], (k / TR_ITEMS) ^ 1);
          if (!ok) break;
          if (lane == 0) {
            ctrl->item[k % TR_ITEMS] = it;
            ctrl->odd[k % TR_ITEMS] = 0u;
            mbar_arrive(smem_u32(&ctrl->item_full[k % TR_ITEMS]));     // (release: the item is visible to whoever sees the phase)
          }
          __syncwarp();
          if (more) load_tiles(it);
        }
        if (lane == 0) {
#pragma unroll
          for (int i = 0; i < 4; ++i) P.rec[4 * blockIdx.x + i] = rec[i];
          if (ran_out) atomicOr(&P.hdr->err, ERR_BAD_PAGE);
        }
        // given up: no copy may still be on its way into this CTA's shared memory when it ends
        if (*reinterpret_cast<const volatile uint32_t*>(abort_flag))
          for (int i = max(0, nq - C::NQ); i < nq; ++i) mbar_wait(smem_u32(&ctrl->q_full[i % C::NQ]), (i / C::NQ) & 1);
      }
      if (lane == 0) {
        if (any_bad) atomicOr(&P.hdr->err, ERR_BAD_PAGE);
        if (!ok) fail();
      }
      if (*reinterpret_cast<const volatile uint32_t*>(abort_flag))
        for (int i = max(0, c - ring); i < c; ++i) mbar_wait(smem_u32(&full[i & 7]), (i >> 3) & 1);
    } else if (warp == 10 || warp == 11) {
      // ================= MMA issue, a warp per group: one thread waits and issues.  It has the scores of at most two key tiles out at a
      // time, one per buffer, and takes what comes first: the weights of the older one (their product), or the next K tile (its
      // scores), which may belong to the next item.
      const int t = warp - 10;
      uint32_t elected;
      asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(elected));
      if (elected) {
        // Q x K tile, both K-major; fp8: two terms of Q, one after the other, against the codes
        constexpr uint32_t ID_S = F8 ? umma_idesc_f16(128, kTreeKeys) : umma_idesc(128, kTreeKeys, 0, 0);
        constexpr uint32_t ID_O = F8 ? umma_idesc_f16(128, D) : umma_idesc(128, D, 0, 1);   // P (tensor memory) x V (MN-major; fp8: K-major)
        constexpr int STRIDE = PAIR ? 1 : 2;       // from one key tile of this group to the next
        const uint64_t q_desc = F8 ? umma_desc_rows<D>(sQP + (PAIR ? t : 0) * C::Q_BYTES) : umma_desc(sQ + (PAIR ? t : 0) * C::Q_BYTES, 16, 1024);
        const uint64_t k_desc = F8 ? umma_desc_rows<D>(sK) : umma_desc(sK, 16, 1024);
        const uint64_t v_desc = F8 ? umma_desc(sV, 16, 1024) : umma_desc(sV, C::HALF_BYTES, 1024);
        const uint32_t tS0 = tbase + C::COL_S + t * 128, tO = tbase + C::COL_O + t * D;
        uint32_t np = 0;                           // bit b: parity of p_full of buffer b
        int out = 0, v0 = 0, v1 = 0;               // key tiles whose product is to come: how many, the older and the younger
        bool open0 = false, open1 = false;         // ... and whether it begins O anew
        int c = PAIR ? 0 : t, end = 0;             // this group's next key tile; end of the present item
        int first = 0, k = 0, nq = 0;              // its first key tile; items so far, those with key tiles
        bool active = false, more = true, ok = true;
        unsigned long long since = 0ull;
        uint32_t idle = 0;
        while (ok && (more || out > 0)) {
          bool moved = false;
          if (out > 0) {
            // O (+)= P . V of the older key tile.  Nothing else can be done while both buffers are taken.
            const int b = (PAIR ? v0 : v0 >> 1) & 1;
            const uint32_t bar_v = smem_u32(&ctrl->v_ok[v0 & 7]), bar_p = smem_u32(&ctrl->p_full[t][b]);
            bool ready;
            if (out == 2 || !more) {
              ok = tree_wait(bar_v, (v0 >> 3) & 1, abort_flag) && tree_wait(bar_p, (np >> b) & 1u, abort_flag);
              ready = ok;
            } else {
              ready = mbar_test_wait(bar_p, (np >> b) & 1u) && mbar_test_wait(bar_v, (v0 >> 3) & 1);
            }
            if (ready) {
              np ^= 1u << b;
              tc_fence_after();
              const uint64_t vd = v_desc + static_cast<uint64_t>((v0 % NV) * (C::TILE_BYTES >> 4));
              uint32_t accum = open0 ? 0u : 1u;
#pragma unroll
              for (int i = 0; i < kTreeKeys / 16; ++i) {
                umma_ts(tO, tS0 + b * 64 + i * 8, vd + (F8 ? i * 2 : i * (2048 >> 4)), ID_O, accum);
                accum = 1u;
              }
              tc_commit(smem_u32(&ctrl->pv_done[t][b]));
              v0 = v1;
              open0 = open1;
              --out;
              moved = true;
            }
          }
          if (more && c >= end) {
            // the item is through (this group's scores of it are issued), or it had no key tile for this group
            if (mbar_test_wait(smem_u32(&ctrl->item_full[k % TR_ITEMS]), (k / TR_ITEMS) & 1)) {
              const TreeItem& it = ctrl->item[k % TR_ITEMS];
              const int n = it.te - it.tb;
              more = it.s >= 0;
              active = !PAIR || it.rows[t] > 0;
              mbar_arrive(smem_u32(&ctrl->item_free[k % TR_ITEMS]));
              ++k;
              moved = true;
              if (more && n > 0) {
                first = end;
                end += n;
                ++nq;
                if (c >= end) tc_commit(smem_u32(&ctrl->q_free[(nq - 1) % C::NQ]));
              }
            }
          } else if (more && (out == 0 || v0 > c - LAG)) {
            const int qb = (nq - 1) % C::NQ, b = (PAIR ? c : c >> 1) & 1;
            if (mbar_test_wait(smem_u32(&ctrl->k_full[c & 7]), (c >> 3) & 1) &&
                (!active || mbar_test_wait(smem_u32(F8 ? &ctrl->q_ok[qb] : &ctrl->q_full[qb]), ((nq - 1) / C::NQ) & 1))) {
              if (active) {
                tc_fence_after();
                uint64_t kd = k_desc + static_cast<uint64_t>((c % NK) * (C::K_BYTES >> 4));
                uint64_t qd = q_desc + static_cast<uint64_t>(qb * QT * (C::Q_BYTES >> 4));
                uint32_t accum = 0u;
#pragma unroll
                for (int hh = 0; hh < (F8 ? 2 : C::HALVES); ++hh) {
#pragma unroll
                  for (int kk = 0; kk < (F8 ? D / 32 : 4); ++kk) {
                    if constexpr (F8) umma_ss_f8(tS0 + b * 64, qd + kk * 2, kd + kk * 2, ID_S, accum);
                    else umma_ss(tS0 + b * 64, qd + kk * 2, kd + kk * 2, ID_S, accum);
                    accum = 1u;
                  }
                  qd += F8 ? (128 * D) >> 4 : C::Q_HALF >> 4;
                  if (!F8) kd += C::HALF_BYTES >> 4;
                }
                tc_commit(smem_u32(&ctrl->s_full[t][b]));
                const bool opens = c - first < STRIDE;
                if (out == 0) {
                  v0 = c;
                  open0 = opens;
                } else {
                  v1 = c;
                  open1 = opens;
                }
                ++out;
              }
              // this group's scores of c and product of c - LAG
              tc_commit(smem_u32(&ctrl->step[c & 7]));
              c += STRIDE;
              if (c >= end) tc_commit(smem_u32(&ctrl->q_free[qb]));    // this group's scores of the item
              moved = true;
            }
          }
          if (moved) {
            idle = 0;
          } else if ((++idle & 63u) == 0u) {
            const unsigned long long now = globaltimer_ns();
            if (idle == 64u) since = now;
            ok = ok && !*reinterpret_cast<const volatile uint32_t*>(abort_flag) && now - since <= kWaitLimitNs;
          }
        }
        if (!ok) fail();
        // nothing that was issued may still be running on the tensor cores when the tensor memory goes back
        tc_commit(smem_u32(&ctrl->drained[t]));
        mbar_wait(smem_u32(&ctrl->drained[t]), 0);
      }
      __syncwarp();
    } else if (F8) {
      // ================= warps 12-15: Q split into two e4m3 terms, V widened to fp16, 16 codes at a time
      const int w = warp - 12, id = w * 32 + lane;
      const TreeItem* ip;
      int nq = 0, nv = 0, rv = 0, ov = 0, meets = 0;       // items with key tiles; V tiles; ring slots of V's codes and of V
      bool ok = true;
      auto load16 = [&](uint32_t src, uint32_t (&x)[4]) {    // 16 codes
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(src) : "memory");
      };
      auto widen = [&](const uint32_t (&x)[4], uint32_t d0, uint32_t d1) {     // ... to two 16-byte chunks
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
        // V(v): codes [page][d][slot], linear; tile [d][64 keys]
        ok = ok && wait(&ctrl->v_full[v & 7], v >> 3);
        if (ok && v >= NV) ok = wait(&ctrl->step[(v - NV + LAG) & 7], (v - NV + LAG) >> 3);
        if (!ok) return;
        const uint32_t src = rV + rv * C::RAW_BYTES, dst = sV + ov * C::TILE_BYTES;
        if (edge_tile) {
          // the guard: which keys hold a NaN code.  Warp w looks at keys 16 w .. + 15, all of d
          uint32_t bad = 0u;
#pragma unroll 1
          for (int dd = lane; dd < D; dd += 32) {
            const int key = w * 16, page = key >> P.bs_log2, in = key & ((1 << P.bs_log2) - 1);
            const uint32_t from = src + ((page * D + dd) << P.bs_log2) + in;
            uint32_t x[4], mine = 0u;
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(from) : "memory");
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              // a byte is NaN when its low seven bits are all set: adding one carries into the eighth
              const uint32_t hit = ((x[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
#pragma unroll
              for (int i = 0; i < 4; ++i) mine |= (hit >> (8 * i + 7) & 1u) << (e * 4 + i);
              x[e] &= ~((hit >> 7) * 0xffu);
            }
            // (written back: the widening below reads it, by other warps too)
            if (mine)
              asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(from), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
            bad |= mine;
          }
          bad = __reduce_or_sync(0xffffffffu, bad);
          if (lane == 0) reinterpret_cast<uint16_t*>(ctrl->v_bad[v & 7])[w] = static_cast<uint16_t>(bad);
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&ctrl->meet_widen));
          ok = wait(&ctrl->meet_widen, meets++);           // (bounded, unlike a named barrier)
          if (!ok) return;
        }
        constexpr int NC = D * 4 / 128;                    // chunks of 16 codes a thread moves: all loads, then all stores
        uint32_t x[NC][4];
#pragma unroll
        for (int e = 0; e < NC; ++e) load16(src + ((e * 128 + id) << 4), x[e]);
#pragma unroll
        for (int e = 0; e < NC; ++e) {
          const int i = e * 128 + id;                      // chunk i, as they lie
          const int page = (i << 4) >> (P.bs_log2 + (D == 128 ? 7 : 6)), in_page = (i << 4) - page * (D << P.bs_log2);
          const int dd = in_page >> P.bs_log2, key = (page << P.bs_log2) + (in_page & ((1 << P.bs_log2) - 1));
          const uint32_t row = dst + dd * 128;
          const int ch = key >> 3;
          widen(x[e], row + ((ch ^ (dd & 7)) << 4), row + (((ch + 1) ^ (dd & 7)) << 4));
        }
        publish(&ctrl->v_ok[v & 7]);
        if (++rv == NR) rv = 0;
        if (++ov == NV) ov = 0;
      };
      // Row `id` of a row tile of Q: q = 2^-e (q1 + q2), q1 = e4m3(2^e q), q2 = e4m3 of the rest, with 2^e the power of two that brings the
      // row's largest magnitude to (224, 448].  A bf16 has 8 bits, the terms 4 and 4: exact down to 2^-9 of the largest, and off by
      // at most 2^-10 * 2^-e below.  An element that is not finite becomes NaN.
      auto read64 = [&](uint32_t src, uint32_t (&x)[32]) {    // 64 elements of the row
#pragma unroll
        for (int i = 0; i < 8; ++i)
          asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[4 * i]), "=r"(x[4 * i + 1]), "=r"(x[4 * i + 2]), "=r"(x[4 * i + 3])
                       : "r"(src + ((i ^ (id & 7)) << 4)) : "memory");
      };
      auto largest = [&](const uint32_t (&x)[32]) {           // magnitudes as whole numbers; NaN and infinities do not count
        uint32_t top = 0u;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const uint32_t lo = (x[i] << 16) & 0x7fffffffu, hi = x[i] & 0x7fff0000u;
          top = max(top, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
        }
        return top;
      };
      auto terms = [&](uint32_t u, float up, uint32_t& t1, uint32_t& t2) {   // of two elements
        float a = __uint_as_float(u << 16) * up, b = __uint_as_float(u & 0xffff0000u) * up;
        a = fabsf(a) <= 448.f ? a : __int_as_float(0x7fffffff);
        b = fabsf(b) <= 448.f ? b : __int_as_float(0x7fffffff);
        unsigned short q1, q2;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(q1) : "f"(b), "f"(a));
        const uint32_t back = cvt_e4m3x2_f16x2(q1);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&back));
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(q2) : "f"(b - f.y), "f"(a - f.x));
        t1 = q1;
        t2 = q2;
      };
      auto put64 = [&](uint32_t row, int i0, const uint32_t (&y)[16]) {      // 64 codes from chunk i0 of a row on
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t at = static_cast<uint32_t>(D == 128 ? (i0 + i) ^ (id & 7) : i ^ ((id >> 1) & 3)) << 4;
          asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(row + at), "r"(y[4 * i]), "r"(y[4 * i + 1]), "r"(y[4 * i + 2]),
                       "r"(y[4 * i + 3]) : "memory");
        }
      };
      auto split64 = [&](const uint32_t (&x)[32], float up, uint32_t (&y1)[16], uint32_t (&y2)[16]) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          uint32_t a1, a2, b1, b2;
          terms(x[2 * i], up, a1, a2);
          terms(x[2 * i + 1], up, b1, b2);
          y1[i] = a1 | (b1 << 16);
          y2[i] = a2 | (b2 << 16);
        }
      };
      auto split_row = [&](int tile, float* factor) {
        const uint32_t src = sQ + tile * C::Q_BYTES + id * 128;
        uint32_t x[32], y1[16], y2[16];
        uint32_t top = 0u;
#pragma unroll 1
        for (int h = 0; h < C::HALVES; ++h) {
          read64(src + h * C::Q_HALF, x);
          top = max(top, largest(x));
        }
        int e = 135 - static_cast<int>(top >> 23) - ((top & 0x7fffffu) > 0x600000u ? 1 : 0);   // 448 = 1.75 * 2^8
        e = top == 0u ? 0 : min(126, e);
        const float up = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
        factor[id] = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
        // the terms' rows; with head_dim 128 they lie over the row itself: a half's second terms wait until the other half is read
        const uint32_t d1 = sQP + tile * C::Q_BYTES + id * D, d2 = d1 + 128 * D;
        read64(src, x);
        split64(x, up, y1, y2);
        put64(d1, 0, y1);
        if constexpr (D == 128) {
          read64(src + C::Q_HALF, x);
          put64(d2, 0, y2);
          split64(x, up, y1, y2);
          put64(d1, 4, y1);
          put64(d2, 4, y2);
        } else {
          put64(d2, 0, y2);
        }
      };
      for (int k = 0; ok && get_item(k, ip); ++k) {
        const TreeItem& it = *ip;
        const int tb = it.tb, te = it.te, edge = it.edge;
        if (te > tb) {
          const int qb = nq % C::NQ;
          ok = wait(&ctrl->q_full[qb], nq / C::NQ);
          ++nq;
          if (!ok) break;
#pragma unroll 1
          for (int i = 0; i < QT; ++i) split_row(qb * QT + i, q_scale + (k % TR_ITEMS * QT + i) * 128);
          publish(&ctrl->q_ok[qb]);
        }
        if (lane == 0) mbar_arrive(smem_u32(&ctrl->scale_ok[k % TR_ITEMS]));
        for (int kt = tb; kt < te && ok; ++kt) do_v(kt >= edge, nv++);
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
            {
              // 32 keys: a key's row of a 64-column block is 128 bytes = 8 chunks, four keys per warp-wide load.  A bf16 is not
              // finite when its eight exponent bits are all set: adding one to them then carries into the sign's place.
              const uint32_t rows = base + w * 32 * 128;
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
              if (lane == 0) ctrl->v_bad[c & 7][w] = bad;
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
    // all eight warps (bounded, unlike a named barrier)
    auto meet_arrive = [&]() {
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ctrl->meet));
    };
    bool owed = false;                 // arrived, but not waited
    auto meet_wait = [&]() {
      wait_all(&ctrl->meet, meets++);
      owed = false;
    };
    auto meet = [&]() {
      meet_arrive();
      meet_wait();
    };
    const TreeItem* ip;
    int c0 = 0;                        // key tiles of the CTA before this item
    uint32_t ns = 0;                   // bit b: parity of s_full (and of p_full, pv_done) of this group's buffer b
    constexpr float kLag = F8 ? 4.f : 8.f, kFactor = 11.f;   // (base 2)
    constexpr float kUnfactor = F8 ? 1.f / 2048.f : 1.f;     // a piece's results leave without the factor
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
      if (F8 && te > tb) {
        wait_all(&ctrl->scale_ok[k % TR_ITEMS], k / TR_ITEMS);
        sc *= q_scale[(k % TR_ITEMS * QT + (PAIR ? t : 0)) * 128 + r];
      }
      if (sc == 0.f) sc = 1.1754944e-38f;               // (all weights alike; 0 * inf would be NaN)
      float m = NEG_INF, mu = 0.f, l = 0.f;             // running maximum (reference), the same or 0 in its place; sum
      bool odd = false;                                 // this row sees a key with a non-finite V
      int last = -1;                                    // this group's last buffer in use
      const int own = PAIR ? tb : tb + ((c0 ^ t) & 1);  // split: group t has the key tiles whose number in the CTA has its parity
      for (int kt = own; mine && kt < te; kt += PAIR ? 1 : 2) {
        const int c = c0 + (kt - tb), b = (PAIR ? c : c >> 1) & 1;
        const bool first = last < 0;
        wait_all(&ctrl->s_full[t][b], ns >> b);
        if (!busy) {
          if (!F8 && owed) meet_wait();
          if (lane == 0) mbar_arrive(smem_u32(&ctrl->p_full[t][b]));
          ns ^= 1u << b;
          last = b;
          continue;
        }
        tc_fence_after();
        uint32_t x[64];
        tmem_ld32(tS + b * 64, *reinterpret_cast<uint32_t(*)[32]>(&x[0]));
        tmem_ld32(tS + b * 64 + 32, *reinterpret_cast<uint32_t(*)[32]>(&x[32]));
        tc_wait_ld();
        const uint32_t pb = ctrl->page_bad[c & 15];
        if (kt >= edge || flip || pb != 0) {
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t vis = sees ? tree_visible(kt * kTreeKeys + q * 32, at, keys, mask) : 0u;
            if (P.bs_log2 == 4) vis &= ~(((pb >> (2 * q)) & 1u ? 0xffffu : 0u) | ((pb >> (2 * q + 1)) & 1u ? 0xffff0000u : 0u));
            else if ((pb >> (q >> (P.bs_log2 - 5))) & 1u) vis = 0u;
            if (flip) {
#pragma unroll
              for (int i = 0; i < 32; ++i) x[q * 32 + i] ^= 0x80000000u;
            }
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (!((vis >> i) & 1u)) x[q * 32 + i] = __float_as_uint(NEG_INF);
          }
          if (kt >= edge) {
            // before the weights go, for they let the guard's word be written anew: does this row see a guarded key?
            wait_all(&ctrl->v_ok[c & 7], c >> 3);
            if (sees) {
#pragma unroll
              for (int q = 0; q < 2; ++q)
                odd |= (*reinterpret_cast<volatile uint32_t*>(&ctrl->v_bad[c & 7][q]) &
                        tree_visible(kt * kTreeKeys + 32 * q, at, keys, mask)) != 0u;
            }
          }
        }
        float m4[4] = {NEG_INF, NEG_INF, NEG_INF, NEG_INF};
#pragma unroll
        for (int i = 0; i < 64; i += 2) m4[(i >> 1) & 3] = max3(m4[(i >> 1) & 3], __uint_as_float(x[i]), __uint_as_float(x[i + 1]));
        float mx = fmaxf(max3(m4[0], m4[1], m4[2]), m4[3]);
        mx = mx == NEG_INF ? NEG_INF : F8 ? ceilf(__fmul_ru(mx, sc)) : mx * sc;
        float alpha = 1.f;
        // The reference moves with the first tile, and when the maximum grew by more than 2^kLag.  (Codes: rounded so that no weight
        // leaves fp16's range where fp32 cannot tell such scores apart any more.)
        bool grow = first || mx > (F8 ? __fadd_rd(m, kLag) : m + kLag);
        if (__any_sync(0xffffffffu, valid && grow)) {
          if (F8) grow = true;
          const float m_new = grow ? fmaxf(m, mx) : m;
          mu = m_new == NEG_INF ? 0.f : m_new;
          alpha = grow ? fast_exp2(m - mu) : 1.f;
          m = m_new;
          if (!first) {
            // scale this row of O, once the product before this one is done
            wait_all(&ctrl->pv_done[t][last], (ns >> last) ^ 1u);
            tc_fence_after();
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
        }
        uint64_t sum0 = 0ull, sum1 = 0ull;
        const float off = F8 ? __fadd_rd(kFactor, -mu) : -mu;
        const uint64_t sc2 = pack_f32x2(sc, sc), mu2 = pack_f32x2(off, off);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float p0, p1;
            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(x[q * 32 + 2 * i]), __uint_as_float(x[q * 32 + 2 * i + 1])), sc2, mu2), p0, p1);
            // PAIR: a quarter on the FMA pipe (8 x 64 tokens 388 -> 379 us under the power cap; split, 256 x 8: 281 -> 287)
            if (PAIR && (i & 3) == 3) {
              tree_exp2_pair(p0, p1);
            } else {
              p0 = fast_exp2(p0);
              p1 = fast_exp2(p1);
            }
            const uint64_t pp = pack_f32x2(p0, p1);
            if (i & 1) sum1 = add_f32x2(sum1, pp);
            else sum0 = add_f32x2(sum0, pp);
            pk[i] = F8 ? pack_f16x2(p0, p1) : pack_bf16x2(p0, p1);
          }
          tmem_st16(tS + b * 64 + q * 16, pk);          // (over scores that have been read)
        }
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (!F8 && owed) meet_wait();                   // (these weights may make O anew: the other group has read the last item's)
        if (lane == 0) mbar_arrive(smem_u32(&ctrl->p_full[t][b]));
        ns ^= 1u << b;
        last = b;
        {
          float a0, a1, b0, b1;
          unpack_f32x2(sum0, a0, a1);
          unpack_f32x2(sum1, b0, b1);
          l = l * alpha + ((a0 + a1) + (b0 + b1));
        }
      }
      // ---- the item's rows
      const bool any = last >= 0;                       // this group had key tiles
      const float vs = F8 ? __ldg(P.v_scale + it.g) : 1.f;
      if (any) {
        wait_all(&ctrl->pv_done[t][last], (ns >> last) ^ 1u);   // the last product is done, and with it those before it
        tc_fence_after();
      }
      // Factors of O_0 and O_1 in this row's output; below 0: the row saw nothing there, and what O holds may be anything.  (A factor of
      // 0 is a weight that vanishes: what is not finite stays so.)
      constexpr float kUnseen = -1.f;
      float f[2] = {kUnseen, kUnseen};
      bool have[2];
      const bool whole = it.part < 0;
      if (PAIR) {
        have[0] = any && t == 0;
        have[1] = any && t == 1;
        f[t] = l == 0.f ? kUnseen : whole ? 1.f / l : kUnfactor;
      } else {
        const int even = tb + (c0 & 1), odds = tb + ((c0 & 1) ^ 1);
        have[0] = te > even;
        have[1] = te > odds;
        if (owed) meet_wait();
        if (odd) atomicOr(&ctrl->odd[k % TR_ITEMS], 1u);
        if (t == 1) ctrl->ml[r] = make_float2(m, l);
        meet();
        odd = *reinterpret_cast<volatile uint32_t*>(&ctrl->odd[k % TR_ITEMS]) != 0u;
        if (t == 0) {
          const float2 other = ctrl->ml[r];
          const float M = fmaxf(m, other.x);
          const bool saw0 = l != 0.f, saw1 = other.y != 0.f;
          f[0] = m == NEG_INF ? 0.f : fast_exp2(m - M);
          f[1] = other.x == NEG_INF ? 0.f : fast_exp2(other.x - M);
          m = M;
          l = l * f[0] + other.y * f[1];
          const float inv = whole ? 1.f / l : kUnfactor;      // (used where something was seen)
          f[0] *= inv;
          f[1] *= inv;
          if (!saw0) f[0] = kUnseen;
          if (!saw1) f[1] = kUnseen;
          ctrl->ml[r] = make_float2(f[0], f[1]);
        }
        meet();
        if (t == 1) {
          const float2 both = ctrl->ml[r];
          f[0] = both.x;
          f[1] = both.y;
        }
        tc_fence_after();                               // (the other group's O: its product was seen to be done before the barrier)
      }
      const bool saw[2] = {!(f[0] < 0.f), !(f[1] < 0.f)};
      f[0] *= vs;
      f[1] *= vs;
      if (mine && busy) {
        // a part of a unit leaves its sums as they are
        float* part = whole ? nullptr : P.partials + (static_cast<int64_t>(it.part) * 2 + (PAIR ? t : 0)) * ((D + 2) * 128) + r;
        if (part && valid && (PAIR || t == 0)) {
          part[D * 128] = m;
          part[(D + 1) * 128] = l * kUnfactor;
        }
        __nv_bfloat16* out0 = P.out + (static_cast<int64_t>(it.row0 + it.tok0 + (PAIR ? t * P.TQ : 0)) * P.Hq + it.g * P.G) * D;
        const int offset = valid ? (rj * P.Hq + rh) * D : -1;     // of this thread's row
        const int q0 = PAIR ? 0 : t * (D / 64), q1 = PAIR ? D / 32 : q0 + D / 64;   // split: half of the columns each
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
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = saw[tt] ? fmaf(__uint_as_float(o[i]), f[tt], v[i]) : v[i];
          }
          if (odd && sees) {
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
      // split: neither group may hand weights of the next item over while the other still reads O.  It waits for that when it has some;
      // over codes at once (the check in the loop over the key tiles cost more there: 317 -> 346 us for 32 x 16 tokens).
      if (!PAIR) {
        meet_arrive();
        if (F8) meet_wait();
        else owed = true;
      }
      c0 += te - tb;
      done_item(k);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 10) tmem_dealloc(tbase, C::TMEM_COLS);
}

// The pieces of the units that shares' ends cut, put together in order: block (share in which the unit begins, row tile, 16 columns),
// a thread per row.     M = max m_j;  out = sum O_j 2^(m_j - M) / sum l_j 2^(m_j - M)
// Bound by the latency of its loads (neighbouring rows are neighbours in memory): the records of all shares that may follow come at
// once, then all maxima, then four pieces at a time.
constexpr int TR_JOIN_COLS = 16;
template <int D, bool PAIR>
__global__ void __launch_bounds__(128)
tree_join_kernel(const __grid_constant__ TreeParams P, int ctas) {
  __shared__ int list[2 * TR_CTAS], last[8], count[8];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int c = blockIdx.x, t = blockIdx.y, q = blockIdx.z, r = threadIdx.x, warp = r >> 5, lane = r & 31;
  static_assert(TR_CTAS <= 257, "two records a thread");
  const int4 head = P.rec[4 * c + 2], whose = P.rec[4 * c + 3];
  int4 x[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int cc = c + 1 + e * 128 + r;
    x[e] = cc < ctas ? P.rec[4 * cc] : make_int4(-1, 0, 0, 0);
  }
  if (head.x < 0) return;
  // the unit's other pieces: first pieces of the shares that follow, up to the one that ends the unit (shares may be empty)
  uint32_t mine[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const bool own = x[e].x == head.x && x[e].y == head.y && x[e].z == head.z;
    const uint32_t ends = __ballot_sync(0xffffffffu, own && x[e].w == 1), owns = __ballot_sync(0xffffffffu, own);
    mine[e] = owns & (ends ? (ends & (0u - ends)) * 2u - 1u : 0xffffffffu);       // up to the one that ends the unit
    if (lane == 0) {
      last[e * 4 + warp] = ends != 0u;
      count[e * 4 + warp] = __popc(mine[e]);
    }
  }
  if (r == 0) list[0] = 2 * c + 1;
  __syncthreads();
  int n = 1;
  bool over = false;
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    if (!over && (w & 3) == warp && (mine[w >> 2] >> lane & 1u))
      list[n + __popc(mine[w >> 2] & ((1u << lane) - 1u))] = 2 * (c + 1 + (w >> 2) * 128 + r);
    if (!over) n += count[w];
    over |= last[w] != 0;
  }
  __syncthreads();
  const int rj = r / P.G, rh = r - rj * P.G;
  const int j = (PAIR ? (2 * head.z + t) * P.TQ : 0) + rj;
  if (rj >= P.TQ || j >= whose.y) return;
  constexpr int64_t TILE_FLOATS = (D + 2) * 128;
  auto part = [&](int p) { return P.partials + (static_cast<int64_t>(list[p]) * 2 + t) * TILE_FLOATS + r; };
  const float NEG_INF = __int_as_float(0xff800000);
  float M = NEG_INF, L = 0.f, o[TR_JOIN_COLS];
#pragma unroll
  for (int i = 0; i < TR_JOIN_COLS; ++i) o[i] = 0.f;
#pragma unroll 8
  for (int p = 0; p < n; ++p) M = fmaxf(M, part(p)[D * 128]);
#pragma unroll 4
  for (int p = 0; p < n; ++p) {
    const float* from = part(p);
    const float m = from[D * 128], l = from[(D + 1) * 128];
    float y[TR_JOIN_COLS];
#pragma unroll
    for (int i = 0; i < TR_JOIN_COLS; ++i) y[i] = from[(q * TR_JOIN_COLS + i) * 128];
    // Saw nothing: what it holds may be anything.  (Scores that are all NaN leave the maximum there too, but not the sum: it stays.)
    if (m == NEG_INF && l == 0.f) continue;
    const float f = fast_exp2(m - M);
    L += l * f;
#pragma unroll
    for (int i = 0; i < TR_JOIN_COLS; ++i) {
      // infinities and NaN of V stand whatever the weight
      const bool odd = (__float_as_uint(y[i]) & 0x7f800000u) == 0x7f800000u;
      o[i] += odd ? y[i] : y[i] * f;
    }
  }
  const float inv = L > 0.f ? 1.f / L : (L != L ? L : 0.f);
  uint4* out = reinterpret_cast<uint4*>(P.out + (static_cast<int64_t>(whose.x + j) * P.Hq + head.y * P.G + rh) * D + q * TR_JOIN_COLS);
#pragma unroll
  for (int i = 0; i < TR_JOIN_COLS / 8; ++i)
    out[i] = make_uint4(pack_bf16x2(o[8 * i] * inv, o[8 * i + 1] * inv), pack_bf16x2(o[8 * i + 2] * inv, o[8 * i + 3] * inv),
                        pack_bf16x2(o[8 * i + 4] * inv, o[8 * i + 5] * inv), pack_bf16x2(o[8 * i + 6] * inv, o[8 * i + 7] * inv));
}

}  // namespace pdattn

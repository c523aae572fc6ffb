// Prompt attention over the paged cache on the 5th-generation tensor cores: prefill_kernel.
//
//   x_t = scale q.k_t, capped by a tanh and biased by distance if asked;  out = softmax_t(x_t) . V over lo <= t < hi
//
// Work.  The query rows of one KV head are packed: row r of a 128-row tile is head r % G of token r / G, so a tile holds
// floor(128 / G) whole tokens and K/V tiles are read once for all G heads.  An item is (sequence, pair of tiles, KV head); a
// persistent CTA walks the 128-key tiles that any row of its pair sees and takes the next item from a counter, late
// (long) ones first.  Sequence s owns the pair slots from cu[s] / (2 tokens-per-tile) + s on: enough of them without a prefix
// sum, so the launch needs no host copy of the lengths (slots without tokens are stepped over).
//
//   S_t[128, 128 keys]  = Q_t . K^T         both from shared memory               t = 0, 1: the two tiles of the pair
//   O_t[128, d]        += P_t . V           P from tensor memory (over S_t's columns), V from shared memory
//
// The pair is what keeps the tensor cores busy: while the softmax warps of one tile work on S_t the products of the other
// run.  Roles: warps 0-3 and 4-7 softmax of tile 0 and 1 (a thread owns a row: no shuffles), warp 8 issues the MMAs, warp 9
// loads Q, K, V (TMA), warp 10 prepares items ahead, warp 11 guards V.  S_t of the next key tile is issued right behind the
// P_t . V of the present one by the same thread, in order, so the buffer that P_t occupies needs no further wait.
//
// Masks are intervals per row.  A key tile that every row of a tile sees whole takes no mask at all; the others ("edge" tiles)
// are masked by select.  A masked weight is 0, and 0 * inf or 0 * NaN would still poison the row, so in edge tiles warp 11 sets
// the non-finite elements of V to 0 before the product and notes the keys; a row that does see such a key adds those elements
// to its output at the end (whatever the weight, infinity and NaN are absorbing).
//
// Numbers: scores, maxima, sums and O in fp32; the weights are rounded to bf16 for the second product (relative 2^-9 each,
// independent: the same size as the final rounding of the output; two terms, as in the decode kernel, would cost half as much
// tensor work again).  The reference of the online softmax follows the running maximum only when that grew by more than 2^8,
// so O is rarely rescaled.
//
// Every wait is bounded; on expiry the CTA raises ERR_TIMEOUT, the waits fall through, the MMA thread drains, tensor memory
// is freed and the CTA returns.
#pragma once

#include <climits>

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
  int window;
  float scale_log2;              // scale * log2(e)
  float cap2;                    // cap * log2(e)
  float cap_k;                   // 2 scale / cap * log2(e)
};

constexpr int PF_KEYS = 128;     // keys of a tile
constexpr int PF_ITEMS = 3;      // items in flight between the warps
constexpr int PF_NTHREADS = 384;
constexpr int PF_LAUNCH_REGS = 168, PF_SOFTMAX_REGS = 208, PF_OTHER_REGS = 88;   // a thread
static_assert(256 * PF_SOFTMAX_REGS + 128 * PF_OTHER_REGS <= PF_NTHREADS * PF_LAUNCH_REGS, "register split");

template <int D>
struct PrefillCfg {
  static constexpr int HALVES = D / 64;
  static constexpr int HALF_BYTES = 128 * 128;              // 128 rows of one 64-column block
  static constexpr int TILE_BYTES = HALVES * HALF_BYTES;    // a Q, K or V tile
  static constexpr int NST = D == 128 ? 5 : 8;              // ring of K and V tiles, in order K0 V0 K1 V1 ...
  static constexpr int CTRL_BYTES = 1024;
  static constexpr int DYN_BYTES = 1024 + (2 + NST) * TILE_BYTES + CTRL_BYTES;
  static constexpr int COL_S = 0, COL_O = 256, TMEM_COLS = 512;
  static_assert(DYN_BYTES <= 232448, "shared memory");
};

struct PrefillItem {
  int s, g, tok0, n;             // sequence, KV head, first token of the pair within the sequence, new tokens of the sequence
  int L, row0;                   // context length; cu_tokens[s]
  int begin[2], end[2];          // key tiles [begin, end) of each tile; begin == end: none
  int max_lo[2], min_hi[2];      // keys [max_lo, min_hi) are seen by every row of the tile
  int rows[2];                   // tokens of each tile
};

struct PrefillCtrl {
  uint64_t full[8], empty[8];                    // ring
  uint64_t q_full[2], q_free[2], s_full[2], p_full[2], pv_done[2];
  uint64_t v_ok[4];                              // V of key tile c has passed the guard (c mod 4)
  uint64_t item_full[PF_ITEMS], item_free[PF_ITEMS];
  uint64_t drained;
  PrefillItem item[PF_ITEMS];
  uint32_t page_bad[4];                          // per key tile (mod 4): bit j set = its page j had a bad id
  uint32_t v_bad[4][4];                          // per key tile: keys whose V held something non-finite
  uint32_t abort, tmem_base;
};
static_assert(sizeof(PrefillCtrl) <= 1024, "control block");

// first and one-past-last key that token j of a sequence sees
__device__ __forceinline__ int2 prefill_interval(const PrefillParams& P, int L, int n, int row0, int prefix, int j) {
  const int pos = L - n + j;
  int lo = 0;
  if (P.window > 0) lo = max(lo, pos - P.window + 1);
  if (P.key_begin) lo = max(lo, __ldg(P.key_begin + row0 + j));
  const int hi = pos < 0 ? 0 : min(L, max(pos + 1, prefix));
  return lo < hi ? make_int2(lo, hi) : make_int2(0, 0);
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
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
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

// CAP: scores capped by a tanh.  GEN: scores brought to base-2 units one by one (distance bias, or a scale that is not
// positive); without it the scale rides in the exponent's multiply-add.
template <int D, bool CAP, bool GEN>
__global__ void __launch_bounds__(PF_NTHREADS, 1)
prefill_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
               const __grid_constant__ CUtensorMap tmV, const __grid_constant__ PrefillParams P) {
  using C = PrefillCfg<D>;
  constexpr int NST = C::NST;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t pad = (1024u - (raw & 1023u)) & 1023u;
  uint8_t* smem = smem_raw + pad;
  const uint32_t sQ = raw + pad, ring = sQ + 2 * C::TILE_BYTES;
  PrefillCtrl* ctrl = reinterpret_cast<PrefillCtrl*>(smem + (2 + NST) * C::TILE_BYTES);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float NEG_INF = __int_as_float(0xff800000);

  if (threadIdx.x == 0) {
    for (int i = 0; i < NST; ++i) {
      mbar_init(smem_u32(&ctrl->full[i]), 1);
      mbar_init(smem_u32(&ctrl->empty[i]), 1);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&ctrl->q_full[t]), 1);
      mbar_init(smem_u32(&ctrl->q_free[t]), 1);
      mbar_init(smem_u32(&ctrl->s_full[t]), 1);
      mbar_init(smem_u32(&ctrl->p_full[t]), 128);
      mbar_init(smem_u32(&ctrl->pv_done[t]), 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(smem_u32(&ctrl->v_ok[i]), 1);
    for (int i = 0; i < PF_ITEMS; ++i) {
      mbar_init(smem_u32(&ctrl->item_full[i]), 1);
      mbar_init(smem_u32(&ctrl->item_free[i]), 11);   // softmax warps, MMA, loads, guard
    }
    mbar_init(smem_u32(&ctrl->drained), 1);
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
  const uint32_t tbase = *reinterpret_cast<volatile uint32_t*>(&ctrl->tmem_base);
  asm volatile("griddepcontrol.wait;" ::: "memory");   // a programmatic dependent of the kernel before it on the stream
  const uint32_t* abort_flag = &ctrl->abort;
  auto fail = [&]() {
    atomicOr(&P.hdr->err, ERR_TIMEOUT);
    atomicExch(&ctrl->abort, 1u);
  };
  // the k-th item of this CTA (false: no more, or a wait ran out); uniform over the warp
  auto get_item = [&](int k, const PrefillItem*& it) -> bool {
    const int e = k % PF_ITEMS;
    if (!__all_sync(0xffffffffu, mbar_wait_abortable(smem_u32(&ctrl->item_full[e]), (k / PF_ITEMS) & 1, abort_flag))) {
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
  // whether key tile kt is masked for some row of the pair
  auto edge = [&](const PrefillItem& it, int kt) {
    bool e = false;
#pragma unroll
    for (int t = 0; t < 2; ++t)
      e |= active(it, t, kt) && (kt * PF_KEYS < it.max_lo[t] || (kt + 1) * PF_KEYS > it.min_hi[t]);
    return e;
  };

  // The softmax threads hold a row of scores each; they take the registers that the others leave.
  if (warp >= 8) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PF_OTHER_REGS));
  if (warp == 10) {
    // ================= items: found one or two ahead of their use
    int next = blockIdx.x;
    for (int k = 0;; ++k) {
      PrefillItem it;
      it.s = -1;
      while (next < P.n_items) {
        const int slots = P.n_items / P.Hkv;
        const int slot = slots - 1 - next / P.Hkv;      // the late pairs of a sequence, which see most keys, first
        it.g = next % P.Hkv;
        int drawn = 0;
        if (lane == 0) drawn = atomicAdd(&P.hdr->counter, 1);
        next = static_cast<int>(gridDim.x) + __shfl_sync(0xffffffffu, drawn, 0);
        // the last sequence whose first slot is at or before this one
        const int TP = 2 * P.TQ;
        int lo = 0, len = P.S;
        while (len > 1) {
          const int step = (len + 31) / 32, i = lane * step;
          const bool below = i < len && __ldg(P.cu_tokens + lo + i) / TP + lo + i <= slot;
          const uint32_t m = __ballot_sync(0xffffffffu, below);
          const int b = m ? 31 - __clz(m) : 0;
          lo += b * step;
          len = min(step, len - b * step);
        }
        const int row0 = __ldg(P.cu_tokens + lo), row1 = __ldg(P.cu_tokens + lo + 1);
        const int tok0 = (slot - (row0 / TP + lo)) * TP;
        if (row0 < 0 || row1 > P.N || tok0 < 0 || tok0 >= row1 - row0) continue;   // a slot without tokens
        it.s = lo;
        it.tok0 = tok0;
        it.row0 = row0;
        it.n = row1 - row0;
        it.L = max(0, __ldg(P.context_lens + lo));
        const int prefix = P.prefix_lens ? __ldg(P.prefix_lens + lo) : 0;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          it.rows[t] = min(P.TQ, max(0, it.n - tok0 - t * P.TQ));
          int lo_min = INT_MAX, lo_max = 0, hi_min = INT_MAX, hi_max = 0;
          for (int j = lane; j < it.rows[t]; j += 32) {
            const int2 v = prefill_interval(P, it.L, it.n, row0, prefix, tok0 + t * P.TQ + j);
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
          it.max_lo[t] = lo_max;
          it.min_hi[t] = hi_min;
        }
        break;
      }
      const int e = k % PF_ITEMS;
      if (!__all_sync(0xffffffffu, mbar_wait_abortable(smem_u32(&ctrl->item_free[e]), ((k / PF_ITEMS) & 1) ^ 1, abort_flag))) {
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
  } else if (warp == 9) {
    // ================= loads
    const int ppt = PF_KEYS >> P.bs_log2;               // pages of a key tile
    const int j = lane & (ppt - 1), h = lane / ppt;
    bool any_bad = false, ok = true;
    int c = 0, issued = 0, nq[2] = {0, 0};
    const PrefillItem* ip;
    for (int k = 0; ok && get_item(k, ip); ++k) {
      const PrefillItem& it = *ip;
      const int32_t* row = P.block_table + static_cast<int64_t>(it.s) * P.MB;
      const int npages = (it.L + (1 << P.bs_log2) - 1) >> P.bs_log2;
      auto page_id = [&](int kt) {
        const int i = kt * ppt + j;
        return i >= npages ? -2 : i < P.MB ? __ldg(row + i) : -1;     // -2: past the end, filled with zeros; -1: bad
      };
      const int k0 = tiles_from(it), k1 = tiles_to(it);
      int id_next = k0 < k1 ? page_id(k0) : 0;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (!ok || it.begin[t] == it.end[t]) continue;
        ok = __all_sync(0xffffffffu, mbar_wait_abortable(smem_u32(&ctrl->q_free[t]), (nq[t] & 1) ^ 1, abort_flag));
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
      for (int kt = k0; kt < k1 && ok; ++kt) {
        int id = id_next;
        if (kt + 1 < k1) id_next = page_id(kt + 1);
        if (!active(it, 0, kt) && !active(it, 1, kt)) continue;
        const bool bad = id != -2 && (id < 0 || id >= P.NB);
        const uint32_t badmask = __ballot_sync(0xffffffffu, bad && h == 0);
        any_bad |= badmask != 0;
        if (id < 0 || id >= P.NB) id = P.NB;            // out-of-bounds coordinate: TMA fills zeros, nothing is read
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const int i = 2 * c + kv, slot = i % NST;
          if (!__all_sync(0xffffffffu, mbar_wait_abortable(smem_u32(&ctrl->empty[slot]), ((i / NST) & 1) ^ 1, abort_flag))) {
            ok = false;
            break;
          }
          const uint32_t bar = smem_u32(&ctrl->full[slot]);
          if (lane == 0) {
            if (kv == 0) ctrl->page_bad[c & 3] = badmask;
            mbar_arrive_expect_tx(bar, static_cast<uint32_t>(C::TILE_BYTES));
          }
          __syncwarp();
          if (h < C::HALVES)
            tma_load_4d(ring + slot * C::TILE_BYTES + h * C::HALF_BYTES + (j << P.bs_log2) * 128, kv ? &tmV : &tmK, h * 64, 0,
                        it.g, id, bar);
          issued = i + 1;
        }
        ++c;
      }
      done_item(k);
    }
    if (lane == 0) {
      if (any_bad) atomicOr(&P.hdr->err, ERR_BAD_PAGE);
      if (!ok) fail();
    }
    if (*reinterpret_cast<const volatile uint32_t*>(abort_flag)) {
      // given up: no copy may still be on its way into this CTA's shared memory when it ends
      for (int i = max(0, issued - NST); i < issued; ++i) mbar_wait(smem_u32(&ctrl->full[i % NST]), (i / NST) & 1);
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (nq[t] > 0) mbar_wait(smem_u32(&ctrl->q_full[t]), (nq[t] - 1) & 1);
    }
  } else if (warp == 8) {
    // ================= MMA issue (one thread)
    const PrefillItem* ip;
    int c = 0;                         // key tiles of this CTA so far
    int nq[2] = {0, 0}, np[2] = {0, 0};
    bool ok = true;
    constexpr uint32_t ID_S = umma_idesc(128, PF_KEYS, 0, 0);   // Q (K-major) x K tile (K-major)
    constexpr uint32_t ID_O = umma_idesc(128, D, 0, 1);         // P (tensor memory) x V tile (MN-major)
    const uint64_t q_desc = umma_desc(sQ, 16, 1024), k_desc = umma_desc(ring, 16, 1024),
                   v_desc = umma_desc(ring, C::HALF_BYTES, 1024);
    for (int k = 0; ok && get_item(k, ip); ++k) {
      const PrefillItem& it = *ip;
      if (lane == 0) {
        const int k1 = tiles_to(it);
        int prev = -1;
        bool first_pv[2] = {true, true}, first_s[2] = {true, true};
        auto wait = [&](uint64_t* bar, uint32_t parity) { ok = ok && mbar_wait_abortable(smem_u32(bar), parity, abort_flag); };
        for (int kt = tiles_from(it); ok; ++kt) {
          while (kt < k1 && !active(it, 0, kt) && !active(it, 1, kt)) ++kt;
          const bool cur = kt < k1;
          if (!cur && prev < 0) break;
          // ring positions: the previous tile is number c - 1, the present one number c
          const int vi = 2 * (c - 1) + 1, ki = 2 * c;
          bool v_seen = false, k_seen = false;
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (prev >= 0 && active(it, t, prev)) {
              if (!v_seen) wait(&ctrl->v_ok[(c - 1) & 3], ((c - 1) >> 2) & 1);
              v_seen = true;
              wait(&ctrl->p_full[t], np[t] & 1);
              ++np[t];
              if (!ok) break;
              tc_fence_after();
              const uint64_t vd = v_desc + static_cast<uint64_t>((vi % NST) * (C::TILE_BYTES >> 4));
              const uint32_t acc0 = first_pv[t] ? 0u : 1u;
              first_pv[t] = false;
#pragma unroll
              for (int ks = 0; ks < PF_KEYS / 16; ++ks)
                umma_ts(tbase + C::COL_O + t * D, tbase + C::COL_S + t * 128 + ks * 8, vd + static_cast<uint64_t>((ks * 2048) >> 4),
                        ID_O, ks ? 1u : acc0);
              tc_commit(smem_u32(&ctrl->pv_done[t]));
            }
            if (cur && active(it, t, kt)) {
              if (first_s[t]) {
                wait(&ctrl->q_full[t], nq[t] & 1);
                ++nq[t];
                first_s[t] = false;
              }
              if (!k_seen) wait(&ctrl->full[ki % NST], (ki / NST) & 1);
              k_seen = true;
              if (!ok) break;
              tc_fence_after();
              const uint64_t kd = k_desc + static_cast<uint64_t>((ki % NST) * (C::TILE_BYTES >> 4));
              const uint64_t qd = q_desc + static_cast<uint64_t>(t * (C::TILE_BYTES >> 4));
#pragma unroll
              for (int hh = 0; hh < C::HALVES; ++hh)
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) {
                  const uint64_t off = static_cast<uint64_t>((hh * C::HALF_BYTES + kk * 32) >> 4);
                  umma_ss(tbase + C::COL_S + t * 128, qd + off, kd + off, ID_S, (hh | kk) ? 1u : 0u);
                }
              tc_commit(smem_u32(&ctrl->s_full[t]));
              if (kt == it.end[t] - 1) tc_commit(smem_u32(&ctrl->q_free[t]));
            }
          }
          if (!ok) break;
          if (prev >= 0) tc_commit(smem_u32(&ctrl->empty[vi % NST]));
          if (!cur) break;
          tc_commit(smem_u32(&ctrl->empty[ki % NST]));
          prev = kt;
          ++c;
        }
      }
      ok = __shfl_sync(0xffffffffu, ok, 0);
      done_item(k);
    }
    if (lane == 0) {
      if (!ok) fail();
      // nothing of this thread may still be running on the tensor cores when the tensor memory goes back
      tc_commit(smem_u32(&ctrl->drained));
      mbar_wait(smem_u32(&ctrl->drained), 0);
    }
    __syncwarp();
  } else if (warp == 11) {
    // ================= guard of V
    const PrefillItem* ip;
    int c = 0;
    bool ok = true;
    for (int k = 0; ok && get_item(k, ip); ++k) {
      const PrefillItem& it = *ip;
      const int k1 = tiles_to(it);
      for (int kt = tiles_from(it); kt < k1; ++kt) {
        if (!active(it, 0, kt) && !active(it, 1, kt)) continue;
        const int i = 2 * c + 1;
        if (!__all_sync(0xffffffffu, mbar_wait_abortable(smem_u32(&ctrl->full[i % NST]), (i / NST) & 1, abort_flag))) {
          ok = false;
          break;
        }
        if (edge(it, kt)) {
          uint32_t bad[4] = {0u, 0u, 0u, 0u};
          const uint32_t base = ring + (i % NST) * C::TILE_BYTES;
          // a row of a 64-column block is 128 bytes = 8 chunks; four rows per warp-wide load
#pragma unroll 4
          for (int x = lane; x < C::TILE_BYTES / 16; x += 32) {
            uint32_t w[4];
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(base + x * 16));
            uint32_t hit = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool lo = (w[e] & 0x7f80u) == 0x7f80u, hi = (w[e] & 0x7f800000u) == 0x7f800000u;
              hit |= lo | hi;
              if (lo) w[e] &= 0xffff0000u;
              if (hi) w[e] &= 0x0000ffffu;
            }
            if (hit) {
              asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(base + x * 16), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
              const int key = (x >> 3) & 127;
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if ((key >> 5) == e) bad[e] |= 1u << (key & 31);
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            bad[e] = __reduce_or_sync(0xffffffffu, bad[e]);
            if (lane == 0) ctrl->v_bad[c & 3][e] = bad[e];
          }
          fence_proxy_async();         // the stores above before the tensor cores' reads
          __syncwarp();
        }
        if (lane == 0) mbar_arrive(smem_u32(&ctrl->v_ok[c & 3]));
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
    const float sc = P.scale_log2;
    // warp-uniform: tensor-memory accesses need the whole warp.  No thread leaves this path early: after a failed wait it
    // carries on, and its further waits return at once.
    auto wait_all = [&](uint64_t* bar, uint32_t parity) {
      if (!__all_sync(0xffffffffu, mbar_wait_abortable(smem_u32(bar), parity, abort_flag)) && lane == 0) fail();
    };
    const PrefillItem* ip;
    int c = 0, nt = 0;                 // key tiles of the CTA, of this tile
    for (int k = 0; get_item(k, ip); ++k) {
      const PrefillItem& it = *ip;
      const int my_begin = it.begin[t], my_end = it.end[t], my_lo = it.max_lo[t], my_hi = it.min_hi[t], my_rows = it.rows[t];
      const int j = it.tok0 + t * P.TQ + rj;            // token within the sequence
      const bool valid = rj < my_rows;
      int lo = 0, hi = 0;
      const int pos = it.L - it.n + j;
      if (valid) {
        const int2 v = prefill_interval(P, it.L, it.n, it.row0, P.prefix_lens ? __ldg(P.prefix_lens + it.s) : 0, j);
        lo = v.x;
        hi = v.y;
      }
      const float slope2 = (GEN && valid && P.slopes) ? -1.4426950408889634f * __ldg(P.slopes + it.g * P.G + rh) : 0.f;
      float m = NEG_INF, l = 0.f;
      int poison_from = INT_MAX, poison_to = -1;        // key tiles with a non-finite V that this row sees
      const int k1 = tiles_to(it);
      for (int kt = tiles_from(it); kt < k1; ++kt) {
        if (kt < my_begin || kt >= my_end) {
          if (active(it, t ^ 1, kt)) ++c;
          continue;
        }
        const int key0 = kt * PF_KEYS;
        wait_all(&ctrl->s_full[t], nt & 1);
        tc_fence_after();
        uint32_t raw_s[4][32];
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_ld32(tS + q * 32, raw_s[q]);
        tc_wait_ld();
        float s[128];
#pragma unroll
        for (int i = 0; i < 128; ++i) s[i] = __uint_as_float(raw_s[i >> 5][i & 31]);
        if (CAP) {
#pragma unroll
          for (int i = 0; i < 128; ++i) {
            // cap tanh(x / cap) = cap (1 - 2 / (1 + exp(2 x / cap))): exact to 2^-21 of the cap, at both ends too
            float rc;
            const float e = fast_exp2(s[i] * P.cap_k) + 1.f;
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rc) : "f"(e));
            s[i] = fmaf(-2.f * P.cap2, rc, P.cap2);
          }
        }
        if (GEN) {
          const float d0 = static_cast<float>(key0 - pos);
#pragma unroll
          for (int i = 0; i < 128; ++i) {
            const float x = CAP ? s[i] : s[i] * sc;
            s[i] = fmaf(slope2, fabsf(d0 + static_cast<float>(i)), x);
          }
        }
        const uint32_t pb = ctrl->page_bad[c & 3];
        if (pb) {
#pragma unroll
          for (int i = 0; i < 128; ++i)
            if ((pb >> (i >> P.bs_log2)) & 1u) s[i] = NEG_INF;
        }
        if (key0 < my_lo || key0 + PF_KEYS > my_hi) {
          const int a = lo - key0, b = hi - key0;
#pragma unroll
          for (int i = 0; i < 128; ++i)
            if (i < a || i >= b) s[i] = NEG_INF;
        }
        float m4[4] = {NEG_INF, NEG_INF, NEG_INF, NEG_INF};
#pragma unroll
        for (int i = 0; i < 128; i += 2) m4[(i >> 1) & 3] = max3(m4[(i >> 1) & 3], s[i], s[i + 1]);
        float mx = fmaxf(max3(m4[0], m4[1], m4[2]), m4[3]);
        constexpr bool SCALED = CAP || GEN;             // s is in base-2 units already
        if (!SCALED) mx = mx == NEG_INF ? NEG_INF : mx * sc;
        const bool first = kt == my_begin;
        const bool grow = first || mx > m + 8.f;
        const float m_new = grow ? fmaxf(m, mx) : m;
        const float mu = m_new == NEG_INF ? 0.f : m_new;
        const float alpha = grow ? fast_exp2(m - mu) : 1.f;
        m = m_new;
        if (__any_sync(0xffffffffu, !first && alpha != 1.f)) {
          // new reference: scale this row of O, once the product before this one is done
          wait_all(&ctrl->pv_done[t], (nt - 1) & 1);
          tc_fence_after();
#pragma unroll 1
          for (int q = 0; q < D / 32; ++q) {
            uint32_t o[32];
            tmem_ld32(tO + q * 32, o);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
            tmem_st32(tO + q * 32, o);
          }
        }
        uint64_t sum0 = 0ull, sum1 = 0ull;
        const uint64_t sc2 = pack_f32x2(sc, sc), mu2 = pack_f32x2(-mu, -mu);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint64_t x = pack_f32x2(s[q * 32 + 2 * i], s[q * 32 + 2 * i + 1]);
            float y0, y1;
            unpack_f32x2(SCALED ? add_f32x2(x, mu2) : fma_f32x2(x, sc2, mu2), y0, y1);
            const float p0 = fast_exp2(y0), p1 = fast_exp2(y1);
            const uint64_t pp = pack_f32x2(p0, p1);
            if (i & 1) sum1 = add_f32x2(sum1, pp);
            else sum0 = add_f32x2(sum0, pp);
            pk[i] = pack_bf16x2(p0, p1);
          }
          tmem_st16(tS + q * 16, pk);
        }
        {
          float a0, a1, b0, b1;
          unpack_f32x2(sum0, a0, a1);
          unpack_f32x2(sum1, b0, b1);
          l = l * alpha + ((a0 + a1) + (b0 + b1));
        }
        if (edge(it, kt)) {
          wait_all(&ctrl->v_ok[c & 3], (c >> 2) & 1);
          uint32_t seen = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int a = max(0, min(32, lo - key0 - 32 * e)), b = max(0, min(32, hi - key0 - 32 * e));
            const uint32_t vis = (b >= 32 ? 0xffffffffu : (1u << b) - 1u) & ~(a >= 32 ? 0xffffffffu : (1u << a) - 1u);
            seen |= *reinterpret_cast<volatile uint32_t*>(&ctrl->v_bad[c & 3][e]) & vis;
          }
          if (seen) {
            poison_from = min(poison_from, kt);
            poison_to = kt;
          }
        }
        tc_wait_st();
        tc_fence_before();
        mbar_arrive(smem_u32(&ctrl->p_full[t]));
        ++nt;
        ++c;
      }
      // ---- the item's rows
      if (my_rows > 0) {
        const bool any = my_begin != my_end;
        if (any) {
          wait_all(&ctrl->pv_done[t], (nt - 1) & 1);
          tc_fence_after();
        }
        const float inv = l > 0.f ? 1.f / l : (l != l ? l : 0.f);
        __nv_bfloat16* orow = P.out + (static_cast<int64_t>(it.row0 + j) * P.Hq + it.g * P.G + rh) * D;
#pragma unroll 1
        for (int q = 0; q < D / 32; ++q) {
          uint32_t o[32];
          if (any) {
            tmem_ld32(tO + q * 32, o);
            tc_wait_ld();
          }
          if (valid) {
            float v[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = any && inv != 0.f ? __uint_as_float(o[i]) * inv : 0.f;
            if (poison_to >= 0) add_guarded<D>(P, it.s, it.g, max(lo, poison_from * PF_KEYS), min(hi, (poison_to + 1) * PF_KEYS), q, v);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<uint4*>(orow + q * 32 + i * 8) =
                  make_uint4(pack_bf16x2(v[8 * i], v[8 * i + 1]), pack_bf16x2(v[8 * i + 2], v[8 * i + 3]),
                             pack_bf16x2(v[8 * i + 4], v[8 * i + 5]), pack_bf16x2(v[8 * i + 6], v[8 * i + 7]));
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

}  // namespace pdattn

// The accepted path of a tree of drafted tokens: accept_kernel moves the K and V of its tokens to the front of the tree's slots.
//
// Block (sequence, KV head).  Token i of the path comes from slot base + accepted[i] and goes to slot base + i.  The places overlap,
// so the block reads everything it moves into registers (at most 64 rows of K and of V), waits for itself and then writes.
// Bound: the launch and three dependent loads (length, path, page id): 256 sequences x 4 heads of 128 4.5 us, 48 x 8 over codes 4.0.
#pragma once

#include "common.cuh"

namespace pdattn {

constexpr int ACCEPT_THREADS = 256;
constexpr int ACCEPT_MAX = 64;        // tokens of a path

struct AcceptParams {
  uint8_t *k, *v;
  int64_t sb, sh, st;                 // strides in bytes (fp8: of the K pool; the V pool has pages [head][D][slot])
  const int32_t *table, *lens, *cu, *accepted, *counts;
  int32_t* err;                       // may be null
  int S, Hkv, MB, NB, bs, stride;     // stride: entries of a row of `accepted`
};

template <int D, bool FP8>
__global__ void __launch_bounds__(ACCEPT_THREADS)
accept_kernel(const __grid_constant__ AcceptParams P) {
  __shared__ int2 src[ACCEPT_MAX], dst[ACCEPT_MAX];        // (page, slot)
  const int s = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
  asm volatile("griddepcontrol.wait;" ::: "memory");       // a programmatic dependent of the kernel before it on the stream
  const int c0 = __ldg(P.cu + s), n = __ldg(P.cu + s + 1) - c0, L = __ldg(P.lens + s), a = __ldg(P.counts + s);
  if (a == 0) return;
  // every block of a sequence comes to the same answer: the sequence is moved as a whole or not at all
  int wrong = a < 0 || a > n || a > P.stride || a > ACCEPT_MAX || L < n ? ERR_BAD_SEQUENCE : 0;
  if (!wrong && tid < a) {
    const int j = __ldg(P.accepted + static_cast<int64_t>(s) * P.stride + tid);
    const int before = tid > 0 ? __ldg(P.accepted + static_cast<int64_t>(s) * P.stride + tid - 1) : -1;
    if (j <= before || j < 0 || j >= n) {
      wrong = ERR_BAD_SEQUENCE;
    } else {
      auto place = [&](int t) {
        const int b = t / P.bs;
        return make_int2(b < P.MB ? __ldg(P.table + static_cast<int64_t>(s) * P.MB + b) : -1, t - b * P.bs);
      };
      const int2 from = place(L - n + j), to = place(L - n + tid);
      src[tid] = from;
      dst[tid] = to;
      if (from.x < 0 || from.x >= P.NB || to.x < 0 || to.x >= P.NB) wrong = ERR_BAD_PAGE;
    }
  }
  if (__syncthreads_or(wrong)) {
    if (wrong && P.err && h == 0) atomicOr(P.err, wrong);
    return;
  }
  constexpr int RC = D * (FP8 ? 1 : 2) / 16;               // 16-byte pieces of a K row
  constexpr int PER = ACCEPT_MAX * RC / ACCEPT_THREADS;
  auto row = [&](uint8_t* pool, const int2& at, int piece) {
    return reinterpret_cast<uint4*>(pool + at.x * P.sb + h * P.sh + at.y * P.st) + piece;
  };
  uint4 k[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int i = (tid + e * ACCEPT_THREADS) / RC, piece = tid % RC;
    if (i < a) k[e] = *row(P.k, src[i], piece);
  }
  if constexpr (!FP8) {
    uint4 v[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = (tid + e * ACCEPT_THREADS) / RC, piece = tid % RC;
      if (i < a) v[e] = *row(P.v, src[i], piece);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = (tid + e * ACCEPT_THREADS) / RC, piece = tid % RC;
      if (i < a) {
        *row(P.k, dst[i], piece) = k[e];
        *row(P.v, dst[i], piece) = v[e];
      }
    }
  } else {
    // V: a token is a column of its page [D][slot]
    constexpr int ROWS = ACCEPT_THREADS / D, PV = ACCEPT_MAX / ROWS;
    const int dd = tid % D, i0 = tid / D;
    auto column = [&](const int2& at) {
      return P.v + (static_cast<int64_t>(at.x) * P.Hkv + h) * (D * P.bs) + dd * P.bs + at.y;
    };
    uint8_t v[PV];
#pragma unroll
    for (int e = 0; e < PV; ++e) {
      if (e * ROWS >= a) break;                            // (short paths pay for their own tokens only)
      if (i0 + e * ROWS < a) v[e] = *column(src[i0 + e * ROWS]);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = (tid + e * ACCEPT_THREADS) / RC, piece = tid % RC;
      if (i < a) *row(P.k, dst[i], piece) = k[e];
    }
#pragma unroll
    for (int e = 0; e < PV; ++e) {
      if (e * ROWS >= a) break;
      if (i0 + e * ROWS < a) *column(dst[i0 + e * ROWS]) = v[e];
    }
  }
}

}  // namespace pdattn

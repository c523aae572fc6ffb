// Page summaries and the choice of pages by them: summarize_kernel, select_kernel.
//
// Summary of a whole page for one KV head: the channelwise minimum and maximum of its keys as int8 codes that share a power of
// two, the smallest 2^e (-40 <= e <= 40) with max |k| <= 127 * 2^e; the minimum rounded down, the maximum up, so that
//   sum_i max(q_i lo_i, q_i hi_i) >= q . k   for every key of the page.
// Query heads are rounded to int8 with a power of two of their own (c_i), and
//   score(page) = max over the heads of the KV group of  2^(e_page + e_head) * sum_i max(c_i lo_i, c_i hi_i).
// The sum is an integer below 2^21 and the powers of two lose nothing, so a score is exact and the chosen pages are the same
// whatever the order of the sums, the renumbering of the pages or the split of the work.
//
// Bound: summarize_kernel by the keys it reads once (a warp per page-head, 16-byte loads, packed minima and maxima); select_kernel
// by the 2 d + 1 bytes it reads per page-head.  The products run on int8 MMAs straight from global memory: a lane's 16-byte loads
// are fragments of two MMAs when the contraction index is permuted alike in both operands, so nothing passes through shared
// memory.  The block that finishes a (sequence, KV head) last picks its pages: no second launch.
//
// Times (replays of a graph): summaries of 12 prompts of 700 to 2100 tokens (8 heads of 128, pages of 16, 38 MB) 9.5 us, of the pages
// that 256 single tokens fill 3.7 us (the launch and three dependent loads); 128 of up to 2048 pages for 48 sequences x 8 KV heads (100 MB)
// 24.6 us, of which 17 are scores (a warp's 16 pages take 2 us, most of it latency), 1.5 the tickets and 4 the choice of the last units;
// 6 sequences x 4 KV heads of up to 250 pages 6.4 us (latency of one block).  Equal parts for a unit's blocks: 25.5 instead of 24.6.
#pragma once

#include <climits>
#include <type_traits>

#include <cuda_fp16.h>

#include "common.cuh"

namespace pdattn {

constexpr int SUM_EXP_MIN = -40, SUM_EXP_MAX = 40;   // exponents of codes
constexpr int SUM_EXP_ODD = 127;                     // a page with a key that is not finite: always chosen first

struct SummaryParams {
  const void* k;                 // bf16 cache, or the code pool of the fp8 cache
  int64_t sb, sh, st;            // strides in elements
  const float* k_scale;          // fp8 cache only
  int8_t *codes, *exps;          // [page][head][min, max][d], [page][head]
  const int32_t *table, *lens;   // pages filled by the last tokens of the sequences ...
  const int32_t* cu;             // null: one token each
  const int32_t* pages;          // ... or the pages of a list
  int32_t* err;                  // may be null
  int S, Hkv, MB, NB, bs, n;     // n: entries of the list, or new tokens
};

// The smallest e within the limits with a <= 127 * 2^e: a = m 2^k with 1 <= m < 2, and 127 = 1.984375 * 2^6.
__device__ __forceinline__ int summary_exponent(float a) {
  const uint32_t u = __float_as_uint(a);
  const int e = static_cast<int>(u >> 23) - 127 - 6 + ((u & 0x7fffffu) > 0x7e0000u ? 1 : 0);
  return max(SUM_EXP_MIN, min(SUM_EXP_MAX, e));
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(static_cast<uint32_t>(127 + e) << 23); }
__device__ __forceinline__ uint32_t code_byte(float x) {   // x: a whole number
  return static_cast<uint32_t>(static_cast<int>(fminf(fmaxf(x, -127.f), 127.f))) & 0xffu;
}

// A warp per page-head.  A row of D elements takes LR lanes of 16 bytes; the warp reads 32 / LR rows at a time.
template <int D, bool FP8>
__device__ __forceinline__ void summarize_page(const SummaryParams& P, int page, int h, int lane) {
  constexpr int EB = FP8 ? 1 : 2, LR = D * EB / 16, ROWS = 32 / LR, E = 16 / EB;
  const int col = lane % LR, row0 = lane / LR;
  const uint8_t* base = static_cast<const uint8_t*>(P.k) + (page * P.sb + h * P.sh + row0 * P.st) * EB + col * 16;
  const int64_t step = ROWS * P.st * EB;
  // packed running extremes: bf16 pairs as they are, e4m3 codes widened to fp16 (exact)
  using V2 = typename std::conditional<FP8, __half2, __nv_bfloat162>::type;
  constexpr int NV = E / 2;
  V2 lo[NV], hi[NV];
  uint32_t odd = 0u;
  auto take = [&](const uint4& w, bool first) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      uint32_t x;
      if constexpr (FP8) {
        x = cvt_e4m3x2_f16x2(u[i >> 1] >> (16 * (i & 1)));
        odd |= (x & 0x7c007c00u) + 0x04000400u;     // all exponent bits set carry into the sign's place
      } else {
        x = u[i];
        odd |= (x & 0x7f807f80u) + 0x00800080u;
      }
      const V2 v = *reinterpret_cast<const V2*>(&x);
      lo[i] = first ? v : __hmin2(lo[i], v);
      hi[i] = first ? v : __hmax2(hi[i], v);
    }
  };
  take(__ldg(reinterpret_cast<const uint4*>(base)), true);
#pragma unroll 8
  for (int r = ROWS; r < P.bs; r += ROWS) take(__ldg(reinterpret_cast<const uint4*>(base + (r / ROWS) * step)), false);
#pragma unroll
  for (int o = LR; o < 32; o <<= 1)
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      lo[i] = __hmin2(lo[i], __shfl_xor_sync(0xffffffffu, lo[i], o));
      hi[i] = __hmax2(hi[i], __shfl_xor_sync(0xffffffffu, hi[i], o));
    }
  float a[E], b[E], top = 0.f;
  const float sc = FP8 ? __ldg(P.k_scale + h) : 1.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float2 x, y;
    if constexpr (FP8) {
      x = __half22float2(lo[i]);
      y = __half22float2(hi[i]);
      x.x *= sc, x.y *= sc, y.x *= sc, y.y *= sc;
    } else {
      x = __bfloat1622float2(lo[i]);
      y = __bfloat1622float2(hi[i]);
    }
    a[2 * i] = fminf(x.x, y.x), a[2 * i + 1] = fminf(x.y, y.y);      // (a negative scale swaps them)
    b[2 * i] = fmaxf(x.x, y.x), b[2 * i + 1] = fmaxf(x.y, y.y);
#pragma unroll
    for (int e = 2 * i; e < 2 * i + 2; ++e) {
      top = fmaxf(top, fmaxf(fabsf(a[e]), fabsf(b[e])));
      if (FP8 && !(fabsf(a[e]) <= 3.4e38f && fabsf(b[e]) <= 3.4e38f)) odd |= 0x8000u;   // (a scale that is not finite)
    }
  }
  const bool any_odd = __any_sync(0xffffffffu, (odd & 0x80008000u) != 0);
  top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
  const int e = summary_exponent(top);
  const float inv = any_odd ? 0.f : power_of_two(-e);
  if (row0 == 0) {
    uint32_t wl[E / 4], wh[E / 4];
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      wl[i] = wh[i] = 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // (a product may vanish in 32 bits beside keys that are far larger; its bound does not)
        const float x = a[4 * i + j], y = b[4 * i + j];
        const float down = fminf(floorf(x * inv), x < 0.f ? -1.f : 127.f), up = fmaxf(ceilf(y * inv), y > 0.f ? 1.f : -127.f);
        wl[i] |= (any_odd ? 0u : code_byte(down)) << (8 * j);
        wh[i] |= (any_odd ? 0u : code_byte(up)) << (8 * j);
      }
    }
    const int64_t at = static_cast<int64_t>(page) * P.Hkv + h;
    uint32_t* out = reinterpret_cast<uint32_t*>(P.codes + at * (2 * D)) + col * (E / 4);
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      out[i] = wl[i];
      out[D / 4 + i] = wh[i];
    }
    if (lane == 0) P.exps[at] = static_cast<int8_t>(any_odd ? SUM_EXP_ODD : e);
  }
}

// Block i: entry i of the list, or slot i of the sequences' filled pages.  Sequence s owns the slots from cu[s] / bs + s on: n new
// tokens fill at most n / bs + 1 pages, so they are enough without a prefix sum.
template <int D, bool FP8>
__global__ void __launch_bounds__(256)
summarize_kernel(const __grid_constant__ SummaryParams P) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int slot = blockIdx.x;
  asm volatile("griddepcontrol.wait;" ::: "memory");   // a programmatic dependent of the kernel before it on the stream
  int page;
  if (P.pages) {
    page = __ldg(P.pages + slot);
    if (page < 0) return;                              // (an entry that names no page)
  } else {
    int s = slot, n = 1, k = 0;
    if (P.cu) {
      // (tokens past the call's number are left out, with the sequences they belong to)
      if (slot == 0 && threadIdx.x == 0 && P.err && __ldg(P.cu + P.S) > P.n) atomicOr(P.err, ERR_BAD_SEQUENCE);
      int lo = 0, len = P.S;                           // the last sequence whose first slot is at or before this one
      while (len > 1) {
        const int step = (len + 31) / 32, i = lane * step;
        const bool below = i < len && __ldg(P.cu + lo + i) / P.bs + lo + i <= slot;
        const uint32_t m = __ballot_sync(0xffffffffu, below);
        const int b = m ? 31 - __clz(m) : 0;
        lo += b * step;
        len = min(step, len - b * step);
      }
      s = lo;
      const int c0 = __ldg(P.cu + s), c1 = __ldg(P.cu + s + 1);
      n = c1 - c0;
      k = slot - (c0 / P.bs + s);
      if (n <= 0 || k < 0 || c1 > P.n) return;
    }
    const int L = __ldg(P.lens + s);
    if (L <= 0) return;
    const int64_t b = static_cast<int64_t>(max(0, L - n) / P.bs) + k;
    if (b >= L / P.bs) return;
    page = b < P.MB ? __ldg(P.table + static_cast<int64_t>(s) * P.MB + b) : -1;
  }
  if (page < 0 || page >= P.NB) {
    if (P.err && threadIdx.x == 0) atomicOr(P.err, ERR_BAD_PAGE);
    return;
  }
  for (int h = warp; h < P.Hkv; h += warps) summarize_page<D, FP8>(P, page, h, lane);
}

// ------------------------------------------------------------------------------------------
// Selection
// ------------------------------------------------------------------------------------------
struct SelectParams {
  const __nv_bfloat16* q;         // [S, Hq, D]
  const int8_t *codes, *exps;
  const int32_t *table, *lens;
  int32_t* selected;              // [S, Hkv, K]
  uint32_t* keys;                 // [S * Hkv, MB] order-preserving keys of the scores
  int32_t* tickets;               // [S * Hkv] blocks that have written their keys; zero between calls
  int32_t* err;
  int S, Hq, Hkv, G, MB, NB, bs, K, first, recent;
  int chunk, chunks;              // pages scored by a block; blocks of a unit
};

constexpr int SEL_THREADS = 256;

// larger scores have larger keys
__device__ __forceinline__ uint32_t score_key(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ void mma_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Exclusive sum over the block of v in the threads' order.
template <class T>
__device__ __forceinline__ T block_exclusive(T v, T* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  T run = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T y = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += y;
  }
  if (lane == 31) warp_sums[warp] = run;
  __syncthreads();
  T before = run - v;
#pragma unroll
  for (int w = 0; w < SEL_THREADS / 32; ++w) before += w < warp ? warp_sums[w] : T(0);
  return before;
}

// The R largest of M keys, ties to the lower index, as ascending page numbers out[0 .. R).  Thread t owns the indices t * each ..
// + each - 1, in registers up to E of them (E = 0: read again in every round).  Keys that this block has just written lie in its shared
// memory.  The R-th largest key is found eight bits at a time, from the highest in which the keys differ: a histogram of the keys that
// agree with it so far, and the bin in which the count from above reaches R, until all of a bin is wanted.  (Bit by bit, with 32
// counts, 2048 keys took 2.5 us longer; without the early end 0.6.)
struct SelectScratch {
  int bins[2][256];
  int warp_counts[SEL_THREADS / 32];
  unsigned long long warp_sums[SEL_THREADS / 32];
  uint32_t ends[2], digit;
  int left, in_bin;
};
static_assert(SEL_THREADS == 256, "a thread per bin");
// (A function of its own: inlined, its registers slowed the scoring loop, 25.5 -> 31 us for 48 sequences to 32,768 tokens.)
template <int E, bool SHARED>
__device__ __noinline__ void take_largest(const uint32_t* keys, int M, int R, int first, int32_t* out, SelectScratch* sh) {
  const int tid = threadIdx.x, lane = tid & 31;
  const int each = E > 0 ? E : (M + SEL_THREADS - 1) / SEL_THREADS;
  const int i0 = tid * each;
  const int mine = max(0, min(each, M - i0));
  auto read = [&](int j) { return SHARED ? keys[i0 + j] : __ldcg(keys + i0 + j); };
  uint32_t x[E > 0 ? E : 1] = {};
  if constexpr (E > 0) {
#pragma unroll
    for (int j = 0; j < E; ++j) x[j] = j < mine ? read(j) : 0u;
  }
  // f(index in the thread's share, key) for all of them
  auto each_key = [&](auto f) {
    if constexpr (E > 0) {
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (j < mine) f(j, x[j]);
    } else {
#pragma unroll 4
      for (int j = 0; j < mine; ++j) f(j, read(j));
    }
  };
  uint32_t largest = 0u, least = 0xffffffffu;
  each_key([&](int, uint32_t k) {
    largest = max(largest, k);
    least = min(least, k);
  });
  if (tid == 0) {
    sh->ends[0] = 0u;
    sh->ends[1] = 0xffffffffu;
  }
  sh->bins[0][tid] = 0;
  __syncthreads();
  largest = __reduce_max_sync(0xffffffffu, largest);
  least = __reduce_min_sync(0xffffffffu, least);
  if (lane == 0) {
    atomicMax(&sh->ends[0], largest);
    atomicMin(&sh->ends[1], least);
  }
  __syncthreads();
  const uint32_t differ = sh->ends[0] ^ sh->ends[1];
  int low = differ ? 32 - __clz(differ) : 0;            // bits below this one are still to be found
  uint32_t t = low >= 32 ? 0u : sh->ends[1] >> low << low;
  int want = R;                                         // of the keys that agree with t in the bits from `low` on
  for (int turn = 0; low > 0; turn ^= 1) {
    const int shift = max(0, low - 8), bits = low - shift;
    each_key([&](int, uint32_t k) {
      if (low >= 32 || (k >> low) == (t >> low)) atomicAdd(&sh->bins[turn][(k >> shift) & ((1u << bits) - 1u)], 1);
    });
    __syncthreads();
    // thread i looks at bin 255 - i: keys in larger bins come before
    const int n = sh->bins[turn][255 - tid];
    sh->bins[turn ^ 1][tid] = 0;
    const int above = block_exclusive(n, sh->warp_counts);
    if (above < want && above + n >= want) {
      sh->digit = static_cast<uint32_t>(255 - tid);
      sh->left = want - above;
      sh->in_bin = n;
    }
    __syncthreads();
    t |= sh->digit << shift;
    want = sh->left;
    low = shift;
    if (want == sh->in_bin) break;                      // all of the bin: the bits below do not matter
  }
  t >>= low;                                            // (low < 32)
  // keys above t, and `want` of those equal to it in order: both counts scanned as one 64-bit word
  int gt = 0, eq = 0;
  each_key([&](int, uint32_t k) {
    gt += (k >> low) > t ? 1 : 0;
    eq += (k >> low) == t ? 1 : 0;
  });
  const unsigned long long before =
      block_exclusive((static_cast<unsigned long long>(gt) << 32) | static_cast<unsigned>(eq), sh->warp_sums);
  int g = static_cast<int>(before >> 32), q = static_cast<int>(before & 0xffffffffull);
  each_key([&](int j, uint32_t k) {
    k >>= low;
    if (k > t || (k == t && q < want)) out[g + min(q, want)] = first + i0 + j;
    if (k > t) ++g;
    if (k == t) ++q;
  });
}

constexpr int SEL_OWN = 2048;     // keys that a block which has a unit to itself keeps in shared memory
template <int D, int NT>   // NT: groups of 8 query heads
__global__ void __launch_bounds__(SEL_THREADS, NT == 1 ? 4 : 2)
select_kernel(const __grid_constant__ SelectParams P) {
  constexpr int RB = 2 * D, NI = RB / 64;
  __shared__ __align__(16) int8_t qc[8 * NT][RB];
  __shared__ int qe[8 * NT];
  __shared__ SelectScratch scratch;
  __shared__ int is_last;
  __shared__ uint32_t own_keys[SEL_OWN];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int unit = blockIdx.x / P.chunks, chunk = blockIdx.x - unit * P.chunks;
  const int s = unit / P.Hkv, g = unit - s * P.Hkv;
  asm volatile("griddepcontrol.wait;" ::: "memory");   // a programmatic dependent of the kernel before it on the stream
  const int L = max(0, __ldg(P.lens + s));
  int nb = L > 0 ? (L - 1) / P.bs + 1 : 0;
  if (nb > P.MB) {                                     // tokens past the end of the table row: left out
    if (chunk == 0 && tid == 0) atomicOr(P.err, ERR_BAD_PAGE);
    nb = P.MB;
  }
  int32_t* out = P.selected + static_cast<int64_t>(unit) * P.K;
  const int R = P.K - P.first - P.recent;              // pages taken by their score
  if (nb <= P.K || R == 0) {
    if (chunk == 0)
      for (int i = tid; i < P.K; i += SEL_THREADS)
        out[i] = nb > P.K ? (i < P.first ? i : nb - P.K + i) : i < nb ? i : -1;
    return;
  }
  const int M = nb - P.first - P.recent;               // pages with a score (M > R)
  const int i0 = chunk * P.chunk;
  if (i0 >= M) return;
  const int i1 = min(M, i0 + P.chunk);
  // ids of a warp's 16 pages, a round ahead of their use
  constexpr int STEP = SEL_THREADS / 32 * 16;          // pages of a round of the block
  const int32_t* row = P.table + static_cast<int64_t>(s) * P.MB + P.first;
  auto page_of = [&](int b0) {
    const int i = b0 + (lane & 15);
    return i < i1 ? __ldg(row + i) : 0;
  };
  int next_id = page_of(i0 + warp * 16);

  // ---- the group's query heads as codes: the parts below zero against the minima, the others against the maxima
  for (int h = warp; h < 8 * NT; h += SEL_THREADS / 32) {
    float x[D / 32];
    float top = 0.f;
    bool odd = false;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      x[j] = h < P.G ? __bfloat162float(P.q[(static_cast<int64_t>(s) * P.Hq + g * P.G + h) * D + j * 32 + lane]) : 0.f;
      odd |= !(fabsf(x[j]) <= 3.4e38f);
      top = fmaxf(top, fabsf(x[j]));
    }
    odd = __any_sync(0xffffffffu, odd);
    top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
    const int e = summary_exponent(top);
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      const int c = odd ? 0 : static_cast<int>(fminf(fmaxf(rintf(x[j] * power_of_two(-e)), -127.f), 127.f));
      qc[h][j * 32 + lane] = static_cast<int8_t>(min(c, 0));
      qc[h][D + j * 32 + lane] = static_cast<int8_t>(max(c, 0));
    }
    if (lane == 0) qe[h] = odd || h >= P.G ? INT_MIN : e;
  }
  __syncthreads();

  // ---- scores, 16 pages a warp at a time
  const int r = lane >> 2, c = lane & 3;
  uint4 bq[NT][NI];
  float pe[NT][2];                                     // 2^e of this lane's two columns, or -1: takes no part
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int i = 0; i < NI; ++i) bq[nt][i] = *reinterpret_cast<const uint4*>(&qc[nt * 8 + r][64 * i + 16 * c]);
#pragma unroll
    for (int e = 0; e < 2; ++e) pe[nt][e] = qe[nt * 8 + 2 * c + e] == INT_MIN ? -1.f : power_of_two(qe[nt * 8 + 2 * c + e]);
  }
  const float NEG_INF = __int_as_float(0xff800000);
  uint32_t* keys = P.keys + static_cast<int64_t>(unit) * P.MB;
  const bool own = M <= P.chunk && M <= SEL_OWN;       // no other block scores for this unit
  bool bad = false;
  for (int b0 = i0 + warp * 16; b0 < i1; b0 += STEP) {
    int id = next_id;
    next_id = page_of(b0 + STEP);
    const bool gone = id < 0 || id >= P.NB;
    bad |= gone;
    if (gone) id = -1;
    int ids[2], ek[2];
    uint4 v[2][NI];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      ids[half] = __shfl_sync(0xffffffffu, id, r + 8 * half);
      const int64_t at = static_cast<int64_t>(max(0, ids[half])) * P.Hkv + g;
#pragma unroll
      for (int j = 0; j < NI; ++j) v[half][j] = __ldg(reinterpret_cast<const uint4*>(P.codes + at * RB + 64 * j + 16 * c));
      ek[half] = __ldg(P.exps + at);
    }
    float best[2] = {NEG_INF, NEG_INF};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      int acc[4] = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        mma_s8(acc, v[0][j].x, v[1][j].x, v[0][j].y, v[1][j].y, bq[nt][j].x, bq[nt][j].y);
        mma_s8(acc, v[0][j].z, v[1][j].z, v[0][j].w, v[1][j].w, bq[nt][j].z, bq[nt][j].w);
      }
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (pe[nt][e] > 0.f)
            best[half] = fmaxf(best[half], static_cast<float>(acc[2 * half + e]) * pe[nt][e] * power_of_two(min(ek[half], SUM_EXP_MAX)));
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      best[half] = fmaxf(best[half], __shfl_xor_sync(0xffffffffu, best[half], 1));
      best[half] = fmaxf(best[half], __shfl_xor_sync(0xffffffffu, best[half], 2));
      if (ek[half] == SUM_EXP_ODD) best[half] = __int_as_float(0x7f800000);
      const int at = b0 + r + 8 * half;
      if (c == 0 && at < i1) {
        const uint32_t key = ids[half] < 0 ? 1u : score_key(best[half]);
        if (own) own_keys[at] = key;
        else __stcg(keys + at, key);
      }
    }
  }
  if (bad) atomicOr(P.err, ERR_BAD_PAGE);

  // ---- the block that comes last takes the unit's pages
  const int blocks = (M + P.chunk - 1) / P.chunk;
  __syncthreads();
  if (blocks > 1) {
    if (tid == 0) {
      int k;
      // (release: this block's keys; acquire: those of the others)
      asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(k) : "l"(P.tickets + unit) : "memory");
      is_last = k == blocks - 1;
      if (is_last) P.tickets[unit] = 0;
    }
    __syncthreads();
    if (!is_last) return;
  }
  for (int i = tid; i < P.first; i += SEL_THREADS) out[i] = i;
  for (int i = tid; i < P.recent; i += SEL_THREADS) out[P.first + R + i] = nb - P.recent + i;
  static_assert(SEL_OWN == SEL_THREADS * 8, "eight keys a thread");
  if (own) take_largest<8, true>(own_keys, M, R, P.first, out + P.first, &scratch);
  else if (M <= SEL_THREADS * 8) take_largest<8, false>(keys, M, R, P.first, out + P.first, &scratch);
  else take_largest<0, false>(keys, M, R, P.first, out + P.first, &scratch);
}

}  // namespace pdattn

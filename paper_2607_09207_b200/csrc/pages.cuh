// Page bookkeeping on the device: which pages of the pool are free, how often each is referenced, and the copies
// that forking and compacting need.
//
// The books are three arrays: ref_counts[p] = references to page p from block-table rows, free_list = the pages with
// none in DESCENDING id (the lowest id is on top, entries at or past free_count are -1), free_count.  This state is a
// function of the reference counts alone, so every operation leaves the same books whatever order its threads ran in.
//
// Bound: the table operations by launches and dependent loads (one block scans the request, a block per row does the
// rows), the rebuild of the free list by one pass over the counts (a cluster of blocks, counts exchanged through
// distributed shared memory, no waiting between launches), the copies by bytes (each page read once, written once).
#pragma once

#include <cooperative_groups.h>

#include "common.cuh"

namespace pdattn {

struct PagePool {
  int32_t *ref, *free_list, *free_count;
  int NB;
};
// Scratch behind the cleared part of the workspace
struct PagesScratch {
  int32_t* err;        // the workspace's sticky error word
  int32_t* head;       // [0]: fork accepted
  int32_t* lens;       // [S] fork: parent lengths
  int32_t* tails;      // [S] fork: page of the child's partial tail, -1 = none
  int32_t* map;        // [NB] compact: new id of page p, -1: nothing references it
};

constexpr int kPagesThreads = 1024;

__device__ __forceinline__ int block_scan_excl(int v, int* warp_sums, int* total) {   // kPagesThreads threads
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sums[wid] = x;
  __syncthreads();
  if (wid == 0) {
    int w = warp_sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += y;
    }
    warp_sums[lane] = w;
  }
  __syncthreads();
  const int excl = x - v + (wid > 0 ? warp_sums[wid - 1] : 0);
  *total = warp_sums[31];
  __syncthreads();
  return excl;
}

__global__ void __launch_bounds__(256)
pages_init_kernel(PagePool pool) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < pool.NB) {
    pool.ref[i] = 0;
    pool.free_list[i] = pool.NB - 1 - i;
  }
  if (i == 0) *pool.free_count = pool.NB;
}

// Whether the `need` topmost entries of the free list are page ids (they always are unless the books were overwritten).
__device__ __forceinline__ bool pages_on_top_valid(const PagePool& pool, int count, int need) {
  bool ok = true;
  for (int r = threadIdx.x; r < need; r += kPagesThreads) {
    const int id = pool.free_list[count - 1 - r];
    ok &= id >= 0 && id < pool.NB;
  }
  return __syncthreads_and(ok) != 0;
}

// ------------------------------------------------------------------------------------------
// Reserve: pages for new_tokens[s] further tokens of every sequence, taken in sequence order, and the lengths
// advanced.  All or nothing: when the pool holds too few pages no row changes.
// ------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(kPagesThreads)
pages_reserve_kernel(PagePool pool, int32_t* __restrict__ table, int32_t* __restrict__ lens,
                     const int32_t* __restrict__ new_tokens, int S, int MB, int bs, int32_t* err) {
  __shared__ int warp_sums[32];
  __shared__ int first[kPagesThreads], from[kPagesThreads], count_of[kPagesThreads];
  __shared__ unsigned long long wanted;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t room = min(static_cast<int64_t>(MB) * bs, static_cast<int64_t>(INT32_MAX));   // (lengths are int32)
  auto request = [&](int s, int& L, int& n) {     // pages the sequence needs; n = tokens granted
    L = lens[s];
    n = new_tokens[s];
    if (L < 0 || n < 0 || static_cast<int64_t>(L) + n > room) {
      n = 0;
      return -1;
    }
    return static_cast<int>((static_cast<int64_t>(L) + n + bs - 1) / bs - (static_cast<int64_t>(L) + bs - 1) / bs);
  };
  const int count = *pool.free_count;
  // The request's total in 64 bits: 1024 rows of a wide table can ask for more pages than 32 hold.  What is granted below is at
  // most the pool, so the sums there fit.
  unsigned long long mine = 0;
  for (int s = tid; s < S; s += kPagesThreads) {
    int L, n;
    const int need = request(s, L, n);
    if (need < 0) atomicOr(err, ERR_BAD_SEQUENCE);   // left as it is; the others are served
    else mine += need;
  }
  if (tid == 0) wanted = 0;
  __syncthreads();
  if (mine > 0) atomicAdd(&wanted, mine);
  __syncthreads();
  const int64_t total = static_cast<int64_t>(wanted);
  if (total > count || count > pool.NB) {
    if (tid == 0) atomicOr(err, ERR_OUT_OF_PAGES);
    return;
  }
  if (!pages_on_top_valid(pool, count, static_cast<int>(total))) {
    if (tid == 0) atomicOr(err, ERR_BAD_PAGE);
    return;
  }
  int taken = 0;
  for (int base = 0; base < S; base += kPagesThreads) {
    int L = 0, n = 0, need = 0;
    if (base + tid < S) need = max(0, request(base + tid, L, n));
    int sum;
    const int excl = block_scan_excl(need, warp_sums, &sum);
    first[tid] = taken + excl;
    from[tid] = static_cast<int>((static_cast<int64_t>(L) + bs - 1) / bs);
    count_of[tid] = need;
    if (n > 0) lens[base + tid] = L + n;
    __syncthreads();
    for (int k = warp; k < min(kPagesThreads, S - base); k += kPagesThreads / 32) {   // a warp per row
      const int f = first[k], c0 = from[k];
      for (int j = lane; j < count_of[k]; j += 32) {
        const int at = count - 1 - (f + j);
        const int id = pool.free_list[at];
        pool.free_list[at] = -1;
        pool.ref[id] = 1;
        table[static_cast<int64_t>(base + k) * MB + c0 + j] = id;
      }
    }
    taken += sum;
    __syncthreads();
  }
  if (tid == 0) *pool.free_count = count - taken;
}

// ------------------------------------------------------------------------------------------
// Fork, first part (one block): checks the request, hands every child with a partial tail page a page of its own, and
// writes the copies that fill those pages.  Refused as a whole: a row out of range, a child that is not empty or
// named twice, a bad tail page, too few free pages.
// ------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(kPagesThreads)
pages_fork_kernel(PagePool pool, const int32_t* __restrict__ table, int32_t* __restrict__ lens,
                  const int32_t* __restrict__ parents, const int32_t* __restrict__ children, int n, int S, int MB, int bs,
                  int32_t* __restrict__ copy_src, int32_t* __restrict__ copy_dst, PagesScratch X) {
  __shared__ int warp_sums[32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tid = threadIdx.x;
  const int64_t room = static_cast<int64_t>(MB) * bs;
  const int count = *pool.free_count;
  // the parents' lengths, before any child's is touched
  bool ok = true;
  int total = 0;
  for (int base = 0; base < n; base += kPagesThreads) {
    int tail = 0;
    if (base + tid < n) {
      const int p = parents[base + tid], c = children[base + tid];
      bool good = p >= 0 && p < S && c >= 0 && c < S;
      int L = 0;
      if (good) {
        L = lens[p];
        good = L >= 0 && L <= room && lens[c] == 0;
        tail = good && L % bs != 0;
        if (tail) {
          const int id = table[static_cast<int64_t>(p) * MB + L / bs];
          if (id < 0 || id >= pool.NB) good = false;
        }
      }
      X.lens[base + tid] = L;
      ok &= good;
    }
    int sum;
    block_scan_excl(tail, warp_sums, &sum);
    total += sum;
  }
  ok = __syncthreads_and(ok) != 0;
  int bits = ok ? 0 : ERR_BAD_SEQUENCE;
  if (ok) {
    // claim the children: a row named twice is claimed twice
    bool mine = true;
    for (int i = tid; i < n; i += kPagesThreads) mine &= atomicCAS(lens + children[i], 0, -1) == 0;
    ok = __syncthreads_and(mine) != 0;
    if (!ok) bits = ERR_BAD_SEQUENCE;
    else if (total > count || count > pool.NB) bits = ERR_OUT_OF_PAGES;
    else if (!pages_on_top_valid(pool, count, total)) bits = ERR_BAD_PAGE;
    if (bits) {
      __syncthreads();
      for (int i = tid; i < n; i += kPagesThreads) lens[children[i]] = 0;   // every one of them was empty
    }
  }
  if (bits) {
    for (int i = tid; i < n; i += kPagesThreads) copy_src[i] = copy_dst[i] = -1;
    if (tid == 0) {
      atomicOr(X.err, bits);
      X.head[0] = 0;
    }
    return;
  }
  int taken = 0;
  for (int base = 0; base < n; base += kPagesThreads) {
    int tail = 0, L = 0, p = 0;
    if (base + tid < n) {
      p = parents[base + tid];
      L = X.lens[base + tid];
      tail = L % bs != 0;
    }
    int sum;
    const int rank = taken + block_scan_excl(tail, warp_sums, &sum);
    if (base + tid < n) {
      int id = -1;
      if (tail) {
        const int at = count - 1 - rank;
        id = pool.free_list[at];
        pool.free_list[at] = -1;
        pool.ref[id] = 1;
        copy_src[rank] = table[static_cast<int64_t>(p) * MB + L / bs];
        copy_dst[rank] = id;
      }
      X.tails[base + tid] = id;
      lens[children[base + tid]] = L;
    }
    taken += sum;
  }
  for (int i = taken + tid; i < n; i += kPagesThreads) copy_src[i] = copy_dst[i] = -1;
  if (tid == 0) {
    *pool.free_count = count - taken;
    X.head[0] = 1;
  }
}

// Fork, second part: block i writes child i's row -- the parent's whole pages, each with one more reference, then the
// child's own tail page, then -1.
__global__ void __launch_bounds__(128)
pages_fork_rows_kernel(PagePool pool, int32_t* __restrict__ table, const int32_t* __restrict__ parents,
                       const int32_t* __restrict__ children, int MB, int bs, PagesScratch X) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (X.head[0] == 0) return;
  const int i = blockIdx.x;
  const int L = X.lens[i], whole = L / bs, tail = X.tails[i];
  const int32_t* from = table + static_cast<int64_t>(parents[i]) * MB;
  int32_t* to = table + static_cast<int64_t>(children[i]) * MB;
  for (int b = threadIdx.x; b < MB; b += blockDim.x) {
    int id = -1;
    if (b < whole) {
      id = from[b];
      if (id >= 0 && id < pool.NB) atomicAdd(pool.ref + id, 1);
      else atomicOr(X.err, ERR_BAD_PAGE);
    } else if (b == whole) {
      id = tail;
    }
    to[b] = id;
  }
}

// ------------------------------------------------------------------------------------------
// Free, first part: block i takes the references of sequence seqs[i] back and empties its row.  The length is
// exchanged for 0, so a sequence that is named twice is freed once.
// ------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(128)
pages_free_kernel(PagePool pool, int32_t* __restrict__ table, int32_t* __restrict__ lens,
                  const int32_t* __restrict__ seqs, int S, int MB, int bs, int32_t* err) {
  __shared__ int len;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int s = seqs[blockIdx.x];
  if (s < 0 || s >= S) {
    if (threadIdx.x == 0) atomicOr(err, ERR_BAD_SEQUENCE);
    return;
  }
  if (threadIdx.x == 0) len = atomicExch(lens + s, 0);
  __syncthreads();
  const int L = len;
  if (L <= 0) {
    if (L < 0 && threadIdx.x == 0) atomicOr(err, ERR_BAD_SEQUENCE);
    return;
  }
  const int64_t need = (static_cast<int64_t>(L) + bs - 1) / bs;
  const int np = static_cast<int>(need < MB ? need : MB);
  if (need > MB && threadIdx.x == 0) atomicOr(err, ERR_BAD_SEQUENCE);
  int32_t* row = table + static_cast<int64_t>(s) * MB;
  for (int b = threadIdx.x; b < MB; b += blockDim.x) {
    if (b < np) {
      const int id = row[b];
      bool good = id >= 0 && id < pool.NB;
      if (good && atomicSub(pool.ref + id, 1) <= 0) {   // a page without references: the books do not match the table
        atomicAdd(pool.ref + id, 1);
        good = false;
      }
      if (!good) atomicOr(err, ERR_BAD_PAGE);
    }
    row[b] = -1;
  }
}

// ------------------------------------------------------------------------------------------
// Trim, first part: block s shortens row s to new_lens[s] tokens and takes back the references of the pages behind them.
// ------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(128)
pages_trim_kernel(PagePool pool, int32_t* __restrict__ table, int32_t* __restrict__ lens,
                  const int32_t* __restrict__ new_lens, int MB, int bs, int32_t* err) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int s = blockIdx.x, L = lens[s], n = new_lens[s];
  if (n < 0 || n > L) {
    if (threadIdx.x == 0) atomicOr(err, ERR_BAD_SEQUENCE);
    return;
  }
  const int64_t had = (static_cast<int64_t>(L) + bs - 1) / bs, keep = (static_cast<int64_t>(n) + bs - 1) / bs;
  if (had > MB && threadIdx.x == 0) atomicOr(err, ERR_BAD_SEQUENCE);
  const int b1 = static_cast<int>(had < MB ? had : MB);
  int32_t* row = table + static_cast<int64_t>(s) * MB;
  for (int64_t b = keep + threadIdx.x; b < b1; b += blockDim.x) {
    const int id = row[b];
    bool good = id >= 0 && id < pool.NB;
    if (good && atomicSub(pool.ref + id, 1) <= 0) {   // a page without references: the books do not match the table
      atomicAdd(pool.ref + id, 1);
      good = false;
    }
    if (!good) atomicOr(err, ERR_BAD_PAGE);
    row[b] = -1;
  }
  __syncthreads();                                    // (every thread has read the length)
  if (threadIdx.x == 0) lens[s] = n;
}

// ------------------------------------------------------------------------------------------
// One pass over the reference counts by a cluster of blocks: the free list of the present counts (COMPACT = false),
// or the moves that make the live pages dense and the books after them (COMPACT = true).  Block r of the cluster owns
// a contiguous range of pages; the ranges' live counts are exchanged through distributed shared memory.
// Compaction: with n live pages, the live pages at or past n move, in ascending order, into the holes below n.
// ------------------------------------------------------------------------------------------
constexpr int kPagesCluster = 8;

template <bool COMPACT>
__global__ void __cluster_dims__(kPagesCluster, 1, 1) __launch_bounds__(kPagesThreads)
pages_books_kernel(PagePool pool, int32_t* __restrict__ copy_src, int32_t* __restrict__ copy_dst, int max_copies,
                   PagesScratch X) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ int warp_sums[32];
  __shared__ int live_of[kPagesCluster];        // live pages of every block's range
  const int tid = threadIdx.x, rank = static_cast<int>(cluster.block_rank());
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int NB = pool.NB;
  // ranges of whole 4-page groups
  const int per = ((NB + kPagesCluster - 1) / kPagesCluster + 3) & ~3;
  const int lo = min(NB, rank * per), hi = min(NB, lo + per);
  auto load4 = [&](int p, bool (&live)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) live[e] = p + e < hi && pool.ref[p + e] > 0;
  };
  int mine = 0;
  for (int p = lo + 4 * tid; p < hi; p += 4 * kPagesThreads) {
    bool live[4];
    load4(p, live);
    mine += live[0] + live[1] + live[2] + live[3];
  }
  int sum;
  block_scan_excl(mine, warp_sums, &sum);
  if (tid < kPagesCluster) *cluster.map_shared_rank(&live_of[rank], tid) = sum;
  cluster.sync();
  int before = 0, n_live = 0;                   // live pages below this block's range; all of them
#pragma unroll
  for (int r = 0; r < kPagesCluster; ++r) {
    before += r < rank ? live_of[r] : 0;
    n_live += live_of[r];
  }
  const int n_free = NB - n_live;
  // how many live pages lie below page n_live (only needed for compaction): each range past it does not count
  int holes = 0;
  if (COMPACT) {
    // the range that page n_live falls into counts its part; exchanged like the totals
    __shared__ int below_of[kPagesCluster];
    int m = 0;
    for (int p = lo + 4 * tid; p < hi && p < n_live; p += 4 * kPagesThreads) {
      bool live[4];
      load4(p, live);
#pragma unroll
      for (int e = 0; e < 4; ++e) m += live[e] && p + e < n_live;
    }
    int s2;
    block_scan_excl(m, warp_sums, &s2);
    if (tid < kPagesCluster) *cluster.map_shared_rank(&below_of[rank], tid) = s2;
    cluster.sync();
    int below = 0;
#pragma unroll
    for (int r = 0; r < kPagesCluster; ++r) below += below_of[r];
    holes = n_live - below;                     // = moves
  }
  for (int base = lo; base < hi; base += 4 * kPagesThreads) {
    const int p = base + 4 * tid;
    bool live[4] = {false, false, false, false};
    if (p < hi) load4(p, live);
    int s3;
    int at = before + block_scan_excl(live[0] + live[1] + live[2] + live[3], warp_sums, &s3);   // live pages below p
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int id = p + e;
      if (id < hi) {
        if (!COMPACT) {
          if (!live[e]) pool.free_list[n_free - 1 - (id - at)] = id;
        } else if (live[e] && id >= n_live) {
          const int k = at - (n_live - holes);
          if (k < max_copies) copy_src[k] = id;
        } else if (!live[e] && id < n_live) {
          const int k = id - at;
          if (k < max_copies) copy_dst[k] = id;
        }
        if (COMPACT) X.map[id] = live[e] && id < n_live ? id : -1;   // (those that move: below)
      }
      at += live[e];
    }
    before += s3;
  }
  const int g = rank * kPagesThreads + tid, G = kPagesCluster * kPagesThreads;
  for (int i = g; i < NB; i += G)
    if (COMPACT) pool.free_list[i] = i < n_free ? NB - 1 - i : -1;
    else if (i >= n_free) pool.free_list[i] = -1;
  if (g == 0) *pool.free_count = n_free;
  if (COMPACT) {
    for (int i = g; i < max_copies; i += G)
      if (i >= holes) copy_src[i] = copy_dst[i] = -1;
    __threadfence();
    cluster.sync();                             // every move is written; the counts are no longer read as they were
    for (int i = g; i < min(holes, max_copies); i += G) {
      const int a = __ldcg(copy_src + i), b = __ldcg(copy_dst + i);
      pool.ref[b] = __ldcg(pool.ref + a);
      pool.ref[a] = 0;
      X.map[a] = b;
    }
  }
  cluster.sync();                               // no block leaves while another may still write to its shared memory
}

// Compaction, second part: block s rewrites the used entries of row s.
__global__ void __launch_bounds__(128)
pages_remap_kernel(PagePool pool, int32_t* __restrict__ table, const int32_t* __restrict__ lens, int MB, int bs,
                   PagesScratch X) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int s = blockIdx.x;
  const int64_t need = (static_cast<int64_t>(lens[s]) + bs - 1) / bs;
  const int np = static_cast<int>(need < 0 ? 0 : need < MB ? need : MB);
  int32_t* row = table + static_cast<int64_t>(s) * MB;
  for (int b = threadIdx.x; b < np; b += blockDim.x) {
    const int id = row[b];
    const int to = id >= 0 && id < pool.NB ? X.map[id] : -1;
    if (to < 0) atomicOr(X.err, ERR_BAD_PAGE);  // an entry that names no live page stays as it is
    else if (to != id) row[b] = to;
  }
}

// ------------------------------------------------------------------------------------------
// Page copies: pair i copies page src[i] to page dst[i] in K and in V (a pair with a negative entry is skipped).
// Unit = (pair, K or V); a block looks at 32 of its units at a time and copies the ones that exist, 16 bytes per
// thread and four loads in flight.
// ------------------------------------------------------------------------------------------
struct CopyParams {
  uint8_t *k, *v;
  const int32_t *src, *dst;
  int64_t sb, sh, st;          // byte strides of block, head, token row
  int n, NB, heads, rows, row_chunks;   // row_chunks: 16-byte chunks of a row
  int dense;                   // the page is one contiguous run
  int32_t* err;
};
constexpr int kCopyThreads = 256;

__global__ void __launch_bounds__(kCopyThreads)
pages_copy_kernel(const __grid_constant__ CopyParams P) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const int units = 2 * P.n;
  const int per_head = P.rows * P.row_chunks, chunks = P.heads * per_head;
  for (int64_t base = blockIdx.x; base < units; base += 32ll * gridDim.x) {
    const int64_t u = base + static_cast<int64_t>(lane) * gridDim.x;
    int a = -1, b = -1;
    if (u < units) {
      a = __ldg(P.src + u / 2);
      b = __ldg(P.dst + u / 2);
    }
    const bool named = a >= 0 && b >= 0;
    const bool good = named && a < P.NB && b < P.NB;
    if (named && !good && P.err && threadIdx.x < 32) atomicOr(P.err, ERR_BAD_PAGE);
    uint32_t todo = __ballot_sync(0xffffffffu, good && a != b);
    while (todo) {
      const int l = __ffs(todo) - 1;
      todo &= todo - 1;
      const int from = __shfl_sync(0xffffffffu, a, l), to = __shfl_sync(0xffffffffu, b, l);
      uint8_t* pool = ((base + static_cast<int64_t>(l) * gridDim.x) & 1) ? P.v : P.k;
      const uint8_t* s = pool + from * P.sb;
      uint8_t* d = pool + to * P.sb;
      auto at = [&](int c) -> int64_t {
        if (P.dense) return static_cast<int64_t>(c) * 16;
        const int h = c / per_head, r = (c - h * per_head) / P.row_chunks;
        return h * P.sh + r * P.st + static_cast<int64_t>(c - h * per_head - r * P.row_chunks) * 16;
      };
      for (int c = threadIdx.x; c < chunks; c += 4 * kCopyThreads) {
        uint4 w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e * kCopyThreads < chunks) w[e] = *reinterpret_cast<const uint4*>(s + at(c + e * kCopyThreads));
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e * kCopyThreads < chunks) *reinterpret_cast<uint4*>(d + at(c + e * kCopyThreads)) = w[e];
      }
    }
  }
}

}  // namespace pdattn

// Rotary positions fused with the KV append: rope_append_kernel.
//
// A new token at position pos has its query and key heads rotated, pair by pair:
//   theta_i = pos * inv_freq[i],   x' = mag (x cos theta_i - y sin theta_i),   y' = mag (y cos theta_i + x sin theta_i)
// with (x, y) = elements (i, i + R/2) of the head (half layout) or (2i, 2i + 1) (interleaved), i < R/2; elements at or
// past R pass through.  q goes to q_out, the rotated k and the untouched v to their slots of the paged cache.
//
// Bound: bytes (every row is read once and written once); a single-token step of a few hundred sequences is bound
// by the launch and two dependent loads (length, page id).
//   - Angles once per token, not once per head: the block's R/2 cosines and sines go through shared memory.
//   - Angles of far positions: the product and the reduction to a turn are done in 64 bits (three operations), the
//     sine and cosine of the reduced turn in 32.  pos * inv_freq in 32 bits would be off by up to 0.03 rad at 10^6.
//   - A thread owns two 16-byte chunks of a row that rotate into each other (half layout: R/2 elements apart;
//     interleaved and pass-through: neighbours), so every load and store is 16 bytes wide and q_out may be q.
//   - 512 threads a block, three blocks an SM: measured on 17,492 prompt tokens of 40 + 8 + 8 heads, 91 us (5.5 TB/s; 256
//     threads with a deeper unroll 95), and on one token of 256 sequences, 28 + 4 + 4 heads, 3.4 us (3.6).
//   - Products and sums in fp32, one rounding per element (bf16 nearest even; e4m3 of value / scale for the fp8 cache).
#pragma once

#include "common.cuh"

namespace pdattn {

constexpr int kRopeThreads = 512;
constexpr int kRopeMaxTokens = 8;      // tokens of a block (one warp each looks its token up)

struct RopeParams {
  const __nv_bfloat16 *q, *k_new, *v_new;
  __nv_bfloat16* q_out;
  void *k_cache, *v_cache;
  const int32_t *block_table, *context_lens, *cu_tokens;   // cu_tokens null: token t belongs to sequence t
  const int32_t* positions;            // of the rotation, per token; null: the token's place in its sequence
  const float *inv_freq, *k_scale, *v_scale;
  int64_t q_ts, k_ts, v_ts;            // token strides of q, k_new, v_new (elements)
  int64_t sb, sh, st;                  // cache strides (elements)
  int32_t* err;
  float magnitude;
  int N, S, Hq, Hkv, bs, MB, NB, R, interleaved, tokens_per_block;
};

// The sequence that token t belongs to: the last s with cu[s] <= t (sequences without tokens are stepped over), or -1
// when t lies behind the last sequence.  One warp; 32 probes per round.
__device__ __forceinline__ int find_sequence(const int32_t* __restrict__ cu, int S, int t, int lane) {
  if (t >= __ldg(cu + S) || t < __ldg(cu)) return -1;
  int lo = 0, n = S;                   // the answer lies in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32;
    const int i = lane * step;
    const bool below = i < n && __ldg(cu + lo + i) <= t;
    const uint32_t m = __ballot_sync(0xffffffffu, below);
    const int k = m ? 31 - __clz(m) : 0;
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}

template <int D, bool FP8>
__global__ void __launch_bounds__(kRopeThreads, 3)
rope_append_kernel(const __grid_constant__ RopeParams P) {
  constexpr int TPR = D / 16;          // threads per row: two 16-byte chunks each
  __shared__ float2 cs[kRopeMaxTokens][D / 2];
  __shared__ int4 info[kRopeMaxTokens];   // (0, or -1: no such token; page or -1: not written; slot; q: 1 rotate, 0 zeros)
  __shared__ int turn_at[kRopeMaxTokens]; // position of the rotation
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int t0 = blockIdx.x * P.tokens_per_block;
  const int nt = min(P.tokens_per_block, P.N - t0);
  asm volatile("griddepcontrol.wait;" ::: "memory");   // a programmatic dependent of the kernel before it on the stream
  if (warp < nt) {
    const int t = t0 + warp;
    const int s = P.cu_tokens ? find_sequence(P.cu_tokens, P.S, t, lane) : t;
    if (lane == 0) {
      int4 v = make_int4(-1, -1, 0, 0);
      int at = 0;
      if (s >= 0) {
        const int after = P.cu_tokens ? __ldg(P.cu_tokens + s + 1) - t : 1;   // new tokens from this one on
        const int pos = __ldg(P.context_lens + s) - after;
        v.x = 0;
        if (pos >= 0) {
          at = P.positions ? __ldg(P.positions + t) : pos;
          v.w = 1;
          v.z = pos % P.bs;
          const int b = pos / P.bs;
          const int page = b < P.MB ? __ldg(P.block_table + static_cast<int64_t>(s) * P.MB + b) : -1;
          if (page >= 0 && page < P.NB) v.y = page;
          else if (P.err) atomicOr(P.err, ERR_BAD_PAGE);
        }
      }
      info[warp] = v;
      turn_at[warp] = at;
    }
  }
  __syncthreads();
  const int half = P.R / 2;
  for (int i = tid; i < nt * half; i += kRopeThreads) {
    const int k = i / half, j = i - k * half;
    double turn = static_cast<double>(turn_at[k]) * static_cast<double>(__ldg(P.inv_freq + j)) * 0.15915494309189535;
    turn -= rint(turn);
    float sn, cn;
    sincospif(static_cast<float>(2.0 * turn), &sn, &cn);
    cs[k][j] = make_float2(cn * P.magnitude, sn * P.magnitude);
  }
  __syncthreads();
  const int rows = P.Hq + 2 * P.Hkv;
  const int rot = P.R / 16;            // chunk pairs of a row that rotate
  const int items = nt * rows * TPR;
#pragma unroll 1
  for (int i = tid; i < items; i += kRopeThreads) {
    const int p = i % TPR, tr = i / TPR;
    const int k = tr / rows, r = tr - k * rows;
    const int4 f = info[k];
    if (f.x < 0) continue;             // behind the last sequence: left as it is
    const int64_t t = t0 + k;
    const bool isq = r < P.Hq, isv = r >= P.Hq + P.Hkv;
    if (!isq && f.y < 0) continue;     // no page for this token
    const int h = isq ? r : isv ? r - P.Hq - P.Hkv : r - P.Hq;
    const __nv_bfloat16* src = isq ? P.q + t * P.q_ts : isv ? P.v_new + t * P.v_ts : P.k_new + t * P.k_ts;
    const bool split = p < rot && !P.interleaved;
    const int c0 = split ? p : 2 * p, c1 = split ? p + rot : 2 * p + 1;
    const uint4 ra = *reinterpret_cast<const uint4*>(src + h * D + c0 * 8);
    const uint4 rb = *reinterpret_cast<const uint4*>(src + h * D + c1 * 8);
    float a[8], b[8];
    {
      const uint32_t wa[4] = {ra.x, ra.y, ra.z, ra.w}, wb[4] = {rb.x, rb.y, rb.z, rb.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        a[2 * e] = __uint_as_float(wa[e] << 16);
        a[2 * e + 1] = __uint_as_float(wa[e] & 0xffff0000u);
        b[2 * e] = __uint_as_float(wb[e] << 16);
        b[2 * e + 1] = __uint_as_float(wb[e] & 0xffff0000u);
      }
    }
    if (!isv && p < rot) {
      const float4* z4 = reinterpret_cast<const float4*>(&cs[k][8 * p]);   // pairs 8p .. 8p + 7
      if (split) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 z = z4[e];
          const float x0 = a[2 * e], y0 = b[2 * e], x1 = a[2 * e + 1], y1 = b[2 * e + 1];
          a[2 * e] = x0 * z.x - y0 * z.y;
          b[2 * e] = y0 * z.x + x0 * z.y;
          a[2 * e + 1] = x1 * z.z - y1 * z.w;
          b[2 * e + 1] = y1 * z.z + x1 * z.w;
        }
      } else {
        auto turn4 = [&](float (&w)[8], const float4* zz) {   // four neighbouring pairs
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float4 z = zz[e];
            const float x0 = w[4 * e], y0 = w[4 * e + 1], x1 = w[4 * e + 2], y1 = w[4 * e + 3];
            w[4 * e] = x0 * z.x - y0 * z.y;
            w[4 * e + 1] = y0 * z.x + x0 * z.y;
            w[4 * e + 2] = x1 * z.z - y1 * z.w;
            w[4 * e + 3] = y1 * z.z + x1 * z.w;
          }
        };
        turn4(a, z4);
        turn4(b, z4 + 2);
      }
    }
    auto packed = [](const float (&w)[8]) {
      return make_uint4(pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3]), pack_bf16x2(w[4], w[5]), pack_bf16x2(w[6], w[7]));
    };
    if (isq) {
      // a token before position 0 (more new tokens than the context holds) has no place to attend from: zeros
      const bool live = f.w != 0;
      __nv_bfloat16* dst = P.q_out + (t * P.Hq + h) * D;
      *reinterpret_cast<uint4*>(dst + c0 * 8) = live ? packed(a) : make_uint4(0, 0, 0, 0);
      *reinterpret_cast<uint4*>(dst + c1 * 8) = live ? packed(b) : make_uint4(0, 0, 0, 0);
    } else if constexpr (!FP8) {
      __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(isv ? P.v_cache : P.k_cache) + f.y * P.sb + h * P.sh + f.z * P.st;
      *reinterpret_cast<uint4*>(dst + c0 * 8) = isv ? ra : packed(a);
      *reinterpret_cast<uint4*>(dst + c1 * 8) = isv ? rb : packed(b);
    } else {
      // K as a row of the page [slot][D], V as a column of the transposed page [D][slot]
      const float sc = __ldg((isv ? P.v_scale : P.k_scale) + h);   // true divisions: the code is decided in fp32
      uint32_t ca[2], cb[2];
      auto codes = [&](const float (&w)[8], uint32_t (&o)[2]) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          unsigned short u0, u1;
          asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(u0) : "f"(__fdiv_rn(w[4 * e + 1], sc)), "f"(__fdiv_rn(w[4 * e], sc)));
          asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(u1) : "f"(__fdiv_rn(w[4 * e + 3], sc)), "f"(__fdiv_rn(w[4 * e + 2], sc)));
          o[e] = static_cast<uint32_t>(u0) | (static_cast<uint32_t>(u1) << 16);
        }
      };
      codes(a, ca);
      codes(b, cb);
      const int64_t page_head = (static_cast<int64_t>(f.y) * P.Hkv + h) * P.bs * D;
      if (!isv) {
        uint8_t* dst = static_cast<uint8_t*>(P.k_cache) + page_head + static_cast<int64_t>(f.z) * D;
        *reinterpret_cast<uint2*>(dst + c0 * 8) = make_uint2(ca[0], ca[1]);
        *reinterpret_cast<uint2*>(dst + c1 * 8) = make_uint2(cb[0], cb[1]);
      } else {
        uint8_t* dst = static_cast<uint8_t*>(P.v_cache) + page_head + f.z;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          dst[(c0 * 8 + e) * P.bs] = static_cast<uint8_t>(ca[e >> 2] >> (8 * (e & 3)));
          dst[(c1 * 8 + e) * P.bs] = static_cast<uint8_t>(cb[e >> 2] >> (8 * (e & 3)));
        }
      }
    }
  }
}

}  // namespace pdattn

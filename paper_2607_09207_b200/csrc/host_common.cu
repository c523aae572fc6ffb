// Host-side helpers shared by the API translation units: see host_common.h.
#include "host_common.h"

#include <cstdio>
#include <mutex>

namespace pdattn {

namespace {
thread_local char g_cuda_err[kCudaErrorTextBytes] = "";
}

char* cuda_error_text() { return g_cuda_err; }

pdattn_status cuda_fail(const char* what, cudaError_t e) {
  snprintf(g_cuda_err, sizeof g_cuda_err, "%s: %s", what, cudaGetErrorString(e));
  return PDATTN_CUDA_ERROR;
}

pdattn_status check_shape(int num_seqs, int Hq, int Hkv, int d, int bs) {
  if (num_seqs < 0 || Hq <= 0 || Hkv <= 0 || d <= 0 || bs <= 0) return PDATTN_INVALID_ARG;
  if (Hq % Hkv != 0) return PDATTN_INVALID_ARG;
  if (d != 64 && d != 128) return PDATTN_UNSUPPORTED;
  if (bs != 16 && bs != 32 && bs != 64) return PDATTN_UNSUPPORTED;
  if (Hq / Hkv > 16) return PDATTN_UNSUPPORTED;
  return PDATTN_OK;
}

// ---- per-device facts ------------------------------------------------------------------------
namespace {
DevInfo g_dev[kMaxDevices];
std::mutex g_dev_mu;
}  // namespace

pdattn_status device_info(int* dev_out, DevInfo** info) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail("cudaGetDevice", e);
  if (dev < 0 || dev >= kMaxDevices) return PDATTN_UNSUPPORTED;
  DevInfo& di = g_dev[dev];
  if (!di.ready) {
    std::lock_guard<std::mutex> lk(g_dev_mu);
    if (!di.ready) {
      int sms = 0, major = 0;
      e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
      if (e != cudaSuccess) return cuda_fail("cudaDeviceGetAttribute", e);
      e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
      if (e != cudaSuccess) return cuda_fail("cudaDeviceGetAttribute", e);
      if (major != 10) {
        snprintf(cuda_error_text(), kCudaErrorTextBytes, "libpdattn is built for sm_100a only (device has major %d)", major);
        return PDATTN_CUDA_ERROR;
      }
      di.sm_count = sms;
      di.ready = true;
    }
  }
  *dev_out = dev;
  *info = &di;
  return PDATTN_OK;
}

// ---- TMA tensor maps ---------------------------------------------------------------------------
namespace {
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn g_encode = nullptr;

pdattn_status get_encode() {
  if (g_encode) return PDATTN_OK;
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult qres;
  cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres);
  if (e != cudaSuccess) return cuda_fail("cudaGetDriverEntryPoint", e);
  if (!fn || qres != cudaDriverEntryPointSuccess) {
    snprintf(cuda_error_text(), kCudaErrorTextBytes, "cuTensorMapEncodeTiled not available in this driver");
    return PDATTN_CUDA_ERROR;
  }
  g_encode = reinterpret_cast<EncodeTiledFn>(fn);
  return PDATTN_OK;
}

struct MapKey {
  const void* ptr;
  int d, bs, hkv, nb, rank;
  int64_t sb, sh, st;
  bool operator==(const MapKey& o) const {
    return ptr == o.ptr && d == o.d && bs == o.bs && hkv == o.hkv && nb == o.nb && rank == o.rank && sb == o.sb &&
           sh == o.sh && st == o.st;
  }
};
struct MapCacheEntry {
  bool valid = false;
  MapKey key;
  CUtensorMap map;
};
thread_local MapCacheEntry g_maps[16];
thread_local int g_map_next = 0;

}  // namespace

// View of a cache as a tensor for TMA, 128-byte swizzle, zero fill out of bounds.
//   rank 4: (dim, slot, kv head, page); one box = one 64-element column block of a page-head,
//           [64, block_size, 1, 1]: head_dim / 64 copies per page-head.
//   rank 5: (dim within column block, slot, column block, kv head, page); one box = a whole
//           page-head [64, block_size, 2, 1, 1], landing in shared memory column block by column
//           block exactly like two rank-4 boxes.  head_dim 128 only.
pdattn_status make_map(const void* ptr, int d, int bs, int hkv, int nb, int64_t sb, int64_t sh, int64_t st, int rank,
                       CUtensorMap* out) {
  MapKey key{ptr, d, bs, hkv, nb, rank, sb, sh, st};
  for (auto& e : g_maps)
    if (rank != kMapQ && e.valid && e.key == key) {
      *out = e.map;
      return PDATTN_OK;
    }
  pdattn_status s = get_encode();
  if (s != PDATTN_OK) return s;
  const cuuint64_t nbu = static_cast<cuuint64_t>(nb > 0 ? nb : 1);
  CUtensorMap m;
  CUresult r;
  if (rank == kMapK8) {
    // fp8 K pool [pages, kv heads, slots, d] of one-byte codes: one box = a page-head, [d, block_size, 1, 1]
    cuuint64_t dims[4] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(bs), static_cast<cuuint64_t>(hkv), nbu};
    cuuint64_t strides[3] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(bs) * d,
                             static_cast<cuuint64_t>(hkv) * bs * d};
    cuuint32_t box[4] = {static_cast<cuuint32_t>(d), static_cast<cuuint32_t>(bs), 1, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    // rows of d bytes: 128-byte swizzle at head_dim 128, 64-byte swizzle at head_dim 64
    r = g_encode(&m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(ptr), dims, strides, box, estr,
                 CU_TENSOR_MAP_INTERLEAVE_NONE, d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                 CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  } else if (rank == kMapV8) {
    // fp8 V pool [pages, kv heads, d, slots] (transposed inside a page): a page-head is d * block_size
    // contiguous bytes and lands in shared memory in the same order, so it is described as rows of 256
    // bytes (8 requests per box; rows of block_size bytes would be 128), no swizzle
    const cuuint64_t rows = static_cast<cuuint64_t>(d) * bs / 256;
    cuuint64_t dims[4] = {256, rows, static_cast<cuuint64_t>(hkv), nbu};
    cuuint64_t strides[3] = {256, static_cast<cuuint64_t>(d) * bs, static_cast<cuuint64_t>(hkv) * d * bs};
    cuuint32_t box[4] = {256, static_cast<cuuint32_t>(rows), 1, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    r = g_encode(&m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(ptr), dims, strides, box, estr,
                 CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                 CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  } else if (rank == kMapQ) {
    // dense query rows [nb tokens, hkv KV heads, sh heads of a KV head, d]; one box = a 64-element column block of the
    // heads of one KV head for bs tokens, row = token * heads + head
    const cuuint64_t G = static_cast<cuuint64_t>(sh), H = static_cast<cuuint64_t>(hkv), dd = static_cast<cuuint64_t>(d);
    cuuint64_t dims[4] = {dd, G, H, nbu};
    cuuint64_t strides[3] = {dd * 2, G * dd * 2, H * G * dd * 2};
    cuuint32_t box[4] = {64, static_cast<cuuint32_t>(G), 1, static_cast<cuuint32_t>(bs)};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    r = g_encode(&m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(ptr), dims, strides, box, estr,
                 CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                 CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  } else if (rank == 5) {
    cuuint64_t dims[5] = {64, static_cast<cuuint64_t>(bs), static_cast<cuuint64_t>(d / 64),
                          static_cast<cuuint64_t>(hkv), nbu};
    cuuint64_t strides[4] = {static_cast<cuuint64_t>(st) * 2, 128, static_cast<cuuint64_t>(sh) * 2,
                             static_cast<cuuint64_t>(sb) * 2};
    cuuint32_t box[5] = {64, static_cast<cuuint32_t>(bs), static_cast<cuuint32_t>(d / 64), 1, 1};
    cuuint32_t estr[5] = {1, 1, 1, 1, 1};
    r = g_encode(&m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(ptr), dims, strides, box, estr,
                 CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                 CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  } else {
    cuuint64_t dims[4] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(bs), static_cast<cuuint64_t>(hkv), nbu};
    cuuint64_t strides[3] = {static_cast<cuuint64_t>(st) * 2, static_cast<cuuint64_t>(sh) * 2,
                             static_cast<cuuint64_t>(sb) * 2};
    cuuint32_t box[4] = {64, static_cast<cuuint32_t>(bs), 1, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    r = g_encode(&m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(ptr), dims, strides, box, estr,
                 CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                 CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  }
  if (r != CUDA_SUCCESS) {
    snprintf(cuda_error_text(), kCudaErrorTextBytes, "cuTensorMapEncodeTiled (rank %d) failed with CUresult %d", rank,
             static_cast<int>(r));
    return PDATTN_CUDA_ERROR;
  }
  *out = m;
  if (rank == kMapQ) return PDATTN_OK;
  MapCacheEntry& e = g_maps[g_map_next];
  g_map_next = (g_map_next + 1) % 16;
  e.valid = true;
  e.key = key;
  e.map = m;
  return PDATTN_OK;
}

}  // namespace pdattn

// Host-side helpers shared by the API translation units of libpdattn: error text, per-device facts, tensor maps,
// programmatic dependent launches.  Defined in host_common.cu; hidden from the library's symbol table.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/pdattn.h"

namespace pdattn {

#define PDATTN_HIDDEN __attribute__((visibility("hidden")))

// Thread-local text of the last CUDA failure, and the status that goes with it.
PDATTN_HIDDEN char* cuda_error_text();
constexpr size_t kCudaErrorTextBytes = 256;
PDATTN_HIDDEN pdattn_status cuda_fail(const char* what, cudaError_t e);

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// The head shapes and page sizes every attention entry point takes.
PDATTN_HIDDEN pdattn_status check_shape(int num_seqs, int Hq, int Hkv, int d, int bs);

// A cap of pdattn_score_args: none (0), or one whose reciprocal and whose multiples fp32 holds.
inline bool valid_cap(float cap) { return cap == 0.f || (cap >= 1e-6f && cap <= 1e6f); }

// ---- per-device facts ------------------------------------------------------------------------
struct DevInfo {
  bool ready = false;
  int sm_count = 0;
  bool attr_set[2][2][3] = {};      // [D==128][NT==2][page size / 32]
  bool probe_attr_set[2][2][3] = {};
  bool chain_attr_set[2][2][3] = {};
  bool win_attr_set[2][3] = {};     // [D==128][page size / 32]
  bool fp8_attr_set[2][2][3] = {};  // [D==128][NT==2][page size / 32]
  bool prefix_fp8_attr_set[2][3] = {};
  bool prefix_attr_set[2][3] = {};  // [D==128][page size / 32]
  bool prefix_umma_attr_set[2][3] = {};
};
constexpr int kMaxDevices = 64;
PDATTN_HIDDEN pdattn_status device_info(int* dev_out, DevInfo** info);

// ---- TMA tensor maps ---------------------------------------------------------------------------
constexpr int kMapK8 = 81, kMapV8 = 82;   // "ranks" of the two fp8 views in make_map
constexpr int kMapQ = 83;                 // ... and of the packed query rows of pdattn_prefill
// View of a cache as a tensor for TMA (see host_common.cu).  The caches' views are kept per thread, pointer and shape; that of
// the query rows, which are new memory in every call, is not.
PDATTN_HIDDEN pdattn_status make_map(const void* ptr, int d, int bs, int hkv, int nb, int64_t sb, int64_t sh, int64_t st,
                                     int rank, CUtensorMap* out);

// ---- launches ------------------------------------------------------------------------------------
// Launch that may begin while the kernel before it on the stream drains (programmatic dependent launch); the
// kernel itself waits (griddepcontrol.wait) before it touches global memory.
template <typename... KArgs, typename... Args>
cudaError_t launch_dependent(void (*kernel)(KArgs...), dim3 grid, int block, size_t smem, cudaStream_t stream, bool dependent,
                             const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = dependent ? 1 : 0;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

}  // namespace pdattn

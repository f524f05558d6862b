// Host side of the few-token operators: device check and launch.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/exo_gemm.h"

namespace exo {
void note_cuda_error(int e);   // what exo_gemm_last_cuda_error reports (api.cu)
// Zeroes device memory and returns when that is done: a plan may be run on any stream at once (api.cu).
cudaError_t clear_now(void* at, size_t bytes);
// Tensor map for copies of `steps` steps of 16 rows of a 4-bit matrix (api.cu, which looks the encoder up).
bool encode_steps_map(CUtensorMap* map, const void* codes, uint64_t rows, uint64_t blocks, uint32_t steps);
// The same for copies of a box of words (2 or 4 bytes) from the rows of a matrix.
bool encode_rows_map(CUtensorMap* map, int word_bytes, const void* base, uint64_t row_words, uint64_t rows, uint64_t row_bytes, uint32_t box_words,
                     uint32_t box_rows);

namespace decode {

constexpr int kMostSmem = 220 * 1024;   // dynamic shared memory a launch may ask for

// What exo_decode_debug_set has set for this call (q4.cu): the bound of its waits for copies in SM clocks (at 2 GHz; 4 s if nothing is
// set), and whose first warp issues none.
struct WaitHook {
  uint64_t clocks;
  int skip;
};
WaitHook take_wait_hook();

inline exo_gemm_status_t cuda_failed(cudaError_t e) {
  note_cuda_error((int)e);
  cudaGetLastError();   // clear the runtime's error state
  return EXO_GEMM_ERR_CUDA;
}

// The current device has to be compute capability 10.x; *sms is its SM count.  Looked up once per device.
inline exo_gemm_status_t device_check(int* sms) {
  static std::atomic<int> seen[64];   // 0: not yet; else SM count, negative where the architecture is another
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return cuda_failed(e);
  int v = device < 64 ? seen[device].load(std::memory_order_relaxed) : 0;
  if (v == 0) {
    int major = 0, n = 0;
    if ((e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device)) != cudaSuccess) return cuda_failed(e);
    if ((e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device)) != cudaSuccess) return cuda_failed(e);
    v = major == 10 ? n : -n;
    if (device < 64) seen[device].store(v, std::memory_order_relaxed);
  }
  if (v < 0) return EXO_GEMM_ERR_ARCH;
  *sms = v;
  return EXO_GEMM_OK;
}

// Alignment of a 4-bit matrix's parts: a lane reads 16 bytes of codes, and the scales and zero points of 128 weights at once.
inline bool q4_aligned(const void* codes, const void* scales, const void* zeros, int group) {
  return ((uintptr_t)codes & 15u) == 0 && (uintptr_t)scales % (unsigned)(256 / group) == 0 && (uintptr_t)zeros % (unsigned)(128 / group) == 0;
}

// Opts a kernel in to kMostSmem, or what it can have, once per device: always to the same size, so that threads which launch one kernel at different
// sizes cannot take it from each other.
inline cudaError_t allow_smem(void* fn) {
  constexpr int kSlots = 512;
  static std::atomic<void*> done[8][kSlots];   // the kernels that have it, by hash of their address
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  std::atomic<void*>* slot = nullptr;
  if (device < 8) {
    for (int i = 0; i < 4; ++i) {
      std::atomic<void*>& s = done[device][(((uintptr_t)fn >> 4) * 0x9e3779b1u + (unsigned)i) % kSlots];
      void* have = s.load(std::memory_order_relaxed);
      if (have == fn) return cudaSuccess;
      if (!have && !slot) slot = &s;
    }
  }
  cudaFuncAttributes a;
  if ((e = cudaFuncGetAttributes(&a, fn)) != cudaSuccess) return e;
  const int room = 227 * 1024 - (int)a.sharedSizeBytes;   // what the kernel's own variables leave
  e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, room < kMostSmem ? room : kMostSmem);
  if (e == cudaSuccess && slot) slot->store(fn, std::memory_order_relaxed);
  return e;
}

// How many clusters of `cluster` CTAs of this kernel the current device holds at once: fewer than its SMs divided by the cluster where
// a GPC's SMs do not divide.  Asked once per device for each kind (an index below 32 that the caller gives to kernel, cluster size
// and shared memory).
inline int resident_clusters(int kind, void* fn, unsigned threads, size_t smem, unsigned cluster, int sms, int ctas_per_sm) {
  static std::atomic<int> known[8][32];
  const int otherwise = ctas_per_sm * sms / (int)cluster;
  if (cluster == 1) return otherwise;
  int device = 0, n = 0;
  if (cudaGetDevice(&device) != cudaSuccess || device >= 8) return otherwise;
  if ((n = known[device][kind].load(std::memory_order_relaxed)) > 0) return n;
  cudaLaunchConfig_t lc{};
  lc.gridDim = dim3(cluster, 1, 1);
  lc.blockDim = dim3(threads, 1, 1);
  lc.dynamicSmemBytes = smem;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = cluster;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  lc.attrs = at;
  lc.numAttrs = 1;
  if (allow_smem(fn) != cudaSuccess || cudaOccupancyMaxActiveClusters(&n, fn, &lc) != cudaSuccess || n < 1) {
    cudaGetLastError();
    n = otherwise;
  }
  known[device][kind].store(n, std::memory_order_relaxed);
  return n;
}

// One launch with programmatic dependent launch and, for cluster > 1, clusters of that many CTAs along x.
inline exo_gemm_status_t launch(void* fn, unsigned grid_x, unsigned grid_y, unsigned threads, size_t smem, unsigned cluster,
                                cudaStream_t stream, void* params, void* params2 = nullptr, void* params3 = nullptr) {
  cudaError_t e;
  // without it a kernel has 48 KB, its own variables included: what it needs beyond `smem` is not known here
  if (smem > 0 && (e = allow_smem(fn)) != cudaSuccess) return cuda_failed(e);
  cudaLaunchConfig_t lc{};
  lc.gridDim = dim3(grid_x, grid_y, 1);
  lc.blockDim = dim3(threads, 1, 1);
  lc.dynamicSmemBytes = smem;
  lc.stream = stream;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  lc.attrs = at;
  lc.numAttrs = cluster > 1 ? 2 : 1;
  void* args[3] = {params, params2, params3};
  e = cudaLaunchKernelExC(&lc, fn, args);
  return e == cudaSuccess ? EXO_GEMM_OK : cuda_failed(e);
}

}  // namespace decode
}  // namespace exo

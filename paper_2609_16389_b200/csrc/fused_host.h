// Host side of exo_fused.h: launches, tensor maps, tile shapes, aligned copies and device memory of plans.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <atomic>
#include <initializer_list>

#include "../../include/exo_fused.h"
#include "decode_host.h"
#include "fused_core.cuh"
#include "plan.h"

namespace exo {
bool encode_operand_map(CUtensorMap* map, int elem_bytes, bool bf16, const void* base, uint64_t inner, uint64_t rows, uint64_t row_bytes,
                        uint32_t box_rows);   // api.cu
bool encode_blocks_map(CUtensorMap* whole, CUtensorMap* rest, int elem_bytes, bool bf16, const void* base, uint64_t inner, uint64_t rows,
                       uint64_t row_bytes, uint64_t parts, uint64_t part_bytes, uint32_t box_rows, uint32_t box_blocks);   // api.cu
bool encode_result_map(CUtensorMap* map, void* base, uint64_t cols, uint64_t rows, uint64_t row_bytes);   // api.cu
exo_gemm_status_t gemm_run_scaled(exo_gemm_plan* plan, const void* A, const void* B, void* C, float alpha, const float* alpha_dev, float beta,
                                  void* cuda_stream);   // api.cu

namespace fused {

// What exo_fused_debug_set has set for the next kernel with products (i8.cu).
struct WaitHook {
  uint64_t clocks;
  int skip;
};
WaitHook take_wait_hook();

using decode::cuda_failed;
using decode::device_check;

struct OnDevice {   // makes `device` the current one while it lives
  int before = -1;
  cudaError_t err;
  explicit OnDevice(int device) {
    err = cudaGetDevice(&before);
    if (err == cudaSuccess && before != device) err = cudaSetDevice(device);
    else before = -1;
  }
  ~OnDevice() {
    if (before >= 0) cudaSetDevice(before);
  }
};

inline int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
// the largest power of two up to 32 that divides an address and a row stride in bytes
inline int align_of(const void* p, int64_t row_bytes) {
  const uint64_t at = (uint64_t)(uintptr_t)p | (uint64_t)row_bytes | 32u;
  return (int)(at & (~at + 1));
}
inline bool is16(int32_t t) { return t == EXO_GEMM_BF16 || t == EXO_GEMM_FP16; }

// One launch with programmatic dependent launch.  args: the kernel's parameters, in order.
inline exo_gemm_status_t launch_args(void* fn, dim3 grid, unsigned threads, size_t smem, unsigned cluster, cudaStream_t stream, void** args) {
  cudaError_t e;
  if (smem > 48 * 1024) {
    // every kernel gets the whole of what a CTA may have, once per device: launches of other sizes cannot lower it for one another
    constexpr int kSlots = 64;
    static std::atomic<void*> done[8][kSlots];
    int device = 0;
    if ((e = cudaGetDevice(&device)) != cudaSuccess) return cuda_failed(e);
    std::atomic<void*>* free_slot = nullptr;
    bool known = false;
    for (int i = 0; device < 8 && i < kSlots && !known && !free_slot; ++i) {
      void* have = done[device][i].load(std::memory_order_relaxed);
      known = have == fn;
      if (!have) free_slot = &done[device][i];
    }
    if (!known) {
      if ((e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit)) != cudaSuccess) return cuda_failed(e);
      if (free_slot) free_slot->store(fn, std::memory_order_relaxed);
    }
  }
  cudaLaunchConfig_t lc{};
  lc.gridDim = grid;
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
  e = cudaLaunchKernelExC(&lc, fn, args);
  return e == cudaSuccess ? EXO_GEMM_OK : cuda_failed(e);
}

constexpr int kThinRows = 128;   // what one tile's accumulator has

// Rows of B and A in a stage's k-block with which three stages leave an SM room for a second CTA.
constexpr int kSharedRows = 288;
// Thin tiles: a width that spreads the columns evenly over the SMs, with a charge per tile for its start and end.  quantum: what a width is a
// multiple of; most: the widest; parts: 2 for a gated product.  More tiles than SMs run two to an SM, which has to have the room.
inline int thin_width(int64_t N, int quantum, int most, int parts, int64_t rows, int sms) {
  const int a_rows = (int)round_up(rows, 8);
  int best = quantum;
  int64_t cost = -1;
  for (int w = quantum; w <= most; w += quantum) {
    const int64_t tiles = (N + w - 1) / w, waves = (tiles + sms - 1) / sms, c = waves * (w + 64);
    if (waves > 1 && w > quantum && parts * w + a_rows > kSharedRows) break;
    if (cost < 0 || c <= cost) { cost = c; best = w; }
  }
  return best;
}
// The ring of a thin tile: three large stages.  A stage costs the issuing warps some 500 clocks whatever it holds, which smaller ones do not
// hide (16 tokens through a block of 4096 x 10240, us in all, with stages of 20, 32, 48 and 66 KB: 56.8, 52.7, 49.5, 48.3).  One CTA per SM takes
// 200 KB; where there are more tiles than SMs two CTAs take 100 KB each, so that one's start and end hide behind the other's copies.
inline void thin_ring(int b_rows, int a_rows, int64_t whole, bool alone, int after, int* per_stage, int* stages) {
  const int block = (b_rows + a_rows) * 128;
  int per = (alone ? 66 : 33) * 1024 / block;
  if (per > 16) per = 16;
  if (per > whole) per = (int)whole;
  if (per < 1) per = 1;
  int n = (alone ? 200 : 100) * 1024 / (per * block);
  if (n < 3) n = 3;
  if (n > kThinMaxStages) n = kThinMaxStages;
  while (n > 1 && thin_smem(n, per, b_rows, a_rows, after) > kSmemLimit) --n;
  *per_stage = per;
  *stages = n;
}

// Accumulator columns of a pair's tile: what fills the waves best, multiples of 64 (128 for a B that lies K x N).  A narrow tile moves more
// operand bytes per product: 2048 x 12288 x 4096, gated, took 1, 0.79, 0.64 and 0.59 of the time per tile with 256, 192, 128 and 64 columns; 30
// stands for a tile's start and end.
inline int pair_bn(int64_t M, int64_t N, bool gated, int multiple, int sms) {
  const int pairs = sms / 2;
  int best = 256;
  int64_t cost = -1;
  for (int bn = 256; bn >= multiple; bn -= multiple) {
    const int64_t w = gated ? bn / 2 : bn, tiles = ((M + 255) / 256) * ((N + w - 1) / w), waves = (tiles + pairs - 1) / pairs;
    const int64_t c = waves * (30 + (bn == 256 ? 256 : bn == 192 ? 203 : bn == 128 ? 165 : 152));
    if (cost < 0 || c < cost) { cost = c; best = bn; }
  }
  return best;
}

// CTAs that share a thin tile's K where the tiles leave SMs idle: as many as the device holds clusters of (15 of 8 CTAs, 33 of 4), with
// twelve k-blocks each, and room for the partial sums.  Whole and shared, us: 2 tokens through 7808 x 512 15.9, 13.8; 8 through 512 x 8192 17.8,
// 13.1; 8 bits, 100 tokens by 256 x 16384 24.2, 12.9, 1 by 1024 x 8192 9.4, 8.5; with eight blocks each, 4 by 1024 x 2048, 5.4, 5.8.
inline int thin_split(int64_t tiles, int warp_bytes, int64_t nkb, int sms) {
  for (int s = 8; s > 1; s /= 2)
    if (tiles * s <= (s == 8 ? sms * 4 / 5 : s == 4 ? sms * 8 / 9 : sms) && nkb >= 12 * s && thin_after(warp_bytes, s) <= 180 * 1024) return s;
  return 1;
}

struct Operand {
  const void* base;
  int64_t rows, inner, ld;   // elements; ld * element size is a multiple of 16
};

// A 16-bit result that the pair kernel stores by TMA: its address a multiple of 16 bytes, ld of 8 values.  Where `cols` is not, a store
// writes up to 7 values beyond them.
struct Result {
  void* at;
  int64_t cols, ld;
};

// A product of A (M rows) and B with operator Op.  b_mn: B lies K x N (N contiguous) instead of N x K.  gave_up: the plan's word, or NULL.
template <class Op, bool B_MN>
exo_gemm_status_t launch_pair(int bn, const Operand& A, const Operand& B, int64_t N, int64_t K, int64_t b_split, bool bf16, int sms,
                              const typename Op::Params& op, std::initializer_list<Result> results, uint32_t* gave_up, cudaStream_t stream) {
  constexpr int ES = Op::kInt8 ? 1 : 2, SUB_K = 128 / ES;
  const int width = Op::kGated ? bn / 2 : bn;
  CoreParams p{};
  p.M = (int32_t)A.rows;
  p.N = (int32_t)N;
  p.nkb = (int32_t)((K + SUB_K - 1) / SUB_K);
  p.width = width;
  p.buffers = Op::kTogether && results.size() + Op::kMore > 2 ? 3 : 2;
  p.stages = pair_stages(bn, p.buffers);
  p.b_split = (int32_t)(Op::kGated ? b_split : bn / 2);
  p.idesc = Op::kInt8 ? (2u << 4 | 1u << 7 | 1u << 10 | (uint32_t)(bn >> 3) << 17 | 16u << 24)   // signed bytes, 32-bit integer sums
                      : make_idesc(bf16 ? EXO_GEMM_BF16 : EXO_GEMM_FP16, 0, B_MN ? 1 : 0, 256, bn);
  p.a = make_staging(0, kBlockM, 1, 2);   // (128 bytes of K per row whatever the type)
  p.b = make_staging(B_MN ? 1 : 0, bn / 2, 1, 2);
  const int32_t tiles_m = (int32_t)((A.rows + 255) / 256), tiles_n = (int32_t)((N + width - 1) / width);
  // Bands of 8 tile columns: the 74 tiles at work then cover about 9 x 8 tiles, whose rows of A and B L2 holds.
  p.raster = make_raster(tiles_m, tiles_n, 8, 0);
  const int64_t tiles = (int64_t)tiles_m * tiles_n;
  if (tiles >= (1LL << 31)) return EXO_GEMM_ERR_UNSUPPORTED;
  CUtensorMap ma, mb;
  if (!encode_operand_map(&ma, ES, bf16, A.base, (uint64_t)A.inner, (uint64_t)A.rows, (uint64_t)(A.ld * ES), 128) ||
      !encode_operand_map(&mb, ES, bf16, B.base, (uint64_t)B.inner, (uint64_t)B.rows, (uint64_t)(B.ld * ES), B_MN ? 64u : (uint32_t)bn / 2))
    return EXO_GEMM_ERR_CUDA;
  const WaitHook hook = take_wait_hook();
  p.waits = Waits{hook.clocks, gave_up};
  p.skip_copies = hook.skip;
  OutMaps mo;
  memset(&mo, 0, sizeof mo);
  int n = 0;
  for (const Result& r : results)
    if (!encode_result_map(&mo.m[n++], r.at, (uint64_t)r.cols, (uint64_t)A.rows, (uint64_t)r.ld * 2)) return EXO_GEMM_ERR_CUDA;
  const int64_t pairs = tiles < sms / 2 ? tiles : sms / 2;
  typename Op::Params o = op;
  void* args[5] = {&ma, &mb, &mo, &p, &o};
  return launch_args((void*)exo_fused_pair_kernel<Op, B_MN>, dim3((unsigned)(2 * pairs)), kNumThreads, (size_t)pair_smem(bn, p.buffers), 2, stream, args);
}

template <class Op, int U>
exo_gemm_status_t launch_thin(int width, const Operand& A, const Operand& B, int64_t N, int64_t K, int64_t b_split, bool bf16,
                              int sms, const typename Op::Params& op, uint32_t* gave_up, cudaStream_t stream) {
  constexpr int ES = Op::kInt8 ? 1 : 2, SUB_K = 128 / ES;
  constexpr int PARTS = Op::kGated ? 2 : 1;
  const int a_rows = (int)round_up(A.rows, 8);
  int64_t tiles = (N + width - 1) / width;
  const int64_t nkb = (K + SUB_K - 1) / SUB_K;
  // Where a tile stages twice as many rows of A as of B, tiles of twice the width and half of K each move a third less: 128 tokens through
  // 4096 x 10240 63.7 us, 57.3; 8 bits, 100 tokens by 2048 x 8192 15.6, 13.3, but 64 tokens by 4096 x 4096, 32 k-blocks, 9.6, 10.9.  (Not where the
  // rows' parts go by the tile.)
  const bool wide = !Op::kTwice && tiles <= sms && a_rows >= 2 * PARTS * width && 2 * PARTS * width <= 256 && nkb >= 48;
  if (wide) {
    width *= 2;
    tiles = (N + width - 1) / width;
  }
  const int bn = PARTS * width;
  CoreParams p{};
  p.M = (int32_t)A.rows;
  p.N = (int32_t)N;
  p.nkb = (int32_t)nkb;
  p.width = width;
  p.a_rows = a_rows;
  const int mma_rows = thin_mma_rows(a_rows);
  p.quad_rows = mma_rows / 4;
  p.whole = (int32_t)(K / SUB_K);
  const int warp_bytes = (width / U + 1) / 2 * PARTS * U * 128;   // of partial sums
  p.split = thin_split(tiles, warp_bytes, p.nkb, sms);
  const int after = thin_after(warp_bytes, p.split);
  thin_ring(bn, a_rows, p.whole / p.split, tiles <= sms, after, &p.per_stage, &p.stages);
  p.idesc = Op::kInt8 ? (2u << 4 | 1u << 7 | 1u << 10 | (uint32_t)(bn >> 3) << 17 | (uint32_t)(mma_rows >> 4) << 24)
                      : make_idesc(bf16 ? EXO_GEMM_BF16 : EXO_GEMM_FP16, 0, 0, mma_rows, bn);
  p.a = make_staging(0, kBlockM, 1, 2);
  p.b = make_staging(0, bn, 1, 2);
  CUtensorMap ma, ma_rest, mb, mb_rest;
  const uint64_t parts = Op::kGated ? 2 : 1, part_bytes = (uint64_t)b_split * (uint64_t)(B.ld * ES);
  if (!encode_blocks_map(&ma, &ma_rest, ES, bf16, A.base, (uint64_t)A.inner, (uint64_t)A.rows, (uint64_t)(A.ld * ES), 1, 0, (uint32_t)a_rows, (uint32_t)p.per_stage) ||
      !encode_blocks_map(&mb, &mb_rest, ES, bf16, B.base, (uint64_t)B.inner, (uint64_t)N, (uint64_t)(B.ld * ES), parts, part_bytes, (uint32_t)width,
                         (uint32_t)p.per_stage))
    return EXO_GEMM_ERR_CUDA;
  const WaitHook hook = take_wait_hook();
  p.waits = Waits{hook.clocks, gave_up};
  p.skip_copies = hook.skip;
  typename Op::Params o = op;
  void* args[6] = {&ma, &ma_rest, &mb, &mb_rest, &p, &o};
  return launch_args((void*)exo_fused_thin_kernel<Op, U>, dim3((unsigned)(tiles * p.split)), kThinThreads,
                     (size_t)thin_smem(p.stages, p.per_stage, bn, a_rows, after), (unsigned)p.split, stream, args);
}

// dst = src, `rows` rows of `inner` 16-bit values; dst's rows start on 16 bytes and have room for a multiple of 8 values.
// beside: behind a kernel of this header whose results it does not touch, and beside it: that kernel has waited for all before it when this
// one starts, and this one ends after it.
exo_gemm_status_t align_rows(void* dst, int64_t dst_ld, const void* src, int64_t src_ld, int64_t inner, int64_t rows, cudaStream_t stream,
                             bool beside = false);   // i8.cu

// Device memory of a plan.
struct Memory {
  static constexpr int kMost = 12;
  void* parts[kMost] = {};
  int count = 0;
  int64_t bytes = 0;
  cudaError_t err = cudaSuccess;
  void* take(int64_t n) {
    void* p = nullptr;
    if (err != cudaSuccess || n <= 0) return nullptr;
    if (count == kMost) { err = cudaErrorMemoryAllocation; return nullptr; }
    err = cudaMalloc(&p, (size_t)n);
    if (err != cudaSuccess) return nullptr;
    parts[count++] = p;
    bytes += n;
    return p;
  }
  // a word of a plan's waits, clear when it returns
  uint32_t* take_word() {
    uint32_t* const p = (uint32_t*)take(sizeof(uint32_t));
    if (p) err = clear_now(p, sizeof(uint32_t));
    return p;
  }
  void give_back() {
    for (int i = 0; i < count; ++i) cudaFree(parts[i]);
    count = 0;
  }
};

unsigned take_gave_up_i8(cudaError_t* e);
unsigned take_gave_up_ffn(cudaError_t* e);
unsigned take_gave_up_ce(cudaError_t* e);
// of this translation unit's kernels, on the current device
static inline unsigned take_gave_up_here(cudaError_t* e) {
  unsigned n = 0, zero = 0;
  *e = cudaMemcpyFromSymbol(&n, fused_gave_up, sizeof n);
  if (*e == cudaSuccess && n) *e = cudaMemcpyToSymbol(fused_gave_up, &zero, sizeof zero);
  return n;
}
// What exo_ffn_check and exo_ce_check do: the plan's own word, and exo_gemm_check of its products.  On the plan's device.
inline exo_gemm_status_t check_plan(uint32_t* gave_up, std::initializer_list<exo_gemm_handle_t> plans) {
  cudaError_t e = cudaDeviceSynchronize();
  uint32_t n = 0;
  if (e == cudaSuccess && gave_up) e = cudaMemcpy(&n, gave_up, sizeof n, cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && n) e = clear_now(gave_up, sizeof n);
  if (e != cudaSuccess) return cuda_failed(e);
  exo_gemm_status_t st = n ? EXO_GEMM_ERR_DEVICE_TIMEOUT : EXO_GEMM_OK;
  for (exo_gemm_handle_t g : plans)
    if (g) {
      const exo_gemm_status_t s = exo_gemm_check(g, nullptr);
      if (st == EXO_GEMM_OK) st = s;
    }
  return st;
}

}  // namespace fused
}  // namespace exo

// 4-bit weights: quantisation, its inverse, and the product of a few tokens with a 4-bit matrix (exo_decode.h).
#include <cooperative_groups.h>

#include "../../include/exo_decode.h"
#include "decode_core.cuh"
#include "decode_host.h"
#include "ptx.cuh"

namespace exo {
namespace decode {
namespace {

// ==== quantisation ===============================================================================================
// A lane holds eight consecutive weights, so a group is 16, 8 or 4 neighbouring lanes and its extremes are a shuffle
// tree; a warp walks along a row, 256 weights at a time.  Bound by memory: 2 (4) bytes in and 1/2 out per weight,
// and the division by the scale (IEEE, so that codes are the formula's) hides behind it.
constexpr int kQuantThreads = 256;
constexpr int kQuantSegment = 4096;   // weights of a row per warp

template <class T, class W> struct Source;   // eight weights as floats, and back
template <class T> struct Source<T, uint16_t> {
  static __device__ __forceinline__ void load(const uint16_t* row, int k, int K, bool aligned, float (&v)[8]) {
    const uint4 r = load8_checked(row, k, K, aligned);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = T::to_float((uint16_t)(w[i / 2] >> (16 * (i % 2))));
  }
  static __device__ __forceinline__ void store(uint16_t* row, int k, int K, bool aligned, const float (&v)[8]) {
    if (aligned && k + 8 <= K) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (uint32_t)T::from_float(v[2 * i]) | (uint32_t)T::from_float(v[2 * i + 1]) << 16;
      *reinterpret_cast<uint4*>(row + k) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (k + i < K) row[k + i] = T::from_float(v[i]);
    }
  }
};
template <class T> struct Source<T, float> {
  static __device__ __forceinline__ void load(const float* row, int k, int K, bool aligned, float (&v)[8]) {
    if (aligned && k + 8 <= K) {
      const float4 a = *reinterpret_cast<const float4*>(row + k), b = *reinterpret_cast<const float4*>(row + k + 4);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = k + i < K ? row[k + i] : 0.f;
    }
  }
  static __device__ __forceinline__ void store(float* row, int k, int K, bool aligned, const float (&v)[8]) {
    if (aligned && k + 8 <= K) {
      *reinterpret_cast<float4*>(row + k) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(row + k + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (k + i < K) row[k + i] = v[i];
    }
  }
};

struct QuantParams {
  int64_t rows, ldw;
  int K, blocks, segments, group;
  void* w;
  uint32_t* codes;
  uint16_t* scales;
  uint8_t* zeros;
  bool aligned;
};

// T: type of the scales.  WT/W: type of the weights (a 16-bit type with its format, or float).
template <class T, class WT, class W>
__global__ void __launch_bounds__(kQuantThreads) exo_q4_quantize_kernel(const QuantParams p) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int64_t item = ((int64_t)blockIdx.x * kQuantThreads + threadIdx.x) >> 5;
  const int64_t row = item / p.segments;
  if (row >= p.rows) return;
  const int seg = (int)(item - row * p.segments);
  const int k_end = min((seg + 1) * (kQuantSegment / 128), p.blocks) * 128;
  const W* src = static_cast<const W*>(p.w) + row * p.ldw;
  const int lanes = p.group / 8, per_row = p.blocks * 128 / p.group;
#pragma unroll 2
  for (int k0 = seg * kQuantSegment; k0 < k_end; k0 += 256) {
    const int k = k0 + 8 * lane;
    float v[8];
    Source<WT, W>::load(src, k, p.K, p.aligned, v);
    float lo = 0.f, hi = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) { lo = fminf(lo, v[i]); hi = fmaxf(hi, v[i]); }
    for (int o = 1; o < lanes; o <<= 1) {
      lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    const float raw = p.zeros ? __fdiv_rn(hi - lo, 15.f) : __fdiv_rn(fmaxf(hi, -lo), 7.f);
    const uint16_t s16 = T::from_float(fminf(raw, T::max_finite()));
    const float s = T::to_float(s16);
    float zero = 8.f;
    if (p.zeros && s > 0.f) zero = fminf(fmaxf(rintf(__fdiv_rn(-lo, s)), 0.f), 15.f);
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float q = s > 0.f ? rintf(__fdiv_rn(v[i], s)) + zero : zero;   // symmetric: -8 .. 7 plus 8
      word |= (uint32_t)fminf(fmaxf(q, 0.f), 15.f) << (4 * (i / 2 + 4 * (i % 2)));
    }
    if (k < k_end) {   // the last pass may hold one block of 128 only
      const int l = lane & 15;
      p.codes[(row * p.blocks + k / 128) * 16 + 4 * (l & 3) + (l >> 2)] = word;
      if ((lane & (lanes - 1)) == 0) {
        p.scales[row * per_row + k / p.group] = s16;
        if (p.zeros) p.zeros[row * per_row + k / p.group] = (uint8_t)zero;
      }
    }
  }
}

template <class T, class WT, class W>
__global__ void __launch_bounds__(kQuantThreads) exo_q4_dequantize_kernel(const QuantParams p) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int64_t item = ((int64_t)blockIdx.x * kQuantThreads + threadIdx.x) >> 5;
  const int64_t row = item / p.segments;
  if (row >= p.rows) return;
  const int seg = (int)(item - row * p.segments);
  const int k_end = min((seg + 1) * (kQuantSegment / 128), p.blocks) * 128;
  W* dst = static_cast<W*>(p.w) + row * p.ldw;
  const int per_row = p.blocks * 128 / p.group;
#pragma unroll 4
  for (int k0 = seg * kQuantSegment; k0 < k_end; k0 += 256) {
    const int k = k0 + 8 * lane;
    if (k < k_end) {
      const int l = lane & 15;
      const uint32_t word = p.codes[(row * p.blocks + k / 128) * 16 + 4 * (l & 3) + (l >> 2)];
      const float s = T::to_float(p.scales[row * per_row + k / p.group]);
      const int zero = p.zeros ? (int)p.zeros[row * per_row + k / p.group] : 8;
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (float)((int)(word >> (4 * (i / 2 + 4 * (i % 2))) & 15u) - zero) * s;
      Source<WT, W>::store(dst, k, p.K, p.aligned, v);
    }
  }
}

// ==== the product of a few tokens with a 4-bit matrix =============================================================
// A CTA's eight warps are `wr` groups of 16 weight rows times 8 / wr parts of its steps of k; the CTAs of a cluster
// share the rows and split k.  The tokens' values for the CTA's part of k are staged in shared memory (rows 64 bytes off
// a multiple of 128, so that a fragment load is free of bank conflicts).  Partial sums meet in shared memory in warp
// order, then in distributed shared memory in rank order.
constexpr int kGemvThreads = 256, kGemvWarps = 8;

struct GemvParams {
  const uint8_t* codes;
  const uint16_t* scales;
  const uint8_t* zeros;
  const uint16_t* x;
  void* y;
  int64_t ldx, ldy, rows;
  int K, tokens, blocks;        // blocks: steps of 128
  int wr;                       // warps across rows: 1, 2, 4 or 8
  int chunk;                    // steps staged at a time
  int y_dtype;
  bool x_aligned;
  float alpha, beta;
};

__host__ __device__ constexpr int gemv_pitch(int chunk) { return chunk * 256 + 64; }   // bytes of a token's staged row

template <class T>
__device__ __forceinline__ void store_y(const GemvParams& p, int token, int64_t row, float v) {
  if (token >= p.tokens || row >= p.rows) return;
  const int64_t at = (int64_t)token * p.ldy + row;
  v *= p.alpha;
  if (p.y_dtype == EXO_GEMM_FP32) {
    float* y = static_cast<float*>(p.y);
    y[at] = p.beta != 0.f ? fmaf(p.beta, y[at], v) : v;
  } else {
    uint16_t* y = static_cast<uint16_t*>(p.y);
    y[at] = T::from_float(p.beta != 0.f ? fmaf(p.beta, T::to_float(y[at]), v) : v);
  }
}

template <class T, int PER, int NT>
__global__ void __launch_bounds__(kGemvThreads) exo_gemv_q4_kernel(const GemvParams p) {
  namespace cg = cooperative_groups;
  extern __shared__ __align__(128) uint8_t smem[];
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), r = (int)cluster.block_rank();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int wr = warp % p.wr, wk = warp / p.wr, nk = kGemvWarps / p.wr;
  const int64_t tile_row = (int64_t)(blockIdx.x / S) * 16 * p.wr;
  const int64_t row0 = min(tile_row + 16 * wr + g, p.rows - 1), row1 = min(tile_row + 16 * wr + g + 8, p.rows - 1);
  const int s_begin = (int)((int64_t)p.blocks * r / S), s_end = (int)((int64_t)p.blocks * (r + 1) / S);
  const int nt = (p.tokens + 7) / 8;

  RowsQ4<T, PER> f;
  f.c0 = p.codes + row0 * p.blocks * 64;
  f.c1 = p.codes + row1 * p.blocks * 64;
  f.s0 = p.scales + row0 * p.blocks * PER;
  f.s1 = p.scales + row1 * p.blocks * PER;
  f.z0 = p.zeros ? p.zeros + row0 * p.blocks * PER : nullptr;
  f.z1 = p.zeros ? p.zeros + row1 * p.blocks * PER : nullptr;

  float acc[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;

  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int pitch = gemv_pitch(p.chunk);
  constexpr int DEPTH = NT <= 2 ? 4 : 2;
  Stream<RowsQ4<T, PER>, DEPTH> stream;
  for (int c = s_begin; c < s_end; c += p.chunk) {
    const int c_end = min(c + p.chunk, s_end);
    stream.preload(f, c + wk, nk, c_end, p.K, t);
    if (c != s_begin) __syncthreads();   // the previous chunk has been read
    const int per_token = (c_end - c) * 16;
    for (int i = threadIdx.x; i < p.tokens * per_token; i += kGemvThreads) {
      const int token = i / per_token, e = i - token * per_token;
      *reinterpret_cast<uint4*>(smem + token * pitch + e * 16) =
          load8_checked(p.x + (int64_t)token * p.ldx, c * 128 + e * 8, p.K, p.x_aligned);
    }
    __syncthreads();
    const uint8_t* mine = smem + g * pitch - c * 256;
    stream.template walk<NT>(f, c + wk, nk, c_end, p.K, t, [&](int i, int k) {
      return 8 * i + g < p.tokens ? *reinterpret_cast<const uint4*>(mine + 8 * i * pitch + 2 * k) : make_uint4(0, 0, 0, 0);
    }, nt, acc);
  }

  // sums over the warps that share rows, then over the cluster
  __syncthreads();
  float4* red = reinterpret_cast<float4*>(smem);                        // [warp][nt][lane]
  float4* part = red + kGemvWarps * nt * 32;                            // [wr][nt][lane]
#pragma unroll
  for (int i = 0; i < NT; ++i)
    if (i < nt) red[(warp * nt + i) * 32 + lane] = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
  __syncthreads();
  const int items = p.wr * nt * 32;
  auto finish = [&](int idx, float4 v) {
    const int l = idx & 31, i = (idx >> 5) % nt, w = (idx >> 5) / nt;
    const int64_t row = tile_row + 16 * w + (l >> 2);
    const int token = 8 * i + 2 * (l & 3);
    store_y<T>(p, token, row, v.x);
    store_y<T>(p, token + 1, row, v.y);
    store_y<T>(p, token, row + 8, v.z);
    store_y<T>(p, token + 1, row + 8, v.w);
  };
  for (int idx = threadIdx.x; idx < items; idx += kGemvThreads) {
    float4 v = red[idx];
    for (int q = 1; q < nk; ++q) {
      const float4 w = red[q * items + idx];
      v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
    }
    if (S == 1) finish(idx, v);
    else part[idx] = v;
  }
  if (S > 1) {
    cluster.sync();
    for (int idx = r * kGemvThreads + threadIdx.x; idx < items; idx += S * kGemvThreads) {
      float4 v = cluster.map_shared_rank(part, 0)[idx];
      for (int q = 1; q < S; ++q) {
        const float4 w = cluster.map_shared_rank(part, q)[idx];
        v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
      }
      finish(idx, v);
    }
    cluster.sync();   // no CTA leaves while another may still read its sums
  }
}

// Y = beta * Y, for alpha == 0 or K == 0
template <class T>
__global__ void __launch_bounds__(kGemvThreads) exo_gemv_q4_scale_kernel(const GemvParams p) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int64_t row = (int64_t)blockIdx.x * kGemvThreads + threadIdx.x;
  for (int token = 0; token < p.tokens; ++token) store_y<T>(p, token, row, 0.f);
}

using GemvFn = void (*)(GemvParams);
template <class T, int PER> GemvFn pick_nt(int nt) {
  return nt == 1 ? exo_gemv_q4_kernel<T, PER, 1> : nt == 2 ? exo_gemv_q4_kernel<T, PER, 2>
         : nt <= 4 ? exo_gemv_q4_kernel<T, PER, 4> : exo_gemv_q4_kernel<T, PER, 8>;
}
template <class T> GemvFn pick_gemv(int group, int nt) {
  return group == 128 ? pick_nt<T, 1>(nt) : group == 64 ? pick_nt<T, 2>(nt) : pick_nt<T, 4>(nt);
}

exo_gemm_status_t check_q4(const exo_q4_t* q) {
  if (!q) return EXO_GEMM_ERR_NULL;
  if (q->rows < 0 || q->K < 0 || q->rows > (1LL << 40) || q->K > (1LL << 30)) return EXO_GEMM_ERR_INVALID_ARG;
  if (q->group != 32 && q->group != 64 && q->group != 128) return EXO_GEMM_ERR_INVALID_ARG;
  if (q->dtype != EXO_GEMM_BF16 && q->dtype != EXO_GEMM_FP16) return EXO_GEMM_ERR_INVALID_ARG;
  return EXO_GEMM_OK;
}
exo_gemm_status_t check_q4_pointers(const exo_q4_t* q) {
  if (!q->codes || !q->scales) return EXO_GEMM_ERR_NULL;
  return q4_aligned(q->codes, q->scales, q->zeros, q->group) ? EXO_GEMM_OK : EXO_GEMM_ERR_ALIGNMENT;
}
int blocks_of(int64_t K) { return (int)((K + 127) / 128); }

template <class T>
void* quant_fn(int w_dtype, bool back) {
  if (w_dtype == EXO_GEMM_FP32) return back ? (void*)exo_q4_dequantize_kernel<T, T, float> : (void*)exo_q4_quantize_kernel<T, T, float>;
  if (w_dtype == EXO_GEMM_BF16) return back ? (void*)exo_q4_dequantize_kernel<T, Bf16, uint16_t> : (void*)exo_q4_quantize_kernel<T, Bf16, uint16_t>;
  return back ? (void*)exo_q4_dequantize_kernel<T, Fp16, uint16_t> : (void*)exo_q4_quantize_kernel<T, Fp16, uint16_t>;
}

exo_gemm_status_t run_quant(const exo_q4_t* q, void* W, int64_t ldw, int32_t w_dtype, bool back, void* cuda_stream) {
  exo_gemm_status_t st = check_q4(q);
  if (st != EXO_GEMM_OK) return st;
  if (ldw < (q->K > 1 ? q->K : 1) || w_dtype < EXO_GEMM_BF16 || w_dtype > EXO_GEMM_FP32) return EXO_GEMM_ERR_INVALID_ARG;
  if (q->rows == 0 || q->K == 0) return EXO_GEMM_OK;
  if (!W) return EXO_GEMM_ERR_NULL;
  if ((st = check_q4_pointers(q)) != EXO_GEMM_OK) return st;
  const int bytes = w_dtype == EXO_GEMM_FP32 ? 4 : 2;
  if ((uintptr_t)W & (unsigned)(bytes - 1)) return EXO_GEMM_ERR_ALIGNMENT;
  int sms = 0;
  if ((st = device_check(&sms)) != EXO_GEMM_OK) return st;
  QuantParams p{};
  p.rows = q->rows; p.ldw = ldw; p.K = (int)q->K; p.blocks = blocks_of(q->K); p.group = q->group;
  p.segments = (p.blocks * 128 + kQuantSegment - 1) / kQuantSegment;
  p.w = W; p.codes = (uint32_t*)q->codes; p.scales = (uint16_t*)q->scales; p.zeros = q->zeros;
  p.aligned = ((uintptr_t)W & 15u) == 0 && (ldw * bytes) % 16 == 0;
  const int64_t ctas = (p.rows * p.segments + kQuantThreads / 32 - 1) / (kQuantThreads / 32);
  if (ctas >= (1LL << 31)) return EXO_GEMM_ERR_UNSUPPORTED;
  void* fn = q->dtype == EXO_GEMM_BF16 ? quant_fn<Bf16>(w_dtype, back) : quant_fn<Fp16>(w_dtype, back);
  return launch(fn, (unsigned)ctas, 1, kQuantThreads, 0, 1, (cudaStream_t)cuda_stream, &p);
}

}  // namespace
}  // namespace decode
}  // namespace exo

using namespace exo::decode;

extern "C" exo_gemm_status_t exo_q4_quantize(const exo_q4_t* q, const void* W, int64_t ldw, int32_t w_dtype, void* cuda_stream) {
  return run_quant(q, const_cast<void*>(W), ldw, w_dtype, false, cuda_stream);
}

extern "C" exo_gemm_status_t exo_q4_dequantize(const exo_q4_t* q, void* W, int64_t ldw, int32_t w_dtype, void* cuda_stream) {
  return run_quant(q, W, ldw, w_dtype, true, cuda_stream);
}

extern "C" exo_gemm_status_t exo_gemv_q4_run(const exo_q4_t* W, int64_t tokens, const void* X, int64_t ldx, void* Y, int64_t ldy,
                                             int32_t y_dtype, float alpha, float beta, void* cuda_stream) {
  exo_gemm_status_t st = check_q4(W);
  if (st != EXO_GEMM_OK) return st;
  if (tokens < 0 || ldx < (W->K > 1 ? W->K : 1) || ldy < (W->rows > 1 ? W->rows : 1)) return EXO_GEMM_ERR_INVALID_ARG;
  if (y_dtype != EXO_GEMM_FP32 && y_dtype != W->dtype) return EXO_GEMM_ERR_INVALID_ARG;
  if (tokens > 64) return EXO_GEMM_ERR_UNSUPPORTED;
  if (tokens == 0 || W->rows == 0) return EXO_GEMM_OK;
  const bool read = alpha != 0.f && W->K > 0;
  if (!Y || (read && !X)) return EXO_GEMM_ERR_NULL;
  if (read && (st = check_q4_pointers(W)) != EXO_GEMM_OK) return st;
  if (((uintptr_t)X & 1u) || ((uintptr_t)Y & (y_dtype == EXO_GEMM_FP32 ? 3u : 1u))) return EXO_GEMM_ERR_ALIGNMENT;
  int sms = 0;
  if ((st = device_check(&sms)) != EXO_GEMM_OK) return st;
  GemvParams p{};
  p.codes = (const uint8_t*)W->codes; p.scales = (const uint16_t*)W->scales; p.zeros = W->zeros;
  p.x = (const uint16_t*)X; p.y = Y; p.ldx = ldx; p.ldy = ldy; p.rows = W->rows;
  p.K = (int)W->K; p.tokens = (int)tokens; p.blocks = blocks_of(W->K);
  p.y_dtype = y_dtype; p.alpha = alpha; p.beta = beta;
  p.x_aligned = ((uintptr_t)X & 15u) == 0 && ldx % 8 == 0;
  const bool bf16 = W->dtype == EXO_GEMM_BF16;
  if (!read) {
    const int64_t ctas = (p.rows + kGemvThreads - 1) / kGemvThreads;
    if (ctas >= (1LL << 31)) return EXO_GEMM_ERR_UNSUPPORTED;
    return launch(bf16 ? (void*)exo_gemv_q4_scale_kernel<Bf16> : (void*)exo_gemv_q4_scale_kernel<Fp16>, (unsigned)ctas, 1,
                  kGemvThreads, 0, 1, (cudaStream_t)cuda_stream, &p);
  }
  // A CTA reads its part of X once for 16 * wr weight rows: more rows for more tokens.  Then the cluster cuts k until the
  // grid fills the device twice, as long as a warp keeps a step.
  p.wr = tokens <= 2 ? 1 : tokens <= 8 ? 4 : 8;
  const int64_t tiles = (p.rows + 16 * p.wr - 1) / (16 * p.wr);
  const int nk = kGemvWarps / p.wr, nt = (p.tokens + 7) / 8;
  int S = 1;
  while (S < 8 && tiles * S < 2 * sms && p.blocks >= 2 * S * nk) S *= 2;
  if (tiles * S >= (1LL << 31)) return EXO_GEMM_ERR_UNSUPPORTED;
  const int mine = (p.blocks + S - 1) / S;
  // staged activations: all of the CTA's part of k where that leaves room for two CTAs per SM
  const int most = (100 * 1024 / p.tokens - 64) / 256;
  p.chunk = mine < most ? mine : most;
  size_t smem = (size_t)p.tokens * gemv_pitch(p.chunk);
  const size_t reduce = (size_t)(kGemvWarps + p.wr) * nt * 512;
  if (smem < reduce) smem = reduce;
  GemvFn fn = bf16 ? pick_gemv<Bf16>(W->group, nt) : pick_gemv<Fp16>(W->group, nt);
  return launch((void*)fn, (unsigned)(tiles * S), 1, kGemvThreads, smem, (unsigned)S, (cudaStream_t)cuda_stream, &p);
}

// 8-bit integers with a scale per row, their products, and what the operators of exo_fused.h share: aligned copies, the state of device-side
// waits.
#include <new>

#include "fused_host.h"

namespace exo {
namespace fused {
namespace {

// ---------------------------------------------------------------- quantisation
// A CTA per row: the largest magnitude, then the codes, from registers.  Bound by memory for many rows (2 + 1 bytes a value) and by the
// latency of a load, a reduction and a store for few.
struct QuantParams {
  const void* x;
  int64_t ldx;
  int8_t* codes;
  int64_t ld;
  float* scales;
  int32_t K;
};
template <class T> struct Element { using type = uint16_t; };
template <> struct Element<float> { using type = float; };

// V values from k on as fp32
template <class T, int V>
__device__ __forceinline__ void load_values(const typename Element<T>::type* x, int k, float (&v)[V]) {
  if constexpr (std::is_same<T, float>::value) {
    if (V == 4) {
      const float4 w = *reinterpret_cast<const float4*>(x + k);
      v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
    } else {
      v[0] = x[k];
    }
  } else if constexpr (V == 8) {
    const uint4 w = *reinterpret_cast<const uint4*>(x + k);
    const float2 a = T::unpack(w.x), b = T::unpack(w.y), c = T::unpack(w.z), d = T::unpack(w.w);
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y; v[4] = c.x; v[5] = c.y; v[6] = d.x; v[7] = d.y;
  } else {
    v[0] = T::unpack(x[k]).x;
  }
}

// Codes: the quotient rounded as IEEE division rounds it, then to the nearest integer, ties to even.  The product with the rounded
// reciprocal is within 2^-22 of the quotient, relative, so both round to the same integer unless the product is within 127 * 2^-22 of a tie; there,
// and for scales whose reciprocal is not a normal number, the division is made.
struct Divider {
  float scale, inverse;
  bool safe;
  __device__ __forceinline__ explicit Divider(float s) : scale(s), inverse(1.f / s), safe(s > 0x1p-120f && s < 0x1p120f) {}
  __device__ __forceinline__ int code(float x) const {
    float q = x * inverse, r = rintf(q);
    if (!safe || fabsf(fabsf(q - r) - 0.5f) < 0x1p-14f) r = rintf(__fdiv_rn(x, scale));
    return (int)fminf(fmaxf(r, -127.f), 127.f);
  }
};

// V: values per load, 16 bytes of them where the rows allow that, else one.  THREADS per row; a thread keeps its first kHeld loads in
// registers, further ones are read again.
constexpr int kHeld = 8;
template <class T, int V, int THREADS>
__global__ void __launch_bounds__(THREADS) exo_i8_quantize_kernel(const QuantParams p) {
  __shared__ float tops[THREADS / 32];
  using E = typename Element<T>::type;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const E* x = (const E*)p.x + (int64_t)blockIdx.x * p.ldx;
  int8_t* codes = p.codes + (int64_t)blockIdx.x * p.ld;
  const int whole = p.K / V * V;   // the values of whole loads; the others one by one
  const int first = threadIdx.x * V;
  constexpr int STEP = THREADS * V;
  float top = 0.f, held[kHeld][V];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    if (first + i * STEP < whole) {
      load_values<T, V>(x, first + i * STEP, held[i]);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) held[i][j] = 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) top = fmaxf(top, fabsf(held[i][j]));
#pragma unroll 4
  for (int k = first + kHeld * STEP; k < whole; k += STEP) {
    float v[V];
    load_values<T, V>(x, k, v);
#pragma unroll
    for (int j = 0; j < V; ++j) top = fmaxf(top, fabsf(v[j]));
  }
  for (int k = whole + threadIdx.x; k < p.K; k += THREADS) {
    float v[1];
    load_values<T, 1>(x, k, v);
    top = fmaxf(top, fabsf(v[0]));
  }
#pragma unroll
  for (int o = 16; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) top = fmaxf(top, tops[w]);
  const float scale = __fdiv_rn(top, 127.f);
  if (threadIdx.x == 0) p.scales[blockIdx.x] = scale;
  const bool zero = !(scale > 0.f);
  const Divider by(zero ? 1.f : scale);
  auto store = [&](int k, const float (&v)[V]) {
    uint32_t w[(V + 3) / 4] = {};
#pragma unroll
    for (int j = 0; j < V; ++j) w[j / 4] |= (uint32_t)((zero ? 0 : by.code(v[j])) & 255) << (8 * (j & 3));
    if constexpr (V == 8) *reinterpret_cast<uint2*>(codes + k) = make_uint2(w[0], w[1]);
    else if constexpr (V == 4) *reinterpret_cast<uint32_t*>(codes + k) = w[0];
    else codes[k] = (int8_t)w[0];
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (first + i * STEP < whole) store(first + i * STEP, held[i]);
  for (int k = first + kHeld * STEP; k < whole; k += STEP) {
    float v[V];
    load_values<T, V>(x, k, v);
    store(k, v);
  }
  for (int k = whole + threadIdx.x; k < p.K; k += THREADS) {
    float v[1];
    load_values<T, 1>(x, k, v);
    codes[k] = (int8_t)(zero ? 0 : by.code(v[0]));
  }
}

// ---------------------------------------------------------------- products
// Integer sums are exact; a token's scale, its channels' scales and alpha are multiplied on in fp32.
struct I8Op {
  static constexpr bool kInt8 = true, kGated = false, kTwice = false;
  static constexpr int kUnit = 32, kBuffers = 2;   // by pairs
  struct Params {
    const float *xs, *ws;
    void* y;
    int64_t ldy;
    int32_t cols, y_dtype, align;   // align: what divides the address of every unit
    int32_t tma;                    // 16-bit results that are stored by TMA
    float alpha, beta;
  };
  template <int U>
  struct State {
    float xs, ws;   // of the row; of column `lane` of the next unit
  };
  template <int U>
  static __device__ __forceinline__ float scale_of(const Params& o, int col, int N) {
    const int k = (int)ptx::lane_id();
    return k < U && col + k < N ? __ldcg(o.ws + col + k) : 0.f;
  }
  template <int U>
  static __device__ __forceinline__ void begin(const Params& o, State<U>& s, int row, bool row_ok, int col, int N) {
    s.xs = row_ok ? __ldcg(o.xs + row) : 0.f;
    s.ws = scale_of<U>(o, col, N);
  }
  template <int U>
  static __device__ __forceinline__ void unit(const Params& o, State<U>& s, Out& out, uint32_t (&v)[U], uint32_t (&)[1], int row, bool row_ok, int col, int n, bool more) {
    float y[U];
    const float ws = s.ws;
    if (more) s.ws = scale_of<U>(o, col + U, o.cols);
#pragma unroll
    for (int k = 0; k < U; ++k) y[k] = (float)(int32_t)v[k] * s.xs * __shfl_sync(0xffffffffu, ws, k) * o.alpha;
    if constexpr (U == 32) {
      if (o.tma) {
        uint32_t w[16];
        if (o.y_dtype == EXO_GEMM_BF16) pack<Bf16, U>(y, w);
        else pack<Fp16, U>(y, w);
        out.put(0, col, w);
        return;
      }
    }
    const int64_t at = (int64_t)row * o.ldy + col;
    const bool whole = n == U && o.align >= 16;
    if (o.y_dtype == EXO_GEMM_FP32) {
      float* const c = (float*)o.y + at;
      if (o.beta != 0.f && row_ok) {
#pragma unroll
        for (int k = 0; k < U; ++k)
          if (k < n) y[k] = fmaf(o.beta, c[k], y[k]);
      }
      if (whole) {
        if (row_ok) store32<U>(c, y, o.align);
        return;
      }
#pragma unroll
      for (int h = 0; h < U / 16; ++h) {
        uint32_t w[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) w[k] = __float_as_uint(y[16 * h + k]);
        out.write<4>(out.buffers + h * kOutBytes, 0, w);
        out.store_rows<4>(h, (float*)o.y + (int64_t)out.row0 * o.ldy + col + 16 * h, 4 * o.ldy, n - 16 * h < 16 ? n - 16 * h : 16, o.align);
      }
      return;
    }
    uint16_t* const c = (uint16_t*)o.y + at;
    if (o.beta != 0.f && row_ok) {
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (k < n) y[k] = fmaf(o.beta, o.y_dtype == EXO_GEMM_BF16 ? Bf16::unpack(c[k]).x : Fp16::unpack(c[k]).x, y[k]);
    }
    uint32_t w[U / 2];
    if (o.y_dtype == EXO_GEMM_BF16) pack<Bf16, U>(y, w);
    else pack<Fp16, U>(y, w);
    if (whole) {
      if (row_ok) store_words<U>(c, w, n, o.align);
    } else {
      out.write<U / 8>(out.buffers, 0, w);
      out.store_rows<2>(0, (uint16_t*)o.y + (int64_t)out.row0 * o.ldy + col, 2 * o.ldy, n, o.align);
    }
  }
  template <int U>
  static __device__ __forceinline__ void end(const Params&, State<U>&, int, bool, int) {}
};

// Y = beta * Y, where there are no products
struct ScaleYParams {
  void* y;
  int64_t ldy, rows, cols;
  int32_t y_dtype;
  float beta;
};
constexpr int kScaleYThreads = 256;
__global__ void __launch_bounds__(kScaleYThreads) exo_i8_scale_kernel(const ScaleYParams p) {
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  for (int64_t i = (int64_t)blockIdx.x * kScaleYThreads + threadIdx.x; i < p.rows * p.cols; i += (int64_t)gridDim.x * kScaleYThreads) {
    const int64_t at = i / p.cols * p.ldy + i % p.cols;
    if (p.y_dtype == EXO_GEMM_FP32) {
      float* c = (float*)p.y + at;
      *c = p.beta != 0.f ? p.beta * *c : 0.f;
    } else if (p.y_dtype == EXO_GEMM_BF16) {
      uint16_t* c = (uint16_t*)p.y + at;
      *c = (uint16_t)Bf16::pack(p.beta != 0.f ? p.beta * Bf16::unpack(*c).x : 0.f, 0.f);
    } else {
      uint16_t* c = (uint16_t*)p.y + at;
      *c = (uint16_t)Fp16::pack(p.beta != 0.f ? p.beta * Fp16::unpack(*c).x : 0.f, 0.f);
    }
  }
}

// ---------------------------------------------------------------- aligned copies
constexpr int kAlignThreads = 128;   // (with 40 registers at most, so that they fit an SM beside a CTA of a pair)
struct AlignParams {
  uint16_t* dst;
  const uint16_t* src;
  int64_t dst_ld, src_ld, inner, rows, chunks;   // chunks: of eight values, per row
  int32_t word;                                  // bytes that divide the address of every source row: 2, 4 or 8
  int32_t beside;
};
// A thread moves eight values at a time: 16 bytes out, in as wide pieces as the source's rows allow; four of them are on their way together.
__global__ void __launch_bounds__(kAlignThreads) exo_fused_align_kernel(const AlignParams p) {
  if (!p.beside) ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int64_t all = p.rows * p.chunks, step = (int64_t)gridDim.x * kAlignThreads;
  for (int64_t i0 = (int64_t)blockIdx.x * kAlignThreads + threadIdx.x; i0 < all; i0 += 4 * step) {
    uint32_t w[4][4];
    int64_t to[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t i = i0 + q * step;
      to[q] = -1;
      if (i >= all) continue;
      const int64_t row = i / p.chunks, k = (i - row * p.chunks) * 8;
      const uint16_t* s = p.src + row * p.src_ld + k;
      to[q] = row * p.dst_ld + k;
      if (k + 8 <= p.inner && p.word >= 8) {
        const uint2 a = *reinterpret_cast<const uint2*>(s), b = *reinterpret_cast<const uint2*>(s + 4);
        w[q][0] = a.x; w[q][1] = a.y; w[q][2] = b.x; w[q][3] = b.y;
      } else if (k + 8 <= p.inner && p.word >= 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[q][j] = reinterpret_cast<const uint32_t*>(s)[j];
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[q][j] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (k + j < p.inner) w[q][j / 2] |= (uint32_t)s[j] << (16 * (j & 1));
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (to[q] >= 0) ptx::st_global_v4(p.dst + to[q], w[q][0], w[q][1], w[q][2], w[q][3]);
  }
  if (p.beside) ptx::grid_dependency_wait();   // what comes after this kernel comes after the one beside it, too
}

std::atomic<int64_t> wait_hook{0};   // milliseconds * 2 + skip

exo_gemm_status_t check_i8(const exo_i8_t* q) {
  if (!q) return EXO_GEMM_ERR_NULL;
  if (q->rows < 0 || q->K < 0 || q->rows > (1LL << 30) || q->K > (1LL << 30) || q->ld < q->K || q->ld > (1LL << 31)) return EXO_GEMM_ERR_INVALID_ARG;
  return EXO_GEMM_OK;
}
exo_gemm_status_t check_i8_memory(const exo_i8_t* q) {
  if (!q->codes || !q->scales) return EXO_GEMM_ERR_NULL;
  return aligned16(q->codes) && q->ld % 16 == 0 && ((uintptr_t)q->scales & 3u) == 0 ? EXO_GEMM_OK : EXO_GEMM_ERR_ALIGNMENT;
}

template <class T, int V> void* quant_fn(bool wide, int threads) {
  if (wide) return threads == 128 ? (void*)exo_i8_quantize_kernel<T, V, 128> : (void*)exo_i8_quantize_kernel<T, V, 512>;
  return threads == 128 ? (void*)exo_i8_quantize_kernel<T, 1, 128> : (void*)exo_i8_quantize_kernel<T, 1, 512>;
}

}  // namespace

WaitHook take_wait_hook() {
  const int64_t v = wait_hook.load(std::memory_order_relaxed) ? wait_hook.exchange(0) : 0;
  return WaitHook{(uint64_t)(v / 2 > 0 ? v / 2 : 4000) * 2000000ull, (int)(v % 2)};   // SM clocks at 2 GHz, an upper bound of theirs
}
unsigned take_gave_up_i8(cudaError_t* e) { return take_gave_up_here(e); }

exo_gemm_status_t align_rows(void* dst, int64_t dst_ld, const void* src, int64_t src_ld, int64_t inner, int64_t rows, cudaStream_t stream, bool beside) {
  AlignParams p{(uint16_t*)dst, (const uint16_t*)src, dst_ld, src_ld, inner, rows, (inner + 7) / 8, align_of(src, src_ld * 2), beside ? 1 : 0};
  // Beside another kernel the CTAs stay until that one ends, so there are as many as find room there.
  int sms = 0;
  const exo_gemm_status_t st = device_check(&sms);
  if (st != EXO_GEMM_OK) return st;
  const int64_t most = (beside ? 4 : 16) * sms, full = (rows * p.chunks + 4 * kAlignThreads - 1) / (4 * kAlignThreads), ctas = full < most ? full : most;
  if (ctas == 0) return EXO_GEMM_OK;
  void* args[1] = {&p};
  return launch_args((void*)exo_fused_align_kernel, dim3((unsigned)ctas), kAlignThreads, 0, 1, stream, args);
}

}  // namespace fused
}  // namespace exo

using namespace exo;
using namespace exo::fused;

extern "C" {

exo_gemm_status_t exo_fused_check(void) {
  cudaError_t e = cudaDeviceSynchronize();
  unsigned n = 0;
  if (e == cudaSuccess) n |= take_gave_up_i8(&e);
  if (e == cudaSuccess) n |= take_gave_up_ffn(&e);
  if (e == cudaSuccess) n |= take_gave_up_ce(&e);
  if (e != cudaSuccess) return cuda_failed(e);
  return n ? EXO_GEMM_ERR_DEVICE_TIMEOUT : EXO_GEMM_OK;
}

exo_gemm_status_t exo_fused_debug_set(int32_t timeout_ms, int32_t skip_copies) {
  if (timeout_ms < 0 || timeout_ms > 10000 || skip_copies < 0 || skip_copies > 1) return EXO_GEMM_ERR_INVALID_ARG;
  exo::fused::wait_hook.store((int64_t)timeout_ms * 2 + skip_copies);
  return EXO_GEMM_OK;
}

exo_gemm_status_t exo_i8_quantize(const exo_i8_t* q, const void* X, int64_t ldx, int32_t x_dtype, void* cuda_stream) {
  exo_gemm_status_t st = check_i8(q);
  if (st != EXO_GEMM_OK) return st;
  if (ldx < (q->K > 1 ? q->K : 1) || x_dtype < EXO_GEMM_BF16 || x_dtype > EXO_GEMM_FP32) return EXO_GEMM_ERR_INVALID_ARG;
  if (q->rows == 0) return EXO_GEMM_OK;
  if (!X && q->K > 0) return EXO_GEMM_ERR_NULL;
  if ((st = check_i8_memory(q)) != EXO_GEMM_OK) return st;
  const int bytes = x_dtype == EXO_GEMM_FP32 ? 4 : 2;
  if ((uintptr_t)X & (unsigned)(bytes - 1)) return EXO_GEMM_ERR_ALIGNMENT;
  int sms = 0;
  if ((st = device_check(&sms)) != EXO_GEMM_OK) return st;
  QuantParams p{X, ldx, q->codes, q->ld, q->scales, (int32_t)q->K};
  const bool wide = align_of(X, ldx * bytes) >= 16;
  // few rows: more threads each, since nothing else hides a row's loads; many: more rows at once
  const int threads = q->rows <= 2 * sms ? 512 : 128;
  void* fn = x_dtype == EXO_GEMM_FP32   ? quant_fn<float, 4>(wide, threads)
             : x_dtype == EXO_GEMM_BF16 ? quant_fn<Bf16, 8>(wide, threads)
                                        : quant_fn<Fp16, 8>(wide, threads);
  void* args[1] = {&p};
  return launch_args(fn, dim3((unsigned)q->rows), (unsigned)threads, 0, 1, (cudaStream_t)cuda_stream, args);
}

exo_gemm_status_t exo_gemm_i8_run(const exo_i8_t* X, const exo_i8_t* W, void* Y, int64_t ldy, int32_t y_dtype, float alpha, float beta, void* cuda_stream) {
  exo_gemm_status_t st;
  if ((st = check_i8(X)) != EXO_GEMM_OK || (st = check_i8(W)) != EXO_GEMM_OK) return st;
  if (X->K != W->K || ldy < (W->rows > 1 ? W->rows : 1) || y_dtype < EXO_GEMM_BF16 || y_dtype > EXO_GEMM_FP32) return EXO_GEMM_ERR_INVALID_ARG;
  if (X->K > 131071) return EXO_GEMM_ERR_UNSUPPORTED;   // 2^17 products of -128 * -128 are more than a 32-bit integer holds
  if (X->rows == 0 || W->rows == 0) return EXO_GEMM_OK;
  const bool read = alpha != 0.f && X->K > 0;
  if (!Y) return EXO_GEMM_ERR_NULL;
  if (read && ((st = check_i8_memory(X)) != EXO_GEMM_OK || (st = check_i8_memory(W)) != EXO_GEMM_OK)) return st;
  const int bytes = y_dtype == EXO_GEMM_FP32 ? 4 : 2;
  if ((uintptr_t)Y & (unsigned)(bytes - 1)) return EXO_GEMM_ERR_ALIGNMENT;
  int sms = 0;
  if ((st = device_check(&sms)) != EXO_GEMM_OK) return st;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  const int64_t M = X->rows, N = W->rows, K = X->K;
  if (!read) {
    ScaleYParams p{Y, ldy, M, N, y_dtype, beta};
    const int64_t ctas = (M * N + kScaleYThreads - 1) / kScaleYThreads;
    void* args[1] = {&p};
    return launch_args((void*)exo_i8_scale_kernel, dim3((unsigned)(ctas < 16 * sms ? ctas : 16 * sms)), kScaleYThreads, 0, 1, stream, args);
  }
  I8Op::Params o{X->scales, W->scales, Y, ldy, (int32_t)N, y_dtype, align_of(Y, ldy * bytes), 0, alpha, beta};
  const Operand A{X->codes, M, K, X->ld}, B{W->codes, N, K, W->ld};
  if (M <= kThinRows) return launch_thin<I8Op, 16>(thin_width(N, 16, 256, 1, M, sms), A, B, N, K, 0, false, sms, o, stream);
  const int bn = pair_bn(M, N, false, 64, sms);
  o.tma = bytes == 2 && beta == 0.f && o.align >= 16 && N % 8 == 0;   // (nothing is written beyond a row's end)
  return o.tma ? launch_pair<I8Op, false>(bn, A, B, N, K, 0, false, sms, o, {Result{Y, N, ldy}}, stream)
               : launch_pair<I8Op, false>(bn, A, B, N, K, 0, false, sms, o, {}, stream);
}

}  // extern "C"

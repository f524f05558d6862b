// 8-bit integers with a scale per row, their products, and what the operators of exo_fused.h share: aligned copies, the state of device-side
// waits.
#include <new>
#include <type_traits>

#include "fused_host.h"

namespace exo {
namespace fused {
namespace {

// ---------------------------------------------------------------- quantisation
// A row's largest magnitude, then its codes, from registers.  For many rows what bounds the kernel is the instructions per value (4096 x 4096 bf16,
// 128 threads a row: 14.7 us, issue slots 61 % busy, where 2 + 1 bytes a value would take 7.7); for few rows a CTA of 512 takes one, and the
// latencies of a load, a reduction and a store are what is left.
struct QuantParams {
  const void* x;
  int64_t ldx;
  int8_t* codes;
  int64_t ld;
  float* scales;
  int64_t rows;
  int32_t K;
};
template <class T> struct Element { using type = uint16_t; };
template <> struct Element<float> { using type = float; };

template <int BYTES> struct Word;
template <> struct Word<16> { using type = uint4; };
template <> struct Word<8> { using type = uint2; };
template <> struct Word<4> { using type = uint32_t; };
template <> struct Word<2> { using type = uint16_t; };
__device__ __forceinline__ uint32_t word_of(const uint4& w, int i) { return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w; }
__device__ __forceinline__ uint32_t word_of(const uint2& w, int i) { return i == 0 ? w.x : w.y; }
__device__ __forceinline__ uint32_t word_of(uint32_t w, int) { return w; }
__device__ __forceinline__ uint32_t word_of(uint16_t w, int) { return w; }

// V consecutive values as they lie in memory, and as fp32
template <class T, int V> struct Held {
  using E = typename Element<T>::type;
  typename Word<V * (int)sizeof(E)>::type w;
  __device__ __forceinline__ void load(const E* x) { w = *reinterpret_cast<const decltype(w)*>(x); }
  __device__ __forceinline__ void values(float (&v)[V]) const {
    if constexpr (std::is_same<T, float>::value) {
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = __uint_as_float(word_of(w, j));
    } else {
#pragma unroll
      for (int j = 0; j < (V + 1) / 2; ++j) {
        const float2 f = T::unpack(word_of(w, j));
        v[2 * j] = f.x;
        if (2 * j + 1 < V) v[2 * j + 1] = f.y;
      }
    }
  }
  __device__ __forceinline__ float largest() const {
    float v[V], top = 0.f;
    values(v);
#pragma unroll
    for (int j = 0; j < V; ++j) top = fmaxf(top, fabsf(v[j]));
    return top;
  }
};

// Codes: the quotient rounded as IEEE division rounds it, then to the nearest integer, ties to even.  The product with the rounded
// reciprocal is within 2^-22 of the quotient, relative, so both round to the same integer unless the product is within 127 * 2^-22 of a tie; there,
// and for scales whose reciprocal is not a normal number, the division is made.  Adding 1.5 * 2^23 rounds to an integer, whose last byte is the
// code's.
struct Divider {
  float scale, inverse, limit;   // limit: how far from an integer the product may be
  __device__ __forceinline__ explicit Divider(float s) : scale(s) {
    const bool safe = s > 0x1p-120f && s < 0x1p120f;
    inverse = safe ? 1.f / s : 0.f;
    limit = safe ? 0.5f - 0x1p-14f : -1.f;
  }
  __device__ __noinline__ uint32_t divided(float x) const {
    return scale > 0.f ? __float_as_uint(fminf(fmaxf(rintf(__fdiv_rn(x, scale)), -127.f), 127.f) + 12582912.f) : 0u;
  }
  template <int V>
  __device__ __forceinline__ void codes(const float (&v)[V], uint32_t (&w)[(V + 3) / 4]) const {
    constexpr float kRound = 12582912.f;
    uint32_t c[V];
    // A branch for every value: those of 16 bits meet ties often (half of a row's largest is one), a warp's 32 rarely all at one of them.
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float q = v[j] * inverse, t = q + kRound;
      c[j] = __float_as_uint(t);
      if (fabsf(q - (t - kRound)) > limit) c[j] = divided(v[j]);   // (NaN and infinities give codes of no meaning)
    }
#pragma unroll
    for (int j = 0; j < (V + 3) / 4; ++j) {
      const uint32_t a = c[4 * j], b = 4 * j + 1 < V ? c[(4 * j + 1) % V] : 0u, d = 4 * j + 2 < V ? c[(4 * j + 2) % V] : 0u,
                     e = 4 * j + 3 < V ? c[(4 * j + 3) % V] : 0u;
      w[j] = __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(d, e, 0x0040), 0x5410);
    }
  }
};

// V: values per load, as many as 16 bytes hold where the rows' addresses allow that.  THREADS per row: a CTA of 512 for few rows, of 128 for many,
// a warp where a row has 1024 values at most.  A thread keeps its
// first HELD loads in registers, further ones are read again, from L1 or L2.  (A warp that keeps a row is so much code that fetching it takes
// longer than reading twice: 4096 x 4096 bf16, 16 loads kept 35 us.)
constexpr int kQuantWarps = 8;   // rows of a CTA, a warp each
template <class T, int V, int THREADS, int HELD>
__global__ void __launch_bounds__(THREADS == 32 ? 32 * kQuantWarps : THREADS) exo_i8_quantize_kernel(const QuantParams p) {
  __shared__ float tops[THREADS / 32];
  using E = typename Element<T>::type;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const int64_t row = THREADS == 32 ? (int64_t)blockIdx.x * kQuantWarps + (threadIdx.x >> 5) : blockIdx.x;
  const int t = THREADS == 32 ? (int)(threadIdx.x & 31u) : (int)threadIdx.x;
  if (row >= p.rows) return;   // (whole warps, where they have a row each)
  const E* x = (const E*)p.x + row * p.ldx;
  int8_t* codes = p.codes + row * p.ld;
  constexpr int STEP = THREADS * V;
  const int whole = p.K / V * V, first = t * V;   // the values of whole loads; the others one by one
  float top = 0.f;
  Held<T, V> held[HELD > 0 ? HELD : 1];
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (first + i * STEP < whole) held[i].load(x + first + i * STEP);
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (first + i * STEP < whole) top = fmaxf(top, held[i].largest());
#pragma unroll 4
  for (int k = first + HELD * STEP; k < whole; k += STEP) {
    Held<T, V> h;
    h.load(x + k);
    top = fmaxf(top, h.largest());
  }
  for (int k = whole + t; k < p.K; k += THREADS) {
    Held<T, 1> h;
    h.load(x + k);
    top = fmaxf(top, h.largest());
  }
#pragma unroll
  for (int o = 16; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if constexpr (THREADS > 32) {
    if ((t & 31) == 0) tops[t >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) top = fmaxf(top, tops[w]);
  }
  const float scale = __fdiv_rn(top, 127.f);
  if (t == 0) p.scales[row] = scale;
  const Divider by(scale);
  auto store = [&](int k, const Held<T, V>& h) {
    float v[V];
    uint32_t w[(V + 3) / 4];
    h.values(v);
    by.codes<V>(v, w);
    if constexpr (V == 8) *reinterpret_cast<uint2*>(codes + k) = make_uint2(w[0], w[1]);
    else if constexpr (V == 4) *reinterpret_cast<uint32_t*>(codes + k) = w[0];
    else if constexpr (V == 2) *reinterpret_cast<uint16_t*>(codes + k) = (uint16_t)w[0];
    else codes[k] = (int8_t)w[0];
  };
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (first + i * STEP < whole) store(first + i * STEP, held[i]);
#pragma unroll 2
  for (int k = first + HELD * STEP; k < whole; k += STEP) {
    Held<T, V> h;
    h.load(x + k);
    store(k, h);
  }
  for (int k = whole + t; k < p.K; k += THREADS) {
    Held<T, 1> h;
    float v[1];
    uint32_t w[1];
    h.load(x + k);
    h.values(v);
    by.codes<1>(v, w);
    codes[k] = (int8_t)w[0];
  }
}

// ---------------------------------------------------------------- products
// Integer sums are exact; a token's scale, its channels' scales and alpha are multiplied on in fp32.
struct I8Op {
  static constexpr bool kInt8 = true, kGated = false, kTwice = false;
  static constexpr int kUnit = 32;         // columns at a time, by pairs
  static constexpr bool kTogether = false;   // results go out together, a buffer each
  static constexpr int kMore = 0;
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

template <class T, int V> void* quant_threads(int threads) {
  return threads == 512 ? (void*)exo_i8_quantize_kernel<T, V, 512, 4> : threads == 128 ? (void*)exo_i8_quantize_kernel<T, V, 128, 4>
                                                                                      : (void*)exo_i8_quantize_kernel<T, V, 32, 0>;
}
// bytes: what divides every row's address
template <class T> void* quant_fn(int bytes, int threads) {
  constexpr int ES = (int)sizeof(typename Element<T>::type);
  if (bytes >= 16) return quant_threads<T, 16 / ES>(threads);
  if (bytes >= 8) return quant_threads<T, 8 / ES>(threads);
  if constexpr (ES == 2) return bytes >= 4 ? quant_threads<T, 2>(threads) : quant_threads<T, 1>(threads);
  else return quant_threads<T, 1>(threads);
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
  QuantParams p{X, ldx, q->codes, q->ld, q->scales, q->rows, (int32_t)q->K};
  const int at = align_of(X, ldx * bytes);
  const int threads = q->rows <= 4 * sms ? 512 : q->K > 1024 ? 128 : 32;
  void* fn = x_dtype == EXO_GEMM_FP32   ? quant_fn<float>(at, threads)
             : x_dtype == EXO_GEMM_BF16 ? quant_fn<Bf16>(at, threads)
                                        : quant_fn<Fp16>(at, threads);
  void* args[1] = {&p};
  const int64_t ctas = threads > 32 ? q->rows : (q->rows + kQuantWarps - 1) / kQuantWarps;
  return launch_args(fn, dim3((unsigned)ctas), threads > 32 ? (unsigned)threads : 32u * kQuantWarps, 0, 1, (cudaStream_t)cuda_stream, args);
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
  if (M <= kThinRows) return launch_thin<I8Op, 16>(thin_width(N, 16, 256, 1, M, sms), A, B, N, K, 0, false, sms, o, nullptr, stream);
  const int bn = pair_bn(M, N, false, 64, sms);
  o.tma = bytes == 2 && beta == 0.f && o.align >= 16 && N % 8 == 0;   // (nothing is written beyond a row's end)
  return o.tma ? launch_pair<I8Op, false>(bn, A, B, N, K, 0, false, sms, o, {Result{Y, N, ldy}}, nullptr, stream)
               : launch_pair<I8Op, false>(bn, A, B, N, K, 0, false, sms, o, {}, nullptr, stream);
}

}  // extern "C"

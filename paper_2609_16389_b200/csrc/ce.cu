// Softmax cross entropy of a head x W^T over a large vocabulary (exo_fused.h).
//
//   forward    per row and half a tile's columns ("part"): the largest logit, the sum of exp(logit - it) and, for smoothed labels, the sum
//              of the logits; a second kernel joins the parts of a row.  The logits themselves stay in tensor memory.  A training call also
//              writes the exponentials, 16 bits each, for as much of the vocabulary as the caller has room for.
//   backward   d = q (softmax - target) in 16 bits, from the kept exponentials by one factor per row and part, or from recomputed logits, a
//              piece of the vocabulary at a time;  dx += d W,  dW = d^T x
//
// With V columns, T rows and width H the products take 2 T V H operations each: one forward, two backward, and one more for what is not
// kept.  A kept exponential costs 2 + 4 bytes of traffic, which is less than recomputing it from H ~ 200 on.
#include <math.h>
#include <new>

#include "fused_host.h"

namespace exo {
namespace fused {
namespace {

// What a kept exponential is multiplied by.  They are at most 1, and fp16 has no normal numbers below 2^-14: from 2^15 on they reach down to 2^-29 of
// their part's largest with all of their bits, and to 2^-39 with one.  bf16 has fp32's range.
template <class T> constexpr float kKeptScale = 1.f;
template <> constexpr float kKeptScale<Fp16> = 32768.f;
constexpr float kTop = 16384.f;   // what the largest |dloss| becomes in q: |d| <= 2^14 in fp16, and 2^-24 / 2^14 is its smallest step

// ---------------------------------------------------------------- parts of the rows
template <class T>
struct StatsOp {
  static constexpr bool kInt8 = false, kGated = false, kTwice = true;
  static constexpr int kUnit = 32;         // columns at a time, by pairs
  static constexpr bool kTogether = false;   // results go out together, a buffer each
  static constexpr int kMore = 0;
  struct Params {
    float *top, *sum, *all;   // [part][row]: largest logit, sum of exponentials, sum of logits (NULL: not wanted)
    float* hit;               // [row]: the target's logit
    const int64_t* target;
    uint16_t* e;              // kept exponentials, rows of lde values, lde a multiple of 64: whole units can be written
    int64_t lde;
    int32_t keep;             // columns kept
    int32_t rows, vocab;
  };
  template <int U>
  struct State {
    float top, sum, all;
    int32_t target;
  };
  template <int U>
  static __device__ __forceinline__ void begin(const Params& o, State<U>& s, int row, bool row_ok, int, int) {
    s.top = -INFINITY;
    s.sum = s.all = 0.f;
    s.target = -1;
    if (row_ok) {
      const int64_t t = o.target[row];
      if (t >= 0 && t < o.vocab) s.target = (int32_t)t;
    }
  }
  template <int U>
  static __device__ __forceinline__ void look(const Params&, State<U>& s, uint32_t (&v)[U], int n) {
    float top[4] = {s.top, s.top, s.top, s.top};
    if (n >= U) {
#pragma unroll
      for (int k = 0; k < U; ++k) top[k & 3] = fmaxf(top[k & 3], __uint_as_float(v[k]));
    } else {
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (k < n) top[k & 3] = fmaxf(top[k & 3], __uint_as_float(v[k]));
    }
    s.top = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
  }
  template <int U>
  static __device__ __forceinline__ void unit(const Params& o, State<U>& s, Out& out, uint32_t (&v)[U], uint32_t (&)[1], int row, bool row_ok, int col, int n, bool) {
    const float top = s.top == -INFINITY ? 0.f : s.top;   // a part without a finite logit: exponentials of -inf, or NaN, as they are
    float e[U];
    if (n >= U) {
#pragma unroll
      for (int k = 0; k < U; ++k) e[k] = __expf(__uint_as_float(v[k]) - top);
      if (o.all) {
#pragma unroll
        for (int k = 0; k < U; ++k) s.all += __uint_as_float(v[k]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < U; ++k) {
        e[k] = k < n ? __expf(__uint_as_float(v[k]) - top) : 0.f;
        if (o.all && k < n) s.all += __uint_as_float(v[k]);
      }
    }
    float sum[4] = {};
#pragma unroll
    for (int k = 0; k < U; ++k) sum[k & 3] += e[k];
    s.sum += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    const int32_t t = s.target - col;
    if (t >= 0 && t < n) {
      float l = 0.f;
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (k == t) l = __uint_as_float(v[k]);
      o.hit[row] = l;   // one thread in all has this column
    }
    if (o.e && col < o.keep) {
      if constexpr (kKeptScale<T> != 1.f) {
#pragma unroll
        for (int k = 0; k < U; ++k) e[k] *= kKeptScale<T>;
      }
      if constexpr (U == 32) {
        uint32_t w[16];
        pack<T, U>(e, w);
        out.put(0, col, w);
      } else if (row_ok) {
        store16<T, U>(o.e + (int64_t)row * o.lde + col, e, U, 16);
      }
    }
  }
  template <int U>
  static __device__ __forceinline__ void end(const Params& o, State<U>& s, int row, bool row_ok, int part) {
    if (!row_ok) return;
    const int64_t at = (int64_t)part * o.rows + row;
    o.top[at] = s.top;
    o.sum[at] = s.sum;
    if (o.all) o.all[at] = s.all;
  }
};

// ---------------------------------------------------------------- d of a piece, from recomputed logits
template <class T>
struct GradOp {
  static constexpr bool kInt8 = false, kGated = false, kTwice = false;
  static constexpr int kUnit = 32;         // columns at a time, by pairs
  static constexpr bool kTogether = false;   // results go out together, a buffer each
  static constexpr int kMore = 0;
  struct Params {
    const float *lse, *q;     // [row]; q: dloss scaled, 0 for an ignored row
    const int64_t* target;
    int64_t first;            // the piece's first column of the vocabulary
    float hot, rest;          // what the target's column loses, and every column: 1 - s and s / vocab
  };
  template <int U>
  struct State {
    float lse, q;
    int64_t target;
  };
  template <int U>
  static __device__ __forceinline__ void begin(const Params& o, State<U>& s, int row, bool row_ok, int, int) {
    s.lse = row_ok ? o.lse[row] : 0.f;
    s.q = row_ok ? o.q[row] : 0.f;
    s.target = row_ok ? o.target[row] - o.first : -1;
  }
  template <int U>
  static __device__ __forceinline__ void unit(const Params& o, State<U>& s, Out& out, uint32_t (&v)[U], uint32_t (&)[1], int row, bool row_ok, int col, int, bool) {
    float d[U];
    const int64_t t = s.target - col;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const float p = __expf(__uint_as_float(v[k]) - s.lse) - o.rest - (t == k ? o.hot : 0.f);
      d[k] = s.q == 0.f ? 0.f : s.q * p;   // (an ignored row's logits may be anything)
    }
    uint32_t w[U / 2];
    pack<T, U>(d, w);
    out.put(0, col, w);
  }
  template <int U>
  static __device__ __forceinline__ void end(const Params&, State<U>&, int, bool, int) {}
};

// What a forward call leaves at the end of `saved`, and the backward call that uses `saved` up takes away.
constexpr uint32_t kMark = 0x6B657074u;

// ---------------------------------------------------------------- rows from their parts
struct JoinParams {
  const float *top, *sum, *all, *hit;
  const int64_t* target;
  float *loss, *lse;
  uint32_t* mark;           // of `saved`, or NULL
  int64_t rows, vocab, ignore;
  int32_t parts;
  float smoothing;
};
constexpr int kJoinThreads = 1024;
// A sum of exponentials relative to `top` as one relative to `base`.  Without a finite logit it is 0, or NaN, and stays that.
__device__ __forceinline__ float weighted(float sum, float top, float base) { return top == -INFINITY ? sum : sum * __expf(top - base); }
// A warp takes every 32nd part of 32 rows, a row per lane; the warps meet in shared memory.
__global__ void __launch_bounds__(kJoinThreads) exo_ce_join_kernel(const JoinParams p) {
  __shared__ float tops[32][33], sums[32][33], alls[32][33];
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * 32 + lane;
  if (p.mark && blockIdx.x == 0 && threadIdx.x == 0) *p.mark = kMark;
  float top = -INFINITY, sum = 0.f, all = 0.f;
  if (row < p.rows) {
    // eight parts at a time: their loads are independent
    for (int i0 = warp; i0 < p.parts; i0 += 8 * 32) {
      float t[8], s[8], m = top;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = i0 + 32 * j;
        t[j] = i < p.parts ? __ldcg(p.top + (int64_t)i * p.rows + row) : -INFINITY;
        s[j] = i < p.parts ? __ldcg(p.sum + (int64_t)i * p.rows + row) : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaxf(m, t[j]);
      const float base = m == -INFINITY ? 0.f : m;
      sum = weighted(sum, top, base);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += weighted(s[j], t[j], base);
      top = m;
    }
    if (p.all) {
#pragma unroll 4
      for (int i = warp; i < p.parts; i += 32) all += __ldcg(p.all + (int64_t)i * p.rows + row);
    }
  }
  tops[warp][lane] = top;
  sums[warp][lane] = sum;
  alls[warp][lane] = all;
  __syncthreads();
  if (warp == 0 && row < p.rows) {
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < 32; ++w) m = fmaxf(m, tops[w][lane]);
    const float base = m == -INFINITY ? 0.f : m;
    float s = 0.f, a = 0.f;
#pragma unroll
    for (int w = 0; w < 32; ++w) {
      s += weighted(sums[w][lane], tops[w][lane], base);
      a += alls[w][lane];
    }
    const float lse = base + logf(s);
    if (p.lse) p.lse[row] = lse;
    if (p.loss) {
      const int64_t t = p.target[row];
      const bool taken = t >= 0 && t < p.vocab && t != p.ignore;
      float loss = 0.f;
      if (taken) {
        loss = lse - (1.f - p.smoothing) * __ldcg(p.hit + row);
        if (p.all) loss -= p.smoothing * (a / (float)p.vocab);
      }
      p.loss[row] = loss;
    }
  }
}

// ---------------------------------------------------------------- q: dloss in the range of 16 bits, and the factor that takes it back
struct ScaleParams {
  const float* dloss;
  const int64_t* target;
  float *q, *factor;
  uint32_t* mark;           // of `saved`, or NULL
  int64_t rows, vocab, ignore;
};
constexpr int kScaleThreads = 1024;
__global__ void __launch_bounds__(kScaleThreads) exo_ce_scale_kernel(const ScaleParams p) {
  __shared__ float tops[32];
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  auto of = [&](int64_t i) {
    const int64_t t = p.target[i];
    return t >= 0 && t < p.vocab && t != p.ignore ? p.dloss[i] : 0.f;
  };
  const bool stale = p.mark && *p.mark != kMark;   // `saved` holds no exponentials (any more): nothing that looks like a gradient comes of it
  float top = 0.f;
  for (int64_t i = threadIdx.x; i < p.rows; i += kScaleThreads) {
    const float d = fabsf(of(i));
    if (d < INFINITY) top = fmaxf(top, d);   // infinities and NaN keep to their own rows
  }
#pragma unroll
  for (int o = 16; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
  __syncthreads();
  top = tops[threadIdx.x & 31];
#pragma unroll
  for (int o = 16; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  // A power of two, so that scaling rounds nothing: the largest |q| is in [2^13, 2^14).  (top == 0: every q is 0 or not finite.)
  int e = 0;
  if (top > 0.f) frexpf(top, &e);   // 2^(e - 1) <= top < 2^e
  e = e < -100 ? -100 : e;          // e <= 128: both factors are normal numbers, between 2^-114 and 2^114
  const float up = ldexpf(kTop, -e), down = ldexpf(1.f / kTop, e);
  if (threadIdx.x == 0) {
    *p.factor = down;
    if (p.mark) *p.mark = 0u;   // (every thread has read it)
  }
  for (int64_t i = threadIdx.x; i < p.rows; i += kScaleThreads) p.q[i] = stale ? NAN : of(i) * up;
}

// ---------------------------------------------------------------- d of the kept part, in place
// Bound by memory: 2 bytes in and 2 out per column.  A thread has eight columns of a row, its factor is one exponential.
struct RescaleParams {
  uint16_t* e;
  const float *top, *lse, *q;
  const int64_t* target;
  int64_t lde, rows, top_rows;   // rows of this launch, and of `top`
  uint32_t chunks;           // of eight columns, per row
  FastDiv by_part;           // columns / part_width
  float hot, rest;
};
constexpr int kRescaleThreads = 256, kRescaleRows = 4;
template <class T>
__global__ void __launch_bounds__(kRescaleThreads) exo_ce_rescale_kernel(const RescaleParams p) {
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const uint32_t chunk = blockIdx.x * kRescaleThreads + threadIdx.x;
  if (chunk >= p.chunks) return;
  const int32_t col = (int32_t)chunk * 8, part = (int32_t)fast_div((uint32_t)col, p.by_part);
  const int64_t row0 = (int64_t)blockIdx.y * kRescaleRows;
  uint32_t w[kRescaleRows][4];
#pragma unroll
  for (int r = 0; r < kRescaleRows; ++r)
    if (row0 + r < p.rows) ptx::ld_global_cg_v4(p.e + (row0 + r) * p.lde + col, w[r][0], w[r][1], w[r][2], w[r][3]);
#pragma unroll
  for (int r = 0; r < kRescaleRows; ++r) {
    const int64_t row = row0 + r;
    if (row >= p.rows) break;
    const float q = p.q[row], f = __expf(p.top[(int64_t)part * p.top_rows + row] - p.lse[row]) * (1.f / kKeptScale<T>);
    const int64_t t = p.target[row] - col;
    float d[8];
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
      const float2 v = T::unpack(w[r][k / 2]);
      d[k] = v.x * f - p.rest - (t == k ? p.hot : 0.f);
      d[k + 1] = v.y * f - p.rest - (t == k + 1 ? p.hot : 0.f);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) d[k] = q == 0.f ? 0.f : q * d[k];
    store16<T, 8>(p.e + row * p.lde + col, d, 8, 16);
  }
}

// ---------------------------------------------------------------- dx from its fp32 sum
struct FinishParams {
  const float *sum, *factor;
  uint16_t* dx;
  int64_t rows, hidden, ldx, ld;   // ld: of the sum
};
constexpr int kFinishThreads = 256;
template <class T>
__global__ void __launch_bounds__(kFinishThreads) exo_ce_finish_kernel(const FinishParams p) {
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const float f = *p.factor;
  const int64_t row = blockIdx.y, col = ((int64_t)blockIdx.x * kFinishThreads + threadIdx.x) * 8;
  if (col >= p.hidden) return;
  float v[8];
  const float4* s = reinterpret_cast<const float4*>(p.sum + row * p.ld + col);
  const float4 a = __ldcg(s), b = __ldcg(s + 1);
  v[0] = a.x * f; v[1] = a.y * f; v[2] = a.z * f; v[3] = a.w * f;
  v[4] = b.x * f; v[5] = b.y * f; v[6] = b.z * f; v[7] = b.w * f;
  const int64_t left = p.hidden - col;
  store16<T, 8>(p.dx + row * p.ldx + col, v, left < 8 ? (int)left : 8, p.ldx % 8 ? 2 : 16);
}

}  // namespace
}  // namespace fused
}  // namespace exo

using namespace exo;
using namespace exo::fused;

struct exo_ce_plan {
  exo_ce_desc_t d;       // leading dimensions and device filled in
  int device, sms;
  bool thin;
  int width, parts;      // columns of a forward tile; two parts each
  int64_t keep, lde;     // columns kept and their leading dimension
  int64_t piece, ldd;    // columns of a recomputed piece
  int bn_piece;
  int64_t ldx, ldw;      // as the kernels see them
  Memory mem;
  uint32_t* gave_up;
  float *top, *sum, *all, *hit, *q, *factor, *dx_sum;
  uint16_t *pieces, *pack_x, *pack_w;
  exo_gemm_handle_t dx[3], dw[3];   // the products of the kept columns, of a whole piece and of the last one
};

namespace {

constexpr int64_t kMostSize = 1 << 24;
constexpr int64_t kMostLd = 1LL << 31;
constexpr int64_t kKeepBytes = 4LL << 30, kPieceBytes = 256LL << 20;

exo_gemm_status_t complete(const exo_ce_desc_t* desc, exo_ce_desc_t* d) {
  if (!desc) return EXO_GEMM_ERR_NULL;
  *d = *desc;
  if (d->tokens < 0 || d->hidden < 1 || d->vocab < 1 || d->tokens > kMostSize || d->hidden > kMostSize || d->vocab > kMostSize)
    return EXO_GEMM_ERR_INVALID_ARG;
  if (!is16(d->dtype) || d->device < -1 || (d->training != 0 && d->training != 1)) return EXO_GEMM_ERR_INVALID_ARG;
  if (d->training && d->grad_dtype != EXO_GEMM_FP32 && d->grad_dtype != d->dtype) return EXO_GEMM_ERR_INVALID_ARG;
  if (!(d->label_smoothing >= 0.f && d->label_smoothing < 1.f)) return EXO_GEMM_ERR_INVALID_ARG;
  if (d->keep_bytes < -1 || d->piece < 0 || d->piece > kMostSize) return EXO_GEMM_ERR_INVALID_ARG;
  if (d->ldx == 0) d->ldx = d->hidden;
  if (d->ldw == 0) d->ldw = d->hidden;
  if (d->ldx < d->hidden || d->ldw < d->hidden || d->ldx > kMostLd || d->ldw > kMostLd) return EXO_GEMM_ERR_INVALID_ARG;
  return EXO_GEMM_OK;
}

void release(exo_ce_plan* p) {
  for (int i = 0; i < 3; ++i) {
    exo_gemm_destroy(p->dx[i]);
    exo_gemm_destroy(p->dw[i]);
  }
  p->mem.give_back();
  delete p;
}

bool placed(const void* m, int64_t ld) { return ((uintptr_t)m & (ld % 8 ? 1u : 15u)) == 0; }

// bytes of the kept exponentials; the parts' largest logits follow them, and the mark
int64_t kept_bytes(const exo_ce_plan* p) { return round_up(p->d.tokens * p->lde * 2, 256); }
constexpr int64_t kMarkBytes = 16;
uint32_t* mark_of(const exo_ce_plan* p, void* saved) { return (uint32_t*)((char*)saved + kept_bytes(p) + 4 * p->d.tokens * p->parts); }

template <class T>
exo_gemm_status_t forward(exo_ce_plan* p, const void* x, const void* W, const int64_t* target, void* saved, cudaStream_t stream) {
  const exo_ce_desc_t& d = p->d;
  typename StatsOp<T>::Params o{};
  o.top = saved ? (float*)((char*)saved + kept_bytes(p)) : p->top;
  o.sum = p->sum;
  o.all = p->all;
  o.hit = p->hit;
  o.target = target;
  o.e = (uint16_t*)saved;
  o.lde = p->lde;
  o.keep = (int32_t)p->keep;
  o.rows = (int32_t)d.tokens;
  o.vocab = (int32_t)d.vocab;
  const Operand X{x, d.tokens, d.hidden, p->ldx}, Wo{W, d.vocab, d.hidden, p->ldw};
  const bool bf16 = d.dtype == EXO_GEMM_BF16;
  if (p->thin) return launch_thin<StatsOp<T>, 16>(p->width, X, Wo, d.vocab, d.hidden, 0, bf16, p->sms, o, p->gave_up, stream);
  return saved ? launch_pair<StatsOp<T>, false>(p->width, X, Wo, d.vocab, d.hidden, 0, bf16, p->sms, o, {Result{saved, p->lde, p->lde}}, p->gave_up, stream)
               : launch_pair<StatsOp<T>, false>(p->width, X, Wo, d.vocab, d.hidden, 0, bf16, p->sms, o, {}, p->gave_up, stream);
}

template <class T>
exo_gemm_status_t recompute(exo_ce_plan* p, const void* x, const void* W, const int64_t* target, const float* lse, int64_t first, int64_t columns,
                            cudaStream_t stream) {
  const exo_ce_desc_t& d = p->d;
  typename GradOp<T>::Params o{};
  o.lse = lse; o.q = p->q; o.target = target; o.first = first;
  o.hot = 1.f - d.label_smoothing;
  o.rest = d.label_smoothing / (float)d.vocab;
  const Operand Wo{(const uint16_t*)W + first * p->ldw, columns, d.hidden, p->ldw};
  return launch_pair<GradOp<T>, false>(p->bn_piece, Operand{x, d.tokens, d.hidden, p->ldx}, Wo, columns, d.hidden, 0, d.dtype == EXO_GEMM_BF16, p->sms, o,
                                       {Result{p->pieces, p->ldd, p->ldd}}, p->gave_up, stream);
}

exo_gemm_status_t products(exo_ce_plan* p, int which, int64_t columns, int64_t ldd, bool several) {
  const exo_ce_desc_t& d = p->d;
  exo_gemm_desc_t g{};
  g.ab_dtype = d.dtype;
  g.c_layout = EXO_GEMM_ROW_MAJOR;
  g.device = p->device;
  g.M = d.tokens; g.N = d.hidden; g.K = columns;          // dx = d W
  g.c_dtype = several ? EXO_GEMM_FP32 : d.dtype;
  g.a_layout = g.b_layout = EXO_GEMM_ROW_MAJOR;
  g.lda = ldd; g.ldb = p->ldw; g.ldc = several ? round_up(d.hidden, 64) : d.ldx;
  exo_gemm_status_t st = exo_gemm_create(&p->dx[which], &g);
  if (st != EXO_GEMM_OK) return st;
  g.M = columns; g.N = d.hidden; g.K = d.tokens;          // dW = d^T x
  g.c_dtype = d.grad_dtype;
  g.a_layout = EXO_GEMM_COL_MAJOR;
  g.lda = ldd; g.ldb = p->ldx; g.ldc = d.ldw;
  return exo_gemm_create(&p->dw[which], &g);
}

}  // namespace

unsigned exo::fused::take_gave_up_ce(cudaError_t* e) { return take_gave_up_here(e); }

extern "C" {

exo_gemm_status_t exo_ce_validate(const exo_ce_desc_t* desc) {
  exo_ce_desc_t d;
  return complete(desc, &d);
}

exo_gemm_status_t exo_ce_create(exo_ce_handle_t* out, const exo_ce_desc_t* desc) {
  if (!out) return EXO_GEMM_ERR_NULL;
  exo_ce_desc_t d;
  exo_gemm_status_t st = complete(desc, &d);
  if (st != EXO_GEMM_OK) return st;
  cudaError_t e;
  if (d.device < 0 && (e = cudaGetDevice(&d.device)) != cudaSuccess) return cuda_failed(e);
  OnDevice on(d.device);
  if (on.err != cudaSuccess) return cuda_failed(on.err);
  int sms = 0;
  if ((st = device_check(&sms)) != EXO_GEMM_OK) return st;
  exo_ce_plan* p = new (std::nothrow) exo_ce_plan{};
  if (!p) return EXO_GEMM_ERR_CUDA;
  p->d = d;
  p->device = d.device;
  p->sms = sms;
  const int64_t T = d.tokens, H = d.hidden, V = d.vocab;
  p->thin = T <= kThinRows;
  p->width = p->thin ? thin_width(V, 32, 256, 1, T, sms) : pair_bn(T, V, false, 64, sms);
  p->parts = (int)((V + p->width - 1) / p->width) * 2;
  p->ldx = d.ldx % 8 ? round_up(H, 64) : d.ldx;
  p->ldw = d.ldw % 8 ? round_up(H, 64) : d.ldw;
  p->lde = p->ldd = 64;
  if (d.training && T > 0) {
    const int64_t most = (d.keep_bytes < 0 ? kKeepBytes : d.keep_bytes) - 4 * T * p->parts - kMarkBytes - 256;
    p->keep = most <= 0 ? 0 : most / (2 * T) / 64 * 64;   // (rows of a multiple of 64)
    if (p->keep >= round_up(V, 64)) p->keep = V;
    else p->keep = p->keep / p->width * p->width;   // whole tiles of the forward product, less than V of them
    if (p->keep > V) p->keep = V;
    p->lde = round_up(p->keep, 64);
    if (p->keep < V) {
      p->piece = d.piece ? round_up(d.piece, 64) : kPieceBytes / (2 * T) / 256 * 256;
      if (p->piece < 256 && !d.piece) p->piece = 256;
      if (p->piece > V - p->keep) p->piece = V - p->keep;
      p->ldd = round_up(p->piece, 64);
      p->bn_piece = pair_bn(T, p->piece, false, 64, sms);
    }
  }
  const int64_t rest = p->piece ? (V - p->keep) % p->piece : 0;
  const bool several = p->piece > 0 && (p->keep > 0 || p->piece < V);   // dx is a sum of more than one product
  if (T > 0) {
    p->gave_up = p->mem.take_word();
    p->top = (float*)p->mem.take(4 * T * p->parts);
    p->sum = (float*)p->mem.take(4 * T * p->parts);
    if (d.label_smoothing > 0.f) p->all = (float*)p->mem.take(4 * T * p->parts);
    p->hit = (float*)p->mem.take(4 * T);
    if (d.ldx % 8) p->pack_x = (uint16_t*)p->mem.take(2 * T * p->ldx);
    if (d.ldw % 8) p->pack_w = (uint16_t*)p->mem.take(2 * V * p->ldw);
    if (d.training) {
      p->q = (float*)p->mem.take(4 * T);
      p->factor = (float*)p->mem.take(16);
      if (several) p->dx_sum = (float*)p->mem.take(4 * T * round_up(H, 64));
      if (p->piece) p->pieces = (uint16_t*)p->mem.take(2 * T * p->ldd);
    }
  }
  if (p->mem.err != cudaSuccess) {
    e = p->mem.err;
    release(p);
    return cuda_failed(e);
  }
  if (d.training) {
    if (T == 0) st = products(p, 0, V, round_up(V, 64), false);   // an empty sum: dW's is zero
    else if (p->keep > 0) st = products(p, 0, p->keep, p->lde, several);
    if (st == EXO_GEMM_OK && p->piece && V - p->keep >= p->piece) st = products(p, 1, p->piece, p->ldd, several);
    if (st == EXO_GEMM_OK && rest) st = products(p, 2, rest, p->ldd, several);
  }
  if (st != EXO_GEMM_OK) {
    release(p);
    return st;
  }
  *out = p;
  return EXO_GEMM_OK;
}

int64_t exo_ce_saved_bytes(exo_ce_handle_t p) { return p && p->keep > 0 ? kept_bytes(p) + 4 * p->d.tokens * p->parts + kMarkBytes : 0; }

exo_gemm_status_t exo_ce_forward(exo_ce_handle_t p, const void* x, const void* W, const int64_t* target, float* loss, float* lse, void* saved,
                                 void* cuda_stream) {
  if (!p) return EXO_GEMM_ERR_NULL;
  const exo_ce_desc_t& d = p->d;
  if (saved && !d.training) return EXO_GEMM_ERR_INVALID_ARG;
  if (d.tokens == 0) return EXO_GEMM_OK;
  if (!x || !W || !target) return EXO_GEMM_ERR_NULL;
  if (!placed(x, d.ldx) || !placed(W, d.ldw) || ((uintptr_t)target & 7u) || ((uintptr_t)loss & 3u) || ((uintptr_t)lse & 3u) || !aligned16(saved))
    return EXO_GEMM_ERR_ALIGNMENT;
  OnDevice on(p->device);
  if (on.err != cudaSuccess) return cuda_failed(on.err);
  cudaStream_t s = (cudaStream_t)cuda_stream;
  exo_gemm_status_t st;
  if (p->pack_x && (st = align_rows(p->pack_x, p->ldx, x, d.ldx, d.hidden, d.tokens, s)) != EXO_GEMM_OK) return st;
  if (p->pack_w && (st = align_rows(p->pack_w, p->ldw, W, d.ldw, d.hidden, d.vocab, s)) != EXO_GEMM_OK) return st;
  if (p->pack_x) x = p->pack_x;
  if (p->pack_w) W = p->pack_w;
  if (p->keep == 0) saved = nullptr;
  st = d.dtype == EXO_GEMM_BF16 ? forward<Bf16>(p, x, W, target, saved, s) : forward<Fp16>(p, x, W, target, saved, s);
  if (st != EXO_GEMM_OK) return st;
  JoinParams j{};
  j.top = saved ? (const float*)((const char*)saved + kept_bytes(p)) : p->top;
  j.sum = p->sum; j.all = p->all; j.hit = p->hit; j.target = target; j.loss = loss; j.lse = lse;
  j.mark = saved ? mark_of(p, saved) : nullptr;
  j.rows = d.tokens; j.vocab = d.vocab; j.ignore = d.ignore_index; j.parts = p->parts; j.smoothing = d.label_smoothing;
  void* args[1] = {&j};
  return launch_args((void*)exo_ce_join_kernel, dim3((unsigned)((d.tokens + 31) / 32)), kJoinThreads, 0, 1, s, args);
}

exo_gemm_status_t exo_ce_backward(exo_ce_handle_t p, const void* x, const void* W, const int64_t* target, const float* lse, const float* dloss, void* saved,
                                  void* dx, void* dW, int32_t accumulate, void* cuda_stream) {
  if (!p) return EXO_GEMM_ERR_NULL;
  const exo_ce_desc_t& d = p->d;
  if (!d.training) return EXO_GEMM_ERR_INVALID_ARG;
  if (!dx && !dW) return EXO_GEMM_OK;
  const int gb = d.grad_dtype == EXO_GEMM_FP32 ? 4 : 2;
  if (dW && ((uintptr_t)dW & (d.ldw * gb % 16 ? (unsigned)gb - 1u : 15u))) return EXO_GEMM_ERR_ALIGNMENT;
  const float beta = accumulate ? 1.f : 0.f;
  if (d.tokens == 0) return dW ? gemm_run_scaled(p->dw[0], nullptr, nullptr, dW, 1.f, nullptr, beta, cuda_stream) : EXO_GEMM_OK;
  const bool recomputes = p->keep < d.vocab;
  if (!target || !lse || !dloss || (p->keep > 0 && !saved) || (!x && (dW || recomputes)) || (!W && (dx || recomputes))) return EXO_GEMM_ERR_NULL;
  if ((x && !placed(x, d.ldx)) || (W && !placed(W, d.ldw)) || (dx && !placed(dx, d.ldx)) || ((uintptr_t)target & 7u) || ((uintptr_t)lse & 3u) ||
      ((uintptr_t)dloss & 3u) || !aligned16(saved))
    return EXO_GEMM_ERR_ALIGNMENT;
  OnDevice on(p->device);
  if (on.err != cudaSuccess) return cuda_failed(on.err);
  cudaStream_t s = (cudaStream_t)cuda_stream;
  exo_gemm_status_t st;
  if (x && p->pack_x && (st = align_rows(p->pack_x, p->ldx, x, d.ldx, d.hidden, d.tokens, s)) != EXO_GEMM_OK) return st;
  if (W && p->pack_w && (st = align_rows(p->pack_w, p->ldw, W, d.ldw, d.hidden, d.vocab, s)) != EXO_GEMM_OK) return st;
  if (p->pack_x) x = p->pack_x;
  if (p->pack_w) W = p->pack_w;

  ScaleParams sp{dloss, target, p->q, p->factor, p->keep > 0 ? mark_of(p, saved) : nullptr, d.tokens, d.vocab, d.ignore_index};
  void* scale_args[1] = {&sp};
  if ((st = launch_args((void*)exo_ce_scale_kernel, dim3(1), kScaleThreads, 0, 1, s, scale_args)) != EXO_GEMM_OK) return st;

  const bool several = p->dx_sum != nullptr;
  bool first = true;
  auto both = [&](int which, const void* dmat, int64_t at) {
    exo_gemm_status_t r = EXO_GEMM_OK;
    const uint16_t* w = (const uint16_t*)W + at * p->ldw;
    if (dx && several) r = gemm_run_scaled(p->dx[which], dmat, w, p->dx_sum, 1.f, nullptr, first ? 0.f : 1.f, cuda_stream);
    else if (dx) r = gemm_run_scaled(p->dx[which], dmat, w, dx, 1.f, p->factor, 0.f, cuda_stream);
    first = false;
    if (r == EXO_GEMM_OK && dW) r = gemm_run_scaled(p->dw[which], dmat, x, (char*)dW + at * d.ldw * gb, 1.f, p->factor, beta, cuda_stream);
    return r;
  };
  if (p->keep > 0) {
    RescaleParams r{};
    r.e = (uint16_t*)saved;
    r.top = (const float*)((const char*)saved + kept_bytes(p));
    r.lse = lse; r.q = p->q; r.target = target;
    r.lde = p->lde; r.top_rows = d.tokens;
    r.chunks = (uint32_t)((p->keep + 7) / 8);
    r.by_part = make_fast_div((uint32_t)p->width / 2);
    r.hot = 1.f - d.label_smoothing;
    r.rest = d.label_smoothing / (float)d.vocab;
    void* args[1] = {&r};
    // rows in the grid's second dimension, which has 65535 at most
    const int64_t rows_per_launch = 65535LL * kRescaleRows;
    for (int64_t r0 = 0; r0 < d.tokens; r0 += rows_per_launch) {
      RescaleParams part = r;
      part.e += r0 * p->lde;
      part.top += r0; part.lse += r0; part.q += r0; part.target += r0;
      const int64_t rows = d.tokens - r0 < rows_per_launch ? d.tokens - r0 : rows_per_launch;
      part.rows = rows;
      args[0] = &part;
      const dim3 grid((r.chunks + kRescaleThreads - 1) / kRescaleThreads, (unsigned)((rows + kRescaleRows - 1) / kRescaleRows));
      void* fn = d.dtype == EXO_GEMM_BF16 ? (void*)exo_ce_rescale_kernel<Bf16> : (void*)exo_ce_rescale_kernel<Fp16>;
      if ((st = launch_args(fn, grid, kRescaleThreads, 0, 1, s, args)) != EXO_GEMM_OK) return st;
    }
    if ((st = both(0, saved, 0)) != EXO_GEMM_OK) return st;
  }
  for (int64_t at = p->keep; at < d.vocab; at += p->piece) {
    const int64_t columns = d.vocab - at < p->piece ? d.vocab - at : p->piece;
    st = d.dtype == EXO_GEMM_BF16 ? recompute<Bf16>(p, x, W, target, lse, at, columns, s) : recompute<Fp16>(p, x, W, target, lse, at, columns, s);
    if (st == EXO_GEMM_OK) st = both(columns == p->piece ? 1 : 2, p->pieces, at);
    if (st != EXO_GEMM_OK) return st;
  }
  if (dx && several) {
    FinishParams f{p->dx_sum, p->factor, (uint16_t*)dx, d.tokens, d.hidden, d.ldx, round_up(d.hidden, 64)};
    void* args[1] = {&f};
    const int64_t rows_per_launch = 65535;
    for (int64_t r0 = 0; r0 < d.tokens; r0 += rows_per_launch) {
      FinishParams part = f;
      part.sum += r0 * f.ld;
      part.dx += r0 * f.ldx;
      args[0] = &part;
      const int64_t rows = d.tokens - r0 < rows_per_launch ? d.tokens - r0 : rows_per_launch;
      const dim3 grid((unsigned)((d.hidden + kFinishThreads * 8 - 1) / (kFinishThreads * 8)), (unsigned)rows);
      void* fn = d.dtype == EXO_GEMM_BF16 ? (void*)exo_ce_finish_kernel<Bf16> : (void*)exo_ce_finish_kernel<Fp16>;
      if ((st = launch_args(fn, grid, kFinishThreads, 0, 1, s, args)) != EXO_GEMM_OK) return st;
    }
  }
  return EXO_GEMM_OK;
}

exo_gemm_status_t exo_ce_check(exo_ce_handle_t p) {
  if (!p) return EXO_GEMM_ERR_NULL;
  OnDevice on(p->device);
  if (on.err != cudaSuccess) return cuda_failed(on.err);
  return check_plan(p->gave_up, {p->dx[0], p->dx[1], p->dx[2], p->dw[0], p->dw[1], p->dw[2]});
}

int64_t exo_ce_workspace_bytes(exo_ce_handle_t p) {
  if (!p) return 0;
  int64_t n = p->mem.bytes;
  for (exo_gemm_handle_t g : {p->dx[0], p->dx[1], p->dx[2], p->dw[0], p->dw[1], p->dw[2]}) {
    exo_gemm_info_t info;
    if (g && exo_gemm_get_info(g, &info) == EXO_GEMM_OK) n += info.workspace_bytes;
  }
  return n;
}

exo_gemm_status_t exo_ce_destroy(exo_ce_handle_t p) {
  if (!p) return EXO_GEMM_OK;
  OnDevice on(p->device);
  if (on.err != cudaSuccess) return cuda_failed(on.err);
  release(p);
  return EXO_GEMM_OK;
}

}  // extern "C"

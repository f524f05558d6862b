// The gated feed-forward block (exo_fused.h).
//
//   forward    h = act(x Wg^T) * (x Wu^T)      one product with two accumulators' columns, act and the product in its epilogue
//              y = h Wd^T
//   backward   dh = dy Wd                      in the epilogue, from the saved g and u: dg, du and h
//              dx = [dg du] [Wg; Wu],  d_gate_up = [dg du]^T x,  d_down = dy^T h
//
// dg and du lie side by side in rows of 2 * inner values, so that dx is one product of depth 2 * inner and both weights' gradients are one.
// The plain products are the library's own (exo_gemm); up to 128 rows, y is a thin product.
#include <new>

#include "fused_host.h"

namespace exo {
namespace fused {
namespace {

// ---------------------------------------------------------------- activations
// 1 / (1 + exp(-x)): beyond the range of expf the quotient is 0 or 1, as it should be.
__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }

// act(g) and, with GRAD, act'(g)
template <int ACT, bool GRAD>
__device__ __forceinline__ void activate(float g, float& a, float& slope) {
  if constexpr (ACT == EXO_ACT_SILU) {
    const float s = sigmoid(g);
    a = g * s;
    if constexpr (GRAD) slope = s * fmaf(g, 1.f - s, 1.f);
  } else if constexpr (ACT == EXO_ACT_GELU) {
    // Phi by erfc: 1 + erf would lose the digits of the left tail.  erfc is the Chebyshev fit of Press et al., Numerical Recipes in C, section 6.2,
    // good to 1.2e-7 of the value everywhere, with fewer instructions than erfcf: the backward pass's epilogue is exposed in products of one wave.
    const float z = 0.70710678118654752f * fabsf(g), t = __fdividef(1.f, fmaf(0.5f, z, 1.f));
    float e = fmaf(t, 0.17087277f, -0.82215223f);
    e = fmaf(t, e, 1.48851587f);
    e = fmaf(t, e, -1.13520398f);
    e = fmaf(t, e, 0.27886807f);
    e = fmaf(t, e, -0.18628806f);
    e = fmaf(t, e, 0.09678418f);
    e = fmaf(t, e, 0.37409196f);
    e = fmaf(t, e, 1.00002368f);
    e = fmaf(t, e, -1.26551223f);
    const float tail = 0.5f * t * __expf(fmaf(-z, z, e)), phi = g < 0.f ? tail : 1.f - tail;
    a = g * phi;
    if constexpr (GRAD) slope = fmaf(g * 0.39894228040143268f, __expf(-0.5f * g * g), phi);
  } else {
    // (1 + tanh(z)) / 2 = 1 / (1 + exp(-2 z))
    constexpr float two_a = 1.5957691216057308f, b = 0.044715f;
    const float s = sigmoid(two_a * g * fmaf(b * g, g, 1.f));
    a = g * s;
    if constexpr (GRAD) {
      const float d = s * (1.f - s);   // 0 where the cube of a large g is infinite
      slope = d > 0.f ? fmaf(g * d, two_a * fmaf(3.f * b * g, g, 1.f), s) : s;
    }
  }
}

// ---------------------------------------------------------------- h = act(g) * u
// Bound by the tensor cores for many rows and by the weights' bytes for few.
template <class T>
struct GatedOp {
  static constexpr bool kInt8 = false, kGated = true, kTwice = false;
  static constexpr int kUnit = 8;         // columns at a time, by pairs
  static constexpr bool kTogether = true;   // results go out together, a buffer each
  static constexpr int kMore = 0;
  struct Params {
    uint16_t *h, *g, *u;   // rows of ld values, ld a multiple of 64: whole units can be written; g and u may be NULL
    int64_t ld;
    int32_t act;
  };
  template <int U>
  struct State {};
  template <int U>
  static __device__ __forceinline__ void begin(const Params&, State<U>&, int, bool, int, int) {}
  template <int ACT, int U>
  static __device__ __forceinline__ void product(const float (&g)[U], const float (&u)[U], float (&h)[U]) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      float a, unused;
      activate<ACT, false>(g[k], a, unused);
      h[k] = a * u[k];
    }
  }
  template <int U>
  static __device__ __forceinline__ void unit(const Params& o, State<U>&, Out& out, uint32_t (&v)[U], uint32_t (&v2)[U], int row, bool row_ok, int col, int, bool more) {
    float g[U], u[U], h[U];
#pragma unroll
    for (int k = 0; k < U; ++k) { g[k] = __uint_as_float(v[k]); u[k] = __uint_as_float(v2[k]); }
    if (o.act == EXO_ACT_SILU) product<EXO_ACT_SILU, U>(g, u, h);
    else if (o.act == EXO_ACT_GELU) product<EXO_ACT_GELU, U>(g, u, h);
    else product<EXO_ACT_GELU_TANH, U>(g, u, h);
    uint32_t w[U / 2];
    if (out.maps) {   // by pairs: 32 columns of up to three results, then a TMA store of each, which leaves out the rows that do not exist
      if ((col & 31) == 0) out.open();
      pack<T, U>(h, w);
      out.piece<U / 8>(0, col, w);
      if (o.g) {
        pack<T, U>(g, w);
        out.piece<U / 8>(1, col, w);
        pack<T, U>(u, w);
        out.piece<U / 8>(2, col, w);
      }
      if (((col + U) & 31) == 0 || !more) out.close(o.g ? 3 : 1, col);   // (columns beyond the last are the rows' padding)
    } else if (row_ok) {
      const int64_t at = (int64_t)row * o.ld + col;
      store16<T, U>(o.h + at, h, U, 16);
      if (o.g) {
        store16<T, U>(o.g + at, g, U, 16);
        store16<T, U>(o.u + at, u, U, 16);
      }
    }
  }
  template <int U>
  static __device__ __forceinline__ void end(const Params&, State<U>&, int, bool, int) {}
};

// ---------------------------------------------------------------- dg, du and h from dh, g and u
template <class T>
struct GatedBackOp {
  static constexpr bool kInt8 = false, kGated = false, kTwice = false;
  static constexpr int kUnit = 16;         // columns at a time, by pairs
  static constexpr bool kTogether = true;   // results go out together, a buffer each
  static constexpr int kMore = 2;   // dg and du, also where they are not stored by TMA
  struct Params {
    const uint16_t *g, *u;
    uint16_t* h;
    int64_t ld;
    uint16_t* dgu;       // rows of ld2 values: dg, then du from value `inner` on
    int64_t ld2;
    int32_t inner, act;
    int32_t aligned;     // dg and du are stored by TMA
    int32_t du_align;    // what divides the address of du's units
  };
  template <int U>
  struct State {
    uint32_t g[U / 2], u[U / 2];   // of the next unit, fetched a unit's time ahead
  };
  template <int U>
  static __device__ __forceinline__ void fetch(const Params& o, State<U>& s, int64_t at) {
    static_assert(U == 16, "a sector of each");
    ld_global_cg_v8(o.g + at, s.g);
    ld_global_cg_v8(o.u + at, s.u);
  }
  template <int U>
  static __device__ __forceinline__ void begin(const Params& o, State<U>& s, int row, bool row_ok, int col, int N) {
    if (row_ok && col < N) fetch<U>(o, s, (int64_t)row * o.ld + col);
  }
  template <int ACT, int U>
  static __device__ __forceinline__ void chain(const uint32_t (&v)[U], const uint32_t (&g)[U / 2], const uint32_t (&u)[U / 2], uint32_t (&dg)[U / 2],
                                               uint32_t (&du)[U / 2], uint32_t (&h)[U / 2]) {
#pragma unroll
    for (int k = 0; k < U; k += 2) {
      const float2 x = T::unpack(g[k / 2]), y = T::unpack(u[k / 2]);
      const float dh0 = __uint_as_float(v[k]), dh1 = __uint_as_float(v[k + 1]);
      float a0, a1, slope0, slope1;
      activate<ACT, true>(x.x, a0, slope0);
      activate<ACT, true>(x.y, a1, slope1);
      dg[k / 2] = T::pack(dh0 * y.x * slope0, dh1 * y.y * slope1);
      du[k / 2] = T::pack(dh0 * a0, dh1 * a1);
      h[k / 2] = T::pack(a0 * y.x, a1 * y.y);
    }
  }
  template <int U>
  static __device__ __forceinline__ void unit(const Params& o, State<U>& s, Out& out, uint32_t (&v)[U], uint32_t (&)[1], int row, bool row_ok, int col, int n,
                                              bool more) {
    uint32_t g[U / 2], u[U / 2], dg[U / 2], du[U / 2], h[U / 2];
#pragma unroll
    for (int j = 0; j < U / 2; ++j) { g[j] = s.g[j]; u[j] = s.u[j]; }
    if (more && row_ok) fetch<U>(o, s, (int64_t)row * o.ld + col + U);
    if (o.act == EXO_ACT_SILU) chain<EXO_ACT_SILU, U>(v, g, u, dg, du, h);
    else if (o.act == EXO_ACT_GELU) chain<EXO_ACT_GELU, U>(v, g, u, dg, du, h);
    else chain<EXO_ACT_GELU_TANH, U>(v, g, u, dg, du, h);
    if ((col & 31) == 0) out.open();
    out.piece<U / 8>(0, col, h);
    out.piece<U / 8>(1, col, dg);
    out.piece<U / 8>(2, col, du);
    if (((col + U) & 31) == 0 || !more) {
      out.close(o.aligned ? 3 : 1, col);   // (columns beyond the last are the rows' padding, or not stored)
      if (!o.aligned) {   // `inner` is not a multiple of 8: du begins inside a 16-byte piece, and dg must not be written beyond its end
        uint16_t* const d = o.dgu + (int64_t)out.row0 * o.ld2 + (col & ~31);
        const int there = (col & 31) + n;
        out.store_rows<2>(1, d, 2 * o.ld2, there, 8);
        out.store_rows<2>(2, d + o.inner, 2 * o.ld2, there, o.du_align);
      }
    }
  }
  template <int U>
  static __device__ __forceinline__ void end(const Params&, State<U>&, int, bool, int) {}
};

// ---------------------------------------------------------------- y, for a few rows
template <class T>
struct PlainOp {
  static constexpr bool kInt8 = false, kGated = false, kTwice = false;
  struct Params {
    uint16_t* y;
    int64_t ld;
    int32_t align;
  };
  template <int U>
  struct State {};
  template <int U>
  static __device__ __forceinline__ void begin(const Params&, State<U>&, int, bool, int, int) {}
  template <int U>
  static __device__ __forceinline__ void unit(const Params& o, State<U>&, Out& out, uint32_t (&v)[U], uint32_t (&)[1], int row, bool row_ok, int col, int n, bool) {
    float y[U];
#pragma unroll
    for (int k = 0; k < U; ++k) y[k] = __uint_as_float(v[k]);
    uint32_t w[U / 2];
    pack<T, U>(y, w);
    if (o.align >= 16 && n == U) {
      if (row_ok) store_words<U>(o.y + (int64_t)row * o.ld + col, w, n, o.align);
    } else {
      out.write<U / 8>(out.buffers, 0, w);
      out.store_rows<2>(0, o.y + (int64_t)out.row0 * o.ld + col, 2 * o.ld, n, o.align);
    }
  }
  template <int U>
  static __device__ __forceinline__ void end(const Params&, State<U>&, int, bool, int) {}
};

}  // namespace
}  // namespace fused
}  // namespace exo

using namespace exo;
using namespace exo::fused;

struct exo_ffn_plan {
  exo_ffn_desc_t d;      // leading dimensions and device filled in
  int device, sms;
  bool thin;
  int width_gated, width_down;         // thin
  int bn_gated, bn_back;               // pairs
  int64_t ldh, ld2;                    // of h (and g, u) and of dg | du
  int64_t ldx, ldy, ld_gate_up, ld_down;   // as the kernels see them: of the aligned copies where there are some
  Memory mem;
  uint32_t* gave_up;
  uint16_t *h, *dgu;
  uint16_t *pack_x, *pack_dy, *pack_gate_up, *pack_down;
  exo_gemm_handle_t down, dx, d_gate_up, d_down;
};

namespace {

constexpr int64_t kMostSize = 1 << 24;
constexpr int64_t kMostLd = 1LL << 31;

// Leading dimensions filled in, then checked.
exo_gemm_status_t complete(const exo_ffn_desc_t* desc, exo_ffn_desc_t* d) {
  if (!desc) return EXO_GEMM_ERR_NULL;
  *d = *desc;
  if (d->tokens < 0 || d->hidden < 1 || d->inner < 1 || d->tokens > kMostSize || d->hidden > kMostSize || d->inner > kMostSize)
    return EXO_GEMM_ERR_INVALID_ARG;
  if (!is16(d->dtype) || d->activation < EXO_ACT_SILU || d->activation > EXO_ACT_GELU_TANH || d->device < -1) return EXO_GEMM_ERR_INVALID_ARG;
  if (d->training != 0 && d->training != 1) return EXO_GEMM_ERR_INVALID_ARG;
  if (d->training && d->grad_dtype != EXO_GEMM_FP32 && d->grad_dtype != d->dtype) return EXO_GEMM_ERR_INVALID_ARG;
  if (d->ldx == 0) d->ldx = d->hidden;
  if (d->ldy == 0) d->ldy = d->hidden;
  if (d->ld_gate_up == 0) d->ld_gate_up = d->hidden;
  if (d->ld_down == 0) d->ld_down = d->inner;
  if (d->ldx < d->hidden || d->ldy < d->hidden || d->ld_gate_up < d->hidden || d->ld_down < d->inner || d->ldx > kMostLd || d->ldy > kMostLd ||
      d->ld_gate_up > kMostLd || d->ld_down > kMostLd)
    return EXO_GEMM_ERR_INVALID_ARG;
  return EXO_GEMM_OK;
}

void release(exo_ffn_plan* p) {
  for (exo_gemm_handle_t g : {p->down, p->dx, p->d_gate_up, p->d_down}) exo_gemm_destroy(g);
  p->mem.give_back();
  delete p;
}

exo_gemm_status_t product(exo_gemm_handle_t* out, const exo_ffn_plan* p, int64_t M, int64_t N, int64_t K, int32_t c_dtype, int32_t a_layout, int64_t lda,
                          int32_t b_layout, int64_t ldb, int64_t ldc) {
  exo_gemm_desc_t g{};
  g.M = M; g.N = N; g.K = K;
  g.ab_dtype = p->d.dtype; g.c_dtype = c_dtype;
  g.a_layout = a_layout; g.b_layout = b_layout; g.c_layout = EXO_GEMM_ROW_MAJOR;
  g.lda = lda; g.ldb = ldb; g.ldc = ldc;
  g.device = p->device;
  return exo_gemm_create(out, &g);
}

// the saved g and u are read 32 bytes at a time
bool aligned32(const void* p) { return ((uintptr_t)p & 31u) == 0; }

// A 16-bit matrix of the caller's: 16-byte aligned where it is used in place, else aligned to its element.
bool placed(const void* m, int64_t ld) { return ((uintptr_t)m & (ld % 8 ? 1u : 15u)) == 0; }

template <class T>
exo_gemm_status_t forward(exo_ffn_plan* p, const void* x, const void* gate_up, const void* down, void* y, uint16_t* saved, cudaStream_t stream) {
  const exo_ffn_desc_t& d = p->d;
  const bool bf16 = d.dtype == EXO_GEMM_BF16;
  typename GatedOp<T>::Params gp{p->h, saved, saved ? saved + d.tokens * p->ldh : nullptr, p->ldh, d.activation};
  const Operand X{x, d.tokens, d.hidden, p->ldx}, GU{gate_up, 2 * d.inner, d.hidden, p->ld_gate_up};
  exo_gemm_status_t st;
  if (!p->thin) {
    const Result H{p->h, p->ldh, p->ldh}, G{gp.g, p->ldh, p->ldh}, U{gp.u, p->ldh, p->ldh};
    st = saved ? launch_pair<GatedOp<T>, false>(p->bn_gated, X, GU, d.inner, d.hidden, d.inner, bf16, p->sms, gp, {H, G, U}, p->gave_up, stream)
               : launch_pair<GatedOp<T>, false>(p->bn_gated, X, GU, d.inner, d.hidden, d.inner, bf16, p->sms, gp, {H}, p->gave_up, stream);
  } else {
    st = launch_thin<GatedOp<T>, 8>(p->width_gated, X, GU, d.inner, d.hidden, d.inner, bf16, p->sms, gp, p->gave_up, stream);
  }
  if (st != EXO_GEMM_OK) return st;
  if (p->pack_down) {   // the copy of down goes on beside the first product
    if ((st = align_rows(p->pack_down, p->ld_down, down, d.ld_down, d.inner, d.hidden, stream, true)) != EXO_GEMM_OK) return st;
    down = p->pack_down;
  }
  if (!p->thin) return gemm_run_scaled(p->down, p->h, down, y, 1.f, nullptr, 0.f, stream);
  typename PlainOp<T>::Params yp{(uint16_t*)y, d.ldy, align_of(y, d.ldy * 2)};
  return launch_thin<PlainOp<T>, 16>(p->width_down, Operand{p->h, d.tokens, d.inner, p->ldh}, Operand{down, d.hidden, d.inner, p->ld_down}, d.hidden, d.inner,
                                     0, bf16, p->sms, yp, p->gave_up, stream);
}

template <class T>
exo_gemm_status_t back(exo_ffn_plan* p, const void* down, const uint16_t* saved, const void* dy, cudaStream_t stream) {
  const exo_ffn_desc_t& d = p->d;
  typename GatedBackOp<T>::Params bp{saved, saved + d.tokens * p->ldh, p->h, p->ldh, p->dgu, p->ld2, (int32_t)d.inner, d.activation,
                                     d.inner % 8 == 0, align_of(p->dgu, 2 * d.inner)};
  const Operand dY{dy, d.tokens, d.hidden, p->ldy}, Wd{down, d.hidden, d.inner, p->ld_down};
  const Result H{p->h, p->ldh, p->ldh}, G{p->dgu, d.inner, p->ld2}, U{p->dgu + d.inner, d.inner, p->ld2};
  const bool bf16 = d.dtype == EXO_GEMM_BF16;
  return bp.aligned ? launch_pair<GatedBackOp<T>, true>(p->bn_back, dY, Wd, d.inner, d.hidden, 0, bf16, p->sms, bp, {H, G, U}, p->gave_up, stream)
                    : launch_pair<GatedBackOp<T>, true>(p->bn_back, dY, Wd, d.inner, d.hidden, 0, bf16, p->sms, bp, {H}, p->gave_up, stream);
}

}  // namespace

unsigned exo::fused::take_gave_up_ffn(cudaError_t* e) { return take_gave_up_here(e); }

extern "C" {

exo_gemm_status_t exo_ffn_validate(const exo_ffn_desc_t* desc) {
  exo_ffn_desc_t d;
  return complete(desc, &d);
}

exo_gemm_status_t exo_ffn_create(exo_ffn_handle_t* out, const exo_ffn_desc_t* desc) {
  if (!out) return EXO_GEMM_ERR_NULL;
  exo_ffn_desc_t d;
  exo_gemm_status_t st = complete(desc, &d);
  if (st != EXO_GEMM_OK) return st;
  cudaError_t e;
  if (d.device < 0 && (e = cudaGetDevice(&d.device)) != cudaSuccess) return cuda_failed(e);
  OnDevice on(d.device);
  if (on.err != cudaSuccess) return cuda_failed(on.err);
  int sms = 0;
  if ((st = device_check(&sms)) != EXO_GEMM_OK) return st;
  exo_ffn_plan* p = new (std::nothrow) exo_ffn_plan{};
  if (!p) return EXO_GEMM_ERR_CUDA;
  p->d = d;
  p->device = d.device;
  p->sms = sms;
  const int64_t T = d.tokens, H = d.hidden, F = d.inner;
  p->thin = T <= kThinRows;
  p->width_gated = thin_width(F, 8, 128, 2, T, sms);
  p->width_down = thin_width(H, 16, 256, 1, T, sms);
  p->bn_gated = pair_bn(T, F, true, 64, sms);
  p->bn_back = pair_bn(T, F, false, 128, sms);
  p->ldh = round_up(F, 64);
  p->ld2 = round_up(2 * F, 64);
  auto packed = [](int64_t ld, int64_t inner) { return ld % 8 ? round_up(inner, 64) : ld; };
  p->ldx = packed(d.ldx, H);
  p->ldy = packed(d.ldy, H);
  p->ld_gate_up = packed(d.ld_gate_up, H);
  p->ld_down = packed(d.ld_down, F);
  if (T > 0) {
    auto take = [&](int64_t values) { return (uint16_t*)p->mem.take(2 * values); };
    p->gave_up = p->mem.take_word();
    p->h = take(T * p->ldh);
    if (d.training) p->dgu = take(T * p->ld2);
    if (d.ldx % 8) p->pack_x = take(T * p->ldx);
    if (d.ldy % 8 && d.training) p->pack_dy = take(T * p->ldy);
    if (d.ld_gate_up % 8) p->pack_gate_up = take(2 * F * p->ld_gate_up);
    if (d.ld_down % 8) p->pack_down = take(H * p->ld_down);
  }
  if (p->mem.err != cudaSuccess) {
    e = p->mem.err;
    release(p);
    return cuda_failed(e);
  }
  const int R = EXO_GEMM_ROW_MAJOR, C = EXO_GEMM_COL_MAJOR;
  if (!p->thin) st = product(&p->down, p, T, H, F, d.dtype, R, p->ldh, C, p->ld_down, d.ldy);
  if (d.training) {
    if (st == EXO_GEMM_OK) st = product(&p->dx, p, T, H, 2 * F, d.dtype, R, p->ld2, R, p->ld_gate_up, d.ldx);
    if (st == EXO_GEMM_OK) st = product(&p->d_gate_up, p, 2 * F, H, T, d.grad_dtype, C, p->ld2, R, p->ldx, d.ld_gate_up);
    if (st == EXO_GEMM_OK) st = product(&p->d_down, p, H, F, T, d.grad_dtype, C, p->ldy, R, p->ldh, d.ld_down);
  }
  if (st != EXO_GEMM_OK) {
    release(p);
    return st;
  }
  *out = p;
  return EXO_GEMM_OK;
}

int64_t exo_ffn_saved_bytes(exo_ffn_handle_t plan) { return plan && plan->d.training ? 4 * plan->d.tokens * plan->ldh : 0; }

exo_gemm_status_t exo_ffn_forward(exo_ffn_handle_t p, const void* x, const void* gate_up, const void* down, void* y, void* saved, void* cuda_stream) {
  if (!p) return EXO_GEMM_ERR_NULL;
  const exo_ffn_desc_t& d = p->d;
  if (saved && !d.training) return EXO_GEMM_ERR_INVALID_ARG;
  if (d.tokens == 0) return EXO_GEMM_OK;
  if (!x || !gate_up || !down || !y) return EXO_GEMM_ERR_NULL;
  if (!placed(x, d.ldx) || !placed(gate_up, d.ld_gate_up) || !placed(down, d.ld_down) || !placed(y, d.ldy) || !aligned32(saved)) return EXO_GEMM_ERR_ALIGNMENT;
  OnDevice on(p->device);
  if (on.err != cudaSuccess) return cuda_failed(on.err);
  cudaStream_t s = (cudaStream_t)cuda_stream;
  exo_gemm_status_t st = EXO_GEMM_OK;
  if (p->pack_x && (st = align_rows(p->pack_x, p->ldx, x, d.ldx, d.hidden, d.tokens, s)) != EXO_GEMM_OK) return st;
  if (p->pack_gate_up && (st = align_rows(p->pack_gate_up, p->ld_gate_up, gate_up, d.ld_gate_up, d.hidden, 2 * d.inner, s)) != EXO_GEMM_OK) return st;
  if (p->pack_x) x = p->pack_x;
  if (p->pack_gate_up) gate_up = p->pack_gate_up;
  return d.dtype == EXO_GEMM_BF16 ? forward<Bf16>(p, x, gate_up, down, y, (uint16_t*)saved, s)
                                  : forward<Fp16>(p, x, gate_up, down, y, (uint16_t*)saved, s);
}

exo_gemm_status_t exo_ffn_backward(exo_ffn_handle_t p, const void* x, const void* gate_up, const void* down, const void* saved, const void* dy, void* dx,
                                   void* d_gate_up, void* d_down, int32_t accumulate, void* cuda_stream) {
  if (!p) return EXO_GEMM_ERR_NULL;
  const exo_ffn_desc_t& d = p->d;
  if (!d.training) return EXO_GEMM_ERR_INVALID_ARG;
  if (!dx && !d_gate_up && !d_down) return EXO_GEMM_OK;
  const bool any = d.tokens > 0;
  if (any && (!down || !saved || !dy || (d_gate_up && !x) || (dx && !gate_up))) return EXO_GEMM_ERR_NULL;
  if (any && (!placed(down, d.ld_down) || !placed(dy, d.ldy) || !aligned32(saved) || (d_gate_up && !placed(x, d.ldx)) ||
              (dx && (!placed(gate_up, d.ld_gate_up) || !placed(dx, d.ldx)))))
    return EXO_GEMM_ERR_ALIGNMENT;
  const int gb = d.grad_dtype == EXO_GEMM_FP32 ? 4 : 2;
  auto grad_placed = [&](const void* m, int64_t ld) { return ((uintptr_t)m & (ld * gb % 16 ? (unsigned)gb - 1u : 15u)) == 0; };
  if ((d_gate_up && !grad_placed(d_gate_up, d.ld_gate_up)) || (d_down && !grad_placed(d_down, d.ld_down))) return EXO_GEMM_ERR_ALIGNMENT;
  OnDevice on(p->device);
  if (on.err != cudaSuccess) return cuda_failed(on.err);
  cudaStream_t s = (cudaStream_t)cuda_stream;
  exo_gemm_status_t st = EXO_GEMM_OK;
  if (any) {
    if (p->pack_down && (st = align_rows(p->pack_down, p->ld_down, down, d.ld_down, d.inner, d.hidden, s)) != EXO_GEMM_OK) return st;
    if (p->pack_dy && (st = align_rows(p->pack_dy, p->ldy, dy, d.ldy, d.hidden, d.tokens, s)) != EXO_GEMM_OK) return st;
    if (d_gate_up && p->pack_x && (st = align_rows(p->pack_x, p->ldx, x, d.ldx, d.hidden, d.tokens, s)) != EXO_GEMM_OK) return st;
    if (dx && p->pack_gate_up && (st = align_rows(p->pack_gate_up, p->ld_gate_up, gate_up, d.ld_gate_up, d.hidden, 2 * d.inner, s)) != EXO_GEMM_OK) return st;
    if (p->pack_down) down = p->pack_down;
    if (p->pack_dy) dy = p->pack_dy;
    if (p->pack_x) x = p->pack_x;
    if (p->pack_gate_up) gate_up = p->pack_gate_up;
    st = d.dtype == EXO_GEMM_BF16 ? back<Bf16>(p, down, (const uint16_t*)saved, dy, s) : back<Fp16>(p, down, (const uint16_t*)saved, dy, s);
    if (st != EXO_GEMM_OK) return st;
  }
  const float beta = accumulate ? 1.f : 0.f;
  if (dx && any && (st = gemm_run_scaled(p->dx, p->dgu, gate_up, dx, 1.f, nullptr, 0.f, cuda_stream)) != EXO_GEMM_OK) return st;
  if (d_gate_up && (st = gemm_run_scaled(p->d_gate_up, p->dgu, x, d_gate_up, 1.f, nullptr, beta, cuda_stream)) != EXO_GEMM_OK) return st;
  if (d_down && (st = gemm_run_scaled(p->d_down, dy, p->h, d_down, 1.f, nullptr, beta, cuda_stream)) != EXO_GEMM_OK) return st;
  return EXO_GEMM_OK;
}

exo_gemm_status_t exo_ffn_check(exo_ffn_handle_t p) {
  if (!p) return EXO_GEMM_ERR_NULL;
  OnDevice on(p->device);
  if (on.err != cudaSuccess) return cuda_failed(on.err);
  return check_plan(p->gave_up, {p->down, p->dx, p->d_gate_up, p->d_down});
}

int64_t exo_ffn_workspace_bytes(exo_ffn_handle_t p) {
  if (!p) return 0;
  int64_t n = p->mem.bytes;
  for (exo_gemm_handle_t g : {p->down, p->dx, p->d_gate_up, p->d_down}) {
    exo_gemm_info_t info;
    if (g && exo_gemm_get_info(g, &info) == EXO_GEMM_OK) n += info.workspace_bytes;
  }
  return n;
}

exo_gemm_status_t exo_ffn_destroy(exo_ffn_handle_t p) {
  if (!p) return EXO_GEMM_OK;
  OnDevice on(p->device);
  if (on.err != cudaSuccess) return cuda_failed(on.err);
  release(p);
  return EXO_GEMM_OK;
}

}  // extern "C"

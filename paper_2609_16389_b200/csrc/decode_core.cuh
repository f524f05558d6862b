// What the few-token kernels share: the fragments of mma.sync, 16 weight rows by 8 tokens at a time, straight from rows of
// weights.
//
// For a few tokens a product is bound by reading the weights, so the kernels are built around the load: a lane
// takes 16 consecutive bytes of a weight row, and the order in which the tensor core sums over k is chosen so that
// those bytes are its fragment.  In m16n8k16 lane 4 g + t holds the A elements of rows g and g + 8 at four
// values of k and the B elements of column g at the same four.  Any assignment of the real k to those places gives the
// same sum as long as A and B agree, so lane t takes eight consecutive k for two instructions: no shuffle and no
// transposition of either operand.
//
// mma.sync and not tcgen05: an operand of tcgen05.mma comes from shared or tensor memory, 64 or 128 rows at a time.
// 4-bit weights have to pass through registers anyway, and 16 rows per warp cut a matrix into pieces fine enough to
// occupy 148 SMs.  m16n8k16 takes a quarter of an SM 8 clocks (ncu, sm__pipe_tensor): at one token 64 of the 178 clocks in
// which memory delivers a step of 16 x 128 4-bit weights, from about 24 tokens on more than that.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "ptx.cuh"

namespace exo {
void note_cuda_error(int e);   // what exo_gemm_last_cuda_error reports (api.cu)

namespace decode {

// ---- the two 16-bit types -----------------------------------------------------------------------------------
struct Bf16 {
  using type = __nv_bfloat16;
  static constexpr uint32_t kNibbleBase = 0x43004300u;   // a pair of 128.0: one unit in the last place is 1
  static __device__ __forceinline__ float to_float(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
  static __device__ __forceinline__ uint16_t from_float(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }
  static __device__ __forceinline__ uint32_t pair(float lo, float hi) {
    const __nv_bfloat162 r = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  static __device__ __forceinline__ float max_finite() { return __uint_as_float(0x7f7f0000u); }
  static __device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  static __device__ __forceinline__ void mma0(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {   // d = a b
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
  }
  static __device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {   // d += a b
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
};
struct Fp16 {
  using type = __half;
  static constexpr uint32_t kNibbleBase = 0x64006400u;   // a pair of 1024.0: one unit in the last place is 1
  static __device__ __forceinline__ float to_float(uint16_t v) { return __half2float(__ushort_as_half(v)); }
  static __device__ __forceinline__ uint16_t from_float(float v) { return __half_as_ushort(__float2half_rn(v)); }
  static __device__ __forceinline__ uint32_t pair(float lo, float hi) {
    const __half2 r = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  static __device__ __forceinline__ float max_finite() { return 65504.f; }
  static __device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  static __device__ __forceinline__ void mma0(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {   // d = a b
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
  }
  static __device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {   // d += a b
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
};

// ---- loads ----------------------------------------------------------------------------------------------------
// Weights: read once, so they leave L1 to the activations.
__device__ __forceinline__ uint4 ldg_weights(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// Eight consecutive 16-bit elements k .. k + 7 of a row; those at and beyond K are 0 and not read.  aligned: the
// row starts on a 16-byte boundary (k is a multiple of 8).
__device__ __forceinline__ uint4 load8_checked(const uint16_t* row, int k, int K, bool aligned) {
  if (aligned && k + 8 <= K) return *reinterpret_cast<const uint4*>(row + k);
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = k + 2 * i < K ? row[k + 2 * i] : 0, hi = k + 2 * i + 1 < K ? row[k + 2 * i + 1] : 0;
    v[i] = lo | hi << 16;
  }
  return make_uint4(v[0], v[1], v[2], v[3]);
}

// ---- activations ----------------------------------------------------------------------------------------------
// The rows of tokens g, 8 + g, 16 + g, ... are `stride` apart.  Rows of tokens that do not exist may hold anything: a
// column of the product depends on its own token alone, and nobody reads theirs.
struct XShared {
  uint32_t base, stride;   // bytes, shared window
  template <int OFF> __device__ __forceinline__ uint4 load(int i) const {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4+%5];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(base + i * stride), "n"(OFF * 2));
    return v;
  }
  __device__ __forceinline__ void advance(int n) { base += 2 * n; }
};

// ---- 4-bit rows -----------------------------------------------------------------------------------------------
// Sixteen rows of 4-bit weights in steps of 128 values of k.  The pointers are the lane's own: rows g and g + 8, at its part of
// the current step.
//   load(n)      the step n ahead of the current one
//   advance(n)   n steps on
//   step(...)    acc += rows x tokens; x.load<OFF>(i) are the lane's eight activations of token 8 i + g, OFF elements
//                behind the current step's (the lane's own 8 t included)
// Only whole steps go through load() and step(); a last part of a step goes through load_tail() and step_tail().
// 4-bit weights, PER groups of 128 / PER weights in a step of 128.  ZEROS: with zero points, else 8 everywhere.
template <class T, int PER, bool ZEROS>
struct RowsQ4 {
  static constexpr int kStep = 128;
  const uint8_t *c0, *c1;        // codes
  const uint16_t *s0, *s1;       // scales
  const uint8_t *z0, *z1;        // zero points
  struct Regs {
    uint4 a, b;
    uint32_t sa[(PER + 1) / 2], sb[(PER + 1) / 2];
    uint32_t za, zb;             // PER bytes
  };

  static __device__ __forceinline__ void load_scales(uint32_t (&v)[(PER + 1) / 2], const uint16_t* p) {
    if constexpr (PER == 1) {
      uint16_t h;
      asm volatile("ld.global.nc.u16 %0, [%1];" : "=h"(h) : "l"(p));
      v[0] = h;
    } else if constexpr (PER == 2) {
      asm volatile("ld.global.nc.u32 %0, [%1];" : "=r"(v[0]) : "l"(p));
    } else {
      asm volatile("ld.global.nc.v2.u32 {%0, %1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "l"(p));
    }
  }
  static __device__ __forceinline__ uint32_t load_zeros(const uint8_t* p) {
    uint32_t v;
    if constexpr (PER == 1) asm volatile("ld.global.nc.u8 %0, [%1];" : "=r"(v) : "l"(p));
    else if constexpr (PER == 2) asm volatile("ld.global.nc.u16 %0, [%1];" : "=r"(v) : "l"(p));
    else asm volatile("ld.global.nc.u32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
  }
  __device__ __forceinline__ void begin(int t) { c0 += 16 * t; c1 += 16 * t; }
  __device__ __forceinline__ void advance(int n) {
    c0 += n * 64; c1 += n * 64;
    s0 += n * PER; s1 += n * PER;
    if constexpr (ZEROS) { z0 += n * PER; z1 += n * PER; }
  }
  __device__ __forceinline__ Regs load(int n) const {
    Regs r;
    r.a = ldg_weights(c0 + n * 64);
    r.b = ldg_weights(c1 + n * 64);
    load_scales(r.sa, s0 + n * PER);
    load_scales(r.sb, s1 + n * PER);
    if constexpr (ZEROS) {
      r.za = load_zeros(z0 + n * PER);
      r.zb = load_zeros(z1 + n * PER);
    }
    return r;
  }
  __device__ __forceinline__ Regs load_tail(int, int) const { return load(0); }   // rows are padded to whole steps

  // The eight weights of a word as four pairs of exact 16-bit numbers code - zero: a code put under the exponent of
  // 128 (bf16) or 1024 (fp16) is that number plus the code, and subtracting the same number plus zero leaves the difference.
  static __device__ __forceinline__ void unpack(uint32_t w, uint32_t base_zero, uint32_t (&p)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t v;
      asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(v) : "r"(w >> (4 * i)), "r"(0x000f000fu), "r"(T::kNibbleBase));   // (w & mask) | base
      p[i] = T::sub2(v, base_zero);
    }
  }
  template <int NT, int OFF, bool TAIL, class X, class N>
  __device__ __forceinline__ void products(const Regs& r, int left, const X& x, N nt, float (&acc)[NT][4]) const {
    const uint32_t wa[4] = {r.a.x, r.a.y, r.a.z, r.a.w}, wb[4] = {r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      if (TAIL && q * (128 / PER) >= left) break;   // groups of padding alone: their scales may be anything
      const uint32_t za = T::kNibbleBase | (ZEROS ? ((r.za >> (8 * q)) & 0xffu) * 0x00010001u : 0x00080008u);
      const uint32_t zb = T::kNibbleBase | (ZEROS ? ((r.zb >> (8 * q)) & 0xffu) * 0x00010001u : 0x00080008u);
      float part[NT][4];
#pragma unroll
      for (int j = 4 / PER * q; j < 4 / PER * (q + 1); ++j) {
        uint32_t pa[4], pb[4];
        unpack(wa[j], za, pa);
        unpack(wb[j], zb, pb);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          if (i == 0 || i < nt) {
            const uint4 b = j == 0 ? x.template load<OFF>(i) : j == 1 ? x.template load<OFF + 32>(i) : j == 2 ? x.template load<OFF + 64>(i) : x.template load<OFF + 96>(i);
            if (j == 4 / PER * q) T::mma0(part[i], pa[0], pb[0], pa[1], pb[1], b.x, b.y);
            else T::mma(part[i], pa[0], pb[0], pa[1], pb[1], b.x, b.y);
            T::mma(part[i], pa[2], pb[2], pa[3], pb[3], b.z, b.w);
          }
        }
      }
      const float sa = T::to_float((uint16_t)(r.sa[q / 2] >> (16 * (q % 2)))), sb = T::to_float((uint16_t)(r.sb[q / 2] >> (16 * (q % 2))));
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        if (i == 0 || i < nt) {
          acc[i][0] = fmaf(sa, part[i][0], acc[i][0]);
          acc[i][1] = fmaf(sa, part[i][1], acc[i][1]);
          acc[i][2] = fmaf(sb, part[i][2], acc[i][2]);
          acc[i][3] = fmaf(sb, part[i][3], acc[i][3]);
        }
      }
    }
  }
  template <int NT, int OFF, class X, class N>
  __device__ __forceinline__ void step(const Regs& r, const X& x, N nt, float (&acc)[NT][4]) const {
    products<NT, OFF, false>(r, 128, x, nt, acc);
  }
  template <int NT, class X, class N>
  __device__ __forceinline__ void step_tail(const Regs& r, int left, const X& x, N nt, float (&acc)[NT][4]) const {
    products<NT, 0, true>(r, left, x, nt, acc);
  }
};

// Scales and zero points of up to STEPS (4 or 8) steps of a lane's rows g and g + 8, loaded together: lane t of four holds those of
// steps t and 4 + t, and hands them out.  Groups of padding alone (whose scales may be anything) get 0.
template <class T, int PER, bool ZEROS, int STEPS>
struct StepScales {
  using F = RowsQ4<T, PER, ZEROS>;
  static constexpr int N = (PER + 1) / 2, H = STEPS / 4;
  uint32_t a[H][N], b[H][N], za[H], zb[H];

  struct Rows {                  // this lane's places in the rows of a tile: their step 0, t further on
    const uint16_t *s0, *s1;
    const uint8_t *z0, *z1;      // NULL: 8
  };
  // steps s .. s + n - 1; left: values of k from step s on
  __device__ __forceinline__ void load(const Rows& r, int s, int n, int left) {
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int step = 4 * h + (threadIdx.x & 3);
#pragma unroll
      for (int i = 0; i < N; ++i) a[h][i] = b[h][i] = 0;
      za[h] = zb[h] = 0;
      if (step < n) {
        const int at = (s + 4 * h) * PER;
        F::load_scales(a[h], r.s0 + at);
        F::load_scales(b[h], r.s1 + at);
        if constexpr (ZEROS) {
          za[h] = r.z0 ? F::load_zeros(r.z0 + at) : 0x08080808u;
          zb[h] = r.z1 ? F::load_zeros(r.z1 + at) : 0x08080808u;
        }
        if (PER > 1 && (step + 1) * 128 > left) {
#pragma unroll
          for (int q = 1; q < PER; ++q)
            if (step * 128 + q * (128 / PER) >= left) {
              a[h][q / 2] &= q % 2 ? 0x0000ffffu : 0xffff0000u;
              b[h][q / 2] &= q % 2 ? 0x0000ffffu : 0xffff0000u;
            }
        }
      }
    }
  }
  // step u, the same for all lanes
  __device__ __forceinline__ void get(int u, uint32_t (&sa)[N], uint32_t (&sb)[N], uint32_t& z0, uint32_t& z1) const {
    const int from = ((threadIdx.x & 31) & 28) | (u & 3);
    auto pick = [&](const uint32_t (&v)[H]) { return H == 1 || u < 4 ? v[0] : v[H - 1]; };
    auto pick_n = [&](const uint32_t (&v)[H][N], int i) { return H == 1 || u < 4 ? v[0][i] : v[H - 1][i]; };
    if constexpr (PER == 1) {
      const uint32_t both = __shfl_sync(0xffffffffu, pick_n(a, 0) | pick_n(b, 0) << 16, from);
      sa[0] = both & 0xffffu;
      sb[0] = both >> 16;
    } else {
#pragma unroll
      for (int q = 0; q < N; ++q) {
        sa[q] = __shfl_sync(0xffffffffu, pick_n(a, q), from);
        sb[q] = __shfl_sync(0xffffffffu, pick_n(b, q), from);
      }
    }
    z0 = z1 = 0;
    if constexpr (ZEROS) {
      if constexpr (PER <= 2) {
        const uint32_t both = __shfl_sync(0xffffffffu, (pick(za) & 0xffffu) | pick(zb) << 16, from);
        z0 = both & 0xffffu;
        z1 = both >> 16;
      } else {
        z0 = __shfl_sync(0xffffffffu, pick(za), from);
        z1 = __shfl_sync(0xffffffffu, pick(zb), from);
      }
    }
  }
};

// ---- a warp's walk over its steps -----------------------------------------------------------------------------
// `n` whole steps, DS apart, with DEPTH steps' loads in flight: preload() issues the first ones (before the
// activations are needed), walk() computes a step and at once refills its registers.  While 2 * DEPTH steps are left
// nothing is checked.  Afterwards f and x point behind the n steps.
template <class F, int DS, int DEPTH>
struct Stream {
  typename F::Regs buf[DEPTH];

  __device__ __forceinline__ void preload(const F& f, int n) {
#pragma unroll
    for (int u = 0; u < DEPTH; ++u)
      if (u < n) buf[u] = f.load(u * DS);
  }
  template <int NT, int U, class X, class N>
  __device__ __forceinline__ void round(const F& f, int n, bool all, const X& x, N nt, float (&acc)[NT][4]) {
    if constexpr (U < DEPTH) {
      if (all || U < n) f.template step<NT, U * DS * F::kStep>(buf[U], x, nt, acc);
      if (all || U + DEPTH < n) buf[U] = f.load((U + DEPTH) * DS);
      round<NT, U + 1>(f, n, all, x, nt, acc);
    }
  }
  template <int NT, class X, class N>
  __device__ __forceinline__ void walk(F& f, int n, X& x, N nt, float (&acc)[NT][4]) {
    while (n >= 2 * DEPTH) {
      round<NT, 0>(f, n, true, x, nt, acc);
      f.advance(DEPTH * DS);
      x.advance(DEPTH * DS * F::kStep);
      n -= DEPTH;
    }
    while (n > 0) {
      round<NT, 0>(f, n, false, x, nt, acc);
      const int done = n < DEPTH ? n : DEPTH;
      f.advance(done * DS);
      x.advance(done * DS * F::kStep);
      n -= done;
    }
  }
};

// All NT tiles of columns, known when compiling: the `nt` of the functions above.
template <int NT> struct All { __device__ constexpr operator int() const { return NT; } };

// 16 bytes of shared memory
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
// A warp's waits for the copies of a piece, bounded by the SM's clock.  One that gives up says so and lets the copies in flight land; the
// warp then neither issues nor awaits any more and goes on to the kernel's end, and the host can learn of it (exo_decode_check).
struct WaitBound {
  uint64_t clocks;
  int skip;         // for tests: the first CTA's first warp issues no copies
};
static __device__ unsigned gave_up;
__device__ __forceinline__ bool wait_on(uint32_t bar, uint32_t parity, uint64_t clocks) {
  const long long begin = clock64();
  do {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (ptx::mbar_try_wait(bar, parity)) return true;
  } while ((uint64_t)(clock64() - begin) <= clocks);
  gave_up = 1;
  for (int i = 0; i < 200; ++i) __nanosleep(1000);
  return false;
}
static __device__ __noinline__ bool wait_on_call(uint32_t bar, uint32_t parity, uint64_t clocks) { return wait_on(bar, parity, clocks); }
struct Copies {
  bool issues, awaits = true;   // issues: this lane, lane 0
  __device__ __forceinline__ explicit Copies(const WaitBound& b) : issues((threadIdx.x & 31) == 0 && !(b.skip && blockIdx.x == 0 && threadIdx.x < 32)) {}
  // CALL: the longer part of the wait is a call.  It frees the integer products' loop (32768 x 16384: 49.9 us, 51.1 inline), and costs
  // the others more than it gives (64 tokens of 64 experts of 4096 x 1536: 547 us, 539 inline).
  template <bool CALL>
  __device__ __forceinline__ void wait(uint32_t bar, uint32_t parity, const WaitBound& b) {
    if (ptx::mbar_try_wait(bar, parity) || !awaits) return;
    if (!(CALL ? wait_on_call(bar, parity, b.clocks) : wait_on(bar, parity, b.clocks))) issues = awaits = false;
  }
};

// This translation unit's word, put back to 0.
static inline unsigned take_gave_up(cudaError_t* e) {
  unsigned v = 0, zero = 0;
  *e = cudaMemcpyFromSymbol(&v, gave_up, sizeof v);
  if (*e == cudaSuccess && v) *e = cudaMemcpyToSymbol(gave_up, &zero, sizeof zero);
  return v;
}

// How many of the steps s, s + ds, ... lie below `end`.
__device__ __forceinline__ int steps_of(int s, int ds, int end) { return s < end ? (end - s + ds - 1) / ds : 0; }

}  // namespace decode
}  // namespace exo

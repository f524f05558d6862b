// What the few-token kernels share: weights streamed from device memory straight into the fragments of
// mma.sync.m16n8k16, 16 weight rows by 8 tokens at a time.
//
// For a few tokens a product is bound by reading the weights, so the kernels are built around the load: a lane
// reads 16 consecutive bytes of a weight row, and the order in which the tensor core sums over k is chosen so that
// those bytes are its fragment.  In m16n8k16 lane 4 g + t holds the A elements of rows g and g + 8 at four
// values of k and the B elements of column g at the same four.  Any assignment of the real k to those places gives the
// same sum as long as A and B agree, so lane t takes eight consecutive k for two instructions: no shuffle, no
// shared-memory pass and no transposition of either operand.
//
// mma.sync and not tcgen05: an operand of tcgen05.mma comes from shared or tensor memory, 64 or 128 rows at a time.
// Here the weights arrive in registers, 4-bit ones have to pass through them anyway, and 16 rows per warp cut a
// matrix into pieces fine enough to occupy 148 SMs.  Up to 64 tokens the legacy path's rate is not the bound.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace exo {
void note_cuda_error(int e);   // what exo_gemm_last_cuda_error reports (api.cu)

namespace decode {

// ---- the two 16-bit types -----------------------------------------------------------------------------------
struct Bf16 {
  using type = __nv_bfloat16;
  static constexpr uint32_t kNibbleBase = 0x43004300u;   // a pair of 128.0: one unit in the last place is 1
  static __device__ __forceinline__ float to_float(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
  static __device__ __forceinline__ uint16_t from_float(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }
  static __device__ __forceinline__ float max_finite() { return __uint_as_float(0x7f7f0000u); }
  static __device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  static __device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
};
struct Fp16 {
  using type = __half;
  static constexpr uint32_t kNibbleBase = 0x64006400u;   // a pair of 1024.0: one unit in the last place is 1
  static __device__ __forceinline__ float to_float(uint16_t v) { return __half2float(__ushort_as_half(v)); }
  static __device__ __forceinline__ uint16_t from_float(float v) { return __half_as_ushort(__float2half_rn(v)); }
  static __device__ __forceinline__ float max_finite() { return 65504.f; }
  static __device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  static __device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
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

// ---- weight formats -------------------------------------------------------------------------------------------
// A format reads 16 weight rows in steps of kStep values of k.  Row pointers are those of the lane's rows g and g + 8.
//   load(s, K)   step s of both rows (values at and beyond K read as 0)
//   step(...)    acc += rows x tokens over that step; xb(i, k) is the lane's part of B: eight activations of token
//                8 i + g at k .. k + 7 (k includes the lane's own 8 t)

// 16-bit weights.  VEC: every row starts on a 16-byte boundary.
template <class T, bool VEC>
struct Rows16 {
  static constexpr int kStep = 32;
  const uint16_t *r0, *r1;
  struct Regs { uint4 a, b; };

  __device__ __forceinline__ Regs load(int s, int K, int t) const {
    const int k = s * kStep + 8 * t;
    Regs r;
    if (VEC && k + 8 <= K) {
      r.a = ldg_weights(r0 + k);
      r.b = ldg_weights(r1 + k);
    } else {
      r.a = load8_checked(r0, k, K, false);
      r.b = load8_checked(r1, k, K, false);
    }
    return r;
  }
  template <int NT, class XB>
  __device__ __forceinline__ void step(const Regs& r, int s, int K, int t, const XB& xb, int nt, float (&acc)[NT][4]) const {
    const int k = s * kStep + 8 * t;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      if (i < nt) {
        const uint4 b = xb(i, k);
        T::mma(acc[i], r.a.x, r.b.x, r.a.y, r.b.y, b.x, b.y);
        T::mma(acc[i], r.a.z, r.b.z, r.a.w, r.b.w, b.z, b.w);
      }
    }
  }
};

// 4-bit weights, PER groups of 128 / PER weights in a step of 128.
template <class T, int PER>
struct RowsQ4 {
  static constexpr int kStep = 128;
  const uint8_t *c0, *c1;        // codes
  const uint16_t *s0, *s1;       // scales
  const uint8_t *z0, *z1;        // zero points (NULL: 8)
  struct Regs {
    uint4 a, b;
    uint32_t sa[(PER + 1) / 2], sb[(PER + 1) / 2];
    uint32_t za, zb;             // PER bytes
  };

  static __device__ __forceinline__ void load_scales(uint32_t (&v)[(PER + 1) / 2], const uint16_t* p) {
    if constexpr (PER == 1) v[0] = __ldg(p);
    else if constexpr (PER == 2) v[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
    else { const uint2 w = __ldg(reinterpret_cast<const uint2*>(p)); v[0] = w.x; v[1] = w.y; }
  }
  static __device__ __forceinline__ uint32_t load_zeros(const uint8_t* p) {
    if constexpr (PER == 1) return __ldg(p);
    else if constexpr (PER == 2) return __ldg(reinterpret_cast<const uint16_t*>(p));
    else return __ldg(reinterpret_cast<const uint32_t*>(p));
  }
  __device__ __forceinline__ Regs load(int s, int, int t) const {
    Regs r;
    r.a = ldg_weights(c0 + (int64_t)s * 64 + 16 * t);
    r.b = ldg_weights(c1 + (int64_t)s * 64 + 16 * t);
    load_scales(r.sa, s0 + (int64_t)s * PER);
    load_scales(r.sb, s1 + (int64_t)s * PER);
    r.za = r.zb = 0x08080808u;
    if (z0 != nullptr) {
      r.za = load_zeros(z0 + (int64_t)s * PER);
      r.zb = load_zeros(z1 + (int64_t)s * PER);
    }
    return r;
  }
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
  template <int NT, class XB>
  __device__ __forceinline__ void step(const Regs& r, int s, int K, int t, const XB& xb, int nt, float (&acc)[NT][4]) const {
    const uint32_t wa[4] = {r.a.x, r.a.y, r.a.z, r.a.w}, wb[4] = {r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const int kq = s * kStep + q * (128 / PER);
      if (PER > 1 && kq >= K) break;   // a group of padding alone: its scale may be anything
      const uint32_t za = T::kNibbleBase | ((r.za >> (8 * q)) & 0xffu) * 0x00010001u;
      const uint32_t zb = T::kNibbleBase | ((r.zb >> (8 * q)) & 0xffu) * 0x00010001u;
      float part[NT][4];
#pragma unroll
      for (int i = 0; i < NT; ++i) part[i][0] = part[i][1] = part[i][2] = part[i][3] = 0.f;
#pragma unroll
      for (int j = 4 / PER * q; j < 4 / PER * (q + 1); ++j) {
        uint32_t pa[4], pb[4];
        unpack(wa[j], za, pa);
        unpack(wb[j], zb, pb);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          if (i < nt) {
            const uint4 b = xb(i, s * kStep + 32 * j + 8 * t);
            T::mma(part[i], pa[0], pb[0], pa[1], pb[1], b.x, b.y);
            T::mma(part[i], pa[2], pb[2], pa[3], pb[3], b.z, b.w);
          }
        }
      }
      const float sa = T::to_float((uint16_t)(r.sa[q / 2] >> (16 * (q % 2)))), sb = T::to_float((uint16_t)(r.sb[q / 2] >> (16 * (q % 2))));
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        if (i < nt) {
          acc[i][0] = fmaf(sa, part[i][0], acc[i][0]);
          acc[i][1] = fmaf(sa, part[i][1], acc[i][1]);
          acc[i][2] = fmaf(sb, part[i][2], acc[i][2]);
          acc[i][3] = fmaf(sb, part[i][3], acc[i][3]);
        }
      }
    }
  }
};

// ---- a warp's walk over its steps -----------------------------------------------------------------------------
// Steps s, s + ds, ... below `end`, with DEPTH steps' loads in flight: preload() issues the first ones (before the
// activations are needed), walk() computes a step and at once refills its registers.
template <class F, int DEPTH>
struct Stream {
  typename F::Regs buf[DEPTH];
  __device__ __forceinline__ void preload(const F& f, int s, int ds, int end, int K, int t) {
#pragma unroll
    for (int u = 0; u < DEPTH; ++u)
      if (s + u * ds < end) buf[u] = f.load(s + u * ds, K, t);
  }
  template <int NT, class XB>
  __device__ __forceinline__ void walk(const F& f, int s, int ds, int end, int K, int t, const XB& xb, int nt, float (&acc)[NT][4]) {
    for (; s < end; s += DEPTH * ds) {
#pragma unroll
      for (int u = 0; u < DEPTH; ++u) {
        const int now = s + u * ds, next = now + DEPTH * ds;
        if (now < end) f.template step<NT>(buf[u], now, K, t, xb, nt, acc);
        if (next < end) buf[u] = f.load(next, K, t);
      }
    }
  }
};

}  // namespace decode
}  // namespace exo

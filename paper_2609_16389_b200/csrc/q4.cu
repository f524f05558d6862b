// 4-bit weights: quantisation, its inverse, and the product of a few tokens with a 4-bit matrix (exo_decode.h).
#include <cooperative_groups.h>

#include <type_traits>

#include "../../include/exo_decode.h"
#include "decode_core.cuh"
#include "decode_host.h"
#include "ptx.cuh"

namespace exo {
namespace decode {
namespace {

// ==== quantisation ===============================================================================================
// A lane holds eight consecutive weights, so a group is 16, 8 or 4 neighbouring lanes and its extremes are a shuffle
// tree; a warp walks along a row, 256 weights at a time.  Memory is the bound (2 or 4 bytes in and 1/2 out per weight) only
// if a weight costs about a dozen instructions: a division takes that many alone.  A group divides by one scale, so the
// quotient is the product with the scale's reciprocal, corrected once by its remainder: with fused operations and a
// correctly rounded reciprocal that is the correctly rounded quotient (P. Markstein, 1990), as the formula has it, wherever
// nothing under- or overflows.
constexpr int kQuantThreads = 256;
constexpr int kQuantSegment = 4096;   // weights of a row per warp

// Eight elements at k .. k + 7 of a row (those at and beyond K are 0, and not written).  ALIGN: bytes that every row's start
// is a multiple of.
template <int BYTES, int ALIGN>
__device__ __forceinline__ void load_eight(const void* row, int k, int K, uint32_t (&w)[2 * BYTES]) {
  const char* p = static_cast<const char*>(row) + (int64_t)k * BYTES;
  if (k + 8 <= K) {
    if constexpr (ALIGN == 16) {
#pragma unroll
      for (int i = 0; i < BYTES / 2; ++i) {
        const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p) + i);
        w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
      }
    } else if constexpr (ALIGN == 8) {
#pragma unroll
      for (int i = 0; i < BYTES; ++i) {
        const uint2 v = __ldcs(reinterpret_cast<const uint2*>(p) + i);
        w[2 * i] = v.x; w[2 * i + 1] = v.y;
      }
    } else if constexpr (ALIGN == 4) {
#pragma unroll
      for (int i = 0; i < 2 * BYTES; ++i) w[i] = __ldcs(reinterpret_cast<const uint32_t*>(p) + i);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(p) + 2 * i;
        w[i] = (uint32_t)h[0] | (uint32_t)h[1] << 16;
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 2 * BYTES; ++i) w[i] = 0;
  for (int i = 0; i < 8; ++i)
    if (k + i < K) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j == i) {
          if constexpr (BYTES == 4) w[j] = reinterpret_cast<const uint32_t*>(p)[j];
          else w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[j] << (16 * (j % 2));
        }
    }
}
template <int BYTES, int ALIGN>
__device__ __forceinline__ void store_eight(void* row, int k, int K, const uint32_t (&w)[2 * BYTES]) {
  char* p = static_cast<char*>(row) + (int64_t)k * BYTES;
  if (k + 8 <= K) {
    if constexpr (ALIGN == 16) {
#pragma unroll
      for (int i = 0; i < BYTES / 2; ++i) __stcs(reinterpret_cast<uint4*>(p) + i, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
    } else if constexpr (ALIGN == 8) {
#pragma unroll
      for (int i = 0; i < BYTES; ++i) reinterpret_cast<uint2*>(p)[i] = make_uint2(w[2 * i], w[2 * i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < 2 * BYTES; ++i) reinterpret_cast<uint32_t*>(p)[i] = w[i];
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (k + i < K) {
      if constexpr (BYTES == 4) reinterpret_cast<uint32_t*>(p)[i] = w[i];
      else reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)(w[i / 2] >> (16 * (i % 2)));
    }
}

// Rows of 16-bit elements at odd addresses can be written by halves only, and a lane that wrote its own eight would touch a sector
// for each: elements 0 .. 255 of a pass change their order in the warp's part of shared memory, so that neighbouring lanes write
// neighbouring elements.  32768 x 4097, us: 98, against 359 without.  At multiples of 4 and 8 bytes the detour loses (111 / 78 and 92 /
// 77), and so it does for reading, which finds the sector's rest in the L1 (164 / 171, 162 / 131 and 150 / 128).
__device__ __forceinline__ void store_halves(uint4* mine, uint16_t* to, int left, const uint32_t (&w)[4]) {
  const int lane = threadIdx.x & 31;
  __syncwarp();                            // what was there has been read
  mine[lane] = make_uint4(w[0], w[1], w[2], w[3]);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (32 * i + lane < left) to[32 * i + lane] = reinterpret_cast<const uint16_t*>(mine)[32 * i + lane];
}

// a / N, correctly rounded (P. Markstein: the product with the rounded reciprocal, corrected by its exact remainder).
template <int N>
__device__ __forceinline__ float divided(float a) {
  if (!(a > 1.0e-30f && a < 1.0e38f)) return __fdiv_rn(a, (float)N);   // where the remainder may underflow, or not be finite
  const float q = a * (1.f / N);
  return fmaf(fmaf(-q, (float)N, a), 1.f / N, q);
}

// Half a warp has a step of 128 weights, eight to a lane.  Measured on a B200 at 65536 x 4096 bf16 in groups of 64: 311 us for both
// directions (207 at the copy bandwidth).  Quantising is bound by its instructions (ncu: 23 per weight, issue slots 79 % used, DRAM 29
// %), its inverse by instructions and memory alike (11 per weight, 69 %, DRAM 38 %).
struct QuantParams {
  int64_t rows, ldw;
  int K, blocks, segments, group;
  void* w;
  uint32_t* codes;
  uint16_t* scales;
  uint8_t* zeros;
};

// T: type of the scales; WT: type of the weights (float: 32 bits).
template <class T, class WT, int ALIGN>
__global__ void __launch_bounds__(kQuantThreads) exo_q4_quantize_kernel(const QuantParams p) {
  constexpr bool WIDE = std::is_same<WT, float>::value;
  constexpr int BYTES = WIDE ? 4 : 2;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int64_t item = ((int64_t)blockIdx.x * kQuantThreads + threadIdx.x) >> 5;
  const int64_t row = item / p.segments;
  if (row >= p.rows) return;
  const int seg = (int)(item - row * p.segments);
  const int k_end = min((seg + 1) * (kQuantSegment / 128), p.blocks) * 128;
  const char* src = static_cast<const char*>(p.w) + row * p.ldw * BYTES;
  const int lanes = p.group / 8, per_row = p.blocks * 128 / p.group, group_log = 31 - __clz(p.group);
  uint32_t* codes = p.codes + row * p.blocks * 16;
  uint16_t* scales = p.scales + row * per_row;
  uint8_t* zeros = p.zeros ? p.zeros + row * per_row : nullptr;
  auto weights = [&](const uint32_t (&w)[2 * BYTES], float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (WIDE) v[i] = __uint_as_float(w[i]);
      else v[i] = WT::to_float((uint16_t)(w[i / 2] >> (16 * (i % 2))));
    }
  };
  uint32_t ahead[2 * BYTES];
  load_eight<BYTES, ALIGN>(src, seg * kQuantSegment + 8 * lane, p.K, ahead);
  for (int k0 = seg * kQuantSegment; k0 < k_end; k0 += 256) {
    const int k = k0 + 8 * lane;
    float v[8];
    weights(ahead, v);
    if (k0 + 256 < k_end) load_eight<BYTES, ALIGN>(src, k + 256, p.K, ahead);
    float lo = 0.f, hi = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) { lo = fminf(lo, v[i]); hi = fmaxf(hi, v[i]); }
    if (!p.zeros) hi = fmaxf(hi, -lo);
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      if (o < lanes) {
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        if (p.zeros) lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      }
    }
    const float raw = p.zeros ? divided<15>(hi - lo) : divided<7>(hi);
    const uint16_t s16 = T::from_float(fminf(raw, T::max_finite()));
    const float s = T::to_float(s16);
    // scales whose quotients are beyond 16, or whose remainders may underflow, or none at all
    const bool plain = s > 1.0e-30f && raw <= T::max_finite();
    const float inverse = __frcp_rn(plain ? s : 1.f);
    auto quotient = [&](float v) {
      const float y = v * inverse;
      return fmaf(fmaf(-y, s, v), inverse, y);
    };
    int zero = 8;
    if (p.zeros && s > 0.f) zero = (int)fminf(fmaxf(rintf(plain ? quotient(-lo) : __fdiv_rn(-lo, s)), 0.f), 15.f);
    uint32_t word = 0;
    if (plain) {
      const int base = 0x4b400000 - zero;       // 1.5 * 2^23 + v has the rounded v in its last bits
#pragma unroll
      for (int i = 0; i < 8; ++i)
        word += (uint32_t)__vimin_s32_relu(__float_as_int(quotient(v[i]) + 12582912.f) - base, 15) << (4 * (i / 2 + 4 * (i % 2)));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float q = s > 0.f ? rintf(__fdiv_rn(v[i], s)) + (float)zero : (float)zero;   // without zero points: -8 .. 7 plus 8
        word |= (uint32_t)fminf(fmaxf(q, 0.f), 15.f) << (4 * (i / 2 + 4 * (i % 2)));
      }
    }
    if (k < k_end) {   // the last pass may hold one block of 128 only
      const int l = lane & 15;
      codes[k / 128 * 16 + 4 * (l & 3) + (l >> 2)] = word;
      if ((lane & (lanes - 1)) == 0) {
        scales[k >> group_log] = s16;
        if (p.zeros) zeros[k >> group_log] = (uint8_t)zero;
      }
    }
  }
}

template <class T, class WT, int ALIGN>
__global__ void __launch_bounds__(kQuantThreads) exo_q4_dequantize_kernel(const QuantParams p) {
  constexpr bool WIDE = std::is_same<WT, float>::value;
  constexpr int BYTES = WIDE ? 4 : 2;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int64_t item = ((int64_t)blockIdx.x * kQuantThreads + threadIdx.x) >> 5;
  const int64_t row = item / p.segments;
  if (row >= p.rows) return;
  const int seg = (int)(item - row * p.segments);
  const int k_end = min((seg + 1) * (kQuantSegment / 128), p.blocks) * 128;
  char* dst = static_cast<char*>(p.w) + row * p.ldw * BYTES;
  const int group_log = 31 - __clz(p.group);
  const int64_t groups = row * (p.blocks * 128 / p.group);
  const uint32_t* codes = p.codes + row * p.blocks * 16 + 4 * (lane & 3) + ((lane & 15) >> 2);
  constexpr int N = 4;   // passes whose loads are in flight together
  constexpr bool HALVES = ALIGN == 2;
  __shared__ uint4 moved[HALVES ? kQuantThreads : 1];
  for (int k0 = seg * kQuantSegment + 8 * lane; k0 - (HALVES ? 8 * lane : 0) < k_end; k0 += N * 256) {   // by halves all lanes take part
    uint32_t word[N];
    float s[N], zero[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int k = k0 + 256 * u;
      if constexpr (HALVES) {
        word[u] = 0;
        s[u] = zero[u] = 0.f;
      }
      if (k < k_end) {
        word[u] = __ldcs(codes + k / 128 * 16);
        s[u] = T::to_float(__ldg(p.scales + groups + (k >> group_log)));
        zero[u] = 8388608.f + (p.zeros ? (float)__ldg(p.zeros + groups + (k >> group_log)) : 8.f);
      }
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int k = k0 + 256 * u;
      if (k - (HALVES ? 8 * lane : 0) < k_end) {
        float v[8];
        uint32_t out[2 * BYTES];
#pragma unroll
        for (int i = 0; i < 8; ++i)   // 2^23 + code, less 2^23 + zero: exact, as is the product with the scale
          v[i] = (__uint_as_float((word[u] >> (4 * (i / 2 + 4 * (i % 2))) & 15u) | 0x4b000000u) - zero[u]) * s[u];
#pragma unroll
        for (int i = 0; i < 2 * BYTES; ++i) {
          if constexpr (WIDE) out[i] = __float_as_uint(v[i]);
          else out[i] = WT::pair(v[2 * i], v[2 * i + 1]);
        }
        if constexpr (HALVES) store_halves(moved + (threadIdx.x & ~31u), reinterpret_cast<uint16_t*>(dst) + (k - 8 * lane), min(p.K, k_end) - (k - 8 * lane), out);
        else store_eight<BYTES, ALIGN>(dst, k, p.K, out);
      }
    }
  }
}

// ==== the product of a few tokens with a 4-bit matrix =============================================================
// The general form, for activations that fit no shared memory (rows of tens of thousands of weights): 16 weight rows and up to
// eight tokens to a CTA, whose eight warps split k; the CTAs of a cluster split it once more.  The activations are staged
// in shared memory a chunk of k at a time (rows 64 bytes off a multiple of 128, so that a fragment load is free of bank
// conflicts).  Partial sums meet in shared memory in warp order, then in distributed shared memory in rank order.
constexpr int kGemvThreads = 256, kGemvWarps = 8;

struct GemvParams {
  const uint8_t* codes;
  const uint16_t* scales;
  const uint8_t* zeros;
  const uint16_t* x;
  void* y;
  int64_t ldx, ldy, rows;
  int K, tokens, blocks;        // blocks: steps of 128
  int chunk;                    // steps staged at a time
  int y_dtype;
  int x_align;                  // bytes that every row of x starts on a multiple of, 16 at most
  bool x_aligned;               // 16 of them
  float alpha, beta;
};

__host__ __device__ constexpr int gemv_pitch(int chunk) { return chunk * 256 + 64; }   // bytes of a token's staged row

// The lane's places in the scales of the tile that begins at `row`, from step k_begin on; rows that do not exist repeat the last
// one, nobody stores theirs.
template <class SC, int PER, bool ZEROS>
__device__ __forceinline__ typename SC::Rows scale_rows(const GemvParams& p, int row, int k_begin) {
  const int lane = threadIdx.x & 31;
  const int64_t r0 = min((int64_t)row + (lane >> 2), p.rows - 1), r1 = min((int64_t)row + (lane >> 2) + 8, p.rows - 1);
  const int64_t at0 = (r0 * p.blocks + k_begin + (lane & 3)) * PER, at1 = (r1 * p.blocks + k_begin + (lane & 3)) * PER;
  return typename SC::Rows{p.scales + at0, p.scales + at1, ZEROS ? p.zeros + at0 : nullptr, ZEROS ? p.zeros + at1 : nullptr};
}

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

template <class T, int PER, bool ZEROS>
__global__ void __launch_bounds__(kGemvThreads, 2) exo_gemv_q4_kernel(const GemvParams p) {
  namespace cg = cooperative_groups;
  extern __shared__ __align__(128) uint8_t smem[];
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), r = (int)cluster.block_rank();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int64_t tile_row = (int64_t)(blockIdx.x / S) * 16;
  const int64_t row0 = min(tile_row + g, p.rows - 1), row1 = min(tile_row + g + 8, p.rows - 1);
  const int first = blockIdx.y * 8, tokens = min(p.tokens - first, 8);   // this CTA's tokens
  const int s_begin = (int)((int64_t)p.blocks * r / S), s_end = (int)((int64_t)p.blocks * (r + 1) / S);
  const int whole = p.K / 128;          // whole steps; a part of one may follow
  using F = RowsQ4<T, PER, ZEROS>;
  float acc[1][4] = {{0.f, 0.f, 0.f, 0.f}};

  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int pitch = gemv_pitch(p.chunk);
  for (int c = s_begin; c < s_end; c += p.chunk) {
    const int c_end = min(c + p.chunk, s_end), s = c + warp;
    F f;
    f.c0 = p.codes + (row0 * p.blocks + s) * 64;
    f.c1 = p.codes + (row1 * p.blocks + s) * 64;
    f.s0 = p.scales + (row0 * p.blocks + s) * PER;
    f.s1 = p.scales + (row1 * p.blocks + s) * PER;
    if constexpr (ZEROS) {
      f.z0 = p.zeros + (row0 * p.blocks + s) * PER;
      f.z1 = p.zeros + (row1 * p.blocks + s) * PER;
    }
    f.begin(t);
    const int n = steps_of(s, kGemvWarps, min(c_end, whole));
    Stream<F, kGemvWarps, 4> stream;
    stream.preload(f, n);
    if (c != s_begin) __syncthreads();   // the previous chunk has been read
    const int per_token = (c_end - c) * 16;
    for (int i = threadIdx.x; i < tokens * per_token; i += kGemvThreads) {
      const int token = i / per_token, e = i - token * per_token;
      *reinterpret_cast<uint4*>(smem + token * pitch + e * 16) =
          load8_checked(p.x + (int64_t)(first + token) * p.ldx, c * 128 + e * 8, p.K, p.x_aligned);
    }
    __syncthreads();
    // columns beyond the tokens read the last row again
    XShared x{ptx::smem_u32(smem) + min(g, tokens - 1) * pitch + warp * 256 + 16 * t, 0};
    stream.template walk<1>(f, n, x, All<1>(), acc);
    if (s + n * kGemvWarps == whole && whole < c_end) f.template step_tail<1>(f.load_tail(0, t), p.K - whole * 128, x, All<1>(), acc);
  }

  // sums over the warps, then over the cluster
  __syncthreads();
  float4* red = reinterpret_cast<float4*>(smem);                        // [warp][lane]
  float4* part = red + kGemvWarps * 32;                                 // [lane]
  red[warp * 32 + lane] = make_float4(acc[0][0], acc[0][1], acc[0][2], acc[0][3]);
  __syncthreads();
  auto finish = [&](float4 v) {
    const int token = first + 2 * t;
    const int64_t row = tile_row + g;
    store_y<T>(p, token, row, v.x);
    store_y<T>(p, token + 1, row, v.y);
    store_y<T>(p, token, row + 8, v.z);
    store_y<T>(p, token + 1, row + 8, v.w);
  };
  auto add = [](float4& v, const float4& w) { v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w; };
  if (warp == 0) {
    float4 v = red[lane];
#pragma unroll
    for (int q = 1; q < kGemvWarps; ++q) add(v, red[q * 32 + lane]);
    if (S == 1) finish(v);
    else part[lane] = v;
  }
  if (S > 1) {
    cluster.sync();
    if (r == 0 && warp == 0) {
      float4 v = part[lane];
      for (int q = 1; q < S; ++q) add(v, cluster.map_shared_rank(part, q)[lane]);
      finish(v);
    }
    cluster.sync();   // no CTA leaves while another may still read its sums
  }
}

// ==== one or two tokens and a large matrix: integer products ========================================================
// Turning 4-bit codes into 16-bit numbers costs the general kernel 11 instructions for eight weights, and at one token
// that, not memory, is what it is bound by (181 clocks a step of 16 x 128 weights, where memory delivers one every 178).
// Integers need three: the codes of a word, masked, are the bytes that mma.m16n8k32 takes as unsigned operands.  The
// activations become signed bytes: per token and step of 128 they are scaled by a power of two to integers of 30
// bits (exact for what is down to 2^-22 of the step's largest in bf16, 2^-19 in fp16; a smaller value is off by at most
// 2^-30 of the largest), whose four balanced digits are four columns of the product.  The columns of few tokens are idle
// otherwise.  A group's sum of (code - zero) * digit is an exact integer; it comes out as the float 1.5 * 2^23 + sum, since
// the accumulator starts with that float's bits less zero * (sum of digits).  From there on everything is fp32: an integer is multiplied by its
// weights' scale, which cannot underflow, then by its activations' with the weight of the top digit in it, so that the top digits' sum is of
// the result's own size.  The lower digits' sums may be four times that: a result that is not finite is summed again in floats.
//
// Weights come through shared memory: each warp keeps a ring of pieces (eight steps of 16 rows) that it fills itself by tiled
// copies.  A lane's parts of a step are 16 bytes of rows g and g + 8.
//
// The digits have to be made by every CTA, so the matrix has to be large before the saved instructions are ahead of the 16-bit
// kernel below.  Measured in a CUDA graph, integer against 16-bit products (us, group 128, bf16):
//                   1024 x 2048  4096 x 4096  8192 x 8192  16384 x 8192  32768 x 16384
//   one token         4.0 / 3.0    5.2 / 5.0  12.2 / 12.6   18.4 / 20.4    49.8 / 67.9
//   two tokens        4.6 / 3.0    6.5 / 5.2  13.2 / 12.9   19.6 / 20.8    58.7 / 68.3
// and with three and four tokens, whose digits take twice the columns, 83 / 71 and 87 / 72 on 32768 x 16384.  Hence two tokens at
// most, and 256 KB of weights for every SM.  32768 x 16384 is 277 MB: one token at 5.6 TB/s, 0.85 of what a copy does (called
// from Python one by one 53 us, 0.80).
constexpr int kFewWarps = 8, kFewThreads = 32 * kFewWarps, kFewPiece = 8, kFewTokens = 2, kFewSteps = 256;   // steps of 1 KB per SM
constexpr int kMagic = 0x4b400000;        // 1.5 * 2^23

struct FewParams {
  GemvParams g;
  int nk_log;       // parts of a tile's steps: 1 << nk_log
  int stages;
  WaitBound wait;
  int digits_at, start_at, step_scale_at, ring_at;   // offsets in shared memory; the sums come first, the barriers before them
};

__device__ __forceinline__ void mma_u8s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// four words of four bytes, transposed
__device__ __forceinline__ void transpose4(const uint32_t (&v)[4], uint32_t (&d)[4]) {
  const uint32_t x0 = __byte_perm(v[0], v[1], 0x5140), x1 = __byte_perm(v[2], v[3], 0x5140);
  const uint32_t y0 = __byte_perm(v[0], v[1], 0x7362), y1 = __byte_perm(v[2], v[3], 0x7362);
  d[0] = __byte_perm(x0, x1, 0x5410); d[1] = __byte_perm(x0, x1, 0x7632);
  d[2] = __byte_perm(y0, y1, 0x5410); d[3] = __byte_perm(y0, y1, 0x7632);
}

// eight 16-bit values to shared memory, asynchronously, by copies of `align` bytes (4, 8 or 16 at least)
__device__ __forceinline__ void copy_eight(uint32_t to, const uint16_t* from, int align) {
  if (align >= 16) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  } else if (align == 8) {
#pragma unroll
    for (int i = 0; i < 2; ++i) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to + 8 * i), "l"(from + 4 * i) : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to + 4 * i), "l"(from + 2 * i) : "memory");
  }
}
__device__ __forceinline__ int rank_part(int blocks, int r, int S) { return (int)((int64_t)blocks * r / S); }

// A row's product with a token in 32-bit floats, value by value: for tokens that have infinities or NaN, which are no integers, and sums of
// digits that overflow.  codes, scales and zeros are the row's, x the token's.
template <class T>
__device__ __noinline__ float sum_in_floats(const uint32_t* codes, const uint16_t* scales, const uint8_t* zeros, const uint16_t* x, int per, int K) {
  float v = 0.f;
  for (int group = 0; group * (128 / per) < K; ++group) {
    const int zero = zeros ? zeros[group] : 8, end = min((group + 1) * (128 / per), K);
    float part = 0.f;
    for (int k = group * (128 / per); k < end; ++k) {
      const int i = k & 7, n = i / 2 + 4 * (i & 1), j = k >> 5 & 3, t = k >> 3 & 3;
      const uint32_t word = codes[k / 128 * 16 + 4 * t + j];
      part = fmaf((float)((int)(word >> (4 * n) & 15u) - zero), T::to_float(x[k]), part);
    }
    v = fmaf(T::to_float(scales[group]), part, v);
  }
  return v;
}

template <class T, int PER, bool ZEROS>
__global__ void __launch_bounds__(kFewThreads, 1) exo_gemv_q4_few_kernel(const FewParams fp, const __grid_constant__ CUtensorMap map) {
  namespace cg = cooperative_groups;
  constexpr int COLS = 8;                  // two tokens of four digits
  const GemvParams& p = fp.g;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int strange;                  // bit t: token t has values that are not finite
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int clusters = gridDim.x / S, cl = blockIdx.x / S;
  const int tiles = (int)((p.rows + 15) / 16), nk = 1 << fp.nk_log;
  const int units = ((tiles - cl + clusters - 1) / clusters) << fp.nk_log;   // of this cluster
  const int k_begin = rank_part(p.blocks, rank, S), k_steps = rank_part(p.blocks, rank + 1, S) - k_begin;
  const int pieces = (k_steps + kFewPiece - 1) / kFewPiece;
  const int stage_bytes = kFewPiece * 1024;
  float* sums = reinterpret_cast<float*>(smem + 256);                        // [unit][token][16]
  const int col_pitch = k_steps * 128 + 16;
  const uint32_t bar = ptx::smem_u32(smem) + warp * 32, ring = ptx::smem_u32(smem + fp.ring_at) + warp * fp.stages * stage_bytes;
  if (lane == 0)
    for (int i = 0; i < fp.stages; ++i) ptx::mbar_init(bar + 8 * i, 1);
  ptx::fence_mbar_init();
  Copies copies(fp.wait);
  if (threadIdx.x == 0) strange = 0;
  __syncwarp();
  // unit u: tile cl + (u >> nk_log) * clusters, part u & (nk - 1) of its pieces
  auto row_of = [&](int u) { return (cl + (u >> fp.nk_log) * clusters) * 16; };
  auto begin_of = [&](int u) { return (pieces * (u & (nk - 1))) >> fp.nk_log; };
  auto end_of = [&](int u) { return (pieces * ((u & (nk - 1)) + 1)) >> fp.nk_log; };

  int iu = warp, ip, islot = 0;            // the next copy
  ip = begin_of(iu);
  auto issue = [&]() {
    if (iu < units) {
      const int row = row_of(iu), step = k_begin + ip * kFewPiece;
      if (copies.issues) {
        ptx::mbar_arrive_expect_tx(bar + 8 * islot, stage_bytes);
        ptx::tma_load_3d(ring + islot * stage_bytes, &map, 0, row, step, bar + 8 * islot);
      }
      islot = islot + 1 == fp.stages ? 0 : islot + 1;
      if (++ip == end_of(iu)) {
        iu += kFewWarps;
        ip = begin_of(iu);
      }
    }
  };
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  for (int i = 0; i < fp.stages; ++i) issue();

  using SC = StepScales<T, PER, ZEROS, 8>;
  typename SC::Rows srows;
  auto load_scales = [&](SC& sc, int piece) {
    const int s = piece * kFewPiece;
    sc.load(srows, s, min(kFewPiece, k_steps - s), p.K - (k_begin + s) * 128);
  };
  int cu = warp;
  int cp = begin_of(cu);
  SC cur, nxt;
  if (cu < units) {
    srows = scale_rows<SC, PER, ZEROS>(p, row_of(cu), k_begin);
    load_scales(cur, cp);
  }

  // the tokens' digits: 16 lanes to a step, eight values each
  uint8_t* digits = smem + fp.digits_at;                                     // [column][k_steps][t][j][8]
  int* start = reinterpret_cast<int*>(smem + fp.start_at);                   // [k_steps * PER][COLS]
  float* step_scale = reinterpret_cast<float*>(smem + fp.step_scale_at);     // [k_steps][2]
  __syncthreads();
  const int all_parts = p.tokens * k_steps * 16;
  auto raw_part = [&](int i) {             // clamped, so that all lanes take part in the shuffles below
    const int item = min(i >> 4, p.tokens * k_steps - 1), token = item / k_steps, s = item - token * k_steps;
    return load8_checked(p.x + (int64_t)token * p.ldx, (k_begin + s) * 128 + 8 * (i & 15), p.K, p.x_aligned);
  };
  uint4 raw_next = raw_part(threadIdx.x);
  for (int i0 = 0; i0 < all_parts; i0 += kFewThreads) {
    const int i = i0 + threadIdx.x, item = min(i >> 4, p.tokens * k_steps - 1), e = i & 15;
    const int token = item / k_steps, s = item - token * k_steps;
    const uint4 raw = raw_next;
    if (i0 + kFewThreads < all_parts) raw_next = raw_part(i + kFewThreads);
    const uint32_t rw[4] = {raw.x, raw.y, raw.z, raw.w};
    float v[8], top = 0.f;
    bool odd = false;
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      v[n] = T::to_float((uint16_t)(rw[n / 2] >> (16 * (n % 2))));
      if (!(fabsf(v[n]) <= 3.4028235e38f)) { v[n] = 0.f; odd = true; }
      top = fmaxf(top, fabsf(v[n]));
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (odd) atomicOr(&strange, 1 << token);
    const int up = 156 - (int)(__float_as_uint(top) >> 23), half = up / 2;   // |v| * 2^up < 2^30; up is 156 at most
    const float factor = __uint_as_float((uint32_t)(half + 127) << 23), factor2 = __uint_as_float((uint32_t)(up - half + 127) << 23);
    uint32_t q[8];
#pragma unroll
    for (int n = 0; n < 8; ++n) q[n] = ((uint32_t)__float2int_rn(v[n] * factor * factor2) + 0x00808080u) ^ 0x00808080u;
    const uint32_t first[4] = {q[0], q[4], q[1], q[5]}, second[4] = {q[2], q[6], q[3], q[7]};   // the order of the codes of a word, low and high
    uint32_t d0[4], d1[4];
    transpose4(first, d0);
    transpose4(second, d1);
    int sum[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      sum[c] = __dp4a((int)d0[c], 0x01010101, __dp4a((int)d1[c], 0x01010101, 0));
#pragma unroll
      for (int o = 1; o < 16 / PER; o <<= 1) sum[c] += __shfl_xor_sync(0xffffffffu, sum[c], o);
    }
    if (i < all_parts) {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<uint2*>(digits + (token * 4 + c) * col_pitch + s * 128 + (e & 3) * 32 + (e >> 2) * 8) = make_uint2(d0[c], d1[c]);
      if (e % (16 / PER) == 0) {
        int* to = start + ((s * PER + e / (16 / PER)) * COLS + token * 4);
#pragma unroll
        for (int c = 0; c < 4; ++c) to[c] = ZEROS ? -sum[c] : kMagic - 8 * sum[c];
      }
      if (e == 0) step_scale[2 * s + token] = ldexpf(1.f, 24 - up);
    }
  }
  __syncthreads();

  float acc[4] = {};
  const uint32_t xat = ptx::smem_u32(digits) + min(g, p.tokens * 4 - 1) * col_pitch + t * 32;   // columns beyond the tokens repeat the last one; nobody reads them
  int cslot = 0;
  uint32_t parity = 0;
  while (cu < units) {
    int nu = cu, np = cp + 1;              // the piece after this one
    const bool ends = np == end_of(cu);
    if (ends) {
      nu += kFewWarps;
      np = begin_of(nu);
      if (nu < units) srows = scale_rows<SC, PER, ZEROS>(p, row_of(nu), k_begin);
    }
    if (nu < units) load_scales(nxt, np);
    copies.wait<true>(bar + 8 * cslot, parity, fp.wait);
    const uint32_t w = ring + cslot * stage_bytes + g * 64 + t * 16;
    const int s0 = cp * kFewPiece, n = min(kFewPiece, k_steps - s0);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (u < n) {
        const uint4 ra = lds128(w + u * 1024), rb = lds128(w + u * 1024 + 512);
        const uint32_t wa[4] = {ra.x, ra.y, ra.z, ra.w}, wb[4] = {rb.x, rb.y, rb.z, rb.w};
        uint32_t sa[(PER + 1) / 2], sb[(PER + 1) / 2], za, zb;
        cur.get(u, sa, sb, za, zb);
        const int s = s0 + u;
        const uint4 x0 = lds128(xat + s * 128), x1 = lds128(xat + s * 128 + 16);
        const uint32_t xl[4] = {x0.x, x0.z, x1.x, x1.z}, xh[4] = {x0.y, x0.w, x1.y, x1.w};
        const float ss = step_scale[2 * s + t / 2];
        float part[4];
#pragma unroll
        for (int q = 0; q < PER; ++q) {
          const int2 c = *reinterpret_cast<const int2*>(start + (s * PER + q) * COLS + 2 * t);
          int d[4] = {c.x, c.y, c.x, c.y};
          if constexpr (ZEROS) {
            const int z0 = (za >> (8 * q)) & 0xff, z1 = (zb >> (8 * q)) & 0xff;
            d[0] = z0 * c.x + kMagic; d[1] = z0 * c.y + kMagic;
            d[2] = z1 * c.x + kMagic; d[3] = z1 * c.y + kMagic;
          }
#pragma unroll
          for (int j = 4 / PER * q; j < 4 / PER * (q + 1); ++j)
            mma_u8s8(d, wa[j] & 0x0f0f0f0fu, wb[j] & 0x0f0f0f0fu, (wa[j] >> 4) & 0x0f0f0f0fu, (wb[j] >> 4) & 0x0f0f0f0fu, xl[j], xh[j]);
          const float fa = T::to_float((uint16_t)(sa[q / 2] >> (16 * (q % 2)))), fb = T::to_float((uint16_t)(sb[q / 2] >> (16 * (q % 2))));
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const float sum = __int_as_float(d[c]) - 12582912.f;
            part[c] = q == 0 ? (c < 2 ? fa : fb) * sum : fmaf(c < 2 ? fa : fb, sum, part[c]);
          }
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] = fmaf(ss, part[c], acc[c]);
      }
    }
    __syncwarp();
    issue();
    cslot = cslot + 1 == fp.stages ? 0 : cslot + 1;
    parity ^= cslot == 0 ? 1u : 0u;
    if (ends) {                            // digits 2 (t % 2) and 2 (t % 2) + 1 of token t / 2, weighted by 256^(digit - 3)
      const float lo = t & 1 ? 0x1p-8f : 0x1p-24f, hi = t & 1 ? 1.f : 0x1p-16f;
      float* out = sums + cu * p.tokens * 16;
      float v0 = fmaf(hi, acc[1], lo * acc[0]), v1 = fmaf(hi, acc[3], lo * acc[2]);
      v0 += __shfl_xor_sync(0xffffffffu, v0, 1);
      v1 += __shfl_xor_sync(0xffffffffu, v1, 1);
      if ((t & 1) == 0 && t / 2 < p.tokens) {
        out[t / 2 * 16 + g] = v0;
        out[t / 2 * 16 + g + 8] = v1;
      }
      acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
    }
    cu = nu; cp = np;
    cur = nxt;
  }
  // one value per row and token: over the parts of k in the CTA, then over the cluster
  if (S > 1) cluster.sync(); else __syncthreads();
  const int values = (units >> fp.nk_log) * p.tokens * 16;
  for (int i = rank * kFewThreads + threadIdx.x; i < values; i += S * kFewThreads) {
    const int tile = i / (p.tokens * 16), at = i - tile * (p.tokens * 16), token = at >> 4;
    const int row = (cl + tile * clusters) * 16 + (at & 15);
    float v = 0.f;
    bool floats = false;
    for (int r = 0; r < S; ++r) {
      const float* from = (S > 1 ? cluster.map_shared_rank(sums, r) : sums) + (tile << fp.nk_log) * p.tokens * 16 + at;
      for (int j = 0; j < nk; ++j) v += from[j * p.tokens * 16];
      floats = floats || ((S > 1 ? *cluster.map_shared_rank(&strange, r) : strange) >> token & 1);
    }
    if ((floats || !(fabsf(v) <= 3.4028235e38f)) && row < p.rows) {
      const int64_t at = (int64_t)row * p.blocks;
      v = sum_in_floats<T>(reinterpret_cast<const uint32_t*>(p.codes) + at * 16, p.scales + at * PER, ZEROS ? p.zeros + at * PER : nullptr,
                           p.x + (int64_t)token * p.ldx, PER, p.K);
    }
    store_y<T>(p, token, row, v);
  }
  if (S > 1) cluster.sync();   // no CTA leaves while another may still read its sums
}

// ==== all others up to 64 tokens =====================================================================================
// The same cut, with 16-bit products: a step's codes become exact 16-bit integers once for NT tiles of
// eight tokens, whose values for the CTA's part of k lie in shared memory for the whole run (rows 64 bytes off a
// multiple of 128, so that a fragment load is free of bank conflicts).  Eight more tokens cost a step 8 matrix instructions and
// four 512-byte loads of activations.  16384 x 8192 (69 MB, 10.7 us at the copy bandwidth), us: 20.4 for one token, 23 for 8, 30 for
// 16, 37 for 24: at one token the unpacking is the bound, and every further tile adds its loads and products, which a warp
// does not overlap with the unpacking (ncu at 24 tokens: issue slots 51 % used, the tensor pipe 35 %, DRAM 20 %).
constexpr int kBatchWarps = 16, kBatchThreads = 32 * kBatchWarps, kBatchPiece = 2;

template <class T, int PER, bool ZEROS, int NT>
__global__ void __launch_bounds__(kBatchThreads, 1) exo_gemv_q4_batch_kernel(const FewParams fp, const __grid_constant__ CUtensorMap map) {
  namespace cg = cooperative_groups;
  using F = RowsQ4<T, PER, ZEROS>;
  const GemvParams& p = fp.g;
  extern __shared__ __align__(128) uint8_t smem[];
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int clusters = gridDim.x / S, cl = blockIdx.x / S;
  const int first = blockIdx.y * 8 * NT, tokens = min(p.tokens - first, 8 * NT);   // this CTA's tokens
  const int tiles = (int)((p.rows + 15) / 16), nk = 1 << fp.nk_log;
  const int units = ((tiles - cl + clusters - 1) / clusters) << fp.nk_log;         // of this cluster
  const int k_begin = rank_part(p.blocks, rank, S), k_steps = rank_part(p.blocks, rank + 1, S) - k_begin;
  const int pieces = (k_steps + kBatchPiece - 1) / kBatchPiece, stage_bytes = kBatchPiece * 1024;
  float* sums = reinterpret_cast<float*>(smem + 512);                              // [unit][token][16]
  uint8_t* xs = smem + fp.digits_at;                                               // [token][pitch]
  const int pitch = k_steps * 256 + 64;
  const uint32_t bar = ptx::smem_u32(smem) + warp * 32, ring = ptx::smem_u32(smem + fp.ring_at) + warp * fp.stages * stage_bytes;
  if (lane == 0) {
    for (int i = 0; i < fp.stages; ++i) ptx::mbar_init(bar + 8 * i, 1);
    ptx::prefetch_tensormap(&map);
  }
  ptx::fence_mbar_init();
  Copies copies(fp.wait);
  __syncwarp();
  auto row_of = [&](int u) { return (cl + (u >> fp.nk_log) * clusters) * 16; };
  auto begin_of = [&](int u) { return (pieces * (u & (nk - 1))) >> fp.nk_log; };
  auto end_of = [&](int u) { return (pieces * ((u & (nk - 1)) + 1)) >> fp.nk_log; };
  int iu = warp, ip = begin_of(iu), islot = 0;            // the next copy
  auto issue = [&]() {
    if (iu < units) {
      if (copies.issues) {
        ptx::mbar_arrive_expect_tx(bar + 8 * islot, stage_bytes);
        ptx::tma_load_3d(ring + islot * stage_bytes, &map, 0, row_of(iu), k_begin + ip * kBatchPiece, bar + 8 * islot);
      }
      islot = islot + 1 == fp.stages ? 0 : islot + 1;
      if (++ip == end_of(iu)) {
        iu += kBatchWarps;
        ip = begin_of(iu);
      }
    }
  };
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  for (int i = 0; i < fp.stages; ++i) issue();

  F f;
  using SC = StepScales<T, PER, ZEROS, 4>;
  typename SC::Rows srows;
  auto load_scales = [&](SC& sc, int piece) {
    const int s = piece * kBatchPiece;
    sc.load(srows, s, min(kBatchPiece, k_steps - s), p.K - (k_begin + s) * 128);
  };
  SC cur, nxt;
  if (warp < units) {
    srows = scale_rows<SC, PER, ZEROS>(p, row_of(warp), k_begin);
    load_scales(cur, begin_of(warp));
  }

  // all of the activations' loads in flight at once, as wide as their rows' alignment lets them be
  const int per_token = k_steps * 16, segments = (per_token + 31) / 32;
  for (int i = warp; i < tokens * segments; i += kBatchWarps) {
    const int token = i / segments, e = (i - token * segments) * 32 + lane, left = p.K - k_begin * 128;
    if (e < per_token) {
      const uint16_t* from = p.x + (int64_t)(first + token) * p.ldx + k_begin * 128;
      uint8_t* to = xs + token * pitch + e * 16;
      if (p.x_align >= 4 && e * 8 + 8 <= left) copy_eight(ptx::smem_u32(to), from + e * 8, p.x_align);
      else *reinterpret_cast<uint4*>(to) = load8_checked(from, e * 8, left, p.x_aligned);
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  // columns beyond the tokens repeat the last one (one tile) or hold what happens to be there; nobody reads them
  const XShared x0{ptx::smem_u32(xs) + (NT == 1 ? min(g, tokens - 1) : g) * pitch + 16 * t, 8u * pitch};
  int cslot = 0;
  uint32_t parity = 0;
  for (int u = warp; u < units; u += kBatchWarps) {
    float acc[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
    const int end = end_of(u);
    for (int c = begin_of(u); c < end; ++c) {
      copies.wait<false>(bar + 8 * cslot, parity, fp.wait);
      const uint32_t w = ring + cslot * stage_bytes + g * 64 + t * 16;
      const int s0 = c * kBatchPiece, n = min(kBatchPiece, k_steps - s0);
      if (c + 1 < end) {
        load_scales(nxt, c + 1);
      } else if (u + kBatchWarps < units) {
        srows = scale_rows<SC, PER, ZEROS>(p, row_of(u + kBatchWarps), k_begin);
        load_scales(nxt, begin_of(u + kBatchWarps));
      }
#pragma unroll
      for (int v = 0; v < kBatchPiece; ++v) {
        if (v < n) {
          typename F::Regs now;
          cur.get(v, now.sa, now.sb, now.za, now.zb);
          now.a = lds128(w + v * 1024);
          now.b = lds128(w + v * 1024 + 512);
          f.template step<NT, 0>(now, XShared{x0.base + (s0 + v) * 256, x0.stride}, All<NT>(), acc);
        }
      }
      cur = nxt;
      __syncwarp();
      issue();
      cslot = cslot + 1 == fp.stages ? 0 : cslot + 1;
      parity ^= cslot == 0 ? 1u : 0u;
    }
    float* out = sums + u * tokens * 16;
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int token = 8 * i + 2 * t + (c & 1);
        if (token < tokens) out[token * 16 + g + 8 * (c >> 1)] = acc[i][c];
      }
  }
  if (S > 1) cluster.sync(); else __syncthreads();
  const int values = (units >> fp.nk_log) * tokens * 16;
  for (int i = rank * kBatchThreads + threadIdx.x; i < values; i += S * kBatchThreads) {
    const int tile = i / (tokens * 16), at = i - tile * (tokens * 16);
    float v = 0.f;
    for (int r = 0; r < S; ++r) {
      const float* from = (S > 1 ? cluster.map_shared_rank(sums, r) : sums) + (tile << fp.nk_log) * tokens * 16 + at;
      for (int j = 0; j < nk; ++j) v += from[j * tokens * 16];
    }
    store_y<T>(p, first + at / 16, (cl + tile * clusters) * 16 + (at & 15), v);
  }
  if (S > 1) cluster.sync();   // no CTA leaves while another may still read its sums
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
using FewFn = void (*)(FewParams, CUtensorMap);
template <class T, bool ZEROS> GemvFn pick_group(int group) {
  return group == 128 ? exo_gemv_q4_kernel<T, 1, ZEROS> : group == 64 ? exo_gemv_q4_kernel<T, 2, ZEROS> : exo_gemv_q4_kernel<T, 4, ZEROS>;
}
template <class T> GemvFn pick_gemv(int group, bool zeros) { return zeros ? pick_group<T, true>(group) : pick_group<T, false>(group); }

// few: the integer kernel; else the 16-bit one with nt tiles of eight tokens
template <class T, int PER, bool ZEROS> FewFn pick_few_tiles(bool few, int nt) {
  return few ? exo_gemv_q4_few_kernel<T, PER, ZEROS>
         : nt == 1 ? exo_gemv_q4_batch_kernel<T, PER, ZEROS, 1> : nt == 2 ? exo_gemv_q4_batch_kernel<T, PER, ZEROS, 2>
         : nt == 3 ? exo_gemv_q4_batch_kernel<T, PER, ZEROS, 3> : exo_gemv_q4_batch_kernel<T, PER, ZEROS, 4>;
}
template <class T, bool ZEROS> FewFn pick_few_group(int group, bool few, int nt) {
  return group == 128 ? pick_few_tiles<T, 1, ZEROS>(few, nt) : group == 64 ? pick_few_tiles<T, 2, ZEROS>(few, nt) : pick_few_tiles<T, 4, ZEROS>(few, nt);
}
template <class T> FewFn pick_few(int group, bool zeros, bool few, int nt) {
  return zeros ? pick_few_group<T, true>(group, few, nt) : pick_few_group<T, false>(group, few, nt);
}

// How the integer kernel is cut: one CTA per SM with pieces of 8 steps, which the copies like best (32768 x 16384, one token:
// 50 us; 55 with two CTAs and pieces of 4).  The cluster cuts k where a CTA's digits would take more than 40 KB.  False: not
// for this size, or the sums do not fit.
bool plan_few(FewParams& fp, const GemvParams& p, int per, int sms, unsigned* ctas, unsigned* cluster, size_t* smem) {
  const int64_t tiles = (p.rows + 15) / 16;
  if (p.tokens > kFewTokens || tiles * p.blocks < (int64_t)sms * kFewSteps) return false;
  int S = 1;
  while (S < 8 && p.blocks >= 2 * S && (int64_t)4 * p.tokens * ((p.blocks + S - 1) / S) * 128 > 40 * 1024) S *= 2;
  const int slice = (p.blocks + S - 1) / S, least = p.blocks / S;
  const int64_t slots = resident_clusters(8 + S, (void*)exo_gemv_q4_few_kernel<Bf16, 1, false>, kFewThreads, 200 * 1024, (unsigned)S, sms, 1);
  const int64_t clusters = tiles < slots ? tiles : slots;
  const int most = (int)((tiles + clusters - 1) / clusters);     // tiles of a cluster
  // parts of k: two pieces each, or fewer where the CTA would otherwise have less than a part for every warp
  fp.nk_log = 0;
  while (fp.nk_log < 3 && (least + kFewPiece - 1) / kFewPiece >= ((most << fp.nk_log) < kFewWarps ? 2 : 4) << fp.nk_log) ++fp.nk_log;
  const int turns = ((most << fp.nk_log) + kFewWarps - 1) / kFewWarps;
  const int pieces = ((slice + kFewPiece - 1) / kFewPiece + (1 << fp.nk_log) - 1) >> fp.nk_log;
  fp.stages = turns * pieces < 2 ? 1 : 2;
  int64_t at = 256 + (int64_t)(most << fp.nk_log) * p.tokens * 64;
  fp.digits_at = (int)at; at += 4 * p.tokens * ((int64_t)slice * 128 + 16);
  fp.start_at = (int)at; at += (int64_t)slice * per * 8 * 4;
  fp.step_scale_at = (int)at; at += (int64_t)slice * 2 * 4;
  at = (at + 127) / 128 * 128;
  fp.ring_at = (int)at;
  at += kFewWarps * fp.stages * kFewPiece * 1024;
  fp.g = p;
  *ctas = (unsigned)(clusters * S);
  *cluster = (unsigned)S;
  *smem = (size_t)at;
  return at <= kMostSmem;
}

// How the kernel for more tokens is cut, one CTA to an SM; nt is the number of tiles of eight tokens that a CTA keeps.  The
// smallest cluster whose CTAs hold their part of the activations and of the sums, on the clusters that the device holds (16384 x 8192,
// 24 tokens: 37 us with the 33 clusters of four that there are, 67 with 37).  Returns an estimate of the time, in 16ths of a
// microsecond or so, or 0 where nothing fits.
int64_t plan_batch(FewParams& fp, const GemvParams& p, int sms, int nt, unsigned* ctas, unsigned* cluster, size_t* smem) {
  const int64_t tiles = (p.rows + 15) / 16, staged = nt == 1 && p.tokens < 8 ? p.tokens : 8 * nt, tokens = p.tokens < 8 * nt ? p.tokens : 8 * nt;
  const int64_t groups = (p.tokens + 8 * nt - 1) / (8 * nt);
  for (int S = 1; S <= 8 && (S == 1 || p.blocks >= S); S *= 2) {
    const int slice = (p.blocks + S - 1) / S, least = p.blocks / S;
    const int64_t x_bytes = staged * ((int64_t)slice * 256 + 64);
    const bool enough = tiles * S >= sms || S == 8 || p.blocks < 2 * S * kBatchWarps;   // a cluster also spreads few rows over the SMs
    if (x_bytes > 110 * 1024 || !enough) continue;
    const int64_t fit = resident_clusters(S, (void*)exo_gemv_q4_batch_kernel<Bf16, 1, false, 1>, kBatchThreads, kMostSmem, (unsigned)S, sms, 1);
    for (int64_t clusters = tiles < fit ? tiles : fit;; clusters = 2 * clusters < tiles ? 2 * clusters : tiles) {   // more turns where the sums would not fit
      const int most = (int)((tiles + clusters - 1) / clusters);
      fp.nk_log = 0;
      while (fp.nk_log < 4 && (most << fp.nk_log) < kBatchWarps && (least + kBatchPiece - 1) / kBatchPiece >= 2 << fp.nk_log) ++fp.nk_log;
      const int turns = ((most << fp.nk_log) + kBatchWarps - 1) / kBatchWarps;
      const int pieces = ((slice + kBatchPiece - 1) / kBatchPiece + (1 << fp.nk_log) - 1) >> fp.nk_log;
      fp.stages = turns * pieces < 2 ? turns * pieces : 2;
      int64_t at = 512 + (int64_t)(most << fp.nk_log) * tokens * 64;
      fp.digits_at = (int)at; at += x_bytes;
      at = (at + 127) / 128 * 128;
      fp.ring_at = (int)at;
      at += kBatchWarps * fp.stages * kBatchPiece * 1024;
      if (at <= kMostSmem) {
        *ctas = (unsigned)(clusters * S);
        *cluster = (unsigned)S;
        *smem = (size_t)at;
        fp.g = p;
        return (clusters * groups + fit - 1) / fit * ((int64_t)turns * pieces * (16 + 7 * nt) + 60);
      }
      if (most <= 1) break;
    }
  }
  return 0;
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

template <class T, class WT, int ALIGN> void* quant_dir(bool back) {
  return back ? (void*)exo_q4_dequantize_kernel<T, WT, ALIGN> : (void*)exo_q4_quantize_kernel<T, WT, ALIGN>;
}
template <class T, class WT> void* quant_align(int align, bool back) {
  if (align == 16) return quant_dir<T, WT, 16>(back);
  if (align == 8) return quant_dir<T, WT, 8>(back);
  if constexpr (std::is_same<WT, float>::value) return quant_dir<T, WT, 4>(back);
  else return align == 4 ? quant_dir<T, WT, 4>(back) : quant_dir<T, WT, 2>(back);
}
template <class T> void* quant_fn(int w_dtype, int align, bool back) {
  return w_dtype == EXO_GEMM_FP32 ? quant_align<T, float>(align, back)
         : w_dtype == EXO_GEMM_BF16 ? quant_align<T, Bf16>(align, back) : quant_align<T, Fp16>(align, back);
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
  const uintptr_t at = (uintptr_t)W | (uintptr_t)(ldw * bytes);   // what every row's start is a multiple of
  const int align = at % 16 == 0 ? 16 : at % 8 == 0 ? 8 : at % 4 == 0 ? 4 : 2;
  const int64_t ctas = (p.rows * p.segments + kQuantThreads / 32 - 1) / (kQuantThreads / 32);
  if (ctas >= (1LL << 31)) return EXO_GEMM_ERR_UNSUPPORTED;
  void* fn = q->dtype == EXO_GEMM_BF16 ? quant_fn<Bf16>(w_dtype, align, back) : quant_fn<Fp16>(w_dtype, align, back);
  return launch(fn, (unsigned)ctas, 1, kQuantThreads, 0, 1, (cudaStream_t)cuda_stream, &p);
}

}  // namespace
unsigned take_gave_up_q4(cudaError_t* e) { return take_gave_up(e); }
unsigned take_gave_up_moe(cudaError_t* e);   // moe.cu

static std::atomic<int64_t> wait_hook{0};   // milliseconds * 4 + skip
WaitHook take_wait_hook() {
  const int64_t v = wait_hook.load(std::memory_order_relaxed) ? wait_hook.exchange(0) : 0;
  return WaitHook{(uint64_t)(v / 4 > 0 ? v / 4 : 4000) * 2000000ull, (int)(v % 4)};
}
}  // namespace decode
}  // namespace exo

using namespace exo::decode;

extern "C" exo_gemm_status_t exo_decode_check(void) {
  cudaError_t e = cudaDeviceSynchronize();
  if (e != cudaSuccess) return cuda_failed(e);
  const unsigned n = take_gave_up_q4(&e) | (e == cudaSuccess ? take_gave_up_moe(&e) : 0u);
  if (e != cudaSuccess) return cuda_failed(e);
  return n ? EXO_GEMM_ERR_DEVICE_TIMEOUT : EXO_GEMM_OK;
}

extern "C" exo_gemm_status_t exo_decode_debug_set(int32_t timeout_ms, int32_t skip_copies) {
  if (timeout_ms < 0 || timeout_ms > 10000 || skip_copies < 0 || skip_copies > 2) return EXO_GEMM_ERR_INVALID_ARG;
  wait_hook.store((int64_t)timeout_ms * 4 + skip_copies);
  return EXO_GEMM_OK;
}

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
  if ((read && ((uintptr_t)X & 1u)) || ((uintptr_t)Y & (y_dtype == EXO_GEMM_FP32 ? 3u : 1u))) return EXO_GEMM_ERR_ALIGNMENT;
  int sms = 0;
  if ((st = device_check(&sms)) != EXO_GEMM_OK) return st;
  GemvParams p{};
  p.codes = (const uint8_t*)W->codes; p.scales = (const uint16_t*)W->scales; p.zeros = W->zeros;
  p.x = (const uint16_t*)X; p.y = Y; p.ldx = ldx; p.ldy = ldy; p.rows = W->rows;
  p.K = (int)W->K; p.tokens = (int)tokens; p.blocks = blocks_of(W->K);
  p.y_dtype = y_dtype; p.alpha = alpha; p.beta = beta;
  const uintptr_t x_at = (uintptr_t)X | (uintptr_t)(ldx * 2);
  p.x_align = x_at % 16 == 0 ? 16 : x_at % 8 == 0 ? 8 : x_at % 4 == 0 ? 4 : 2;
  p.x_aligned = p.x_align == 16;
  const bool bf16 = W->dtype == EXO_GEMM_BF16;
  if (!read) {
    const int64_t ctas = (p.rows + kGemvThreads - 1) / kGemvThreads;
    if (ctas >= (1LL << 31)) return EXO_GEMM_ERR_UNSUPPORTED;
    return launch(bf16 ? (void*)exo_gemv_q4_scale_kernel<Bf16> : (void*)exo_gemv_q4_scale_kernel<Fp16>, (unsigned)ctas, 1,
                  kGemvThreads, 0, 1, (cudaStream_t)cuda_stream, &p);
  }
  if (p.rows < (1LL << 31) - 16) {
    FewParams fp{};
    size_t smem = 0;
    unsigned ctas = 0, cluster = 1, groups = 1;
    int nt = 0;
    const bool few = plan_few(fp, p, 128 / W->group, sms, &ctas, &cluster, &smem);
    if (!few) {
      // A CTA's tokens: with more the weights are read and unpacked less often, with fewer its activations and sums leave room for
      // smaller clusters and longer turns.  The estimate is a line through 8, 16 and 24 tokens.  16384 x 8192, us, with 1, 2, 3 and 4
      // tiles of eight to a CTA: 32 tokens 90, 59, 67, 69; 64 tokens 180, 119, 106, 137; 4096 x 4096, 64 tokens 46, 31, 27, 24.
      int64_t best = 0;
      for (int n = 1; n <= 4 && n <= (p.tokens + 7) / 8; ++n) {
        FewParams q{};
        size_t bytes = 0;
        unsigned c = 0, cl = 1;
        const int64_t cost = plan_batch(q, p, sms, n, &c, &cl, &bytes);
        if (cost > 0 && (nt == 0 || cost < best)) { best = cost; nt = n; fp = q; ctas = c; cluster = cl; smem = bytes; }
      }
      if (nt > 0) groups = (unsigned)((p.tokens + 8 * nt - 1) / (8 * nt));
    }
    if (few || nt > 0) {
      const WaitHook hook = take_wait_hook();
      fp.wait = WaitBound{hook.clocks, hook.skip == 1};
      CUtensorMap map;
      if (!exo::encode_steps_map(&map, p.codes, (uint64_t)p.rows, (uint64_t)p.blocks, few ? kFewPiece : kBatchPiece)) return EXO_GEMM_ERR_CUDA;
      FewFn fn = bf16 ? pick_few<Bf16>(W->group, W->zeros, few, nt) : pick_few<Fp16>(W->group, W->zeros, few, nt);
      return launch((void*)fn, ctas, groups, few ? kFewThreads : kBatchThreads, smem, cluster, (cudaStream_t)cuda_stream, &fp, &map);
    }
  }
  // Activations or sums that fit no CTA: the general kernel.  The cluster cuts k until the grid fills the device twice, as long as
  // a warp keeps a step.
  const int64_t tiles = (p.rows + 15) / 16;
  int S = 1;
  while (S < 8 && tiles * S < 2 * sms && p.blocks >= 2 * S * kGemvWarps) S *= 2;
  if (tiles * S >= (1LL << 31)) return EXO_GEMM_ERR_UNSUPPORTED;
  // staged activations: all of the CTA's part of k where that leaves room for two CTAs per SM
  const int mine = (p.blocks + S - 1) / S, staged = p.tokens < 8 ? p.tokens : 8, most = (100 * 1024 / staged - 64) / 256;
  p.chunk = mine < most ? mine : most;
  size_t smem = (size_t)staged * gemv_pitch(p.chunk);
  if (smem < (kGemvWarps + 1) * 512) smem = (kGemvWarps + 1) * 512;
  GemvFn fn = bf16 ? pick_gemv<Bf16>(W->group, W->zeros) : pick_gemv<Fp16>(W->group, W->zeros);
  return launch((void*)fn, (unsigned)(tiles * S), (unsigned)((p.tokens + 7) / 8), kGemvThreads, smem, (unsigned)S, (cudaStream_t)cuda_stream, &p);
}

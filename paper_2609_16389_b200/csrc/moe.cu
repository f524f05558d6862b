// A whole mixture-of-experts layer for a few tokens (exo_decode.h), in three kernels that follow one another by
// programmatic dependent launch:
//
//   route   logits = x * router^T; its last CTA picks each token's experts and lists, for every taken expert, its tokens
//   up      a = w_e * silu(gate_e x) * (up_e x) for every taken expert and its tokens
//   down    y = sum of down_e a over the taken experts
//
// The layer is bound by reading the taken experts' weights once.  All three stream weight rows into mma fragments
// (decode_core.cuh); a fragment's eight columns are the expert's own tokens, gathered.
#include <cooperative_groups.h>

#include <new>

#include "../../include/exo_decode.h"
#include "decode_core.cuh"
#include "decode_host.h"
#include "ptx.cuh"

namespace exo {
namespace decode {

constexpr int kMaxTokens = 64, kMaxExperts = 512, kMaxShared = 8, kMaxTopK = 16;

struct Active { int expert, base, count, pad; };   // a taken expert: its tokens are entries base .. base + count - 1

namespace {

// ---- what the kernels are given --------------------------------------------------------------------------------
struct Stack {              // one stack of expert matrices
  const void* w;
  const uint16_t* scales;
  const uint8_t* zeros;
  int64_t ld, expert_rows;
  int rows, K;              // of one expert
};

struct MoeParams {
  const uint16_t *x, *router;
  int64_t ldx, ldy, ld_router, ldh;
  uint16_t* y;
  int* index;               // may be NULL
  float* weight;            // may be NULL
  Stack gate, up, down;
  int tokens, hidden, inner, experts, shared, top_k;
  bool renormalize, x_aligned;
  float routed_scale;
  // workspace
  unsigned* arrivals;
  int* n_active;
  Active* active;
  int* entry_token;
  float* entry_weight;
  float* logits;            // tokens x experts
  uint16_t* h;              // entries x ldh
};

// Row formats by number: 0 = 16-bit rows anywhere, 1 = 16-bit rows on 16-byte boundaries, 2 + n = 4-bit, 2^n groups in 128.
template <class T, int FMT> struct FormatOf { using type = RowsQ4<T, 1 << (FMT - 2)>; };
template <class T> struct FormatOf<T, 0> { using type = Rows16<T, false>; };
template <class T> struct FormatOf<T, 1> { using type = Rows16<T, true>; };

template <class T, int FMT>
__device__ __forceinline__ typename FormatOf<T, FMT>::type rows_of(const Stack& m0, int64_t row0, const Stack& m1, int64_t row1) {
  typename FormatOf<T, FMT>::type f;
  if constexpr (FMT < 2) {
    f.r0 = static_cast<const uint16_t*>(m0.w) + row0 * m0.ld;
    f.r1 = static_cast<const uint16_t*>(m1.w) + row1 * m1.ld;
  } else {
    constexpr int PER = 1 << (FMT - 2);
    const int64_t blocks = (m0.K + 127) / 128;
    f.c0 = static_cast<const uint8_t*>(m0.w) + row0 * blocks * 64;
    f.c1 = static_cast<const uint8_t*>(m1.w) + row1 * blocks * 64;
    f.s0 = m0.scales + row0 * blocks * PER;
    f.s1 = m1.scales + row1 * blocks * PER;
    f.z0 = m0.zeros ? m0.zeros + row0 * blocks * PER : nullptr;
    f.z1 = m1.zeros ? m1.zeros + row1 * blocks * PER : nullptr;
  }
  return f;
}

template <int NT> __device__ __forceinline__ void clear(float (&acc)[NT][4]) {
#pragma unroll
  for (int i = 0; i < NT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
}
__device__ __forceinline__ void add(float4& v, const float4& w) { v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w; }

// ==== route =======================================================================================================
// 16 experts per cluster; k is cut over the cluster's CTAs and their 16 warps, so that one token's logits are a
// couple of loads per lane.  The last CTA to arrive holds every logit in L2 and does the rest alone: a warp per token.
constexpr int kRouteThreads = 512, kRouteWarps = kRouteThreads / 32;

// Larger for larger logits, never 0; NaN above all.
__device__ __forceinline__ uint32_t key_of(float l) {
  if (isnan(l)) return 0xffffffffu;
  const uint32_t u = __float_as_uint(l + 0.f);   // -0 counts as 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct RouteTables {
  unsigned long long tokens_of[kMaxExperts + kMaxShared];   // bit t: token t takes the expert
  int base[kMaxExperts + kMaxShared];
  int taken[kMaxTokens * kMaxTopK];
  float weight[kMaxTokens * kMaxTopK];
};

__device__ void route_tokens(const MoeParams& p, RouteTables& tb) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int all = p.experts + p.shared;
  for (int e = threadIdx.x; e < all; e += kRouteThreads)
    tb.tokens_of[e] = e < p.experts ? 0ull : ~0ull >> (64 - p.tokens);
  __syncthreads();
  for (int token = warp; token < p.tokens; token += kRouteWarps) {
    const float* l = p.logits + (int64_t)token * p.experts;
    float mine[kMaxExperts / 32];
    uint32_t key[kMaxExperts / 32];
#pragma unroll
    for (int j = 0; j < kMaxExperts / 32; ++j) {
      const int e = 32 * j + lane;
      key[j] = 0;
      if (e < p.experts) { mine[j] = __ldcg(l + e); key[j] = key_of(mine[j]); }
    }
    int my_expert = 0;        // lane r keeps the r-th taken one
    float my_logit = 0.f, top = 0.f;
    for (int r = 0; r < p.top_k; ++r) {
      uint32_t best = 0;
      int at = 0;
      float val = 0.f;
#pragma unroll
      for (int j = 0; j < kMaxExperts / 32; ++j)
        if (32 * j < p.experts && key[j] > best) { best = key[j]; at = 32 * j + lane; val = mine[j]; }
      const uint32_t most = __reduce_max_sync(0xffffffffu, best);
      const int e = (int)__reduce_min_sync(0xffffffffu, best == most ? (uint32_t)at : 0xffffffffu);
      val = __shfl_sync(0xffffffffu, val, e & 31);
      if (r == 0) top = val;
      if (lane == r) { my_expert = e; my_logit = val; }
#pragma unroll
      for (int j = 0; j < kMaxExperts / 32; ++j)
        if (32 * j + lane == e) key[j] = 0;
    }
    float total;
    if (p.renormalize) {
      total = lane < p.top_k ? expf(my_logit - top) : 0.f;
    } else {
      total = 0.f;
#pragma unroll
      for (int j = 0; j < kMaxExperts / 32; ++j)
        if (32 * j + lane < p.experts) total += expf(mine[j] - top);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    if (lane < p.top_k) {
      const float w = expf(my_logit - top) / total * p.routed_scale;
      const int at = token * p.top_k + lane;
      tb.taken[at] = my_expert;
      tb.weight[at] = w;
      atomicOr(&tb.tokens_of[my_expert], 1ull << token);
      if (p.index) p.index[at] = my_expert;
      if (p.weight) p.weight[at] = w;
    }
  }
  __syncthreads();
  if (warp == 0) {   // the taken experts in order, and where each one's tokens begin
    int base = 0, n = 0;
    for (int e0 = 0; e0 < all; e0 += 32) {
      const int e = e0 + lane;
      const int count = e < all ? __popcll(tb.tokens_of[e]) : 0;
      int sum = count;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += v;
      }
      const unsigned some = __ballot_sync(0xffffffffu, count > 0);
      if (count > 0) {
        tb.base[e] = base + sum - count;
        p.active[n + __popc(some & ((1u << lane) - 1u))] = Active{e, base + sum - count, count, 0};
      }
      base += __shfl_sync(0xffffffffu, sum, 31);
      n += __popc(some);
    }
    if (lane == 0) *p.n_active = n;
  }
  __syncthreads();
  const int per = p.top_k + p.shared;
  for (int i = threadIdx.x; i < p.tokens * per; i += kRouteThreads) {
    const int token = i / per, slot = i - token * per;
    const int e = slot < p.top_k ? tb.taken[token * p.top_k + slot] : p.experts + slot - p.top_k;
    const int at = tb.base[e] + __popcll(tb.tokens_of[e] & ((1ull << token) - 1ull));
    p.entry_token[at] = token;
    p.entry_weight[at] = slot < p.top_k ? tb.weight[token * p.top_k + slot] : 1.f;
  }
}

template <class T, bool VEC, int NT>
__global__ void __launch_bounds__(kRouteThreads) exo_moe_route_kernel(const MoeParams p) {
  namespace cg = cooperative_groups;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ RouteTables tables;
  __shared__ bool last;
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), r = (int)cluster.block_rank();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int e0 = (int)(blockIdx.x / S) * 16;
  const int nt = (p.tokens + 7) / 8;
  Rows16<T, VEC> f;
  f.r0 = p.router + (int64_t)min(e0 + g, p.experts - 1) * p.ld_router;
  f.r1 = p.router + (int64_t)min(e0 + g + 8, p.experts - 1) * p.ld_router;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  float acc[NT][4];
  clear(acc);
  const int steps = (p.hidden + 31) / 32, ds = S * kRouteWarps, s = r * kRouteWarps + warp;
  Stream<Rows16<T, VEC>, 2> stream;
  stream.preload(f, s, ds, steps, p.hidden, t);
  stream.template walk<NT>(f, s, ds, steps, p.hidden, t, [&](int i, int k) {
    const int token = 8 * i + g;
    return token < p.tokens ? load8_checked(p.x + token * p.ldx, k, p.hidden, p.x_aligned) : make_uint4(0, 0, 0, 0);
  }, nt, acc);
  float4* red = reinterpret_cast<float4*>(smem);   // [warp][nt][lane]
  float4* part = red + kRouteWarps * nt * 32;
#pragma unroll
  for (int i = 0; i < NT; ++i)
    if (i < nt) red[(warp * nt + i) * 32 + lane] = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
  __syncthreads();
  const int items = nt * 32;
  for (int idx = threadIdx.x; idx < items; idx += kRouteThreads) {
    float4 v = red[idx];
    for (int q = 1; q < kRouteWarps; ++q) add(v, red[q * items + idx]);
    part[idx] = v;
  }
  cluster.sync();
  for (int idx = r * kRouteThreads + threadIdx.x; idx < items; idx += S * kRouteThreads) {
    float4 v = cluster.map_shared_rank(part, 0)[idx];
    for (int q = 1; q < S; ++q) add(v, cluster.map_shared_rank(part, q)[idx]);
    const int token = 8 * (idx >> 5) + 2 * (idx & 3), e = e0 + ((idx & 31) >> 2);
    const float vals[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int tk = token + (q & 1), ex = e + 8 * (q >> 1);
      if (tk < p.tokens && ex < p.experts) __stcg(p.logits + (int64_t)tk * p.experts + ex, vals[q]);
    }
  }
  __threadfence();
  cluster.sync();   // also: no CTA leaves while another may still read its sums
  if (threadIdx.x == 0) {
    const unsigned n = atomicAdd(p.arrivals, 1u);
    last = n + 1 == gridDim.x;
    if (last) { *p.arrivals = 0; __threadfence(); }
  }
  __syncthreads();
  if (last) route_tokens(p, tables);
}

// ==== up ==========================================================================================================
// A CTA computes 8 inner values of one taken expert for its tokens: the 16 rows of a fragment are eight rows of gate and
// the same eight of up, so that a lane ends with both factors of an activation.  Eight warps cut `hidden`.
constexpr int kUpThreads = 256, kUpWarps = 8;

template <class T, int FMT, int NT>
__global__ void __launch_bounds__(kUpThreads) exo_moe_up_kernel(const MoeParams p) {
  __shared__ float4 red[kUpWarps * NT * 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();   // after the wait: `down` may then read the tables of `route` before it waits itself
  if ((int)blockIdx.y >= __ldcg(p.n_active)) return;
  const int4 raw = __ldcg(reinterpret_cast<const int4*>(p.active + blockIdx.y));
  const Active a{raw.x, raw.y, raw.z, raw.w};
  const int f0 = blockIdx.x * 8, nt = (a.count + 7) / 8;
  const int64_t row = min(f0 + g, p.inner - 1);
  using F = typename FormatOf<T, FMT>::type;
  const F f = rows_of<T, FMT>(p.gate, a.expert * p.gate.expert_rows + row, p.up, a.expert * p.up.expert_rows + row);
  const int steps = (p.hidden + F::kStep - 1) / F::kStep;
  constexpr int DEPTH = NT <= 2 ? 4 : 2;
  Stream<F, DEPTH> stream;
  stream.preload(f, warp, kUpWarps, steps, p.hidden, t);
  const uint16_t* xrow[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
    xrow[i] = 8 * i + g < a.count ? p.x + (int64_t)__ldcg(p.entry_token + a.base + 8 * i + g) * p.ldx : nullptr;
  float acc[NT][4];
  clear(acc);
  stream.template walk<NT>(f, warp, kUpWarps, steps, p.hidden, t, [&](int i, int k) {
    return xrow[i] ? load8_checked(xrow[i], k, p.hidden, p.x_aligned) : make_uint4(0, 0, 0, 0);
  }, nt, acc);
#pragma unroll
  for (int i = 0; i < NT; ++i)
    if (i < nt) red[(warp * nt + i) * 32 + lane] = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
  __syncthreads();
  for (int idx = threadIdx.x; idx < nt * 32; idx += kUpThreads) {
    float4 v = red[idx];
    for (int q = 1; q < kUpWarps; ++q) add(v, red[q * nt * 32 + idx]);
    const int n = 8 * (idx >> 5) + 2 * (idx & 3), col = f0 + ((idx & 31) >> 2);
    if (col < p.inner) {
      const float gate[2] = {v.x, v.y}, up[2] = {v.z, v.w};
#pragma unroll
      for (int q = 0; q < 2; ++q)
        if (n + q < a.count) {
          const float w = __ldcg(p.entry_weight + a.base + n + q);
          p.h[(int64_t)(a.base + n + q) * p.ldh + col] = T::from_float(w * (gate[q] / (1.f + expf(-gate[q])) * up[q]));
        }
    }
  }
}

// ==== down ========================================================================================================
// A cluster computes 16 rows of y for all tokens.  Its warps share the steps of all taken experts, one after another,
// in equal ranges; a warp adds what an expert gives onto its own sums in shared memory, by token.  The sums meet
// in warp order and then in rank order.
constexpr int kDownThreads = 256, kDownWarps = 8;

template <class T, int FMT, int NT>
__global__ void __launch_bounds__(kDownThreads) exo_moe_down_kernel(const MoeParams p) {
  namespace cg = cooperative_groups;
  extern __shared__ __align__(128) uint8_t smem[];
  float* sums = reinterpret_cast<float*>(smem);               // [warp][token][row]
  float* part = sums + kDownWarps * p.tokens * 16;            // [token][row]
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), r = (int)cluster.block_rank();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int row0 = (int)(blockIdx.x / S) * 16;
  using F = typename FormatOf<T, FMT>::type;
  const int steps = (p.inner + F::kStep - 1) / F::kStep;
  // `route` is complete: `up` started this kernel after it had waited for that
  const int64_t total = (int64_t)__ldcg(p.n_active) * steps;
  const int64_t workers = (int64_t)S * kDownWarps, q = r * kDownWarps + warp;
  int64_t pos = total * q / workers;
  const int64_t end = total * (q + 1) / workers;
  for (int i = threadIdx.x; i < kDownWarps * p.tokens * 16; i += kDownThreads) sums[i] = 0.f;
  __syncthreads();
  float* mine = sums + warp * p.tokens * 16;
  constexpr int DEPTH = NT <= 2 ? 4 : 2;
  Stream<F, DEPTH> stream;
  bool waited = false;
  while (pos < end) {
    const int at = (int)(pos / steps), s0 = (int)(pos - (int64_t)at * steps);
    const int s1 = (int)min((int64_t)steps, s0 + (end - pos));
    const int4 raw = __ldcg(reinterpret_cast<const int4*>(p.active + at));
    const Active a{raw.x, raw.y, raw.z, raw.w};
    const int nt = (a.count + 7) / 8;
    const int64_t first = a.expert * p.down.expert_rows;
    const F f = rows_of<T, FMT>(p.down, first + min(row0 + g, p.hidden - 1), p.down, first + min(row0 + g + 8, p.hidden - 1));
    stream.preload(f, s0, 1, s1, p.inner, t);
    int token[NT][2];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int c = 0; c < 2; ++c)
        token[i][c] = 8 * i + 2 * t + c < a.count ? __ldcg(p.entry_token + a.base + 8 * i + 2 * t + c) : -1;
    if (!waited) { ptx::grid_dependency_wait(); waited = true; }   // `up` is complete
    const uint16_t* hrow = p.h + (int64_t)(a.base + g) * p.ldh;
    float acc[NT][4];
    clear(acc);
    stream.template walk<NT>(f, s0, 1, s1, p.inner, t, [&](int i, int k) {
      if (8 * i + g >= a.count) return make_uint4(0, 0, 0, 0);
      const uint16_t* hk = hrow + (int64_t)8 * i * p.ldh;
      return k + 8 <= p.inner ? __ldcg(reinterpret_cast<const uint4*>(hk + k)) : load8_checked(hk, k, p.inner, false);
    }, nt, acc);
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (token[i][c] >= 0) {
          mine[token[i][c] * 16 + g] += acc[i][c];
          mine[token[i][c] * 16 + g + 8] += acc[i][2 + c];
        }
    __syncwarp();
    pos += s1 - s0;
  }
  if (!waited) ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  __syncthreads();
  auto finish = [&](int idx, float v) {
    const int row = row0 + (idx & 15);
    if (row < p.hidden) p.y[(int64_t)(idx >> 4) * p.ldy + row] = T::from_float(v);
  };
  for (int idx = threadIdx.x; idx < p.tokens * 16; idx += kDownThreads) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kDownWarps; ++w) v += sums[w * p.tokens * 16 + idx];
    if (S == 1) finish(idx, v);
    else part[idx] = v;
  }
  if (S > 1) {
    cluster.sync();
    for (int idx = r * kDownThreads + threadIdx.x; idx < p.tokens * 16; idx += S * kDownThreads) {
      float v = 0.f;
      for (int o = 0; o < S; ++o) v += cluster.map_shared_rank(part, o)[idx];
      finish(idx, v);
    }
    cluster.sync();
  }
}

// ---- kernels by type, format and token count --------------------------------------------------------------------
template <class T, bool VEC> void* pick_route(int nt) {
  return nt == 1 ? (void*)exo_moe_route_kernel<T, VEC, 1> : nt == 2 ? (void*)exo_moe_route_kernel<T, VEC, 2> : (void*)exo_moe_route_kernel<T, VEC, 8>;
}
template <class T, int FMT> void* pick_up_nt(int nt) {
  return nt == 1 ? (void*)exo_moe_up_kernel<T, FMT, 1> : nt == 2 ? (void*)exo_moe_up_kernel<T, FMT, 2> : (void*)exo_moe_up_kernel<T, FMT, 8>;
}
template <class T, int FMT> void* pick_down_nt(int nt) {
  return nt == 1 ? (void*)exo_moe_down_kernel<T, FMT, 1> : nt == 2 ? (void*)exo_moe_down_kernel<T, FMT, 2> : (void*)exo_moe_down_kernel<T, FMT, 8>;
}
template <class T> void* pick_up(int fmt, int nt) {
  switch (fmt) {
    case 0: return pick_up_nt<T, 0>(nt);
    case 1: return pick_up_nt<T, 1>(nt);
    case 2: return pick_up_nt<T, 2>(nt);
    case 3: return pick_up_nt<T, 3>(nt);
    default: return pick_up_nt<T, 4>(nt);
  }
}
template <class T> void* pick_down(int fmt, int nt) {
  switch (fmt) {
    case 0: return pick_down_nt<T, 0>(nt);
    case 1: return pick_down_nt<T, 1>(nt);
    case 2: return pick_down_nt<T, 2>(nt);
    case 3: return pick_down_nt<T, 3>(nt);
    default: return pick_down_nt<T, 4>(nt);
  }
}

bool rows_aligned(const void* w, int64_t ld) { return ((uintptr_t)w & 15u) == 0 && ld % 8 == 0; }

exo_gemm_status_t check_stack(const exo_moe_matrix_t& m, int64_t rows, int64_t K, int q4_group) {
  if (!m.w) return EXO_GEMM_ERR_NULL;
  if (m.expert_rows < rows || m.expert_rows > (1LL << 32)) return EXO_GEMM_ERR_INVALID_ARG;
  if (q4_group) {
    if (!m.scales) return EXO_GEMM_ERR_NULL;
    if (!q4_aligned(m.w, m.scales, m.zeros, q4_group)) return EXO_GEMM_ERR_ALIGNMENT;
  } else {
    if (m.scales || m.zeros || m.ld < K) return EXO_GEMM_ERR_INVALID_ARG;
    if ((uintptr_t)m.w & 1u) return EXO_GEMM_ERR_ALIGNMENT;
  }
  return EXO_GEMM_OK;
}

Stack stack_of(const exo_moe_matrix_t& m, int64_t rows, int64_t K) {
  return Stack{m.w, (const uint16_t*)m.scales, m.zeros, m.ld, m.expert_rows, (int)rows, (int)K};
}

struct DeviceGuard {
  int prev = -1;
  bool switched = false;
  cudaError_t err;
  explicit DeviceGuard(int dev) {
    err = cudaGetDevice(&prev);
    if (err == cudaSuccess && dev >= 0 && dev != prev) {
      err = cudaSetDevice(dev);
      switched = err == cudaSuccess;
    }
  }
  ~DeviceGuard() {
    if (switched) cudaSetDevice(prev);
  }
};

}  // namespace
}  // namespace decode
}  // namespace exo

using namespace exo::decode;

struct exo_moe_plan {
  exo_moe_desc_t desc;
  int device, sms;
  int64_t ldh, bytes;
  uint8_t* ws;
  int64_t at_active, at_token, at_weight, at_logits, at_h;   // offsets into ws; the arrival counter and n_active come first
};

extern "C" {

exo_gemm_status_t exo_moe_validate(const exo_moe_desc_t* d) {
  if (!d) return EXO_GEMM_ERR_NULL;
  if (d->hidden < 1 || d->inner < 1 || d->hidden > (1 << 24) || d->inner > (1 << 24)) return EXO_GEMM_ERR_INVALID_ARG;
  if (d->experts < 1 || d->shared < 0 || d->top_k < 1 || d->top_k > d->experts || d->max_tokens < 1) return EXO_GEMM_ERR_INVALID_ARG;
  if (d->dtype != EXO_GEMM_BF16 && d->dtype != EXO_GEMM_FP16) return EXO_GEMM_ERR_INVALID_ARG;
  if (d->q4_group != 0 && d->q4_group != 32 && d->q4_group != 64 && d->q4_group != 128) return EXO_GEMM_ERR_INVALID_ARG;
  if ((d->renormalize != 0 && d->renormalize != 1) || d->device < -1) return EXO_GEMM_ERR_INVALID_ARG;
  if (d->experts > kMaxExperts || d->shared > kMaxShared || d->top_k > kMaxTopK || d->max_tokens > kMaxTokens) return EXO_GEMM_ERR_UNSUPPORTED;
  return EXO_GEMM_OK;
}

exo_gemm_status_t exo_moe_create(exo_moe_handle_t* out, const exo_moe_desc_t* d) {
  if (!out) return EXO_GEMM_ERR_NULL;
  exo_gemm_status_t st = exo_moe_validate(d);
  if (st != EXO_GEMM_OK) return st;
  DeviceGuard guard(d->device);
  if (guard.err != cudaSuccess) return cuda_failed(guard.err);
  int sms = 0;
  if ((st = device_check(&sms)) != EXO_GEMM_OK) return st;
  exo_moe_plan* plan = new (std::nothrow) exo_moe_plan();
  if (!plan) return EXO_GEMM_ERR_CUDA;
  plan->desc = *d;
  plan->device = d->device >= 0 ? d->device : guard.prev;
  plan->sms = sms;
  plan->ldh = (d->inner + 127) / 128 * 128;
  const int64_t entries = (int64_t)d->max_tokens * (d->top_k + d->shared);
  int64_t at = 256;
  auto take = [&at](int64_t bytes) { const int64_t here = at; at += (bytes + 255) / 256 * 256; return here; };
  plan->at_active = take((int64_t)(d->experts + d->shared) * (int64_t)sizeof(Active));
  plan->at_token = take(entries * 4);
  plan->at_weight = take(entries * 4);
  plan->at_logits = take((int64_t)d->max_tokens * d->experts * 4);
  plan->at_h = take(entries * plan->ldh * 2);
  plan->bytes = at;
  cudaError_t e = cudaMalloc((void**)&plan->ws, (size_t)plan->bytes);
  if (e == cudaSuccess) {
    e = cudaMemset(plan->ws, 0, 256);
    if (e != cudaSuccess) cudaFree(plan->ws);
  }
  if (e != cudaSuccess) {
    delete plan;
    return cuda_failed(e);
  }
  *out = plan;
  return EXO_GEMM_OK;
}

exo_gemm_status_t exo_moe_run(exo_moe_handle_t plan, const exo_moe_weights_t* w, int64_t tokens, const void* x, int64_t ldx,
                              void* y, int64_t ldy, int32_t* index, float* weight, void* cuda_stream) {
  if (!plan || !w) return EXO_GEMM_ERR_NULL;
  const exo_moe_desc_t& d = plan->desc;
  if (tokens < 0 || tokens > d.max_tokens || ldx < d.hidden || ldy < d.hidden || w->ld_router < d.hidden) return EXO_GEMM_ERR_INVALID_ARG;
  if (tokens == 0) return EXO_GEMM_OK;
  if (!x || !y || !w->router) return EXO_GEMM_ERR_NULL;
  const bool q4 = d.q4_group != 0;
  exo_gemm_status_t st;
  if ((st = check_stack(w->gate, d.inner, d.hidden, d.q4_group)) != EXO_GEMM_OK) return st;
  if ((st = check_stack(w->up, d.inner, d.hidden, d.q4_group)) != EXO_GEMM_OK) return st;
  if ((st = check_stack(w->down, d.hidden, d.inner, d.q4_group)) != EXO_GEMM_OK) return st;
  if ((((uintptr_t)x | (uintptr_t)y | (uintptr_t)w->router) & 1u) || (((uintptr_t)index | (uintptr_t)weight) & 3u)) return EXO_GEMM_ERR_ALIGNMENT;
  DeviceGuard guard(plan->device);
  if (guard.err != cudaSuccess) return cuda_failed(guard.err);

  MoeParams p{};
  p.x = (const uint16_t*)x; p.router = (const uint16_t*)w->router; p.y = (uint16_t*)y;
  p.ldx = ldx; p.ldy = ldy; p.ld_router = w->ld_router; p.ldh = plan->ldh;
  p.index = index; p.weight = weight;
  p.gate = stack_of(w->gate, d.inner, d.hidden);
  p.up = stack_of(w->up, d.inner, d.hidden);
  p.down = stack_of(w->down, d.hidden, d.inner);
  p.tokens = (int)tokens; p.hidden = (int)d.hidden; p.inner = (int)d.inner;
  p.experts = d.experts; p.shared = d.shared; p.top_k = d.top_k;
  p.renormalize = d.renormalize != 0; p.routed_scale = d.routed_scale;
  p.x_aligned = rows_aligned(x, ldx);
  p.arrivals = (unsigned*)plan->ws;
  p.n_active = (int*)(plan->ws + 128);
  p.active = (Active*)(plan->ws + plan->at_active);
  p.entry_token = (int*)(plan->ws + plan->at_token);
  p.entry_weight = (float*)(plan->ws + plan->at_weight);
  p.logits = (float*)(plan->ws + plan->at_logits);
  p.h = (uint16_t*)(plan->ws + plan->at_h);

  const bool bf16 = d.dtype == EXO_GEMM_BF16;
  const int nt = (p.tokens + 7) / 8;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;

  // route: 16 experts per cluster; a warp keeps a step of 32
  int S = 1;
  const int steps = (p.hidden + 31) / 32;
  while (S < 8 && steps >= 2 * S * kRouteWarps) S *= 2;
  const bool router_aligned = rows_aligned(w->router, w->ld_router);
  void* fn = bf16 ? (router_aligned ? pick_route<Bf16, true>(nt) : pick_route<Bf16, false>(nt))
                  : (router_aligned ? pick_route<Fp16, true>(nt) : pick_route<Fp16, false>(nt));
  st = launch(fn, (unsigned)((p.experts + 15) / 16 * S), 1, kRouteThreads, (size_t)(kRouteWarps + 1) * nt * 512, (unsigned)S, stream, &p);
  if (st != EXO_GEMM_OK) return st;

  const int q4_fmt = d.q4_group == 128 ? 2 : d.q4_group == 64 ? 3 : 4;
  const int64_t most = (int64_t)p.tokens * p.top_k < p.experts ? (int64_t)p.tokens * p.top_k : p.experts;
  const int taken = (int)most + p.shared;   // the most experts this run can take
  const int up_fmt = q4 ? q4_fmt : rows_aligned(w->gate.w, w->gate.ld) && rows_aligned(w->up.w, w->up.ld) ? 1 : 0;
  st = launch(bf16 ? pick_up<Bf16>(up_fmt, nt) : pick_up<Fp16>(up_fmt, nt), (unsigned)((p.inner + 7) / 8), (unsigned)taken, kUpThreads,
              0, 1, stream, &p);
  if (st != EXO_GEMM_OK) return st;

  // down: cut until the grid fills the device four times, as long as a warp keeps two steps
  const int down_fmt = q4 ? q4_fmt : rows_aligned(w->down.w, w->down.ld) ? 1 : 0;
  const int64_t tiles = (p.hidden + 15) / 16, all_steps = (int64_t)taken * ((p.inner + (q4 ? 127 : 31)) / (q4 ? 128 : 32));
  S = 1;
  while (S < 8 && tiles * S < 4 * plan->sms && all_steps >= 4 * S * kDownWarps) S *= 2;
  return launch(bf16 ? pick_down<Bf16>(down_fmt, nt) : pick_down<Fp16>(down_fmt, nt), (unsigned)(tiles * S), 1, kDownThreads,
                (size_t)(kDownWarps + 1) * p.tokens * 64, (unsigned)S, stream, &p);
}

int64_t exo_moe_workspace_bytes(exo_moe_handle_t plan) { return plan ? plan->bytes : 0; }

exo_gemm_status_t exo_moe_destroy(exo_moe_handle_t plan) {
  if (!plan) return EXO_GEMM_OK;
  DeviceGuard guard(plan->device);
  const cudaError_t e = cudaFree(plan->ws);
  delete plan;
  return e == cudaSuccess ? EXO_GEMM_OK : cuda_failed(e);
}

}  // extern "C"

// A whole mixture-of-experts layer for a few tokens (exo_decode.h): a routing kernel and two kernels for the experts, that follow
// one another by programmatic dependent launch:
//
//   route   logits = x * router^T; each token's experts, and for every taken expert its tokens
//   up      a = w_e * silu(gate_e x) * (up_e x) for every taken expert and its tokens
//   down    y = sum of down_e a over the taken experts
//
// The layer is bound by reading the taken experts' weights once.  A fragment (decode_core.cuh) is 16 weight rows by eight of the
// expert's own tokens.  Measured on a B200 (CUDA graph of passes, three sets of inputs in turn): 8 of 64 experts of 2048 x 1024 in
// bf16, one token, 29.5 us for 101 MB (15.4 at the copy bandwidth): 5.4 are routing, and `up` and `down` each have a start of 2 to 4 us and an end
// of 1 to 2 in which memory is idle (alone, `up` draws 44 % of the nominal bandwidth and `down` 27 %); 64 tokens, 6 of 64 and a shared one of
// 4096 x 1536, 538 us for 2.45 GB (374).  4-bit experts are held up by their unpacking (2 of 8 of 4096 x 8192, one token, 51 us; 15.9), from 17
// tokens on by their activations from L2 too (24 tokens 309 us, 64 tokens 729; 63).
#include <cooperative_groups.h>

#include <new>

#include "../../include/exo_decode.h"
#include "decode_core.cuh"
#include "decode_host.h"
#include "ptx.cuh"

namespace exo {
namespace decode {

constexpr int kHalvesTokens = 4;   // the inner activations of an expert of up to this many tokens are kept in two 16-bit parts
constexpr int kMaxTokens = 64, kMaxExperts = 512, kMaxShared = 8, kMaxTopK = 16;

struct Active { int expert, base, count, cost_before; };   // a taken expert: its tokens are entries base .. base + count - 1

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
  int taken;                // the most experts this run can take
  bool renormalize, x_aligned;
  float routed_scale;
  // workspace
  unsigned* arrivals;
  int* n_active;
  Active* active;
  int* entry_token;
  float* entry_weight;
  float* logits;            // tokens x experts
  uint16_t* h;              // inner activations, two rows of ldh for every entry (halves_of)
  const uint16_t* xs;       // x itself, or (copy_x) route's copy in rows of ldxs elements, a multiple of 128, filled with zeros
  int64_t ldxs;
  bool copy_x;
  int up_piece, down_piece;
  WaitBound up_wait, down_wait;
};

// Weight formats by number: 0 = 16-bit rows anywhere, 1 = 16-bit rows on 16-byte boundaries, 2 + n = 4-bit, 2^n groups in 128.

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

template <int EPL>   // experts per lane
__device__ __forceinline__ void route_tokens(const MoeParams& p, const float* logits, RouteTables& tb) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int all = p.experts + p.shared;
  for (int e = threadIdx.x; e < all; e += kRouteThreads)
    tb.tokens_of[e] = e < p.experts ? 0ull : ~0ull >> (64 - p.tokens);
  __syncthreads();
  for (int token = warp; token < p.tokens; token += kRouteWarps) {
    const float* l = logits + (int64_t)token * p.experts;
    float mine[EPL];
    uint32_t key[EPL];
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
      const int e = 32 * j + lane;
      key[j] = 0;
      if (e < p.experts) { mine[j] = l[e]; key[j] = key_of(mine[j]); }
    }
    int my_expert = 0;        // lane r keeps the r-th taken one
    float my_logit = 0.f, top = 0.f;
    for (int r = 0; r < p.top_k; ++r) {
      uint32_t best = 0;
      int at = 0;
      float val = 0.f;
#pragma unroll
      for (int j = 0; j < EPL; ++j)
        if (32 * j < p.experts && key[j] > best) { best = key[j]; at = 32 * j + lane; val = mine[j]; }
      const uint32_t most = __reduce_max_sync(0xffffffffu, best);
      const int e = (int)__reduce_min_sync(0xffffffffu, best == most ? (uint32_t)at : 0xffffffffu);
      val = __shfl_sync(0xffffffffu, val, e & 31);
      if (r == 0) top = val;
      if (lane == r) { my_expert = e; my_logit = val; }
#pragma unroll
      for (int j = 0; j < EPL; ++j)
        if (32 * j + lane == e) key[j] = 0;
    }
    float total;
    if (p.renormalize) {
      total = lane < p.top_k ? expf(my_logit - top) : 0.f;
    } else {
      total = 0.f;
#pragma unroll
      for (int j = 0; j < EPL; ++j)
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

__device__ __forceinline__ void route_all(const MoeParams& p, const float* logits, RouteTables& tb) {
  if (p.experts <= 64) route_tokens<2>(p, logits, tb);
  else if (p.experts <= 128) route_tokens<4>(p, logits, tb);
  else route_tokens<16>(p, logits, tb);
}

// x in rows that start on 16-byte boundaries and end in zeros, for `up`
__device__ __forceinline__ void copy_rows(const MoeParams& p) {
  const int per = (int)(p.ldxs / 8);
  for (int i = blockIdx.x * kRouteThreads + threadIdx.x; i < p.tokens * per; i += gridDim.x * kRouteThreads) {
    const int token = i / per, e = i - token * per;
    *reinterpret_cast<uint4*>(const_cast<uint16_t*>(p.xs) + token * p.ldxs + 8 * e) = load8_checked(p.x + token * p.ldx, 8 * e, p.hidden, p.x_aligned);
  }
}

// The same for up to 8 tokens and 128 experts as one cluster of eight CTAs: a CTA has up to 16 of the experts, its warps cut k, and
// the logits go straight into the first CTA's shared memory.  No memory fence, counter or second reading.
// The layer with it and with the general form (us): 64 experts of 2048 x 1024, one token 30.1 / 31.2, 4 tokens 68.1 / 69.0; 60 of
// 1416 x 1000, 6 tokens 44.7 / 46.4; 64 of 4096 x 1536, 4 tokens 142.4 / 143.0, 8 tokens 233 / 231.
constexpr int kOneCtas = 8, kOneTokens = 8, kOneExperts = 16 * kOneCtas;

template <class T, bool VEC>
__global__ void __launch_bounds__(kRouteThreads) exo_moe_route_one_kernel(const MoeParams p) {
  namespace cg = cooperative_groups;
  __shared__ float4 red[kRouteWarps * 32];
  __shared__ float logits[kOneTokens * kOneExperts];     // [token][expert], of the first CTA
  __shared__ RouteTables tables;
  cg::cluster_group cluster = cg::this_cluster();
  const int r = (int)cluster.block_rank(), lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int e0 = p.experts * r / kOneCtas, mine = p.experts * (r + 1) / kOneCtas - e0;
  const uint16_t* r0 = p.router + (int64_t)min(e0 + min(g, mine - 1), p.experts - 1) * p.ld_router;
  const uint16_t* r1 = p.router + (int64_t)min(e0 + min(g + 8, mine - 1), p.experts - 1) * p.ld_router;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  if (mine > 0) {
    if (mine <= 8) r1 = r0;
    const uint16_t* x = p.x + (int64_t)min(g, p.tokens - 1) * p.ldx;
    float acc[1][4];
    clear(acc);
    const int steps = (p.hidden + 31) / 32;
    constexpr int N = 4;           // steps whose loads are in flight together
    for (int s0 = warp; s0 < steps; s0 += N * kRouteWarps) {
      uint4 wa[N], wb[N], b[N];
#pragma unroll
      for (int u = 0; u < N; ++u) {
        const int k = (s0 + u * kRouteWarps) * 32 + 8 * t;
        if (VEC && p.x_aligned && k + 8 <= p.hidden) {
          wa[u] = ldg_weights(r0 + k);
          wb[u] = ldg_weights(r1 + k);
          b[u] = *reinterpret_cast<const uint4*>(x + k);
        } else {
          wa[u] = load8_checked(r0, k, p.hidden, VEC);
          wb[u] = load8_checked(r1, k, p.hidden, VEC);
          b[u] = load8_checked(x, k, p.hidden, p.x_aligned);
        }
      }
#pragma unroll
      for (int u = 0; u < N; ++u) {
        T::mma(acc[0], wa[u].x, wb[u].x, wa[u].y, wb[u].y, b[u].x, b[u].y);
        T::mma(acc[0], wa[u].z, wb[u].z, wa[u].w, wb[u].w, b[u].z, b[u].w);
      }
    }
    red[warp * 32 + lane] = make_float4(acc[0][0], acc[0][1], acc[0][2], acc[0][3]);
  }
  if (p.copy_x) copy_rows(p);
  cluster.sync();      // this CTA's sums are there, and the first CTA runs
  if (warp == 0 && mine > 0) {
    float4 v = red[lane];
#pragma unroll
    for (int q = 1; q < kRouteWarps; ++q) add(v, red[q * 32 + lane]);
    float* to = cluster.map_shared_rank(logits, 0);
    const float vals[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int token = 2 * t + (q & 1), e = g + 8 * (q >> 1);
      if (token < p.tokens && e < mine) to[token * p.experts + e0 + e] = vals[q];
    }
  }
  cluster.sync();
  if (r == 0) route_all(p, logits, tables);
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
  const uint16_t* r0 = p.router + (int64_t)min(e0 + g, p.experts - 1) * p.ld_router;
  const uint16_t* r1 = p.router + (int64_t)min(e0 + g + 8, p.experts - 1) * p.ld_router;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  if (p.copy_x) copy_rows(p);
  float acc[NT][4];
  clear(acc);
  const int steps = (p.hidden + 31) / 32, ds = S * kRouteWarps;
  for (int s = r * kRouteWarps + warp; s < steps; s += ds) {
    const int k = s * 32 + 8 * t;
    const uint4 wa = load8_checked(r0, k, p.hidden, VEC), wb = load8_checked(r1, k, p.hidden, VEC);
#pragma unroll
    for (int i = 0; i < NT; ++i)
      if (i < nt) {
        const uint4 b = load8_checked(p.x + (int64_t)min(8 * i + g, p.tokens - 1) * p.ldx, k, p.hidden, p.x_aligned);
        T::mma(acc[i], wa.x, wb.x, wa.y, wb.y, b.x, b.y);
        T::mma(acc[i], wa.z, wb.z, wa.w, wb.w, b.z, b.w);
      }
  }
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
  if (!last) return;
  route_all(p, p.logits, tables);
}

// Rows of h: an expert's begin at twice its first entry, and hold an entry each, or (1) its two parts.
__device__ __forceinline__ int halves_of(int count) { return count <= kHalvesTokens ? 1 : 0; }

// Inner activations from lane l's part of tile i: gate in x, y and up in z, w for two tokens.  Rounding them to 16 bits would cost
// as much accuracy as rounding y does.  Where an expert has up to four tokens, the columns of their fragment have room for the rounding's
// remainder too, as a token of its own, and `down` adds both; with more tokens one 16-bit value is kept, as for any 16-bit matrix product.
// (Two parts for every expert of up to 8 or 32 tokens take further tiles of `down`: 64 tokens of 64 experts of 4096 x 1536, 539 us,
// 567 and 583.)
template <class T>
__device__ __forceinline__ void store_inner(const MoeParams& p, const float* weight, const Active& a, int f0, int i, int l, const float4& sums) {
  const int n = 8 * i + 2 * (l & 3), col = f0 + (l >> 2);
  if (col >= p.inner) return;
  const float gate[2] = {sums.x, sums.y}, up[2] = {sums.z, sums.w};
  const int halves = halves_of(a.count);
#pragma unroll 1   // the code of eight tiles twice over costs the 4-bit kernel registers (64 tokens of 8 experts of 4096 x 8192: 770 us, 733 so)
  for (int q = 0; q < 2; ++q)
    if (n + q < a.count) {
      const float gq = q ? gate[1] : gate[0], uq = q ? up[1] : up[0], v = weight[a.base + n + q] * (gq / (1.f + expf(-gq)) * uq);
      uint16_t* to = p.h + (2 * (int64_t)a.base + ((n + q) << halves)) * p.ldh + col;
      if (halves && fabsf(v) <= 3.4028235e38f) {   // beyond the type's range the first part is its largest value, the second the rest
        const uint16_t hi = T::from_float(fminf(fmaxf(v, -T::max_finite()), T::max_finite()));
        to[0] = hi;
        to[p.ldh] = T::from_float(v - T::to_float(hi));
      } else {
        to[0] = T::from_float(v);
        if (halves) to[p.ldh] = 0;
      }
    }
}

// ==== the taken experts' weights ====================================================================================
// A warp's own ring of pieces: `piece` steps (64 bytes of a row each, an odd number of them, so that the rows of a fragment
// lie in different banks) of 16 rows, brought by tiled copies that the warp issues itself and waits for itself.
constexpr int kMoeWarps = 8, kMoeThreads = 32 * kMoeWarps, kMoeStages = 2, kMostPiece = 7;
constexpr int kPairSmem = 110 * 1024;   // dynamic shared memory with which two CTAs fit an SM

struct Ring {
  uint32_t bar, base;
  int stage_bytes, pitch, put = 0, take = 0;
  uint32_t parity = 0;
  Copies copies;

  __device__ __forceinline__ explicit Ring(const WaitBound& b) : copies(b) {}
  __device__ __forceinline__ void begin(uint8_t* bars, uint8_t* stages, int piece, int warp, int lane) {
    pitch = piece * 64;
    stage_bytes = 16 * pitch;
    bar = ptx::smem_u32(bars) + warp * kMoeStages * 8;
    base = ptx::smem_u32(stages) + warp * kMoeStages * stage_bytes;
    if (lane == 0)
      for (int i = 0; i < kMoeStages; ++i) ptx::mbar_init(bar + 8 * i, 1);
    ptx::fence_mbar_init();
    __syncwarp();
  }
  // a piece of rows r0 .. r0 + 7 of one map and r1 .. r1 + 7 of the other, or (m1 == nullptr) of 16 rows of one
  __device__ __forceinline__ void copy(const CUtensorMap* m0, int r0, const CUtensorMap* m1, int r1, int x) {
    if (!copies.issues) return;
    ptx::mbar_arrive_expect_tx(bar + 8 * put, stage_bytes);
    ptx::tma_load_2d(base + put * stage_bytes, m0, x, r0, bar + 8 * put);
    if (m1) ptx::tma_load_2d(base + put * stage_bytes + 8 * pitch, m1, x, r1, bar + 8 * put);
  }
  __device__ __forceinline__ void copied() { put = put + 1 == kMoeStages ? 0 : put + 1; }
  __device__ __forceinline__ uint32_t wait(const WaitBound& b) { copies.wait<false>(bar + 8 * take, parity, b); return base + take * stage_bytes; }
  __device__ __forceinline__ void taken() {
    take = take + 1 == kMoeStages ? 0 : take + 1;
    parity ^= take == 0 ? 1u : 0u;
  }
};

// What a warp needs to multiply a piece, by format.  The activations of a tile are loaded while the tile, or the piece, before
// it is multiplied: first(row, s, n) at the very beginning, then multiply() with the place of the next piece.
//   xr(i)   the lane's row of tile i at the piece's first k
//   next    the lane's row of tile 0 at the next piece's first k, of n_next steps (0: there is none)
// The scales of 4-bit weights come a piece ahead too: scales() asks for the next piece's, scales_here() takes them.
template <class T>
struct Piece16 {
  static constexpr int kStep = 32, kWords = 32;     // weights of a step, and elements of the tensor map
  uint4 x[2][kMostPiece];
  __device__ __forceinline__ void scales(const Stack&, int64_t, const Stack&, int64_t, int, int) {}
  __device__ __forceinline__ void scales_here() {}
  template <int B> __device__ __forceinline__ void load(const uint16_t* row, int n) {
#pragma unroll
    for (int u = 0; u < kMostPiece; ++u)
      if (u < n) x[B][u] = *reinterpret_cast<const uint4*>(row + 32 * u);
  }
  __device__ __forceinline__ void first(const uint16_t* row, int n) { load<0>(row, n); }
  template <int NT, int I, class XR>
  __device__ __forceinline__ void tile(uint32_t w, int pitch, int n, const XR& xr, const uint16_t* next, int n_next, int nt, float (&acc)[NT][4]) {
    if constexpr (I < NT) {
      if (I == 0 || I < nt) {
        if (I + 1 < nt) load<(I + 1) % 2>(xr(I + 1), n);
        else load<(I + 1) % 2>(next, n_next);
#pragma unroll
        for (int u = 0; u < kMostPiece; ++u)
          if (u < n) {
            const uint4 a = lds128(w + u * 64), b = lds128(w + 8 * pitch + u * 64);
            T::mma(acc[I], a.x, b.x, a.y, b.y, x[I % 2][u].x, x[I % 2][u].y);
            T::mma(acc[I], a.z, b.z, a.w, b.w, x[I % 2][u].z, x[I % 2][u].w);
          }
        tile<NT, I + 1>(w, pitch, n, xr, next, n_next, nt, acc);
      }
    }
  }
  template <int NT, class XR>
  __device__ __forceinline__ void multiply(uint32_t w, int pitch, int, int n, const XR& xr, const uint16_t* next, int n_next, int nt, float (&acc)[NT][4]) {
    tile<NT, 0>(w, pitch, n, xr, next, n_next, nt, acc);
    if (NT == 1 || (nt & 1)) {
#pragma unroll
      for (int u = 0; u < kMostPiece; ++u) x[0][u] = x[1][u];
    }
  }
};

template <class T, int PER>
struct PieceQ4 {
  using F = RowsQ4<T, PER, true>;
  using SC = StepScales<T, PER, true, 8>;
  static constexpr int kStep = 128, kWords = 16;
  SC now, next_scales;
  uint4 x[4];
  // the scales of steps s .. s + n - 1 of row0 of one stack and row1 of the other, for the piece after the one at hand
  __device__ __forceinline__ void scales(const Stack& m0, int64_t row0, const Stack& m1, int64_t row1, int s, int n) {
    const int t = threadIdx.x & 3;
    const int64_t groups = (int64_t)((m0.K + 127) / 128) * PER, at0 = row0 * groups + t * PER, at1 = row1 * groups + t * PER;
    next_scales.load(typename SC::Rows{m0.scales + at0, m1.scales + at1, m0.zeros ? m0.zeros + at0 : nullptr, m1.zeros ? m1.zeros + at1 : nullptr},
                     s, n, m0.K - s * 128);
  }
  __device__ __forceinline__ void scales_here() { now = next_scales; }
  __device__ __forceinline__ void activations(const uint16_t* xr) {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = *reinterpret_cast<const uint4*>(xr + 32 * j);
  }
  __device__ __forceinline__ void first(const uint16_t* row, int) { activations(row); }
  struct FirstTile {
    const uint4 (&v)[4];
    template <int OFF> __device__ __forceinline__ uint4 load(int) const { return v[OFF / 32]; }
  };
  template <class XR> struct Tiles {
    const XR& xr;
    int at;
    template <int OFF> __device__ __forceinline__ uint4 load(int i) const { return *reinterpret_cast<const uint4*>(xr(i) + at + OFF); }
  };
  template <int NT, class XR>
  __device__ __forceinline__ void multiply(uint32_t w, int pitch, int, int n, const XR& xr, const uint16_t* next, int n_next, int nt, float (&acc)[NT][4]) {
    F f;
    if (NT == 1 || nt == 1) {   // the next step's activations while this one is multiplied
      float one[1][4] = {{acc[0][0], acc[0][1], acc[0][2], acc[0][3]}};
      for (int u = 0; u < n; ++u) {
        typename F::Regs r;
        now.get(u, r.sa, r.sb, r.za, r.zb);
        r.a = lds128(w + u * 64);
        r.b = lds128(w + 8 * pitch + u * 64);
        const uint4 mine[4] = {x[0], x[1], x[2], x[3]};
        if (u + 1 < n) activations(xr(0) + (u + 1) * 128);
        else if (n_next) activations(next);
        f.template step<1, 0>(r, FirstTile{mine}, All<1>(), one);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[0][i] = one[0][i];
    } else {
      for (int u = 0; u < n; ++u) {
        typename F::Regs r;
        now.get(u, r.sa, r.sb, r.za, r.zb);
        r.a = lds128(w + u * 64);
        r.b = lds128(w + 8 * pitch + u * 64);
        f.template step<NT, 0>(r, Tiles<XR>{xr, u * 128}, nt, acc);
      }
      if (n_next) activations(next);
    }
  }
};
template <class T, int FMT> struct PieceOf { using type = PieceQ4<T, 1 << (FMT - 2)>; };
template <class T> struct PieceOf<T, 1> { using type = Piece16<T>; };

// A CTA cuts its items into parts while it has fewer units than this: two turns of its warps, or one where the sums are large.  With two
// turns for two tiles of tokens the sums (32 KB) and the routing tables left no room for a second CTA of 4-bit experts: 16 tokens,
// 8 of 64 of 4096 x 1536, 245 us; 203 with one turn.
__host__ __device__ constexpr int part_limit(int nt) { return nt == 1 ? 2 * kMoeWarps : kMoeWarps; }

constexpr int kUnitsAhead = 4;

// The routing tables, copied to shared memory (table_bytes() of it).  Every CTA reads the same few lines at the same time, so it
// reads each of them once and no more than a run of this size can fill.
struct Tables {
  Active* active;
  int* token;
  float* weight;
};
__host__ __device__ inline int table_bytes(const MoeParams& p) {
  return p.taken * (int)sizeof(Active) + p.tokens * (p.top_k + p.shared) * 8;
}
__device__ __forceinline__ Tables copy_tables(uint8_t* at, int& n_active, const MoeParams& p) {
  const int entries = p.tokens * (p.top_k + p.shared);
  Tables tb;
  tb.active = reinterpret_cast<Active*>(at);
  tb.token = reinterpret_cast<int*>(at + p.taken * sizeof(Active));
  tb.weight = reinterpret_cast<float*>(tb.token + entries);
  for (int i = threadIdx.x; i < p.taken; i += kMoeThreads) *reinterpret_cast<int4*>(&tb.active[i]) = __ldcg(reinterpret_cast<const int4*>(p.active) + i);
  for (int i = (int)threadIdx.x - 32; i < entries; i += kMoeThreads)
    if (i >= 0) tb.token[i] = __ldcg(p.entry_token + i);
  for (int i = (int)threadIdx.x - 64; i < entries; i += kMoeThreads)
    if (i >= 0) tb.weight[i] = __ldcg(p.entry_weight + i);
  if (threadIdx.x == kMoeThreads - 1) n_active = __ldcg(p.n_active);
  __syncthreads();
  return tb;
}

// ==== up ==========================================================================================================
// An item is 8 inner values of one taken expert for its tokens: the 16 rows of a fragment are eight rows of gate and the
// same eight of up, so that a lane ends with both factors of an activation.  The grid shares the items out; a CTA's warps
// take its items one by one, or, where there are fewer items than warps, parts of their `hidden`, whose sums meet in
// shared memory in order.
template <class T, int FMT, int NT>
__global__ void __launch_bounds__(kMoeThreads, NT <= 2 || FMT == 1 ? 2 : 1)
exo_moe_up_ring_kernel(const MoeParams p, const __grid_constant__ CUtensorMap gate_map, const __grid_constant__ CUtensorMap up_map) {
  using P = typename PieceOf<T, FMT>::type;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int active_shared, next_unit, ahead_of[kMoeWarps][kUnitsAhead];
  __shared__ __align__(8) uint8_t bars[kMoeWarps * kMoeStages * 8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  Ring ring(p.up_wait);
  ring.begin(bars, smem, p.up_piece, warp, lane);
  float4* sums = reinterpret_cast<float4*>(smem + kMoeWarps * kMoeStages * ring.stage_bytes);   // [unit][tile][lane]
  const int tiles = (p.inner + 7) / 8, steps = (p.hidden + P::kStep - 1) / P::kStep, pieces = (steps + p.up_piece - 1) / p.up_piece;
  if (threadIdx.x == 0) next_unit = kMoeWarps;
  if (lane == 0) { ptx::prefetch_tensormap(&gate_map); ptx::prefetch_tensormap(&up_map); }
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();   // after the wait: `down` may then read the tables of `route` before it waits itself
  const Tables tb = copy_tables(reinterpret_cast<uint8_t*>(sums + 2 * part_limit(NT) * NT * 32), active_shared, p);
  const int n_active = active_shared;
  const int items = n_active * tiles;
  const int mine = (int)blockIdx.x < items ? (items - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x : 0;
  int nk_log = 0;
  while (nk_log < 3 && (mine << nk_log) < part_limit(NT) && (2 << nk_log) <= pieces) ++nk_log;
  const int units = mine << nk_log, nk = 1 << nk_log;
  auto begin_of = [&](int u) { return (pieces * (u & (nk - 1))) >> nk_log; };
  auto end_of = [&](int u) { return (pieces * ((u & (nk - 1)) + 1)) >> nk_log; };
  // items by expert, the last first: the shared experts, who have all tokens, are last
  auto item_of = [&](int u) { return (int)blockIdx.x + (u >> nk_log) * (int)gridDim.x; };
  auto expert_of = [&](int item) { return n_active - 1 - item / tiles; };
  // A warp takes its first unit by its number and any other when its copies get there; the numbers of the units between the
  // copies and the products (at most one per stage, the one that is open, and the end) wait in shared memory.
  int* ahead = ahead_of[warp];
  int iu = warp, ip = begin_of(warp), igate = 0, iup = 0, put = 1;
  if (lane == 0) ahead[0] = warp;
  auto open = [&]() {
    const int item = item_of(iu), f0 = item % tiles * 8, expert = tb.active[expert_of(item)].expert;
    igate = (int)(expert * p.gate.expert_rows) + f0;
    iup = (int)(expert * p.up.expert_rows) + f0;
  };
  auto issue = [&]() {
    if (iu < units) {
      ring.copy(&gate_map, igate, &up_map, iup, ip * p.up_piece * P::kWords);
      ring.copied();
      if (++ip == end_of(iu)) {
        if (lane == 0) {
          iu = atomicAdd(&next_unit, 1);
          ahead[put % kUnitsAhead] = iu;
        }
        iu = __shfl_sync(0xffffffffu, iu, 0);
        ++put;
        if (iu < units) {
          ip = begin_of(iu);
          open();
        }
      }
    }
  };
  if (iu < units) open();
  for (int i = 0; i < kMoeStages; ++i) issue();
  __syncwarp();

  // the lane's row of activations for tile i of an item's tokens; columns without a token repeat the last one's
  auto row_of = [&](const Active& a, int i) { return p.xs + (int64_t)tb.token[a.base + min(8 * i + g, a.count - 1)] * p.ldxs + 8 * t; };
  auto steps_at = [&](int c) { return min(p.up_piece, steps - c * p.up_piece); };
  P piece;
  auto ask_scales = [&](int u, int c) {
    const int item = item_of(u), expert = tb.active[expert_of(item)].expert;
    const int64_t row = min(item % tiles * 8 + g, p.inner - 1);
    piece.scales(p.gate, expert * p.gate.expert_rows + row, p.up, expert * p.up.expert_rows + row, c * p.up_piece, steps_at(c));
  };
  if (warp < units) {
    ask_scales(warp, begin_of(warp));
    piece.first(row_of(tb.active[expert_of(item_of(warp))], 0) + begin_of(warp) * p.up_piece * P::kStep, steps_at(begin_of(warp)));
  }
  for (int u = warp, took = 1; u < units; ++took) {
    const int item = item_of(u), f0 = item % tiles * 8;
    const Active a = tb.active[expert_of(item)];
    const int nt = (a.count + 7) / 8;
    const uint16_t* xrow[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) xrow[i] = row_of(a, i);
    float acc[NT][4];
    clear(acc);
    const int end = end_of(u);
    int after = units;                 // the unit after this one
    for (int c = begin_of(u); c < end; ++c) {
      const int s = c * p.up_piece, n = steps_at(c);
      const uint16_t* next = xrow[0] + (s + p.up_piece) * P::kStep;
      int n_next = c + 1 < end ? steps_at(c + 1) : 0;
      piece.scales_here();
      if (c + 1 < end) {
        ask_scales(u, c + 1);
      } else {
        after = ahead[took % kUnitsAhead];   // its copies have begun, or there is none
        if (after < units) {
          ask_scales(after, begin_of(after));
          next = row_of(tb.active[expert_of(item_of(after))], 0) + begin_of(after) * p.up_piece * P::kStep;
          n_next = steps_at(begin_of(after));
        }
      }
      const uint32_t w = ring.wait(p.up_wait) + g * ring.pitch + 16 * t;
      piece.template multiply<NT>(w, ring.pitch, s, n, [&](int i) { return xrow[i] + s * P::kStep; }, next, n_next, nt, acc);
      __syncwarp();
      ring.taken();
      issue();
      __syncwarp();
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      if (i < nt) {
        const float4 v = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
        if (nk_log == 0) store_inner<T>(p, tb.weight, a, f0, i, lane, v);
        else sums[(u * NT + i) * 32 + lane] = v;
      }
    }
    u = after;
  }
  if (nk_log > 0) {
    __syncthreads();
    for (int idx = threadIdx.x; idx < mine * NT * 32; idx += kMoeThreads) {
      const int k = idx / (NT * 32), i = (idx >> 5) % NT;
      const int item = (int)blockIdx.x + k * (int)gridDim.x;
      const Active a = tb.active[expert_of(item)];
      if (8 * i >= a.count) continue;
      float4 v = sums[((k << nk_log) * NT + i) * 32 + (idx & 31)];
      for (int q = 1; q < nk; ++q) add(v, sums[(((k << nk_log) + q) * NT + i) * 32 + (idx & 31)]);
      store_inner<T>(p, tb.weight, a, (item % tiles) * 8, i, idx & 31, v);
    }
  }
}

// ==== down ========================================================================================================
// A cluster computes 16 rows of y for all tokens.  Its warps share the steps of all taken experts, one after another,
// in equal ranges; a warp adds what an expert gives onto its own sums in shared memory, by token.  The sums meet
// in warp order and then in rank order.
template <class T, int FMT, int NT>
__global__ void __launch_bounds__(kMoeThreads, NT <= 2 || FMT == 1 ? 2 : 1)
exo_moe_down_ring_kernel(const MoeParams p, const __grid_constant__ CUtensorMap map) {
  namespace cg = cooperative_groups;
  using P = typename PieceOf<T, FMT>::type;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int all_costs, active_shared;
  __shared__ __align__(8) uint8_t bars[kMoeWarps * kMoeStages * 8];
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), r = (int)cluster.block_rank();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int row0 = (int)(blockIdx.x / S) * 16;
  Ring ring(p.down_wait);
  ring.begin(bars, smem, p.down_piece, warp, lane);
  float* sums = reinterpret_cast<float*>(smem + kMoeWarps * kMoeStages * ring.stage_bytes);   // [warp][token][row]
  float* part = sums + kMoeWarps * p.tokens * 16;             // [token][row]
  const int steps = (p.inner + P::kStep - 1) / P::kStep;
  if (lane == 0) ptx::prefetch_tensormap(&map);
  // `route` is complete: `up` started this kernel after it had waited for that
  for (int i = threadIdx.x; i < kMoeWarps * p.tokens * 16; i += kMoeThreads) sums[i] = 0.f;
  const Tables tb = copy_tables(reinterpret_cast<uint8_t*>(part + p.tokens * 16), active_shared, p);
  const int n_active = active_shared;
  // A step costs a warp its weights and then its tiles of tokens: three parts and two for every tile.  Equal shares of that.
  auto cost_of = [&](int at) { return 3 + 2 * (((tb.active[at].count << halves_of(tb.active[at].count)) + 7) / 8); };
  if (warp == 0) {
    int before = 0;
    for (int e0 = 0; e0 < n_active; e0 += 32) {
      int sum = e0 + lane < n_active ? cost_of(e0 + lane) : 0;
      const int own = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += v;
      }
      if (e0 + lane < n_active) tb.active[e0 + lane].cost_before = before + sum - own;
      before += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (lane == 0) all_costs = before;
  }
  __syncthreads();
  const int64_t total = (int64_t)all_costs * steps;
  const int64_t workers = (int64_t)S * kMoeWarps, q = r * kMoeWarps + warp;
  auto place = [&](int64_t cost, int& at, int& s) {   // the step that begins at or after this point
    int lo = 0, hi = n_active;                        // the last expert that begins at or before it
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if ((int64_t)tb.active[mid].cost_before * steps <= cost) lo = mid; else hi = mid;
    }
    const int c = cost_of(lo);
    at = lo;
    s = (int)((cost - (int64_t)tb.active[lo].cost_before * steps + c - 1) / c);
    if (s >= steps) { s = 0; ++at; }
  };
  int at, s, end_at, end_s;
  place(total * q / workers, at, s);
  place(total * (q + 1) / workers, end_at, end_s);
  float* mine = sums + warp * p.tokens * 16;
  // steps of expert e that are this warp's end here
  auto stop_of = [&](int e) { return e < end_at ? steps : end_s; };
  auto any = [&](int e, int from) { return e < end_at || (e == end_at && from < end_s); };
  int iat = at, is = s;                               // the next copy
  auto issue = [&]() {
    if (any(iat, is)) {
      ring.copy(&map, (int)(tb.active[iat].expert * p.down.expert_rows) + row0, nullptr, 0, is * P::kWords);
      ring.copied();
      is = min(is + p.down_piece, stop_of(iat));
      if (is == steps) { is = 0; ++iat; }
    }
  };
  for (int i = 0; i < kMoeStages; ++i) issue();
  ptx::grid_dependency_wait();     // `up` is complete
  ptx::grid_launch_dependents();
  // rows behind an expert's are other entries', or spare ones
  auto row_at = [&](int e, int from) { return p.h + (2 * (int64_t)tb.active[e].base + g) * p.ldh + 8 * t + from * P::kStep; };
  P piece;
  auto ask_scales = [&](int e, int from, int n) {
    const int64_t first = tb.active[e].expert * p.down.expert_rows;
    piece.scales(p.down, first + min(row0 + g, p.hidden - 1), p.down, first + min(row0 + g + 8, p.hidden - 1), from, n);
  };
  if (any(at, s)) {
    const int n = min(p.down_piece, stop_of(at) - s);
    ask_scales(at, s, n);
    piece.first(row_at(at, s), n);
  }
  while (any(at, s)) {
    const Active a = tb.active[at];
    const int halves = halves_of(a.count), columns = a.count << halves, nt = (columns + 7) / 8, stop = stop_of(at);
    float acc[NT][4];
    clear(acc);
    while (s < stop) {
      const int n = min(p.down_piece, stop - s), after = s + n;
      const uint16_t* here = row_at(at, s);
      const bool more = after < stop;
      const int ne = more ? at : at + 1, nf = more ? after : 0;
      const int n_next = any(ne, nf) ? min(p.down_piece, stop_of(ne) - nf) : 0;
      const uint16_t* next = n_next ? row_at(ne, nf) : here;
      piece.scales_here();
      if (n_next) ask_scales(ne, nf, n_next);
      const uint32_t w = ring.wait(p.down_wait) + g * ring.pitch + 16 * t;
      piece.template multiply<NT>(w, ring.pitch, s, n, [&](int i) { return here + (int64_t)8 * i * p.ldh; }, next, n_next, nt, acc);
      __syncwarp();
      ring.taken();
      issue();
      s = after;
    }
#pragma unroll
    for (int i = 0; i < NT; ++i)
      if (i < nt) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int n = 8 * i + 2 * t + c;
          if (n < columns) {   // both parts of an activation are the same lane's
            float* to = mine + tb.token[a.base + (n >> halves)] * 16 + g;
            to[0] += acc[i][c];
            to[8] += acc[i][2 + c];
          }
        }
      }
    __syncwarp();
    s = 0;
    ++at;
  }
  __syncthreads();
  auto finish = [&](int idx, float v) {
    const int row = row0 + (idx & 15);
    if (row < p.hidden) p.y[(int64_t)(idx >> 4) * p.ldy + row] = T::from_float(v);
  };
  for (int idx = threadIdx.x; idx < p.tokens * 16; idx += kMoeThreads) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kMoeWarps; ++w) v += sums[w * p.tokens * 16 + idx];
    if (S == 1) finish(idx, v);
    else part[idx] = v;
  }
  if (S > 1) {
    cluster.sync();
    for (int idx = r * kMoeThreads + threadIdx.x; idx < p.tokens * 16; idx += S * kMoeThreads) {
      float v = 0.f;
      for (int o = 0; o < S; ++o) v += cluster.map_shared_rank(part, o)[idx];
      finish(idx, v);
    }
    cluster.sync();
  }
}

// ==== 16-bit rows that a tiled copy cannot address ==================================================================
// Rows that do not start on 16-byte boundaries are read element by element, straight into the fragments: right at any
// leading dimension, and slow (us, 8 of 64 experts: one token 2048 x 1024 32, 2044 x 1020 92, 2047 x 1023 81; 16 tokens 143, 573 and 485; 6 of 64 and a
// shared one, 64 tokens, 4096 x 1536 540, 4095 x 1535 1538).
constexpr int kPlainThreads = 256, kPlainWarps = 8;

// Steps of 32 from s on, ds apart, of the lane's rows r0 and r1; the lane's activations of tile i begin at x0 + i * stride, or at
// rows[i] where x0 is NULL.
template <class T, int NT>
__device__ __forceinline__ void plain_steps(const uint16_t* r0, const uint16_t* r1, const uint16_t* x0, int64_t stride, const uint16_t* const (&rows)[NT],
                                            int s, int ds, int end, int K, int t, int nt, float (&acc)[NT][4]) {
  for (; s < end; s += ds) {
    const int k = s * 32 + 8 * t;
    const uint4 wa = load8_checked(r0, k, K, false), wb = load8_checked(r1, k, K, false);
#pragma unroll
    for (int i = 0; i < NT; ++i)
      if (i < nt) {
        const uint4 b = *reinterpret_cast<const uint4*>((x0 ? x0 + i * stride : rows[i]) + s * 32);
        T::mma(acc[i], wa.x, wb.x, wa.y, wb.y, b.x, b.y);
        T::mma(acc[i], wa.z, wb.z, wa.w, wb.w, b.z, b.w);
      }
  }
}

template <class T, int NT>
__global__ void __launch_bounds__(kPlainThreads) exo_moe_up_plain_kernel(const MoeParams p) {
  __shared__ float4 red[kPlainWarps * NT * 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();   // after the wait: `down` may then read the tables of `route` before it waits itself
  if ((int)blockIdx.y >= __ldcg(p.n_active)) return;
  const int4 raw = __ldcg(reinterpret_cast<const int4*>(p.active + blockIdx.y));
  const Active a{raw.x, raw.y, raw.z, raw.w};
  const int f0 = blockIdx.x * 8, nt = (a.count + 7) / 8;
  const int64_t row = min(f0 + g, p.inner - 1);
  const uint16_t* r0 = static_cast<const uint16_t*>(p.gate.w) + (a.expert * p.gate.expert_rows + row) * p.gate.ld;
  const uint16_t* r1 = static_cast<const uint16_t*>(p.up.w) + (a.expert * p.up.expert_rows + row) * p.up.ld;
  const uint16_t* xrow[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
    xrow[i] = p.xs + (int64_t)__ldcg(p.entry_token + a.base + min(8 * i + g, a.count - 1)) * p.ldxs + 8 * t;
  float acc[NT][4];
  clear(acc);
  plain_steps<T, NT>(r0, r1, nullptr, 0, xrow, warp, kPlainWarps, (p.hidden + 31) / 32, p.hidden, t, nt, acc);
#pragma unroll
  for (int i = 0; i < NT; ++i)
    if (i < nt) red[(warp * nt + i) * 32 + lane] = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
  __syncthreads();
  for (int idx = threadIdx.x; idx < nt * 32; idx += kPlainThreads) {
    float4 v = red[idx];
    for (int q = 1; q < kPlainWarps; ++q) add(v, red[q * nt * 32 + idx]);
    store_inner<T>(p, p.entry_weight, a, f0, idx >> 5, idx & 31, v);
  }
}

template <class T, int NT>
__global__ void __launch_bounds__(kPlainThreads) exo_moe_down_plain_kernel(const MoeParams p) {
  extern __shared__ __align__(128) uint8_t smem[];
  float* sums = reinterpret_cast<float*>(smem);               // [warp][token][row]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int row0 = (int)blockIdx.x * 16, steps = (p.inner + 31) / 32;
  for (int i = threadIdx.x; i < kPlainWarps * p.tokens * 16; i += kPlainThreads) sums[i] = 0.f;
  __syncthreads();
  float* mine = sums + warp * p.tokens * 16;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int n_active = __ldcg(p.n_active);
  for (int at = 0; at < n_active; ++at) {
    const int4 raw = __ldcg(reinterpret_cast<const int4*>(p.active + at));
    const Active a{raw.x, raw.y, raw.z, raw.w};
    const int halves = halves_of(a.count), columns = a.count << halves, nt = (columns + 7) / 8;
    const int64_t first = a.expert * p.down.expert_rows;
    const uint16_t* r0 = static_cast<const uint16_t*>(p.down.w) + (first + min(row0 + g, p.hidden - 1)) * p.down.ld;
    const uint16_t* r1 = static_cast<const uint16_t*>(p.down.w) + (first + min(row0 + g + 8, p.hidden - 1)) * p.down.ld;
    float acc[NT][4];
    clear(acc);
    const uint16_t* none[NT] = {};
    plain_steps<T, NT>(r0, r1, p.h + (2 * (int64_t)a.base + g) * p.ldh + 8 * t, 8 * p.ldh, none, warp, kPlainWarps, steps, p.inner, t, nt, acc);
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int n = 8 * i + 2 * t + c;
        if (i < nt && n < columns) {
          float* to = mine + __ldcg(p.entry_token + a.base + (n >> halves)) * 16 + g;
          to[0] += acc[i][c];
          to[8] += acc[i][2 + c];
        }
      }
    __syncwarp();
  }
  __syncthreads();
  for (int idx = threadIdx.x; idx < p.tokens * 16; idx += kPlainThreads) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kPlainWarps; ++w) v += sums[w * p.tokens * 16 + idx];
    const int row = row0 + (idx & 15);
    if (row < p.hidden) p.y[(int64_t)(idx >> 4) * p.ldy + row] = T::from_float(v);
  }
}

// ---- kernels by type, format and token count --------------------------------------------------------------------
template <class T, bool VEC> void* pick_route(int nt) {
  return nt == 1 ? (void*)exo_moe_route_kernel<T, VEC, 1> : nt == 2 ? (void*)exo_moe_route_kernel<T, VEC, 2> : (void*)exo_moe_route_kernel<T, VEC, 8>;
}
template <class T, int FMT> void* pick_up_nt(int nt) {
  if constexpr (FMT == 0)
    return nt == 1 ? (void*)exo_moe_up_plain_kernel<T, 1> : nt == 2 ? (void*)exo_moe_up_plain_kernel<T, 2> : (void*)exo_moe_up_plain_kernel<T, 8>;
  else
    return nt == 1 ? (void*)exo_moe_up_ring_kernel<T, FMT, 1> : nt == 2 ? (void*)exo_moe_up_ring_kernel<T, FMT, 2> : (void*)exo_moe_up_ring_kernel<T, FMT, 8>;
}
template <class T, int FMT> void* pick_down_nt(int nt) {
  if constexpr (FMT == 0)
    return nt == 1 ? (void*)exo_moe_down_plain_kernel<T, 1> : nt == 2 ? (void*)exo_moe_down_plain_kernel<T, 2> : (void*)exo_moe_down_plain_kernel<T, 8>;
  else
    return nt == 1 ? (void*)exo_moe_down_ring_kernel<T, FMT, 1> : nt == 2 ? (void*)exo_moe_down_ring_kernel<T, FMT, 2> : (void*)exo_moe_down_ring_kernel<T, FMT, 8>;
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

// Tensor map of a stack for pieces of `steps` steps of `box_rows` rows.
bool stack_map(CUtensorMap* map, const Stack& m, int64_t all, bool q4, int steps, int box_rows) {
  const uint64_t rows = (uint64_t)((all - 1) * m.expert_rows + m.rows), blocks = (uint64_t)(m.K + 127) / 128;
  return q4 ? exo::encode_rows_map(map, 4, m.w, blocks * 16, rows, blocks * 64, (uint32_t)steps * 16, (uint32_t)box_rows)
            : exo::encode_rows_map(map, 2, m.w, (uint64_t)m.K, rows, (uint64_t)m.ld * 2, (uint32_t)steps * 32, (uint32_t)box_rows);
}

bool rows_aligned(const void* w, int64_t ld) { return ((uintptr_t)w & 15u) == 0 && ld % 8 == 0; }

// all: experts of the stack
exo_gemm_status_t check_stack(const exo_moe_matrix_t& m, int64_t rows, int64_t K, int64_t all, int q4_group) {
  if (!m.w) return EXO_GEMM_ERR_NULL;
  if (m.expert_rows < rows || m.expert_rows > (1LL << 40)) return EXO_GEMM_ERR_INVALID_ARG;
  if (all * m.expert_rows > 0x7fffffffLL - 16) return EXO_GEMM_ERR_UNSUPPORTED;   // row numbers are 32 bits in a tensor map's copies
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

namespace exo {
namespace decode {
unsigned take_gave_up_moe(cudaError_t* e) { return take_gave_up(e); }
}  // namespace decode
}  // namespace exo

using namespace exo::decode;

struct exo_moe_plan {
  exo_moe_desc_t desc;
  int device, sms;
  int64_t ldh, ldxs, bytes;
  uint8_t* ws;
  int64_t at_active, at_token, at_weight, at_logits, at_xs, at_h;   // offsets into ws; the arrival counter and n_active come first
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
  plan->ldxs = (d->hidden + 127) / 128 * 128;
  plan->at_xs = take((int64_t)d->max_tokens * plan->ldxs * 2);
  plan->at_h = take((2 * entries + 8) * plan->ldh * 2);   // a last tile of eight may read rows behind the last one
  plan->bytes = at;
  cudaError_t e = cudaMalloc((void**)&plan->ws, (size_t)plan->bytes);
  if (e == cudaSuccess) {
    e = exo::clear_now(plan->ws, (size_t)plan->bytes);   // the counter, and the padding of the inner activations
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
  const int64_t all = d.experts + d.shared;
  exo_gemm_status_t st;
  if ((st = check_stack(w->gate, d.inner, d.hidden, all, d.q4_group)) != EXO_GEMM_OK) return st;
  if ((st = check_stack(w->up, d.inner, d.hidden, all, d.q4_group)) != EXO_GEMM_OK) return st;
  if ((st = check_stack(w->down, d.hidden, d.inner, all, d.q4_group)) != EXO_GEMM_OK) return st;
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
  p.taken = (int)((int64_t)p.tokens * p.top_k < p.experts ? (int64_t)p.tokens * p.top_k : p.experts) + p.shared;
  p.renormalize = d.renormalize != 0; p.routed_scale = d.routed_scale;
  p.x_aligned = rows_aligned(x, ldx);
  p.arrivals = (unsigned*)plan->ws;
  p.n_active = (int*)(plan->ws + 128);
  p.active = (Active*)(plan->ws + plan->at_active);
  p.entry_token = (int*)(plan->ws + plan->at_token);
  p.entry_weight = (float*)(plan->ws + plan->at_weight);
  p.logits = (float*)(plan->ws + plan->at_logits);
  p.h = (uint16_t*)(plan->ws + plan->at_h);

  p.copy_x = !(p.x_aligned && d.hidden % 128 == 0);
  p.xs = p.copy_x ? (const uint16_t*)(plan->ws + plan->at_xs) : p.x;
  p.ldxs = p.copy_x ? plan->ldxs : ldx;
  // Pieces: larger ones suit the copies, smaller ones leave room for a second CTA on the SM, which covers the first one's
  // start and end (5 steps: 80 KB of ring), up to 16 tokens, whose sums leave room for it.  5 steps against 7 (us): 16 bits, 64 experts of
  // 4096 x 1536 and a shared one, 8 tokens 234 / 243, 9 tokens 254 / 271, 16 tokens 319 / 343, 20 tokens 411 / 414, 64 tokens 645 / 538; 8 of 64 of
  // 2048 x 1024, 16 tokens 136 / 141.  4 bits, 8 experts of 4096 x 8192, one token 50.6 / 55.8, 16 tokens 162 / 209, 24 tokens 311 / 302, 64 tokens
  // 728 / 715: 5 for all.
  p.up_piece = p.down_piece = !q4 && p.tokens > 16 ? 7 : 5;

  const WaitHook hook = take_wait_hook();
  p.up_wait = WaitBound{hook.clocks, hook.skip == 1};
  p.down_wait = WaitBound{hook.clocks, hook.skip == 2};

  const bool bf16 = d.dtype == EXO_GEMM_BF16;
  const int nt = (p.tokens + 7) / 8;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;

  // formats and tensor maps, before anything is launched
  const int q4_fmt = d.q4_group == 128 ? 2 : d.q4_group == 64 ? 3 : 4, step = q4 ? 128 : 32, nt_kernel = nt <= 2 ? nt : 8;
  const int up_fmt = q4 ? q4_fmt : rows_aligned(w->gate.w, w->gate.ld) && rows_aligned(w->up.w, w->up.ld) ? 1 : 0;
  const int down_fmt = q4 ? q4_fmt : rows_aligned(w->down.w, w->down.ld) ? 1 : 0;
  CUtensorMap gate, up, down;
  if (up_fmt && (!stack_map(&gate, p.gate, all, q4, p.up_piece, 8) || !stack_map(&up, p.up, all, q4, p.up_piece, 8))) return EXO_GEMM_ERR_CUDA;
  if (down_fmt && !stack_map(&down, p.down, all, q4, p.down_piece, 16)) return EXO_GEMM_ERR_CUDA;

  const bool router_aligned = rows_aligned(w->router, w->ld_router);
  int S = 1;
  void* fn;
  if (p.tokens <= kOneTokens && p.experts <= kOneExperts && (int64_t)p.experts * p.hidden <= 1 << 20) {   // at most 256 KB of the router to a CTA
    fn = bf16 ? (router_aligned ? (void*)exo_moe_route_one_kernel<Bf16, true> : (void*)exo_moe_route_one_kernel<Bf16, false>)
              : (router_aligned ? (void*)exo_moe_route_one_kernel<Fp16, true> : (void*)exo_moe_route_one_kernel<Fp16, false>);
    st = launch(fn, kOneCtas, 1, kRouteThreads, 0, kOneCtas, stream, &p);
  } else {   // 16 experts per cluster; a warp keeps a step of 32
    const int steps = (p.hidden + 31) / 32;
    while (S < 8 && steps >= 2 * S * kRouteWarps) S *= 2;
    fn = bf16 ? (router_aligned ? pick_route<Bf16, true>(nt) : pick_route<Bf16, false>(nt))
              : (router_aligned ? pick_route<Fp16, true>(nt) : pick_route<Fp16, false>(nt));
    st = launch(fn, (unsigned)((p.experts + 15) / 16 * S), 1, kRouteThreads, (size_t)(kRouteWarps + 1) * nt * 512, (unsigned)S, stream, &p);
  }
  if (st != EXO_GEMM_OK) return st;

  fn = bf16 ? pick_up<Bf16>(up_fmt, nt) : pick_up<Fp16>(up_fmt, nt);
  if (up_fmt == 0) {
    st = launch(fn, (unsigned)((p.inner + 7) / 8), (unsigned)p.taken, kPlainThreads, 0, 1, stream, &p);
  } else {
    const size_t smem = (size_t)kMoeWarps * kMoeStages * p.up_piece * 1024 + (size_t)2 * part_limit(nt_kernel) * nt_kernel * 512 + table_bytes(p);
    const int64_t items = (int64_t)p.taken * ((p.inner + 7) / 8), slots = (int64_t)(smem <= kPairSmem ? 2 : 1) * plan->sms;
    st = launch(fn, (unsigned)(items < slots ? items : slots), 1, kMoeThreads, smem, 1, stream, &p, &gate, &up);
  }
  if (st != EXO_GEMM_OK) return st;

  const int64_t tiles = (p.hidden + 15) / 16, all_steps = (int64_t)p.taken * ((p.inner + step - 1) / step);
  fn = bf16 ? pick_down<Bf16>(down_fmt, nt) : pick_down<Fp16>(down_fmt, nt);
  if (down_fmt == 0)
    return launch(fn, (unsigned)tiles, 1, kPlainThreads, (size_t)kPlainWarps * p.tokens * 64, 1, stream, &p);
  // The cluster size with the shortest estimate: a turn of the CTAs that fit costs their start and end (4 us, and more for
  // the sums of many tokens) and the weights at an SM's share of the bandwidth, 44 GB/s.
  const size_t smem = (size_t)kMoeWarps * kMoeStages * p.down_piece * 1024 + (size_t)(kMoeWarps + 1) * p.tokens * 64 + table_bytes(p);
  const int fit = smem <= kPairSmem && !(q4 && nt_kernel > 2) ? 2 : 1;   // (eight tiles of 4-bit experts take all registers)
  S = 1;
  double best = 0.0;
  for (int c = 1; c <= 8 && (c == 1 || all_steps >= (int64_t)c * kMoeWarps); c *= 2) {
    const double us = (double)((tiles * c + fit * plan->sms - 1) / (fit * plan->sms)) * (4.0 + 0.1 * p.tokens + (double)all_steps * 1024.0 / c / (44e3 / fit));
    if (c == 1 || us < best) { best = us; S = c; }
  }
  return launch(fn, (unsigned)(tiles * S), 1, kMoeThreads, smem, (unsigned)S, stream, &p, &down);
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

// Products whose epilogue is an operator: the two kernels behind exo_fused.h.
//
// exo_fused_pair_kernel   persistent, a pair of CTAs (tcgen05 cta_group::2) per tile of 256 rows x up to 256 accumulator columns, two
//                         accumulators in tensor memory, so that a tile's epilogue runs beside the next tile's main loop
// exo_fused_thin_kernel   up to 128 rows (a few tokens): one tile per CTA, two CTAs per SM; what counts is the stream of B's rows
//
// The operator is a class `Op`: its epilogue takes a row's accumulator columns in units of U, and for a gated product (Op::kGated) two units
// at once, the second from `gap` columns further on.  There the rows of B that a tile stages are `gap` rows of gate and `gap` rows of up:
// CTA 0 of a pair stages the ones and CTA 1 the others, which is how a pair splits B anyway, so both projections are one product.
//
// A row of the accumulator is a lane's, so a warp's access to memory is to 32 rows.  Operands of an epilogue are asked for a unit ahead, in whole
// 32-byte sectors (a training step's backward kernel, 1024 tokens of 1024 x 2816: 3.3 us less than with 16 bytes); 16-bit results go through
// shared memory and TMA stores where their rows allow that (the pair kernel's Out; 8192 x 32000 x 4096 with the exponentials kept: 1432 us with
// stores from registers, 1404), and rows that start anywhere are stored by neighbouring lanes (8 bits, 320 x 1865 x 3648: 34.5 us a row per lane, 18.1).
//
// Every wait is bounded: one that gives up records that with its plan, all roles leave their loops, tensor memory is freed and the kernel returns.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "gemm_params.h"
#include "ptx.cuh"

namespace exo {
namespace fused {

struct Bf16 {
  using type = __nv_bfloat16;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
  }
  static __device__ __forceinline__ float2 unpack(uint32_t w) { return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&w)); }
};
struct Fp16 {
  using type = __half;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
  }
  static __device__ __forceinline__ float2 unpack(uint32_t w) { return __half22float2(*reinterpret_cast<__half2*>(&w)); }
};

struct Waits {
  uint64_t clocks;     // bound of every wait, in SM clocks
  uint32_t* gave_up;   // the plan's count of waits that gave up; NULL for operators without a plan, which share their file's
};

struct CoreParams {
  int32_t M, N;        // rows of A, and columns of the result (columns of gate, for a gated product)
  int32_t nkb;         // k-blocks: 128 bytes of a row of A and of B
  int32_t stages;
  int32_t width;       // result columns of a tile
  int32_t b_split;     // pair: how many rows of B lie between what CTA 0 and what CTA 1 stage
  int32_t a_rows;      // thin: rows of A staged, M rounded up to 8
  int32_t quad_rows;   // thin: rows in a lane quadrant of the accumulator: 16 where the MMAs have 64 rows, 32 where they have 128
  int32_t per_stage;   // thin: k-blocks of a stage
  int32_t whole;       // thin: k-blocks that are whole; the last one may not be
  int32_t buffers;     // pair: of an epilogue warp, for results
  int32_t split;       // thin: CTAs (a cluster of 1, 2, 4 or 8) that share a tile's K
  uint32_t idesc;
  OperandStaging a, b;
  Raster raster;
  Waits waits;
  int32_t skip_copies;    // test hook: CTA 0 leaves out the copies of its first k-block
};

constexpr int kPairBarrierBytes = 512;
constexpr int kPairMaxStages = 10;
constexpr int kOutBytes = 2048;      // a buffer for results of an epilogue warp: 32 rows x 32 values of 16 bits
constexpr int kThinThreads = 320;    // producer, MMA issuer, eight epilogue warps
constexpr int kThinMaxStages = 16;
constexpr int kThinBarrierBytes = 512;

EXO_CX int pair_stage_bytes(int bn) { return kATileBytes + bn / 2 * 128; }
EXO_CX int pair_stages(int bn, int buffers) {
  const int n = (kSmemLimit - 1024 - kPairBarrierBytes - kEpiWarps * buffers * kOutBytes) / pair_stage_bytes(bn);
  return n > kPairMaxStages ? kPairMaxStages : n;
}
EXO_CX int pair_smem(int bn, int buffers) {
  return pair_stages(bn, buffers) * pair_stage_bytes(bn) + kEpiWarps * buffers * kOutBytes + kPairBarrierBytes + 1024;
}
// The MMAs read 64 or 128 rows of A whatever a stage holds of it: what follows the rows staged becomes accumulator rows that nobody reads, and
// behind the last stage it is room that the ring keeps.
EXO_CX int thin_mma_rows(int a_rows) { return a_rows <= 64 ? 64 : 128; }
// What the epilogue keeps in the ring, when that is idle: buffers for results, and the partial sums of the other CTAs of a cluster, warp_bytes of
// each warp.
EXO_CX int thin_after(int warp_bytes, int split) { return kEpiWarps * (2 * kOutBytes + (split - 1) * warp_bytes); }
EXO_CX int thin_smem(int stages, int per_stage, int b_rows, int a_rows, int after) {
  const int ring = stages * per_stage * (b_rows + a_rows) * 128 + (thin_mma_rows(a_rows) - a_rows) * 128;
  return 1024 + kThinBarrierBytes + 512 + (ring > after ? ring : after);
}

// ---------------------------------------------------------------- bounded waits
// Waits that gave up in this translation unit's kernels on this device, whoever's they were (exo_fused_check).
static __device__ uint32_t fused_gave_up;

static __device__ __noinline__ bool wait_slow(uint32_t bar, uint32_t parity, uint64_t clocks, uint32_t* gave_up) {
  const long long t0 = clock64();
  uint32_t* const word = gave_up ? gave_up : &fused_gave_up;
  uint32_t n = 0;
  for (;;) {
    if (ptx::mbar_try_wait(bar, parity)) return true;
    if ((++n & 63u) == 0u) {
      if (*(volatile uint32_t*)word != 0u) return false;   // another role, or an earlier launch that nobody has asked about
      if ((uint64_t)(clock64() - t0) > clocks) {
        atomicAdd(word, 1u);
        if (gave_up) atomicAdd(&fused_gave_up, 1u);
        return false;
      }
    }
  }
}
__device__ __forceinline__ bool wait_on(uint32_t bar, uint32_t parity, const Waits& w) {
#pragma unroll 1
  for (int i = 0; i < 8; ++i)
    if (ptx::mbar_try_wait(bar, parity)) return true;
  return wait_slow(bar, parity, w.clocks, w.gave_up);
}
// the same for a whole warp: true if no lane gave up
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, const Waits& w) {
  return __all_sync(0xffffffffu, wait_on(bar, parity, w)) != 0;
}

__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, const OperandStaging& op) {
  return ((uint64_t)op.desc_hi << 32) | (((addr & 0x3FFFFu) >> 4) | (op.lbo_enc << 16));
}

// A barrier that orders nothing: a release would wait for the results' stores, some 0.9 us at a kernel's end.
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }

// ---------------------------------------------------------------- tensor-core instructions of exo_fused.h only
template <int CTA_GROUP>
__device__ __forceinline__ void umma_i8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  if constexpr (CTA_GROUP == 1)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
template <class Op, int CTA_GROUP>
__device__ __forceinline__ void umma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (Op::kInt8) umma_i8<CTA_GROUP>(d, a, b, idesc, accumulate);
  else ptx::umma_f16<CTA_GROUP>(d, a, b, idesc, accumulate);
}

// 32 bytes of a lane, a whole sector: what a warp's rows cost is the sectors they ask for.
__device__ __forceinline__ void ld_global_cg_v8(const void* at, uint32_t (&r)[8]) {
  asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "l"(at) : "memory");
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, int32_t z, int32_t w, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}

__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[32]) { ptx::tmem_ld_32x32(taddr, r); }
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                 "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr) : "memory");
}

template <class T, int U>
__device__ __forceinline__ void pack(const float (&v)[U], uint32_t (&w)[U / 2]) {
#pragma unroll
  for (int k = 0; k < U / 2; ++k) w[k] = T::pack(v[2 * k], v[2 * k + 1]);
}

// ---------------------------------------------------------------- a row's U values to memory
// `align`: a power of two up to 32 that divides the address of every unit.  n <= U values exist; the others are not written.
template <int U>
__device__ __forceinline__ void store_words(void* at, const uint32_t (&w)[U / 2], int n, int align) {
  char* const c = static_cast<char*>(at);
  if (n >= U && align >= 16) {
    if (U >= 16 && align >= 32) {
#pragma unroll
      for (int j = 0; j < U / 16; ++j) ptx::st_global_v8(c + 32 * j, &w[8 * j]);
    } else {
#pragma unroll
      for (int j = 0; j < U / 8; ++j) ptx::st_global_v4(c + 16 * j, w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (k < n) reinterpret_cast<uint16_t*>(c)[k] = (uint16_t)(w[k / 2] >> (16 * (k & 1)));
  }
}
template <class T, int U>
__device__ __forceinline__ void store16(void* at, const float (&v)[U], int n, int align) {
  uint32_t w[U / 2];
  pack<T, U>(v, w);
  store_words<U>(at, w, n, align);
}
template <int U>
__device__ __forceinline__ void store32(void* at, const float (&v)[U], int align) {   // align: 16 at least
  char* const c = static_cast<char*>(at);
  uint32_t w[U];
#pragma unroll
  for (int k = 0; k < U; ++k) w[k] = __float_as_uint(v[k]);
  if (align >= 32) {
#pragma unroll
    for (int j = 0; j < U / 8; ++j) ptx::st_global_v8(c + 32 * j, &w[8 * j]);
  } else {
#pragma unroll
    for (int j = 0; j < U / 4; ++j) ptx::st_global_v4(c + 16 * j, w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
  }
}

// Where a warp of the pair kernel puts its results, 32 columns of 16 bits at a time: into a buffer, from there by a TMA store.  The buffers'
// rows of 64 bytes are swizzled as the tensor maps say: 16-byte piece j of row r lies at j ^ (r / 2 % 4).
struct OutMaps {
  CUtensorMap m[3];
};
struct Out {
  const OutMaps* maps;    // NULL in the thin kernel, which stores rows only
  uint32_t buffers, turn;
  int32_t row0, rows;     // the warp's first row, and how many of its rows exist
  // N pieces of the lane's row, from piece `first` on
  template <int N>
  __device__ __forceinline__ void write(uint32_t at, uint32_t first, const uint32_t (&w)[4 * N]) {
    const uint32_t lane = ptx::lane_id(), row = at + lane * 64u, x = (lane >> 1) & 3u;
#pragma unroll
    for (uint32_t j = 0; j < (uint32_t)N; ++j) ptx::st_shared_v4(row + (((first + j) ^ x) << 4), w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
  }
  // one result at a time, two buffers in turn
  __device__ __forceinline__ void put(int map, int col, const uint32_t (&w)[16]) {
    const uint32_t at = buffers + turn * kOutBytes;
    if (ptx::elect_one()) ptx::bulk_wait_read<1>();   // the store before the last has read this buffer
    __syncwarp();
    write<4>(at, 0, w);
    ptx::fence_proxy_async_smem();
    __syncwarp();
    if (ptx::elect_one()) {
      ptx::tma_store_2d(&maps->m[map], col, row0, at);
      ptx::bulk_commit();
    }
    turn ^= 1u;
  }
  // Results whose rows start anywhere: a row's `n` elements of ES bytes (64 bytes of it are in the buffer) are stored by neighbouring lanes, in
  // pieces of what divides every row's address.  A row per lane would take 32 lines of memory for every instruction instead.
  template <int ES, int W>
  __device__ __forceinline__ void pieces(uint32_t at, char* dst, int64_t row_bytes, int n) {
    constexpr int PER = W / ES, LANES = 64 / W;   // elements of a piece, pieces of a row
    const int lane = (int)ptx::lane_id(), e = lane % LANES * PER;
    const uint32_t byte = (uint32_t)(e * ES);
    for (int r = lane / LANES; r < rows; r += 32 / LANES) {
      const uint32_t from = at + (uint32_t)r * 64u + ((((byte >> 4) ^ ((uint32_t)r >> 1)) & 3u) << 4) + (byte & 15u);
      char* const to = dst + (int64_t)r * row_bytes + byte;
      if (e + PER <= n) {
        if constexpr (W == 2) {
          uint16_t v;
          asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(from) : "memory");
          *reinterpret_cast<uint16_t*>(to) = v;
        } else if constexpr (W == 4) {
          uint32_t v;
          asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(from) : "memory");
          *reinterpret_cast<uint32_t*>(to) = v;
        } else {
          uint2 v;
          asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(from) : "memory");
          *reinterpret_cast<uint2*>(to) = v;
        }
      } else {
        for (int k = 0; k < n - e; ++k) {   // the end of a row inside a piece
          if constexpr (ES == 2) {
            uint16_t v;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(from + 2u * (uint32_t)k) : "memory");
            reinterpret_cast<uint16_t*>(to)[k] = v;
          } else {
            uint32_t v;
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(from + 4u * (uint32_t)k) : "memory");
            reinterpret_cast<uint32_t*>(to)[k] = v;
          }
        }
      }
    }
  }
  // dst: the first row's first element
  template <int ES>
  __device__ __forceinline__ void store_rows(int buffer, void* dst, int64_t row_bytes, int n, int align) {
    const uint32_t at = buffers + (uint32_t)buffer * kOutBytes;
    __syncwarp();
    if (align >= 8) pieces<ES, 8>(at, static_cast<char*>(dst), row_bytes, n);
    else if (ES == 4 || align >= 4) pieces<ES, 4>(at, static_cast<char*>(dst), row_bytes, n);
    else if constexpr (ES == 2) pieces<ES, 2>(at, static_cast<char*>(dst), row_bytes, n);
    __syncwarp();
  }
  // several results together, N * 8 columns at a time: open, piece each, and close behind the 32nd column or the last
  __device__ __forceinline__ void open() {
    if (ptx::elect_one()) ptx::bulk_wait_read<0>();
    __syncwarp();
  }
  template <int N>
  __device__ __forceinline__ void piece(int buffer, int col, const uint32_t (&w)[4 * N]) {
    write<N>(buffers + (uint32_t)buffer * kOutBytes, (uint32_t)(col >> 3) & 3u, w);
  }
  __device__ __forceinline__ void close(int results, int col) {
    ptx::fence_proxy_async_smem();
    __syncwarp();
    if (ptx::elect_one()) {
      for (int i = 0; i < results; ++i) ptx::tma_store_2d(&maps->m[i], col & ~31, row0, buffers + (uint32_t)i * kOutBytes);
      ptx::bulk_commit();
    }
  }
};
// The partial sums of a tile that the other CTAs of a cluster have left in this one's shared memory: per CTA and unit U columns (twice, for a
// gated product) of a word per lane.
struct Peers {
  uint32_t count, at, step;   // step: bytes between two CTAs' sums
};
template <bool INT, int U>
__device__ __forceinline__ void add_peers(const Peers& p, uint32_t offset, uint32_t (&v)[U]) {
  const uint32_t lane = ptx::lane_id();
  for (uint32_t i = 0; i < p.count; ++i) {   // in the order of K
    const uint32_t from = p.at + i * p.step + offset + lane * 4u;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      uint32_t w;
      asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(from + 128u * (uint32_t)k) : "memory");
      v[k] = INT ? v[k] + w : __float_as_uint(__uint_as_float(v[k]) + __uint_as_float(w));
    }
  }
}
template <int U>
__device__ __forceinline__ void give_to_peer(uint32_t cluster_at, const uint32_t (&v)[U]) {
  const uint32_t to = cluster_at + ptx::lane_id() * 4u;
#pragma unroll
  for (int k = 0; k < U; ++k) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to + 128u * (uint32_t)k), "r"(v[k]) : "memory");
}

// ---------------------------------------------------------------- the epilogue of one warp: 32 rows, `units` units of U columns
// tacc: the warp's lanes of the accumulator, at its first unit's column; release() hands the accumulator back after the last read.
// s: what Op::begin has fetched for the row and the first unit, before the accumulator was complete; a unit fetches for the next one.
template <class Op, int U, bool PEERS, class Release>
__device__ __forceinline__ void run_units(const typename Op::Params& o, typename Op::template State<U>& s, Out& out, uint32_t tacc, uint32_t gap, int row, bool row_ok, int col,
                                          int units, int N, int part, const Peers& peers, const Release& release) {
  constexpr uint32_t kUnitBytes = (Op::kGated ? 2 : 1) * U * 128;
  const int left = N > col ? (N - col + U - 1) / U : 0;
  if (units > left) units = left;
  if constexpr (Op::kTwice) {   // a first look at the columns
#pragma unroll 1
    for (int i = 0; i < units; ++i) {
      uint32_t v[U];
      tmem_ld(tacc + (uint32_t)(i * U), v);
      ptx::tmem_ld_wait();
      if constexpr (PEERS) add_peers<Op::kInt8, U>(peers, (uint32_t)i * kUnitBytes, v);
      Op::template look<U>(o, s, v, N - col - i * U);
    }
  }
  if (units == 0) release();
#pragma unroll 1
  for (int i = 0; i < units; ++i) {
    uint32_t v[U], v2[Op::kGated ? U : 1];
    tmem_ld(tacc + (uint32_t)(i * U), v);
    if constexpr (Op::kGated) tmem_ld(tacc + gap + (uint32_t)(i * U), v2);
    ptx::tmem_ld_wait();
    if (i + 1 == units) release();
    if constexpr (PEERS) {
      add_peers<Op::kInt8, U>(peers, (uint32_t)i * kUnitBytes, v);
      if constexpr (Op::kGated) add_peers<Op::kInt8, U>(peers, (uint32_t)i * kUnitBytes + U * 128, v2);
    }
    const int n = N - col - i * U;
    Op::template unit<U>(o, s, out, v, v2, row, row_ok, col + i * U, n < U ? n : U, i + 1 < units);
  }
  Op::end(o, s, row, row_ok, part);
}

// ---------------------------------------------------------------- pairs of CTAs, persistent
// Roles as in the library's plain product: warps 0 and 10 copy A and B, warp 1 issues the MMAs (CTA 0) and owns tensor memory, warps 2 to 9
// are the epilogue, two per lane quadrant, each of them half of the tile's columns.
template <class Op, bool B_MN>
__global__ void __launch_bounds__(kNumThreads, 1)
exo_fused_pair_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const __grid_constant__ OutMaps tm_out,
                      const __grid_constant__ CoreParams p, const __grid_constant__ typename Op::Params o) {
  constexpr int SUB_K = Op::kInt8 ? 128 : 64;          // elements of a k-block
  constexpr uint32_t TMEM_COLS = 512, ACC = 256;       // columns of both accumulators, and between them
  const int32_t width = p.width;                       // result columns of a tile
  const uint32_t b_rows = (uint32_t)(Op::kGated ? width : width / 2), stage_bytes = (uint32_t)kATileBytes + b_rows * 128u, stages = (uint32_t)p.stages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t stage0 = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u, out0 = stage0 + stages * stage_bytes, bar0 = out0 + kEpiWarps * (uint32_t)p.buffers * kOutBytes;
  auto full_bar = [&](uint32_t s) { return bar0 + 8u * s; };
  auto empty_bar = [&](uint32_t s) { return bar0 + 8u * (kPairMaxStages + s); };
  auto tfull_bar = [&](uint32_t a) { return bar0 + 8u * (2 * kPairMaxStages + a); };
  auto tempty_bar = [&](uint32_t a) { return bar0 + 8u * (2 * kPairMaxStages + 2 + a); };
  const uint32_t tmem_slot = bar0 + 8u * (2 * kPairMaxStages + 4);
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  const uint32_t rank = ptx::cluster_ctarank();
  const int64_t worker = blockIdx.x / 2, workers = gridDim.x / 2, tiles = raster_total(p.raster);
  const int32_t nkb = p.nkb;

  if (warp == 2) {
    if (lane == 0) {
      ptx::prefetch_tensormap(&tm_a);
      ptx::prefetch_tensormap(&tm_b);
    }
    for (uint32_t i = lane; i < 2u * kPairMaxStages + 4u; i += 32u) ptx::mbar_init(bar0 + 8u * i, i >= 2u * kPairMaxStages + 2u ? kEpiWarps * 2 : 1);
    ptx::fence_mbar_init();
  }
  if (warp == 1) {
    ptx::tmem_alloc<2>(tmem_slot, TMEM_COLS);
    ptx::tmem_relinquish<2>();
  }
  ptx::cluster_arrive();
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::cluster_wait();   // the peer's barriers and tensor memory exist before anything remote touches them
  ptx::tc_fence_after_sync();
  uint32_t tmem_base;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem_base) : "r"(tmem_slot) : "memory");
  bool ok = true;

  if (warp == 0 || warp == (uint32_t)kProducerBWarp) {
    const bool do_a = warp == 0;
    uint32_t s = 0, ph = 0;
    const uint32_t full0 = ptx::map_to_cta(full_bar(0), 0u);   // both CTAs' copies are counted on CTA 0's barrier
    ptx::grid_dependency_wait();
    bool skip = p.skip_copies != 0 && blockIdx.x == 0;
    for (int64_t t = worker; t < tiles && ok; t += workers) {
      const TileCoord tc = raster_decode(p.raster, t);
      const int32_t a0 = tc.m * 256 + (int32_t)rank * 128, b0 = tc.n * width + (int32_t)rank * p.b_split;
      for (int32_t kb = 0; kb < nkb; ++kb) {
        ok = wait_warp(empty_bar(s), ph ^ 1u, p.waits);
        if (!ok) break;
        if (ptx::elect_one()) {
          if (rank == 0 && do_a) ptx::mbar_arrive_expect_tx(full_bar(s), stage_bytes * 2);
          const uint32_t a_dst = stage0 + s * stage_bytes, b_dst = a_dst + kATileBytes, bar = full0 + 8u * s;
          if (skip) {
          } else if (do_a) {
            ptx::tma_load_2d_pair(a_dst, &tm_a, kb * SUB_K, a0, bar);
          } else if constexpr (!B_MN) {
            ptx::tma_load_2d_pair(b_dst, &tm_b, kb * SUB_K, b0, bar);
          } else {
            for (uint32_t b = 0; b < b_rows / 64; ++b) ptx::tma_load_2d_pair(b_dst + b * 8192u, &tm_b, b0 + 64 * (int32_t)b, kb * SUB_K, bar);
          }
        }
        skip = false;
        if (++s == stages) { s = 0; ph ^= 1u; }
      }
    }
    for (uint32_t i = 0; i < stages && ok; ++i) {   // no stage release may still be on its way to this CTA
      ok = wait_warp(empty_bar(s), ph ^ 1u, p.waits);
      if (++s == stages) { s = 0; ph ^= 1u; }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      ptx::grid_dependency_wait();
      uint32_t s = 0, ph = 0, acc = 0, acc_ph = 0;
      const uint32_t a_step = p.a.k_step_enc, b_step = p.b.k_step_enc, idesc = p.idesc;
      for (int64_t t = worker; t < tiles && ok; t += workers) {
        ok = wait_warp(tempty_bar(acc), acc_ph ^ 1u, p.waits);   // both CTAs' epilogues have read it
        if (!ok) break;
        ptx::tc_fence_after_sync();
        const uint32_t d = tmem_base + acc * ACC;
        for (int32_t kb = 0; kb < nkb; ++kb) {
          ok = wait_warp(full_bar(s), ph, p.waits);
          if (!ok) break;
          ptx::tc_fence_after_sync();
          const uint64_t a_desc = smem_desc(stage0 + s * stage_bytes, p.a), b_desc = smem_desc(stage0 + s * stage_bytes + kATileBytes, p.b);
          if (ptx::elect_one()) {
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k)   // 32 bytes of K each
              umma<Op, 2>(d, a_desc + k * a_step, b_desc + k * b_step, idesc, (kb > 0 || k > 0) ? 1u : 0u);
            ptx::umma_commit<2>(empty_bar(s), 3);
            if (kb == nkb - 1) ptx::umma_commit<2>(tfull_bar(acc), 3);
          }
          if (++s == stages) { s = 0; ph ^= 1u; }
        }
        if ((acc ^= 1u) == 0u) acc_ph ^= 1u;
      }
    }
  } else {
    ptx::grid_dependency_wait();
    if (warp == 2) ptx::grid_launch_dependents();   // (behind the wait: a kernel that starts now comes after all that this one waited for)
    const uint32_t quad = warp & 3u;
    const int32_t half = (int32_t)((warp - 2u) >> 2);
    const uint32_t tempty0 = ptx::map_to_cta(tempty_bar(0), 0u);
    // the tile's columns, 32 at a time: the first half of them, rounded up, is the first warp's of a lane quadrant
    constexpr int U = Op::kUnit, PER = 32 / U;
    const int32_t all = width / 32, skipped = (half ? (all + 1) / 2 : 0) * PER, units = (half ? all / 2 : (all + 1) / 2) * PER;
    Out out{&tm_out, out0 + (warp - 2u) * ((uint32_t)p.buffers * kOutBytes), 0u, 0, 0};
    uint32_t acc = 0, acc_ph = 0;
    for (int64_t t = worker; t < tiles; t += workers) {
      const TileCoord tc = raster_decode(p.raster, t);
      const int32_t row0 = tc.m * 256 + (int32_t)rank * 128 + (int32_t)quad * 32, row = row0 + (int32_t)lane;
      const int32_t col = tc.n * width + skipped * U;
      out.row0 = row0;
      out.rows = p.M - row0 < 32 ? p.M - row0 : 32;
      typename Op::template State<U> state;
      Op::template begin<U>(o, state, row, row < p.M, col, p.N);
      ok = wait_warp(tfull_bar(acc), acc_ph, p.waits);
      if (!ok) break;
      ptx::tc_fence_after_sync();
      // (Handed back only for a tile to come: an arrival that nobody waits for could reach a CTA that has gone.)
      const bool wanted = t + 2 * workers < tiles;
      auto release = [&]() {
        if (!wanted) return;
        ptx::tc_fence_before_sync();
        __syncwarp();
        if (ptx::elect_one()) ptx::mbar_arrive_cluster(tempty0 + 8u * acc);
      };
      if (row0 >= p.M) {
        release();
      } else {
        const uint32_t tacc = tmem_base + ((quad * 32u) << 16) + acc * ACC + (uint32_t)(skipped * U);
        run_units<Op, U, false>(o, state, out, tacc, (uint32_t)width, row, row < p.M, col, units, p.N, tc.n * 2 + half, Peers{}, release);
      }
      if ((acc ^= 1u) == 0u) acc_ph ^= 1u;
    }
    __syncwarp();
    if (ptx::elect_one()) ptx::bulk_wait_read<0>();   // the stores have read this CTA's shared memory
    __syncwarp();
  }

  if (!ok)
    for (int i = 0; i < 200; ++i) __nanosleep(1000);   // a wait was abandoned: copies and MMAs in flight land first
  ptx::tc_fence_before_sync();
  __syncthreads();
  // The peer's shared and tensor memory stay valid until both CTAs are done; every arrival and copy that reaches over has been waited for.
  cluster_arrive_relaxed();
  ptx::cluster_wait();
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc<2>(tmem_base, TMEM_COLS);
  }
}

// ---------------------------------------------------------------- a few rows: one tile per CTA
// A stage is `per_stage` k-blocks of the tile's rows of B (gate's and up's for a gated product) and of the a_rows rows of A, a copy each:
// issuing a copy takes a few hundred clocks, in which an SM's share of memory bandwidth is some 8 KB.  Up to 64 rows the MMAs have 64: what
// such an MMA takes is the reading of its operands from shared memory, mostly A's.  There a lane quadrant of the accumulator holds 16 rows.
// U: columns of an epilogue unit.
template <class Op, int U>
__global__ void __launch_bounds__(kThinThreads, 2)
exo_fused_thin_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_a_rest, const __grid_constant__ CUtensorMap tm_b,
                      const __grid_constant__ CUtensorMap tm_b_rest, const __grid_constant__ CoreParams p, const __grid_constant__ typename Op::Params o) {
  constexpr int SUB_K = Op::kInt8 ? 128 : 64;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t stage0 = (ptx::smem_u32(smem_raw) + kThinBarrierBytes + 1023u) & ~1023u, bar0 = stage0 - kThinBarrierBytes;
  auto full_bar = [&](uint32_t s) { return bar0 + 8u * s; };
  auto empty_bar = [&](uint32_t s) { return bar0 + 8u * (kThinMaxStages + s); };
  const uint32_t tfull_bar = bar0 + 8u * (2 * kThinMaxStages), tmem_slot = tfull_bar + 8u;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  const uint32_t width = (uint32_t)p.width, bn = Op::kGated ? 2u * width : width;
  const uint32_t b_bytes = bn * 128u, a_bytes = (uint32_t)p.a_rows * 128u, stages = (uint32_t)p.stages;   // b_bytes, a_bytes: of a k-block
  const uint32_t stage_bytes = (b_bytes + a_bytes) * (uint32_t)p.per_stage, a_at = b_bytes * (uint32_t)p.per_stage;
  uint32_t tmem_cols = 32;
  while (tmem_cols < bn) tmem_cols *= 2;
  const uint32_t split = (uint32_t)p.split, rank = split > 1 ? ptx::cluster_ctarank() : 0u, tile = blockIdx.x / split;
  const int32_t kb_first = (int32_t)((int64_t)p.nkb * rank / split), nkb = (int32_t)((int64_t)p.nkb * (rank + 1) / split);   // this CTA's k-blocks
  const int32_t whole = p.whole < nkb ? p.whole : nkb, per = p.per_stage, col0 = (int32_t)(tile * width);

  if (warp == 0) {
    if (lane == 0) {
      ptx::prefetch_tensormap(&tm_a);
      ptx::prefetch_tensormap(&tm_b);
    }
    for (uint32_t i = lane; i < 2u * kThinMaxStages + 1u; i += 32u) ptx::mbar_init(bar0 + 8u * i, 1);
    ptx::fence_mbar_init();
  }
  if (warp == 1) {
    ptx::tmem_alloc<1>(tmem_slot, tmem_cols);
    ptx::tmem_relinquish<1>();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  uint32_t tmem_base;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem_base) : "r"(tmem_slot) : "memory");
  bool ok = true;

  if (warp == 0) {
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();   // (behind the wait: a kernel that starts now comes after all that this one waited for)
    uint32_t s = 0, ph = 0;
    bool skip = p.skip_copies != 0 && blockIdx.x == 0;
    for (int32_t kb = kb_first; kb < nkb; kb += kb < whole ? (kb + per > whole ? whole - kb : per) : 1) {
      ok = wait_warp(empty_bar(s), ph ^ 1u, p.waits);
      if (!ok) break;
      if (ptx::elect_one()) {
        const uint32_t dst = stage0 + s * stage_bytes, bar = full_bar(s);
        if (kb < whole) {   // (blocks beyond the last whole one arrive as zeros, another CTA's are not used)
          ptx::mbar_arrive_expect_tx(bar, stage_bytes);
          if (!skip) {
            tma_load_4d(dst, &tm_b, 0, col0, 0, kb, bar);
            tma_load_4d(dst + a_at, &tm_a, 0, 0, 0, kb, bar);
          }
        } else {
          ptx::mbar_arrive_expect_tx(bar, b_bytes + a_bytes);
          if (!skip) {
            ptx::tma_load_3d(dst, &tm_b_rest, kb * SUB_K, col0, 0, bar);
            ptx::tma_load_3d(dst + a_at, &tm_a_rest, kb * SUB_K, 0, 0, bar);
          }
        }
      }
      skip = false;
      if (++s == stages) { s = 0; ph ^= 1u; }
    }
  } else if (warp == 1) {
    ptx::grid_dependency_wait();
    uint32_t s = 0, ph = 0;
    const uint32_t a_step = p.a.k_step_enc, b_step = p.b.k_step_enc, idesc = p.idesc;
    for (int32_t kb = kb_first; kb < nkb;) {
      const int32_t blocks = kb < whole ? (kb + per > whole ? whole - kb : per) : 1;
      ok = wait_warp(full_bar(s), ph, p.waits);
      if (!ok) break;
      ptx::tc_fence_after_sync();
      const uint64_t b_desc = smem_desc(stage0 + s * stage_bytes, p.b), a_desc = smem_desc(stage0 + s * stage_bytes + a_at, p.a);
      if (ptx::elect_one()) {
        for (int32_t j = 0; j < blocks; ++j) {
          const uint64_t a_j = a_desc + (uint32_t)j * (a_bytes >> 4), b_j = b_desc + (uint32_t)j * (b_bytes >> 4);
#pragma unroll
          for (uint32_t k = 0; k < 4; ++k) umma<Op, 1>(tmem_base, a_j + k * a_step, b_j + k * b_step, idesc, (kb > kb_first || j > 0 || k > 0) ? 1u : 0u);
        }
        ptx::umma_commit<1>(empty_bar(s), 1);
        if (kb + blocks == nkb) ptx::umma_commit<1>(tfull_bar, 1);
      }
      kb += blocks;
      if (++s == stages) { s = 0; ph ^= 1u; }
    }
    ok = ok && wait_warp(tfull_bar, 0u, p.waits);
  }
  const uint32_t quad = warp & 3u;
  const int32_t half = (int32_t)((warp - 2u) >> 2), row0 = (int32_t)quad * p.quad_rows, row = row0 + (int32_t)lane;
  const int32_t all = (int32_t)width / U, skipped = half ? (all + 1) / 2 : 0, mine = half ? all / 2 : (all + 1) / 2, col = col0 + skipped * U;
  const bool row_ok = (int32_t)lane < p.quad_rows && row < p.M;
  typename Op::template State<U> state;
  if (warp >= 2) {
    ptx::grid_dependency_wait();
    Op::template begin<U>(o, state, row, row_ok, col, p.N);
  }
  const bool all_ok = __syncthreads_and(ok) != 0;   // the epilogue's warps wait here for the accumulator, taking no issue slots
  const uint32_t tacc = tmem_base + ((quad * 32u) << 16) + (uint32_t)(skipped * U);
  // a warp's place for its sums in the first CTA of the cluster: [CTA][warp][unit]
  constexpr uint32_t kUnitBytes = (Op::kGated ? 2 : 1) * U * 128;
  const uint32_t most = (uint32_t)(all + 1) / 2u, peer_step = kEpiWarps * most * kUnitBytes;
  const uint32_t peer_at = stage0 + kEpiWarps * 2 * kOutBytes + (warp - 2u) * most * kUnitBytes;
  if (split > 1) {
    ptx::cluster_arrive();
    ptx::cluster_wait();   // the first CTA's ring is idle
    if (rank > 0 && warp >= 2 && all_ok && row0 < p.M) {
      ptx::tc_fence_after_sync();
      const uint32_t to = ptx::map_to_cta(peer_at + (rank - 1u) * peer_step, 0u);
      for (int32_t i = 0; i < mine; ++i) {
        uint32_t v[U];
        tmem_ld(tacc + (uint32_t)(i * U), v);
        ptx::tmem_ld_wait();
        give_to_peer<U>(to + (uint32_t)i * kUnitBytes, v);
        if constexpr (Op::kGated) {
          tmem_ld(tacc + width + (uint32_t)(i * U), v);
          ptx::tmem_ld_wait();
          give_to_peer<U>(to + (uint32_t)i * kUnitBytes + U * 128, v);
        }
      }
    }
    ptx::cluster_arrive();
    ptx::cluster_wait();   // the sums are there
  }
  if (rank == 0 && warp >= 2 && all_ok && row0 < p.M) {
    ptx::tc_fence_after_sync();
    const int32_t there = p.M - row0 < p.quad_rows ? p.M - row0 : p.quad_rows;
    Out out{nullptr, stage0 + (warp - 2u) * (2 * kOutBytes), 0u, row0, there};   // (the ring is idle: every MMA has read its stage)
    const Peers peers{split - 1u, peer_at, peer_step};
    run_units<Op, U, true>(o, state, out, tacc, width, row, row_ok, col, mine, p.N, (int)tile * 2 + half, peers, [] {});
  }
  if (!ok)
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc<1>(tmem_base, tmem_cols);
  }
}

}  // namespace fused
}  // namespace exo

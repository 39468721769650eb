// Tensor-core path of gated linear attention (bf16, d = 128): what its kernels share.
//
// Steps of 128 tokens.  Tiles are [2][128 rows][64 columns] bf16, 32 KiB, rows of 128 bytes with the 128-byte swizzle: as TMA brings q, k, v and do
// (rows = tokens), and as the state kernel writes the images of a state (rows = keys, columns = value channels).  Such a tile
// is an operand either way round: K-major over its columns, MN-major over its rows.  What threads make of P, dS and the scaled keys goes to
// tensor memory as A operand; what they write to shared memory for the tensor cores is the walk's tile of the state, and zeros behind the end of a sequence.
#pragma once

#include <cuda.h>

#include <type_traits>

#include "gla.cuh"
#include "../fp32_common.cuh"
#include "../tc_common.cuh"
#include "../tc_mma.cuh"

namespace ha_la {
namespace gla {

using namespace ptx;

constexpr int kComputeWarps = 16;

// The walk and the gradient kernel run 20 warps: 16 that compute, then producer, MMA issue, gates and one for dg or, in the walk, for o.  96 registers a
// thread are what an SM has for them; in the walk the last four hand some over, since a few bytes of spills cost 3% (with ~227 KiB of shared memory there is
// hardly any L1 left for the stack).  A launch that brought fewer than kRegs would wait for ever for them, so the launcher asks.
constexpr int kRoleThreads = 32 * (kComputeWarps + 4), kRegs = 96, kComputeRegs = 104, kOtherRegs = 64;
static_assert(32 * (kComputeWarps * kComputeRegs + 4 * kOtherRegs) <= kRoleThreads * kRegs && kRoleThreads * kRegs <= 65536, "register split");
__device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kComputeRegs)); }
__device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs)); }

constexpr double kLog2e = 1.4426950408889634;

// Log-gates of a step's tokens 4 lane .. 4 lane + 3 (one warp; 0 past the end), and cumulative, times log2 e, in 64 bits.
__device__ __forceinline__ float4 fetch_gates(const float* g, int HV, int j, Geom c, int lane) {
  float4 x;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int t = 4 * lane + e;
    (&x.x)[e] = t < c.L ? g[(size_t)(c.tok0 + t) * HV + j] : 0.f;
  }
  return x;
}
__device__ __forceinline__ void scan_gates(float4 x, int lane, double (&G)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) G[e] = gate((&x.x)[e]) * kLog2e;
  G[1] += G[0];
  G[2] += G[1];
  G[3] += G[2];
  double s = G[3];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double y = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += y;
  }
  const double before = s - G[3];
#pragma unroll
  for (int e = 0; e < 4; ++e) G[e] += before;
}

// What e^{G_i - G_j} is made of.  Off the diagonal blocks of 16 tokens it factors through the gates at the blocks' edges, all exponents
// <= 0: er[i] = 2^(G_i - R_I), ec[j] = 2^(R_{J+1} - G_j), bb[I][J] = 2^(R_I - R_{J+1}) (zero where J >= I), R_I = G of block I's first token.
// Near the diagonal it is taken of the difference, G = hi + lo: sums of closed gates leave a float no bits for what comes behind.
struct StepGates { float hi[kStep], lo[kStep], er[kStep], ec[kStep], bb[64]; };
struct LaneGates { float4 hi, lo, er, ec; float2 bb; };    // a lane's share of them

__device__ __forceinline__ LaneGates lane_gates(const double (&G)[4], int lane) {
  const double R = __shfl_sync(0xffffffffu, G[0], lane & ~3), R1 = __shfl_sync(0xffffffffu, G[0], min((lane & ~3) + 4, 31));
  LaneGates x;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    (&x.hi.x)[e] = (float)G[e];
    (&x.lo.x)[e] = (float)(G[e] - (double)(&x.hi.x)[e]);
    (&x.er.x)[e] = ex2((float)(G[e] - R));
    (&x.ec.x)[e] = ex2(fminf((float)(R1 - G[e]), 0.f));    // (the last block's, which nothing uses, would be of the wrong sign)
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int I = (2 * lane + e) >> 3, J = (2 * lane + e) & 7;
    const double rI = __shfl_sync(0xffffffffu, G[0], 4 * I), rJ = __shfl_sync(0xffffffffu, G[0], min(4 * J + 4, 31));
    (&x.bb.x)[e] = J < I ? ex2((float)(rI - rJ)) : 0.f;
  }
  return x;
}
__device__ __forceinline__ void put_gates(StepGates* s, const LaneGates& x, int lane) {
  reinterpret_cast<float4*>(s->hi)[lane] = x.hi;
  reinterpret_cast<float4*>(s->lo)[lane] = x.lo;
  reinterpret_cast<float4*>(s->er)[lane] = x.er;
  reinterpret_cast<float4*>(s->ec)[lane] = x.ec;
  reinterpret_cast<float2*>(s->bb)[lane] = x.bb;
}

// Rows L .. 127 of a tile to zero, by `n` threads: what lies behind a sequence may be NaN, and zero weights would not mask that.
__device__ __forceinline__ void clear_rows(uint8_t* tile, int L, int tid, int n) {
#pragma unroll 1
  for (int i = tid; i < (kStep - L) * 16; i += n)
    *reinterpret_cast<uint4*>(tile + (i & 1) * 16384 + (L + (i >> 4)) * 128 + ((i >> 1) & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
}

// Four lanes that hold four 16-byte pieces of a row each exchange them: v[i] becomes this lane's piece of the row of lane i of the four.  A warp's
// store of v[i] then covers 64 bytes of eight rows instead of 16 of thirty-two: a store takes the memory pipe a cycle for every 128-byte line it touches.
__device__ __forceinline__ void exchange(uint4& first, uint4& second, bool keep_second, int with) {
  const uint4 send = keep_second ? first : second;
  uint4 got;
  got.x = __shfl_xor_sync(0xffffffffu, send.x, with);
  got.y = __shfl_xor_sync(0xffffffffu, send.y, with);
  got.z = __shfl_xor_sync(0xffffffffu, send.z, with);
  got.w = __shfl_xor_sync(0xffffffffu, send.w, with);
  if (keep_second) first = got;
  else second = got;
}
__device__ __forceinline__ void exchange4(uint4 (&v)[4], int lane) {
  exchange(v[0], v[1], lane & 1, 1);
  exchange(v[2], v[3], lane & 1, 1);
  exchange(v[0], v[2], lane & 2, 2);
  exchange(v[1], v[3], lane & 2, 2);
}

// mbar_wait, with a look ahead of it (mbarrier.try_wait costs its caller some 150 cycles even when the phase is over) and its loop not unrolled: at some
// sixty places that is most of the gradient kernel's instructions, for which its warps waited a quarter of their time.  (As a function of its own it is
// shorter still, but what is live across a call does not all stay in registers, and there is hardly any L1 left for the stack.)
__device__ __forceinline__ void wait_for(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  if (mbar_test_wait(bar, parity)) return;
#pragma unroll 1
  for (uint32_t it = 0; it < kSpinLimit; ++it) {
    if (mbar_try_wait(bar, parity)) return;
    if ((it & 255u) == 255u && *abort_flag) return;
  }
  *abort_flag = 1;
}

// A tile's descriptors as B operand: over its columns (k index = columns, N = rows) or over its rows (k index = rows, N = columns), and
// what a step of 16 k adds.
__device__ __forceinline__ uint64_t desc_cols(uint32_t tile) { return smem_desc(tile, 16, 1024, kSwizzle128B); }
__device__ __forceinline__ uint64_t desc_rows(uint32_t tile) { return smem_desc(tile, 16384, 1024, kSwizzle128B); }
__device__ __forceinline__ uint32_t step_cols(int ks) { return (uint32_t)((ks >> 2) * 16384 + (ks & 3) * 32) >> 4; }
__device__ __forceinline__ uint32_t step_rows(int ks) { return (uint32_t)(ks * 2048) >> 4; }
constexpr uint32_t kIdCols = idesc_bf16(128, 128, false, false), kIdRows = idesc_bf16(128, 128, false, true);

// D (+)= A B over 128 k, one thread: both tiles over their columns; A over its columns and B over its rows; A in tensor memory.
__device__ __forceinline__ void mma_cols(uint32_t d, uint32_t a, uint32_t b, bool add) {
  const uint64_t da = desc_cols(a), db = desc_cols(b);
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) umma_ss(d, da + step_cols(ks), db + step_cols(ks), kIdCols, add || ks > 0);
}
__device__ __forceinline__ void mma_rows(uint32_t d, uint32_t a, uint32_t b, bool add) {
  const uint64_t da = desc_cols(a), db = desc_rows(b);
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) umma_ss(d, da + step_cols(ks), db + step_rows(ks), kIdRows, add || ks > 0);
}
// (`pitch`: columns from one 16 k of A to the next)
template <int pitch = 8>
__device__ __forceinline__ void mma_tmem_rows(uint32_t d, uint32_t a, uint32_t b, bool add) {
  const uint64_t db = desc_rows(b);
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) umma_ts(d, a + pitch * ks, db + step_rows(ks), kIdRows, add || ks > 0);
}

// Sequences as the state kernel walks them
struct Seqs {
  const int32_t *tok0, *len, *chunk0, *order;              // the plan kernel's tables, or NULL: equal-length rows
  int T_row, cps;
};

struct TcWork {
  uint8_t* image;                                          // backward: [slot][V-head] states in front of the steps as tiles, two bf16 pieces
  uint8_t* image_back;                                     // ... gradients behind them
  float *part, *part_back;                                 // [sequence][segment][V-head] fp32 states
  float *total, *total_back;                               // ... and decays
  float4* shared;                                          // backward: dq and dk that the gradient kernel's CTAs add up over a run's V-heads
  float* sums;                                             // ... and what their warps pass on for dg
};

struct TcCall {
  const Call* c;
  CUtensorMap q, k, v, d_o, o;                             // d_o: backward, o: forward
  Seqs seqs;
  TcWork w;
  int nseg;
};

int segments(const Problem& p, bool back);
size_t tc_bytes(const Problem& p, bool back, TcWork* tw, Work* w, void* base);
cudaError_t launch_tc_forward(const Call& c, PlanView plan, const TcWork& w, cudaStream_t stream);
cudaError_t launch_tc_backward(const Call& c, PlanView plan, const TcWork& w, cudaStream_t stream);
cudaError_t launch_tc_states(const TcCall& t, bool sums, cudaStream_t stream);
cudaError_t launch_tc_walk(const TcCall& t, cudaStream_t stream);
size_t local_back_bytes();
int heads_per_run(const Problem& p);
cudaError_t launch_tc_local_back(const TcCall& t, cudaStream_t stream);

}  // namespace gla

bool make_map_tile(CUtensorMap* m, const void* base, int T, int H);   // tc.cu

}  // namespace ha_la

// States of gated linear attention on the tensor cores.  For the gradients: the state in front of every step and the gradient of the
// state behind it, as bf16 tiles that their kernel takes as operands.  For sequences in segments, forward and backward: each segment's sum from zero.
//
//   forward   h  <- e^{G_L} h  + sum_j (e^{G_L - G_j} k_j) v_j^T                       in the order of the steps
//   reverse   dh <- e^{G_L} dh + scale e^{G_0} sum_i (e^{G_i - G_0} q_i) do_i^T        against it
// A CTA walks a run of a (sequence, V-head)'s steps, a whole state in registers (32 values of a key's row to each of 512 threads).  A step is one
// product, D[key][value channel] = A B: A the scaled keys, transposed to tensor memory (lane = key channel, columns = tokens) as two bf16
// pieces, 2^-17 of the value left out, so that the sum keeps the accuracy of fp32 (and nothing left out of the token next to the state, whose
// weight is one: with scale e^{G_0} in the weights dh0 had 1.5 times the error); B the values' tile as it is.  Nothing of the product waits for
// the state, so the next step's keys are scaled under this one's product, and the chain through the steps is one multiply-add.
//
// A step's image goes to shared memory as it will lie in memory, and one bulk copy of 64 KiB takes it out under the next step: four rows of 4096 tokens,
// 16 heads, 88 us, and 148 of the gradient kernel behind it; with stores of the warps (by way of shared memory, 64 bytes of eight rows at a time) 12 us more.
// What bounds it: the tiles and images through HBM when many CTAs run (128 KiB a step), else for images what an SM stores, and for sums the
// scaling warps' instructions (0.9 us a step).
// Few (sequence, V-head) pairs are cut into segments: gla_combine_kernel (simt.cu) chains the sums.
#include "tc.cuh"

namespace ha_la {
namespace gla {

namespace {

constexpr int kSlots = 5;                                  // tiles of two and a half steps
constexpr int kThreads = 32 * (kComputeWarps + 4);         // compute warps, producer, MMA issue, gates, images out
constexpr uint32_t OFF_IMAGE = kSlots * kTileBytes;        // a step's image on its way out, two pieces
constexpr uint32_t OFF_W = OFF_IMAGE + 2 * kTileBytes;     // [2] weights of a step's tokens, its decay, its sum's factor
constexpr uint32_t kWeightB = (kStep + 4) * 4;
constexpr uint32_t OFF_BAR = OFF_W + 2 * kWeightB;
constexpr int kBars = 2 * kSlots + 10;
constexpr uint32_t kSmem = OFF_BAR + kBars * 8 + 16;
static_assert(kSmem <= 227 * 1024, "shared memory budget");
constexpr uint32_t TM_A = 0, TM_D = 256;                   // operand: [2] (hi 64 | lo 64 columns); product: [2] 128 columns

struct StateParams {
  const float* g;
  Seqs seqs;
  const float* first[2];                                   // [direction] start states, [sequence][V-head], or NULL
  float* last;                                             // dh0, or NULL
  uint8_t* image[2];
  float *part[2], *total[2];
  int HK, HV, nseg;
  float scale;
  int32_t* status;
};

// IMAGES: the states as tiles, of two bf16 pieces each; without, the segments' sums from zero
template <bool IMAGES>
__global__ void __launch_bounds__(kThreads, 1)
gla_tc_state_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                    const __grid_constant__ CUtensorMap map_do, StateParams p) {
  extern __shared__ __align__(1024) uint8_t sm[];
  uint64_t* bar = reinterpret_cast<uint64_t*>(sm + OFF_BAR);
  uint64_t* full = bar;                                    // [kSlots] tiles: keys, values of a step, and so on
  uint64_t* empty = bar + kSlots;                          // [kSlots] keys scaled, product complete
  uint64_t* weights = bar + 2 * kSlots;                    // [2] of step c in set c % 2
  uint64_t* product = weights + 2;                         // [2]
  uint64_t* taken = product + 2;                           // the image has been read
  uint64_t* used = taken + 1;                              // [2] weights done with
  uint64_t* operand = used + 2;                            // [2] scaled keys in tensor memory
  uint64_t* put = operand + 2;                             // the image is there
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const bool rev = blockIdx.y;
  const int seg = blockIdx.x % p.nseg, nj = blockIdx.x / p.nseg, j = nj % p.HV, jq = j / (p.HV / p.HK);

  if (tid == 0) {
    for (int i = 0; i < kBars; ++i) mbar_init(&bar[i], &bar[i] >= used ? kComputeWarps : 1);
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 0) tmem_alloc(tmem_slot, 512);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // this CTA's steps: c = 0 .. count - 1 in the order it walks them
  int n = nj / p.HV, tok0 = n * p.seqs.T_row, len = p.seqs.T_row, slot0 = n * p.seqs.cps;
  if (p.seqs.tok0) {
    n = p.seqs.order[n];                                   // (the longest sequences first)
    tok0 = p.seqs.tok0[n];
    len = p.seqs.len[n];
    slot0 = p.seqs.chunk0[n];
  }
  const int steps = (len + kStep - 1) / kStep, per_seg = (steps + p.nseg - 1) / p.nseg;
  const int s0 = min(seg * per_seg, steps);
  const bool unused = !IMAGES && seg == (rev ? 0 : p.nseg - 1);   // (nothing starts from what the last segment adds)
  const int count = unused ? 0 : min(per_seg, steps - s0);
  auto index = [&](int c) { return s0 + (rev ? count - 1 - c : c); };   // step of the sequence
  auto geom = [&](int c) { return Geom{tok0 + index(c) * kStep, min(kStep, len - index(c) * kStep)}; };

  if (warp == kComputeWarps) {
    // ------------------------------------------------------------ tiles
    if (elect_one()) {
      int slot = 0;
      uint32_t round = 0;
      for (int x = 0; x < 2 * count; ++x) {
        if (round > 0) wait_for(&empty[slot], (round - 1) & 1, abort_flag);
        if (*abort_flag) break;
        mbar_expect_tx(&full[slot], kTileBytes);
        tma_load_4d(sm + slot * kTileBytes, x & 1 ? (rev ? &map_do : &map_v) : (rev ? &map_q : &map_k), &full[slot], 0, x & 1 ? j : jq, geom(x >> 1).tok0, 0);
        if (++slot == kSlots) { slot = 0; ++round; }
      }
    }
    __syncwarp();
  } else if (warp == kComputeWarps + 1) {
    // ------------------------------------------------------------ products
    if (elect_one()) {
      for (int c = 0; c < count; ++c) {
        const int b = c & 1, sk = 2 * c % kSlots, sv = (2 * c + 1) % kSlots;
        wait_for(&full[sv], ((2 * c + 1) / kSlots) & 1, abort_flag);
        wait_for(&operand[b], (c >> 1) & 1, abort_flag);
        mbar_arrive(&empty[sk]);
        tc_fence_after_sync();
        const uint32_t tile = smem_u32(sm + sv * kTileBytes);
        mma_tmem_rows(TM_D + 128 * b, TM_A + 128 * b, tile, false);
        mma_tmem_rows(TM_D + 128 * b, TM_A + 128 * b + 64, tile, true);
        umma_commit(&product[b]);
        umma_commit(&empty[sv]);
      }
    }
    __syncwarp();
  } else if (warp == kComputeWarps + 3) {
    // ------------------------------------------------------------ images out
    if (IMAGES && elect_one()) {
      for (int c = 0; c < count; ++c) {
        wait_for(put, c & 1, abort_flag);
        if (*abort_flag) break;
        bulk_store(p.image[rev] + ((size_t)(slot0 + index(c)) * p.HV + j) * (2 * kTileBytes), sm + OFF_IMAGE, 2 * kTileBytes);
        bulk_store_read();
        mbar_arrive(taken);
      }
      bulk_store_done();
    }
    __syncwarp();
  } else if (warp == kComputeWarps + 2) {
    // ------------------------------------------------------------ gates
    float4 raw = count > 0 ? fetch_gates(p.g, p.HV, j, geom(0), lane) : make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c = 0; c < count; ++c) {
      double G[4];
      scan_gates(raw, lane, G);
      if (c + 1 < count) raw = fetch_gates(p.g, p.HV, j, geom(c + 1), lane);
      if (c > 1) wait_for(&used[c & 1], ((c >> 1) - 1) & 1, abort_flag);
      __syncwarp();
      float* w = reinterpret_cast<float*>(sm + OFF_W + (c & 1) * kWeightB);
      const double GL = __shfl_sync(0xffffffffu, G[3], 31), G0 = __shfl_sync(0xffffffffu, G[0], 0);
      float4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) (&x.x)[e] = ex2((float)(rev ? G[e] - G0 : GL - G[e]));
      reinterpret_cast<float4*>(w)[lane] = x;
      if (lane == 0) {
        w[kStep] = ex2((float)GL);
        w[kStep + 1] = rev ? p.scale * ex2((float)G0) : 1.f;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&weights[c & 1]);
      __syncwarp();
    }
  } else {
    // ------------------------------------------------------------ scaling, state
    const int q = warp & 3, g = warp >> 2;                 // lanes 32 q .. (keys), columns: tokens of the operand or value channels 32 g ..
    const int key = 32 * q + lane;
    const uint32_t lanes = static_cast<uint32_t>(32 * q) << 16;
    float h[32];                                           // [key][32 g ..]
    const size_t unit = (size_t)n * p.HV + j, part = ((size_t)n * p.nseg + seg) * p.HV + j;
    const size_t at = (size_t)key * kStep + 32 * g;
    {
      const float* src = !IMAGES ? nullptr : p.nseg > 1 ? p.part[rev] + part * 16384 : p.first[rev] ? p.first[rev] + unit * 16384 : nullptr;
#pragma unroll
      for (int k = 0; k < 32; k += 4) {
        const float4 x = src ? *reinterpret_cast<const float4*>(src + at + k) : make_float4(0.f, 0.f, 0.f, 0.f);
        h[k] = x.x; h[k + 1] = x.y; h[k + 2] = x.z; h[k + 3] = x.w;
      }
    }
    float total = 1.f;
    auto scale_keys = [&](int c) {
      const int b = c & 1, L = geom(c).L, sk = 2 * c % kSlots, sv = (2 * c + 1) % kSlots;
      uint8_t* tile = sm + sk * kTileBytes;
      wait_for(&weights[b], (c >> 1) & 1, abort_flag);
      wait_for(&full[sk], (2 * c / kSlots) & 1, abort_flag);
      __syncwarp();
      if (L < kStep) {                                     // (rows behind the sequence may be NaN, which no weight of zero masks)
        wait_for(&full[sv], ((2 * c + 1) / kSlots) & 1, abort_flag);
        clear_rows(tile, L, tid, 32 * kComputeWarps);
        clear_rows(sm + sv * kTileBytes, L, tid, 32 * kComputeWarps);
        fence_proxy_async_smem();
        __syncwarp();
        asm volatile("bar.sync 1, %0;" ::"n"(32 * kComputeWarps) : "memory");
      }
      // 16 keys x 16 tokens at a time, transposed by ldmatrix; this lane's tokens are 2 (lane % 4), + 1 of each eight
      const float* w = reinterpret_cast<const float*>(sm + OFF_W + b * kWeightB) + 32 * g + 2 * (lane & 3);
      const uint32_t keys = smem_u32(tile) + (q >> 1) * 16384;
#pragma unroll
      for (int tk = 0; tk < 32; tk += 16) {
        const float2 f0 = *reinterpret_cast<const float2*>(w + tk), f1 = *reinterpret_cast<const float2*>(w + tk + 8);
#pragma unroll
        for (int hl = 0; hl < 2; ++hl) {
          uint32_t x[4], hi[4], lo[4];
          ldsm4t(x, keys + sw128_offset(32 * g + tk + (lane >> 4) * 8 + (lane & 7), (4 * q + 2 * hl + ((lane >> 3) & 1)) & 7));
#pragma unroll
          for (int e = 0; e < 4; ++e) split_bf16(mul2(unpack_bf16(x[e]), e < 2 ? f0 : f1), hi[e], lo[e]);
          const uint32_t at = TM_A + 128 * b + lanes + (static_cast<uint32_t>(16 * hl) << 16) + 16 * g + tk / 2;
          tmem_st_16x128b_x2(at, hi);
          tmem_st_16x128b_x2(at + 64, lo);
        }
      }
      tmem_st_wait();
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&operand[b]);
    };
    if (count > 0) scale_keys(0);
    for (int c = 0; c < count; ++c) {
      const int b = c & 1;
      if (c + 1 < count) scale_keys(c + 1);
      if constexpr (IMAGES) {
        if (c > 0) wait_for(taken, (c - 1) & 1, abort_flag);
        uint8_t* row = sm + OFF_IMAGE + (g >> 1) * 16384 + key * 128;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint4 hi, lo;
#pragma unroll
          for (int w = 0; w < 4; ++w) split_bf16(make_float2(h[8 * k + 2 * w], h[8 * k + 2 * w + 1]), (&hi.x)[w], (&lo.x)[w]);
          const int at = ((4 * (g & 1) + k) ^ (key & 7)) << 4;
          *reinterpret_cast<uint4*>(row + at) = hi;
          *reinterpret_cast<uint4*>(row + kTileBytes + at) = lo;
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(put);
      }
      const float2 f = *reinterpret_cast<const float2*>(sm + OFF_W + b * kWeightB + kStep * 4);
      wait_for(&product[b], (c >> 1) & 1, abort_flag);
      __syncwarp();
      tc_fence_after_sync();
      uint32_t d[32];
      tmem_ld32(TM_D + 128 * b + lanes + 32 * g, d);
      tmem_ld_wait();
#pragma unroll
      for (int k = 0; k < 32; k += 2) {
        const float2 x = fma2(make_float2(f.x, f.x), make_float2(h[k], h[k + 1]), mul2(make_float2(f.y, f.y), as_f2(d[k], d[k + 1])));
        h[k] = x.x;
        h[k + 1] = x.y;
      }
      total *= f.x;
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&used[b]);
    }
    float* dst = !IMAGES ? p.part[rev] + part * 16384 : rev && seg == 0 && p.last ? p.last + unit * 16384 : nullptr;
    if (dst) {
#pragma unroll
      for (int k = 0; k < 32; k += 4) *reinterpret_cast<float4*>(dst + at + k) = make_float4(h[k], h[k + 1], h[k + 2], h[k + 3]);
    }
    if (!IMAGES && tid == 0) p.total[rev][part] = total;
  }
  tc_fence_before_sync();
  __syncthreads();
  if (tid == 0 && *abort_flag) report_timeout(p.status);
  __syncthreads();
  if (warp == 0) tmem_dealloc(*tmem_slot, 512);
}

}  // namespace

cudaError_t launch_tc_states(const TcCall& t, bool sums, cudaStream_t stream) {
  const Call& c = *t.c;
  StateParams p = {};
  p.g = c.a.g; p.seqs = t.seqs;
  p.first[0] = c.a.h0; p.first[1] = c.a.dhT;
  p.last = c.a.dh0;
  p.image[0] = t.w.image; p.image[1] = t.w.image_back;
  p.part[0] = t.w.part; p.part[1] = t.w.part_back;
  p.total[0] = t.w.total; p.total[1] = t.w.total_back;
  p.HK = c.p.HK; p.HV = c.p.HV; p.nseg = t.nseg; p.scale = c.p.scale; p.status = c.a.status_word;
  const dim3 grid((unsigned)((size_t)c.p.N * c.p.HV * t.nseg), c.back ? 2 : 1);
  auto kernel = sums ? gla_tc_state_kernel<false> : gla_tc_state_kernel<true>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
  return e != cudaSuccess ? e : start(kernel, grid, kThreads, kSmem, stream, t.q, t.k, t.v, t.d_o, p);
}

}  // namespace gla
}  // namespace ha_la

// Gated linear attention forward on the tensor cores, in one walk: a CTA takes a run of a (sequence, V-head)'s steps in order, with the state in registers
// (32 values of a key's row to each of 512 threads), and leaves their outputs on the way.
//
//   o_i = scale [e^{G_i} (q_i h) + sum_{j <= i} e^{G_i - G_j} (q_i . k_j) v_j]        h <- e^{G_L} h + sum_j (e^{G_L - G_j} k_j) v_j^T
// Products of 128^3 a step: S = Q K^T; Q h, with h as a bf16 tile that the threads write to shared memory; P V, P = decay and mask of S, rounded to
// bf16 (o is rounded to bf16 anyway), added to Q h, whose rows have been scaled where they lie; and K' V, K' the scaled keys, transposed to
// tensor memory as two bf16 pieces, 2^-17 of the value left out, so that the state keeps the accuracy of fp32.  Tensor memory, four regions of
// 128 columns: S, and P over it (a warp writes 16 columns of P, 8 words, over the first half of the 16 accumulator columns that it alone has read);
// Q h + P V; K'; K' V.
//   threads   P(c)   scale Q h(c)   h(c + 1) and its tile   K'(c + 1)   o(c) out
//   products  ...    K' V(c)        P V(c)  S(c + 1)        Q h(c + 1)  K' V(c + 1)
// so each product runs under what the threads do next, and nothing but q, k, v and o goes through HBM.
// o goes out by a tensor store from where V lay, which is of no more use then; a last step of fewer tokens by plain stores.
// What bounds it: a step's phases, 2.6 to 2.9 us: 12000 instructions of a warp, four at a time, and looking at seven barriers, some 200 cycles each.
// HBM would allow 2.6 us with 128 CTAs (128 KiB a step): eight sequences of 7914 to 15654 tokens, 16 heads 365 us, 4.2 TB/s on the average.
// Outputs as a kernel of their own over stored states took 573 us; eight more warps for o 388, the state's and the outputs' phases in different
// warps 500 (seven warps to a scheduler, spills); 96 registers with 16 bytes of spills instead of 104 without + 10; o by exchanges between lanes and stores of
// 64 bytes a row 376; o from where Q lay 486 (that slot is wanted a step sooner).
// Few (sequence, V-head) pairs are cut into segments: gla_tc_state_kernel sums each from zero, gla_combine_kernel (simt.cu) chains the sums, and this
// kernel walks all segments from their true starts.
#include "tc.cuh"

namespace ha_la {
namespace gla {

namespace {

constexpr int kSlots = 6, kTiles = 3;                      // Q, K, V of two steps
struct WalkGates : StepGates { float el[kStep], total, pad[3]; };   // and e^{G_L - G_j}, e^{G_L}
constexpr uint32_t OFF_H = kSlots * kTileBytes;            // the state in front of the step as a tile
constexpr uint32_t OFF_G = OFF_H + kTileBytes;
constexpr uint32_t OFF_BAR = OFF_G + sizeof(WalkGates);
constexpr int kBars = 2 * kSlots + 10;
constexpr uint32_t kSmem = OFF_BAR + kBars * 8 + 16;
static_assert(kSmem <= 227 * 1024 && sizeof(WalkGates) % 16 == 0, "shared memory budget");
constexpr uint32_t TM_S = 0, TM_O = 128, TM_K = 256, TM_D = 384;

struct WalkParams {
  const float* g;
  Seqs seqs;
  const float* first;                                      // start states, [sequence][V-head], or NULL
  const float* part;                                       // ... of segments, [sequence][segment][V-head]
  float* last;
  void* o;
  int HK, HV, nseg;
  float scale;
  int32_t* status;
};

__global__ void __launch_bounds__(kRoleThreads, 1)
gla_tc_walk_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                   const __grid_constant__ CUtensorMap map_o, WalkParams p) {
  extern __shared__ __align__(1024) uint8_t sm[];
  WalkGates* s = reinterpret_cast<WalkGates*>(sm + OFF_G);
  uint64_t* bar = reinterpret_cast<uint64_t*>(sm + OFF_BAR);
  uint64_t *full = bar, *empty = bar + kSlots;             // [kSlots]
  uint64_t* one = bar + 2 * kSlots;                        // by one thread or by the tensor cores: gates; products complete: S, Q h, K' V, P V
  uint64_t *gates = one, *b_s = one + 1, *b_qh = one + 2, *b_d = one + 3, *b_o = one + 4;
  uint64_t* all = one + 5;                                 // by the compute warps: gates done with; P there and Q h scaled; K' there; O read and the state's tile written; o there
  uint64_t *g_free = all, *e_p = all + 1, *e_k = all + 2, *e_h = all + 3, *put = all + 4;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int seg = blockIdx.x % p.nseg, nj = blockIdx.x / p.nseg, j = nj % p.HV, jq = j / (p.HV / p.HK);

  if (tid == 0) {
    for (int i = 0; i < kBars; ++i) mbar_init(&bar[i], &bar[i] >= all ? kComputeWarps : 1);
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 0) tmem_alloc(tmem_slot, 512);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // this CTA's steps: c = 0 .. count - 1
  int n = nj / p.HV, tok0 = n * p.seqs.T_row, len = p.seqs.T_row;
  if (p.seqs.tok0) {
    n = p.seqs.order[n];                                   // (the longest sequences first)
    tok0 = p.seqs.tok0[n];
    len = p.seqs.len[n];
  }
  const int steps = (len + kStep - 1) / kStep, per_seg = (steps + p.nseg - 1) / p.nseg;
  const int s0 = min(seg * per_seg, steps), count = min(per_seg, steps - s0);
  auto geom = [&](int c) { return Geom{tok0 + (s0 + c) * kStep, min(kStep, len - (s0 + c) * kStep)}; };

  if (warp >= kComputeWarps) {
    give_registers();
    if (warp == kComputeWarps) {
      // ------------------------------------------------------------ tiles
      if (elect_one()) {
        int slot = 0;
        uint32_t round = 0;
        for (int c = 0; c < count && !*abort_flag; ++c) {
          const int t0 = geom(c).tok0;
#pragma unroll 1
          for (int t = 0; t < kTiles; ++t) {
            if (round > 0) wait_for(&empty[slot], (round - 1) & 1, abort_flag);
            if (*abort_flag) break;
            mbar_expect_tx(&full[slot], kTileBytes);
            tma_load_4d(sm + slot * kTileBytes, t == 0 ? &map_q : t == 1 ? &map_k : &map_v, &full[slot], 0, t == 2 ? j : jq, t0, 0);
            if (++slot == kSlots) { slot = 0; ++round; }
          }
        }
      }
      __syncwarp();
    } else if (warp == kComputeWarps + 1) {
      // ------------------------------------------------------------ products
      if (elect_one()) {
        const uint32_t h = smem_u32(sm + OFF_H);
        for (int c = -1; c < count; ++c) {
          const int at = kTiles * (c & 1), next = kTiles - at;
          const uint32_t ph = c & 1, fill = (c >> 1) & 1, fill_next = ((c + 1) >> 1) & 1;
          const uint32_t q = smem_u32(sm + at * kTileBytes), v = q + 2 * kTileBytes;
          auto wait = [&](uint64_t* b, uint32_t parity) {
            wait_for(b, parity, abort_flag);
            tc_fence_after_sync();
          };
          if (c >= 0) {
            wait(e_h, ph);
            mma_rows(TM_O, q, h, false);                     // Q h
            umma_commit(b_qh);
            umma_commit(&empty[at]);
            umma_commit(&empty[at + 1]);                   // (K: K' is there, S was complete)
            wait(&full[at + 2], fill);
            wait(e_k, ph);
            mma_tmem_rows(TM_D, TM_K, v, false);             // K' V
            mma_tmem_rows(TM_D, TM_K + 64, v, true);
            umma_commit(b_d);
            wait(e_p, ph);
            mma_tmem_rows<16>(TM_O, TM_S, v, true);          // + P V
            umma_commit(b_o);
          }
          if (c + 1 < count) {
            wait(&full[next], fill_next);
            wait(&full[next + 1], fill_next);
            mma_cols(TM_S, smem_u32(sm + next * kTileBytes), smem_u32(sm + (next + 1) * kTileBytes), false);
            umma_commit(b_s);
          }
        }
      }
      __syncwarp();
    } else if (warp == kComputeWarps + 2) {
      // ------------------------------------------------------------ gates
      float4 raw = count > 0 ? fetch_gates(p.g, p.HV, j, geom(0), lane) : make_float4(0.f, 0.f, 0.f, 0.f);
      for (int c = 0; c < count; ++c) {
        double G[4];
        scan_gates(raw, lane, G);
        if (c + 1 < count) raw = fetch_gates(p.g, p.HV, j, geom(c + 1), lane);
        const LaneGates x = lane_gates(G, lane);
        const double GL = __shfl_sync(0xffffffffu, G[3], 31);
        float4 el;
#pragma unroll
        for (int e = 0; e < 4; ++e) (&el.x)[e] = ex2((float)(GL - G[e]));
        if (c > 0) wait_for(g_free, (c - 1) & 1, abort_flag);
        __syncwarp();
        put_gates(s, x, lane);
        reinterpret_cast<float4*>(s->el)[lane] = el;
        if (lane == 0) s->total = ex2((float)GL);
        __syncwarp();
        if (lane == 0) mbar_arrive(gates);
        __syncwarp();
      }
    } else {
      // ------------------------------------------------------------ outputs, out of where V was
#pragma unroll 1
      for (int c = 0; c < count; ++c) {
        wait_for(put, c & 1, abort_flag);
        if (__any_sync(0xffffffffu, *abort_flag)) break;
        const Geom at = geom(c);
        const uint8_t* tile = sm + (kTiles * (c & 1) + 2) * kTileBytes;
        if (at.L == kStep) {
          if (lane == 0) {
            tma_store_4d(&map_o, tile, 0, j, at.tok0, 0);
            bulk_store_read();
          }
        } else {                                           // (not over the next sequence's rows)
          uint4* dst = reinterpret_cast<uint4*>(p.o) + ((size_t)at.tok0 * p.HV + j) * 16;
#pragma unroll 4
          for (int x = lane; x < at.L * 16; x += 32)
            dst[(size_t)(x >> 4) * p.HV * 16 + (x & 15)] = *reinterpret_cast<const uint4*>(tile + (x & 8) * 2048 + (x >> 4) * 128 + (((x ^ (x >> 4)) & 7) << 4));
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&empty[kTiles * (c & 1) + 2]);
        __syncwarp();
      }
      if (lane == 0) bulk_store_done();
      __syncwarp();
    }
  } else {
    take_registers();
    // ------------------------------------------------------------ decay and mask, state, scaled keys, outputs
    const int q = warp & 3, g = warp >> 2, i = 32 * q + lane;     // row i (token, key) of tensor memory; columns 32 g ..
    const uint32_t lanes = static_cast<uint32_t>(32 * q) << 16, slice = lanes + 32 * g;
    auto arrive = [&](uint64_t* b) {
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(b);
    };
    auto wait = [&](uint64_t* b, uint32_t parity) {
      wait_for(b, parity, abort_flag);
      __syncwarp();
      tc_fence_after_sync();
    };
    float h[32];                                           // [key][32 g ..]
    const size_t unit = (size_t)n * p.HV + j;
    const size_t at_state = (size_t)i * kStep + 32 * g;
    {
      const float* src = p.nseg > 1 ? p.part + (((size_t)n * p.nseg + seg) * p.HV + j) * 16384 : p.first ? p.first + unit * 16384 : nullptr;
#pragma unroll
      for (int k = 0; k < 32; k += 4) {
        const float4 x = src ? *reinterpret_cast<const float4*>(src + at_state + k) : make_float4(0.f, 0.f, 0.f, 0.f);
        h[k] = x.x; h[k + 1] = x.y; h[k + 2] = x.z; h[k + 3] = x.w;
      }
    }
#pragma unroll 1
    for (int c = -1; c < count; ++c) {
      const uint32_t ph = c & 1;
      if (c >= 0) {
        // ---- P, 16 columns at a time: blocks 0 .. 2 q + 1 of the quarter's rows, zeros behind
        const float hi = s->hi[i], lo = s->lo[i], total = s->total;
        wait(b_s, ph);
#pragma unroll
        for (int b = g; b < 8; b += 4) {
          const uint32_t at = TM_S + lanes + 16 * b;
          uint32_t w[8] = {};
          if (b < 2 * q + 2) {
            uint32_t r[16];
            tmem_ld16(at, r);
            float2 dec[8];
            if (b >> 1 != q) {
              const float f = s->er[i] * s->bb[8 * (i >> 4) + b];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float4 e = *reinterpret_cast<const float4*>(&s->ec[16 * b + 4 * k]);
                dec[2 * k] = mul2(make_float2(f, f), make_float2(e.x, e.y));
                dec[2 * k + 1] = mul2(make_float2(f, f), make_float2(e.z, e.w));
              }
            } else {
              const int to = i - 16 * b;                   // the row's own column
#pragma unroll
              for (int k = 0; k < 16; k += 4) {
                const float4 x = *reinterpret_cast<const float4*>(&s->hi[16 * b + k]), y = *reinterpret_cast<const float4*>(&s->lo[16 * b + k]);
#pragma unroll
                for (int e = 0; e < 4; ++e) (&dec[(k + e) / 2].x)[e & 1] = k + e <= to ? ex2((hi - (&x.x)[e]) + (lo - (&y.x)[e])) : 0.f;
              }
              tmem_ld_wait();
#pragma unroll
              for (int k = 0; k < 16; ++k) r[k] = k <= to ? r[k] : 0u;   // (S of rows behind the sequence may be NaN)
            }
            tmem_ld_wait();
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = pack_bf16(mul2(dec[k], as_f2(r[2 * k], r[2 * k + 1])));
          }
          tmem_st8(at, w);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(g_free);
        // ---- Q h times e^{G_i}
        const float eg = ex2(hi + lo);
        wait(b_qh, ph);
#pragma unroll
        for (int k = 0; k < 32; k += 16) {
          uint32_t r[16];
          tmem_ld16(TM_O + slice + k, r);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const float2 x = mul2(make_float2(eg, eg), as_f2(r[e], r[e + 1]));
            r[e] = __float_as_uint(x.x);
            r[e + 1] = __float_as_uint(x.y);
          }
          tmem_st16(TM_O + slice + k, r);
        }
        tmem_st_wait();
        arrive(e_p);
        // ---- state behind the step
        wait(b_d, ph);
#pragma unroll
        for (int k = 0; k < 32; k += 16) {
          uint32_t d[16];
          tmem_ld16(TM_D + slice + k, d);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const float2 x = fma2(make_float2(total, total), make_float2(h[k + e], h[k + e + 1]), as_f2(d[e], d[e + 1]));
            h[k + e] = x.x;
            h[k + e + 1] = x.y;
          }
        }
      }
      if (c + 1 < count) {
        // ---- its tile (Q h of this step is complete); scaled keys of the next step
        uint8_t* row = sm + OFF_H + (g >> 1) * 16384 + i * 128;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint4 x;
#pragma unroll
          for (int w = 0; w < 4; ++w) (&x.x)[w] = pack_bf16(make_float2(h[8 * k + 2 * w], h[8 * k + 2 * w + 1]));
          *reinterpret_cast<uint4*>(row + (((4 * (g & 1) + k) ^ (i & 7)) << 4)) = x;
        }
        fence_proxy_async_smem();
        const int slot = kTiles * ((c + 1) & 1) + 1, L = geom(c + 1).L;
        const uint32_t fill = ((c + 1) >> 1) & 1;
        uint8_t* tile = sm + slot * kTileBytes;
        wait_for(gates, (c + 1) & 1, abort_flag);
        wait_for(&full[slot], fill, abort_flag);
        __syncwarp();
        if (L < kStep) {                                   // (rows behind the sequence may be NaN, which no weight of zero masks)
          wait_for(&full[slot + 1], fill, abort_flag);
          clear_rows(tile, L, tid, 32 * kComputeWarps);
          clear_rows(tile + kTileBytes, L, tid, 32 * kComputeWarps);
          fence_proxy_async_smem();
          __syncwarp();
          asm volatile("bar.sync 1, %0;" ::"n"(32 * kComputeWarps) : "memory");
        }
        // 16 keys x 16 tokens at a time, transposed by ldmatrix; this lane's tokens are 2 (lane % 4), + 1 of each eight
        const float* w = s->el + 32 * g + 2 * (lane & 3);
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
            const uint32_t at = TM_K + lanes + (static_cast<uint32_t>(16 * hl) << 16) + 16 * g + tk / 2;
            tmem_st_16x128b_x2(at, hi);
            tmem_st_16x128b_x2(at + 64, lo);
          }
        }
        tmem_st_wait();
        arrive(e_k);
      }
      uint4 o[4] = {};
      if (c >= 0) {
        wait(b_o, ph);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          uint32_t r[16];
          tmem_ld16(TM_O + slice + 16 * k, r);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 8; ++e)
            (&o[2 * k + (e >> 2)].x)[e & 3] = pack_bf16(mul2(make_float2(p.scale, p.scale), as_f2(r[2 * e], r[2 * e + 1])));
        }
      }
      if (c + 1 < count) arrive(e_h);
      if (c >= 0) {
        uint8_t* row = sm + (kTiles * (c & 1) + 2) * kTileBytes + (g >> 1) * 16384 + i * 128;   // (P V is complete, and V of no more use)
#pragma unroll
        for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4*>(row + (((4 * (g & 1) + k) ^ (i & 7)) << 4)) = o[k];
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(put);
      }
    }
    float* dst = seg == p.nseg - 1 && p.last ? p.last + unit * 16384 : nullptr;
    if (dst) {
#pragma unroll
      for (int k = 0; k < 32; k += 4) *reinterpret_cast<float4*>(dst + at_state + k) = make_float4(h[k], h[k + 1], h[k + 2], h[k + 3]);
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (tid == 0 && *abort_flag) report_timeout(p.status);
  __syncthreads();
  if (warp == 0) tmem_dealloc(*tmem_slot, 512);
}

}  // namespace

cudaError_t launch_tc_walk(const TcCall& t, cudaStream_t stream) {
  const Call& c = *t.c;
  WalkParams p;
  p.g = c.a.g; p.seqs = t.seqs; p.first = c.a.h0; p.part = t.w.part; p.last = c.a.hT; p.o = c.a.o;
  p.HK = c.p.HK; p.HV = c.p.HV; p.nseg = t.nseg; p.scale = c.p.scale; p.status = c.a.status_word;
  cudaFuncAttributes has;
  cudaError_t e = cudaFuncGetAttributes(&has, gla_tc_walk_kernel);
  if (e == cudaSuccess && has.numRegs < kRegs) e = cudaErrorInvalidKernelImage;
  if (e == cudaSuccess) e = cudaFuncSetAttribute(gla_tc_walk_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
  const unsigned ctas = (unsigned)((size_t)c.p.N * c.p.HV * t.nseg);
  return e != cudaSuccess ? e : start(gla_tc_walk_kernel, dim3(ctas), kRoleThreads, kSmem, stream, t.q, t.k, t.v, t.o, p);
}

}  // namespace gla
}  // namespace ha_la

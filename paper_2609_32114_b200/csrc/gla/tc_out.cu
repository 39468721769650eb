// Outputs of gated linear attention on the tensor cores, step by step and independent of one another once the states are there.
//
//   o_i = scale [e^{G_i} (q_i h) + sum_{j <= i} e^{G_i - G_j} (q_i . k_j) v_j]
// A persistent CTA per SM takes (step, V-head) units.  Per unit three products of 128^3: S = Q K^T and Q h with both operands in shared memory (h as the
// image that the state kernel left), then P V with P = decay and mask of S, rounded to bf16 (o is rounded to bf16 anyway), in tensor memory.
// Tiles come through a ring of six 32-KiB slots in the order Q, K, h, V, so that the next unit's arrive under this one's work.
// What bounds it: 160 KiB a unit from L2 or HBM; a unit's dependent phases (a product ~700 cycles, P ~600, the store of o ~600) stay below that.
#include "tc.cuh"

namespace ha_la {
namespace gla {

namespace {

constexpr int kSlots = 6, kTiles = 4;                      // Q, K, h, V
constexpr int kThreads = 32 * (kComputeWarps + 3);
constexpr uint32_t OFF_G = kSlots * kTileBytes;            // [2] gates
constexpr uint32_t OFF_BAR = OFF_G + 2 * sizeof(StepGates);
constexpr int kBars = 2 * kSlots + 7;
constexpr uint32_t kSmem = OFF_BAR + kBars * 8 + 16;
static_assert(kSmem <= 227 * 1024 && OFF_G % 16 == 0 && sizeof(StepGates) % 16 == 0, "shared memory budget");
constexpr uint32_t TM_S = 0, TM_O1 = 128, TM_O2 = 256, TM_P = 384;

struct OutParams {
  const float* g;
  Chunks chunks;
  const uint8_t* image;
  void* o;
  int HK, HV;
  float scale;
  long long units;
  int32_t* status;
};

__global__ void __launch_bounds__(kThreads, 1)
gla_tc_out_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, OutParams p) {
  extern __shared__ __align__(1024) uint8_t sm[];
  uint64_t* bar = reinterpret_cast<uint64_t*>(sm + OFF_BAR);
  uint64_t* full = bar;                                    // [kSlots]
  uint64_t* empty = bar + kSlots;
  uint64_t* gates = bar + 2 * kSlots;                      // [2] of unit u in set u % 2
  uint64_t* used = gates + 2;                              // [2] ... done with: the unit's outputs are out of tensor memory too
  uint64_t* made_s = used + 2;
  uint64_t* made_p = made_s + 1;
  uint64_t* made_o = made_p + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < kBars; ++i) mbar_init(&bar[i], &bar[i] == used || &bar[i] == used + 1 || &bar[i] == made_p ? kComputeWarps : 1);
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 0) tmem_alloc(tmem_slot, 512);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  struct Unit { Geom c; int j; size_t sj; };               // sj: slot x V-heads + V-head; L = 0: no unit (a packed batch's unused slots come last)
  auto unit = [&](int u) {
    const long long i = blockIdx.x + (long long)u * gridDim.x;
    Unit x{{0, 0}, 0, 0};
    if (i >= p.units) return x;
    const int slot = (int)((unsigned)i / (unsigned)p.HV);
    x.j = (int)i - slot * p.HV;
    x.sj = (size_t)i;
    x.c = geom_of(p.chunks, slot);
    return x;
  };
  const int R = p.HV / p.HK;

  if (warp == kComputeWarps) {
    // ------------------------------------------------------------ tiles
    if (elect_one()) {
      int slot = 0;
      uint32_t round = 0;
      auto next = [&]() {                                  // the ring's next slot, free
        if (round > 0) wait_for(&empty[slot], (round - 1) & 1, abort_flag);
        return !*abort_flag;
      };
      auto done = [&]() { if (++slot == kSlots) { slot = 0; ++round; } };
      Unit x = unit(0);
      for (int u = 0; x.c.L > 0 && !*abort_flag; ++u) {
        const Unit after = unit(u + 1);
        for (int t = 0; t < kTiles; ++t) {
          if (!next()) break;
          uint8_t* dst = sm + slot * kTileBytes;
          mbar_expect_tx(&full[slot], kTileBytes);
          if (t == 2) bulk_load(dst, p.image + x.sj * kTileBytes, kTileBytes, &full[slot]);
          else tma_load_4d(dst, t == 0 ? &map_q : t == 1 ? &map_k : &map_v, &full[slot], 0, t == 3 ? x.j : x.j / R, x.c.tok0, 0);
          done();
        }
        x = after;
      }
    }
    __syncwarp();
  } else if (warp == kComputeWarps + 1) {
    // ------------------------------------------------------------ products
    if (elect_one()) {
      Unit x = unit(0);
      for (int u = 0; x.c.L > 0; ++u) {
        const Unit after = unit(u + 1);                    // (its look-ups under the waits, here and below)
        int s[kTiles];
        uint32_t ph[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          s[t] = (kTiles * u + t) % kSlots;
          ph[t] = ((kTiles * u + t) / kSlots) & 1;
        }
        auto tile = [&](int t) { return smem_u32(sm + s[t] * kTileBytes); };
        wait_for(&full[s[0]], ph[0], abort_flag);
        wait_for(&full[s[1]], ph[1], abort_flag);
        tc_fence_after_sync();
        mma_cols(TM_S, tile(0), tile(1), false);           // (the unit before has read its S: its P was made)
        umma_commit(made_s);
        umma_commit(&empty[s[1]]);
        wait_for(&full[s[2]], ph[2], abort_flag);
        if (u > 0) wait_for(&used[(u - 1) & 1], ((u - 1) >> 1) & 1, abort_flag);
        tc_fence_after_sync();
        mma_rows(TM_O1, tile(0), tile(2), false);
        umma_commit(&empty[s[0]]);
        umma_commit(&empty[s[2]]);
        wait_for(&full[s[3]], ph[3], abort_flag);
        wait_for(made_p, u & 1, abort_flag);
        tc_fence_after_sync();
        mma_tmem_rows(TM_O2, TM_P, tile(3), false);
        umma_commit(made_o);
        umma_commit(&empty[s[3]]);
        x = after;
      }
    }
    __syncwarp();
  } else if (warp == kComputeWarps + 2) {
    // ------------------------------------------------------------ gates
    Unit x = unit(0);
    float4 raw = fetch_gates(p.g, p.HV, x.j, x.c, lane);
    for (int u = 0; x.c.L > 0; ++u) {
      double G[4];
      scan_gates(raw, lane, G);
      x = unit(u + 1);
      raw = fetch_gates(p.g, p.HV, x.j, x.c, lane);        // (nothing where there is no unit)
      if (u > 1) wait_for(&used[u & 1], ((u >> 1) - 1) & 1, abort_flag);
      __syncwarp();
      fill_gates(reinterpret_cast<StepGates*>(sm + OFF_G) + (u & 1), G, lane);
      __syncwarp();
      if (lane == 0) mbar_arrive(&gates[u & 1]);
      __syncwarp();
    }
  } else {
    // ------------------------------------------------------------ decay and mask, outputs
    const int q = warp & 3, g = warp >> 2, i = 32 * q + lane;     // row i, columns 32 g ..
    const uint32_t lanes = static_cast<uint32_t>(32 * q) << 16;
    if (g > q) {                                           // above the diagonal: zeros, once
      const uint32_t z[16] = {};
      tmem_st16(TM_P + lanes + 16 * g, z);
      tmem_st_wait();
    }
    Unit x = unit(0);
    for (int u = 0; x.c.L > 0; ++u) {
      const Unit after = unit(u + 1);
      const StepGates* s = reinterpret_cast<const StepGates*>(sm + OFF_G) + (u & 1);
      wait_for(&gates[u & 1], (u >> 1) & 1, abort_flag);
      if (x.c.L < kStep) {                                 // (rows behind the sequence: their zero in P is not enough for NaN)
        const int sv = (kTiles * u + 3) % kSlots;
        wait_for(&full[sv], ((kTiles * u + 3) / kSlots) & 1, abort_flag);
        clear_rows(sm + sv * kTileBytes, x.c.L, tid, 32 * kComputeWarps);
        fence_proxy_async_smem();
      }
      wait_for(made_s, u & 1, abort_flag);
      __syncwarp();
      tc_fence_after_sync();
      if (g <= q) {
        uint32_t r[32], w[16];
        tmem_ld32(TM_S + lanes + 32 * g, r);
        tmem_ld_wait();
        if (g < q) {
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const float f = s->er[i] * s->bb[8 * (i >> 4) + 2 * g + b];
#pragma unroll
            for (int k = 0; k < 16; k += 4) {
              const float4 e = *reinterpret_cast<const float4*>(&s->ec[32 * g + 16 * b + k]);
              const int at = 16 * b + k;
              w[at / 2] = pack_bf16(__uint_as_float(r[at]) * (f * e.x), __uint_as_float(r[at + 1]) * (f * e.y));
              w[at / 2 + 1] = pack_bf16(__uint_as_float(r[at + 2]) * (f * e.z), __uint_as_float(r[at + 3]) * (f * e.w));
            }
          }
        } else {
          const float hi = s->hi[i], lo = s->lo[i];
#pragma unroll
          for (int k = 0; k < 32; k += 4) {
            const float4 a = *reinterpret_cast<const float4*>(&s->hi[32 * g + k]), b = *reinterpret_cast<const float4*>(&s->lo[32 * g + k]);
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              v[e] = k + e <= lane ? __uint_as_float(r[k + e]) * ex2((hi - (&a.x)[e]) + (lo - (&b.x)[e])) : 0.f;
            w[k / 2] = pack_bf16(v[0], v[1]);
            w[k / 2 + 1] = pack_bf16(v[2], v[3]);
          }
        }
        tmem_st16(TM_P + lanes + 16 * g, w);
        tmem_st_wait();
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(made_p);
      const float eg = p.scale * s->eg[i];
      wait_for(made_o, u & 1, abort_flag);
      __syncwarp();
      tc_fence_after_sync();
      uint32_t a[32], b[32];
      tmem_ld32(TM_O1 + lanes + 32 * g, a);
      tmem_ld32(TM_O2 + lanes + 32 * g, b);
      tmem_ld_wait();
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&used[u & 1]);
      auto val = [&](int k) { return fmaf(eg, __uint_as_float(a[k]), p.scale * __uint_as_float(b[k])); };
      uint4 o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        o[k] = make_uint4(pack_bf16(val(8 * k), val(8 * k + 1)), pack_bf16(val(8 * k + 2), val(8 * k + 3)),
                          pack_bf16(val(8 * k + 4), val(8 * k + 5)), pack_bf16(val(8 * k + 6), val(8 * k + 7)));
      exchange4(o, lane);
      const int row = 32 * q + (lane & ~3);
      __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.o) + ((size_t)(x.c.tok0 + row) * p.HV + x.j) * 128 + 32 * g + 8 * (lane & 3);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (row + k < x.c.L) *reinterpret_cast<uint4*>(dst + (size_t)k * p.HV * 128) = o[k];
      x = after;
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (tid == 0 && *abort_flag) report_timeout(p.status);
  __syncthreads();
  if (warp == 0) tmem_dealloc(*tmem_slot, 512);
}

}  // namespace

cudaError_t launch_tc_out(const TcCall& t, cudaStream_t stream) {
  const Call& c = *t.c;
  OutParams p;
  p.g = c.a.g; p.chunks = c.chunks; p.image = t.w.image; p.o = c.a.o;
  p.HK = c.p.HK; p.HV = c.p.HV; p.scale = c.p.scale; p.status = c.a.status_word;
  p.units = (long long)c.p.max_chunks * c.p.HV;
  if (p.units == 0) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(gla_tc_out_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
  const unsigned grid = (unsigned)(p.units < sm_count() ? p.units : sm_count());
  return e != cudaSuccess ? e : start(gla_tc_out_kernel, dim3(grid), kThreads, kSmem, stream, t.q, t.k, t.v, p);
}

}  // namespace gla
}  // namespace ha_la

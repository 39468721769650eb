// Gradients of gated linear attention on the tensor cores, step by step and independent of one another once the states in front of the steps and the
// gradients behind them are there (gla.cuh has the formulas).
//
// A persistent CTA per SM takes (step, V-head) units: sixteen products of 128^3 a unit,
//   S = Q K^T   dP = dO V^T   and both transposed, as the operands dS (rows i), dS^T and P^T (rows j) are wanted by lanes of tensor memory;
//   dq: dS K, dO h^T    dk: dS^T Q, V dh^T    dv: P^T dO, K dh
// The parts by the states are products of their own, for their rows are scaled by e^{G_i} (e^{G_L - G_j}) behind them, and because x_i and y_j, what
// dg is a sum of, come of them alone: with h and dh as two bf16 pieces they keep the accuracy of fp32.  E = S dS is taken of the fp32
// accumulators.  P and dS are rounded to bf16 for the products that give dq, dk and dv, and dv takes the first piece of dh alone, 2^-8 of it left out:
// all three are rounded to bf16 anyway.
//
// Shared memory has seven slots for a unit's tiles: K, Q, dO, V, two pieces of h, two of dh.  V makes room for the second piece of dh once the scores are
// made and is loaded again, out of L2, where the first piece of h was: so all pieces are there for <h, dh> while the products for dq run, and the slots come free
// over the length of a unit, each for what is needed next.  (An SM gets some 32 bytes a cycle when all load, 1000 cycles for a tile.  With <h, dh> at the
// end the last piece of dh and the next unit's K came 4000 cycles late each, of 25000 a unit then; 20000 now.)  Tensor memory: four regions of 128 columns,
//   R0: S, then dS | dq by h | dv by P      R1: dP | dq by dS | dk by dS      R2: S^T, then P^T | dv by dh      R3: dP^T, then dS^T | dk by dh
// An operand lies over the scores that it is made of: a warp writes 16 columns of it, 8 words, over the first half of the 16 accumulator columns
// that it alone has read, and a product's steps of 16 k go from one such place to the next.  So all four scores become operands in one phase, in which
// the blocks of 32 x 16 on either side of the diagonal (dS below it, the transposed ones above) share out evenly: ten to the four warps of a quarter.
// One more warp scans the next unit's gates and another adds up dg; the sums over a row's columns, which four warps share, pass through a
// few KiB of workspace that stay in L2.
// What bounds it: 352 KiB of tiles, images and gradients a unit, and a unit's dependent phases.  2048 units (four rows of 4096
// tokens, 16 heads): 148 us, 10.7 us a unit of an SM; 1104 pairs of units that share a q/k head 181 us.
#include "tc.cuh"

namespace ha_la {
namespace gla {

namespace {

constexpr int kSlots = 7;
// And G_L = ghi + glo; and which unit these are the gates of: first token, tokens (0: no more units), V-head, V-head of the run; its run's and its q/k head
struct BackGates : StepGates { float ghi, glo; int part_head, qk_head; int4 unit; };
constexpr uint32_t OFF_G = kSlots * kTileBytes;
constexpr uint32_t OFF_BAR = OFF_G + sizeof(BackGates);
constexpr int kBars = 2 * kSlots + 12;
constexpr uint32_t kSmem = OFF_BAR + kBars * 8 + 16;
static_assert(kSmem <= 227 * 1024 && sizeof(BackGates) % 16 == 0, "shared memory budget");
constexpr uint32_t R0 = 0, R1 = 128, R2 = 256, R3 = 384;
enum { kK, kQ, kDO, kV, kHH, kHL, kDH, kDL, kV2, kTiles };   // tiles in the order they are loaded; kDL lies where kV was, kV2 where kHH was

struct BackParams {
  const float* g;
  Chunks chunks;
  const uint8_t *image, *image_back;
  void *dq, *dk, *dv;
  float *dg, *part_q, *part_k;                             // part_q, part_k: [token][run of V-heads][128] fp32, where a q/k head has several runs, or NULL
  float* sums;                                             // [CTA][2][kSums]
  float4* shared;                                          // [CTA][dq, dk][8][512 threads], runs of several V-heads
  int HK, HV, per;                                         // per: V-heads of a run
  float scale;
  long long units;
  int32_t* status;
};

// Slot of a tile of the CTA's unit u, and the parity of its fill there.  Q, dO and V have slots of their own; K, the pieces of h and the first of dh go round
// four, each unit where the next one of that order was the unit before.
__device__ __forceinline__ int slot_of(int tile, int u) {
  if (tile == kQ) return 4;
  if (tile == kDO) return 5;
  if (tile == kV || tile == kDL) return 6;
  return ((tile == kK ? 0 : tile == kHL ? 1 : tile == kDH ? 3 : 2) + u) & 3;
}
__device__ __forceinline__ uint32_t fill_of(int tile, int u) {
  if (tile == kQ || tile == kDO) return u & 1;
  if (tile == kV || tile == kDL) return tile == kDL;
  const int since = (slot_of(tile, u) - 2) & 3;            // the first unit in which this slot was filled twice
  return (u + ((u + 3 - since) >> 2) + (tile == kV2 ? 1 : 0)) & 1;
}

__global__ void __launch_bounds__(kRoleThreads, 1)
gla_tc_back_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                   const __grid_constant__ CUtensorMap map_do, BackParams p) {
  extern __shared__ __align__(1024) uint8_t sm[];
  BackGates* s = reinterpret_cast<BackGates*>(sm + OFF_G);
  uint64_t* bar = reinterpret_cast<uint64_t*>(sm + OFF_BAR);
  uint64_t *full = bar, *empty = bar + kSlots;             // [kSlots]
  uint64_t* one = bar + 2 * kSlots;                        // by one thread or by the tensor cores:
  uint64_t *gates = one, *b_s = one + 1, *b_dq = one + 2, *b_dv = one + 3, *b_dk = one + 4;
  uint64_t* all = one + 5;                                 // by the compute warps:
  uint64_t *g_free = all, *clean = all + 1, *e_s = all + 2, *e_d = all + 3, *e_q = all + 4, *e_v = all + 5, *e_k = all + 6;   // (e_q, e_v, e_k and b_dq, b_dv, b_dk in a row)
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < kBars; ++i) mbar_init(&bar[i], &bar[i] == g_free ? kComputeWarps + 1 : &bar[i] >= all ? kComputeWarps : 1);
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 0) tmem_alloc(tmem_slot, 512);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // A CTA takes runs of `per` V-heads that share a q/k head, of one step: dq and dk add up over them.
  struct Unit { Geom c; int j, r; size_t sj; };            // r: V-head of the run; L = 0: no unit
  const int R = p.HV / p.HK, runs = p.HV / p.per;
  auto unit = [&](int u) {
    const int n = u / p.per;
    const long long i = blockIdx.x + (long long)n * gridDim.x;
    Unit x{{0, 0}, 0, 0, 0};
    if (i >= p.units) return x;
    const int slot = (int)((unsigned)i / (unsigned)runs);
    x.r = u - n * p.per;
    x.j = ((int)i - slot * runs) * p.per + x.r;
    x.sj = (size_t)slot * p.HV + x.j;
    x.c = geom_of(p.chunks, slot);
    return x;
  };
  constexpr int kSums = 2 * 4 * kStep + kComputeWarps;     // [4][128] x + R - C, [4][128] y, [16] parts of <h, dh>
  float* sums = p.sums + (size_t)blockIdx.x * 2 * kSums;

  if (warp >= kComputeWarps) {
    if (warp == kComputeWarps) {
      // ------------------------------------------------------------ tiles
      if (elect_one()) {
        Unit x{{0, 1}, 0, 0, 0};
        for (int u = -1; x.c.L > 0 && !*abort_flag; ++u) {
          const Unit after = unit(u + 1);                    // (its look-ups under the waits, here and below)
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            if (u < 0) break;
            const int at = slot_of(t, u);
            wait_for(&empty[at], fill_of(t, u) ^ 1, abort_flag);
            if (*abort_flag) break;
            uint8_t* dst = sm + at * kTileBytes;
            mbar_expect_tx(&full[at], kTileBytes);
            if (t == kQ) tma_load_4d(dst, &map_q, &full[at], 0, x.j / R, x.c.tok0, 0);
            else if (t == kK) tma_load_4d(dst, &map_k, &full[at], 0, x.j / R, x.c.tok0, 0);
            else if (t == kDO) tma_load_4d(dst, &map_do, &full[at], 0, x.j, x.c.tok0, 0);
            else if (t == kV || t == kV2) tma_load_4d(dst, &map_v, &full[at], 0, x.j, x.c.tok0, 0);
            else bulk_load(dst, (t < kDH ? p.image : p.image_back) + (2 * x.sj + (t == kHL || t == kDL)) * kTileBytes, kTileBytes, &full[at]);
          }
          x = after;
        }
      }
      __syncwarp();
    } else if (warp == kComputeWarps + 1) {
      // ------------------------------------------------------------ products
      if (elect_one()) {
        Unit x{{0, 1}, 0, 0, 0};
        uint32_t tails = 0;
        int last_k = 0;
        for (int u = -1; x.c.L > 0; ++u) {
          const Unit after = unit(u + 1);
          if (u < 0) {
            x = after;
            continue;
          }
          const uint32_t ph = u & 1;
          auto tile = [&](int t) { return smem_u32(sm + slot_of(t, u) * kTileBytes); };
          auto wait = [&](uint64_t* b, uint32_t parity) {
            wait_for(b, parity, abort_flag);
            tc_fence_after_sync();
          };
          auto loaded = [&](int t) { wait(&full[slot_of(t, u)], fill_of(t, u)); };
          loaded(kQ);
          loaded(kK);
          if (x.c.L < kStep) wait(clean, tails++ & 1);
          if (u > 0) wait(e_v, ph ^ 1);
          mma_cols(R0, tile(kQ), tile(kK), false);           // S
          mma_cols(R2, tile(kK), tile(kQ), false);           // S^T
          if (u > 0) {
            wait(e_k, ph ^ 1);
            mbar_arrive(&empty[last_k]);                     // (its products are complete)
          }
          loaded(kDO);
          loaded(kV);
          mma_cols(R1, tile(kDO), tile(kV), false);          // dP
          mma_cols(R3, tile(kV), tile(kDO), false);          // dP^T
          umma_commit(b_s);
          umma_commit(&empty[slot_of(kV, u)]);
          wait(e_s, ph);
          mma_tmem_rows<16>(R1, R0, tile(kK), false);        // dS K
          loaded(kHH);
          mma_cols(R0, tile(kDO), tile(kHH), false);         // dO h^T
          loaded(kHL);
          mma_cols(R0, tile(kDO), tile(kHL), true);
          umma_commit(b_dq);
          wait(e_d, ph);
          umma_commit(&empty[slot_of(kHH, u)]);
          umma_commit(&empty[slot_of(kHL, u)]);
          wait(e_q, ph);
          mma_tmem_rows<16>(R1, R3, tile(kQ), false);        // dS^T Q
          umma_commit(&empty[slot_of(kQ, u)]);
          mma_tmem_rows<16>(R0, R2, tile(kDO), false);       // P^T dO
          umma_commit(&empty[slot_of(kDO, u)]);
          loaded(kDH);
          mma_rows(R2, tile(kK), tile(kDH), false);          // K dh
          umma_commit(b_dv);
          loaded(kV2);
          mma_cols(R3, tile(kV2), tile(kDH), false);         // V dh^T
          loaded(kDL);
          mma_cols(R3, tile(kV2), tile(kDL), true);
          umma_commit(b_dk);
          umma_commit(&empty[slot_of(kV2, u)]);
          umma_commit(&empty[slot_of(kDH, u)]);
          umma_commit(&empty[slot_of(kDL, u)]);
          last_k = slot_of(kK, u);
          x = after;
        }
      }
      __syncwarp();
    } else if (warp == kComputeWarps + 2) {
      // ------------------------------------------------------------ gates
      Unit x = unit(0);
      float4 raw = fetch_gates(p.g, p.HV, x.j, x.c, lane);
#pragma unroll 1
      for (int u = 0;; ++u) {                              // (behind the last unit: that there are no more)
        const Unit after = x.c.L > 0 ? unit(u + 1) : x;
        double G[4];
        scan_gates(raw, lane, G);
        raw = fetch_gates(p.g, p.HV, after.j, after.c, lane);
        const LaneGates mine = lane_gates(G, lane);
        const double GL = __shfl_sync(0xffffffffu, G[3], 31);
        if (u > 0) wait_for(g_free, (u - 1) & 1, abort_flag);
        __syncwarp();
        put_gates(s, mine, lane);
        if (lane == 0) {
          s->ghi = (float)GL;
          s->glo = (float)(GL - (double)(float)GL);
          s->unit = make_int4(x.c.tok0, x.c.L, x.j, x.r);
          s->part_head = x.j / p.per;
          s->qk_head = x.j / R;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(gates);
        __syncwarp();
        if (x.c.L <= 0) break;
        x = after;
      }
    } else {
      // ------------------------------------------------------------ dg
#pragma unroll 1
      for (int u = 0;; ++u) {
        wait_for(gates, u & 1, abort_flag);
        __syncwarp();
        const int4 at = s->unit;
        const float total = ex2(s->ghi + s->glo);
        const bool gave_up = __any_sync(0xffffffffu, *abort_flag);
        if (lane == 0) mbar_arrive(g_free);                // (and the sums of the unit before have been read)
        if (at.y <= 0 || gave_up) break;
        wait_for(e_k, u & 1, abort_flag);                  // (the last of the unit's sums are written ahead of it)
        __syncwarp();
        const float* f = sums + (u & 1) * kSums;
        double z[4] = {0.0, 0.0, 0.0, 0.0}, y[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4 a = __ldcg(reinterpret_cast<const float4*>(f + g * kStep) + lane), b = __ldcg(reinterpret_cast<const float4*>(f + 4 * kStep + g * kStep) + lane);
#pragma unroll
          for (int e = 0; e < 4; ++e) { z[e] += (&a.x)[e]; y[e] += (&b.x)[e]; }
        }
        double dot = lane < kComputeWarps ? (double)__ldcg(f + 8 * kStep + lane) : 0.0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
        dot *= total;
        z[2] += z[3]; z[1] += z[2]; z[0] += z[1];          // z: over this and later tokens, y: over earlier ones
        const double y3 = y[3], y012 = y[0] + y[1] + y[2];
        double zs = z[0], ys = y012 + y3;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const double a = __shfl_down_sync(0xffffffffu, zs, o), b = __shfl_up_sync(0xffffffffu, ys, o);
          if (lane + o < 32) zs += a;
          if (lane >= o) ys += b;
        }
        const double behind = zs - z[0], front = ys - (y012 + y3);
        const double yy[4] = {front, front + y[0], front + y[0] + y[1], front + y012};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (4 * lane + e < at.y) p.dg[(size_t)(at.x + 4 * lane + e) * p.HV + at.z] = (float)(z[e] + behind + yy[e] + dot);
      }
    }
  } else {
    // ------------------------------------------------------------ operands, gradients
    const int q = warp & 3, g = warp >> 2, i = 32 * q + lane;     // row (token, key), columns 32 g ..
    const uint32_t lanes = static_cast<uint32_t>(32 * q) << 16;
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
    int u = 0;
    auto seen = [&](int t) {                               // (loaded long ago; this thread's own look at it)
      wait_for(&full[slot_of(t, u)], fill_of(t, u), abort_flag);
      __syncwarp();
    };
    // 16-byte piece k of this thread's 32 columns in its row of the tile in a slot
    auto piece = [&](int at, int k) {
      return *reinterpret_cast<const uint4*>(sm + at * kTileBytes + (g >> 1) * 16384 + i * 128 + (((4 * (g & 1) + k) ^ (i & 7)) << 4));
    };
    float4* acc = p.per > 1 ? p.shared + (size_t)blockIdx.x * 2 * 8 * 512 + tid : nullptr;
    // What the loop over units executes has to stay small, or the warps wait for their instructions: one body for the operands below and above the
    // diagonal, one for the three gradients.
    struct { Geom c; int j, r, out; } x;                   // out: head of dq, dk
    const bool by_run = p.part_q;
    for (;; ++u) {
      {
        const uint32_t ph = u & 1;
        wait_for(gates, ph, abort_flag);
        __syncwarp();
        const int4 at_unit = s->unit;
        x = {{at_unit.x, __any_sync(0xffffffffu, *abort_flag) ? 0 : at_unit.y}, at_unit.z, at_unit.w, by_run ? s->part_head : s->qk_head};
        if (x.c.L <= 0) break;
        if (x.c.L < kStep) {                               // (rows behind the sequence may be NaN)
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            wait_for(&full[slot_of(t, u)], fill_of(t, u), abort_flag);
            clear_rows(sm + slot_of(t, u) * kTileBytes, x.c.L, tid, 32 * kComputeWarps);
          }
          fence_proxy_async_smem();
          arrive(clean);
        }
        const float hi = s->hi[i], lo = s->lo[i];
        const float eg = p.scale * ex2(hi + lo), el = ex2((s->ghi - hi) + (s->glo - lo));

        // ---- operands, 16 columns at a time: dS (row i, columns j <= i), then with the roles of rows and columns exchanged P^T and dS^T;
        // z: R_i - C_i of these columns
        wait(b_s, ph);
        const uint32_t slice = lanes + 32 * g;
        float z = 0.f;
        {                                                  // zeros on the other side of the diagonal
          const uint32_t none[8] = {};
          if (g > q) {
            tmem_st8(R0 + slice, none);
            tmem_st8(R0 + slice + 16, none);
          }
          if (g < q) {
            tmem_st8(R2 + slice, none);
            tmem_st8(R2 + slice + 16, none);
            tmem_st8(R3 + slice, none);
            tmem_st8(R3 + slice + 16, none);
          }
        }
#pragma unroll 1
        for (int n = g; n < 10; n += 4) {                  // block n of the quarter: 2 q + 2 below the diagonal, then 8 - 2 q above
          const bool above = n >= 2 * q + 2;
          const int b = above ? n - 2 : n;                 // block of 16 columns
          const uint32_t at = lanes + 16 * b;
          uint32_t rs[16], rp[16], wp[8], ws[8];
          tmem_ld16((above ? R2 : R0) + at, rs);
          tmem_ld16((above ? R3 : R1) + at, rp);
          float2 dec[8];                                   // decay, mask and scale
          if (b >> 1 != q) {
            const float f = p.scale * (above ? s->ec[i] * s->bb[8 * b + (i >> 4)] : s->er[i] * s->bb[8 * (i >> 4) + b]);
            const float* e = (above ? s->er : s->ec) + 16 * b;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float4 c = *reinterpret_cast<const float4*>(e + 4 * k);
              dec[2 * k] = mul2(make_float2(f, f), make_float2(c.x, c.y));
              dec[2 * k + 1] = mul2(make_float2(f, f), make_float2(c.z, c.w));
            }
          } else {
            const float sign = above ? 1.f : -1.f;
            const int to = i - 16 * b;                     // the row's own column
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float2 a = fma2(*reinterpret_cast<const float2*>(&s->hi[16 * b + 2 * k]), make_float2(sign, sign), make_float2(-sign * hi, -sign * hi)),
                           c = fma2(*reinterpret_cast<const float2*>(&s->lo[16 * b + 2 * k]), make_float2(sign, sign), make_float2(-sign * lo, -sign * lo));
              dec[k].x = (above ? 2 * k >= to : 2 * k <= to) ? p.scale * ex2(a.x + c.x) : 0.f;
              dec[k].y = (above ? 2 * k + 1 >= to : 2 * k + 1 <= to) ? p.scale * ex2(a.y + c.y) : 0.f;
            }
          }
          tmem_ld_wait();
          float2 zz = make_float2(0.f, 0.f);
          const int diag = i - 16 * b;                     // the column whose E counts for neither (none, where it is not of these 16)
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float2 sc = as_f2(rs[2 * k], rs[2 * k + 1]), ds = mul2(dec[k], as_f2(rp[2 * k], rp[2 * k + 1]));
            wp[k] = pack_bf16(mul2(dec[k], sc));
            ws[k] = pack_bf16(ds);
            zz = fma2(make_float2(2 * k == diag ? 0.f : ds.x, 2 * k + 1 == diag ? 0.f : ds.y), sc, zz);
          }
          z += above ? -(zz.x + zz.y) : zz.x + zz.y;
          tmem_st8((above ? R3 : R0) + at, ws);
          if (above) tmem_st8(R2 + at, wp);
        }
        tmem_st_wait();
        arrive(e_s);
        if (lane == 0) mbar_arrive(g_free);

        // ---- <h, dh>, under the products for dq
        float* mine = sums + ph * kSums;
        {
          float2 d = make_float2(0.f, 0.f);
          seen(kHH);
          seen(kHL);
          seen(kDH);
          seen(kDL);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint4 h1 = piece(slot_of(kHH, u), k), h2 = piece(slot_of(kHL, u), k), d1 = piece(slot_of(kDH, u), k), d2 = piece(slot_of(kDL, u), k);
#pragma unroll
            for (int w = 0; w < 4; ++w)
              d = fma2(add2(unpack_bf16((&h1.x)[w]), unpack_bf16((&h2.x)[w])), add2(unpack_bf16((&d1.x)[w]), unpack_bf16((&d2.x)[w])), d);
          }
          arrive(e_d);
          float sum = d.x + d.y;
#pragma unroll
          for (int e = 16; e > 0; e >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, e);
          if (lane == 0) __stcg(mine + 8 * kStep + warp, sum);
        }

        // ---- dq, dv, dk: a f + c, a the part by the state; with the sums x_i, y_i of a f . (the row of q, k) ahead of e_q, e_k
#pragma unroll 1
        for (int o = 0; o < 3; ++o) {
          asm volatile("" : "+r"(o));                      // (not three copies of the body)
          wait(b_dq + o, ph);
          if (o != 1) seen(o == 0 ? kQ : kK);
          const float f = o == 0 ? eg : el;
          const bool parts = o != 1 && by_run;
          const int heads = o == 1 ? p.HV : by_run ? runs : p.HK;
          const size_t row0 = ((size_t)(x.c.tok0 + 32 * q) * heads + (o == 1 ? x.j : x.out)) * 128 + 32 * g, pitch = (size_t)heads * 128;
          uint32_t a[32], c[32];
          tmem_ld32((o == 0 ? R0 : o == 1 ? R2 : R3) + slice, a);
          tmem_ld32((o == 1 ? R0 : R1) + slice, c);
          tmem_ld_wait();
          if (o != 1) {
            float2 d = make_float2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint4 t = piece(o == 0 ? slot_of(kQ, u) : slot_of(kK, u), k);
#pragma unroll
              for (int w = 0; w < 4; ++w) d = fma2(as_f2(a[8 * k + 2 * w], a[8 * k + 2 * w + 1]), unpack_bf16((&t.x)[w]), d);
            }
            // (behind the sequence y is of whatever V's second loading brought)
            __stcg(mine + (o == 0 ? 0 : 4 * kStep) + g * kStep + i, i < x.c.L ? fmaf(f, d.x + d.y, o == 0 ? z : 0.f) : 0.f);
          }
          arrive(e_q + o);
#pragma unroll
          for (int k = 0; k < 32; k += 2) {
            const float2 v = fma2(as_f2(a[k], a[k + 1]), make_float2(f, f), as_f2(c[k], c[k + 1]));
            a[k] = __float_as_uint(v.x);
            a[k + 1] = __float_as_uint(v.y);
          }
          if (o != 1 && acc) {                             // added to what the run's V-heads before left, and left for the next ones
            float4* part = acc + (o == 0 ? 0 : 8 * 512);
            if (x.r > 0) {
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const float4 y = __ldcg(part + 512 * k);
                const float2 v0 = add2(as_f2(a[4 * k], a[4 * k + 1]), make_float2(y.x, y.y)), v1 = add2(as_f2(a[4 * k + 2], a[4 * k + 3]), make_float2(y.z, y.w));
                a[4 * k] = __float_as_uint(v0.x); a[4 * k + 1] = __float_as_uint(v0.y);
                a[4 * k + 2] = __float_as_uint(v1.x); a[4 * k + 3] = __float_as_uint(v1.y);
              }
            }
            if (x.r < p.per - 1) {
#pragma unroll
              for (int k = 0; k < 8; ++k)
                __stcg(part + 512 * k, make_float4(__uint_as_float(a[4 * k]), __uint_as_float(a[4 * k + 1]), __uint_as_float(a[4 * k + 2]), __uint_as_float(a[4 * k + 3])));
              continue;
            }
          }
          const int row = lane & ~3, left = x.c.L - 32 * q - row;
          if (parts) {
            float* dst = (o == 0 ? p.part_q : p.part_k) + row0 + row * pitch + 4 * (lane & 3);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              uint4 v[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) v[k] = make_uint4(a[16 * half + 4 * k], a[16 * half + 4 * k + 1], a[16 * half + 4 * k + 2], a[16 * half + 4 * k + 3]);
              exchange4(v, lane);
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (k < left) *reinterpret_cast<uint4*>(dst + k * pitch + 16 * half) = v[k];
            }
          } else {
            uint4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
              v[k] = make_uint4(pack_bf16(as_f2(a[8 * k], a[8 * k + 1])), pack_bf16(as_f2(a[8 * k + 2], a[8 * k + 3])),
                                pack_bf16(as_f2(a[8 * k + 4], a[8 * k + 5])), pack_bf16(as_f2(a[8 * k + 6], a[8 * k + 7])));
            exchange4(v, lane);
            __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(o == 0 ? p.dq : o == 1 ? p.dv : p.dk) + row0 + row * pitch + 8 * (lane & 3);
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (k < left) *reinterpret_cast<uint4*>(dst + k * pitch) = v[k];
          }
        }
      }
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (tid == 0 && *abort_flag) report_timeout(p.status);
  __syncthreads();
  if (warp == 0) tmem_dealloc(*tmem_slot, 512);
}

}  // namespace

// V-heads of a q/k head that one CTA takes one behind the other, so that dq and dk add up on the way: as many as leave two runs to an SM.
int heads_per_run(const Problem& p) {
  const int R = p.HV / p.HK;
  for (int per = R; per > 1; --per)
    if (R % per == 0 && (long long)p.max_chunks * (p.HV / per) >= 2 * sm_count()) return per;
  return 1;
}

size_t local_back_bytes() { return (size_t)sm_count() * 2 * (2 * 4 * kStep + kComputeWarps) * 4; }

cudaError_t launch_tc_local_back(const TcCall& t, cudaStream_t stream) {
  const Call& c = *t.c;
  BackParams p;
  p.g = c.a.g; p.chunks = c.chunks; p.image = t.w.image; p.image_back = t.w.image_back;
  p.dq = c.a.dq; p.dk = c.a.dk; p.dv = c.a.dv; p.dg = c.a.dg;
  p.per = heads_per_run(c.p);
  p.part_q = c.p.HV / p.per != c.p.HK ? c.w.dq : nullptr;
  p.part_k = c.p.HV / p.per != c.p.HK ? c.w.dk : nullptr;
  p.sums = t.w.sums; p.shared = t.w.shared;
  p.HK = c.p.HK; p.HV = c.p.HV; p.scale = c.p.scale; p.status = c.a.status_word;
  p.units = (long long)c.p.max_chunks * (c.p.HV / p.per);
  if (p.units == 0) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(gla_tc_back_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
  const unsigned grid = (unsigned)(p.units < sm_count() ? p.units : sm_count());
  return e != cudaSuccess ? e : start(gla_tc_back_kernel, dim3(grid), kRoleThreads, kSmem, stream, t.q, t.k, t.v, t.d_o, p);
}

}  // namespace gla
}  // namespace ha_la

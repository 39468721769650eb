// Attention of new tokens to cached latent rows, tensor cores: bf16, rows of 512 + 64, pages of 16 rows or more.
//
// All heads (and new tokens) of a sequence read the same rows, whose first 512 values are keys and values at once, so a row is brought once for up to 32
// query rows and HBM bounds it: 1152 bytes a row, 2 x 1088 multiply-adds a query row.  What fills a matrix instruction's 128 rows are not the queries, of
// which there may be sixteen, but the cache's rows and the latent channels:
//   S^T = C q^T     (128 cached rows x NR queries; nine chunks of 64 channels)
//   O^T += V^T P^T  (4 x 128 channels x NR queries; V = the first eight chunks of C, read the other way round from the same shared memory)
// with P^T through shared memory.  A softmax thread has a cached row, so a query's maximum is spread over 128 threads: they take the exact one for a
// segment's first rows and whenever a score exceeds it by 2^8 (one vote), and each adds up its own weights until the end.
//
// Work is cut into units of 128 rows of all sequences one behind the other, in equal parts for the CTAs, one an SM: long and short contexts, few or many,
// load all of them evenly.  A sequence that several CTAs share leaves unnormalised parts, joined by a second kernel in order.
#include <algorithm>

#include "latent.cuh"
#include "../gla/tc.cuh"

namespace ha_la {

bool make_map_4d(CUtensorMap* m, const void* base, const unsigned long long (&size)[4], const unsigned long long (&stride)[3], const unsigned (&tile)[4]);   // tc.cu

namespace mix {
namespace {

using namespace ptx;
using gla::wait_for;

constexpr int kThreads = 192, kPairs = 5, kLatent = 512, kRow = 576;      // threads: softmax, copies, products; slots of 128 channels
constexpr uint32_t kPairB = 32768, kRopeB = 16384;

template <int NR> struct Cfg {
  static constexpr uint32_t OFF_ROPE = kPairs * kPairB, OFF_Q = OFF_ROPE + kRopeB, OFF_P = OFF_Q + NR * 1152, OFF_BAR = OFF_P + NR * 256;
  static constexpr size_t kSmem = OFF_BAR + 256;
  static constexpr uint32_t kTmO = 0, kTmS = 4 * NR, kTmCols = NR == 32 ? 256 : 128;
  // P^T: a cached row's weights side by side, NR bf16 values, swizzled over that width
  static constexpr uint64_t kSwizzle = NR == 32 ? kSwizzle64B : kSwizzle32B;
  static constexpr uint32_t kPRow = NR * 2, kIdS = idesc_bf16(128, NR, false, false), kIdO = idesc_bf16(128, NR, true, true);
};

__device__ __forceinline__ int units_of(const TokenParams& p, int n) { return (rows_of(p, n) + 127) >> 7; }

// Units of the sequences in front of sequence `before`, and of all; by all of a CTA's threads.
struct Count { long long before, all; };
template <int THREADS> __device__ __forceinline__ Count count_units(const TokenParams& p, int before) {
  __shared__ long long s_part[2][THREADS / 32];
  long long a = 0, b = 0;
  for (int n = threadIdx.x; n < p.N; n += THREADS) {
    const int u = units_of(p, n);
    b += u;
    if (n < before) a += u;
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, o);
    b += __shfl_xor_sync(0xffffffffu, b, o);
  }
  if ((threadIdx.x & 31) == 0) {
    s_part[0][threadIdx.x >> 5] = a;
    s_part[1][threadIdx.x >> 5] = b;
  }
  __syncthreads();
  Count c = {0, 0};
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    c.before += s_part[0][w];
    c.all += s_part[1][w];
  }
  return c;
}

// A CTA's part of the units, segment by segment: tiles [t0, t1) of sequence n for query block rb, of `tiles`.
struct Walk {
  long long u, u1, base;
  int n, blocks, rb, t0, t1, tiles;
  __device__ __forceinline__ bool next(const TokenParams& p) {
    if (u >= u1) return false;
    while ((tiles = units_of(p, n)) == 0 || u >= base + (long long)blocks * tiles) {
      base += (long long)blocks * tiles;
      if (++n >= p.N) return false;                        // (not to be: the units add up)
    }
    const long long in = u - base;
    rb = (int)(in / tiles);
    t0 = (int)(in - (long long)rb * tiles);
    t1 = (int)min((long long)tiles, t0 + (u1 - u));
    u += t1 - t0;
    return true;
  }
};

// Largest (or sum) of v[j] over the lanes of a warp, j left in lane j (NR 16: in lanes j and j + 16).
template <int NR, bool MAX> __device__ __forceinline__ float spread(float (&v)[NR]) {
  const int lane = threadIdx.x & 31;
  auto join = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
#pragma unroll
  for (int off = NR / 2; off; off >>= 1) {
    const bool up = lane & off;
#pragma unroll
    for (int j = 0; j < off; ++j) {
      const float keep = up ? v[j + off] : v[j], send = up ? v[j] : v[j + off];
      v[j] = join(keep, __shfl_xor_sync(0xffffffffu, send, off));
    }
  }
  if (NR == 16) v[0] = join(v[0], __shfl_xor_sync(0xffffffffu, v[0], 16));
  return v[0];
}

__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ bool softmax_any(bool x) {
  uint32_t y;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbar.red.or.pred p, 2, 128, q;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(y) : "r"((uint32_t)x) : "memory");
  return y != 0;
}

template <int NR>
__global__ void __launch_bounds__(kThreads, 1)
latent_token_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_c, TokenParams p) {
  using C = Cfg<NR>;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* const sm = smem;
  __shared__ int s_n;
  __shared__ long long s_base, s_scan[kThreads / 32];
  __shared__ __align__(16) float s_m[NR], s_f[NR], s_red[4][NR];
  uint64_t* const bar = reinterpret_cast<uint64_t*>(sm + C::OFF_BAR);
  uint64_t *const q_full = bar, *const q_free = bar + 1, *const rope_full = bar + 2, *const rope_free = bar + 3, *const scores = bar + 4, *const done = bar + 6;
  uint64_t *const pair_full = bar + 7, *const pair_free = pair_full + kPairs, *const weights = pair_free + kPairs;
  constexpr int kBars = 7 + 2 * kPairs + 1;
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bar + kBars);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < kBars; ++i) mbar_init(&bar[i], &bar[i] >= weights ? 4 : 1);
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 0) tmem_alloc(tmem_slot, C::kTmCols);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tm = *tmem_slot;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0) check_tokens(p);

  // the CTA's part: where its first unit lies
  const int all_rows = p.T * p.H, blocks = (all_rows + NR - 1) / NR;
  Walk walk;
  walk.blocks = blocks;
  {
    const int per = (p.N + kThreads - 1) / kThreads, n0 = min(tid * per, p.N), n1 = min(n0 + per, p.N);
    long long mine = 0;
    for (int n = n0; n < n1; ++n) mine += units_of(p, n);
    long long upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    if (lane == 31) s_scan[warp] = upto;
    __syncthreads();
    long long all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w < warp) upto += s_scan[w];
      all += s_scan[w];
    }
    all *= blocks;
    walk.u = all * blockIdx.x / gridDim.x;
    walk.u1 = all * (blockIdx.x + 1) / gridDim.x;
    long long at = (upto - mine) * blocks;
    if (walk.u < walk.u1 && at <= walk.u && walk.u < upto * blocks) {
      int n = n0;
      for (long long step; walk.u >= at + (step = (long long)units_of(p, n) * blocks); ++n) at += step;
      s_n = n;
      s_base = at;
    }
    __syncthreads();
    if (walk.u < walk.u1) {
      walk.n = s_n;
      walk.base = s_base;
    }
  }
  const int page = 1 << p.page_log, box = min(page, 128), boxes = 128 / box;   // rows of a copy, copies for 128 rows

  if (warp == 4) {
    // ------------------------------------------------------------ tiles: a lane to a copy
    int seg = 0, tile = 0;                                 // of the CTA so far
    while (walk.next(p)) {
      const int len = rows_of(p, walk.n);
      if (seg > 0) wait_for(q_free, (seg - 1) & 1, abort_flag);
      __syncwarp();
      if (elect_one()) {
        mbar_expect_tx(q_full, NR * 1152);
        tma_load_4d(sm + C::OFF_Q, &map_q, q_full, 0, walk.n * all_rows + walk.rb * NR, 0, 0);
      }
      __syncwarp();
      auto row_at = [&](int t) -> int {                    // this lane's piece of tile t: the cache's row, or -1
        const int j = t * 128 + lane % boxes * box;
        return t < walk.t1 && j < len ? (int)cache_row(p, walk.n, j) : -1;
      };
      int row = row_at(walk.t0);
      for (int t = walk.t0; t < walk.t1; ++t, ++tile) {
        const int next = row_at(t + 1), have = min(boxes, (min(len - t * 128, 128) + box - 1) / box);
        if (tile > 0) wait_for(rope_free, (tile - 1) & 1, abort_flag);
        __syncwarp();
        if (*abort_flag) break;
        if (lane == 0) mbar_expect_tx(rope_full, (uint32_t)(have * box) * 128);
        __syncwarp();
        if (lane < have) tma_load_4d(sm + C::OFF_ROPE + lane * box * 128, &map_c, rope_full, 0, row, 8, 0);
        __syncwarp();
        for (int b = 0; b < 4; ++b) {
          const int x = tile * 4 + b, slot = x % kPairs;
          if (x >= kPairs) wait_for(&pair_free[slot], (x / kPairs - 1) & 1, abort_flag);
          __syncwarp();
          if (*abort_flag) break;
          if (lane == 0) mbar_expect_tx(&pair_full[slot], (uint32_t)(have * box) * 256);
          __syncwarp();
          const int half = lane / boxes;
          if (half < 2 && lane % boxes < have)
            tma_load_4d(sm + slot * kPairB + half * 16384 + lane % boxes * box * 128, &map_c, &pair_full[slot], 0, row, 2 * b + half, 0);
          __syncwarp();
        }
        row = next;
      }
      ++seg;
      if (*abort_flag) break;
    }
  } else if (warp == 5) {
    // ------------------------------------------------------------ products
    if (elect_one()) {
      const uint32_t sq = smem_u32(sm + C::OFF_Q), sp = smem_u32(sm + C::OFF_P), rope = smem_u32(sm + C::OFF_ROPE);
      const uint64_t dp = smem_desc(sp, 16, 8 * C::kPRow, C::kSwizzle);
      auto part = [&](uint32_t d, uint32_t chunk, int c, bool add) {      // 64 channels' share of the scores
        const uint64_t da = gla::desc_cols(chunk), db = smem_desc(sq + c * NR * 128, 16, 1024, kSwizzle128B);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) umma_ss(d, da + 2 * ks, db + 2 * ks, C::kIdS, add || ks > 0);
      };
      int seg = 0, tile = 0;
      while (walk.next(p)) {
        wait_for(q_full, seg & 1, abort_flag);
        auto add_values = [&](int i, bool start) {         // weights of the CTA's tile i (a segment's first come once O has been read)
          wait_for(weights, i & 1, abort_flag);
          tc_fence_after_sync();
          for (int b = 0; b < 4; ++b) {
            const int slot = (i * 4 + b) % kPairs;
            const uint64_t da = gla::desc_rows(smem_u32(sm + slot * kPairB));
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) umma_ss(tm + C::kTmO + NR * b, da + gla::step_rows(ks), dp + ((ks * 16 * C::kPRow) >> 4), C::kIdO, !start || ks > 0);
            umma_commit(&pair_free[slot]);
          }
        };
        for (int t = walk.t0; t < walk.t1; ++t, ++tile) {
          const uint32_t d = tm + C::kTmS + NR * (tile & 1);
          wait_for(rope_full, tile & 1, abort_flag);
          if (*abort_flag) break;
          tc_fence_after_sync();
          part(d, rope, 8, false);
          umma_commit(rope_free);
          for (int b = 0; b < 4; ++b) {
            const int x = tile * 4 + b, slot = x % kPairs;
            // (the values of the tile before give this one's rows their place)
            if (b == 1 && t > walk.t0) add_values(tile - 1, t == walk.t0 + 1);
            wait_for(&pair_full[slot], (x / kPairs) & 1, abort_flag);
            tc_fence_after_sync();
            part(d, smem_u32(sm + slot * kPairB), 2 * b, true);
            part(d, smem_u32(sm + slot * kPairB) + 16384, 2 * b + 1, true);
          }
          umma_commit(&scores[tile & 1]);
        }
        umma_commit(q_free);
        if (*abort_flag) break;
        add_values(tile - 1, walk.t1 == walk.t0 + 1);
        umma_commit(done);
        ++seg;
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax: a thread to a cached row
    const int row = tid;
    const uint32_t lanes = static_cast<uint32_t>(32 * warp) << 16;
    const float to_log2 = p.scale * 1.4426950408889634f;
    int seg = 0, tile = 0;
    while (walk.next(p)) {
      const int len = rows_of(p, walk.n), r0 = walk.rb * NR, rows = min(NR, all_rows - r0), low = len - p.T + 1;
      float l[NR];
#pragma unroll
      for (int r = 0; r < NR; ++r) l[r] = 0.f;
      if (tid < NR) s_m[tid] = kNegInf;
      softmax_sync();
      for (int t = walk.t0; t < walk.t1; ++t, ++tile) {
        wait_for(&scores[tile & 1], (tile >> 1) & 1, abort_flag);
        __syncwarp();
        tc_fence_after_sync();
        uint32_t raw[NR];
        if constexpr (NR == 32) tmem_ld32(tm + C::kTmS + NR * (tile & 1) + lanes, raw);
        else tmem_ld16(tm + C::kTmS + NR * (tile & 1) + lanes, raw);
        tmem_ld_wait();
        const int j = t * 128 + row;
        float s[NR];
        const bool partly = t * 128 + 128 > low + (p.T > 1 ? r0 / p.H : 0);   // (of the block's first token)
#pragma unroll
        for (int r = 0; r < NR; ++r) s[r] = __uint_as_float(raw[r]) * to_log2;
        if (partly) {
#pragma unroll
          for (int r = 0; r < NR; ++r) s[r] = j < low + (p.T > 1 ? (r0 + r) / p.H : 0) && j < len ? s[r] : kNegInf;
        }
        bool over = t == walk.t0;
#pragma unroll
        for (int r = 0; r < NR; r += 4) {
          const float4 m = *reinterpret_cast<const float4*>(&s_m[r]);
          over |= s[r] > m.x + 8.f || s[r + 1] > m.y + 8.f || s[r + 2] > m.z + 8.f || s[r + 3] > m.w + 8.f;
        }
        if (softmax_any(over)) {
          float v[NR];
#pragma unroll
          for (int r = 0; r < NR; ++r) v[r] = s[r];
          const float top = spread<NR, true>(v);
          if (lane < NR) s_red[warp][lane] = top;
          softmax_sync();
          if (tid < NR) {
            const float m = s_m[tid], next = fmaxf(fmaxf(m, fmaxf(s_red[0][tid], s_red[1][tid])), fmaxf(s_red[2][tid], s_red[3][tid]));
            s_f[tid] = m == kNegInf ? 0.f : ex2(m - next);
            s_m[tid] = next;
          }
          softmax_sync();
          if (t > walk.t0) {
#pragma unroll
            for (int r = 0; r < NR; ++r) l[r] *= s_f[r];
            // (the products that these scores stood behind are done, so O is whole)
#pragma unroll 1
            for (int b = 0; b < 4; ++b) {
              uint32_t o[16];
#pragma unroll
              for (int r = 0; r < NR; r += 16) {
                tmem_ld16(tm + C::kTmO + NR * b + r + lanes, o);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * s_f[r + e]);
                tmem_st16(tm + C::kTmO + NR * b + r + lanes, o);
              }
            }
            tmem_st_wait();
          }
        }
        uint32_t w[NR / 2];
#pragma unroll
        for (int r = 0; r < NR; r += 4) {
          const float4 m = *reinterpret_cast<const float4*>(&s_m[r]);
          float e[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float mx = (&m.x)[x];
            e[x] = ex2(s[r + x] - (mx == kNegInf ? 0.f : mx));
            l[r + x] += e[x];
          }
          w[r / 2] = pack_bf16(e[0], e[1]);
          w[r / 2 + 1] = pack_bf16(e[2], e[3]);
        }
#pragma unroll
        for (int c = 0; c < NR / 8; ++c) {
          const uint32_t at = NR == 32 ? sw64_offset(row, c) : static_cast<uint32_t>(row * 32 + ((c ^ ((row >> 2) & 1)) << 4));
          *reinterpret_cast<uint4*>(sm + C::OFF_P + at) = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
        }
        if (len - t * 128 < 128) {                         // rows that are not the sequence's may be NaN, which no weight of zero masks
          for (int b = 0; b < 4; ++b) gla::clear_rows(sm + (tile * 4 + b) % kPairs * kPairB, len - t * 128, tid, 128);
        }
        fence_proxy_async_smem();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(weights);
        __syncwarp();
      }
      const float mine = spread<NR, false>(l);
      if (lane < NR) s_red[warp][lane] = mine;
      softmax_sync();
      if (tid < NR) s_f[tid] = (s_red[0][tid] + s_red[1][tid]) + (s_red[2][tid] + s_red[3][tid]);
      softmax_sync();
      const bool whole = walk.t0 == 0 && walk.t1 == walk.tiles;
      const size_t q_row = (size_t)walk.n * all_rows + r0, slot = ((size_t)blockIdx.x * 2 + (seg > 0)) * NR;
      wait_for(done, seg & 1, abort_flag);
      __syncwarp();
      tc_fence_after_sync();
#pragma unroll 1
      for (int b = 0; b < 4; ++b) {
        uint32_t o[NR];
        if constexpr (NR == 32) tmem_ld32(tm + C::kTmO + NR * b + lanes, o);
        else tmem_ld16(tm + C::kTmO + NR * b + lanes, o);
        tmem_ld_wait();
        const int c = 128 * b + row;
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          if (r >= rows) break;
          const float x = __uint_as_float(o[r]);
          if (whole) reinterpret_cast<__nv_bfloat16*>(p.o)[(q_row + r) * kLatent + c] = __float2bfloat16_rn(s_f[r] > 0.f ? x / s_f[r] : 0.f);
          else p.part_o[(slot + r) * kLatent + c] = x;
        }
      }
      if (tid < rows) {
        const float sum = s_f[tid], m = s_m[tid];
        if (!whole) *reinterpret_cast<float2*>(p.part_ml + (slot + tid) * 2) = make_float2(m, sum);
        else if (p.lse) p.lse[q_row + tid] = sum > 0.f ? (m + log2f(sum)) * 0.6931471805599453f : kNegInf;
      }
      softmax_sync();                                      // (s_m and s_f are used again)
      ++seg;
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (tid == 0 && *abort_flag) report_timeout(p.status);
  __syncthreads();
  if (warp == 0) tmem_dealloc(*tmem_slot, C::kTmCols);
}

// Joins the parts of a query row that several CTAs have made, a warp to every eighth of them, 128 channels to a CTA.
constexpr int kJoin = 256;
__global__ void __launch_bounds__(kJoin) latent_join_kernel(TokenParams p, int NR, int G) {
  __shared__ float s_w[kJoin], s_top[kJoin / 32], s_sum[kJoin / 32];
  __shared__ __align__(16) float4 s_o[kJoin / 32][32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, all_rows = p.T * p.H, blocks = (all_rows + NR - 1) / NR;
  const int c0 = (blockIdx.x & 3) * 128, row = blockIdx.x >> 2, n = row / all_rows, r = row - n * all_rows, rb = r / NR;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const Count c = count_units<kJoin>(p, n);
  const long long total = c.all * blocks, tiles = units_of(p, n), u = c.before * blocks + rb * tiles;
  __nv_bfloat16* const out = reinterpret_cast<__nv_bfloat16*>(p.o) + (size_t)row * kLatent + c0;
  if (tiles == 0) {
    if (tid < 32) *reinterpret_cast<uint2*>(out + 4 * tid) = make_uint2(0u, 0u);
    if (tid == 0 && c0 == 0 && p.lse) p.lse[row] = kNegInf;
    return;
  }
  const int from = (int)(((u + 1) * G - 1) / total), to = (int)(((u + tiles) * G - 1) / total);
  if (from == to) return;                                  // (written by the one CTA that had it)
  auto slot_of = [&](int cta) { return ((size_t)cta * 2 + (total * cta / G < u)) * NR + r - rb * NR; };
  const int parts = to - from + 1;                         // <= G <= kJoin
  float2 ml = make_float2(kNegInf, 0.f);
  // (with fewer units than CTAs, some of those between have none)
  if (tid < parts && total * (from + tid) / G < total * (from + tid + 1) / G) ml = *reinterpret_cast<const float2*>(p.part_ml + slot_of(from + tid) * 2);
  float top = ml.x;
#pragma unroll
  for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) s_top[warp] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kJoin / 32; ++w) top = fmaxf(top, s_top[w]);
  const float w = ml.x == kNegInf ? 0.f : ex2(ml.x - top);
  s_w[tid] = w;
  float sum = w * ml.y;
#pragma unroll
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_sum[warp] = sum;
  __syncthreads();
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < kJoin / 32; ++i) sum += s_sum[i];
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int i = warp; i < parts; i += kJoin / 32) {
    const float4 x = *reinterpret_cast<const float4*>(p.part_o + slot_of(from + i) * kLatent + c0 + 4 * lane);
    const float f = s_w[i];
    if (f > 0.f) {                                         // (a part in which the row saw nothing)
      acc.x = fmaf(f, x.x, acc.x); acc.y = fmaf(f, x.y, acc.y); acc.z = fmaf(f, x.z, acc.z); acc.w = fmaf(f, x.w, acc.w);
    }
  }
  s_o[warp][lane] = acc;
  __syncthreads();
  if (tid < 32) {
    float4 o = s_o[0][tid];
#pragma unroll
    for (int i = 1; i < kJoin / 32; ++i) {
      const float4 x = s_o[i][tid];
      o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    *reinterpret_cast<uint2*>(out + 4 * tid) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    if (tid == 0 && c0 == 0 && p.lse) p.lse[row] = sum > 0.f ? (top + log2f(sum)) * 0.6931471805599453f : kNegInf;
  }
}

// Query rows to a CTA
int rows_for(const TokenParams& p) { return p.T * p.H <= 16 ? 16 : 32; }

template <int NR> cudaError_t launch(const TokenParams& p, const CUtensorMap& map_c, int ctas, cudaStream_t stream) {
  typedef unsigned long long u64;
  const u64 rows = (u64)p.N * p.T * p.H;
  const u64 size[4] = {64, rows, 9, 1}, stride[3] = {kRow * 2, 128, 128};
  const unsigned q_box[4] = {64, NR, 9, 1};
  CUtensorMap map_q;
  if (!make_map_4d(&map_q, p.q, size, stride, q_box)) return cudaErrorInvalidValue;
  cudaError_t e = allow_smem<latent_token_tc_kernel<NR>>(Cfg<NR>::kSmem);
  if (e == cudaSuccess) e = start(latent_token_tc_kernel<NR>, dim3((unsigned)ctas), kThreads, Cfg<NR>::kSmem, stream, map_q, map_c, p);
  return e == cudaSuccess ? start(latent_join_kernel, dim3((unsigned)(rows * 4)), kJoin, 0, stream, p, NR, ctas) : e;
}

int ctas() { return std::min(sm_count(), kJoin); }

}  // namespace

size_t token_tc_bytes(const TokenParams& p) { return align_up((size_t)ctas() * 2 * rows_for(p) * (kLatent + 2) * 4, 256); }

cudaError_t launch_token_tc(const TokenParams& given, void* workspace, cudaStream_t stream) {
  typedef unsigned long long u64;
  TokenParams p = given;
  p.part_o = reinterpret_cast<float*>(workspace);
  p.part_ml = p.part_o + (size_t)ctas() * 2 * rows_for(p) * kLatent;
  const unsigned box = (unsigned)std::min(1 << p.page_log, 128);
  const u64 size[4] = {64, std::max<u64>((u64)p.pages << p.page_log, 1), 9, 1}, stride[3] = {kRow * 2, 128, 128};
  const unsigned tile[4] = {64, box, 1, 1};
  CUtensorMap map_c;
  // (no page: no row to read, any address will do for the map)
  if (!make_map_4d(&map_c, p.pages > 0 ? p.cache : p.q, size, stride, tile)) return cudaErrorInvalidValue;
  return rows_for(p) == 16 ? launch<16>(p, map_c, ctas(), stream) : launch<32>(p, map_c, ctas(), stream);
}

}  // namespace mix
}  // namespace ha_la

// Attention of new tokens to cached latent rows, tensor cores: bf16, rows of 512 + 64, pages of 16 rows or more.
//
// All heads (and new tokens) of a sequence read the same rows, whose first 512 values are keys and values at once, so a row is brought once for up to 64
// query rows and HBM bounds it: 1152 bytes a row, 2 x 1088 multiply-adds a query row.  What fills a matrix instruction's rows are not the queries, of
// which there may be sixteen, but the cache's rows and the latent channels:
//   S^T = C q^T     (64 cached rows x NR queries; nine chunks of 64 channels)
//   O^T += V^T P^T  (4 x 128 channels x NR queries; V = the first eight chunks of C, read the other way round from the same shared memory)
// with P^T through shared memory.  A softmax thread has a cached row (lanes 0 .. 15 of four warps, which is where a product of 64 rows leaves them), so a
// query's maximum is spread over 64 threads: they take the exact one for a segment's first rows and whenever a score exceeds it by 2^8 (one vote), and
// each adds up its own weights until the end.
// The scores of the next 64 rows are made ahead of the products with these rows' values, and shared memory holds two to two and a half such tiles: copies are
// under way all the time.  (64 contexts of 500 to 16000 rows, 32 heads: 122 to 126 us a call; 128 rows at a time, of which shared memory holds one and a quarter, 156.)
// Tiles that follow one another take an SM 1.76 us each, 6.2 TB/s over all SMs (148 contexts of 8192 rows less 148 of 4096, with 16 heads 1.63, with 64 2.15); 45.6 of them an
// SM are 80 us of those 64 contexts'.  The rest is what a call has once: two launches, lengths and pages looked up, the first tiles, which come one by one, and the parts'
// joining, 10 us by itself.  (One tile an SM: 22 us a call.)
//
// Work is cut into units of 64 rows of all sequences one behind the other, in equal parts for the CTAs, one an SM: long and short contexts, few or many,
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

constexpr int kThreads = 192, kTile = 64, kLatent = 512, kRow = 576;      // threads: softmax, copies, products
constexpr int kAhead = 2;                                  // tiles on their way to L2 or further (one: 130 us a call, three 125, four 132: the copy engine does this too)
constexpr uint32_t kChunkB = 8192, kPairB = 2 * kChunkB;   // 64 rows x 64 channels; two of them

template <int NR> struct Cfg {
  static constexpr int kPairs = NR == 64 ? 8 : 10, kRopes = NR == 64 ? 1 : 2;   // slots of 128 channels, of the positional ones
  static constexpr uint32_t kPRow = NR * 2, kPB = kTile * kPRow;
  static constexpr uint32_t OFF_ROPE = kPairs * kPairB, OFF_Q = OFF_ROPE + kRopes * kChunkB, OFF_P = OFF_Q + NR * 1152, OFF_BAR = OFF_P + 2 * kPB;
  static constexpr size_t kSmem = OFF_BAR + 320;
  static constexpr uint32_t kTmO = 0, kTmS = 4 * NR, kTmCols = NR == 64 ? 512 : NR == 32 ? 256 : 128;
  // P^T: a cached row's weights side by side, NR bf16 values, swizzled over that width
  static constexpr uint64_t kSwizzle = NR == 64 ? kSwizzle128B : NR == 32 ? kSwizzle64B : kSwizzle32B;
  static constexpr uint32_t kIdS = idesc_bf16(kTile, NR, false, false), kIdO = idesc_bf16(128, NR, true, true);
};

__device__ __forceinline__ int units_of(const TokenParams& p, int n) { return (rows_of(p, n) + kTile - 1) / kTile; }

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

// Largest (or sum) of v[j] over the lanes of a warp: that of column j in v[j / 32] of lane j % 32 (NR 16: in lanes j and j + 16).
template <int NR, bool MAX> __device__ __forceinline__ void spread(float (&v)[NR]) {
  const int lane = threadIdx.x & 31;
  auto join = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
  constexpr int W = NR < 32 ? NR : 32;
#pragma unroll
  for (int h = 0; h < NR / W; ++h) {
    float* const w = v + h * W;
#pragma unroll
    for (int off = W / 2; off; off >>= 1) {
      const bool up = lane & off;
#pragma unroll
      for (int j = 0; j < off; ++j) {
        const float keep = up ? w[j + off] : w[j], send = up ? w[j] : w[j + off];
        w[j] = join(keep, __shfl_xor_sync(0xffffffffu, send, off));
      }
    }
    if (W == 16) w[0] = join(w[0], __shfl_xor_sync(0xffffffffu, w[0], 16));
    v[h] = w[0];
  }
}

template <int NR> __device__ __forceinline__ void load_columns(uint32_t at, uint32_t (&r)[NR]) {
  if constexpr (NR == 16) {
    tmem_ld16(at, r);
  } else {
#pragma unroll
    for (int c = 0; c < NR; c += 32) tmem_ld32(at + c, *reinterpret_cast<uint32_t(*)[32]>(r + c));
  }
  tmem_ld_wait();
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
  constexpr int kPairs = C::kPairs, kRopes = C::kRopes;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* const sm = smem;
  __shared__ int s_n;
  __shared__ long long s_base, s_scan[kThreads / 32];
  __shared__ __align__(16) float s_m[NR], s_f[NR], s_red[4][NR];
  uint64_t* const bar = reinterpret_cast<uint64_t*>(sm + C::OFF_BAR);
  uint64_t *const q_full = bar, *const q_free = bar + 1, *const added = bar + 2, *const scores = bar + 4, *const rope_full = bar + 6, *const rope_free = rope_full + kRopes;
  uint64_t *const pair_full = rope_free + kRopes, *const pair_free = pair_full + kPairs, *const weights = pair_free + kPairs;      // weights: [2]
  constexpr int kBars = 6 + 2 * kRopes + 2 * kPairs + 2;
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bar + kBars);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  static_assert(kBars * 8 + 8 <= 320, "barriers");
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
  const int page = 1 << p.page_log, box = min(page, kTile), boxes = kTile / box;   // rows of a copy, copies for a tile's rows

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
        const int j = t * kTile + lane % boxes * box;
        return t < walk.t1 && j < len ? (int)cache_row(p, walk.n, j) : -1;
      };
      // A tile's rows lie together (page by page), its copies take 128 bytes of each at a time: brought to L2 as they lie, some tiles ahead.
      auto ahead = [&](int row) {
        if (lane < boxes && row >= 0)
          asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(reinterpret_cast<const uint8_t*>(p.cache) + (size_t)row * (kRow * 2)), "r"(box * kRow * 2) : "memory");
      };
      int rows_ahead[kAhead];                              // of tiles t, t + 1, ..
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        rows_ahead[i] = row_at(walk.t0 + i);
        if (i > 0) ahead(rows_ahead[i]);
      }
      for (int t = walk.t0; t < walk.t1; ++t, ++tile) {
        const int row = rows_ahead[0], next = row_at(t + kAhead), have = min(boxes, (min(len - t * kTile, kTile) + box - 1) / box), r = tile % kRopes;
        if (tile >= kRopes) wait_for(&rope_free[r], (tile / kRopes - 1) & 1, abort_flag);
        __syncwarp();
        if (*abort_flag) break;
        if (lane == 0) mbar_expect_tx(&rope_full[r], (uint32_t)(have * box) * 128);
        __syncwarp();
        if (lane < have) tma_load_4d(sm + C::OFF_ROPE + r * kChunkB + lane * box * 128, &map_c, &rope_full[r], 0, row, 8, 0);
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
            tma_load_4d(sm + slot * kPairB + half * kChunkB + lane % boxes * box * 128, &map_c, &pair_full[slot], 0, row, 2 * b + half, 0);
          __syncwarp();
        }
        ahead(next);
#pragma unroll
        for (int i = 1; i < kAhead; ++i) rows_ahead[i - 1] = rows_ahead[i];
        rows_ahead[kAhead - 1] = next;
      }
      ++seg;
      if (*abort_flag) break;
    }
  } else if (warp == 5) {
    // ------------------------------------------------------------ products
    if (elect_one()) {
      const uint32_t sq = smem_u32(sm + C::OFF_Q), rope = smem_u32(sm + C::OFF_ROPE);
      auto part = [&](uint32_t d, uint32_t chunk, int c, bool add) {      // 64 channels' share of the scores
        const uint64_t da = gla::desc_cols(chunk), db = smem_desc(sq + c * NR * 128, 16, 1024, kSwizzle128B);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) umma_ss(d, da + 2 * ks, db + 2 * ks, C::kIdS, add || ks > 0);
      };
      auto make_scores = [&](int i) {                      // of the CTA's tile i
        const uint32_t d = tm + C::kTmS + NR * (i & 1);
        const int r = i % kRopes;
        wait_for(&rope_full[r], (i / kRopes) & 1, abort_flag);
        tc_fence_after_sync();
        part(d, rope + r * kChunkB, 8, false);
        umma_commit(&rope_free[r]);
        for (int b = 0; b < 4; ++b) {
          const int x = i * 4 + b, slot = x % kPairs;
          wait_for(&pair_full[slot], (x / kPairs) & 1, abort_flag);
          tc_fence_after_sync();
          part(d, smem_u32(sm + slot * kPairB), 2 * b, true);
          part(d, smem_u32(sm + slot * kPairB) + kChunkB, 2 * b + 1, true);
        }
        umma_commit(&scores[i & 1]);
      };
      auto add_values = [&](int i, bool start) {           // (a segment's first weights come once the softmax warps have read O)
        wait_for(&weights[i & 1], (i >> 1) & 1, abort_flag);
        tc_fence_after_sync();
        const uint64_t dp = smem_desc(smem_u32(sm + C::OFF_P) + (i & 1) * C::kPB, 16, 8 * C::kPRow, C::kSwizzle);
        for (int b = 0; b < 4; ++b) {
          const int slot = (i * 4 + b) % kPairs;
          const uint64_t da = smem_desc(smem_u32(sm + slot * kPairB), kChunkB, 1024, kSwizzle128B);
#pragma unroll
          for (int ks = 0; ks < kTile / 16; ++ks)
            umma_ss(tm + C::kTmO + NR * b, da + gla::step_rows(ks), dp + ((ks * 16 * C::kPRow) >> 4), C::kIdO, !start || ks > 0);
          umma_commit(&pair_free[slot]);
        }
        umma_commit(&added[i & 1]);
      };
      int seg = 0, tile = 0;
      while (walk.next(p)) {
        wait_for(q_full, seg & 1, abort_flag);
        make_scores(tile);
        for (int t = walk.t0; t < walk.t1; ++t, ++tile) {
          if (t + 1 < walk.t1) make_scores(tile + 1);
          else umma_commit(q_free);
          if (*abort_flag) break;
          add_values(tile, t == walk.t0);
        }
        if (*abort_flag) break;
        ++seg;
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax: a thread to a cached row, lanes 0 .. 15
    const int row = 16 * warp + (lane & 15);
    const bool mine = lane < 16;
    const uint32_t lanes = static_cast<uint32_t>(32 * warp) << 16;
    const float to_log2 = p.scale * kLog2e;
    int seg = 0, tile = 0;
    while (walk.next(p)) {
      const int len = rows_of(p, walk.n), r0 = walk.rb * NR, rows = min(NR, all_rows - r0), low = len - p.T + 1;
      float l[NR];
#pragma unroll
      for (int r = 0; r < NR; ++r) l[r] = 0.f;
      // (columns behind the sequence's hold another's queries: nothing exceeds their maximum, so they have no say in when this one is rescaled)
      if (tid < NR) s_m[tid] = tid < rows ? kNegInf : INFINITY;
      softmax_sync();
      for (int t = walk.t0; t < walk.t1; ++t, ++tile) {
        wait_for(&scores[tile & 1], (tile >> 1) & 1, abort_flag);
        __syncwarp();
        tc_fence_after_sync();
        uint32_t raw[NR];
        load_columns<NR>(tm + C::kTmS + NR * (tile & 1) + lanes, raw);
        const int j = t * kTile + row;
        float s[NR];
        const bool partly = (t + 1) * kTile > low + (p.T > 1 ? r0 / p.H : 0);   // (of the block's first token)
#pragma unroll
        for (int r = 0; r < NR; ++r) s[r] = mine ? __uint_as_float(raw[r]) * to_log2 : kNegInf;
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
          spread<NR, true>(v);
#pragma unroll
          for (int h = 0; h < (NR + 31) / 32; ++h)
            if (lane < NR) s_red[warp][32 * h + lane] = v[h];
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
            // (these scores stood behind the values of the tile two back, so this barrier is in its phase)
            wait_for(&added[(tile - 1) & 1], ((tile - 1) >> 1) & 1, abort_flag);
            __syncwarp();
            tc_fence_after_sync();
#pragma unroll 1
            for (int c = 0; c < 4 * NR; c += 16) {
              uint32_t o[16];
              tmem_ld16(tm + C::kTmO + c + lanes, o);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * s_f[c % NR + e]);
              tmem_st16(tm + C::kTmO + c + lanes, o);
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
        if (mine) {
#pragma unroll
          for (int c = 0; c < NR / 8; ++c) {
            const uint32_t at = NR == 64 ? sw128_offset(row, c) : NR == 32 ? sw64_offset(row, c) : static_cast<uint32_t>(row * 32 + ((c ^ ((row >> 2) & 1)) << 4));
            *reinterpret_cast<uint4*>(sm + C::OFF_P + (tile & 1) * C::kPB + at) = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
          }
        }
        const int have = len - t * kTile;
        if (have < kTile) {                                // rows that are not the sequence's may be NaN, which no weight of zero masks
          for (int i = tid; i < (kTile - have) * 64; i += 128) {   // 16 bytes of chunk i / 8 % 8 and its rows
            const int chunk = (i >> 3) & 7;
            *reinterpret_cast<uint4*>(sm + (tile * 4 + (chunk >> 1)) % kPairs * kPairB + (chunk & 1) * kChunkB + (have + (i >> 6)) * 128 + (i & 7) * 16) =
                make_uint4(0u, 0u, 0u, 0u);
          }
        }
        fence_proxy_async_smem();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&weights[tile & 1]);
        __syncwarp();
      }
      spread<NR, false>(l);
#pragma unroll
      for (int h = 0; h < (NR + 31) / 32; ++h)
        if (lane < NR) s_red[warp][32 * h + lane] = l[h];
      softmax_sync();
      if (tid < NR) s_f[tid] = (s_red[0][tid] + s_red[1][tid]) + (s_red[2][tid] + s_red[3][tid]);
      softmax_sync();
      const bool whole = walk.t0 == 0 && walk.t1 == walk.tiles;
      const size_t q_row = (size_t)walk.n * all_rows + r0, slot = ((size_t)blockIdx.x * 2 + (seg > 0)) * NR;
      wait_for(&added[(tile - 1) & 1], ((tile - 1) >> 1) & 1, abort_flag);
      __syncwarp();
      tc_fence_after_sync();
#pragma unroll 1
      for (int c = 0; c < 4 * NR; c += 16) {
        uint32_t o[16];
        tmem_ld16(tm + C::kTmO + c + lanes, o);
        tmem_ld_wait();
        const int channel = 128 * (c / NR) + tid;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int r = c % NR + e;
          if (r >= rows) break;
          const float x = __uint_as_float(o[e]);
          if (whole) reinterpret_cast<__nv_bfloat16*>(p.o)[(q_row + r) * kLatent + channel] = __float2bfloat16_rn(s_f[r] > 0.f ? x / s_f[r] : 0.f);
          else p.part_o[(slot + r) * kLatent + channel] = x;
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

// Joins the parts of a sequence's query rows that several CTAs have made, in order.  WARPS to a row share the parts out: all eight of a CTA, 128 channels to a
// CTA, where a few sequences have been cut into many parts; one, with all channels, where many have been cut into a few (64 contexts: 41 us the first way).
constexpr int kJoin = 256, kJoinWarps = kJoin / 32;
template <int WARPS>
__global__ void __launch_bounds__(kJoin) latent_join_kernel(TokenParams p, int NR, int G) {
  constexpr int ROWS = kJoinWarps / WARPS, Q = WARPS == 1 ? 4 : 1;         // rows of a CTA; 128 channels that a warp has
  __shared__ float s_w[ROWS][kJoin], s_top[kJoinWarps], s_sum[kJoinWarps];
  __shared__ __align__(16) float4 s_o[WARPS == 1 ? 1 : kJoinWarps][32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, all_rows = p.T * p.H, blocks = (all_rows + NR - 1) / NR;
  const int per = (all_rows + ROWS - 1) / ROWS * (4 / Q), n = blockIdx.x / per, x = blockIdx.x - n * per;
  const int r = x / (4 / Q) * ROWS + warp / WARPS, c0 = x % (4 / Q) * 128, rb = min(r, all_rows - 1) / NR;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const Count c = count_units<kJoin>(p, n);
  const long long total = c.all * blocks, tiles = units_of(p, n), u = c.before * blocks + rb * tiles;
  const bool mine = r < all_rows;
  const size_t row = (size_t)n * all_rows + r;
  __nv_bfloat16* const out = reinterpret_cast<__nv_bfloat16*>(p.o) + row * kLatent + c0 + 4 * lane;
  const bool first = warp % WARPS == 0 && mine;            // the warp that writes
  if (tiles == 0) {
    if (first) {
#pragma unroll
      for (int k = 0; k < Q; ++k) *reinterpret_cast<uint2*>(out + 128 * k) = make_uint2(0u, 0u);
      if (lane == 0 && c0 == 0 && p.lse) p.lse[row] = kNegInf;
    }
    return;
  }
  // CTA i had the units from total i / G on; with fewer units than CTAs some had none
  const int from = (int)(((u + 1) * G - 1) / total), to = (int)(((u + tiles) * G - 1) / total), parts = to - from + 1;    // <= G <= kJoin
  const bool split = mine && from < to;                    // (else written by the one CTA that had it)
  const size_t in = r - rb * NR, slot0 = ((size_t)from * 2 + (total * from / G < u)) * NR + in;
  auto slot_of = [&](int i) { return i == 0 ? slot0 : (size_t)(from + i) * 2 * NR + in; };
  float top = kNegInf, sum = 0.f;
  if constexpr (WARPS == 1) {
    if (!split) return;
    for (int i = lane; i < parts; i += 32) {
      float2 ml = make_float2(kNegInf, 0.f);
      if (total * (from + i) / G < total * (from + i + 1) / G) ml = *reinterpret_cast<const float2*>(p.part_ml + slot_of(i) * 2);
      const float next = fmaxf(top, ml.x);
      sum = next == kNegInf ? 0.f : sum * ex2(top - next) + ml.y * ex2(ml.x - next);
      top = next;
      s_w[warp][i] = ml.x;
    }
    const float mine_top = top;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    sum *= mine_top == kNegInf ? 0.f : ex2(mine_top - top);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    for (int i = lane; i < parts; i += 32) s_w[warp][i] = s_w[warp][i] == kNegInf ? 0.f : ex2(s_w[warp][i] - top);
    __syncwarp();
  } else {
    float2 ml = make_float2(kNegInf, 0.f);
    if (split && tid < parts && total * (from + tid) / G < total * (from + tid + 1) / G) ml = *reinterpret_cast<const float2*>(p.part_ml + slot_of(tid) * 2);
    top = ml.x;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) s_top[warp] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) top = fmaxf(top, s_top[w]);
    const float w = ml.x == kNegInf ? 0.f : ex2(ml.x - top);
    s_w[0][tid] = w;
    sum = w * ml.y;
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < kJoinWarps; ++i) sum += s_sum[i];
    if (!split) return;                                    // (all of the CTA: it has one row)
  }
  float4 acc[Q] = {};
  const float* const weight = s_w[warp / WARPS];
#pragma unroll 4
  for (int i = warp % WARPS; i < parts; i += WARPS) {
    const float f = weight[i];
    if (f > 0.f) {                                         // (else the row saw nothing there, or there is no such part)
      const float* const from_part = p.part_o + slot_of(i) * kLatent + c0 + 4 * lane;
#pragma unroll
      for (int k = 0; k < Q; ++k) {
        const float4 y = *reinterpret_cast<const float4*>(from_part + 128 * k);
        acc[k].x = fmaf(f, y.x, acc[k].x); acc[k].y = fmaf(f, y.y, acc[k].y); acc[k].z = fmaf(f, y.z, acc[k].z); acc[k].w = fmaf(f, y.w, acc[k].w);
      }
    }
  }
  if constexpr (WARPS > 1) {
    s_o[warp][lane] = acc[0];
    __syncthreads();
    if (!first) return;
#pragma unroll
    for (int i = 1; i < kJoinWarps; ++i) {
      const float4 y = s_o[i][lane];
      acc[0].x += y.x; acc[0].y += y.y; acc[0].z += y.z; acc[0].w += y.w;
    }
  }
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
  for (int k = 0; k < Q; ++k) *reinterpret_cast<uint2*>(out + 128 * k) = make_uint2(pack_bf16(acc[k].x * inv, acc[k].y * inv), pack_bf16(acc[k].z * inv, acc[k].w * inv));
  if (lane == 0 && c0 == 0 && p.lse) p.lse[row] = sum > 0.f ? (top + log2f(sum)) * 0.6931471805599453f : kNegInf;
}

// Query rows to a CTA: as few blocks of them as there can be, for each reads the cache once more
int rows_for(const TokenParams& p) { return p.T * p.H <= 16 ? 16 : p.T * p.H <= 32 ? 32 : 64; }

template <int NR> cudaError_t launch(const TokenParams& p, const CUtensorMap& map_c, int ctas, cudaStream_t stream) {
  typedef unsigned long long u64;
  const u64 rows = (u64)p.N * p.T * p.H;
  const u64 size[4] = {64, rows, 9, 1}, stride[3] = {kRow * 2, 128, 128};
  const unsigned q_box[4] = {64, NR, 9, 1};
  CUtensorMap map_q;
  if (!make_map_4d(&map_q, p.q, size, stride, q_box)) return cudaErrorInvalidValue;
  cudaError_t e = allow_smem<latent_token_tc_kernel<NR>>(Cfg<NR>::kSmem);
  if (e == cudaSuccess) e = start(latent_token_tc_kernel<NR>, dim3((unsigned)ctas), kThreads, Cfg<NR>::kSmem, stream, map_q, map_c, p);
  if (e != cudaSuccess) return e;
  // (parts to a row, where lengths are alike: CTAs over query blocks)
  const long long blocks = (long long)p.N * ((p.T * p.H + NR - 1) / NR), all = p.T * p.H;
  return blocks * 16 <= ctas ? start(latent_join_kernel<kJoinWarps>, dim3((unsigned)(rows * 4)), kJoin, 0, stream, p, NR, ctas)
                             : start(latent_join_kernel<1>, dim3((unsigned)(p.N * ((all + kJoinWarps - 1) / kJoinWarps))), kJoin, 0, stream, p, NR, ctas);
}

int ctas() { return std::min(sm_count(), kJoin); }

}  // namespace

size_t token_tc_bytes(const TokenParams& p) { return align_up((size_t)ctas() * 2 * rows_for(p) * (kLatent + 2) * 4, 256); }

cudaError_t launch_token_tc(const TokenParams& given, void* workspace, cudaStream_t stream) {
  typedef unsigned long long u64;
  TokenParams p = given;
  p.part_o = reinterpret_cast<float*>(workspace);
  p.part_ml = p.part_o + (size_t)ctas() * 2 * rows_for(p) * kLatent;
  const unsigned box = (unsigned)std::min(1 << p.page_log, kTile);
  const u64 size[4] = {64, std::max<u64>((u64)p.pages << p.page_log, 1), 9, 1}, stride[3] = {kRow * 2, 128, 128};
  const unsigned tile[4] = {64, box, 1, 1};
  CUtensorMap map_c;
  // (no page: no row to read, any address will do for the map)
  if (!make_map_4d(&map_c, p.pages > 0 ? p.cache : p.q, size, stride, tile)) return cudaErrorInvalidValue;
  return rows_for(p) == 16 ? launch<16>(p, map_c, ctas(), stream) : rows_for(p) == 32 ? launch<32>(p, map_c, ctas(), stream) : launch<64>(p, map_c, ctas(), stream);
}

}  // namespace mix
}  // namespace ha_la

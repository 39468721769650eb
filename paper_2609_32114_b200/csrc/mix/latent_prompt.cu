// Attention of a prompt on expanded keys and values, tensor cores: bf16, 128 + 64 key channels, 128 value channels.
//
// A CTA has 128 TILES queries of a head and goes through the keys 128 at a time: S = Q K^T (128 x 128, twelve steps of 16 channels, the last four of
// them on the positional key that all heads share), P = 2^(S - m) in bf16 over S's place in tensor memory, O += P V with P as the operand from there.
// With two tiles of queries the tensor cores work on one while the softmax warps, a thread to a query, are on the other's scores: the products of
// both are 2560 cycles a round, their exponentials 2048, and K and V are read once for 256 queries.  A round takes some 4700, all that is around the rounds
// included (4096 tokens, 32 heads: 275,000 cycles for 58.8 of them an SM, the tensor cores busy for 53 %): a tile's scores, softmax and values wait for each other.  8192 tokens,
// 32 heads: 580 us, 1184 TFLOP/s of the causal half; 684 after some seconds of nothing else, when the power cap holds the clocks at 1580 MHz.
// m need not be the largest score, only near it: O and l are rescaled when a score exceeds m by 2^8, which after the first keys is rare, so O is hardly
// ever read back.  P <= 2^8 loses nothing in bf16, and l adds up the weights as they are before that rounding, in fp32.
#include <algorithm>

#include "latent.cuh"
#include "../gla/tc.cuh"

namespace ha_la {

bool make_map_4d(CUtensorMap* m, const void* base, const unsigned long long (&size)[4], const unsigned long long (&stride)[3], const unsigned (&tile)[4]);   // tc.cu

namespace mix {
namespace {

using namespace ptx;
using gla::wait_for;

constexpr uint32_t kQB = 49152, kKB = 49152, kVB = 32768, kRopeAt = 32768;
constexpr uint32_t kTmS = 0, kTmO = 256;                   // columns: S (and P) of tile t at 128 t, O at 256 + 128 t

template <int TILES> struct Cfg {
  static constexpr int kSoft = 4 * TILES, kThreads = 32 * (kSoft + 2), kVStages = TILES == 1 ? 2 : 1;
  static constexpr uint32_t OFF_K = TILES * kQB, OFF_V = OFF_K + 2 * kKB, OFF_BAR = OFF_V + kVStages * kVB;
  static constexpr size_t kSmem = OFF_BAR + 256;
};

struct Range { int q0, q, k0, k, r0; };                    // a sequence's queries and keys, the CTA's first query
// Keys that query i sees, and steps of 128 keys for the queries of tile t.
__device__ __forceinline__ int seen_by(const Range& g, int i) { return max(0, min(g.k, g.k - g.q + 1 + i)); }
__device__ __forceinline__ int steps_of(const Range& g, int t) {
  const int first = g.r0 + 128 * t;
  return first < g.q ? (seen_by(g, min(first + 127, g.q - 1)) + 127) / 128 : 0;
}

template <int TILES>
__global__ void __launch_bounds__(Cfg<TILES>::kThreads, 1)
latent_prompt_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_kn, const __grid_constant__ CUtensorMap map_kr,
                        const __grid_constant__ CUtensorMap map_v, PromptParams p) {
  using C = Cfg<TILES>;
  constexpr int VS = C::kVStages;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* const sm = smem;
  uint64_t* const bar = reinterpret_cast<uint64_t*>(sm + C::OFF_BAR);
  uint64_t* const q_full = bar;                            // [TILES]
  uint64_t* const k_full = q_full + TILES;                 // [2]
  uint64_t* const k_free = k_full + 2;                     // [2]
  uint64_t* const v_full = k_free + 2;                     // [VS]
  uint64_t* const v_free = v_full + VS;                    // [VS]
  uint64_t* const scores = v_free + VS;                    // [TILES]
  uint64_t* const added = scores + TILES;                  // [TILES] P V is in O
  uint64_t* const weights = added + TILES;                 // [TILES] by the four softmax warps of the tile
  constexpr int kBars = 3 * TILES + 4 + 2 * VS + TILES;
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bar + kBars);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int nh = p.q_seqs.N * p.H, b = p.blocks - 1 - (int)(blockIdx.x / nh), n = (int)(blockIdx.x % nh) / p.H, h = (int)(blockIdx.x % nh) % p.H;
  if (tid == 0) {
    for (int i = 0; i < kBars; ++i) mbar_init(&bar[i], &bar[i] >= weights ? 4 : 1);
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 0) tmem_alloc(tmem_slot, 512);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tm = *tmem_slot;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0) check_spans(p);
  const Span s = span_of(p, n);
  const Range g = {s.q0, s.q, s.k0, s.k, b * 128 * TILES};
  int steps[TILES], most = 0;
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    steps[t] = steps_of(g, t);
    most = max(most, steps[t]);
  }

  if (warp == C::kSoft) {
    // ------------------------------------------------------------ tiles
    if (elect_one()) {
      if (most > 0) {
#pragma unroll
        for (int t = 0; t < TILES; ++t)
          if (steps[t] > 0) {
            mbar_expect_tx(&q_full[t], kQB);
            tma_load_4d(sm + t * kQB, &map_q, &q_full[t], 0, g.q0 + g.r0 + 128 * t, 0, h);
          }
      }
      auto keys = [&](int i) {
        const int st = i & 1;
        if (i >= 2) wait_for(&k_free[st], ((i >> 1) - 1) & 1, abort_flag);
        if (*abort_flag) return;
        mbar_expect_tx(&k_full[st], kKB);
        tma_load_4d(sm + C::OFF_K + st * kKB, &map_kn, &k_full[st], 0, g.k0 + 128 * i, 0, h);
        tma_load_4d(sm + C::OFF_K + st * kKB + kRopeAt, &map_kr, &k_full[st], 0, g.k0 + 128 * i, 0, 0);
      };
      if (most > 0) keys(0);
      for (int i = 0; i < most; ++i) {
        if (i + 1 < most) keys(i + 1);
        const int st = i % VS;
        if (i >= VS) wait_for(&v_free[st], ((i / VS) - 1) & 1, abort_flag);
        if (*abort_flag) break;
        mbar_expect_tx(&v_full[st], kVB);
        tma_load_4d(sm + C::OFF_V + st * kVB, &map_v, &v_full[st], 0, g.k0 + 128 * i, 0, h);
      }
    }
    __syncwarp();
  } else if (warp == C::kSoft + 1) {
    // ------------------------------------------------------------ products
    if (elect_one()) {
      auto make_scores = [&](int t, int i) {
        const uint64_t dq = gla::desc_cols(smem_u32(sm + t * kQB)), dk = gla::desc_cols(smem_u32(sm + C::OFF_K + (i & 1) * kKB));
#pragma unroll
        for (int ks = 0; ks < 12; ++ks) umma_ss(tm + kTmS + 128 * t, dq + gla::step_cols(ks), dk + gla::step_cols(ks), gla::kIdCols, ks > 0);
        umma_commit(&scores[t]);
      };
      if (most > 0) wait_for(&k_full[0], 0, abort_flag);
#pragma unroll
      for (int t = 0; t < TILES; ++t)
        if (steps[t] > 0) {
          wait_for(&q_full[t], 0, abort_flag);
          tc_fence_after_sync();
          make_scores(t, 0);
        }
      if (most > 0) umma_commit(&k_free[0]);
      for (int i = 0; i < most; ++i) {
        wait_for(&v_full[i % VS], (i / VS) & 1, abort_flag);
        bool keys_there = false;
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
          if (i >= steps[t]) continue;
          wait_for(&weights[t], i & 1, abort_flag);
          if (*abort_flag) break;
          tc_fence_after_sync();
          gla::mma_tmem_rows(tm + kTmO + 128 * t, tm + kTmS + 128 * t, smem_u32(sm + C::OFF_V + (i % VS) * kVB), i > 0);
          umma_commit(&added[t]);
          if (t == TILES - 1 || i >= steps[TILES - 1]) umma_commit(&v_free[i % VS]);   // (the last that reads these values, and ahead of the next scores)
          if (i + 1 < steps[t]) {
            if (!keys_there) wait_for(&k_full[(i + 1) & 1], ((i + 1) >> 1) & 1, abort_flag);
            keys_there = true;
            tc_fence_after_sync();
            make_scores(t, i + 1);                         // behind the product that reads the weights there, in the tensor cores' order
          }
        }
        if (i + 1 < most) umma_commit(&k_free[(i + 1) & 1]);
        if (*abort_flag) break;
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax: a thread to a query
    const int t = warp >> 2, quad = warp & 3, row = 32 * quad + lane, i_q = g.r0 + 128 * t + row;
    const int limit = i_q < g.q ? seen_by(g, i_q) : 0;     // (rows of the tile behind the sequence hold another's queries, which have no say in when this one is rescaled)
    const uint32_t lanes = static_cast<uint32_t>(32 * quad) << 16, S = tm + kTmS + 128 * t + lanes, O = tm + kTmO + 128 * t + lanes;
    const float to_log2 = p.scale * 1.4426950408889634f;
    const int count = t == 0 ? steps[0] : steps[TILES - 1];
    float m = kNegInf, l = 0.f;
    for (int i = 0; i < count; ++i) {
      wait_for(&scores[t], i & 1, abort_flag);
      __syncwarp();
      tc_fence_after_sync();
      uint32_t raw[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32(S + 32 * c, raw[c]);
      tmem_ld_wait();
      const int lim = limit - 128 * i;
      if (__any_sync(0xffffffffu, lim < 128)) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int e = 0; e < 32; ++e) raw[c][e] = 32 * c + e < lim ? raw[c][e] : 0xff800000u;
      }
      // Weights by the m of before, the scores' maximum on the side; where that m will not do any more, which after the first keys is rare, once more by the new one.
      float2 sum;
      float top;
      auto weigh = [&](float base) {
        float2 part[2] = {};
        float tops[2] = {kNegInf, kNegInf};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float2 s = as_f2(raw[c][e], raw[c][e + 1]);
            tops[(e >> 1) & 1] = fmaxf(tops[(e >> 1) & 1], fmaxf(s.x, s.y));
            const float2 x = fma2(s, make_float2(to_log2, to_log2), make_float2(-base, -base));
            const float2 y = make_float2(ex2(x.x), ex2(x.y));
            part[(e >> 1) & 1] = add2(part[(e >> 1) & 1], y);
            w[e / 2] = pack_bf16(y);
          }
          tmem_st16(S + 16 * c, w);
        }
        sum = add2(part[0], part[1]);
        top = fmaxf(tops[0], tops[1]) * to_log2;
      };
      if (i == 0) {
        float tops[4] = {kNegInf, kNegInf, kNegInf, kNegInf};
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int e = 0; e < 32; ++e) tops[e & 3] = fmaxf(tops[e & 3], __uint_as_float(raw[c][e]));
        m = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * to_log2;
      }
      weigh(m == kNegInf ? 0.f : m);
      if (__any_sync(0xffffffffu, top > m + 8.f)) {
        const float next = fmaxf(m, top), f = m == kNegInf ? 0.f : ex2(m - next);
        m = next;
        l *= f;
        if (i > 0) {
          wait_for(&added[t], (i - 1) & 1, abort_flag);
          __syncwarp();
          tc_fence_after_sync();
#pragma unroll 1
          for (int c = 0; c < 8; ++c) {
            uint32_t o[16];
            tmem_ld16(O + 16 * c, o);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            tmem_st16(O + 16 * c, o);
          }
        }
        weigh(m == kNegInf ? 0.f : m);
      }
      l += sum.x + sum.y;
      tmem_st_wait();
      const int keys = g.k - 128 * i;                      // what lies behind the sequence may be NaN, which no weight of zero masks
      if (keys < 128) {
        wait_for(&v_full[i % VS], (i / VS) & 1, abort_flag);
        gla::clear_rows(sm + C::OFF_V + (i % VS) * kVB, keys, tid & 127, 128);
        fence_proxy_async_smem();
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&weights[t]);
      __syncwarp();
    }
    if (count > 0) wait_for(&added[t], (count - 1) & 1, abort_flag);
    __syncwarp();
    tc_fence_after_sync();
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const int rows = min(128, g.q - g.r0 - 128 * t);       // of this tile
    __nv_bfloat16* const out = reinterpret_cast<__nv_bfloat16*>(p.o) + ((size_t)(g.q0 + g.r0 + 128 * t) * p.H + h) * 128;
#pragma unroll 1
    for (int c = 0; c < 4; ++c) {
      uint32_t o[32];
      if (count > 0) {
        tmem_ld32(O + 32 * c, o);
        tmem_ld_wait();
      }
      uint4 v[4];
#pragma unroll
      for (int e = 0; e < 16; ++e)
        (&v[e / 4].x)[e % 4] = count > 0 ? pack_bf16(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv) : 0u;
      gla::exchange4(v, lane);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 32 * quad + (lane & ~3) + e;
        if (r < rows) *reinterpret_cast<uint4*>(out + (size_t)r * p.H * 128 + 32 * c + 8 * (lane & 3)) = v[e];
      }
    }
    if (p.lse && row < rows) p.lse[(size_t)(g.q0 + i_q) * p.H + h] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : kNegInf;
  }
  tc_fence_before_sync();
  __syncthreads();
  if (tid == 0 && *abort_flag) report_timeout(p.status);
  __syncthreads();
  if (warp == 0) tmem_dealloc(*tmem_slot, 512);
}

template <int TILES> cudaError_t launch(const CUtensorMap (&m)[4], PromptParams p, cudaStream_t stream) {
  using C = Cfg<TILES>;
  p.blocks = (p.q_seqs.max_len + 128 * TILES - 1) / (128 * TILES);
  const long long grid = (long long)p.blocks * p.q_seqs.N * p.H;
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  const cudaError_t e = allow_smem<latent_prompt_tc_kernel<TILES>>(C::kSmem);
  return e != cudaSuccess ? e : start(latent_prompt_tc_kernel<TILES>, dim3((unsigned)grid), C::kThreads, C::kSmem, stream, m[0], m[1], m[2], m[3], p);
}

}  // namespace

// [token][64 columns] tiles one behind the other, of one head
cudaError_t launch_prompt_tc(const PromptParams& p, cudaStream_t stream) {
  typedef unsigned long long u64;
  const u64 T = p.q_seqs.T_total, K = std::max(p.k_seqs.T_total, 1), H = p.H;
  const unsigned q_box[4] = {64, 128, 3, 1}, k_box[4] = {64, 128, 2, 1}, r_box[4] = {64, 128, 1, 1};
  CUtensorMap m[4];
  // (no key at all: a map of the queries stands in, and is not read)
  const bool none = p.k_seqs.T_total == 0;
  const u64 q_size[4] = {64, T, 3, H}, q_stride[3] = {(u64)p.qs * 2, 128, 384};
  const u64 k_size[4] = {64, K, 2, H}, kn_stride[3] = {(u64)p.kns * 2, 128, (u64)p.kn_hs * 2}, v_stride[3] = {(u64)p.vs * 2, 128, (u64)p.v_hs * 2};
  const u64 r_size[4] = {64, K, 1, 1}, r_stride[3] = {(u64)p.krs * 2, 128, 128};
  if (!make_map_4d(&m[0], p.q, q_size, q_stride, q_box)) return cudaErrorInvalidValue;
  if (none) {
    m[1] = m[2] = m[3] = m[0];
  } else if (!make_map_4d(&m[1], p.kn, k_size, kn_stride, k_box) || !make_map_4d(&m[2], p.kr, r_size, r_stride, r_box) ||
             !make_map_4d(&m[3], p.v, k_size, v_stride, k_box)) {
    return cudaErrorInvalidValue;
  }
  // Two tiles of queries to a CTA where that still gives every SM one; else they are shared out singly.
  const long long pairs = (long long)p.q_seqs.N * p.H * ((p.q_seqs.max_len + 255) / 256);
  return pairs >= sm_count() ? launch<2>(m, p, stream) : launch<1>(m, p, stream);
}

}  // namespace mix
}  // namespace ha_la

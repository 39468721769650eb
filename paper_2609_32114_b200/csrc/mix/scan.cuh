// Selective state space scan (ha_la_scan* in ha_la.h): what its kernels and their host code share.
//
//   delta = softplus(dt + dt_bias)    a = e^{delta A}    u = delta x    h_t = a_t h_{t-1} + u_t B_t    p_t = <C_t, h_t> + D x_t    y = p silu(z)
// backwards, with g = dy silu(z) and dh the gradient of h_t from t's output and everything behind it:
//   dh_t = C_t g_t + a_{t+1} dh_{t+1}    f = dh a h_{t-1}    dA = sum_t f delta    ddelta = <f, A> + x <dh, B>    dx = delta <dh, B> + D g
//   dB_t = sum_c dh u    dC_t = sum_c g h_t    dz = dy p silu'(z)    ddt = ddelta softplus'(dt + dt_bias)    dD = sum_t g x
// Every (channel, state) is a recurrence of its own, e^{delta A} differs in all three indices, so nothing of it is a matrix product: a value
// (token, channel, state) costs an exponential (the SM makes 16 a cycle) and four multiply-adds (128 a cycle).
#pragma once

#include "mix.cuh"
#include "../tc_mma.cuh"

namespace ha_la {
namespace mix {

struct ScanParams {
  Seqs seqs;
  int C, S, G, per_group;                                  // channels; states; groups; channels to a group
  int blocks;                                              // channel blocks of a group
  int softplus, packed, vec, bc_vec;                       // vec: rows can be read and written several channels at a time; bc_vec: B and C four states
  int seg_log, segs;                                       // tokens to a segment (a power of two) and segments of a row; 31: sequences whole
  long long xs, dts, bs, cs, zs;
  const void *x, *dt, *B, *C_, *z, *dy;
  const float *A, *D, *dt_bias, *h0, *dhT;
  void *y, *dx, *ddt, *dz;
  float *hT, *dh0;
  float *seg_h, *seg_delta, *first;                        // [slot][C][padded S], [slot][C]; h0 of a call that works in place
  float *ckpt;                                             // [slot of 8 tokens][C][padded S]
  float *part_bc;                                          // [channel block][token][2][padded S]
  float *part_a, *part_d;                                  // [sequence][C][S], [sequence][2][C]
  int32_t* status;
};

constexpr int kCkpt = 8, kCkptLog = 3;                     // tokens from one kept state to the next

constexpr float kLn2 = 0.6931471805599453f;

// softplus(v) = max(v, 0) + log1p(e^-|v|), with log1p(e) = 2 artanh(s), s = e / (2 + e) <= 1/3: a small step is as exact as e is, where a logarithm of 1 + e
// would have lost its bits.  artanh(s) / s as a polynomial in s^2 through its Chebyshev points on [0, 1/9], off by 8e-9 with these coefficients.  e itself is off by
// 2^-22 and, its exponent being rounded, |v| 2^-23.6: 1.8e-6 of a step of e^-29, nothing to speak of beside the rest for steps that do something.  (Carrying what the
// exponent loses, or expf, changes no result's error and costs a scan of 4096 tokens 1.3 % and 4 %.)
__device__ __forceinline__ float softplus(float v) {
  const float e = ex2(-fabsf(v) * kLog2e), s = e * reciprocal(2.f + e), q = s * s;
  float r = fmaf(0.14078889f, q, 0.13982579f);
  r = fmaf(r, q, 0.20012298f); r = fmaf(r, q, 0.33333161f); r = fmaf(r, q, 1.f);
  return fmaf(2.f * s, r, fmaxf(v, 0.f));
}

// A step's decay e^{delta A}, with A2 = A log2(e).  ex2 comes out too small on the average, by 2e-8 of itself for exponents of -1/256 to -1 (half of that below, twice as
// much above), and where decays are near one that adds up over all the tokens that a state lasts.  The exponent is raised by as much, where it costs nothing: the average
// is then within 1.2e-8 for all exponents above -1.  Of an exponent of zero 2^x is still exactly one.  (Error of dA, two rows of 2048 tokens, 4096 channels: 1.8e-6 without
// and 0.8e-6 with it; the plain form's exponentials 0.9e-6.)
constexpr float kRaise = 0x1.8p-26f;
__device__ __forceinline__ float decay(float delta, float A2) { return ex2(fmaf(delta, A2, kRaise)); }
__device__ __forceinline__ float2 decay2(float delta, float2 A2) {
  const float2 x = ptx::fma2(make_float2(delta, delta), A2, make_float2(kRaise, kRaise));
  return make_float2(ex2(x.x), ex2(x.y));
}

// What a slot of 2^log tokens stands for: sequence n has those from (tok0 >> log) + n on (packed) or n * per_row on.
__device__ __forceinline__ int slot_of(const Seqs& s, int n, int tok0, int log, int per_row) { return s.cu ? (tok0 >> log) + n : n * per_row; }

// V values of a row that may not be aligned, or end (channels from `left` on are zero), as they are in memory: nothing waits for them until they are unpacked.
template <typename In, int V> struct Raw { uint32_t w[V * sizeof(In) / 4]; };
template <typename In, int V> __device__ __forceinline__ Raw<In, V> load_row(const In* p, bool vec, int left) {
  constexpr int W = V * sizeof(In) / 4;
  Raw<In, V> r;
  if (vec && left >= V) {
    if constexpr (W >= 4) {
#pragma unroll
      for (int i = 0; i < W; i += 4) {
        const uint4 x = reinterpret_cast<const uint4*>(p)[i / 4];
        r.w[i] = x.x; r.w[i + 1] = x.y; r.w[i + 2] = x.z; r.w[i + 3] = x.w;
      }
    } else if constexpr (W == 2) {
      const uint2 x = *reinterpret_cast<const uint2*>(p);
      r.w[0] = x.x; r.w[1] = x.y;
    } else {
      r.w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
    return r;
  }
#pragma unroll
  for (int i = 0; i < W; ++i) {
    if constexpr (sizeof(In) == 4) r.w[i] = i < left ? __float_as_uint(p[i]) : 0u;
    else r.w[i] = (2 * i < left ? (uint32_t)reinterpret_cast<const uint16_t*>(p)[2 * i] : 0u) |
                  (2 * i + 1 < left ? (uint32_t)reinterpret_cast<const uint16_t*>(p)[2 * i + 1] << 16 : 0u);
  }
  return r;
}
template <typename In, int V> __device__ __forceinline__ Vec<V> unpack_row(const Raw<In, V>& r) {
  Vec<V> v;
#pragma unroll
  for (int i = 0; i < V * (int)sizeof(In) / 4; ++i) {
    if constexpr (sizeof(In) == 4) v.v[i] = __uint_as_float(r.w[i]);
    else unpack2(r.w[i], v.v + 2 * i);
  }
  return v;
}
template <typename In, int V> __device__ __forceinline__ void store_row(In* p, bool vec, int left, const Vec<V>& r) {
  if (vec && left >= V) return store_v<V>(p, r);
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < left) p[i] = from_f32<In>(r.v[i]);
}

// Pieces of 16 bytes in a row of what one side writes and the other reads: exchanged within their neighbourhood, so that eight threads that are neighbours meet all
// banks on both sides (without that, reads of the sums took four times as long and bounded the kernel).
__device__ __forceinline__ int sum_piece(int u) { return u ^ ((u >> 3) & 3); }        // four lanes' sums
__device__ __forceinline__ int step_piece(int u) { return u ^ ((u >> 3) & 1); }       // delta and delta x of two channels

// `bytes` from global to shared memory in the background, if that can be (`fast`: aligned and whole), else by way of registers.
template <typename In, int V> __device__ __forceinline__ void stage_row(uint8_t* to, const In* from, bool fast, int left) {
  if (fast && left >= V) {
    const uint32_t dst = static_cast<uint32_t>(__cvta_generic_to_shared(to));
    if constexpr (V * sizeof(In) == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(from), "n"(V * sizeof(In)) : "memory");
  } else {
    *reinterpret_cast<Raw<In, V>*>(to) = load_row<In, V>(from, false, left);
  }
}

// Sums of v[0 .. n) over the lanes that differ in bits `top`, top / 2, .. (`bits` of them), spread out: a lane keeps the sums of the places whose
// index it spells with those bits, n >> bits of them (one, if there are fewer places than lanes).
template <int n, int bits> __device__ __forceinline__ void spread_sum(float (&v)[n], int top) {
  const int lane = threadIdx.x & 31;
  int half = n / 2;
#pragma unroll
  for (int b = 0; b < bits; ++b) {
    const int off = top >> b;
    if (half >= 1) {
      const bool up = lane & off;
#pragma unroll
      for (int j = 0; j < n / 2; ++j)
        if (j < half) {
          const float keep = up ? v[j + half] : v[j], send = up ? v[j] : v[j + half];
          v[j] = keep + __shfl_xor_sync(0xffffffffu, send, off);
        }
      half >>= 1;
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], off);
    }
  }
}

constexpr __host__ __device__ int ilog2(int x) { return x <= 1 ? 0 : 1 + ilog2(x / 2); }

}  // namespace mix
}  // namespace ha_la

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

namespace ha_la {
namespace mix {

struct ScanParams {
  Seqs seqs;
  int C, S, G, per_group;                                  // channels; states; groups; channels to a group
  int blocks;                                              // channel blocks of a group
  int softplus, packed, vec;                               // vec: rows can be read and written several channels at a time
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

// softplus(v) = max(v, 0) + log1p(e^-|v|), with log1p(e) = 2 artanh(s), s = e / (2 + e) <= 1/3, by its power series (s^15 / 15 < 5e-9):
// small steps keep all of their bits, where a logarithm of 1 + e would have lost them.
__device__ __forceinline__ float softplus(float v) {
  const float e = __expf(-fabsf(v)), s = __fdividef(e, 2.f + e), q = s * s;
  float r = 1.f / 13.f;
  r = fmaf(r, q, 1.f / 11.f); r = fmaf(r, q, 1.f / 9.f); r = fmaf(r, q, 1.f / 7.f); r = fmaf(r, q, 1.f / 5.f); r = fmaf(r, q, 1.f / 3.f);
  r = fmaf(r, q, 1.f);
  return fmaf(2.f * s, r, fmaxf(v, 0.f));
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// What a slot of 2^log tokens stands for: sequence n has those from (tok0 >> log) + n on (packed) or n * per_row on.
__device__ __forceinline__ int slot_of(const Seqs& s, int n, int tok0, int log, int per_row) { return s.cu ? (tok0 >> log) + n : n * per_row; }

// V values of a row that may not be aligned, or end (channels from `left` on are zero).
template <typename In, int V> __device__ __forceinline__ Vec<V> load_row(const In* p, bool vec, int left) {
  if (vec && left >= V) return load_v<V>(p);
  Vec<V> r;
#pragma unroll
  for (int i = 0; i < V; ++i) r.v[i] = i < left ? to_f32(p[i]) : 0.f;
  return r;
}
template <typename In, int V> __device__ __forceinline__ void store_row(In* p, bool vec, int left, const Vec<V>& r) {
  if (vec && left >= V) return store_v<V>(p, r);
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < left) p[i] = from_f32<In>(r.v[i]);
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

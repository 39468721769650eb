// Gated linear attention in fp32 on the CUDA cores (fp32 inputs, or d = 64): chunks of 64 tokens, every kernel chunk-parallel but the scan.
//
//   gla_state_kernel    a chunk's addition to the state (backward: and to the gradient of the state)     chunks x V-heads
//   gla_combine_kernel  states in front of the chunks, gradients behind them, by elements                sequences x V-heads x pieces of a state
//   gla_out_kernel      o                                                                                chunks x V-heads
//   gla_back_kernel     dq, dk, dv, dg                                                                   chunks x V-heads
//   gla_sum_kernel      dq, dk of q/k heads that several V-heads share, from their parts in order
//
// A product of a chunk is 64 rows by d (or 64) columns, 4 rows and every sixteenth column to a thread; the operands lie in shared memory with
// rows padded by 4 floats, so that 16-byte reads of neighbouring rows hit different banks.  In calls of few chunks (`few`) the first and third kernel
// give a CTA 16 rows, one to a thread, and four times the CTAs.  Reads of operands from shared memory and the fp32 multiply-adds bound it: eight rows of 600
// tokens, 16 heads, d = 128: additions 83 us (shared memory's pipe 74 % busy, fp32 52 %), outputs 194 (60 %, 43 %), gradients 720 (one CTA of 256
// threads to an SM: 50 %, 30 %).
#include "gla.cuh"

namespace ha_la {
namespace gla {

namespace {

constexpr int kTok = 64, kThreads = 256, kPad = 4;

struct SimtParams {
  Chunks chunks;
  Work w;
  const void *q, *k, *v, *d_o;
  const float* g;
  void *o, *dq, *dk, *dv;
  float* dg;
  int HK, HV;
  float scale;
  bool shared_heads;                                       // dq, dk go to Work's fp32 parts
};

// ---------------------------------------------------------------- pieces

// `rows` (64) tokens x D, zeros past the chunk's end
template <typename In, int D>
__device__ __forceinline__ void load_rows(float* dst, const void* src, int tok0, int L, int heads, int head, int rows = kTok) {
#pragma unroll 4
  for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads) {
    const int t = i / (D / 4), c = i % (D / 4) * 4;
    const float4 x = t < L ? load4(reinterpret_cast<const In*>(src) + ((size_t)(tok0 + t) * heads + head) * D + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    *reinterpret_cast<float4*>(dst + t * (D + kPad) + c) = x;
  }
}

// G_t of the chunk's tokens as the sum of two floats: differences of far tokens keep their low bits.  Tokens past the end have g = 0.
struct Gates { float hi[kTok], lo[kTok]; };
__device__ __forceinline__ void load_gates(Gates& s, const float* g, int tok0, int L, int HV, int j) {
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    const double g0 = 2 * lane < L ? gate(g[(size_t)(tok0 + 2 * lane) * HV + j]) : 0.0;
    const double g1 = 2 * lane + 1 < L ? gate(g[(size_t)(tok0 + 2 * lane + 1) * HV + j]) : 0.0;
    double sum = g0 + g1;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double y = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += y;
    }
    const double even = sum - g1;                          // (up to and with token 2 lane)
    s.hi[2 * lane] = (float)even;
    s.lo[2 * lane] = (float)(even - (double)(float)even);
    s.hi[2 * lane + 1] = (float)sum;
    s.lo[2 * lane + 1] = (float)(sum - (double)(float)sum);
  }
}
__device__ __forceinline__ float decay(const Gates& s, int to, int from) {   // e^{G_to - G_from}
  return expf((s.hi[to] - s.hi[from]) + (s.lo[to] - s.lo[from]));
}
__device__ __forceinline__ float decay0(const Gates& s, int to) { return expf(s.hi[to] + s.lo[to]); }

// acc[r][m] += rows R ty + r, columns tx + 16 m of A B (nn), A B^T (nt), A^T B (tn), over n
template <int R, int M>
__device__ __forceinline__ void nn(float (&acc)[R][M], const float* A, int lda, const float* B, int ldb, int n) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  for (int k = 0; k < n; k += 4) {
    float4 a[R];
#pragma unroll
    for (int r = 0; r < R; ++r) a[r] = *reinterpret_cast<const float4*>(A + (R * ty + r) * lda + k);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const float b = B[(k + kk) * ldb + tx + 16 * m];
#pragma unroll
        for (int r = 0; r < R; ++r) acc[r][m] = fmaf((&a[r].x)[kk], b, acc[r][m]);
      }
  }
}
template <int R, int M>
__device__ __forceinline__ void nt(float (&acc)[R][M], const float* A, int lda, const float* B, int ldb, int n) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  for (int k = 0; k < n; k += 4) {
    float4 a[R];
#pragma unroll
    for (int r = 0; r < R; ++r) a[r] = *reinterpret_cast<const float4*>(A + (R * ty + r) * lda + k);
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const float4 b = *reinterpret_cast<const float4*>(B + (tx + 16 * m) * ldb + k);
#pragma unroll
      for (int r = 0; r < R; ++r)
        acc[r][m] = fmaf(a[r].x, b.x, fmaf(a[r].y, b.y, fmaf(a[r].z, b.z, fmaf(a[r].w, b.w, acc[r][m]))));
    }
  }
}
template <int R, int M>
__device__ __forceinline__ void tn(float (&acc)[R][M], const float* A, int lda, const float* B, int ldb, int n) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll 4
  for (int k = 0; k < n; ++k) {
    float a[R];
    if constexpr (R == 4) *reinterpret_cast<float4*>(a) = *reinterpret_cast<const float4*>(A + k * lda + 4 * ty);
    else a[0] = A[k * lda + ty];
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const float b = B[k * ldb + tx + 16 * m];
#pragma unroll
      for (int r = 0; r < R; ++r) acc[r][m] = fmaf(a[r], b, acc[r][m]);
    }
  }
}
template <int R, int M> __device__ __forceinline__ void zero(float (&acc)[R][M]) {
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int m = 0; m < M; ++m) acc[r][m] = 0.f;
}

// ---------------------------------------------------------------- a chunk's addition to the state

// (16 R of its rows to a CTA: R = 1 in calls of few chunks, see `few`)
template <typename In, int D, int R, bool REV>
__global__ void __launch_bounds__(kThreads) gla_state_kernel(SimtParams p) {
  constexpr int LD = D + kPad, ROWS = 16 * R, LA = ROWS + kPad;
  extern __shared__ __align__(16) float sm[];
  __shared__ Gates G;
  float *a = sm, *b = sm + kTok * LA;
  const int part = blockIdx.x % (D / ROWS), unit = blockIdx.x / (D / ROWS), slot = unit / p.HV, j = unit % p.HV, jq = j / (p.HV / p.HK);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const Geom c = geom_of(p.chunks, slot);
  if (c.L <= 0) return;
  load_gates(G, p.g, c.tok0, c.L, p.HV, j);
  load_rows<In, D>(b, REV ? p.d_o : p.v, c.tok0, c.L, p.HV, j);
  const In* src = reinterpret_cast<const In*>(REV ? p.q : p.k) + part * ROWS;
  constexpr int kMine = kTok * (ROWS / 4) / kThreads;      // float4 of this CTA's rows to a thread
  float4 x[kMine];
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int at = threadIdx.x + kThreads * i, t = at / (ROWS / 4), cc = at % (ROWS / 4) * 4;
    x[i] = t < c.L ? load4(src + ((size_t)(c.tok0 + t) * p.HK + jq) * D + cc) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kMine; ++i) {                        // times their tokens' weights
    const int at = threadIdx.x + kThreads * i, t = at / (ROWS / 4), cc = at % (ROWS / 4) * 4;
    const float w = REV ? p.scale * decay0(G, t) : decay(G, kTok - 1, t);
    *reinterpret_cast<float4*>(a + t * LA + cc) = make_float4(x[i].x * w, x[i].y * w, x[i].z * w, x[i].w * w);
  }
  if (!REV && part == 0 && threadIdx.x == 0) p.w.total[(size_t)slot * p.HV + j] = decay0(G, kTok - 1);
  __syncthreads();
  float acc[R][D / 16];
  zero(acc);
  tn(acc, a, LA, b, LD, kTok);
  float* out = (REV ? p.w.dh : p.w.h) + ((size_t)slot * p.HV + j) * D * D + (size_t)part * ROWS * D;
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int m = 0; m < D / 16; ++m) out[(size_t)(R * ty + r) * D + tx + 16 * m] = acc[r][m];
}

// ---------------------------------------------------------------- the scan

struct CombineParams {
  const float* total;
  float* s;                                                // Work::h or dh
  const float* first;                                      // h0 (dhT) or NULL
  float* last;                                             // hT (dh0) or NULL
  const int32_t* seq_chunk0;
  int cps, HV, per_state;                                  // floats of a state
};

constexpr int kAhead = 8;                                  // chunks read ahead of the one that is added

template <bool REV>
__global__ void __launch_bounds__(kThreads) gla_combine_kernel(CombineParams p) {
  const int pieces = p.per_state / (4 * kThreads);
  const int nj = blockIdx.x / pieces, n = nj / p.HV, j = nj % p.HV;
  const size_t at = (size_t)(blockIdx.x % pieces) * 4 * kThreads + 4 * threadIdx.x;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int c0 = p.seq_chunk0 ? p.seq_chunk0[n] : n * p.cps, count = p.seq_chunk0 ? p.seq_chunk0[n + 1] - c0 : p.cps;
  float4 h = p.first ? *reinterpret_cast<const float4*>(p.first + (size_t)nj * p.per_state + at) : make_float4(0.f, 0.f, 0.f, 0.f);
  auto slot = [&](int c) { return (size_t)(c0 + (REV ? count - 1 - c : c)) * p.HV + j; };
  float4 add[kAhead];
  float dec[kAhead];
  auto fetch = [&](int i, int c) {
    if (c < count) {
      add[i] = *reinterpret_cast<const float4*>(p.s + slot(c) * p.per_state + at);
      dec[i] = p.total[slot(c)];
    }
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) fetch(i, i);
  for (int c = 0; c < count; c += kAhead)
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (c + i < count) {
        const float4 x = add[i];
        const float d = dec[i];
        fetch(i, c + i + kAhead);
        *reinterpret_cast<float4*>(p.s + slot(c + i) * p.per_state + at) = h;
        h = make_float4(fmaf(d, h.x, x.x), fmaf(d, h.y, x.y), fmaf(d, h.z, x.z), fmaf(d, h.w, x.w));
      }
  if (p.last) *reinterpret_cast<float4*>(p.last + (size_t)nj * p.per_state + at) = h;
}

// ---------------------------------------------------------------- outputs

// (16 R tokens to a CTA.  R = 4: keys, state and values in turn in one place, so that several CTAs share an SM; R = 1: all at once, read ahead)
template <typename In, int D, int R>
__global__ void __launch_bounds__(kThreads) gla_out_kernel(SimtParams p) {
  constexpr int LD = D + kPad, LP = kTok + kPad, M = D / 16, ROWS = 16 * R;
  extern __shared__ __align__(16) float sm[];
  __shared__ Gates G;
  float *q = sm, *P = q + ROWS * LD, *k = P + ROWS * LP, *v = R == 1 ? k + kTok * LD : k, *hs = R == 1 ? v + kTok * LD : k;
  const int part = blockIdx.x % (kTok / ROWS), unit = blockIdx.x / (kTok / ROWS), r0 = part * ROWS, upto = r0 + ROWS;
  const int slot = unit / p.HV, j = unit % p.HV, jq = j / (p.HV / p.HK), ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const Geom c = geom_of(p.chunks, slot);
  if (c.L <= r0) return;
  const float* h = p.w.h + ((size_t)slot * p.HV + j) * D * D;
  auto load_state = [&](int at, int rows) {
#pragma unroll 8
    for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads) {
      const int t = i / (D / 4), cc = i % (D / 4) * 4;
      *reinterpret_cast<float4*>(hs + t * LD + cc) = *reinterpret_cast<const float4*>(h + (size_t)(at + t) * D + cc);
    }
  };
  load_gates(G, p.g, c.tok0, c.L, p.HV, j);
  load_rows<In, D>(q, p.q, c.tok0 + r0, c.L - r0, p.HK, jq, ROWS);
  load_rows<In, D>(k, p.k, c.tok0, c.L, p.HK, jq, upto);
  if (R == 1) {
    load_state(0, D);
    load_rows<In, D>(v, p.v, c.tok0, c.L, p.HV, j, upto);
  }
  __syncthreads();
  float s[R][4];
  zero(s);
  nt(s, q, LD, k, LD, D);                                  // (R = 1: beyond this CTA's rows of whatever lies there, which the mask leaves out)
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int i = r0 + R * ty + r, jj = tx + 16 * m;
      P[(R * ty + r) * LP + jj] = i >= jj ? s[r][m] * decay(G, i, jj) : 0.f;
    }
  // q h first, times e^{G_i}; then P v on top
  float acc[R][M];
  zero(acc);
  if (R == 1) {
    nn(acc, q, LD, hs, LD, D);
  } else {
#pragma unroll 1
    for (int half = 0; half < D / 64; ++half) {
      __syncthreads();
      load_state(64 * half, 64);
      __syncthreads();
      nn(acc, q + 64 * half, LD, hs, LD, 64);
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float e = decay0(G, r0 + R * ty + r);
#pragma unroll
    for (int m = 0; m < M; ++m) acc[r][m] *= e;
  }
  __syncthreads();
  if (R != 1) {
    load_rows<In, D>(v, p.v, c.tok0, c.L, p.HV, j);
    __syncthreads();
  }
  nn(acc, P, LP, v, LD, upto);
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (r0 + R * ty + r < c.L) {
      In* o = reinterpret_cast<In*>(p.o) + ((size_t)(c.tok0 + r0 + R * ty + r) * p.HV + j) * D;
#pragma unroll
      for (int m = 0; m < M; ++m) o[tx + 16 * m] = from_f32<In>(p.scale * acc[r][m]);
    }
}

// ---------------------------------------------------------------- gradients

__device__ __forceinline__ float over_tx(float x) {        // sum over the 16 threads that share rows
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

constexpr int kStage = 32;                                 // rows of a state in shared memory

template <typename In, int D>
__global__ void __launch_bounds__(kThreads) gla_back_kernel(SimtParams p) {
  constexpr int LD = D + kPad, LP = kTok + kPad, M = D / 16;
  extern __shared__ __align__(16) float sm[];
  __shared__ Gates G;
  __shared__ float xs[kTok], ys[kTok], colsum[kThreads / 32][kTok], dots[kThreads / 32];
  float *q = sm, *k = q + kTok * LD, *v = k + kTok * LD, *d_o = v + kTok * LD, *P = d_o + kTok * LD, *dS = P + kTok * LP, *st = dS + kTok * LP;
  const int slot = blockIdx.x / p.HV, j = blockIdx.x % p.HV, jq = j / (p.HV / p.HK);
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15, warp = tid >> 5, lane = tid & 31;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const Geom c = geom_of(p.chunks, slot);
  if (c.L <= 0) return;
  load_gates(G, p.g, c.tok0, c.L, p.HV, j);
  load_rows<In, D>(q, p.q, c.tok0, c.L, p.HK, jq);
  load_rows<In, D>(k, p.k, c.tok0, c.L, p.HK, jq);
  load_rows<In, D>(v, p.v, c.tok0, c.L, p.HV, j);
  load_rows<In, D>(d_o, p.d_o, c.tok0, c.L, p.HV, j);
  __syncthreads();
  const float* h = p.w.h + ((size_t)slot * p.HV + j) * D * D;
  const float* dh = p.w.dh + ((size_t)slot * p.HV + j) * D * D;
  {
    float s[4][4], dp[4][4], col[4] = {0.f, 0.f, 0.f, 0.f};
    zero(s);
    zero(dp);
    nt(s, q, LD, k, LD, D);
    nt(dp, d_o, LD, v, LD, D);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 4 * ty + r;
      float row = 0.f;
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const int jj = tx + 16 * m;
        const float dec = i >= jj ? p.scale * decay(G, i, jj) : 0.f, ds = dp[r][m] * dec;
        P[i * LP + jj] = s[r][m] * dec;
        dS[i * LP + jj] = ds;
        const float e = i > jj ? s[r][m] * ds : 0.f;
        row += e;
        col[m] += e;
      }
      row = over_tx(row);
      if (tx == 0) xs[i] = row;
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      col[m] += __shfl_xor_sync(0xffffffffu, col[m], 16);
      if (lane < 16) colsum[warp][tx + 16 * m] = col[m];
    }
    float dot = 0.f;
    for (int i = 4 * tid; i < D * D; i += 4 * kThreads) {
      const float4 a = *reinterpret_cast<const float4*>(h + i), b = *reinterpret_cast<const float4*>(dh + i);
      dot += a.x * b.x + a.y * b.y + a.z * b.z + a.w * b.w;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
    if (lane == 0) dots[warp] = dot;
  }
  // kStage rows of a state into shared memory
  auto stage = [&](const float* src, int r0) {
    __syncthreads();
    for (int i = tid; i < kStage * (D / 4); i += kThreads) {
      const int t = i / (D / 4), cc = i % (D / 4) * 4;
      *reinterpret_cast<float4*>(st + t * LD + cc) = *reinterpret_cast<const float4*>(src + (size_t)(r0 + t) * D + cc);
    }
    __syncthreads();
  };
  auto put = [&](void* out, float* part, int heads, int head, const float (&acc)[4][M]) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (4 * ty + r < c.L) {
        const size_t t = c.tok0 + 4 * ty + r;
#pragma unroll
        for (int m = 0; m < M; ++m) {
          if (part) part[(t * p.HV + j) * D + tx + 16 * m] = acc[r][m];
          else reinterpret_cast<In*>(out)[(t * heads + head) * D + tx + 16 * m] = from_f32<In>(acc[r][m]);
        }
      }
  };
  float acc[4][M];
  // dq
  zero(acc);
#pragma unroll
  for (int r0 = 0; r0 < D; r0 += kStage) {
    stage(h, r0);
    float t[4][2];
    zero(t);
    nt(t, d_o, LD, st, LD, D);
#pragma unroll
    for (int r = 0; r < 4; ++r) { acc[r][r0 / 16] = t[r][0]; acc[r][r0 / 16 + 1] = t[r][1]; }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const float e = p.scale * decay0(G, 4 * ty + r);
    float x = 0.f;
#pragma unroll
    for (int m = 0; m < M; ++m) {
      acc[r][m] *= e;
      x = fmaf(acc[r][m], q[(4 * ty + r) * LD + tx + 16 * m], x);
    }
    x = over_tx(x);
    if (tx == 0) xs[4 * ty + r] += x;                      // (the thread that put the row's sum of E there)
  }
  nn(acc, dS, LP, k, LD, kTok);
  put(p.dq, p.shared_heads ? p.w.dq : nullptr, p.HK, jq, acc);
  // dk, and dv's part by the state: the same rows of dh
  float dv[4][M];
  zero(dv);
#pragma unroll
  for (int r0 = 0; r0 < D; r0 += kStage) {
    stage(dh, r0);
    float t[4][2];
    zero(t);
    nt(t, v, LD, st, LD, D);
#pragma unroll
    for (int r = 0; r < 4; ++r) { acc[r][r0 / 16] = t[r][0]; acc[r][r0 / 16 + 1] = t[r][1]; }
    nn(dv, k + r0, LD, st, LD, kStage);
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const float e = decay(G, kTok - 1, 4 * ty + r);
    float y = 0.f;
#pragma unroll
    for (int m = 0; m < M; ++m) {
      acc[r][m] *= e;
      dv[r][m] *= e;
      y = fmaf(acc[r][m], k[(4 * ty + r) * LD + tx + 16 * m], y);
    }
    y = over_tx(y);
    if (tx == 0) ys[4 * ty + r] = y;
  }
  tn(acc, dS, LP, q, LD, kTok);
  put(p.dk, p.shared_heads ? p.w.dk : nullptr, p.HK, jq, acc);
  tn(dv, P, LP, d_o, LD, kTok);
  put(p.dv, nullptr, p.HV, j, dv);
  __syncthreads();
  if (tid < c.L) {
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) s += dots[w];
    s *= decay0(G, kTok - 1);
    for (int i = tid; i < kTok; ++i) {
      s += xs[i];
#pragma unroll
      for (int w = 0; w < kThreads / 32; ++w) s -= colsum[w][i];
    }
    for (int i = 0; i < tid; ++i) s += ys[i];
    p.dg[(size_t)(c.tok0 + tid) * p.HV + j] = (float)s;
  }
}

// ---------------------------------------------------------------- heads that share q and k

struct SumParams { const float *dq, *dk; void *out_q, *out_k; size_t n; int R, per_head; };   // n: elements of dq

template <typename In>
__global__ void __launch_bounds__(kThreads) gla_sum_kernel(SumParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const size_t i = ((size_t)blockIdx.x * kThreads + threadIdx.x) * 4;
  if (i >= p.n) return;
  const size_t head = i / p.per_head;
  const float* src = (blockIdx.y ? p.dk : p.dq) + head * p.R * p.per_head + i % p.per_head;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int r = 0; r < p.R; ++r) {
    const float4 x = *reinterpret_cast<const float4*>(src + (size_t)r * p.per_head);
    s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
  }
  In* out = reinterpret_cast<In*>(blockIdx.y ? p.out_k : p.out_q) + i;
  out[0] = from_f32<In>(s.x); out[1] = from_f32<In>(s.y); out[2] = from_f32<In>(s.z); out[3] = from_f32<In>(s.w);
}

// ---------------------------------------------------------------- host

constexpr size_t smem_state(int D, int R) { return kTok * (D + 16 * R + 2 * kPad) * 4u; }
constexpr size_t smem_out(int D, int R) { return (16 * R * (D + kTok + 2 * kPad) + (R == 1 ? 2 * kTok + D : kTok) * (D + kPad)) * 4u; }
constexpr size_t smem_back(int D) { return (4u * kTok * (D + kPad) + 2 * kTok * (kTok + kPad) + kStage * (D + kPad)) * 4; }
static_assert(smem_back(128) + 8192 <= 227 * 1024, "shared memory budget");

SimtParams params_of(const Call& c) {
  SimtParams s;
  s.chunks = c.chunks; s.w = c.w;
  s.q = c.a.q; s.k = c.a.k; s.v = c.a.v; s.d_o = c.a.do_; s.g = c.a.g;
  s.o = c.a.o; s.dq = c.a.dq; s.dk = c.a.dk; s.dv = c.a.dv; s.dg = c.a.dg;
  s.HK = c.p.HK; s.HV = c.p.HV; s.scale = c.p.scale; s.shared_heads = c.p.HV != c.p.HK;
  return s;
}

// `parts` CTAs to a (chunk, V-head)
cudaError_t launch(void (*kernel)(SimtParams), int parts, size_t smem, const Call& c, cudaStream_t stream) {
  const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return start(kernel, dim3((unsigned)((size_t)c.p.max_chunks * c.p.HV * parts)), kThreads, smem, stream, params_of(c));
}

// Rows of a thread in the chunks' additions and outputs: 1, with four times the CTAs, where all of these run at once (three to an SM at d = 64, one at 128:
// 61 and 143 KiB).  us with 4 and with 1, fp32: one chunk at d = 64 22 and 13, 40 chunks x V-heads 22 and 21, 160 34 and 45; d = 128, 4 of them 42 and 22, 80 45 and 57.
bool few(const Call& c) { return (long long)c.p.max_chunks * c.p.HV * 4 <= sm_count() * (c.p.dk == 64 ? 3 : 1); }

template <typename In, int D, int R>
cudaError_t chunks_forward(const Call& c, cudaStream_t stream) { return launch(gla_state_kernel<In, D, R, false>, D / (16 * R), smem_state(D, R), c, stream); }
template <typename In, int D, int R>
cudaError_t chunks_reverse(const Call& c, cudaStream_t stream) { return launch(gla_state_kernel<In, D, R, true>, D / (16 * R), smem_state(D, R), c, stream); }

template <typename In, int D>
cudaError_t forward(const Call& c, cudaStream_t stream) {
  if (c.p.max_chunks > 0) {
    const cudaError_t e = few(c) ? chunks_forward<In, D, 1>(c, stream) : chunks_forward<In, D, 4>(c, stream);
    if (e != cudaSuccess) return e;
  }
  const cudaError_t e = launch_combine(c, false, stream);
  if (e != cudaSuccess || c.p.max_chunks == 0) return e;
  return few(c) ? launch(gla_out_kernel<In, D, 1>, kTok / 16, smem_out(D, 1), c, stream) : launch(gla_out_kernel<In, D, 4>, 1, smem_out(D, 4), c, stream);
}

template <typename In, int D>
cudaError_t backward(const Call& c, cudaStream_t stream) {
  cudaError_t e = cudaSuccess;
  if (c.p.max_chunks > 0) {
    e = few(c) ? chunks_forward<In, D, 1>(c, stream) : chunks_forward<In, D, 4>(c, stream);
    if (e == cudaSuccess) e = few(c) ? chunks_reverse<In, D, 1>(c, stream) : chunks_reverse<In, D, 4>(c, stream);
    if (e == cudaSuccess) e = launch_combine(c, false, stream);
  }
  if (e == cudaSuccess) e = launch_combine(c, true, stream);
  if (e != cudaSuccess || c.p.max_chunks == 0) return e;
  e = launch(gla_back_kernel<In, D>, 1, smem_back(D), c, stream);
  return e == cudaSuccess ? launch_head_sums(c, c.p.HV, stream) : e;
}

}  // namespace

size_t simt_bytes(const Problem& p, bool back, Work* w, void* base) {
  char* b = reinterpret_cast<char*>(base);
  const size_t units = (size_t)p.max_chunks * p.HV, state = units * p.dk * p.dv * 4, parts = (size_t)p.T_total * p.HV * p.dk * 4;
  const size_t shared = back && p.HV != p.HK ? parts : 0;
  const size_t at = align_up(units * 4, 1024);
  if (w) {
    w->total = reinterpret_cast<float*>(b);
    w->h = reinterpret_cast<float*>(b + at);
    w->dh = reinterpret_cast<float*>(b + at + state);
    w->dq = reinterpret_cast<float*>(b + at + 2 * state);
    w->dk = reinterpret_cast<float*>(b + at + 2 * state + shared);
  }
  return at + (back ? 2 : 1) * state + 2 * shared;
}

// Forward: the states in front of the chunks and hT.  Reverse: the gradients behind them and dh0.
cudaError_t launch_combine(const Call& c, bool reverse, cudaStream_t stream) {
  CombineParams p;
  p.total = c.w.total;
  p.s = reverse ? c.w.dh : c.w.h;
  p.first = reverse ? c.a.dhT : c.a.h0;
  p.last = reverse ? c.a.dh0 : (c.back ? nullptr : c.a.hT);
  p.seq_chunk0 = c.chunks.seq_chunk0;
  p.cps = c.chunks.cps; p.HV = c.p.HV; p.per_state = c.p.dk * c.p.dv;
  const dim3 grid((unsigned)((size_t)c.p.N * c.p.HV * (p.per_state / (4 * kThreads))));
  return reverse ? start(gla_combine_kernel<true>, grid, kThreads, 0, stream, p) : start(gla_combine_kernel<false>, grid, kThreads, 0, stream, p);
}

cudaError_t launch_chain(const float* total, float* s, const float* first, int count, int N, int HV, int per_state, bool reverse, cudaStream_t stream) {
  const CombineParams p{total, s, first, nullptr, nullptr, count, HV, per_state};
  const dim3 grid((unsigned)((size_t)N * HV * (per_state / (4 * kThreads))));
  return reverse ? start(gla_combine_kernel<true>, grid, kThreads, 0, stream, p) : start(gla_combine_kernel<false>, grid, kThreads, 0, stream, p);
}

cudaError_t launch_head_sums(const Call& c, int parts, cudaStream_t stream) {
  if (parts == c.p.HK || c.p.T_total == 0) return cudaSuccess;   // (empty sequences have chunk slots, but no token)
  SumParams p;
  p.dq = c.w.dq; p.dk = c.w.dk; p.out_q = c.a.dq; p.out_k = c.a.dk;
  p.n = (size_t)c.p.T_total * c.p.HK * c.p.dk; p.R = parts / c.p.HK; p.per_head = c.p.dk;
  const dim3 grid((unsigned)((p.n / 4 + kThreads - 1) / kThreads), 2);
  return c.p.dtype == HA_LA_BF16 ? start(gla_sum_kernel<__nv_bfloat16>, grid, kThreads, 0, stream, p) : start(gla_sum_kernel<float>, grid, kThreads, 0, stream, p);
}

cudaError_t launch_simt_forward(const Call& c, cudaStream_t stream) {
  const bool bf16 = c.p.dtype == HA_LA_BF16, big = c.p.dk == 128;
  if (bf16) return big ? forward<__nv_bfloat16, 128>(c, stream) : forward<__nv_bfloat16, 64>(c, stream);
  return big ? forward<float, 128>(c, stream) : forward<float, 64>(c, stream);
}

cudaError_t launch_simt_backward(const Call& c, cudaStream_t stream) {
  const bool bf16 = c.p.dtype == HA_LA_BF16, big = c.p.dk == 128;
  if (bf16) return big ? backward<__nv_bfloat16, 128>(c, stream) : backward<__nv_bfloat16, 64>(c, stream);
  return big ? backward<float, 128>(c, stream) : backward<float, 64>(c, stream);
}

}  // namespace gla
}  // namespace ha_la

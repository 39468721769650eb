// Short causal convolution per channel (ha_la_conv* in ha_la.h): y_t = act(bias + sum_j w[j] x_{t-K+1+j}), K = 2, 3 or 4.
//
// One read of x and one write of y are all that has to move, and 2 K operations a value are nothing beside it, so HBM bounds it.  A thread
// has V channels (8 bytes) of a run of consecutive tokens: the K - 1 inputs in front stay in registers from token to token, only a run's first ones are
// read twice.  A run is taken apart at sequence starts, in front of which h0's inputs stand, so the inner loops know no boundaries.  (35 k tokens of 8192
// channels 223 us; gradients of 16384 tokens of 4096 channels 107.)
//
// Backwards, with p_t the sum ahead of the activation (made again), e_t = dy_t act'(p_t):
//   dx_t = sum_j w[K-1-j] e_{t+j}  (+ dhT's part for the last K - 1 tokens)    dw[j] = sum_t e_t x_{t-K+1+j}    db = sum_t e_t
// the K - 1 tokens behind a run are read again for their e.  Sums over tokens: a run in registers, runs by a second kernel in 64 bits and
// in order, so the same bits every time.
#include <algorithm>
#include <type_traits>

#include "mix.cuh"
#include "../tc_mma.cuh"

namespace ha_la {
namespace mix {
namespace {

struct ConvParams {
  Seqs seqs;
  int C, run, groups, runs;                                // tokens to a run; CTAs side by side for a run's channels; runs
  long long stride;                                        // of x
  const void *x, *h0, *dy, *dhT;
  const float *w, *bias;
  void *y, *hT, *dx, *dh0;
  float* part;                                             // [run][K + 1][C]: sums for dw and db
  int32_t* status;
};

constexpr int kThreads = 128;
constexpr int kBytes = 8;                                  // of a token to a thread: with 16 the taps' registers leave too few warps (prompts 261 us for 223)

// A thread's values of a token as they are in memory: nothing waits for them until they are unpacked.
template <typename In, int V> struct Piece { In v[V]; };
template <typename In, int V> __device__ __forceinline__ Piece<In, V> fetch(const In* p) {
  constexpr int B = V * sizeof(In);
  Piece<In, V> r;
  if constexpr (B == kBytes) *reinterpret_cast<uint2*>(&r) = *reinterpret_cast<const uint2*>(p);
  else r.v[0] = *p;
  return r;
}
template <typename In, int V> __device__ __forceinline__ Vec<V> unpack(const Piece<In, V>& r) {
  Vec<V> x;
#pragma unroll
  for (int v = 0; v < V; ++v) x.v[v] = to_f32(r.v[v]);
  return x;
}

// A thread's pieces of the tokens ahead, in shared memory by asynchronous copies: kRing batches of U tokens, whose places nobody else looks at.  In registers they
// would take so many that too few warps were left to wait for them (16384 tokens x 4096 channels: 140 us, and 107 this way with a branch-free loop).
constexpr int kRing = 4;
__device__ __forceinline__ void copy8(uint8_t* to, const void* from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(to))), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_sent() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 2) : "memory"); }

// a b + c, two values to an instruction
template <int V> __device__ __forceinline__ Vec<V> fma_v(const Vec<V>& a, const Vec<V>& b, const Vec<V>& c) {
  Vec<V> r;
  if constexpr (V % 2 == 0) {
#pragma unroll
    for (int v = 0; v < V; v += 2) {
      const float2 x = ptx::fma2(make_float2(a.v[v], a.v[v + 1]), make_float2(b.v[v], b.v[v + 1]), make_float2(c.v[v], c.v[v + 1]));
      r.v[v] = x.x;
      r.v[v + 1] = x.y;
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) r.v[v] = fmaf(a.v[v], b.v[v], c.v[v]);
  }
  return r;
}

template <int K, int V> struct Taps { Vec<V> w[K], b; };

template <int K, int V> __device__ __forceinline__ void load_taps(Taps<K, V>& t, const ConvParams& p, int c) {
  constexpr int L = V >= 4 ? 4 : V;                        // (a thread's K V weights lie together)
  float flat[K * V];
#pragma unroll
  for (int i = 0; i < K * V; i += L) {
    const Vec<L> w = load_v<L>(p.w + (size_t)c * K + i);
#pragma unroll
    for (int l = 0; l < L; ++l) flat[i + l] = w.v[l];
  }
  Vec<V> none = {};
  t.b = none;
  if (p.bias) t.b = load_v<V>(p.bias + c);
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < K; ++j) t.w[j].v[v] = flat[v * K + j];
}

// The input at position `pos` of the sequence, which may lie in front of it.
template <typename In, int K, int V> __device__ __forceinline__ Vec<V> input_at(const ConvParams& p, int n, int tok0, int pos, int c) {
  if (pos >= 0) return load_v<V>(reinterpret_cast<const In*>(p.x) + (size_t)(tok0 + pos) * p.stride + c);
  if (p.h0) return load_v<V>(reinterpret_cast<const In*>(p.h0) + ((size_t)n * (K - 1) + (K - 1 + pos)) * p.C + c);
  Vec<V> z = {};
  return z;
}

template <int K, int V> __device__ __forceinline__ Vec<V> sum_of(const Taps<K, V>& t, const Vec<V> (&win)[K - 1], const Vec<V>& x) {
  Vec<V> s = t.b;
#pragma unroll
  for (int j = 0; j < K - 1; ++j) s = fma_v<V>(t.w[j], win[j], s);
  return fma_v<V>(t.w[K - 1], x, s);
}

template <int K, int V> __device__ __forceinline__ void push(Vec<V> (&win)[K - 1], const Vec<V>& x) {
#pragma unroll
  for (int j = 1; j < K - 1; ++j) win[j - 1] = win[j];
  win[K - 2] = x;
}

// The sequence of token t: the CTA's first warp looks it up.  Everybody has to come here.
__device__ __forceinline__ int seq_of_token(const Seqs& s, int t) {
  __shared__ int found;
  if (!s.cu) return s.T_row > 0 ? t / s.T_row : 0;
  if (threadIdx.x < 32) {
    const int n = find_seq(s, t);
    if (threadIdx.x == 0) found = n;
  }
  __syncthreads();
  return found;
}

// Rows behind the runs: the last inputs of a sequence, for whoever goes on from there.
template <typename In, int K, int V> __device__ __forceinline__ void last_inputs(const ConvParams& p, int n, int c) {
  const Seq q = seq_of(p.seqs, n);
  if (!p.hT || q.len < 0) return;
#pragma unroll
  for (int i = 0; i < K - 1; ++i)
    store_v<V>(reinterpret_cast<In*>(p.hT) + ((size_t)n * (K - 1) + i) * p.C + c, input_at<In, K, V>(p, n, q.tok0, q.len - (K - 1) + i, c));
}

template <typename In, int K, int V, bool SILU>
__global__ void __launch_bounds__(kThreads) conv_kernel(ConvParams p) {
  constexpr int U = 8;                                     // tokens whose loads are in flight together (four: 266 us for 223, sixteen: 255)
  const int row = blockIdx.x / p.groups, c = ((blockIdx.x - row * p.groups) * kThreads + threadIdx.x) * V;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0) check_seqs(p.seqs, p.status);
  if (row >= p.runs) {
    if (c < p.C) last_inputs<In, K, V>(p, row - p.runs, c);
    return;
  }
  int t = row * p.run;
  const int t1 = t + min(p.run, p.seqs.T_total - t);
  int n = seq_of_token(p.seqs, t);
  if (c >= p.C) return;
  Taps<K, V> taps;
  load_taps<K, V>(taps, p, c);
  const In* x = reinterpret_cast<const In*>(p.x) + c;
  In* y = reinterpret_cast<In*>(p.y) + c;
  while (t < t1) {
    Seq q = seq_of(p.seqs, n);
    while (n + 1 < p.seqs.N && q.len >= 0 && q.tok0 + q.len <= t) q = seq_of(p.seqs, ++n);
    if (q.len < 0 || t < q.tok0 || t >= q.tok0 + q.len) break;            // (offsets that do not fit)
    const int end = min(t1, q.tok0 + q.len);
    Vec<V> win[K - 1];
#pragma unroll
    for (int j = 0; j < K - 1; ++j) win[j] = input_at<In, K, V>(p, n, q.tok0, t - q.tok0 - (K - 1) + j, c);
    auto token = [&](int at, const Vec<V>& now) {
      Vec<V> s = sum_of<K, V>(taps, win, now);
      if (SILU) {
#pragma unroll
        for (int v = 0; v < V; ++v) s.v[v] *= sigmoid(s.v[v]);
      }
      store_v<V>(y + (size_t)at * p.C, s);
      push<K, V>(win, now);
    };
    for (; t + U <= end; t += U) {
      Piece<In, V> in[U];
#pragma unroll
      for (int i = 0; i < U; ++i) in[i] = fetch<In, V>(x + (size_t)(t + i) * p.stride);
#pragma unroll
      for (int i = 0; i < U; ++i) token(t + i, unpack<In, V>(in[i]));
    }
    for (; t < end; ++t) token(t, load_v<V>(x + (size_t)t * p.stride));
  }
}

// e = dy act'(s)
template <int V, bool SILU> __device__ __forceinline__ void through_act(Vec<V>& d, const Vec<V>& s) {
  if (!SILU) return;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const float g = sigmoid(s.v[v]);
    d.v[v] *= g * fmaf(s.v[v], 1.f - g, 1.f);
  }
}

// dh0 of a sequence: what its first tokens take from in front of it, and dhT's part where the sequence is shorter than K - 1.
template <typename In, int K, int V, bool SILU> __device__ __forceinline__ void front_back(const ConvParams& p, int n, int c) {
  const Seq q = seq_of(p.seqs, n);
  if (!p.dh0 || q.len < 0) return;
  Taps<K, V> taps;
  load_taps<K, V>(taps, p, c);
  Vec<V> d[K - 1] = {}, win[K - 1];
#pragma unroll
  for (int j = 0; j < K - 1; ++j) win[j] = input_at<In, K, V>(p, n, q.tok0, j - (K - 1), c);
#pragma unroll
  for (int u = 0; u < K - 1; ++u) {
    if (u >= q.len) break;
    const Vec<V> now = input_at<In, K, V>(p, n, q.tok0, u, c);
    Vec<V> e = load_v<V>(reinterpret_cast<const In*>(p.dy) + (size_t)(q.tok0 + u) * p.C + c);
    through_act<V, SILU>(e, sum_of<K, V>(taps, win, now));
    push<K, V>(win, now);
#pragma unroll
    for (int j = 0; j < K - 1; ++j)                        // tap j of token u reads place u + j of what lies in front
      if (u + j < K - 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) d[u + j].v[v] = fmaf(taps.w[j].v[v], e.v[v], d[u + j].v[v]);
      }
  }
#pragma unroll
  for (int i = 0; i < K - 1; ++i) {
    if (p.dhT && i >= q.len) {
      const Vec<V> g = load_v<V>(reinterpret_cast<const In*>(p.dhT) + ((size_t)n * (K - 1) + i - q.len) * p.C + c);
#pragma unroll
      for (int v = 0; v < V; ++v) d[i].v[v] += g.v[v];
    }
    store_v<V>(reinterpret_cast<In*>(p.dh0) + ((size_t)n * (K - 1) + i) * p.C + c, d[i]);
  }
}

template <typename In, int K, int V, bool SILU>
__global__ void __launch_bounds__(kThreads) conv_back_kernel(ConvParams p) {
  constexpr int U = 4;
  const int row = blockIdx.x / p.groups, c = ((blockIdx.x - row * p.groups) * kThreads + threadIdx.x) * V;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0) check_seqs(p.seqs, p.status);
  if (row >= p.runs) {
    if (c < p.C) front_back<In, K, V, SILU>(p, row - p.runs, c);
    return;
  }
  int t = row * p.run;
  const int t1 = t + min(p.run, p.seqs.T_total - t);
  int n = seq_of_token(p.seqs, t);
  if (c >= p.C) return;
  Taps<K, V> taps;
  load_taps<K, V>(taps, p, c);
  const In *x = reinterpret_cast<const In*>(p.x) + c, *dy = reinterpret_cast<const In*>(p.dy) + c;
  In* dx = reinterpret_cast<In*>(p.dx) + c;
  Vec<V> dw[K] = {}, db = {};
  while (t < t1) {
    Seq q = seq_of(p.seqs, n);
    while (n + 1 < p.seqs.N && q.len >= 0 && q.tok0 + q.len <= t) q = seq_of(p.seqs, ++n);
    if (q.len < 0 || t < q.tok0 || t >= q.tok0 + q.len) break;
    const int end = q.tok0 + q.len, mine = min(t1, end), last = min(mine + K - 1, end);   // own tokens; those whose e is needed
    Vec<V> win[K - 1], acc[K] = {};                        // acc[j]: dx of the token j ahead
#pragma unroll
    for (int j = 0; j < K - 1; ++j) win[j] = input_at<In, K, V>(p, n, q.tok0, t - q.tok0 - (K - 1) + j, c);
    auto emit = [&](int at, Vec<V>& a) {
      if (p.dhT && at >= end - (K - 1)) {
        const Vec<V> g = load_v<V>(reinterpret_cast<const In*>(p.dhT) + ((size_t)n * (K - 1) + at - (end - (K - 1))) * p.C + c);
#pragma unroll
        for (int v = 0; v < V; ++v) a.v[v] += g.v[v];
      }
      store_v<V>(dx + (size_t)at * p.C, a);
    };
    const int first = t;
    // (`inside`: one of the run's own tokens with K - 1 of the run in front of it, which is most of them, without a branch)
    auto token = [&](auto inside, int u, const Vec<V>& now, Vec<V> e) {
      through_act<V, SILU>(e, sum_of<K, V>(taps, win, now));
      if (inside.value || u < mine) {
#pragma unroll
        for (int j = 0; j < K - 1; ++j) dw[j] = fma_v<V>(e, win[j], dw[j]);
        dw[K - 1] = fma_v<V>(e, now, dw[K - 1]);
#pragma unroll
        for (int v = 0; v < V; ++v) db.v[v] += e.v[v];
      }
      push<K, V>(win, now);
#pragma unroll
      for (int j = K - 1; j > 0; --j) acc[j] = fma_v<V>(taps.w[K - 1 - j], e, acc[j - 1]);
#pragma unroll
      for (int v = 0; v < V; ++v) acc[0].v[v] = taps.w[K - 1].v[v] * e.v[v];
      if (inside.value || u - (K - 1) >= first) store_v<V>(dx + (size_t)(u - (K - 1)) * p.C, acc[K - 1]);
    };
    int u = t;
    if constexpr (V * sizeof(In) == kBytes) {
      __shared__ __align__(16) uint8_t ring[kRing * U * 2][kThreads][8];
      auto send = [&](int b) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int at = first + b * U + i, place = (b % kRing * U + i) * 2;
          if (at < last) {
            copy8(ring[place][threadIdx.x], x + (size_t)at * p.stride);
            copy8(ring[place + 1][threadIdx.x], dy + (size_t)at * p.C);
          }
        }
        copies_sent();
      };
      for (int b = 0; b < kRing - 1; ++b) send(b);
#pragma unroll 1
      for (int b = 0; u < last; ++b) {
        copies_wait();
        auto from_ring = [&](auto inside, int i) {
          const int place = (b % kRing * U + i) * 2;
          token(inside, u + i, unpack<In, V>(fetch<In, V>(reinterpret_cast<const In*>(ring[place][threadIdx.x]))),
                unpack<In, V>(fetch<In, V>(reinterpret_cast<const In*>(ring[place + 1][threadIdx.x]))));
        };
        if (b > 0 && u + U <= mine) {
#pragma unroll
          for (int i = 0; i < U; ++i) from_ring(std::true_type(), i);
        } else {
#pragma unroll 1
          for (int i = 0; i < U && u + i < last; ++i) from_ring(std::false_type(), i);
        }
        u += U;
        send(b + kRing - 1);
      }
    }
    for (; u < last; ++u) token(std::false_type(), u, load_v<V>(x + (size_t)u * p.stride), load_v<V>(dy + (size_t)u * p.C));
#pragma unroll
    for (int j = K - 2; j >= 0; --j)                       // (the tokens that no later one of the sequence follows K - 1 behind)
      if (last - 1 - j >= first && last - 1 - j < mine) emit(last - 1 - j, acc[j]);
    t = mine;
  }
  float* part = p.part + (size_t)row * (K + 1) * p.C + c;
#pragma unroll
  for (int v = 0; v < V; ++v) {
#pragma unroll
    for (int j = 0; j < K; ++j) part[(size_t)j * p.C + v] = dw[j].v[v];
    part[(size_t)K * p.C + v] = db.v[v];
  }
}

__global__ void __launch_bounds__(kThreads) conv_sum_kernel(const float* part, int runs, int C, int K, float* dw, float* db) {
  const long long i = (long long)blockIdx.x * kThreads + threadIdx.x, per = (long long)C * (K + 1);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (i >= per) return;
  double s = 0;
#pragma unroll 8
  for (int r = 0; r < runs; ++r) s += part[(size_t)r * per + i];
  const int j = (int)(i / C), c = (int)(i - (long long)j * C);
  if (j < K) dw[(size_t)c * K + j] = (float)s;
  else if (db) db[c] = (float)s;
}

// One token: a thread reads its channels' inputs before it writes the new state over them.
template <typename In, int K, int V, bool SILU>
__global__ void __launch_bounds__(kThreads) conv_decode_kernel(ConvParams p) {
  const int n = blockIdx.x / p.groups, c = ((blockIdx.x - n * p.groups) * kThreads + threadIdx.x) * V;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (c >= p.C) return;
  Vec<V> win[K - 1];
#pragma unroll
  for (int j = 0; j < K - 1; ++j) win[j] = input_at<In, K, V>(p, n, n, j - (K - 1), c);
  const Vec<V> now = load_v<V>(reinterpret_cast<const In*>(p.x) + (size_t)n * p.stride + c);
  Taps<K, V> taps;
  load_taps<K, V>(taps, p, c);
  Vec<V> s = sum_of<K, V>(taps, win, now);
  if (SILU) {
#pragma unroll
    for (int v = 0; v < V; ++v) s.v[v] *= sigmoid(s.v[v]);
  }
  store_v<V>(reinterpret_cast<In*>(p.y) + (size_t)n * p.C + c, s);
  push<K, V>(win, now);
#pragma unroll
  for (int j = 0; j < K - 1; ++j) store_v<V>(reinterpret_cast<In*>(p.hT) + ((size_t)n * (K - 1) + j) * p.C + c, win[j]);
}

enum Form { kForward, kBackward, kToken };

template <typename In, int K, int V, bool SILU> cudaError_t launch(Form f, const ConvParams& p, long long grid, cudaStream_t stream) {
  void (*k)(ConvParams) = f == kForward ? conv_kernel<In, K, V, SILU> : f == kBackward ? conv_back_kernel<In, K, V, SILU> : conv_decode_kernel<In, K, V, SILU>;
  return start(k, dim3((unsigned)grid), kThreads, 0, stream, p);
}
template <typename In, int V> cudaError_t launch_taps(Form f, int K, bool silu, const ConvParams& p, long long grid, cudaStream_t stream) {
  switch (K) {
    case 2: return silu ? launch<In, 2, V, true>(f, p, grid, stream) : launch<In, 2, V, false>(f, p, grid, stream);
    case 3: return silu ? launch<In, 3, V, true>(f, p, grid, stream) : launch<In, 3, V, false>(f, p, grid, stream);
    default: return silu ? launch<In, 4, V, true>(f, p, grid, stream) : launch<In, 4, V, false>(f, p, grid, stream);
  }
}

// Tokens to a run.  Short ones give the SMs something to do; long ones read less twice and, backward, leave fewer sums, all of them at once on the SMs
// (4 CTAs each: 107 us; 1.4 rounds of them 137).
int run_of(long long tokens, int C, int V, bool back) {
  const long long warps = (C + 32 * V - 1) / (32 * V), want = (long long)sm_count() * (back ? 16 : 32);
  const long long run = tokens * warps / want + back;
  return (int)std::min<long long>(std::max<long long>(run, back ? 8 : 4), back ? 512 : 32);
}

int check(const ha_la_conv_args* a, ConvParams* p, bool packed_ok) {
  if (!a) return HA_LA_ERR_INVALID_ARG;
  if (a->dtype != HA_LA_BF16 && a->dtype != HA_LA_FP32) return HA_LA_ERR_INVALID_ARG;
  if (a->batch < (packed_ok ? 1 : 0) || a->channels < 1 || a->x_stride < 0 || (a->x_stride > 0 && a->x_stride < a->channels)) return HA_LA_ERR_INVALID_ARG;
  if (a->activation != HA_LA_ACT_SILU && a->activation != HA_LA_ACT_NONE) return HA_LA_ERR_INVALID_ARG;
  if (a->taps < 1) return HA_LA_ERR_INVALID_ARG;
  if (a->taps < 2 || a->taps > 4 || a->channels > (1 << 24)) return HA_LA_ERR_UNSUPPORTED;
  *p = ConvParams{};
  if (!make_seqs(&p->seqs, a->cu_seqlens, a->batch, a->seqlen, packed_ok ? a->num_seqs : 0, a->max_seqlen)) return HA_LA_ERR_INVALID_ARG;
  if ((long long)a->batch * a->seqlen > 0x7fffffffLL - 256) return HA_LA_ERR_UNSUPPORTED;
  p->C = a->channels;
  p->stride = a->x_stride ? a->x_stride : a->channels;
  p->x = a->x; p->w = a->w; p->bias = a->bias; p->h0 = a->h0; p->y = a->y; p->hT = a->hT;
  p->dy = a->dy; p->dhT = a->dhT; p->dx = a->dx; p->dh0 = a->dh0;
  p->status = a->status_word;
  return HA_LA_OK;
}

// Values to a thread: kBytes, if every token of every tensor starts on a 16-byte boundary, else one.
int width_of(const ha_la_conv_args* a, const ConvParams& p, bool back) {
  const int e = a->dtype == HA_LA_BF16 ? 2 : 4;
  const uintptr_t at = any_of(a->x, a->h0, a->w, a->bias, back ? a->dy : nullptr, back ? a->dhT : nullptr, back ? a->dx : a->y, back ? a->dh0 : a->hT);
  return at % 16 == 0 && (p.C | p.stride) * e % 16 == 0 ? kBytes / e : 1;
}

void shape(ConvParams* p, int V, bool back) {
  p->groups = (p->C + V * kThreads - 1) / (V * kThreads);
  p->run = run_of(p->seqs.T_total, p->C, V, back);
  p->runs = (int)(((long long)p->seqs.T_total + p->run - 1) / p->run);
}

// The workspace is for the narrow threads too, whatever the pointers are: the most runs that either has.
size_t part_bytes(const ha_la_conv_args* a, ConvParams p) {
  int most = 0;
  for (int V : {kBytes / (a->dtype == HA_LA_BF16 ? 2 : 4), 1}) {
    shape(&p, V, true);
    most = std::max(most, p.runs);
  }
  return align_up(std::max<size_t>((size_t)most * (a->taps + 1) * a->channels * 4, 1), 256);
}

int run(const ha_la_conv_args* a, Form f, cudaStream_t stream) {
  ConvParams p;
  const int rc = check(a, &p, f != kToken);
  if (rc != HA_LA_OK) return rc;
  const bool back = f == kBackward;
  if (f == kToken && (a->seqlen != 1 || a->cu_seqlens || a->num_seqs)) return HA_LA_ERR_INVALID_ARG;
  if (f != kToken && a->num_seqs > 0 && !a->cu_seqlens) return HA_LA_ERR_INVALID_ARG;
  const uintptr_t one = a->dtype == HA_LA_BF16 ? 1 : 3;
  if (any_of(a->x, a->h0, a->y, a->hT, a->dy, a->dhT, a->dx, a->dh0) & one) return HA_LA_ERR_INVALID_ARG;
  if (any_of(a->w, a->bias, a->dw, a->db, a->cu_seqlens, a->status_word) & 3) return HA_LA_ERR_INVALID_ARG;
  if (!a->w) return HA_LA_ERR_INVALID_ARG;
  if (f == kForward && a->hT && a->hT == a->h0) return HA_LA_ERR_INVALID_ARG;
  if (p.seqs.T_total > 0 && (!a->x || (back ? !a->dy || !a->dx : !a->y))) return HA_LA_ERR_INVALID_ARG;
  if (back && !a->dw) return HA_LA_ERR_INVALID_ARG;
  if (f == kToken && p.seqs.N > 0 && !a->hT) return HA_LA_ERR_INVALID_ARG;
  if (back && (!a->workspace || ((uintptr_t)a->workspace & 255) || a->workspace_bytes < part_bytes(a, p))) return HA_LA_ERR_WORKSPACE;
  const int V = width_of(a, p, back);
  shape(&p, V, back);
  p.part = reinterpret_cast<float*>(a->workspace);
  const bool rows = f == kToken || (back ? p.dh0 != nullptr : p.hT != nullptr);
  const long long grid = (long long)p.groups * ((f == kToken ? 0 : p.runs) + (rows ? p.seqs.N : 0));
  if (grid > 0x7fffffffLL) return HA_LA_ERR_UNSUPPORTED;
  cudaError_t e = cudaSuccess;
  const bool silu = a->activation == HA_LA_ACT_SILU;
  if (grid > 0) {
    if (a->dtype == HA_LA_BF16)
      e = V > 1 ? launch_taps<__nv_bfloat16, 4>(f, a->taps, silu, p, grid, stream) : launch_taps<__nv_bfloat16, 1>(f, a->taps, silu, p, grid, stream);
    else
      e = V > 1 ? launch_taps<float, 2>(f, a->taps, silu, p, grid, stream) : launch_taps<float, 1>(f, a->taps, silu, p, grid, stream);
  }
  if (e == cudaSuccess && back) {
    const long long per = (long long)p.C * (a->taps + 1);
    e = start(conv_sum_kernel, dim3((unsigned)((per + kThreads - 1) / kThreads)), kThreads, 0, stream, (const float*)p.part, p.runs, p.C, a->taps, a->dw, a->db);
  }
  return e == cudaSuccess ? HA_LA_OK : HA_LA_ERR_CUDA;
}

}  // namespace
}  // namespace mix
}  // namespace ha_la

using namespace ha_la;

extern "C" {

int ha_la_conv_workspace_bytes(const ha_la_conv_args* a, size_t* out_bytes) {
  if (!out_bytes) return HA_LA_ERR_INVALID_ARG;
  mix::ConvParams p;
  const int rc = mix::check(a, &p, true);
  if (rc != HA_LA_OK) return rc;
  *out_bytes = mix::part_bytes(a, p);
  return HA_LA_OK;
}
int ha_la_conv(const ha_la_conv_args* a, void* s) { return mix::run(a, mix::kForward, reinterpret_cast<cudaStream_t>(s)); }
int ha_la_conv_backward(const ha_la_conv_args* a, void* s) { return mix::run(a, mix::kBackward, reinterpret_cast<cudaStream_t>(s)); }
int ha_la_conv_decode(const ha_la_conv_args* a, void* s) { return mix::run(a, mix::kToken, reinterpret_cast<cudaStream_t>(s)); }

}  // extern "C"

// Short causal convolution per channel (ha_la_conv* in ha_la.h): y_t = act(bias + sum_j w[j] x_{t-K+1+j}), K = 2, 3 or 4.
//
// One read of x and one write of y are all that has to move, and 2 K operations a value are nothing beside it, so HBM bounds it.  A thread
// has V channels (16 bytes forward, 8 backward, where registers for the sums of dw take the room) of a run of consecutive tokens: the K - 1
// inputs in front stay in registers from token to token, only a run's first ones are read twice.  A run is taken apart at sequence
// starts, in front of which h0's inputs stand, so the inner loops know no boundaries.
//
// Backwards, with p_t the sum ahead of the activation (made again), e_t = dy_t act'(p_t):
//   dx_t = sum_j w[K-1-j] e_{t+j}  (+ dhT's part for the last K - 1 tokens)    dw[j] = sum_t e_t x_{t-K+1+j}    db = sum_t e_t
// the K - 1 tokens behind a run are read again for their e.  Sums over tokens: a run in registers, runs by a second kernel in 64 bits and
// in order, so the same bits every time.
#include <algorithm>

#include "mix.cuh"

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

template <int K, int V> struct Taps { float w[K][V], b[V]; };

template <int K, int V> __device__ __forceinline__ void load_taps(Taps<K, V>& t, const ConvParams& p, int c) {
  constexpr int L = V >= 4 ? 4 : V;                        // (a thread's K V weights lie together)
  float flat[K * V];
#pragma unroll
  for (int i = 0; i < K * V; i += L) {
    const Vec<L> w = load_v<L>(p.w + (size_t)c * K + i);
#pragma unroll
    for (int l = 0; l < L; ++l) flat[i + l] = w.v[l];
  }
  Vec<V> b = {};
  if (p.bias) b = load_v<V>(p.bias + c);
#pragma unroll
  for (int v = 0; v < V; ++v) {
#pragma unroll
    for (int j = 0; j < K; ++j) t.w[j][v] = flat[v * K + j];
    t.b[v] = b.v[v];
  }
}

// The input at position `pos` of the sequence, which may lie in front of it.
template <typename In, int K, int V> __device__ __forceinline__ Vec<V> input_at(const ConvParams& p, int n, int tok0, int pos, int c) {
  if (pos >= 0) return load_v<V>(reinterpret_cast<const In*>(p.x) + (size_t)(tok0 + pos) * p.stride + c);
  if (p.h0) return load_v<V>(reinterpret_cast<const In*>(p.h0) + ((size_t)n * (K - 1) + (K - 1 + pos)) * p.C + c);
  Vec<V> z = {};
  return z;
}

template <int K, int V> __device__ __forceinline__ Vec<V> sum_of(const Taps<K, V>& t, const Vec<V> (&win)[K - 1], const Vec<V>& x) {
  Vec<V> s;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    s.v[v] = t.b[v];
#pragma unroll
    for (int j = 0; j < K - 1; ++j) s.v[v] = fmaf(t.w[j][v], win[j].v[v], s.v[v]);
    s.v[v] = fmaf(t.w[K - 1][v], x.v[v], s.v[v]);
  }
  return s;
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
  constexpr int U = 4;                                     // tokens whose loads are in flight together
  const int row = blockIdx.x / p.groups, c = ((blockIdx.x - row * p.groups) * kThreads + threadIdx.x) * V;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0) check_seqs(p.seqs, p.status);
  if (row >= p.runs) {
    if (c < p.C) last_inputs<In, K, V>(p, row - p.runs, c);
    return;
  }
  int t = row * p.run;
  const int t1 = min(t + p.run, p.seqs.T_total);
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
      Vec<V> in[U];
#pragma unroll
      for (int i = 0; i < U; ++i) in[i] = load_v<V>(x + (size_t)(t + i) * p.stride);
#pragma unroll
      for (int i = 0; i < U; ++i) token(t + i, in[i]);
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
        for (int v = 0; v < V; ++v) d[u + j].v[v] = fmaf(taps.w[j][v], e.v[v], d[u + j].v[v]);
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
  const int t1 = min(t + p.run, p.seqs.T_total);
  int n = seq_of_token(p.seqs, t);
  if (c >= p.C) return;
  Taps<K, V> taps;
  load_taps<K, V>(taps, p, c);
  const In *x = reinterpret_cast<const In*>(p.x) + c, *dy = reinterpret_cast<const In*>(p.dy) + c;
  In* dx = reinterpret_cast<In*>(p.dx) + c;
  float dw[K][V] = {}, db[V] = {};
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
    auto token = [&](int u, const Vec<V>& now, Vec<V> e) {
      through_act<V, SILU>(e, sum_of<K, V>(taps, win, now));
      if (u < mine) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
          db[v] += e.v[v];
#pragma unroll
          for (int j = 0; j < K - 1; ++j) dw[j][v] = fmaf(e.v[v], win[j].v[v], dw[j][v]);
          dw[K - 1][v] = fmaf(e.v[v], now.v[v], dw[K - 1][v]);
        }
      }
      push<K, V>(win, now);
#pragma unroll
      for (int j = K - 1; j >= 0; --j) {
#pragma unroll
        for (int v = 0; v < V; ++v) acc[j].v[v] = fmaf(taps.w[K - 1 - j][v], e.v[v], j ? acc[j - 1].v[v] : 0.f);
      }
      if (u - (K - 1) >= first) emit(u - (K - 1), acc[K - 1]);
    };
    int u = t;
    for (; u + U <= last; u += U) {
      Vec<V> in[U], d[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        in[i] = load_v<V>(x + (size_t)(u + i) * p.stride);
        d[i] = load_v<V>(dy + (size_t)(u + i) * p.C);
      }
#pragma unroll
      for (int i = 0; i < U; ++i) token(u + i, in[i], d[i]);
    }
    for (; u < last; ++u) token(u, load_v<V>(x + (size_t)u * p.stride), load_v<V>(dy + (size_t)u * p.C));
#pragma unroll
    for (int j = K - 2; j >= 0; --j)                       // (the tokens that no later one of the sequence follows K - 1 behind)
      if (last - 1 - j >= first && last - 1 - j < mine) emit(last - 1 - j, acc[j]);
    t = mine;
  }
  float* part = p.part + (size_t)row * (K + 1) * p.C + c;
#pragma unroll
  for (int v = 0; v < V; ++v) {
#pragma unroll
    for (int j = 0; j < K; ++j) part[(size_t)j * p.C + v] = dw[j][v];
    part[(size_t)K * p.C + v] = db[v];
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
  constexpr int VB = V > 1 ? V / 2 : 1;
  void (*k)(ConvParams) = f == kForward ? conv_kernel<In, K, V, SILU> : f == kBackward ? conv_back_kernel<In, K, VB, SILU> : conv_decode_kernel<In, K, V, SILU>;
  return start(k, dim3((unsigned)grid), kThreads, 0, stream, p);
}
template <typename In, int V> cudaError_t launch_taps(Form f, int K, bool silu, const ConvParams& p, long long grid, cudaStream_t stream) {
  switch (K) {
    case 2: return silu ? launch<In, 2, V, true>(f, p, grid, stream) : launch<In, 2, V, false>(f, p, grid, stream);
    case 3: return silu ? launch<In, 3, V, true>(f, p, grid, stream) : launch<In, 3, V, false>(f, p, grid, stream);
    default: return silu ? launch<In, 4, V, true>(f, p, grid, stream) : launch<In, 4, V, false>(f, p, grid, stream);
  }
}

// Tokens to a run.  Long ones read less twice and leave fewer sums, short ones give the SMs something to do: aim at 8 (forward) and 12 warps an SM.
int run_of(long long tokens, int C, int V, bool back) {
  const long long warps = (C + 32 * V - 1) / (32 * V), want = (long long)sm_count() * (back ? 12 : 16);
  long long run = tokens * warps / want;
  return (int)std::min<long long>(std::max<long long>(run, back ? 8 : 4), back ? 128 : 32);
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

// Values to a thread: 16 bytes forward and 8 backward, if every token of every tensor starts so aligned, else one.
int width_of(const ha_la_conv_args* a, const ConvParams& p, bool back) {
  const int e = a->dtype == HA_LA_BF16 ? 2 : 4, V = a->dtype == HA_LA_BF16 ? (back ? 4 : 8) : (back ? 2 : 4);
  const uintptr_t at = any_of(a->x, a->h0, back ? a->dy : nullptr, back ? a->dhT : nullptr, back ? a->dx : a->y, back ? a->dh0 : a->hT);
  return at % (V * e) == 0 && any_of(a->w, a->bias) % 16 == 0 && p.C % V == 0 && p.stride % V == 0 ? V : 1;
}

void shape(ConvParams* p, int V, bool back) {
  p->groups = (p->C + V * kThreads - 1) / (V * kThreads);
  p->run = run_of(p->seqs.T_total, p->C, V, back);
  p->runs = (p->seqs.T_total + p->run - 1) / p->run;
}

// The workspace is for the narrow threads too, whatever the pointers are: the most runs that either has.
size_t part_bytes(const ha_la_conv_args* a, ConvParams p) {
  int most = 0;
  for (int V : {a->dtype == HA_LA_BF16 ? 4 : 2, 1}) {
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
      e = V > 1 ? launch_taps<__nv_bfloat16, 8>(f, a->taps, silu, p, grid, stream) : launch_taps<__nv_bfloat16, 1>(f, a->taps, silu, p, grid, stream);
    else
      e = V > 1 ? launch_taps<float, 4>(f, a->taps, silu, p, grid, stream) : launch_taps<float, 1>(f, a->taps, silu, p, grid, stream);
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

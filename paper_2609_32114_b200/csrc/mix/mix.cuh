// What the short convolution, the selective scan and latent attention share: sequences of a packed batch without a chunk table,
// token strides, launches.
#pragma once

#include <atomic>

#include "../common.cuh"

namespace ha_la {
namespace mix {

// Where the sequences are.  There is no table made ahead of the kernels (a launch of its own): whoever needs a sequence looks its two
// offsets up and checks them, so that no offset, whatever it holds, leads out of the token axis.
struct Seqs {
  const int32_t* cu;                                       // NULL: rows of T_row tokens
  int N, T_total, T_row, max_len;
};

struct Seq { int tok0, len; };                             // len -1: offsets that do not fit

__device__ __forceinline__ Seq seq_of(const Seqs& s, int n) {
  if (!s.cu) return {n * s.T_row, s.T_row};
  const int a = s.cu[n], b = s.cu[n + 1];
  const bool ok = a >= 0 && b >= a && b <= s.T_total && b - a <= s.max_len && (n > 0 || a == 0) && (n < s.N - 1 || b == s.T_total);
  return {ok ? a : 0, ok ? b - a : -1};
}

// One CTA's threads look at all sequences and report.
__device__ __forceinline__ void check_seqs(const Seqs& s, int32_t* status) {
  if (!s.cu || !status) return;
  for (int n = threadIdx.x; n < s.N; n += blockDim.x)
    if (seq_of(s, n).len < 0) report_status(status, HA_LA_ERR_DEVICE_CHECK);
}

// The last sequence that starts at token t or ahead of it, and more generally the last n with cu[n] / step + add n <= t (step a power of two by its
// logarithm): 32 places at once by the threads of a warp, so two look-ups one behind the other for a thousand sequences.  Always in [0, N).
__device__ __forceinline__ int find_seq(const Seqs& s, int t, int log_step = 0, int add = 0) {
  int lo = 0, hi = s.N;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, n = lo + (int)(threadIdx.x & 31) * step;
    const unsigned before = __ballot_sync(0xffffffffu, n < hi && (s.cu[n] >> log_step) + add * n <= t);
    lo += before ? (31 - __clz(before)) * step : 0;
    hi = min(hi, lo + step);
  }
  return lo;
}

inline bool make_seqs(Seqs* s, const int32_t* cu, int batch, int seqlen, int num_seqs, int max_seqlen) {
  const bool packed = cu || num_seqs > 0;
  if (batch < 0 || seqlen < 0 || (packed && (batch != 1 || num_seqs < 1 || max_seqlen < 0))) return false;
  s->cu = cu;
  s->N = packed ? num_seqs : batch;
  s->T_row = seqlen;
  s->T_total = (int)((long long)batch * seqlen);           // (callers refuse more than 31 bits)
  s->max_len = packed && max_seqlen > 0 && max_seqlen < seqlen ? max_seqlen : seqlen;
  return true;
}

template <typename... Args>
cudaError_t start(void (*kernel)(Args...), dim3 grid, int threads, size_t smem, cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// A kernel's shared memory limit, raised once per device.  `regs`: registers of a thread that its roles share out among themselves; with fewer at launch
// they would wait for ever.
template <auto kern> cudaError_t allow_smem(size_t smem, int regs = 0) {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return cudaErrorInvalidDevice;
  if (dev < 64 && (done.load() >> dev & 1)) return cudaSuccess;
  cudaFuncAttributes has;
  cudaError_t e = cudaFuncGetAttributes(&has, kern);
  if (e == cudaSuccess && has.numRegs < regs) e = cudaErrorInvalidKernelImage;
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess && dev < 64) done.fetch_or(1ull << dev);
  return e;
}

template <typename... P> uintptr_t any_of(P... p) { return (... | (uintptr_t)p); }

// V consecutive values; 16 bytes at a time where V of them fill that.
template <int V> struct Vec { float v[V]; };

__device__ __forceinline__ void unpack2(uint32_t w, float* v) {
  v[0] = __uint_as_float(w << 16);
  v[1] = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&p);
}
template <int V> __device__ __forceinline__ Vec<V> load_v(const __nv_bfloat16* p) {
  Vec<V> r;
  if constexpr (V == 8) {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    unpack2(w.x, r.v); unpack2(w.y, r.v + 2); unpack2(w.z, r.v + 4); unpack2(w.w, r.v + 6);
  } else if constexpr (V == 4) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    unpack2(w.x, r.v); unpack2(w.y, r.v + 2);
  } else if constexpr (V == 2) {
    unpack2(*reinterpret_cast<const uint32_t*>(p), r.v);
  } else {
    r.v[0] = to_f32(*p);
  }
  return r;
}
template <int V> __device__ __forceinline__ Vec<V> load_v(const float* p) {
  Vec<V> r;
  if constexpr (V >= 4) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const float4 w = *reinterpret_cast<const float4*>(p + i);
      r.v[i] = w.x; r.v[i + 1] = w.y; r.v[i + 2] = w.z; r.v[i + 3] = w.w;
    }
  } else if constexpr (V == 2) {
    const float2 w = *reinterpret_cast<const float2*>(p);
    r.v[0] = w.x; r.v[1] = w.y;
  } else {
    r.v[0] = *p;
  }
  return r;
}
template <int V> __device__ __forceinline__ void store_v(__nv_bfloat16* p, const Vec<V>& r) {
  if constexpr (V == 8) *reinterpret_cast<uint4*>(p) = make_uint4(pack2(r.v[0], r.v[1]), pack2(r.v[2], r.v[3]), pack2(r.v[4], r.v[5]), pack2(r.v[6], r.v[7]));
  else if constexpr (V == 4) *reinterpret_cast<uint2*>(p) = make_uint2(pack2(r.v[0], r.v[1]), pack2(r.v[2], r.v[3]));
  else if constexpr (V == 2) *reinterpret_cast<uint32_t*>(p) = pack2(r.v[0], r.v[1]);
  else *p = from_f32<__nv_bfloat16>(r.v[0]);
}
template <int V> __device__ __forceinline__ void store_v(float* p, const Vec<V>& r) {
  if constexpr (V >= 4) {
#pragma unroll
    for (int i = 0; i < V; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(r.v[i], r.v[i + 1], r.v[i + 2], r.v[i + 3]);
  } else if constexpr (V == 2) *reinterpret_cast<float2*>(p) = make_float2(r.v[0], r.v[1]);
  else *p = r.v[0];
}

constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float ex2(float x) {            // 2^x, zero for very negative x
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float sigmoid(float z) { return reciprocal(1.f + ex2(-z * kLog2e)); }

}  // namespace mix
}  // namespace ha_la

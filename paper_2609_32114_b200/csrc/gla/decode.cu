// One token per sequence of gated linear attention: ha_la_gla_decode in ha_la.h.
//
//   h' = e^g h + k v^T     o = scale h'^T q
// One pass over the state: unlike the delta rule's step (decode.cu) nothing has to be known of the whole state before a row of it
// is rewritten, so a row goes from load to store by itself and only the sum for o crosses threads.  It is bound by HBM, 8 d_k d_v bytes for 5 d_k d_v
// operations per (sequence, V-head); one CTA of four warps per 64 value channels, four channels of D / 8 rows to a thread, all of a
// thread's loads in flight together, streaming accesses (a state is used once per step).
#include "gla.cuh"

namespace ha_la {
namespace gla {

namespace {

struct DecodeParams {
  const void *q, *k, *v;
  const float *g, *h_in;
  float* h_out;
  void* o;
  int HK, HV;
  float scale;
};

constexpr int kCols = 64, kThreads = 128;
constexpr int kRows = kThreads / (kCols / 4);              // state rows that the CTA reads at once

template <typename In, int D>
__global__ void __launch_bounds__(kThreads, 4) gla_decode_kernel(DecodeParams p) {
  constexpr int NR = D / kRows;                            // rows per thread
  __shared__ float sk[D], sq[D];
  __shared__ __align__(16) float spart[kRows][kCols];
  const int tid = threadIdx.x;
  const int row0 = tid / (kCols / 4), c4 = (blockIdx.x % (D / kCols)) * kCols + tid % (kCols / 4) * 4;
  const size_t nj = blockIdx.x / (D / kCols);              // (sequence, V-head)
  const size_t n = nj / p.HV;
  const int jq = (int)(nj - n * p.HV) / (p.HV / p.HK);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  float4 h[NR];
  const size_t base = nj * D * D + (size_t)row0 * D + c4;
#pragma unroll
  for (int i = 0; i < NR; ++i)
    h[i] = p.h_in ? __ldcs(reinterpret_cast<const float4*>(p.h_in + base + (size_t)i * kRows * D)) : make_float4(0.f, 0.f, 0.f, 0.f);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (tid < D) {
    const size_t qk = (n * p.HK + jq) * D + tid;
    sk[tid] = to_f32(reinterpret_cast<const In*>(p.k)[qk]);
    sq[tid] = to_f32(reinterpret_cast<const In*>(p.q)[qk]);
  }
  const float4 v = load4(reinterpret_cast<const In*>(p.v) + nj * D + c4);
  const float dec = expf(p.g[nj]);
  __syncthreads();
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const float k = sk[row0 + i * kRows], q = sq[row0 + i * kRows];
    h[i].x = fmaf(dec, h[i].x, k * v.x); h[i].y = fmaf(dec, h[i].y, k * v.y);
    h[i].z = fmaf(dec, h[i].z, k * v.z); h[i].w = fmaf(dec, h[i].w, k * v.w);
    __stcs(reinterpret_cast<float4*>(p.h_out + base + (size_t)i * kRows * D), h[i]);
    acc.x = fmaf(h[i].x, q, acc.x); acc.y = fmaf(h[i].y, q, acc.y); acc.z = fmaf(h[i].z, q, acc.z); acc.w = fmaf(h[i].w, q, acc.w);
  }
  *reinterpret_cast<float4*>(&spart[row0][c4 % kCols]) = acc;
  __syncthreads();
  if (tid < kCols) {
    float o = 0.f;
#pragma unroll
    for (int r = 0; r < kRows; ++r) o += spart[r][tid];
    reinterpret_cast<In*>(p.o)[nj * D + (blockIdx.x % (D / kCols)) * kCols + tid] = from_f32<In>(p.scale * o);
  }
}

}  // namespace

}  // namespace gla
}  // namespace ha_la

using namespace ha_la;

extern "C" int ha_la_gla_decode(const ha_la_decode_args* a, void* cuda_stream) {
  if (!a) return HA_LA_ERR_INVALID_ARG;
  if (a->dtype != HA_LA_BF16 && a->dtype != HA_LA_FP32) return HA_LA_ERR_INVALID_ARG;
  if (a->num_seqs < 0 || a->num_qk_heads < 1 || a->num_v_heads < 1 || a->num_v_heads % a->num_qk_heads != 0) return HA_LA_ERR_INVALID_ARG;
  if (a->d_k < 1 || a->d_v < 1) return HA_LA_ERR_INVALID_ARG;
  if (a->d_k != a->d_v || (a->d_k != 64 && a->d_k != 128)) return HA_LA_ERR_UNSUPPORTED;
  if (!(a->scale == a->scale)) return HA_LA_ERR_INVALID_ARG;
  const unsigned long long heads = (unsigned long long)a->num_seqs * a->num_v_heads;
  if (heads > 0x7fffffffULL / (a->d_k / gla::kCols)) return HA_LA_ERR_UNSUPPORTED;
  if (heads == 0) return HA_LA_OK;
  if (!a->q || !a->k || !a->v || !a->g || !a->h_out || !a->o) return HA_LA_ERR_INVALID_ARG;
  const uintptr_t al16 = (uintptr_t)a->q | (uintptr_t)a->k | (uintptr_t)a->v | (uintptr_t)a->o | (uintptr_t)a->h_in | (uintptr_t)a->h_out;
  if ((al16 & 15) || ((uintptr_t)a->g & 3)) return HA_LA_ERR_INVALID_ARG;
  const gla::DecodeParams p{a->q, a->k, a->v, a->g, a->h_in, a->h_out, a->o, a->num_qk_heads, a->num_v_heads, a->scale};
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  const bool bf16 = a->dtype == HA_LA_BF16, big = a->d_k == 128;
  void (*k)(gla::DecodeParams) = bf16 ? (big ? gla::gla_decode_kernel<__nv_bfloat16, 128> : gla::gla_decode_kernel<__nv_bfloat16, 64>)
                                      : (big ? gla::gla_decode_kernel<float, 128> : gla::gla_decode_kernel<float, 64>);
  return gla::start(k, dim3((unsigned)(heads * (a->d_k / gla::kCols))), gla::kThreads, 0, stream, p) == cudaSuccess ? HA_LA_OK : HA_LA_ERR_CUDA;
}

// Attention over latent rows on the CUDA cores, for what the tensor-core kernels do not take: fp32, other head sizes, tensors that are not aligned.
//
// A CTA has eight query rows that see the same keys (consecutive queries of a head; heads of a sequence's new tokens), one to a warp, and brings 32 keys
// at a time to shared memory in fp32.  A lane makes one key's score, then holds every 32nd channel of the output.  Bound by shared-memory reads, two
// for each multiply-add.
#include "latent.cuh"

namespace ha_la {
namespace mix {
namespace {

constexpr int kRows = 8, kKeys = 32, kThreads = 32 * kRows;
static_assert(kMostValue <= 8 * 32 && kMostLatent <= 16 * 32, "a lane's channels");

// One CTA: rows r < rows with their limits (keys that row r sees), queries in s_q; `key(j, c)` and `value(j, c)` bring element c of key j.
template <int CH, typename Key, typename Value, typename Out>
__device__ __forceinline__ void attend(float* sm, int rows, int my_keys, int keys, int dk, int dv, bool shared, float scale, Key key, Value value, Out out) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, pitch = dk + 1 + (dk & 1);      // (odd: lanes read a column each)
  float* const s_q = sm;
  float* const s_k = s_q + kRows * dk;
  float* const s_v = shared ? s_k : s_k + kKeys * pitch;
  const int vp = shared ? pitch : dv;
  float m = kNegInf, l = 0.f, acc[CH] = {};
  for (int j0 = 0; j0 < keys; j0 += kKeys) {
    __syncthreads();
    const int have = min(kKeys, keys - j0);
    for (int j = warp; j < have; j += kRows) {
      for (int c = lane; c < dk; c += 32) s_k[j * pitch + c] = key(j0 + j, c);
      if (!shared)
        for (int c = lane; c < dv; c += 32) s_v[j * vp + c] = value(j0 + j, c);
    }
    __syncthreads();
    const int seen = min(have, my_keys - j0);
    if (warp >= rows || seen <= 0) continue;
    float s = 0.f;
    const float *qr = s_q + warp * dk, *kr = s_k + min(lane, have - 1) * pitch;
    for (int c = 0; c < dk; ++c) s = fmaf(qr[c], kr[c], s);
    s = lane < seen ? s * scale : kNegInf;
    float top = s;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float mn = fmaxf(m, top), rescale = m == kNegInf ? 0.f : exp2f(m - mn), w = s > kNegInf ? exp2f(s - mn) : 0.f;
    m = mn;
    float sum = w;
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    l = fmaf(l, rescale, sum);
#pragma unroll
    for (int i = 0; i < CH; ++i) acc[i] *= rescale;
    for (int j = 0; j < seen; ++j) {
      const float wj = __shfl_sync(0xffffffffu, w, j);
#pragma unroll
      for (int i = 0; i < CH; ++i)
        if (i * 32 + lane < dv) acc[i] = fmaf(wj, s_v[j * vp + i * 32 + lane], acc[i]);
    }
  }
  if (warp >= rows) return;
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int i = 0; i < CH; ++i)
    if (i * 32 + lane < dv) out(warp, i * 32 + lane, acc[i] * inv, 0.f, false);
  if (lane == 0) out(warp, 0, 0.f, l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : kNegInf, true);
}

size_t smem_of(int dk, int dv, bool shared) { return sizeof(float) * ((size_t)kRows * dk + (size_t)kKeys * (dk + 1 + (dk & 1)) + (shared ? 0 : (size_t)kKeys * dv)); }

template <typename In>
__global__ void __launch_bounds__(kThreads) latent_prompt_kernel(PromptParams p) {
  extern __shared__ __align__(16) float sm[];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0) check_spans(p);
  const int per = p.blocks * p.H, n = blockIdx.x / per, b = (blockIdx.x - n * per) / p.H, h = blockIdx.x % p.H;
  const Span s = span_of(p, n);
  const int i0 = b * kRows, rows = min(kRows, s.q - i0), dk = p.dn + p.dr;
  if (rows <= 0) return;
  const In *q = reinterpret_cast<const In*>(p.q), *kn = reinterpret_cast<const In*>(p.kn) + h * p.kn_hs, *kr = reinterpret_cast<const In*>(p.kr),
           *v = reinterpret_cast<const In*>(p.v) + h * p.v_hs;
  const float to_log2 = p.scale * 1.4426950408889634f;
  for (int e = threadIdx.x; e < rows * dk; e += kThreads) sm[e] = to_f32(q[(size_t)(s.q0 + i0 + e / dk) * p.qs + (size_t)h * dk + e % dk]);
  auto limit = [&](int i) { return max(0, min(s.k, s.k - s.q + 1 + i)); };
  attend<8>(sm, rows, limit(i0 + (threadIdx.x >> 5)), limit(i0 + rows - 1), dk, p.dv, false, to_log2,
            [&](int j, int c) {
              const size_t t = s.k0 + j;
              return c < p.dn ? to_f32(kn[t * p.kns + c]) : to_f32(kr[t * p.krs + c - p.dn]);
            },
            [&](int j, int c) { return to_f32(v[(size_t)(s.k0 + j) * p.vs + c]); },
            [&](int r, int c, float x, float lse, bool is_lse) {
              const size_t row = (size_t)(s.q0 + i0 + r) * p.H + h;
              if (!is_lse) reinterpret_cast<In*>(p.o)[row * p.dv + c] = from_f32<In>(x);
              else if (p.lse) p.lse[row] = lse;
            });
}

template <typename In>
__global__ void __launch_bounds__(kThreads) latent_token_kernel(TokenParams p) {
  extern __shared__ __align__(16) float sm[];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0) check_tokens(p);
  const int all = p.T * p.H, blocks = (all + kRows - 1) / kRows, n = blockIdx.x / blocks, r0 = (blockIdx.x - n * blocks) * kRows;
  const int rows = min(kRows, all - r0), dk = p.dl + p.dr, len = rows_of(p, n);
  const In *q = reinterpret_cast<const In*>(p.q) + ((size_t)n * all + r0) * dk, *cache = reinterpret_cast<const In*>(p.cache);
  for (int e = threadIdx.x; e < rows * dk; e += kThreads) sm[e] = to_f32(q[e]);
  auto limit = [&](int r) { return max(0, len - p.T + 1 + r / p.H); };
  attend<16>(sm, rows, limit(min(r0 + (int)(threadIdx.x >> 5), all - 1)), limit(r0 + rows - 1), dk, p.dl, true, p.scale * 1.4426950408889634f,
             [&](int j, int c) { return to_f32(cache[cache_row(p, n, j) * dk + c]); }, [&](int, int) { return 0.f; },
             [&](int r, int c, float x, float lse, bool is_lse) {
               const size_t row = (size_t)n * all + r0 + r;
               if (!is_lse) reinterpret_cast<In*>(p.o)[row * p.dl + c] = from_f32<In>(x);
               else if (p.lse) p.lse[row] = lse;
             });
}

// `most`: for the largest head sizes that the library takes, whatever this call's are; a limit of the call's own would be another host thread's to lower.
template <auto kern, typename P> cudaError_t go(const P& p, long long grid, size_t smem, size_t most, cudaStream_t stream) {
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  const cudaError_t e = allow_smem<kern>(most);
  return e == cudaSuccess ? start(kern, dim3((unsigned)grid), kThreads, smem, stream, p) : e;
}

}  // namespace

cudaError_t launch_prompt_simt(bool bf16, const PromptParams& given, cudaStream_t stream) {
  PromptParams p = given;
  p.blocks = (p.q_seqs.max_len + kRows - 1) / kRows;
  const long long grid = (long long)p.q_seqs.N * p.blocks * p.H;
  const size_t smem = smem_of(p.dn + p.dr, p.dv, false), most = smem_of(kMostNope + kMostRope, kMostValue, false);
  return bf16 ? go<latent_prompt_kernel<__nv_bfloat16>>(p, grid, smem, most, stream) : go<latent_prompt_kernel<float>>(p, grid, smem, most, stream);
}

cudaError_t launch_token_simt(bool bf16, const TokenParams& p, cudaStream_t stream) {
  const long long grid = p.N * (((long long)p.T * p.H + kRows - 1) / kRows);
  const size_t smem = smem_of(p.dl + p.dr, p.dl, true), most = smem_of(kMostLatent + kMostRope, kMostLatent, true);
  return bf16 ? go<latent_token_kernel<__nv_bfloat16>>(p, grid, smem, most, stream) : go<latent_token_kernel<float>>(p, grid, smem, most, stream);
}

}  // namespace mix
}  // namespace ha_la

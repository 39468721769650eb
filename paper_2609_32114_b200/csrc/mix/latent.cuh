// Attention over latent rows (ha_la_latent_* in ha_la.h): what its kernels and their host code share.
//
// Online softmax: with m the largest score so far, l = sum e^{s - m}, acc = sum e^{s - m} v; a larger score rescales both.  Exponentials are
// powers of two of scores times scale log2(e).
#pragma once

#include "mix.cuh"

namespace ha_la {
namespace mix {

constexpr float kNegInf = -INFINITY;
constexpr int kMostNope = 256, kMostRope = 128, kMostValue = 256, kMostLatent = 512;      // channels that calls may have

struct PromptParams {
  Seqs q_seqs, k_seqs;
  int H, dn, dr, dv, blocks;                               // blocks: of queries, of the longest sequence
  float scale;
  long long qs, kns, krs, vs, kn_hs, v_hs;
  const void *q, *kn, *kr, *v;
  void* o;
  float* lse;
  int32_t* status;
};

// One sequence's queries and keys; len -1 where either does not fit.
struct Span { int q0, q, k0, k; };
__device__ __forceinline__ Span span_of(const PromptParams& p, int n) {
  const Seq a = seq_of(p.q_seqs, n), b = seq_of(p.k_seqs, n);
  return {a.tok0, b.len < 0 ? -1 : a.len, b.tok0, b.len};
}
__device__ __forceinline__ void check_spans(const PromptParams& p) {
  check_seqs(p.q_seqs, p.status);
  check_seqs(p.k_seqs, p.status);
}

struct TokenParams {
  int N, T, H, dl, dr, page_log, pages, max_pages;
  float scale;
  const void *q, *cache;
  const int32_t *table, *lengths;
  void* o;
  float* lse;
  float *part_o, *part_ml;                                 // tensor cores: parts of sequences (latent_decode.cu)
  int32_t* status;
};

// Cached rows of a sequence; 0 if the length does not fit.
constexpr int kMostRows = 0x7fffffff - 255;                // (tables may name a page again and again; row numbers are 32 bits, tiles ahead of the last one included)
__device__ __forceinline__ int rows_of(const TokenParams& p, int n) {
  const int len = p.lengths[n];
  return len >= 0 && len <= kMostRows && (long long)len <= ((long long)p.max_pages << p.page_log) ? len : 0;
}
// One CTA's threads look at all lengths and report; a page that does not exist is reported by whoever wants a row of it.
__device__ __forceinline__ void check_tokens(const TokenParams& p) {
  if (!p.status) return;
  for (int n = threadIdx.x; n < p.N; n += blockDim.x)
    if (rows_of(p, n) != p.lengths[n]) report_status(p.status, HA_LA_ERR_DEVICE_CHECK);
}
// The cache's row of a sequence's row: in range whatever the table says.
__device__ __forceinline__ long long cache_row(const TokenParams& p, int n, int j) {
  int page = p.table[(long long)n * p.max_pages + (j >> p.page_log)];
  if (page < 0 || page >= p.pages) {
    report_status(p.status, HA_LA_ERR_DEVICE_CHECK);
    page = 0;
  }
  return ((long long)page << p.page_log) + (j & ((1 << p.page_log) - 1));
}

cudaError_t launch_prompt_simt(bool bf16, const PromptParams& p, cudaStream_t stream);
cudaError_t launch_prompt_tc(const PromptParams& p, cudaStream_t stream);
size_t token_tc_bytes(const TokenParams& p);
cudaError_t launch_token_tc(const TokenParams& p, void* workspace, cudaStream_t stream);
cudaError_t launch_token_simt(bool bf16, const TokenParams& p, cudaStream_t stream);

}  // namespace mix
}  // namespace ha_la

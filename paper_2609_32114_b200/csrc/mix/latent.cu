// C ABI of attention over latent rows: checks, dispatch.  See include/ha_la.h.
#include "latent.cuh"

using namespace ha_la;

namespace {

int check(const ha_la_latent_prefill_args* a, mix::PromptParams* p) {
  if (!a) return HA_LA_ERR_INVALID_ARG;
  if (a->dtype != HA_LA_BF16 && a->dtype != HA_LA_FP32) return HA_LA_ERR_INVALID_ARG;
  if (a->batch < 1 || a->num_heads < 1 || a->d_nope < 1 || a->d_rope < 0 || a->d_v < 1 || !(a->scale == a->scale)) return HA_LA_ERR_INVALID_ARG;
  if (a->d_nope > mix::kMostNope || a->d_rope > mix::kMostRope || a->d_v > mix::kMostValue || a->num_heads > 65535) return HA_LA_ERR_UNSUPPORTED;
  *p = mix::PromptParams{};
  if (!mix::make_seqs(&p->q_seqs, a->cu_seqlens, a->batch, a->seqlen, a->num_seqs, a->max_seqlen) ||
      !mix::make_seqs(&p->k_seqs, a->cu_seqlens_k, a->batch, a->seqlen_k, a->num_seqs, 0))
    return HA_LA_ERR_INVALID_ARG;
  if ((long long)a->batch * a->seqlen > 0x7fffffffLL - 256 || (long long)a->batch * a->seqlen_k > 0x7fffffffLL - 256) return HA_LA_ERR_UNSUPPORTED;
  p->H = a->num_heads; p->dn = a->d_nope; p->dr = a->d_rope; p->dv = a->d_v; p->scale = a->scale;
  const long long H = a->num_heads;
  auto stride = [](int64_t given, long long own, long long least, long long* out) {
    *out = given ? given : own;
    return *out >= least;
  };
  if (!stride(a->q_stride, H * (p->dn + p->dr), H * (p->dn + p->dr), &p->qs) || !stride(a->kr_stride, p->dr, p->dr, &p->krs) ||
      !stride(a->kn_head_stride, p->dn, p->dn, &p->kn_hs) || !stride(a->v_head_stride, p->dv, p->dv, &p->v_hs) ||
      !stride(a->kn_stride, H * p->kn_hs, p->dn, &p->kns) || !stride(a->v_stride, H * p->v_hs, p->dv, &p->vs))
    return HA_LA_ERR_INVALID_ARG;
  p->q = a->q; p->kn = a->kn; p->kr = a->kr; p->v = a->v; p->o = a->o; p->lse = a->lse; p->status = a->status_word;
  return HA_LA_OK;
}

// (a scale that is not positive would turn the largest score around, or mask with 0 * infinity)
bool on_tensor_cores(const ha_la_latent_prefill_args* a, const mix::PromptParams& p) {
  return a->dtype == HA_LA_BF16 && p.dn == 128 && p.dr == 64 && p.dv == 128 && p.scale > 0.f && mix::any_of(a->q, a->kn, a->kr, a->v, a->o) % 16 == 0 &&
         ((p.qs | p.kns | p.krs | p.vs | p.kn_hs | p.v_hs) & 7) == 0;
}

int check(const ha_la_latent_decode_args* a, mix::TokenParams* p) {
  if (!a) return HA_LA_ERR_INVALID_ARG;
  if (a->dtype != HA_LA_BF16 && a->dtype != HA_LA_FP32) return HA_LA_ERR_INVALID_ARG;
  if (a->num_seqs < 0 || a->new_tokens < 1 || a->num_heads < 1 || a->d_latent < 1 || a->d_rope < 0 || a->page_size < 1 || (a->page_size & (a->page_size - 1)) ||
      a->num_pages < 0 || a->max_pages < 0 || !(a->scale == a->scale))
    return HA_LA_ERR_INVALID_ARG;
  if (a->d_latent > mix::kMostLatent || a->d_rope > mix::kMostRope || (long long)a->new_tokens * a->num_heads > (1 << 20)) return HA_LA_ERR_UNSUPPORTED;
  if ((long long)a->num_pages * a->page_size > 0x7fffffffLL || (long long)a->num_seqs * a->new_tokens * a->num_heads > 0x7fffffffLL) return HA_LA_ERR_UNSUPPORTED;
  *p = mix::TokenParams{};
  p->N = a->num_seqs; p->T = a->new_tokens; p->H = a->num_heads; p->dl = a->d_latent; p->dr = a->d_rope;
  while ((1 << p->page_log) < a->page_size) ++p->page_log;
  p->pages = a->num_pages;
  p->max_pages = a->num_pages > 0 ? a->max_pages : 0;      // (without a page no length fits but zero)
  p->scale = a->scale;
  p->q = a->q; p->cache = a->cache; p->table = a->page_table; p->lengths = a->lengths; p->o = a->o; p->lse = a->lse; p->status = a->status_word;
  return HA_LA_OK;
}

// By sizes; a tensor that is not aligned goes the other way, which needs less room.
bool on_tensor_cores(const ha_la_latent_decode_args* a, const mix::TokenParams& p) {
  return a->dtype == HA_LA_BF16 && p.dl == 512 && p.dr == 64 && p.page_log >= 4 && p.scale > 0.f && (long long)p.N * p.T * p.H <= 0x7fffffffLL / 4;
}

}  // namespace

extern "C" {

const char* ha_la_latent_prefill_path(const ha_la_latent_prefill_args* a) {
  mix::PromptParams p;
  return check(a, &p) != HA_LA_OK ? nullptr : on_tensor_cores(a, p) ? "tc" : "simt";
}

int ha_la_latent_prefill(const ha_la_latent_prefill_args* a, void* cuda_stream) {
  mix::PromptParams p;
  const int rc = check(a, &p);
  if (rc != HA_LA_OK) return rc;
  if ((a->num_seqs > 0) != (a->cu_seqlens != nullptr) || (a->cu_seqlens != nullptr) != (a->cu_seqlens_k != nullptr)) return HA_LA_ERR_INVALID_ARG;
  const bool bf16 = a->dtype == HA_LA_BF16;
  if (mix::any_of(a->q, a->kn, a->kr, a->v, a->o) & (bf16 ? 1 : 3)) return HA_LA_ERR_INVALID_ARG;
  if (mix::any_of(a->lse, a->cu_seqlens, a->cu_seqlens_k, a->status_word) & 3) return HA_LA_ERR_INVALID_ARG;
  if (p.q_seqs.T_total == 0) return HA_LA_OK;
  if (!a->q || !a->o) return HA_LA_ERR_INVALID_ARG;
  if (p.k_seqs.T_total > 0 && (!a->kn || !a->v || (a->d_rope > 0 && !a->kr))) return HA_LA_ERR_INVALID_ARG;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = on_tensor_cores(a, p) ? mix::launch_prompt_tc(p, stream) : mix::launch_prompt_simt(bf16, p, stream);
  return e == cudaSuccess ? HA_LA_OK : HA_LA_ERR_CUDA;
}

const char* ha_la_latent_decode_path(const ha_la_latent_decode_args* a) {
  mix::TokenParams p;
  return check(a, &p) != HA_LA_OK ? nullptr : on_tensor_cores(a, p) && mix::any_of(a->q, a->cache, a->o) % 16 == 0 ? "tc" : "simt";
}

int ha_la_latent_decode_workspace_bytes(const ha_la_latent_decode_args* a, size_t* out_bytes) {
  if (!out_bytes) return HA_LA_ERR_INVALID_ARG;
  mix::TokenParams p;
  const int rc = check(a, &p);
  if (rc == HA_LA_OK) *out_bytes = on_tensor_cores(a, p) ? mix::token_tc_bytes(p) : 256;
  return rc;
}

int ha_la_latent_decode(const ha_la_latent_decode_args* a, void* cuda_stream) {
  mix::TokenParams p;
  const int rc = check(a, &p);
  if (rc != HA_LA_OK) return rc;
  if (p.N == 0) return HA_LA_OK;
  const bool bf16 = a->dtype == HA_LA_BF16;
  if (!a->q || !a->lengths || !a->o || (a->num_pages > 0 && !a->cache) || (a->max_pages > 0 && !a->page_table)) return HA_LA_ERR_INVALID_ARG;
  if (mix::any_of(a->q, a->cache, a->o) & (bf16 ? 1 : 3)) return HA_LA_ERR_INVALID_ARG;
  if (mix::any_of(a->lse, a->page_table, a->lengths, a->status_word) & 3) return HA_LA_ERR_INVALID_ARG;
  size_t need = 0;
  ha_la_latent_decode_workspace_bytes(a, &need);
  if (!a->workspace || ((uintptr_t)a->workspace & 255) || a->workspace_bytes < need) return HA_LA_ERR_WORKSPACE;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  const bool tc = on_tensor_cores(a, p) && mix::any_of(a->q, a->cache, a->o) % 16 == 0;
  const cudaError_t e = tc ? mix::launch_token_tc(p, a->workspace, stream) : mix::launch_token_simt(bf16, p, stream);
  return e == cudaSuccess ? HA_LA_OK : HA_LA_ERR_CUDA;
}

}  // extern "C"

// C ABI of gated linear attention: checks, workspace, dispatch.  See include/ha_la.h.
#include "tc.cuh"

using namespace ha_la;

namespace {

bool on_tensor_cores(const Problem& p) { return p.dtype == HA_LA_BF16 && p.dk == 128; }

// Shapes only.  Fills `p`.
int make_problem(const ha_la_gla_args* a, Problem* p) {
  if (!a) return HA_LA_ERR_INVALID_ARG;
  if (a->dtype != HA_LA_BF16 && a->dtype != HA_LA_FP32) return HA_LA_ERR_INVALID_ARG;
  if (a->batch < 1 || a->seqlen < 0) return HA_LA_ERR_INVALID_ARG;
  if (a->num_qk_heads < 1 || a->num_v_heads < 1 || a->num_v_heads % a->num_qk_heads != 0) return HA_LA_ERR_INVALID_ARG;
  if (a->d_k < 1 || a->d_v < 1) return HA_LA_ERR_INVALID_ARG;
  if (a->d_k != a->d_v || (a->d_k != 64 && a->d_k != 128)) return HA_LA_ERR_UNSUPPORTED;
  if (!(a->scale == a->scale)) return HA_LA_ERR_INVALID_ARG;
  const bool varlen = a->cu_seqlens != nullptr || a->num_seqs > 0;
  if (varlen && (a->batch != 1 || a->num_seqs < 1 || a->max_seqlen < 0)) return HA_LA_ERR_INVALID_ARG;
  const long long rows = (long long)a->batch * a->seqlen;
  if (rows > 0x7fffffffLL - 128) return HA_LA_ERR_UNSUPPORTED;   // token rows are indexed in int32
  *p = Problem{};
  p->variant = HA_LA_GDN;
  p->dtype = a->dtype;
  p->N = varlen ? a->num_seqs : a->batch;
  p->T_total = (int)rows;
  p->T_row = a->seqlen;
  p->HK = a->num_qk_heads;
  p->HV = a->num_v_heads;
  p->dk = a->d_k;
  p->dv = a->d_v;
  p->scale = a->scale;
  p->varlen = varlen ? 1 : 0;
  p->step = on_tensor_cores(*p) ? 128 : 64;
  const long long step = p->step;
  long long chunks;
  if (varlen) {
    p->max_len = (a->max_seqlen > 0 && a->max_seqlen < a->seqlen) ? a->max_seqlen : a->seqlen;
    chunks = (p->T_total + (step - 1) * p->N) / step;
  } else {
    p->max_len = a->seqlen;
    chunks = (long long)a->batch * ((a->seqlen + step - 1) / step);
  }
  p->max_seq_chunks = (int)((p->max_len + step - 1) / step);
  // CTAs are counted in 31 bits: chunks x V-heads (x parts of a chunk), sequences x V-heads x pieces of a state, pieces of dq
  if (chunks * p->HV > 0x7fffffffLL / (on_tensor_cores(*p) ? 1 : 2) || (long long)p->N * p->HV > 0x7fffffffLL / (p->dk * p->dv / 1024)) return HA_LA_ERR_UNSUPPORTED;
  if (rows * p->HK > 0x7fffffffLL * 8) return HA_LA_ERR_UNSUPPORTED;
  p->max_chunks = (int)chunks;
  p->planned_runs = p->runs = p->segments = 1;
  return HA_LA_OK;
}

size_t plan_part(const Problem& p) { return p.varlen ? plan_bytes(p) : 0; }

size_t bytes_of(const Problem& p, bool back) {
  const size_t n = on_tensor_cores(p) ? gla::tc_bytes(p, back, nullptr, nullptr, nullptr) : gla::simt_bytes(p, back, nullptr, nullptr);
  return align_up(plan_part(p) + (n > 0 ? n : 1), 256);
}

template <typename... P> uintptr_t any_of(P... p) { return (... | (uintptr_t)p); }

int run(const ha_la_gla_args* a, bool back, cudaStream_t stream) {
  gla::Call c = {};
  const int rc = make_problem(a, &c.p);
  if (rc != HA_LA_OK) return rc;
  c.a = *a;
  c.back = back;
  if (c.p.varlen && !a->cu_seqlens) return HA_LA_ERR_INVALID_ARG;
  if (any_of(a->g, a->cu_seqlens, a->status_word, back ? a->dg : nullptr) & 3) return HA_LA_ERR_INVALID_ARG;
  if (c.p.T_total > 0) {
    if (!a->q || !a->k || !a->v || !a->g) return HA_LA_ERR_INVALID_ARG;
    if (back ? !a->do_ || !a->dq || !a->dk || !a->dv || !a->dg : !a->o) return HA_LA_ERR_INVALID_ARG;
  }
  uintptr_t al16 = any_of(a->q, a->k, a->v, a->h0);
  al16 |= back ? any_of(a->do_, a->dhT, a->dq, a->dk, a->dv, a->dh0) : any_of(a->o, a->hT);
  if (al16 & 15) return HA_LA_ERR_INVALID_ARG;
  if (!a->workspace || ((uintptr_t)a->workspace & 255) || a->workspace_bytes < bytes_of(c.p, back)) return HA_LA_ERR_WORKSPACE;
  PlanView plan = {};
  if (c.p.varlen) {
    plan = plan_view(a->workspace, c.p);
    if (launch_plan(c.p, a->cu_seqlens, plan, a->status_word, stream) != cudaSuccess) return HA_LA_ERR_CUDA;
  }
  c.chunks = {plan.chunk_tok0, plan.chunk_len, plan.seq_chunk0, c.p.T_row, c.p.max_seq_chunks, c.p.step};
  void* scratch = reinterpret_cast<char*>(a->workspace) + plan_part(c.p);
  cudaError_t e;
  if (on_tensor_cores(c.p)) {
    gla::TcWork w = {};
    gla::tc_bytes(c.p, back, &w, &c.w, scratch);
    e = back ? gla::launch_tc_backward(c, plan, w, stream) : gla::launch_tc_forward(c, plan, w, stream);
  } else {
    gla::simt_bytes(c.p, back, &c.w, scratch);
    e = back ? gla::launch_simt_backward(c, stream) : gla::launch_simt_forward(c, stream);
  }
  return e == cudaSuccess ? HA_LA_OK : HA_LA_ERR_CUDA;
}

}  // namespace

extern "C" {

int ha_la_gla_workspace_bytes(const ha_la_gla_args* args, int backward, size_t* out_bytes) {
  if (!out_bytes) return HA_LA_ERR_INVALID_ARG;
  Problem p;
  const int rc = make_problem(args, &p);
  if (rc != HA_LA_OK) return rc;
  *out_bytes = bytes_of(p, backward != 0);
  return HA_LA_OK;
}

const char* ha_la_gla_path(const ha_la_gla_args* args) {
  Problem p;
  if (make_problem(args, &p) != HA_LA_OK) return nullptr;
  return on_tensor_cores(p) ? "tc" : "simt";
}

int ha_la_gla_prefill(const ha_la_gla_args* a, void* cuda_stream) { return run(a, false, reinterpret_cast<cudaStream_t>(cuda_stream)); }
int ha_la_gla_backward(const ha_la_gla_args* a, void* cuda_stream) { return run(a, true, reinterpret_cast<cudaStream_t>(cuda_stream)); }

}  // extern "C"

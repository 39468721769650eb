// Gated linear attention (ha_la_gla_* in ha_la.h): what its kernels and their host code share.
//
// A sequence is cut into chunks of `step` tokens (64 in fp32, 128 on the tensor cores).  With G the cumulative log-gate within a chunk,
// G_L its total, h the state in front of the chunk and dh the gradient of the state behind it, D_ij = e^{G_i - G_j} (j <= i):
//   S_ij = q_i . k_j    dP_ij = do_i . v_j    P = S D    dS = dP D
//   o  = scale [P v + e^{G_i} (q h)]                            h'  = e^{G_L} h + sum_j e^{G_L - G_j} k_j v_j^T
//   dq = scale [dS k + e^{G_i} (do h^T)]                        dh' = e^{G_L} dh + scale sum_i e^{G_i} q_i do_i^T   (in front of the chunk)
//   dk = scale dS^T q + e^{G_L - G_j} (v dh^T)
//   dv = scale P^T do + e^{G_L - G_j} (k dh)
//   dg_t = sum_{i >= t} x_i + sum_{j < t} y_j + e^{G_L} <h, dh> + sum_{i >= t > j} E_ij
//     x_i = scale e^{G_i} q_i . (h do_i),  y_j = e^{G_L - G_j} k_j . (dh v_j),  E = scale S dS: all that goes from before token t to it or behind it
// so that the states in front of (behind) all chunks are a scan of small matrices that each chunk makes by itself, and everything else is
// chunk-local.  No term of dg is a difference of large ones but the sums over E: sum over i >= t of (row i's sum - column i's sum), which
// leaves the roundings of all of the chunk's pairs behind, up to 2^-18 of their magnitudes.  (On the tensor cores rows and columns are
// sums of scores that were made separately.)
#pragma once

#include "common.cuh"

namespace ha_la {
namespace gla {

struct Chunks {                                            // where the chunks are: the plan kernel's table, or equal-length rows
  const int32_t *tok0, *len, *seq_chunk0;                  // NULL: chunk c of row n is slot n * cps + c
  int T_row, cps, step;
};

struct Geom { int tok0, L; };

__device__ __forceinline__ Geom geom_of(const Chunks& c, int slot) {
  if (c.len) return {c.tok0[slot], c.len[slot]};
  const int row = slot / c.cps, i = slot - row * c.cps;
  return {row * c.T_row + i * c.step, min(c.step, c.T_row - i * c.step)};
}

// A gate closes a token's past off long before -1000 (e^-104 is zero in fp32); as low as that at most, a chunk's sum keeps what comes
// behind a closed gate.
__device__ __forceinline__ double gate(float g) { return g < -1000.f ? -1000.0 : (double)g; }

struct Work {                                              // workspace behind the chunk table; h, dh: [slot][V-head][d_k][d_v] fp32
  float* total;                                            // [slot][V-head] e^{G_L}
  float* h;                                                // what a chunk adds to the state, then the state in front of it
  float* dh;                                               // backward: what it adds to the gradient, then the gradient behind it
  float *dq, *dk;                                          // backward, several V-heads per QK-head: fp32 parts [token][V-head or run of them][d]
};

struct Call {                                              // one call, as the launchers take it
  Problem p;
  ha_la_gla_args a;
  Chunks chunks;
  Work w;
  bool back;
};

size_t simt_bytes(const Problem& p, bool back, Work* w, void* base);
cudaError_t launch_simt_forward(const Call& c, cudaStream_t stream);
cudaError_t launch_simt_backward(const Call& c, cudaStream_t stream);
cudaError_t launch_combine(const Call& c, bool reverse, cudaStream_t stream);
// N x HV chains of `count` states each, one behind the other at [n][i][head]: total, s in place, from `first` (or zero)
cudaError_t launch_chain(const float* total, float* s, const float* first, int count, int N, int HV, int per_state, bool reverse, cudaStream_t stream);
cudaError_t launch_head_sums(const Call& c, int parts, cudaStream_t stream);   // of dq, dk: `parts` per token, HK heads

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

}  // namespace gla
}  // namespace ha_la

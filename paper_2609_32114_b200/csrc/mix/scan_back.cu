// Selective scan backward; see scan.cuh for the formulas.
//
// The states in front of every eight tokens come from a run of the forward recurrence (scan.cu).  Here a CTA goes through a sequence's tokens from the
// last to the first, 16 at a time, for CH channels: four warps make the eight tokens' states and decays from the kept one, hold them in registers
// (128 of them) and come back through them, so that a value costs two exponentials in all and the states never go through memory one by one.  Four
// other warps bring the next 16 tokens and finish the last ones.  Sums over states (dx, ddelta, p) and over channels (dB, dC) cross the lanes of a warp: with
// two channels and four states to a thread both are short (6 and 7 shuffles a token for 256 values); dB and dC then go over the warps in shared memory and
// over the channel blocks in a second kernel, in order.  What bounds it is the issue slots: some 150 instructions a token and warp.
#include "scan.cuh"

namespace ha_la {
namespace mix {
namespace {

constexpr int kThreads = 256, kTile = 16, SP = 4, CP = 2;

template <int LS> struct BackShape {
  static constexpr int LC = 32 / LS, WC = CP * LC, CH = 4 * WC, NP = SP * LS;
  // shared memory, in floats
  static constexpr int du = 0, g = du + 2 * kTile * CH * 2, b = g + 2 * kTile * CH, c = b + 2 * kTile * NP, res = c + 2 * kTile * NP,
                       bc = res + 2 * 3 * kTile * CH, floats = bc + 2 * 4 * kTile * 2 * NP;
};

template <typename In, int LS, bool GATE>
__global__ void __launch_bounds__(kThreads) scan_back_kernel(ScanParams p) {
  using S = BackShape<LS>;
  constexpr int LC = S::LC, CH = S::CH, NP = S::NP, E = CH / 8, BC = kTile * NP / 128;
  extern __shared__ __align__(16) float sm[];
  float* const s_du = sm + S::du;
  float* const s_g = sm + S::g;
  float* const s_b = sm + S::b;
  float* const s_c = sm + S::c;
  float* const s_res = sm + S::res;                        // [buffer][<dh, B>, <f, A> / ln 2, <C, h>][token][channel]
  float* const s_bc = sm + S::bc;                          // [buffer][warp][token][dB, dC][state]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int nb = p.blocks * p.G, n = blockIdx.x / nb, cb = blockIdx.x - n * nb, group = cb / p.blocks;
  const int c_in = (cb - group * p.blocks) * CH, left = min(CH, p.per_group - c_in), c0 = group * p.per_group + c_in;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const Seq q = seq_of(p.seqs, n);
  const int len = max(q.len, 0), tok0 = q.tok0, tiles = (len + kTile - 1) / kTile;
  const size_t state = (size_t)p.C * p.S;

  if (warp < 4) {
    const int cl = lane % LC, s0 = lane / LC * SP, g = lane / LC;
    int c[CP];
    bool mine[CP];
    float A[CP][SP], dh[CP][SP], dA[CP][SP] = {};
#pragma unroll
    for (int i = 0; i < CP; ++i) {
      c[i] = warp * S::WC + i * LC + cl;
      mine[i] = c[i] < left;
#pragma unroll
      for (int s = 0; s < SP; ++s) {
        const bool ok = mine[i] && s0 + s < p.S;
        const size_t at = (size_t)(c0 + c[i]) * p.S + s0 + s;
        A[i][s] = ok ? p.A[at] * kLog2e : 0.f;
        dh[i][s] = ok && p.dhT && q.len >= 0 ? p.dhT[n * state + at] : 0.f;
      }
    }
    const int ck0 = slot_of(p.seqs, n, tok0, kCkptLog, (p.seqs.T_row + kCkpt - 1) / kCkpt);
    Vec<SP> kept[CP] = {};
    auto fetch = [&](int chunk) {                          // the states in front of it
#pragma unroll
      for (int i = 0; i < CP; ++i)
        if (mine[i] && chunk >= 0 && chunk * kCkpt < len) kept[i] = load_v<SP>(p.ckpt + ((size_t)(ck0 + chunk) * p.C + c0 + c[i]) * NP + s0);
    };
    fetch((len - 1) >> kCkptLog);
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < tiles; ++i) {
      const int tile = tiles - 1 - i, buf = i & 1;
#pragma unroll 1
      for (int half = kTile / kCkpt - 1; half >= 0; --half) {
        const int chunk = tile * (kTile / kCkpt) + half, r0 = half * kCkpt;
        if (chunk * kCkpt >= len) continue;
        float first[CP][SP], h[kCkpt][CP][SP], a[kCkpt][CP][SP];
#pragma unroll
        for (int u = 0; u < CP; ++u)
#pragma unroll
          for (int s = 0; s < SP; ++s) first[u][s] = kept[u].v[s];
        fetch(chunk - 1);
#pragma unroll
        for (int j = 0; j < kCkpt; ++j) {
          const Vec<SP> bv = load_v<SP>(s_b + (buf * kTile + r0 + j) * NP + s0);
#pragma unroll
          for (int u = 0; u < CP; ++u) {
            const float2 du = *reinterpret_cast<const float2*>(s_du + ((buf * kTile + r0 + j) * CH + c[u]) * 2);
#pragma unroll
            for (int s = 0; s < SP; ++s) {
              a[j][u][s] = ex2(du.x * A[u][s]);
              h[j][u][s] = fmaf(a[j][u][s], j ? h[j - 1][u][s] : first[u][s], du.y * bv.v[s]);
            }
          }
        }
#pragma unroll
        for (int j = kCkpt - 1; j >= 0; --j) {
          const int r = r0 + j;
          const Vec<SP> bv = load_v<SP>(s_b + (buf * kTile + r) * NP + s0), cv = load_v<SP>(s_c + (buf * kTile + r) * NP + s0);
          float to_x[8] = {}, to_b[8] = {};                // by kind and channel; dB, dC
#pragma unroll
          for (int u = 0; u < CP; ++u) {
            const float2 du = *reinterpret_cast<const float2*>(s_du + ((buf * kTile + r) * CH + c[u]) * 2);
            const float gy = s_g[(buf * kTile + r) * CH + c[u]];
#pragma unroll
            for (int s = 0; s < SP; ++s) {
              dh[u][s] = fmaf(gy, cv.v[s], dh[u][s]);
              to_x[u] = fmaf(dh[u][s], bv.v[s], to_x[u]);
              if (GATE) to_x[4 + u] = fmaf(h[j][u][s], cv.v[s], to_x[4 + u]);
              to_b[s] = fmaf(dh[u][s], du.y, to_b[s]);
              to_b[4 + s] = fmaf(h[j][u][s], gy, to_b[4 + s]);
              dh[u][s] *= a[j][u][s];
              const float f = dh[u][s] * (j ? h[j - 1][u][s] : first[u][s]);
              to_x[2 + u] = fmaf(f, A[u][s], to_x[2 + u]);
              dA[u][s] = fmaf(f, du.x, dA[u][s]);
            }
          }
          spread_sum<8, ilog2(LS)>(to_x, 16);              // a lane's places: the top bits of g
          spread_sum<8, ilog2(LC)>(to_b, LC / 2);          // ... of cl
          constexpr int nx = LS >= 8 ? 1 : 8 / LS, nbc = LC >= 8 ? 1 : 8 / LC;
          const int px = LS >= 8 ? g / (LS / 8) : g * nx, pb = LC >= 8 ? cl / (LC / 8) : cl * nbc;
#pragma unroll
          for (int e = 0; e < nx; ++e) {
            const int kind = (px + e) / CP, u = (px + e) % CP;
            if (kind < (GATE ? 3 : 2) && (LS < 16 || g % 2 == 0)) s_res[((buf * 3 + kind) * kTile + r) * CH + warp * S::WC + u * LC + cl] = to_x[e];
          }
#pragma unroll
          for (int e = 0; e < nbc; ++e)
            s_bc[((((buf * 4 + warp) * kTile + r) * 2) + (pb + e) / SP) * NP + s0 + (pb + e) % SP] = to_b[e];
        }
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < CP; ++i)
#pragma unroll
      for (int s = 0; s < SP; ++s)
        if (mine[i] && s0 + s < p.S) {
          const size_t at = n * state + (size_t)(c0 + c[i]) * p.S + s0 + s;
          p.part_a[at] = dA[i][s];
          if (p.dh0 && q.len >= 0) p.dh0[at] = dh[i][s];
        }
    __syncthreads();
    return;
  }

  // ---- the helping warps: a token and E channels to a thread
  const int ht = tid - 128, row = ht / 8, c = ht % 8 * E, have = left - c;
  const bool vec = p.vec;
  const In *x = reinterpret_cast<const In*>(p.x) + c0 + c, *dt = reinterpret_cast<const In*>(p.dt) + c0 + c, *z = reinterpret_cast<const In*>(p.z) + c0 + c,
           *dy = reinterpret_cast<const In*>(p.dy) + c0 + c;
  const In *B = reinterpret_cast<const In*>(p.B) + (size_t)group * p.S, *C = reinterpret_cast<const In*>(p.C_) + (size_t)group * p.S;
  Vec<E> bias = {}, skip = {};
  float dD[E] = {}, dbias[E] = {};
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (p.dt_bias && e < have) bias.v[e] = p.dt_bias[c0 + c + e];
    if (p.D && e < have) skip.v[e] = p.D[c0 + c + e];
  }
  using Row = Raw<In, E>;
  Row rx = {}, rd = {}, rz = {}, rg = {};
  In rb[BC], rc[BC];
  auto rows = [&](int tile, Row& ax, Row& ad, Row& az, Row& ag) {
    const int t = tile * kTile + row;
    if (t >= len) return;
    ax = load_row<In, E>(x + (size_t)(tok0 + t) * p.xs, vec, have);
    ad = load_row<In, E>(dt + (size_t)(tok0 + t) * p.dts, vec, have);
    if (GATE) az = load_row<In, E>(z + (size_t)(tok0 + t) * p.zs, vec, have);
    ag = load_row<In, E>(dy + (size_t)(tok0 + t) * p.C, vec, have);
  };
  auto fetch = [&](int tile) {
    rows(tile, rx, rd, rz, rg);
#pragma unroll
    for (int j = 0; j < BC; ++j) {
      const int f = j * 128 + ht, r = tile * kTile + f / NP, s = f % NP;
      const bool ok = r < len && s < p.S;
      rb[j] = ok ? B[(size_t)(tok0 + r) * p.bs + s] : from_f32<In>(0.f);
      rc[j] = ok ? C[(size_t)(tok0 + r) * p.cs + s] : from_f32<In>(0.f);
    }
  };
  auto put = [&](int tile, int buf) {
    const bool in = tile * kTile + row < len;
    const Vec<E> vx = unpack_row<In, E>(rx), vd = unpack_row<In, E>(rd), vz = unpack_row<In, E>(rz), vg = unpack_row<In, E>(rg);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const bool ok = in && e < have;
      const float v = vd.v[e] + bias.v[e], delta = ok ? (p.softplus ? softplus(v) : v) : 0.f;
      *reinterpret_cast<float2*>(s_du + ((buf * kTile + row) * CH + c + e) * 2) = make_float2(delta, ok ? delta * vx.v[e] : 0.f);
      float gy = ok ? vg.v[e] : 0.f;
      if (GATE && ok) gy *= vz.v[e] * sigmoid(vz.v[e]);
      s_g[(buf * kTile + row) * CH + c + e] = gy;
    }
#pragma unroll
    for (int j = 0; j < BC; ++j) {
      const int f = j * 128 + ht;
      s_b[(buf * kTile + f / NP) * NP + f % NP] = to_f32(rb[j]);
      s_c[(buf * kTile + f / NP) * NP + f % NP] = to_f32(rc[j]);
    }
  };
  auto finish = [&](int tile, int buf, const Row& x_in, const Row& d_in, const Row& z_in, const Row& g_in) {
    const int t = tile * kTile + row;
    if (t < len) {
      const Vec<E> ax = unpack_row<In, E>(x_in), ad = unpack_row<In, E>(d_in), az = unpack_row<In, E>(z_in), ag = unpack_row<In, E>(g_in);
      Vec<E> dx, ddt, dz;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int at = row * CH + c + e;
        const float from_b = s_res[buf * 3 * kTile * CH + at], from_a = s_res[(buf * 3 + 1) * kTile * CH + at];
        const float v = ad.v[e] + bias.v[e], delta = p.softplus ? softplus(v) : v;
        float gy = ag.v[e];
        if (GATE) {
          const float sg = sigmoid(az.v[e]), out = fmaf(skip.v[e], ax.v[e], s_res[(buf * 3 + 2) * kTile * CH + at]);
          dz.v[e] = gy * out * sg * fmaf(az.v[e], 1.f - sg, 1.f);
          gy *= az.v[e] * sg;
        }
        dx.v[e] = fmaf(delta, from_b, skip.v[e] * gy);
        ddt.v[e] = fmaf(from_a, kLn2, ax.v[e] * from_b);
        if (p.softplus) ddt.v[e] *= sigmoid(v);
        dD[e] = fmaf(gy, ax.v[e], dD[e]);
        dbias[e] += ddt.v[e];
      }
      const size_t at = (size_t)(tok0 + t) * p.C + c0 + c;
      store_row<In, E>(reinterpret_cast<In*>(p.dx) + at, vec, have, dx);
      store_row<In, E>(reinterpret_cast<In*>(p.ddt) + at, vec, have, ddt);
      if (GATE) store_row<In, E>(reinterpret_cast<In*>(p.dz) + at, vec, have, dz);
    }
    constexpr int per = 2 * NP;
    for (int f = ht; f < kTile * per; f += 128) {
      const int r = f / per, t2 = tile * kTile + r;
      if (t2 >= len) break;
      const float* o = s_bc + (buf * 4 * kTile + r) * per + f % per;
      p.part_bc[((size_t)cb * p.seqs.T_total + tok0 + t2) * per + f % per] = (o[0] + o[kTile * per]) + (o[2 * kTile * per] + o[3 * kTile * per]);
    }
  };
  if (tiles > 0) {
    fetch(tiles - 1);
    put(tiles - 1, 0);
    if (tiles > 1) fetch(tiles - 2);
  }
  __syncthreads();
  Row ax = {}, ad = {}, az = {}, ag = {};                  // of the tile that is gone through now
#pragma unroll 1
  for (int i = 0; i <= tiles; ++i) {
    if (i + 1 < tiles) {
      put(tiles - 2 - i, (i + 1) & 1);
      if (i + 2 < tiles) fetch(tiles - 3 - i);
    }
    if (i > 0) finish(tiles - i, (i - 1) & 1, ax, ad, az, ag);
    if (i < tiles) {
      rows(tiles - 1 - i, ax, ad, az, ag);
      __syncthreads();
    }
  }
  // over the rows: through the places of the results, which nobody reads any more but the helping warps themselves
  __syncthreads();
  float* const s_sum = s_res;                              // [row][dD, dbias][channel]
#pragma unroll
  for (int e = 0; e < E; ++e) {
    s_sum[(row * 2) * CH + c + e] = dD[e];
    s_sum[(row * 2 + 1) * CH + c + e] = dbias[e];
  }
  asm volatile("bar.sync 1, 128;" ::: "memory");
  if (ht < 2 * CH) {
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < kTile; ++r) sum += s_sum[r * 2 * CH + ht];
    const int cc = ht % CH;
    if (cc < left) p.part_d[((size_t)n * 2 + ht / CH) * p.C + c0 + cc] = sum;
  }
}

// Over the sequences, in order: dA, dD, ddt_bias.
__global__ void __launch_bounds__(128) scan_sum_kernel(ScanParams p, float* dA, float* dD, float* ddt_bias) {
  const long long i = (long long)blockIdx.x * 128 + threadIdx.x, as = (long long)p.C * p.S;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  double s = 0;
  if (i < as) {
    for (int n = 0; n < p.seqs.N; ++n) s += p.part_a[n * as + i];
    dA[i] = (float)s;
  } else if (i < as + 2LL * p.C) {
    const long long j = i - as;
    for (int n = 0; n < p.seqs.N; ++n) s += p.part_d[n * 2LL * p.C + j];
    float* const out = j < p.C ? dD : ddt_bias;
    if (out) out[j < p.C ? j : j - p.C] = (float)s;
  }
}

// Over the channel blocks of a group, in order: dB and dC.
template <typename In>
__global__ void __launch_bounds__(128) scan_bc_kernel(ScanParams p, int np, In* dB, In* dC) {
  const long long i = (long long)blockIdx.x * 128 + threadIdx.x, per = 2LL * np;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const long long tg = i / per;
  const int r = (int)(i - tg * per), s = r % np;
  if (tg >= (long long)p.seqs.T_total * p.G || s >= p.S) return;
  const long long t = tg / p.G, g = tg - t * p.G, step = (long long)p.seqs.T_total * per;
  const float* part = p.part_bc + (g * p.blocks * p.seqs.T_total + t) * per + r;
  float sum = 0.f;
#pragma unroll 8
  for (int b = 0; b < p.blocks; ++b) sum += part[b * step];
  (r < np ? dB : dC)[tg * p.S + s] = from_f32<In>(sum);
}

template <typename In, int LS> cudaError_t launch(const ScanParams& p, cudaStream_t stream) {
  const size_t smem = BackShape<LS>::floats * sizeof(float);
  void (*k)(ScanParams) = p.z ? scan_back_kernel<In, LS, true> : scan_back_kernel<In, LS, false>;
  cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(k), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  const long long grid = (long long)p.seqs.N * p.blocks * p.G;
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  return start(k, dim3((unsigned)grid), kThreads, smem, stream, p);
}

template <typename In> cudaError_t launch_all(const ScanParams& p, int np, const ha_la_scan_args& a, cudaStream_t stream) {
  cudaError_t e = np == 16 ? launch<In, 4>(p, stream) : np == 32 ? launch<In, 8>(p, stream) : launch<In, 16>(p, stream);
  const long long sums = (long long)p.C * p.S + 2LL * p.C, bc = (long long)p.seqs.T_total * p.G * 2 * np;
  if (e == cudaSuccess && bc > 0)
    e = start(scan_bc_kernel<In>, dim3((unsigned)((bc + 127) / 128)), 128, 0, stream, p, np, reinterpret_cast<In*>(a.dB), reinterpret_cast<In*>(a.dC));
  if (e == cudaSuccess) e = start(scan_sum_kernel, dim3((unsigned)((sums + 127) / 128)), 128, 0, stream, p, a.dA, a.D ? a.dD : nullptr, a.dt_bias ? a.ddt_bias : nullptr);
  return e;
}

}  // namespace

int scan_back_channels(int padded_states) { return padded_states == 16 ? BackShape<4>::CH : padded_states == 32 ? BackShape<8>::CH : BackShape<16>::CH; }

cudaError_t launch_scan_back(bool bf16, ScanParams p, int padded_states, const ha_la_scan_args& a, cudaStream_t stream) {
  return bf16 ? launch_all<__nv_bfloat16>(p, padded_states, a, stream) : launch_all<float>(p, padded_states, a, stream);
}

}  // namespace mix
}  // namespace ha_la

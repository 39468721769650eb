// Selective scan backward; see scan.cuh for the formulas.
//
// The states in front of every eight tokens come from a run of the forward recurrence (scan.cu).  Here a CTA goes through a sequence's tokens from the
// last to the first, 16 at a time, for CH channels: eight warps make eight tokens' states from the kept one, hold them in registers and come back
// through them, so that the states never go through memory one by one; a decay is made three times in all, which is cheaper than the registers that would
// keep it (622 us against 667 with decays kept, two rows of 2048 tokens and 4096 channels; 634 since dA is summed by eights and in 64 bits).  Eight other warps bring the
// next 16 tokens and finish the last ones.  Sums over states (dx, ddelta, p) and over channels (dB, dC) cross the lanes of a warp, 10 shuffles a token; dB and
// dC then go over the warps in shared memory and over the channel blocks in a second kernel, in order.  What bounds it is the length of a token's own chain,
// products, two sums across lanes, results, with two such warps to a scheduler: issue slots are 54 % used.  (Four warps with two channels to a thread:
// 706 us; kept states sent for one part ahead instead of a tile: 758.)
#include "scan.cuh"

namespace ha_la {
namespace mix {
namespace {

constexpr int kWarps = 8, kScan = 32 * kWarps, kThreads = kScan + 256, kTile = 16, SP = 4;   // recurrence warps and threads
constexpr int kFlush = 4;                                  // tiles whose sums over tokens are in 32 bits: more of them lose what each adds to a long sequence's sum

template <typename In, int LS> struct BackShape {
  static constexpr int LC = 32 / LS, CH = kWarps * LC, NP = SP * LS;
  static constexpr int E = CH >= 32 ? CH / 16 : 2, TPR = CH / E;           // channels of a helping thread, threads to a token
  static constexpr int RES = kTile * CH + 8;                             // (three kinds that a warp writes at once, in banks of their own)
  // shared memory, in floats; then rows on their way, as they are in memory: x, dt, z, dy of four tiles, B and C of two
  static constexpr int du = 0, g = du + 2 * kTile * CH * 2, b = g + 2 * kTile * CH, c = b + 2 * kTile * NP, res = c + 2 * kTile * NP,
                       bc = res + 2 * 3 * RES, floats = bc + 2 * kWarps * kTile * 2 * NP;
  static constexpr int kRowB = E * sizeof(In), kQuadB = 4 * sizeof(In), QUADS = 2 * kTile * NP / 4, BC = (QUADS + 255) / 256;
  static constexpr size_t OFF_ROWS = floats * 4, OFF_BC = OFF_ROWS + 4 * 4 * 256 * kRowB;
  // ... and in 64 bits, a place to a thread: dA of the recurrence's, dD and the steps' gradients of the helping ones
  static constexpr size_t OFF_DA = OFF_BC + 2 * BC * 256 * kQuadB, OFF_DD = OFF_DA + SP * kScan * 8, bytes = OFF_DD + 2 * E * 256 * 8;
  static_assert(bytes <= 227 * 1024 && OFF_DA % 8 == 0, "shared memory");
};

template <typename In, int LS, bool GATE>
__global__ void __launch_bounds__(kThreads) scan_back_kernel(ScanParams p) {
  using S = BackShape<In, LS>;
  constexpr int LC = S::LC, CH = S::CH, NP = S::NP, E = S::E, BC = S::BC;
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

  if (warp < kWarps) {
    const int cl = lane % LC, g = lane / LC, s0 = g * SP, c = warp * LC + cl, du_at = step_piece(c / 2) * 4 + c % 2 * 2;
    const bool mine = c < left;
    float2 A[SP / 2], dh[SP / 2], dA[SP / 2] = {};         // (two states to an instruction)
#pragma unroll
    for (int s = 0; s < SP; ++s) {
      const bool ok = mine && s0 + s < p.S;
      const size_t at = (size_t)(c0 + c) * p.S + s0 + s;
      (&A[s / 2].x)[s % 2] = ok ? p.A[at] * kLog2e : 0.f;
      (&dh[s / 2].x)[s % 2] = ok && p.dhT && q.len >= 0 ? p.dhT[n * state + at] : 0.f;
    }
    double* const total = reinterpret_cast<double*>(reinterpret_cast<uint8_t*>(sm) + S::OFF_DA) + tid;
#pragma unroll
    for (int s = 0; s < SP; ++s) total[s * kScan] = 0;
    const int ck0 = slot_of(p.seqs, n, tok0, kCkptLog, (p.seqs.T_row + kCkpt - 1) / kCkpt);
    constexpr int PARTS = kTile / kCkpt;
    Vec<SP> kept[PARTS] = {};                              // the states in front of a tile's parts, sent for a tile ahead
    auto fetch = [&](int tile, int part) {
      const int chunk = tile * PARTS + part;
      if (mine && chunk >= 0 && chunk * kCkpt < len) kept[part] = load_v<SP>(p.ckpt + ((size_t)(ck0 + chunk) * p.C + c0 + c) * NP + s0);
    };
#pragma unroll
    for (int part = 0; part < PARTS; ++part) fetch(tiles - 1, part);
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < tiles; ++i) {
      const int tile = tiles - 1 - i, buf = i & 1;
#pragma unroll
      for (int part = PARTS - 1; part >= 0; --part) {
        const int r0 = part * kCkpt;
        if (tile * kTile + r0 >= len) {
          fetch(tile - 1, part);
          continue;
        }
        float2 first[SP / 2], h[kCkpt][SP / 2], sum_A[SP / 2];
#pragma unroll
        for (int s = 0; s < SP / 2; ++s) first[s] = make_float2(kept[part].v[2 * s], kept[part].v[2 * s + 1]);
        fetch(tile - 1, part);
        const float *const du0 = s_du + (buf * kTile + r0) * CH * 2 + du_at, *const g0 = s_g + (buf * kTile + r0) * CH + c;
        const float *const b0 = s_b + (buf * kTile + r0) * NP + s0, *const cc0 = s_c + (buf * kTile + r0) * NP + s0;
#pragma unroll
        for (int j = 0; j < kCkpt; ++j) {
          const Vec<SP> bv = load_v<SP>(b0 + j * NP);
          const float2 du = *reinterpret_cast<const float2*>(du0 + j * CH * 2);
#pragma unroll
          for (int s = 0; s < SP / 2; ++s) {
            h[j][s] = ptx::fma2(decay2(du.x, A[s]), j ? h[j - 1][s] : first[s], ptx::mul2(make_float2(du.y, du.y), make_float2(bv.v[2 * s], bv.v[2 * s + 1])));
          }
        }
#pragma unroll
        for (int j = kCkpt - 1; j >= 0; --j) {
          const Vec<SP> bv = load_v<SP>(b0 + j * NP), cv = load_v<SP>(cc0 + j * NP);
          const float2 du = *reinterpret_cast<const float2*>(du0 + j * CH * 2);
          const float gy = g0[j * CH];
          const float2 g2 = make_float2(gy, gy), u2 = make_float2(du.y, du.y);
          float to_x[4], to_b[8];                          // <dh, B>, <f, A>, <C, h>; dB, dC
          float2 from_b, from_a, out = make_float2(0.f, 0.f);
#pragma unroll
          for (int s = 0; s < SP / 2; ++s) {
            const float2 b2 = make_float2(bv.v[2 * s], bv.v[2 * s + 1]), c2 = make_float2(cv.v[2 * s], cv.v[2 * s + 1]);
            dh[s] = ptx::fma2(g2, c2, dh[s]);
            from_b = s ? ptx::fma2(dh[s], b2, from_b) : ptx::mul2(dh[s], b2);
            if (GATE) out = s ? ptx::fma2(h[j][s], c2, out) : ptx::mul2(h[j][s], c2);
            const float2 db = ptx::mul2(dh[s], u2), dc = ptx::mul2(h[j][s], g2);
            dh[s] = ptx::mul2(dh[s], decay2(du.x, A[s]));    // (made again: kept, decays take as many registers as the states)
            const float2 f = ptx::mul2(dh[s], j ? h[j - 1][s] : first[s]);
            from_a = s ? ptx::fma2(f, A[s], from_a) : ptx::mul2(f, A[s]);
            sum_A[s] = j == kCkpt - 1 ? ptx::mul2(f, make_float2(du.x, du.x)) : ptx::fma2(f, make_float2(du.x, du.x), sum_A[s]);
            to_b[2 * s] = db.x; to_b[2 * s + 1] = db.y;
            to_b[SP + 2 * s] = dc.x; to_b[SP + 2 * s + 1] = dc.y;
          }
          to_x[0] = from_b.x + from_b.y; to_x[1] = from_a.x + from_a.y; to_x[2] = out.x + out.y; to_x[3] = 0.f;
          spread_sum<4, ilog2(LS)>(to_x, 16);              // a lane's kind: the top two bits of g
          spread_sum<8, ilog2(LC)>(to_b, LC / 2);          // ... its places: the top bits of cl
          constexpr int nbc = LC >= 8 ? 1 : 8 / LC;
          const int kind = g / (LS / 4), pb = LC >= 8 ? cl / (LC / 8) : cl * nbc, r = r0 + j;
          if (kind < (GATE ? 3 : 2) && g % (LS / 4) == 0) s_res[(buf * 3 + kind) * S::RES + r * CH + c] = to_x[0];
#pragma unroll
          for (int e = 0; e < nbc; ++e) s_bc[((buf * kWarps + warp) * kTile + r) * 2 * NP + (pb + e) / SP * NP + s0 + (pb + e) % SP] = to_b[e];
        }
#pragma unroll
        for (int s = 0; s < SP / 2; ++s) dA[s] = ptx::add2(dA[s], sum_A[s]);   // (eight tokens at a time: token by token it is off by a third more)
      }
      if (i % kFlush == kFlush - 1) {
#pragma unroll
        for (int s = 0; s < SP; ++s) {
          total[s * kScan] += (&dA[s / 2].x)[s % 2];
          (&dA[s / 2].x)[s % 2] = 0.f;
        }
      }
      __syncthreads();
    }
#pragma unroll
    for (int s = 0; s < SP; ++s)
      if (mine && s0 + s < p.S) {
        const size_t at = n * state + (size_t)(c0 + c) * p.S + s0 + s;
        p.part_a[at] = (float)(total[s * kScan] + (&dA[s / 2].x)[s % 2]);
        if (p.dh0 && q.len >= 0) p.dh0[at] = (&dh[s / 2].x)[s % 2];
      }
    __syncthreads();
    return;
  }

  // ---- the helping warps: E channels of a token to a thread
  const int ht = tid - kScan, row = ht / S::TPR, c = ht % S::TPR * E, have = row < kTile ? left - c : 0;
  const bool vec = p.vec;
  const In *x = reinterpret_cast<const In*>(p.x) + c0 + c, *dt = reinterpret_cast<const In*>(p.dt) + c0 + c, *z = reinterpret_cast<const In*>(p.z) + c0 + c,
           *dy = reinterpret_cast<const In*>(p.dy) + c0 + c;
  const In *B = reinterpret_cast<const In*>(p.B) + (size_t)group * p.S, *C = reinterpret_cast<const In*>(p.C_) + (size_t)group * p.S;
  Vec<E> bias = {}, skip = {};
  float dD[E] = {}, dbias[E] = {};
  double* const totals = reinterpret_cast<double*>(reinterpret_cast<uint8_t*>(sm) + S::OFF_DD);       // [dD, dbias][channel of a thread][thread]
  auto flush = [&] {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      totals[e * 256 + ht] += dD[e];
      totals[(E + e) * 256 + ht] += dbias[e];
      dD[e] = dbias[e] = 0.f;
    }
  };
#pragma unroll
  for (int e = 0; e < 2 * E; ++e) totals[e * 256 + ht] = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (p.dt_bias && e < have) bias.v[e] = p.dt_bias[c0 + c + e];
    if (p.D && e < have) skip.v[e] = p.D[c0 + c + e];
  }
  // A thread's pieces, which nobody else looks at: rows of the i-th tile from the end in place i % 4 (they are wanted again for the results), B and C in place i % 2
  uint8_t* const own = reinterpret_cast<uint8_t*>(sm) + S::OFF_ROWS + ht * S::kRowB;
  auto row_at = [&](int i, int kind) { return own + ((i & 3) * 4 + kind) * 256 * S::kRowB; };
  auto row_of = [&](int i, int kind) { return unpack_row<In, E>(*reinterpret_cast<const Raw<In, E>*>(row_at(i, kind))); };
  auto bc_at = [&](int i, int j) { return reinterpret_cast<uint8_t*>(sm) + S::OFF_BC + (((i & 1) * BC + j) * 256 + ht) * S::kQuadB; };
  auto tile_of = [&](int i) { return tiles - 1 - i; };
  auto quad = [&](int j, int& which, int& r, int& s) {      // of B or C: its token and first state; false: there is none
    const int f = j * 256 + ht, in = f % (S::QUADS / 2) * 4;
    which = f / (S::QUADS / 2);
    r = in / NP;
    s = in % NP;
    return f < S::QUADS;
  };
  auto fetch = [&](int i) {
    const int t = tile_of(i) * kTile + row;
    if (t < len && have > 0) {
      stage_row<In, E>(row_at(i, 0), x + (size_t)(tok0 + t) * p.xs, vec, have);
      stage_row<In, E>(row_at(i, 1), dt + (size_t)(tok0 + t) * p.dts, vec, have);
      if (GATE) stage_row<In, E>(row_at(i, 2), z + (size_t)(tok0 + t) * p.zs, vec, have);
      stage_row<In, E>(row_at(i, 3), dy + (size_t)(tok0 + t) * p.C, vec, have);
    }
#pragma unroll
    for (int j = 0; j < BC; ++j) {
      int which, r, s;
      const bool ok = quad(j, which, r, s);
      const int tq = tile_of(i) * kTile + r;
      if (ok && tq < len) stage_row<In, 4>(bc_at(i, j), which ? C + (size_t)(tok0 + tq) * p.cs + s : B + (size_t)(tok0 + tq) * p.bs + s, p.bc_vec, p.S - s);
    }
  };
  auto put = [&](int i) {
    const int buf = i & 1;
    if (row < kTile) {
      const bool in = tile_of(i) * kTile + row < len;
      const Vec<E> vx = row_of(i, 0), vd = row_of(i, 1), vz = row_of(i, 2), vg = row_of(i, 3);
      Vec<E> gy;
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        float4 w;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const bool ok = in && e + k < have;
          const float v = vd.v[e + k] + bias.v[e + k], delta = ok ? (p.softplus ? softplus(v) : v) : 0.f;
          (&w.x)[2 * k] = delta;
          (&w.x)[2 * k + 1] = ok ? delta * vx.v[e + k] : 0.f;
          gy.v[e + k] = ok ? (GATE ? vg.v[e + k] * (vz.v[e + k] * sigmoid(vz.v[e + k])) : vg.v[e + k]) : 0.f;
        }
        *reinterpret_cast<float4*>(s_du + (buf * kTile + row) * CH * 2 + step_piece((c + e) / 2) * 4) = w;
      }
      store_v<E>(s_g + (buf * kTile + row) * CH + c, gy);
    }
#pragma unroll
    for (int j = 0; j < BC; ++j) {
      int which, r, s;
      if (!quad(j, which, r, s)) continue;
      Vec<4> w = {};
      if (tile_of(i) * kTile + r < len) w = unpack_row<In, 4>(*reinterpret_cast<const Raw<In, 4>*>(bc_at(i, j)));
      store_v<4>((which ? s_c : s_b) + (buf * kTile + r) * NP + s, w);
    }
  };
  auto finish = [&](int i) {
    const int buf = i & 1, t = tile_of(i) * kTile + row;
    if (t < len && have > 0) {
      const Vec<E> ax = row_of(i, 0), ad = row_of(i, 1), az = row_of(i, 2), ag = row_of(i, 3);
      const float* const res = s_res + buf * 3 * S::RES + row * CH + c;
      const Vec<E> from_b = load_v<E>(res), from_a = load_v<E>(res + S::RES);
      Vec<E> out = {};
      if (GATE) out = load_v<E>(res + 2 * S::RES);
      Vec<E> dx, ddt, dz;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float v = ad.v[e] + bias.v[e], delta = p.softplus ? softplus(v) : v;
        float gy = ag.v[e];
        if (GATE) {
          const float sg = sigmoid(az.v[e]);
          dz.v[e] = gy * fmaf(skip.v[e], ax.v[e], out.v[e]) * sg * fmaf(az.v[e], 1.f - sg, 1.f);
          gy *= az.v[e] * sg;
        }
        dx.v[e] = fmaf(delta, from_b.v[e], skip.v[e] * gy);
        ddt.v[e] = fmaf(from_a.v[e], kLn2, ax.v[e] * from_b.v[e]);
        if (p.softplus) ddt.v[e] *= sigmoid(v);
        if (e < have) {
          dD[e] = fmaf(gy, ax.v[e], dD[e]);
          dbias[e] += ddt.v[e];
        }
      }
      const size_t at = (size_t)(tok0 + t) * p.C + c0 + c;
      store_row<In, E>(reinterpret_cast<In*>(p.dx) + at, vec, have, dx);
      store_row<In, E>(reinterpret_cast<In*>(p.ddt) + at, vec, have, ddt);
      if (GATE) store_row<In, E>(reinterpret_cast<In*>(p.dz) + at, vec, have, dz);
    }
    constexpr int per = 2 * NP;
#pragma unroll
    for (int f = ht; f < kTile * per; f += 256) {
      const int r = f / per, t2 = tile_of(i) * kTile + r;
      if (t2 >= len) break;
      const float* o = s_bc + (buf * kWarps * kTile + r) * per + f % per;
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) sum += o[w * kTile * per];
      p.part_bc[((size_t)cb * p.seqs.T_total + tok0 + t2) * per + f % per] = sum;
    }
  };
  auto sent = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };
  // What is wanted for the next tile has been sent for two tiles before.
  if (tiles > 0) fetch(0);
  sent();
  if (tiles > 1) fetch(1);
  sent();
  asm volatile("cp.async.wait_group 1;" ::: "memory");
  if (tiles > 0) put(0);
  if (tiles > 2) fetch(2);
  sent();
  __syncthreads();
#pragma unroll 1
  for (int i = 0; i <= tiles; ++i) {
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    if (i + 1 < tiles) put(i + 1);
    if (i > 0) finish(i - 1);
    if (i % kFlush == 0) flush();
    if (i + 3 < tiles) fetch(i + 3);
    sent();
    if (i < tiles) __syncthreads();
  }
  // over the rows
  flush();
  __syncthreads();
  if (ht < 2 * CH) {
    const int kind = ht / CH, cc = ht % CH;
    double sum = 0;
#pragma unroll
    for (int r = 0; r < kTile; ++r) sum += totals[(kind * E + cc % E) * 256 + r * S::TPR + cc / E];
    if (cc < left) p.part_d[((size_t)n * 2 + kind) * p.C + c0 + cc] = (float)sum;
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
  constexpr size_t smem = BackShape<In, LS>::bytes;
  void (*k)(ScanParams) = p.z ? scan_back_kernel<In, LS, true> : scan_back_kernel<In, LS, false>;
  const cudaError_t e = p.z ? allow_smem<scan_back_kernel<In, LS, true>>(smem) : allow_smem<scan_back_kernel<In, LS, false>>(smem);
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

int scan_back_channels(int padded_states) { return padded_states == 16 ? BackShape<float, 4>::CH : padded_states == 32 ? BackShape<float, 8>::CH : BackShape<float, 16>::CH; }

cudaError_t launch_scan_back(bool bf16, ScanParams p, int padded_states, const ha_la_scan_args& a, cudaStream_t stream) {
  return bf16 ? launch_all<__nv_bfloat16>(p, padded_states, a, stream) : launch_all<float>(p, padded_states, a, stream);
}

}  // namespace mix
}  // namespace ha_la

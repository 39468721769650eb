// Selective scan forward and for one token; see scan.cuh for the formulas.
//
// A CTA has CH channels of a sequence (or of a segment of one) and goes through its tokens in order, 32 at a time.  Four warps hold the states, SP of them
// and 32 / LS channels to a warp's lanes, and do nothing but the recurrence, two states to an instruction; eight others make delta and delta x of the next
// 32 tokens (once a channel, not once a state), bring B and C, and finish the outputs of the last 32.  Their inputs come by asynchronous copies two tiles
// ahead, a thread's own pieces in shared memory; sums over a channel's lanes go through shared memory too.  (4096 tokens x 4096 channels: 155 us, 415 before
// both; eight sequences of 100 to 8000 tokens: 847.)
// Bounds, from the counters of the latter: the 20 special-function results of a (token, channel) with 16 states take 1.25 cycles of an SM at 16 a cycle,
// wavefronts of loads and stores 1.4, of 2.0 in all.  Few channels are spread over all SMs by giving a thread fewer states (SP 4, 2, 1) first, and only then
// are sequences cut into segments, whose states are made first, by all at once, at the price of every exponential twice.
#include <algorithm>

#include "scan.cuh"

namespace ha_la {
namespace mix {
namespace {

constexpr int kThreads = 384, kTile = 32;
constexpr int kRegs = 80, kScanRegs = 128, kHelpRegs = 56; // a thread's at launch, and as the roles share them out
static_assert(128 * kScanRegs + 256 * kHelpRegs <= kThreads * kRegs && 2 * kThreads * kRegs <= 65536, "register split");
enum Mode { kOut, kEnds, kKeep };                          // outputs; states behind segments; states in front of every 8 tokens

// Dynamic shared memory: what the recurrence takes, two tiles; rows on their way, as they are in memory (a thread's own pieces side by side).
template <typename In, int SP, int LS> struct Stage {
  static constexpr int CH = 128 / LS, NP = SP * LS, E = CH >= 16 ? CH / 8 : 2, BC = kTile * NP / 4 / 128;
  static constexpr uint32_t kRowB = E * sizeof(In), kQuadB = 4 * sizeof(In);
  static constexpr uint32_t OFF_B = 2 * kTile * CH * 8, OFF_C = OFF_B + 2 * kTile * NP * 4, OFF_X = OFF_C + 2 * kTile * NP * 4;
  static constexpr uint32_t OFF_DT = OFF_X + 4 * 256 * kRowB, OFF_Z = OFF_DT + 2 * 256 * kRowB, OFF_BC = OFF_Z + 2 * 256 * kRowB;
  static constexpr size_t bytes = OFF_BC + 2 * 256 * BC * kQuadB;
};

template <typename In, int SP, int LS, Mode M>
__global__ void __launch_bounds__(kThreads, 2) scan_kernel(ScanParams p) {
  constexpr int LC = 32 / LS, CH = 4 * LC, NP = SP * LS;   // channels of a warp, of the CTA; states
  constexpr int E = CH >= 16 ? CH / 8 : 2, TPR = CH / E;   // channels of a helping thread, threads to a token
  constexpr int BC = kTile * NP / 4 / 128;                 // quads of B (or C) that a helping thread brings
  using St = Stage<In, SP, LS>;
  extern __shared__ __align__(16) uint8_t dyn[];
  float4(*const s_du)[kTile][CH / 2] = reinterpret_cast<float4(*)[kTile][CH / 2]>(dyn);
  float(*const s_b)[kTile][NP] = reinterpret_cast<float(*)[kTile][NP]>(dyn + St::OFF_B);
  float(*const s_c)[kTile][NP] = reinterpret_cast<float(*)[kTile][NP]>(dyn + St::OFF_C);
  // (an object of its own, so that the compiler may move reads of the others ahead of what is written here)
  __shared__ __align__(16) float s_y[M == kOut ? 2 : 1][M == kOut ? kTile : 1][CH * LS];
  __shared__ int s_n;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int nb = p.blocks * p.G, unit = blockIdx.x / nb, cb = blockIdx.x - unit * nb, group = cb / p.blocks;
  const int c_in = (cb - group * p.blocks) * CH, left = min(CH, p.per_group - c_in), c0 = group * p.per_group + c_in;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0) check_seqs(p.seqs, p.status);
  // which sequence, and which tokens of it
  int n = unit, k = 0;
  if (p.seg_log < 31) {
    if (p.seqs.cu) {
      if (warp == 0) {
        const int f = find_seq(p.seqs, unit, p.seg_log, 1);
        if (lane == 0) s_n = f;
      }
      __syncthreads();
      n = s_n;
    } else {
      n = unit / p.segs;
    }
  }
  const Seq q = seq_of(p.seqs, n);
  if (q.len < 0) return;
  const int slot0 = p.seg_log < 31 ? slot_of(p.seqs, n, q.tok0, p.seg_log, p.segs) : 0;
  if (p.seg_log < 31) k = unit - slot0;
  const int L = p.seg_log < 31 ? 1 << p.seg_log : q.len;
  if (k < 0 || (k > 0 && (k > (q.len - 1) >> p.seg_log || p.seg_log == 31))) return;       // (a slot that no token falls to)
  const int start = k * (p.seg_log < 31 ? L : 0), len = min(L, q.len - start), tok0 = q.tok0 + start;
  if (M == kEnds && start + len >= q.len) {                // nobody asks for the state behind the last segment
    if (k > 0 || !p.first) return;
  }
  const int tiles = (len + kTile - 1) / kTile;

  if (warp < 4) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kScanRegs));
    const int c = warp * LC + lane % LC, s0 = lane / LC * SP, ch = c0 + c;
    const bool mine = c < left;
    float A[SP], h[SP];
#pragma unroll
    for (int s = 0; s < SP; ++s) {
      A[s] = mine && s0 + s < p.S ? p.A[(size_t)ch * p.S + s0 + s] * kLog2e : 0.f;
      h[s] = 0.f;
    }
    const size_t at = (size_t)ch * p.S + s0, state = (size_t)p.C * p.S;
    const bool moved = M == kOut && p.first;               // (in place, and in segments: hT may be written already)
    if (mine && k == 0) {
      if (moved) {
#pragma unroll
        for (int s = 0; s < SP; ++s) h[s] = p.first[((size_t)n * p.C + ch) * NP + s0 + s];
      } else if (p.h0) {
#pragma unroll
        for (int s = 0; s < SP; ++s)
          if (s0 + s < p.S) h[s] = p.h0[n * state + at + s];
      }
      if (M == kEnds && p.first) {
#pragma unroll
        for (int s = 0; s < SP; ++s) p.first[((size_t)n * p.C + ch) * NP + s0 + s] = h[s];
      }
    } else if (mine && M == kOut) {                        // through the segments in front; segment 0's end has h0 in it
#pragma unroll 4
      for (int j = 0; j < k; ++j) {
        const size_t sl = (size_t)(slot0 + j) * p.C + ch;
        const float total = p.seg_delta[sl];
        const Vec<SP> end = load_v<SP>(p.seg_h + sl * NP + s0);
#pragma unroll
        for (int s = 0; s < SP; ++s) h[s] = fmaf(ex2(A[s] * total), h[s], end.v[s]);
      }
    }
    if (M == kEnds && start + len >= q.len) return;
    constexpr int U = 8;
    const int du_at = step_piece(c / 2) * 2 + c % 2, sum = c * LS + lane / LC, y_at = sum_piece(sum / 4) * 4 + sum % 4;
    float total = 0.f;
    const int ck0 = M == kKeep ? slot_of(p.seqs, n, q.tok0, kCkptLog, (p.seqs.T_row + kCkpt - 1) / kCkpt) : 0;
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < tiles; ++i) {
      const int b = i & 1;
      float part = 0.f;
#pragma unroll 2
      for (int t0 = 0; t0 < kTile; t0 += U) {
        float yv[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
          if (M == kKeep && j % kCkpt == 0) {
            const int tk = i * kTile + t0 + j;
            if (mine && tk < len) {
              Vec<SP> now;
#pragma unroll
              for (int s = 0; s < SP; ++s) now.v[s] = h[s];
              store_v<SP>(p.ckpt + ((size_t)(ck0 + (tk >> kCkptLog)) * p.C + ch) * NP + s0, now);
            }
          }
          const float2 du = reinterpret_cast<const float2*>(&s_du[b][t0 + j][0])[du_at];
          const Vec<SP> bv = load_v<SP>(&s_b[b][t0 + j][s0]);
          if (M == kEnds) part += du.x;
          Vec<SP> cv;
          if (M == kOut) cv = load_v<SP>(&s_c[b][t0 + j][s0]);
          float y = 0.f;
          if constexpr (SP == 1) {
            h[0] = fmaf(decay(du.x, A[0]), h[0], du.y * bv.v[0]);
            if (M == kOut) y = h[0] * cv.v[0];
          } else {                                         // (two states to an instruction)
            float2 y2 = make_float2(0.f, 0.f);
#pragma unroll
            for (int s = 0; s < SP; s += 2) {
              const float2 hn = ptx::fma2(decay2(du.x, make_float2(A[s], A[s + 1])), make_float2(h[s], h[s + 1]),
                                          ptx::mul2(make_float2(du.y, du.y), make_float2(bv.v[s], bv.v[s + 1])));
              h[s] = hn.x;
              h[s + 1] = hn.y;
              if (M == kOut) y2 = s ? ptx::fma2(hn, make_float2(cv.v[s], cv.v[s + 1]), y2) : ptx::mul2(hn, make_float2(cv.v[s], cv.v[s + 1]));
            }
            y = y2.x + y2.y;
          }
          yv[j] = y;
        }
        if (M == kOut) {
#pragma unroll
          for (int j = 0; j < U; ++j) s_y[b][t0 + j][y_at] = yv[j];
        }
      }
      total += part;
      __syncthreads();
    }
    if (mine) {
      if (M == kEnds) {
        const size_t sl = (size_t)(slot0 + k) * p.C + ch;
#pragma unroll
        for (int s = 0; s < SP; ++s) p.seg_h[sl * NP + s0 + s] = h[s];
        if (s0 == 0) p.seg_delta[sl] = total;
      } else if (M == kOut && p.hT && start + len >= q.len) {
#pragma unroll
        for (int s = 0; s < SP; ++s)
          if (s0 + s < p.S) p.hT[n * state + at + s] = h[s];
      }
    }
    return;
  }

  // ---- the helping warps: E channels of a token to a thread
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kHelpRegs));
  if (M == kEnds && start + len >= q.len) return;
  const int ht = tid - 128, row = ht / TPR, c = ht % TPR * E, have = row < kTile ? left - c : 0;
  const bool vec = p.vec;
  const In *x = reinterpret_cast<const In*>(p.x) + c0 + c, *dt = reinterpret_cast<const In*>(p.dt) + c0 + c;
  const In *B = reinterpret_cast<const In*>(p.B) + (size_t)group * p.S, *C = reinterpret_cast<const In*>(p.C_) + (size_t)group * p.S;
  const In* z = reinterpret_cast<const In*>(p.z) + c0 + c;
  Vec<E> bias = {}, skip = {};
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (p.dt_bias && e < have) bias.v[e] = p.dt_bias[c0 + c + e];
    if (M == kOut && p.D && e < have) skip.v[e] = p.D[c0 + c + e];
  }
  // A thread's pieces, which nobody else looks at: x of tile i in place i % 4 (it is wanted again for the outputs), the others in place i % 2
  uint8_t* const own = dyn + ht * St::kRowB;
  auto x_at = [&](int i) { return own + St::OFF_X + (i & 3) * 256 * St::kRowB; };
  auto dt_at = [&](int i) { return own + St::OFF_DT + (i & 1) * 256 * St::kRowB; };
  auto z_at = [&](int i) { return own + St::OFF_Z + (i & 1) * 256 * St::kRowB; };
  auto bc_at = [&](int i, int j) { return dyn + St::OFF_BC + (((i & 1) * BC + j) * 256 + ht) * St::kQuadB; };
  const In* const bc = ht < 128 ? B : C;                   // the first 128 threads bring B, the others C
  const long long bc_step = ht < 128 ? p.bs : p.cs;
  const bool bc_mine = ht < 128 || M == kOut;
  auto fetch = [&](int i) {
    const int t = i * kTile + row;
    if (t < len && have > 0) {
      stage_row<In, E>(x_at(i), x + (size_t)(tok0 + t) * p.xs, vec, have);
      stage_row<In, E>(dt_at(i), dt + (size_t)(tok0 + t) * p.dts, vec, have);
    }
#pragma unroll
    for (int j = 0; j < BC; ++j) {
      const int f = (j * 128 + (ht & 127)) * 4, r = i * kTile + f / NP, s = f % NP;
      if (bc_mine && r < len) stage_row<In, 4>(bc_at(i, j), bc + (size_t)(tok0 + r) * bc_step + s, p.bc_vec, p.S - s);
    }
  };
  auto fetch_z = [&](int i) {
    const int t = i * kTile + row;
    if (M == kOut && p.z && t < len && have > 0) stage_row<In, E>(z_at(i), z + (size_t)(tok0 + t) * p.zs, vec, have);
  };
  auto put = [&](int i) {                                  // ... as the other warps take them
    const int b = i & 1;
    if (row < kTile) {
      const bool ok = i * kTile + row < len;
      const Vec<E> vx = unpack_row<In, E>(*reinterpret_cast<const Raw<In, E>*>(x_at(i))), vd = unpack_row<In, E>(*reinterpret_cast<const Raw<In, E>*>(dt_at(i)));
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        float4 w;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float u = vd.v[e + k] + bias.v[e + k], delta = ok && e + k < have ? (p.softplus ? softplus(u) : u) : 0.f;
          (&w.x)[2 * k] = delta;
          (&w.x)[2 * k + 1] = ok && e + k < have ? delta * vx.v[e + k] : 0.f;
        }
        s_du[b][row][step_piece((c + e) / 2)] = w;
      }
    }
#pragma unroll
    for (int j = 0; j < BC; ++j) {
      const int f = (j * 128 + (ht & 127)) * 4, r = f / NP, s = f % NP;
      Vec<4> w = {};
      if (i * kTile + r < len) w = unpack_row<In, 4>(*reinterpret_cast<const Raw<In, 4>*>(bc_at(i, j)));
      if (bc_mine) store_v<4>(ht < 128 ? &s_b[b][r][s] : &s_c[b][r][s], w);
    }
  };
  auto finish = [&](int i) {
    const int t = i * kTile + row;
    if (t >= len || have <= 0) return;
    const Vec<E> xi = unpack_row<In, E>(*reinterpret_cast<const Raw<In, E>*>(x_at(i))), zi = unpack_row<In, E>(*reinterpret_cast<const Raw<In, E>*>(z_at(i)));
    Vec<E> y = {};
#pragma unroll
    for (int k = 0; k < E * LS / 4; ++k) {
      const float4 part = *reinterpret_cast<const float4*>(&s_y[i & 1][M == kOut ? row : 0][sum_piece(c * LS / 4 + k) * 4]);
      y.v[k / (LS / 4)] += (part.x + part.y) + (part.z + part.w);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (p.D) y.v[e] = fmaf(skip.v[e], xi.v[e], y.v[e]);
      if (p.z) y.v[e] *= zi.v[e] * sigmoid(zi.v[e]);
    }
    store_row<In, E>(reinterpret_cast<In*>(p.y) + (size_t)(tok0 + t) * p.C + c0 + c, vec, have, y);
  };
  auto sent = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };
  // What is wanted while tile i is gone through has been sent for two tiles before.
  if (tiles > 0) {
    fetch(0);
    fetch_z(0);
  }
  sent();
  if (tiles > 1) fetch(1);
  sent();
  asm volatile("cp.async.wait_group 1;" ::: "memory");
  if (tiles > 0) put(0);
  if (tiles > 2) fetch(2);                                 // (its place was tile 0's)
  sent();
  __syncthreads();
#pragma unroll 1
  for (int i = 0; i <= tiles; ++i) {
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    if (i + 1 < tiles) put(i + 1);
    if (M == kOut && i > 0) finish(i - 1);
    if (i + 3 < tiles) fetch(i + 3);
    if (i + 1 < tiles) fetch_z(i + 1);
    sent();
    if (i < tiles) __syncthreads();
  }
}

// One token: a state is read and written once, so HBM bounds it (8 S bytes a channel).  LS lanes to a channel, four states each; a thread
// takes its channel of two sequences, whose states are on their way together, with one look at A; neighbouring lanes have neighbouring states, and B and C come
// four states at a time where they are aligned.  (256 sequences, 4096 channels, 16 states: 29.6 us, 4.8 TB/s; with neighbouring lanes on neighbouring
// channels, single values of B and C and four sequences 39.9.)
template <typename In, int LS, bool VEC>
__global__ void __launch_bounds__(128) scan_decode_kernel(ScanParams p) {
  constexpr int LC = 32 / LS, U = 2;
  const int lane = threadIdx.x & 31, s0 = lane % LS * 4;
  const int c = (blockIdx.x * 4 + (threadIdx.x >> 5)) * LC + lane / LS, ch = min(c, p.C - 1), group = ch / p.per_group;
  const bool mine = c < p.C;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const size_t state = (size_t)p.C * p.S, at = (size_t)ch * p.S + s0;
  auto four = [&](const float* a) {
    Vec<4> r = {};
    if (VEC) {
      const float4 w = __ldcs(reinterpret_cast<const float4*>(a));
      r.v[0] = w.x; r.v[1] = w.y; r.v[2] = w.z; r.v[3] = w.w;
    } else {
#pragma unroll
      for (int s = 0; s < 4; ++s)
        if (s0 + s < p.S) r.v[s] = a[s];
    }
    return r;
  };
  const Vec<4> A = VEC ? load_v<4>(p.A + at) : four(p.A + at);
  const float bias = p.dt_bias ? p.dt_bias[ch] : 0.f, skip = p.D ? p.D[ch] : 0.f;
  for (int n0 = blockIdx.y * U; n0 < p.seqs.N; n0 += gridDim.y * U) {
    Vec<4> h[U] = {};
    float x[U], dt[U], z[U];
    Vec<4> b[U], cc[U];
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (n0 + i < p.seqs.N && p.h0) h[i] = four(p.h0 + (n0 + i) * state + at);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int n = min(n0 + i, p.seqs.N - 1);
      x[i] = to_f32(reinterpret_cast<const In*>(p.x)[n * p.xs + ch]);
      dt[i] = to_f32(reinterpret_cast<const In*>(p.dt)[n * p.dts + ch]);
      z[i] = p.z ? to_f32(reinterpret_cast<const In*>(p.z)[n * p.zs + ch]) : 0.f;
      const In *B = reinterpret_cast<const In*>(p.B) + n * p.bs + (size_t)group * p.S + s0, *C = reinterpret_cast<const In*>(p.C_) + n * p.cs + (size_t)group * p.S + s0;
      if (VEC && p.bc_vec) {
        b[i] = load_v<4>(B); cc[i] = load_v<4>(C);
      } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          b[i].v[s] = s0 + s < p.S ? to_f32(B[s]) : 0.f;
          cc[i].v[s] = s0 + s < p.S ? to_f32(C[s]) : 0.f;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const float v = dt[i] + bias, delta = p.softplus ? softplus(v) : v, u = delta * x[i];
      float y = 0.f;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        h[i].v[s] = fmaf(decay(delta, A.v[s] * kLog2e), h[i].v[s], u * b[i].v[s]);
        y = fmaf(h[i].v[s], cc[i].v[s], y);
      }
#pragma unroll
      for (int off = LS / 2; off > 0; off >>= 1) y += __shfl_xor_sync(0xffffffffu, y, off);
      if (!mine || n0 + i >= p.seqs.N) continue;
      float* o = p.hT + (n0 + i) * state + at;
      if (VEC) {
        __stcs(reinterpret_cast<float4*>(o), make_float4(h[i].v[0], h[i].v[1], h[i].v[2], h[i].v[3]));
      } else {
#pragma unroll
        for (int s = 0; s < 4; ++s)
          if (s0 + s < p.S) o[s] = h[i].v[s];
      }
      if (s0 == 0) {
        y = fmaf(skip, x[i], y);
        if (p.z) y *= z[i] * sigmoid(z[i]);
        reinterpret_cast<In*>(p.y)[(size_t)(n0 + i) * p.C + ch] = from_f32<In>(y);
      }
    }
  }
}

int padded(int S) { return S <= 16 ? 16 : S <= 32 ? 32 : 64; }

struct Shape { int sp, ls, ch; };

// States to a thread: the most (the fewest shared-memory reads and sums a value) that still gives three SMs of four a CTA.  1024 tokens, 16 states, us, four, two
// and one to a thread: 128, 256, 512 CTAs 42, 48, 82; 64, 128, 256 42, 30, 42; 32, 64, 128 35, 29, 30; 512, 1024, 2048 131, 158, 285.  (Eight, two lanes to a channel: 68 for 64
// CTAs, and 998 instead of 848 for eight sequences of 100 to 8000 tokens and 4096 channels.)
Shape shape_of(int S, long long rows, int per_group, int G) {
  const int np = padded(S);
  Shape last = {};
  for (int sp = np == 16 ? 4 : 8; sp >= np / 16; sp /= 2) {
    const int ls = np / sp, ch = 128 / ls;
    last = {sp, ls, ch};
    if (rows * ((per_group + ch - 1) / ch) * G >= sm_count() * 3 / 4) break;
  }
  return last;
}

// Segments: tokens to one, by its logarithm, or 31.  Two passes over the tokens and a launch more have to pay.
int segment_log(const ScanParams& p, const Shape& s) {
  const long long ctas = (long long)p.seqs.N * ((p.per_group + s.ch - 1) / s.ch) * p.G;
  const int longest = p.seqs.max_len;
  if (ctas * 4 > sm_count() || longest < 512) return 31;
  int log = 7;
  while (((long long)1 << log) * sm_count() < ctas * longest && log < 30) ++log;
  return ((long long)2 << log) * 2 <= longest ? log : 31;
}

template <typename In, int SP, int LS> cudaError_t launch(Mode m, const ScanParams& p, long long units, cudaStream_t stream) {
  const long long grid = units * p.blocks * p.G;
  if (grid == 0) return cudaSuccess;
  constexpr size_t smem = Stage<In, SP, LS>::bytes;
  void (*k)(ScanParams) = m == kOut ? scan_kernel<In, SP, LS, kOut> : m == kEnds ? scan_kernel<In, SP, LS, kEnds> : scan_kernel<In, SP, LS, kKeep>;
  const cudaError_t e = m == kOut ? allow_smem<scan_kernel<In, SP, LS, kOut>>(smem, kRegs) : m == kEnds ? allow_smem<scan_kernel<In, SP, LS, kEnds>>(smem, kRegs)
                                                                                                  : allow_smem<scan_kernel<In, SP, LS, kKeep>>(smem, kRegs);
  return e == cudaSuccess ? start(k, dim3((unsigned)grid), kThreads, smem, stream, p) : e;
}

template <typename In> cudaError_t launch_shape(Mode m, const Shape& s, const ScanParams& p, long long units, cudaStream_t stream) {
  switch (s.sp * 100 + s.ls) {
    case 404: return launch<In, 4, 4>(m, p, units, stream);
    case 208: return launch<In, 2, 8>(m, p, units, stream);
    case 116: return launch<In, 1, 16>(m, p, units, stream);
    case 804: return launch<In, 8, 4>(m, p, units, stream);
    case 408: return launch<In, 4, 8>(m, p, units, stream);
    case 216: return launch<In, 2, 16>(m, p, units, stream);
    case 808: return launch<In, 8, 8>(m, p, units, stream);
    default: return launch<In, 4, 16>(m, p, units, stream);
  }
}

int check(const ha_la_scan_args* a, ScanParams* p, bool token) {
  if (!a) return HA_LA_ERR_INVALID_ARG;
  if (a->dtype != HA_LA_BF16 && a->dtype != HA_LA_FP32) return HA_LA_ERR_INVALID_ARG;
  if (a->batch < (token ? 0 : 1) || a->channels < 1 || a->groups < 1 || a->states < 1 || a->channels % a->groups) return HA_LA_ERR_INVALID_ARG;
  if (a->softplus != 0 && a->softplus != 1) return HA_LA_ERR_INVALID_ARG;
  if (a->states > 64 || a->channels > (1 << 24)) return HA_LA_ERR_UNSUPPORTED;
  *p = ScanParams{};
  if (!make_seqs(&p->seqs, a->cu_seqlens, a->batch, a->seqlen, token ? 0 : a->num_seqs, a->max_seqlen)) return HA_LA_ERR_INVALID_ARG;
  if ((long long)a->batch * a->seqlen > 0x7fffffffLL - 256) return HA_LA_ERR_UNSUPPORTED;
  const long long gs = (long long)a->groups * a->states;
  p->C = a->channels; p->S = a->states; p->G = a->groups; p->per_group = a->channels / a->groups;
  p->softplus = a->softplus;
  p->packed = !token && (a->cu_seqlens || a->num_seqs > 0);
  auto stride = [&](int64_t given, long long own, long long* out) {
    *out = given ? given : own;
    return given == 0 || given >= own;
  };
  if (!stride(a->x_stride, p->C, &p->xs) || !stride(a->dt_stride, p->C, &p->dts) || !stride(a->z_stride, p->C, &p->zs) ||
      !stride(a->b_stride, gs, &p->bs) || !stride(a->c_stride, gs, &p->cs))
    return HA_LA_ERR_INVALID_ARG;
  p->x = a->x; p->dt = a->dt; p->B = a->B; p->C_ = a->C; p->z = a->z; p->dy = a->dy;
  p->A = a->A; p->D = a->D; p->dt_bias = a->dt_bias; p->h0 = a->h0; p->dhT = a->dhT;
  p->y = a->y; p->dx = a->dx; p->ddt = a->ddt; p->dz = a->dz; p->hT = a->hT; p->dh0 = a->dh0;
  p->status = a->status_word;
  p->seg_log = 31;
  return HA_LA_OK;
}

// Sizes of a forward call: shape, segments, slots.
struct Plan { Shape s; long long units; size_t bytes; };

Plan forward_plan(ScanParams* p) {
  Plan f = {};
  f.s = shape_of(p->S, p->seqs.N, p->per_group, p->G);
  p->blocks = (p->per_group + f.s.ch - 1) / f.s.ch;
  p->seg_log = segment_log(*p, f.s);
  p->segs = 1;
  f.units = p->seqs.N;
  if (p->seg_log < 31) {
    const long long L = 1LL << p->seg_log;
    p->segs = (int)((p->seqs.T_row + L - 1) / L);
    f.units = p->packed ? (long long)(p->seqs.T_total >> p->seg_log) + p->seqs.N : (long long)p->seqs.N * p->segs;
    const size_t np = padded(p->S);
    f.bytes = align_up((size_t)f.units * p->C * (np + 1) * 4, 256) + align_up((size_t)p->seqs.N * p->C * np * 4, 256);
  }
  if (f.bytes == 0) f.bytes = 256;
  return f;
}

bool aligned_states(const ha_la_scan_args* a, const ScanParams& p) {
  const int e = a->dtype == HA_LA_BF16 ? 2 : 4;
  return any_of(a->B, a->C) % (4 * e) == 0 && ((p.bs | p.cs | p.S) & 3) == 0;
}

bool aligned_rows(const ha_la_scan_args* a, const ScanParams& p, bool back) {
  const int e = a->dtype == HA_LA_BF16 ? 2 : 4;
  uintptr_t at = any_of(a->x, a->dt, a->z);
  at |= back ? any_of(a->dy, a->dx, a->ddt, a->dz) : any_of(a->y);
  const long long steps = p.xs | p.dts | p.C | (a->z ? p.zs : 0) | (p.G > 1 ? p.per_group : 0);
  return at % 16 == 0 && steps * e % 16 == 0;
}

}  // namespace

// What the backward pass takes of the forward one: states in front of every eight tokens.
cudaError_t launch_scan_keep(bool bf16, ScanParams p, cudaStream_t stream) {
  p.seg_log = 31;
  const Shape s = shape_of(p.S, p.seqs.N, p.per_group, p.G);
  p.blocks = (p.per_group + s.ch - 1) / s.ch;
  return bf16 ? launch_shape<__nv_bfloat16>(kKeep, s, p, p.seqs.N, stream) : launch_shape<float>(kKeep, s, p, p.seqs.N, stream);
}
cudaError_t launch_scan_back(bool bf16, ScanParams p, int padded_states, const ha_la_scan_args& a, cudaStream_t stream);   // scan_back.cu
int scan_back_channels(int padded_states);

namespace {

size_t backward_bytes(ScanParams* p) {
  const size_t np = padded(p->S), ch = scan_back_channels((int)np), blocks = (p->per_group + ch - 1) / ch * p->G, T = p->seqs.T_total;
  const size_t slots = (T >> kCkptLog) + p->seqs.N + 1;
  p->blocks = (int)(blocks / p->G);
  return align_up(slots * p->C * np * 4, 256) + align_up(blocks * T * 2 * np * 4, 256) + align_up((size_t)p->seqs.N * p->C * p->S * 4, 256) +
         align_up((size_t)p->seqs.N * p->C * 2 * 4, 256) + 256;
}

int run(const ha_la_scan_args* a, bool back, cudaStream_t stream) {
  ScanParams p;
  const int rc = check(a, &p, false);
  if (rc != HA_LA_OK) return rc;
  if (a->num_seqs > 0 && !a->cu_seqlens) return HA_LA_ERR_INVALID_ARG;
  const bool bf16 = a->dtype == HA_LA_BF16;
  if (any_of(a->x, a->dt, a->B, a->C, a->z, a->y, a->dy, a->dx, a->ddt, a->dB, a->dC, a->dz) & (bf16 ? 1 : 3)) return HA_LA_ERR_INVALID_ARG;
  if (any_of(a->A, a->D, a->dt_bias, a->h0, a->hT, a->dhT, a->dA, a->dD, a->ddt_bias, a->dh0, a->cu_seqlens, a->status_word) & 3) return HA_LA_ERR_INVALID_ARG;
  if (!a->A) return HA_LA_ERR_INVALID_ARG;
  if (p.seqs.T_total > 0 && (!a->x || !a->dt || !a->B || !a->C)) return HA_LA_ERR_INVALID_ARG;
  if (p.seqs.T_total > 0 && (back ? !a->dy || !a->dx || !a->ddt || !a->dB || !a->dC || (a->z && !a->dz) : !a->y)) return HA_LA_ERR_INVALID_ARG;
  if (back && (!a->dA || (a->D && !a->dD) || (a->dt_bias && !a->ddt_bias))) return HA_LA_ERR_INVALID_ARG;
  p.vec = aligned_rows(a, p, back);
  p.bc_vec = aligned_states(a, p);
  if (!a->workspace || ((uintptr_t)a->workspace & 255)) return HA_LA_ERR_WORKSPACE;
  char* ws = reinterpret_cast<char*>(a->workspace);
  if (back) {
    if (a->workspace_bytes < backward_bytes(&p)) return HA_LA_ERR_WORKSPACE;
    const size_t np = padded(p.S), T = p.seqs.T_total, slots = (T >> kCkptLog) + p.seqs.N + 1;
    // (rows: a row's first slot is its number times the slots of a row, at most one more than its tokens / 8)
    const int back_blocks = p.blocks;
    p.ckpt = reinterpret_cast<float*>(ws); ws += align_up(slots * p.C * np * 4, 256);
    p.part_bc = reinterpret_cast<float*>(ws); ws += align_up((size_t)back_blocks * p.G * T * 2 * np * 4, 256);
    p.part_a = reinterpret_cast<float*>(ws); ws += align_up((size_t)p.seqs.N * p.C * p.S * 4, 256);
    p.part_d = reinterpret_cast<float*>(ws);
    if ((long long)p.seqs.N * p.C > 0x7fffffffLL || (long long)T * p.G > 0x7fffffffLL / 2) return HA_LA_ERR_UNSUPPORTED;
    cudaError_t e = launch_scan_keep(bf16, p, stream);
    p.blocks = back_blocks;
    if (e == cudaSuccess) e = launch_scan_back(bf16, p, (int)np, *a, stream);
    return e == cudaSuccess ? HA_LA_OK : HA_LA_ERR_CUDA;
  }
  const Plan f = forward_plan(&p);
  if (a->workspace_bytes < f.bytes) return HA_LA_ERR_WORKSPACE;
  if (f.units * p.blocks * p.G > 0x7fffffffLL) return HA_LA_ERR_UNSUPPORTED;
  cudaError_t e = cudaSuccess;
  if (p.seg_log < 31) {
    const size_t np = padded(p.S);
    p.seg_h = reinterpret_cast<float*>(ws);
    p.seg_delta = p.seg_h + (size_t)f.units * p.C * np;
    if (p.hT && p.hT == p.h0) p.first = reinterpret_cast<float*>(ws + align_up((size_t)f.units * p.C * (np + 1) * 4, 256));
    e = bf16 ? launch_shape<__nv_bfloat16>(kEnds, f.s, p, f.units, stream) : launch_shape<float>(kEnds, f.s, p, f.units, stream);
  }
  if (e == cudaSuccess) e = bf16 ? launch_shape<__nv_bfloat16>(kOut, f.s, p, f.units, stream) : launch_shape<float>(kOut, f.s, p, f.units, stream);
  return e == cudaSuccess ? HA_LA_OK : HA_LA_ERR_CUDA;
}

template <typename In> cudaError_t launch_decode(const ScanParams& p, bool vec, cudaStream_t stream) {
  const int ls = padded(p.S) / 4, per_cta = 4 * (32 / ls);
  const int gx = (p.C + per_cta - 1) / per_cta, n4 = (p.seqs.N + 1) / 2;
  const int gy = std::min(n4, std::max(1, sm_count() * 32 / gx));          // (32 CTAs an SM: 29.6 us; 16 30.2, 128 33.0)
  void (*k)(ScanParams) = ls == 4 ? (vec ? scan_decode_kernel<In, 4, true> : scan_decode_kernel<In, 4, false>)
                        : ls == 8 ? (vec ? scan_decode_kernel<In, 8, true> : scan_decode_kernel<In, 8, false>)
                                  : (vec ? scan_decode_kernel<In, 16, true> : scan_decode_kernel<In, 16, false>);
  return start(k, dim3((unsigned)gx, (unsigned)std::min(gy, 65535)), 128, 0, stream, p);
}

}  // namespace
}  // namespace mix
}  // namespace ha_la

using namespace ha_la;

extern "C" {

int ha_la_scan_workspace_bytes(const ha_la_scan_args* a, int backward, size_t* out_bytes) {
  if (!out_bytes) return HA_LA_ERR_INVALID_ARG;
  mix::ScanParams p;
  const int rc = mix::check(a, &p, false);
  if (rc != HA_LA_OK) return rc;
  *out_bytes = backward ? mix::backward_bytes(&p) : mix::forward_plan(&p).bytes;
  return HA_LA_OK;
}
int ha_la_scan(const ha_la_scan_args* a, void* s) { return mix::run(a, false, reinterpret_cast<cudaStream_t>(s)); }
int ha_la_scan_backward(const ha_la_scan_args* a, void* s) { return mix::run(a, true, reinterpret_cast<cudaStream_t>(s)); }

int ha_la_scan_decode(const ha_la_scan_args* a, void* cuda_stream) {
  mix::ScanParams p;
  const int rc = mix::check(a, &p, true);
  if (rc != HA_LA_OK) return rc;
  if (a->seqlen != 1 || a->cu_seqlens || a->num_seqs) return HA_LA_ERR_INVALID_ARG;
  if (p.seqs.N == 0) return HA_LA_OK;
  const bool bf16 = a->dtype == HA_LA_BF16;
  if (!a->x || !a->dt || !a->A || !a->B || !a->C || !a->y || !a->hT) return HA_LA_ERR_INVALID_ARG;
  if (mix::any_of(a->x, a->dt, a->B, a->C, a->z, a->y) & (bf16 ? 1 : 3)) return HA_LA_ERR_INVALID_ARG;
  if (mix::any_of(a->A, a->D, a->dt_bias, a->h0, a->hT) & 3) return HA_LA_ERR_INVALID_ARG;
  p.bc_vec = mix::aligned_states(a, p);
  const bool vec = p.S == mix::padded(p.S) && mix::any_of(a->A, a->h0, a->hT) % 16 == 0;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = bf16 ? mix::launch_decode<__nv_bfloat16>(p, vec, stream) : mix::launch_decode<float>(p, vec, stream);
  return e == cudaSuccess ? HA_LA_OK : HA_LA_ERR_CUDA;
}

}  // extern "C"

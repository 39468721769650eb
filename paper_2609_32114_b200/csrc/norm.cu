// The norms on both sides of a block (ha_la_gated_norm, ha_la_add_norm in ha_la.h), forward and backward.
//
//   gated_norm   y = x rs w act(z)                     rs = 1 / sqrt(mean(x^2) + eps) of the row
//     backward   with dn = dy w act(z):  dx = rs (dn - x rs^2 mean(dn x)),  dz = dy x rs w act'(z),  dw = sum over rows of dy x rs act(z)
//   add_norm     r' = r + s f,  f = x or x rx w_post;  y = r' rs w
//     backward   with dn = dy w:  dr = dr' + rs (dn - r' rs^2 mean(dn r')),  dw = sum dy r' rs;  df = s dr, and with a norm behind the block
//                dw_post = sum df x rx,  dx = rx (dm - x rx^2 mean(dm x)) with dm = df w_post
// Grouped so that no value is of a higher power of the row's size than the first: dx = rs dn + (x rs) m with m = -(rs mean(dn x)) rs.  (rs^3 alone
// leaves fp32 for rows of 1e13 and of 1e-13.)
// Nothing is kept from the forward pass: the row is there anyway, so its norm costs no traffic.  The sums that do not wait for one another
// go through one reduction (mean(dn x) is taken of x, not of x rs), so a row needs one, two with w_post.
//
// What bounds them is HBM, and latency in small calls; in large bf16 ones HBM is busy for half of its cycles only.  Counters, 262144 rows of 128 and 16384 of 2048 with both norms:
// forward 46 us (issue slots 68 % used, the pipe of exponentials and quotients 50 %) and 76 (the pipe of shared memory and exchanges 72 %, the sums of two
// norms); backward 73 (issue 66 %) and 91 (61 %), by 16 warps of 122 to 128 registers on an SM, which wait for their own arithmetic more
// than for loads.  fp32 moves twice the bytes by much the same instructions: 5.1 to 6.2 TB/s.  A row lies in registers, 16 bytes of each tensor to a thread: rows of up to 32
// vectors are shared by 1, 2, 4 .. 32 neighbouring lanes, longer ones by a CTA.  A row that does not start on a 16-byte boundary is
// read in aligned vectors all the same, with the neighbours' values at its ends masked: a group's rows are a multiple of 8 apart, so the
// column that an element of a thread holds is the same in every row, weights stay in registers and so do the sums for dw, which
// a second kernel adds up over CTAs in order (no atomics: the same bits every time).  Rows in flight: the backward loops copy the next rows to shared
// memory asynchronously, each thread for itself; with the next row in registers instead 262144 rows of 128 took 89 us instead of 73, 16384
// of 2048 with both norms 105 instead of 91.
#include "common.cuh"
#include "tc_mma.cuh"

namespace ha_la {

namespace {

constexpr int kSubThreads = 256;                         // CTA of the short rows (several rows to a warp or to a CTA)
constexpr int kMaxCols = 16384;
constexpr int kReduceThreads = 1024;

struct NormParams {
  const void *x, *z, *r, *dy, *dr_out;                   // z: the gate; r: residual stream (backward: behind the addition)
  const float *w, *w_post;
  void *y, *r_out, *dx, *dz, *dr;
  float *part;                                           // backward: [CTA][1 or 2][cols] sums of a CTA's rows
  long long rows;
  int cols, group;                                       // group: lanes that share a row (short rows)
  int sigmoid;
  float eps, scale;
};

// ---------------------------------------------------------------- vectors of a row

template <typename In, int VEC> struct Raw { In e[VEC]; };
template <> struct Raw<__nv_bfloat16, 8> { uint4 v; };
template <> struct Raw<float, 4> { float4 v; };

__device__ __forceinline__ void to_floats(const Raw<__nv_bfloat16, 8>& a, float (&f)[8]) {
  const uint32_t w[4] = {a.v.x, a.v.y, a.v.z, a.v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void to_floats(const Raw<float, 4>& a, float (&f)[4]) { f[0] = a.v.x; f[1] = a.v.y; f[2] = a.v.z; f[3] = a.v.w; }
template <typename In> __device__ __forceinline__ void to_floats(const Raw<In, 1>& a, float (&f)[1]) { f[0] = to_f32(a.e[0]); }
__device__ __forceinline__ Raw<__nv_bfloat16, 8> from_floats(const float (&f)[8], __nv_bfloat16) {
  Raw<__nv_bfloat16, 8> a;
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  a.v = make_uint4(w[0], w[1], w[2], w[3]);
  return a;
}
__device__ __forceinline__ Raw<float, 4> from_floats(const float (&f)[4], float) { return {make_float4(f[0], f[1], f[2], f[3])}; }
template <typename In> __device__ __forceinline__ Raw<In, 1> from_floats(const float (&f)[1], In) { return {{from_f32<In>(f[0])}}; }

// Elementwise arithmetic on what a thread holds of a row, two to an instruction where there are two.
template <int N> struct Vec {
  float v[N];
  __device__ __forceinline__ float& operator[](int i) { return v[i]; }
  __device__ __forceinline__ float operator[](int i) const { return v[i]; }
};
template <int N> __device__ __forceinline__ Vec<N> all_of(float x) {
  Vec<N> r;
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = x;
  return r;
}
template <int N> __device__ __forceinline__ Vec<N> mul(const Vec<N>& a, const Vec<N>& b) {
  Vec<N> r;
  if constexpr (N == 1) r[0] = a[0] * b[0];
  else {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 x = ptx::mul2(make_float2(a[i], a[i + 1]), make_float2(b[i], b[i + 1]));
      r[i] = x.x;
      r[i + 1] = x.y;
    }
  }
  return r;
}
template <int N> __device__ __forceinline__ Vec<N> fma(const Vec<N>& a, const Vec<N>& b, const Vec<N>& c) {
  Vec<N> r;
  if constexpr (N == 1) r[0] = fmaf(a[0], b[0], c[0]);
  else {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 x = ptx::fma2(make_float2(a[i], a[i + 1]), make_float2(b[i], b[i + 1]), make_float2(c[i], c[i + 1]));
      r[i] = x.x;
      r[i + 1] = x.y;
    }
  }
  return r;
}
template <int N> __device__ __forceinline__ Vec<N> mul(const Vec<N>& a, float b) { return mul(a, all_of<N>(b)); }
template <int N> __device__ __forceinline__ Vec<N> fma(const Vec<N>& a, float b, const Vec<N>& c) { return fma(a, all_of<N>(b), c); }
// s + the sum of a b
template <int N> __device__ __forceinline__ float dot(const Vec<N>& a, const Vec<N>& b, float s) {
  if constexpr (N == 1) return fmaf(a[0], b[0], s);
  else {
    float2 x = make_float2(s, 0.f);
#pragma unroll
    for (int i = 0; i < N; i += 2) x = ptx::fma2(make_float2(a[i], a[i + 1]), make_float2(b[i], b[i + 1]), x);
    return x.x + x.y;
  }
}

// Which part of a row a thread holds: NV vectors of VEC elements, the group's threads one behind the other, the first one's first vector `shift`
// elements in front of the row's start, on a 16-byte boundary.
// FULL: rows are whole vectors, so they all start on a boundary.
template <typename In, int VEC, int NV, bool SUB, bool FULL>
struct Rows {
  int t, threads, shift, cols;
  long long row, step, rows, total;                      // this group's first row, rows between its rows
  // Of rows that start anywhere: the bits of a vector that are the row's, and for a vector at one of its ends (not both) the pieces of 8, 4 and
  // 2 bytes that it is stored in, as 1 + the piece's place or 0.  The same for every row of the group; kept for the first vector of a thread only.
  uint4 mask;
  uint32_t pieces;
  __device__ __forceinline__ explicit Rows(const NormParams& p) {
    threads = SUB ? p.group : blockDim.x;
    t = SUB ? threadIdx.x & (p.group - 1) : threadIdx.x;
    const int groups = SUB ? kSubThreads / p.group : 1;
    row = SUB ? (long long)blockIdx.x * groups + threadIdx.x / p.group : blockIdx.x;
    step = (long long)gridDim.x * groups;                // (a multiple of VEC unless a group has one row only)
    rows = p.rows;
    cols = p.cols;
    total = p.rows * p.cols;
    shift = FULL ? 0 : (int)((row * cols) & (VEC - 1));
    pieces = 0;
    if constexpr (!FULL && VEC > 1) {
      const int first = max(0, -col(0, 0)), end = min(VEC, cols - col(0, 0));   // elements of the vector that are the row's
      uint32_t m[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        m[k] = 0;
#pragma unroll
        for (int e = k * VEC / 4; e < (k + 1) * VEC / 4; ++e)
          if (e >= first && e < end) m[k] |= VEC == 4 ? 0xffffffffu : 0xffffu << 16 * (e & 1);
      }
      mask = make_uint4(m[0], m[1], m[2], m[3]);
      if (end - first > 0 && end - first < VEC && (first == 0 || end == VEC)) {
        // a run from `first` up to the vector's end: the smaller pieces come first; one from its start up to `end`: the larger ones do
        const int unit = 16 / VEC, n = (end - first) * unit;   // bytes
        const int base = first * unit;
        int at2 = -1, at4 = -1, at8 = -1;
        if (first > 0) {
          int o = base;
          if (n & 2) { at2 = o; o += 2; }
          if (n & 4) { at4 = o; o += 4; }
          if (n & 8) at8 = o;
        } else {
          int o = 0;
          if (n & 8) { at8 = o; o += 8; }
          if (n & 4) { at4 = o; o += 4; }
          if (n & 2) at2 = o;
        }
        pieces = (uint32_t)(at8 + 1) | (uint32_t)(at4 + 1) << 8 | (uint32_t)(at2 + 1) << 16 | 1u << 24;
      }
    }
  }
  // the loop over a group's rows goes on as long as any group of the CTA has one: its threads meet in the sums
  __device__ __forceinline__ bool on(long long r) const {
    return SUB ? r - threadIdx.x / threads < rows : r < rows;
  }
  // Is there such a row?  Of the `together` rows that are worked on at once the first always is, but in CTAs of short rows, which have places left over:
  // all zeros, so that their scale is infinite with eps = 0, and zero times that must not get into a sum over rows.
  __device__ __forceinline__ bool there(long long r, int together) const { return (!SUB && together == 1) || r < rows; }
  __device__ __forceinline__ int col(int i, int e) const { return VEC * (t + i * threads) - (FULL ? 0 : shift) + e; }
  __device__ __forceinline__ bool in(int i, int e) const { return FULL ? col(i, 0) < cols : (unsigned)col(i, e) < (unsigned)cols; }
  __device__ __forceinline__ bool any(int i) const { return FULL ? col(i, 0) < cols : col(i, VEC - 1) >= 0 && col(i, 0) < cols; }
  __device__ __forceinline__ bool whole(int i) const { return FULL ? col(i, 0) < cols : col(i, 0) >= 0 && col(i, VEC - 1) < cols; }
  __device__ __forceinline__ Raw<In, VEC> load(const void* base, long long r, int i) const {
    Raw<In, VEC> a = {};
    if (r < rows && any(i)) {
      const long long at = r * cols + col(i, 0);         // (>= 0: a whole vector of the tensor, or the one at its end)
      const In* src = reinterpret_cast<const In*>(base) + at;
      if (FULL || at + VEC <= total) a = *reinterpret_cast<const Raw<In, VEC>*>(src);
      else {
        In* e = reinterpret_cast<In*>(&a);
        for (int k = 0; k < VEC && at + k < total; ++k) e[k] = src[k];
      }
    }
    return a;
  }
  __device__ __forceinline__ Vec<VEC> unpack(const Raw<In, VEC>& a, int i) const {
    Vec<VEC> f;
    if constexpr (!FULL && VEC > 1 && NV == 1) {
      uint4 w = *reinterpret_cast<const uint4*>(&a);
      w.x &= mask.x; w.y &= mask.y; w.z &= mask.z; w.w &= mask.w;
      to_floats(*reinterpret_cast<const Raw<In, VEC>*>(&w), f.v);
      return f;
    }
    to_floats(a, f.v);
    if (!FULL && VEC > 1 && !whole(i)) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[e] = in(i, e) ? f[e] : 0.f;
    }
    return f;
  }
  __device__ __forceinline__ void store(void* base, long long r, int i, const Vec<VEC>& f) const {
    if (r >= rows || !any(i)) return;
    In* dst = reinterpret_cast<In*>(base) + r * cols + col(i, 0);
    if (whole(i)) {
      *reinterpret_cast<Raw<In, VEC>*>(dst) = from_floats(f.v, In());
    } else if (!FULL && VEC > 1 && NV == 1 && pieces) {
      const Raw<In, VEC> a = from_floats(f.v, In());
      const uint4 w = *reinterpret_cast<const uint4*>(&a);
      char* to = reinterpret_cast<char*>(dst);
      auto word = [&](int o) { return o < 8 ? (o < 4 ? w.x : w.y) : (o < 12 ? w.z : w.w); };   // of byte o
      const int at8 = (int)(pieces & 255) - 1, at4 = (int)(pieces >> 8 & 255) - 1, at2 = (int)(pieces >> 16 & 255) - 1;
      if (at8 >= 0) *reinterpret_cast<uint2*>(to + at8) = make_uint2(word(at8), word(at8 + 4));
      if (at4 >= 0) *reinterpret_cast<uint32_t*>(to + at4) = word(at4);
      if (VEC == 8 && at2 >= 0) *reinterpret_cast<uint16_t*>(to + at2) = (uint16_t)(word(at2) >> 8 * (at2 & 2));
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (in(i, e)) dst[e] = from_f32<In>(f[e]);
    }
  }
  __device__ __forceinline__ Vec<VEC> vector(const float* w, int i) const {
    Vec<VEC> f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[e] = in(i, e) ? w[col(i, e)] : 0.f;
    return f;
  }
};

// The next rows' vectors of N tensors, a thread's own.  Where a row is one or two vectors to a thread, copied asynchronously to shared memory ahead
// of the kRows rows that are worked on together (one's arithmetic under the other's sums); else the next row's in registers.  Copies of less than 16
// bytes (the tensor's end, no row) fill up with zeros.
template <typename In, int VEC, int NV, int THREADS, bool FULL, int N>
struct Ahead {
  static constexpr bool kAsync = VEC > 1 && NV <= 2 && THREADS <= 512, SUB = THREADS == kSubThreads;
  static constexpr int kRows = kAsync && NV == 1 ? 2 : 1, kStages = kAsync ? 3 * kRows : 1;   // rows in shared memory
  Raw<In, VEC> raw[N][NV];
  const void* base[N];
  int st = 0;
  __device__ __forceinline__ uint4* slot(int stage, int n, int i) const {
    extern __shared__ __align__(16) uint4 ahead_rows[];
    return ahead_rows + ((stage * N + n) * NV + i) * (int)blockDim.x + threadIdx.x;
  }
  __device__ __forceinline__ void fetch(const Rows<In, VEC, NV, SUB, FULL>& at, long long row, int stage) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if constexpr (kAsync) {
        if (base[n]) {
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            const bool there = row < at.rows && at.any(i);
            const long long from = there ? row * at.cols + at.col(i, 0) : 0, left = (at.total - from) * (long long)sizeof(In);
            const int bytes = there ? (!FULL && left < 16 ? (int)left : 16) : 0;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(slot(stage, n, i))),
                         "l"(reinterpret_cast<const In*>(base[n]) + from), "r"(bytes) : "memory");
          }
        }
      } else if (base[n]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) raw[n][i] = at.load(base[n], row, i);
      }
    }
    if constexpr (kAsync) asm volatile("cp.async.commit_group;" ::: "memory");
  }
  __device__ __forceinline__ void start(const Rows<In, VEC, NV, SUB, FULL>& at) {
#pragma unroll
    for (int k = 0; k < (kAsync ? kStages - kRows : 1); ++k) fetch(at, at.row + k * at.step, k);
  }
  // the vectors of `row` and the next one or none to use(p, n, i, raw); copies for later ones
  template <typename F> __device__ __forceinline__ void next(const Rows<In, VEC, NV, SUB, FULL>& at, long long row, F use) {
    if constexpr (kAsync) {
#pragma unroll
      for (int p = 0; p < kRows; ++p) {
        int to = st + kStages - kRows + p;
        fetch(at, row + (kStages - kRows + p) * at.step, to >= kStages ? to - kStages : to);
      }
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - kRows) : "memory");
#pragma unroll
      for (int p = 0; p < kRows; ++p)
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int i = 0; i < NV; ++i)
            if (base[n]) use(p, n, i, *reinterpret_cast<const Raw<In, VEC>*>(slot(st + p, n, i)));
      st = st + kRows == kStages ? 0 : st + kRows;
    } else {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (base[n]) use(0, n, i, raw[n][i]);
      fetch(at, row + at.step, 0);
    }
  }
};
constexpr size_t ahead_bytes(int vec, int nv, int threads, int tensors) {
  return vec > 1 && nv <= 2 && threads <= 512 ? (size_t)6 * tensors * threads * 16 : 0;   // (nv == 1: six rows, nv == 2: three)
}

// Sums of N values over the threads that share a row; every thread gets them.  `slot`: this call's shared memory, two used in turn
// so that one barrier is enough.
template <int N, bool SUB>
__device__ __forceinline__ void row_sum(float (&v)[N], int group, float (*slot)[N]) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    if (SUB && o >= group) continue;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  }
  if constexpr (!SUB) {
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) slot[threadIdx.x >> 5][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = lane < warps ? slot[lane][i] : 0.f;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      v[i] = s;
    }
  }
}

// s = 1 / (1 + e^-z) and 1 - s, both from e^-|z| <= 1, so that neither is a difference of near numbers.
__device__ __forceinline__ float sigmoid_of(float z, float* rest = nullptr) {
  const float e = ptx::ex2(-1.4426950408889634f * fabsf(z));
  float big;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(big) : "f"(1.f + e));
  const float small = e * big;
  if (rest) *rest = z < 0.f ? big : small;
  return z < 0.f ? small : big;
}

// A CTA's sums over its rows, from the threads' registers to part[CTA][which][cols]: short rows are added up group by group in shared memory.
template <typename In, int VEC, int NV, bool SUB, bool FULL>
__device__ __forceinline__ void put_sums(const Rows<In, VEC, NV, SUB, FULL>& at, const Vec<VEC> (&acc)[NV], float* part, float* sum, int group) {
  if constexpr (!SUB) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (at.in(i, e)) part[at.col(i, e)] = acc[i][e];
  } else {
    const int mine = threadIdx.x / group, groups = kSubThreads / group;
    __syncthreads();
    for (int c = threadIdx.x; c < at.cols; c += kSubThreads) sum[c] = 0.f;
    for (int g = 0; g < groups; ++g) {
      __syncthreads();
      if (g == mine) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (at.in(0, e)) sum[at.col(0, e)] += acc[0][e];
      }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < at.cols; c += kSubThreads) part[c] = sum[c];
  }
}

// ---------------------------------------------------------------- kernels (THREADS: kSubThreads for the short rows, else the most a CTA has)

template <typename In, int VEC, int NV, int THREADS, bool FULL>
__global__ void __launch_bounds__(THREADS == 257 ? 256 : THREADS) gated_norm_kernel(NormParams p) {
  constexpr bool SUB = THREADS == kSubThreads;
  __shared__ float red[2][32][1];
  const Rows<In, VEC, NV, SUB, FULL> at(p);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  Vec<VEC> w[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) w[i] = at.vector(p.w, i);
  int turn = 0;
  for (long long row = at.row; at.on(row); row += at.step) {
    Raw<In, VEC> rx[NV], rz[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) rx[i] = at.load(p.x, row, i);
    if (p.z) {
#pragma unroll
      for (int i = 0; i < NV; ++i) rz[i] = at.load(p.z, row, i);
    }
    float s[1] = {0.f};
    Vec<VEC> x[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      x[i] = at.unpack(rx[i], i);
      s[0] = dot(x[i], x[i], s[0]);
    }
    row_sum<1, SUB>(s, p.group, red[turn]);
    turn ^= 1;
    const float rs = rsqrtf(s[0] / at.cols + p.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      Vec<VEC> y = mul(mul(x[i], rs), w[i]);
      if (p.z) {
        Vec<VEC> z = at.unpack(rz[i], i);
#pragma unroll
        for (int e = 0; e < VEC; ++e) z[e] = p.sigmoid ? sigmoid_of(z[e]) : z[e] * sigmoid_of(z[e]);
        y = mul(y, z);
      }
      at.store(p.y, row, i, y);
    }
  }
}

template <typename In, int VEC, int NV, int THREADS, bool FULL>
__global__ void __launch_bounds__(THREADS == 257 ? 256 : THREADS, THREADS <= 257 ? 2 : 1) gated_norm_back_kernel(NormParams p) {
  constexpr bool SUB = THREADS == kSubThreads;
  __shared__ float red[2][32][2 * Ahead<In, VEC, NV, THREADS, FULL, 3>::kRows];
  __shared__ float sum[SUB ? 32 * VEC : 1];
  const Rows<In, VEC, NV, SUB, FULL> at(p);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  Vec<VEC> w[NV], dw[NV];
  Ahead<In, VEC, NV, THREADS, FULL, 3> rows;
  rows.base[0] = p.x; rows.base[1] = p.dy; rows.base[2] = p.z;
  rows.start(at);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    w[i] = at.vector(p.w, i);
    dw[i] = all_of<VEC>(0.f);
  }
  int turn = 0;
  constexpr int P = decltype(rows)::kRows;
  for (long long row = at.row; at.on(row); row += P * at.step) {
    Vec<VEC> x[P][NV], d[P][NV], a[P][NV], slope[P][NV];   // a = act(z)
    rows.next(at, row, [&](int q, int n, int i, const Raw<In, VEC>& v) { (n == 0 ? x[q][i] : n == 1 ? d[q][i] : a[q][i]) = at.unpack(v, i); });
    float s[2 * P];
#pragma unroll
    for (int q = 0; q < P; ++q) {
      s[2 * q] = s[2 * q + 1] = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (p.z) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            float rest;
            const float z = a[q][i][e], g = sigmoid_of(z, &rest);
            a[q][i][e] = p.sigmoid ? g : z * g;
            slope[q][i][e] = p.sigmoid ? g * rest : fmaf(a[q][i][e], rest, g);   // (silu: g (1 + z rest))
          }
          slope[q][i] = mul(slope[q][i], mul(d[q][i], w[i]));   // dz = slope d w x rs
          d[q][i] = mul(d[q][i], a[q][i]);
        }
        s[2 * q] = dot(x[q][i], x[q][i], s[2 * q]);
        s[2 * q + 1] = dot(mul(d[q][i], w[i]), x[q][i], s[2 * q + 1]);
      }
    }
    row_sum<2 * P, SUB>(s, p.group, red[turn]);
    turn ^= 1;
#pragma unroll
    for (int q = 0; q < P; ++q) {
      const float rs = rsqrtf(s[2 * q] / at.cols + p.eps), m = -(rs * (s[2 * q + 1] / at.cols)) * rs;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const Vec<VEC> t = mul(d[q][i], rs), n = mul(x[q][i], rs);
        at.store(p.dx, row + q * at.step, i, fma(t, w[i], mul(n, m)));
        if (at.there(row + q * at.step, P)) dw[i] = fma(t, x[q][i], dw[i]);
        if (p.z) at.store(p.dz, row + q * at.step, i, mul(slope[q][i], n));
      }
    }
  }
  put_sums(at, dw, p.part + (size_t)blockIdx.x * p.cols, sum, p.group);
}

template <typename In, int VEC, int NV, int THREADS, bool FULL, bool POST>
__global__ void __launch_bounds__(THREADS == 257 ? 256 : THREADS) add_norm_kernel(NormParams p) {
  constexpr bool SUB = THREADS == kSubThreads;
  __shared__ float red[2][32][1];
  const Rows<In, VEC, NV, SUB, FULL> at(p);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  Vec<VEC> w[NV], wp[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    w[i] = at.vector(p.w, i);
    if (POST) wp[i] = at.vector(p.w_post, i);
  }
  int turn = 0;
  for (long long row = at.row; at.on(row); row += at.step) {
    Raw<In, VEC> rx[NV], rr[NV];
    Vec<VEC> x[NV], r[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      rx[i] = at.load(p.x, row, i);
      rr[i] = at.load(p.r, row, i);
    }
    float s[1] = {0.f}, fs = p.scale;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      x[i] = at.unpack(rx[i], i);
      if (POST) {
        s[0] = dot(x[i], x[i], s[0]);
        x[i] = mul(x[i], wp[i]);
      }
    }
    if (POST) {
      row_sum<1, SUB>(s, p.group, red[turn]);
      turn ^= 1;
      fs = p.scale * rsqrtf(s[0] / at.cols + p.eps);
      s[0] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      r[i] = fma(x[i], fs, at.unpack(rr[i], i));
      s[0] = dot(r[i], r[i], s[0]);
      at.store(p.r_out, row, i, r[i]);
    }
    row_sum<1, SUB>(s, p.group, red[turn]);
    turn ^= 1;
    const float rs = rsqrtf(s[0] / at.cols + p.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) at.store(p.y, row, i, mul(mul(r[i], rs), w[i]));
  }
}

template <typename In, int VEC, int NV, int THREADS, bool FULL, bool POST>
__global__ void __launch_bounds__(THREADS == 257 ? 256 : THREADS, THREADS <= 257 ? 2 : 1) add_norm_back_kernel(NormParams p) {
  constexpr bool SUB = THREADS == kSubThreads;
  constexpr int kR = Ahead<In, VEC, NV, THREADS, FULL, 3>::kRows;
  __shared__ float red[2][32][3 * kR];
  __shared__ float red1[2][32][kR];
  __shared__ float sum[SUB ? 32 * VEC : 1];
  const Rows<In, VEC, NV, SUB, FULL> at(p);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  Vec<VEC> w[NV], wp[NV], dw[NV], dwp[NV];
  Ahead<In, VEC, NV, THREADS, FULL, POST ? 4 : 3> rows;
  rows.base[0] = p.r; rows.base[1] = p.dy; rows.base[2] = p.dr_out;
  if constexpr (POST) rows.base[3] = p.x;
  rows.start(at);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    w[i] = at.vector(p.w, i);
    if (POST) wp[i] = at.vector(p.w_post, i);
    dw[i] = dwp[i] = all_of<VEC>(0.f);
  }
  int turn = 0;
  constexpr int P = decltype(rows)::kRows;
  for (long long row = at.row; at.on(row); row += P * at.step) {
    Vec<VEC> r[P][NV], d[P][NV], x[P][NV], g[P][NV];
#pragma unroll
    for (int q = 0; q < P; ++q)
#pragma unroll
      for (int i = 0; i < NV; ++i) g[q][i] = all_of<VEC>(0.f);
    rows.next(at, row, [&](int q, int n, int i, const Raw<In, VEC>& v) {
      (n == 0 ? r[q][i] : n == 1 ? d[q][i] : n == 2 ? g[q][i] : x[q][i]) = at.unpack(v, i);
    });
    float s[3 * P], u[P];
#pragma unroll
    for (int q = 0; q < P; ++q) {
      s[3 * q] = s[3 * q + 1] = s[3 * q + 2] = u[q] = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        s[3 * q] = dot(r[q][i], r[q][i], s[3 * q]);
        s[3 * q + 1] = dot(mul(d[q][i], w[i]), r[q][i], s[3 * q + 1]);
        if (POST) s[3 * q + 2] = dot(x[q][i], x[q][i], s[3 * q + 2]);
      }
    }
    row_sum<3 * P, SUB>(s, p.group, red[turn]);
#pragma unroll
    for (int q = 0; q < P; ++q) {
      const float rs = rsqrtf(s[3 * q] / at.cols + p.eps), m = -(rs * (s[3 * q + 1] / at.cols)) * rs;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const Vec<VEC> t = mul(d[q][i], rs);
        if (at.there(row + q * at.step, P)) dw[i] = fma(t, r[q][i], dw[i]);
        r[q][i] = fma(t, w[i], fma(mul(r[q][i], rs), m, g[q][i]));     // dr
        if (POST) u[q] = dot(mul(r[q][i], wp[i]), x[q][i], u[q]);
        at.store(p.dr, row + q * at.step, i, r[q][i]);
        r[q][i] = mul(r[q][i], p.scale);                               // df
        if (!POST) at.store(p.dx, row + q * at.step, i, r[q][i]);
      }
    }
    if (POST) {
      row_sum<P, SUB>(u, p.group, red1[turn]);
#pragma unroll
      for (int q = 0; q < P; ++q) {
        const float rx = rsqrtf(s[3 * q + 2] / at.cols + p.eps), mx = -(rx * (p.scale * u[q] / at.cols)) * rx;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const Vec<VEC> t = mul(r[q][i], rx);
          if (at.there(row + q * at.step, P)) dwp[i] = fma(t, x[q][i], dwp[i]);
          at.store(p.dx, row + q * at.step, i, fma(t, wp[i], mul(mul(x[q][i], rx), mx)));
        }
      }
    }
    turn ^= 1;
  }
  float* part = p.part + (size_t)blockIdx.x * (POST ? 2 : 1) * p.cols;
  put_sums(at, dw, part, sum, p.group);
  if (POST) put_sums(at, dwp, part + p.cols, sum, p.group);
}

// Sums of the CTAs' sums: a warp's lanes have 32 neighbouring columns, the 32 warps every 32nd CTA.  blockIdx.y: which vector.
__global__ void __launch_bounds__(kReduceThreads) norm_reduce_kernel(const float* part, int ctas, int cols, int both, float* dw, float* dw_post) {
  __shared__ float s[kReduceThreads / 32][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  float a[4] = {0.f, 0.f, 0.f, 0.f};
  if (c < cols) {
    const float* src = part + (size_t)blockIdx.y * cols + c;
    const size_t stride = (size_t)both * cols;
    int i = warp;
    constexpr int kWarps = kReduceThreads / 32;
    for (; i + 3 * kWarps < ctas; i += 4 * kWarps)
#pragma unroll
      for (int k = 0; k < 4; ++k) a[k] += src[(i + k * kWarps) * stride];
    for (; i < ctas; i += kWarps) a[0] += src[i * stride];
  }
  s[warp][lane] = (a[0] + a[1]) + (a[2] + a[3]);
  __syncthreads();
  if (warp == 0 && c < cols) {
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < kReduceThreads / 32; ++k) t += s[k][lane];
    (blockIdx.y ? dw_post : dw)[c] = t;
  }
}

// ---------------------------------------------------------------- host

struct Shape { int vec, nv, group, threads, groups; bool sub, full; };   // group: lanes of a row (sub), groups: rows of a CTA at once

// `fast`: every tensor 16-byte aligned
Shape shape_of(int cols, bool bf16, bool fast, bool back) {
  Shape s;
  s.vec = fast ? (bf16 ? 8 : 4) : 1;
  s.full = cols % s.vec == 0;
  const int vectors = !s.full ? (cols + s.vec - 1) / s.vec + 1 : cols / s.vec;   // of the worst start
  s.sub = vectors <= 32;
  s.group = 1;
  s.nv = 1;
  if (s.sub) {
    while (s.group < vectors) s.group *= 2;
    s.threads = kSubThreads;
    s.groups = kSubThreads / s.group;
  } else {
    // backward, where a thread has more to keep: up to 256 threads with a vector each, then up to 1024 with two and more
    while (s.nv * (back && s.nv == 1 ? 256 : 1024) < vectors) s.nv *= 2;
    s.threads = ((vectors + s.nv - 1) / s.nv + 31) / 32 * 32;
    s.groups = 1;
  }
  return s;
}

// CTAs: one per `groups` rows up to `most` threads on an SM; rows of a group a multiple of 8 apart where it has several.
int ctas_of(const Shape& s, long long rows, int most_threads) {
  const long long need = (rows + s.groups - 1) / s.groups;
  const long long most = (long long)sm_count() * (most_threads / s.threads > 0 ? most_threads / s.threads : 1);
  long long n = need < most ? need : most;
  if (n < need) n = (n + 7) / 8 * 8;
  return (int)(n > 0 ? n : 1);
}

// Threads of an SM: the backward kernels' CTAs keep sums, so there are no more of them than run at a time (see pick), this many at most.
constexpr int kBackThreads = 1024, kForwardThreads = 16384;

int back_ctas(int cols, bool bf16, long long rows) {     // (of the workspace: either way of reading)
  const int a = ctas_of(shape_of(cols, bf16, true, true), rows, kBackThreads), b = ctas_of(shape_of(cols, bf16, false, true), rows, kBackThreads);
  return a > b ? a : b;
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

enum Kind { kGated, kGatedBack, kAdd, kAddBack };

template <typename In, int VEC, int NV, int THREADS, bool FULL, bool BACK>
cudaError_t pick(Kind kind, const NormParams& p, int& ctas, int threads, cudaStream_t stream) {
  void (*k)(NormParams) = nullptr;
  size_t smem = 0;
  if constexpr (BACK) {
    if (kind == kGatedBack) k = gated_norm_back_kernel<In, VEC, NV, THREADS, FULL>;
    else k = p.w_post ? add_norm_back_kernel<In, VEC, NV, THREADS, FULL, true> : add_norm_back_kernel<In, VEC, NV, THREADS, FULL, false>;
    const int tensors = kind == kAddBack && p.w_post ? 4 : 3;
    smem = ahead_bytes(VEC, NV, threads, tensors);
    // (the kernel's most, whatever this call takes: another thread's call of another width may be between this and its launch)
    const size_t most_smem = ahead_bytes(VEC, NV, THREADS == 257 ? 256 : THREADS, tensors);
    cudaError_t e = smem > 0 ? cudaFuncSetAttribute(reinterpret_cast<const void*>(k), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most_smem) : cudaSuccess;
    int resident = 1;
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, k, threads, smem);
    if (e != cudaSuccess) return e;
    const int most = (sm_count() * (resident > 0 ? resident : 1) + 7) / 8 * 8;   // (rows of a CTA stay a multiple of 8 apart)
    if (ctas > most) ctas = most;
  } else {
    if (kind == kGated) k = gated_norm_kernel<In, VEC, NV, THREADS, FULL>;
    else k = p.w_post ? add_norm_kernel<In, VEC, NV, THREADS, FULL, true> : add_norm_kernel<In, VEC, NV, THREADS, FULL, false>;
  }
  return start(k, dim3((unsigned)ctas), threads, smem, stream, p);
}

// (THREADS of longer rows: 257 stands for up to 256, told apart from the short rows' CTAs)
template <typename In, int VEC, bool FULL, bool BACK>
cudaError_t by_length(Kind kind, const NormParams& p, const Shape& s, int& ctas, cudaStream_t stream) {
  if (s.sub) return pick<In, VEC, 1, kSubThreads, FULL, BACK>(kind, p, ctas, s.threads, stream);
  if (s.nv == 1) {
    if (s.threads <= 256) return pick<In, VEC, 1, 257, FULL, BACK>(kind, p, ctas, s.threads, stream);
    if constexpr (!BACK)
      return s.threads <= 512 ? pick<In, VEC, 1, 512, FULL, BACK>(kind, p, ctas, s.threads, stream) : pick<In, VEC, 1, 1024, FULL, BACK>(kind, p, ctas, s.threads, stream);
  }
  if (s.nv == 2) {
    if constexpr (BACK) {
      if (s.threads <= 256) return pick<In, VEC, 2, 257, FULL, BACK>(kind, p, ctas, s.threads, stream);
      if (s.threads <= 512) return pick<In, VEC, 2, 512, FULL, BACK>(kind, p, ctas, s.threads, stream);
    }
    return pick<In, VEC, 2, 1024, FULL, BACK>(kind, p, ctas, s.threads, stream);
  }
  constexpr int kMostVectors = kMaxCols / VEC + (FULL ? 0 : 1);
  if constexpr (kMostVectors > 2 * 1024) {
    if (s.nv == 4) return pick<In, VEC, 4, 1024, FULL, BACK>(kind, p, ctas, s.threads, stream);
  }
  if constexpr (kMostVectors > 4 * 1024) {
    if (s.nv == 8) return pick<In, VEC, 8, 1024, FULL, BACK>(kind, p, ctas, s.threads, stream);
  }
  if constexpr (kMostVectors > 8 * 1024) return pick<In, VEC, 16, 1024, FULL, BACK>(kind, p, ctas, s.threads, stream);
  return cudaErrorInvalidValue;
}

// (element by element all rows are whole)
template <typename In, int VEC>
cudaError_t by_start(Kind kind, const NormParams& p, const Shape& s, int& ctas, cudaStream_t stream) {
  if constexpr (VEC > 1) {
    if (!s.full) return kind == kGated || kind == kAdd ? by_length<In, VEC, false, false>(kind, p, s, ctas, stream) : by_length<In, VEC, false, true>(kind, p, s, ctas, stream);
  }
  return kind == kGated || kind == kAdd ? by_length<In, VEC, true, false>(kind, p, s, ctas, stream) : by_length<In, VEC, true, true>(kind, p, s, ctas, stream);
}

cudaError_t run(Kind kind, NormParams& p, int dtype, uintptr_t addresses, float* dw, float* dw_post, cudaStream_t stream) {
  const bool bf16 = dtype == HA_LA_BF16, fast = !(addresses & 15), back = kind == kGatedBack || kind == kAddBack;
  const Shape s = shape_of(p.cols, bf16, fast, back);
  p.group = s.group;
  int ctas = ctas_of(s, p.rows, back ? kBackThreads : kForwardThreads);
  cudaError_t e = bf16 ? (fast ? by_start<__nv_bfloat16, 8>(kind, p, s, ctas, stream) : by_start<__nv_bfloat16, 1>(kind, p, s, ctas, stream))
                       : (fast ? by_start<float, 4>(kind, p, s, ctas, stream) : by_start<float, 1>(kind, p, s, ctas, stream));
  if (e != cudaSuccess || !back) return e;
  const int both = dw_post ? 2 : 1;
  return start(norm_reduce_kernel, dim3((unsigned)((p.cols + 31) / 32), (unsigned)both), kReduceThreads, 0, stream,
               (const float*)p.part, ctas, p.cols, both, dw, dw_post);
}

int check(int dtype, long long rows, int cols, float eps) {
  if (dtype != HA_LA_BF16 && dtype != HA_LA_FP32) return HA_LA_ERR_INVALID_ARG;
  if (rows < 0 || cols < 1 || !(eps >= 0.f)) return HA_LA_ERR_INVALID_ARG;
  if (cols > kMaxCols || rows > (1LL << 46) / cols) return HA_LA_ERR_UNSUPPORTED;
  return HA_LA_OK;
}

// the tensors of `dtype` have to start on one of its elements, fp32 vectors too
bool misaligned(int dtype, uintptr_t tensors, uintptr_t vectors) { return (tensors & (dtype == HA_LA_BF16 ? 1 : 3)) || (vectors & 3); }

template <typename... P> uintptr_t any_of(P... p) { return (... | (uintptr_t)p); }

int bytes(int dtype, long long rows, int cols, float eps, int both, size_t* out) {
  if (!out) return HA_LA_ERR_INVALID_ARG;
  const int rc = check(dtype, rows, cols, eps);
  if (rc != HA_LA_OK) return rc;
  *out = align_up((size_t)back_ctas(cols, dtype == HA_LA_BF16, rows) * both * cols * sizeof(float), 256);
  return HA_LA_OK;
}

// Gradients of weights without a row
int no_rows(float* dw, float* dw_post, int cols, cudaStream_t stream) {
  if (cudaMemsetAsync(dw, 0, sizeof(float) * cols, stream) != cudaSuccess) return HA_LA_ERR_CUDA;
  if (dw_post && cudaMemsetAsync(dw_post, 0, sizeof(float) * cols, stream) != cudaSuccess) return HA_LA_ERR_CUDA;
  return HA_LA_OK;
}

bool workspace_ok(const void* ws, size_t have, size_t need) { return ws && !((uintptr_t)ws & 255) && have >= need; }

}  // namespace

}  // namespace ha_la

using namespace ha_la;

extern "C" {

int ha_la_gated_norm_workspace_bytes(const ha_la_gated_norm_args* a, size_t* out_bytes) {
  if (!a) return HA_LA_ERR_INVALID_ARG;
  return bytes(a->dtype, a->rows, a->cols, a->eps, 1, out_bytes);
}

int ha_la_gated_norm(const ha_la_gated_norm_args* a, void* cuda_stream) {
  if (!a) return HA_LA_ERR_INVALID_ARG;
  const int rc = check(a->dtype, a->rows, a->cols, a->eps);
  if (rc != HA_LA_OK) return rc;
  if (a->z && a->activation != HA_LA_ACT_SILU && a->activation != HA_LA_ACT_SIGMOID) return HA_LA_ERR_INVALID_ARG;
  if (a->rows == 0) return HA_LA_OK;
  if (!a->x || !a->w || !a->y) return HA_LA_ERR_INVALID_ARG;
  const uintptr_t at = any_of(a->x, a->z, a->y);
  if (misaligned(a->dtype, at, (uintptr_t)a->w)) return HA_LA_ERR_INVALID_ARG;
  NormParams p = {};
  p.x = a->x; p.z = a->z; p.w = a->w; p.y = a->y;
  p.rows = a->rows; p.cols = a->cols; p.eps = a->eps;
  p.sigmoid = a->activation == HA_LA_ACT_SIGMOID;
  return run(kGated, p, a->dtype, at, nullptr, nullptr, reinterpret_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? HA_LA_OK : HA_LA_ERR_CUDA;
}

int ha_la_gated_norm_backward(const ha_la_gated_norm_args* a, void* cuda_stream) {
  if (!a) return HA_LA_ERR_INVALID_ARG;
  size_t need = 0;
  const int rc = bytes(a->dtype, a->rows, a->cols, a->eps, 1, &need);
  if (rc != HA_LA_OK) return rc;
  if (a->z && a->activation != HA_LA_ACT_SILU && a->activation != HA_LA_ACT_SIGMOID) return HA_LA_ERR_INVALID_ARG;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (!a->dw || ((uintptr_t)a->dw & 3)) return HA_LA_ERR_INVALID_ARG;
  if (a->rows == 0) return no_rows(a->dw, nullptr, a->cols, stream);
  if (!a->x || !a->w || !a->dy || !a->dx || (a->z && !a->dz)) return HA_LA_ERR_INVALID_ARG;
  const uintptr_t at = any_of(a->x, a->z, a->dy, a->dx, a->z ? a->dz : nullptr);
  if (misaligned(a->dtype, at, (uintptr_t)a->w)) return HA_LA_ERR_INVALID_ARG;
  if (!workspace_ok(a->workspace, a->workspace_bytes, need)) return HA_LA_ERR_WORKSPACE;
  NormParams p = {};
  p.x = a->x; p.z = a->z; p.w = a->w; p.dy = a->dy; p.dx = a->dx; p.dz = a->dz;
  p.part = reinterpret_cast<float*>(a->workspace);
  p.rows = a->rows; p.cols = a->cols; p.eps = a->eps;
  p.sigmoid = a->activation == HA_LA_ACT_SIGMOID;
  return run(kGatedBack, p, a->dtype, at, a->dw, nullptr, stream) == cudaSuccess ? HA_LA_OK : HA_LA_ERR_CUDA;
}

int ha_la_add_norm_workspace_bytes(const ha_la_add_norm_args* a, size_t* out_bytes) {
  if (!a) return HA_LA_ERR_INVALID_ARG;
  return bytes(a->dtype, a->rows, a->cols, a->eps, a->w_post ? 2 : 1, out_bytes);
}

int ha_la_add_norm(const ha_la_add_norm_args* a, void* cuda_stream) {
  if (!a) return HA_LA_ERR_INVALID_ARG;
  const int rc = check(a->dtype, a->rows, a->cols, a->eps);
  if (rc != HA_LA_OK) return rc;
  if (!(a->scale == a->scale)) return HA_LA_ERR_INVALID_ARG;
  if (a->rows == 0) return HA_LA_OK;
  if (!a->x || !a->r || !a->w || !a->y || !a->r_out) return HA_LA_ERR_INVALID_ARG;
  const uintptr_t at = any_of(a->x, a->r, a->y, a->r_out);
  if (misaligned(a->dtype, at, any_of(a->w, a->w_post))) return HA_LA_ERR_INVALID_ARG;
  NormParams p = {};
  p.x = a->x; p.r = a->r; p.w = a->w; p.w_post = a->w_post; p.y = a->y; p.r_out = a->r_out;
  p.rows = a->rows; p.cols = a->cols; p.eps = a->eps; p.scale = a->scale;
  return run(kAdd, p, a->dtype, at, nullptr, nullptr, reinterpret_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? HA_LA_OK : HA_LA_ERR_CUDA;
}

int ha_la_add_norm_backward(const ha_la_add_norm_args* a, void* cuda_stream) {
  if (!a) return HA_LA_ERR_INVALID_ARG;
  size_t need = 0;
  const int rc = bytes(a->dtype, a->rows, a->cols, a->eps, a->w_post ? 2 : 1, &need);
  if (rc != HA_LA_OK) return rc;
  if (!(a->scale == a->scale)) return HA_LA_ERR_INVALID_ARG;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (!a->dw || (a->w_post && !a->dw_post) || (any_of(a->dw, a->dw_post) & 3)) return HA_LA_ERR_INVALID_ARG;
  float* dw_post = a->w_post ? a->dw_post : nullptr;
  if (a->rows == 0) return no_rows(a->dw, dw_post, a->cols, stream);
  if (!a->r_out || !a->w || !a->dy || !a->dx || !a->dr || (a->w_post && !a->x)) return HA_LA_ERR_INVALID_ARG;
  const uintptr_t at = any_of(a->w_post ? a->x : nullptr, a->r_out, a->dy, a->dr_out, a->dx, a->dr);
  if (misaligned(a->dtype, at, any_of(a->w, a->w_post))) return HA_LA_ERR_INVALID_ARG;
  if (!workspace_ok(a->workspace, a->workspace_bytes, need)) return HA_LA_ERR_WORKSPACE;
  NormParams p = {};
  p.x = a->x; p.r = a->r_out; p.w = a->w; p.w_post = a->w_post; p.dy = a->dy; p.dr_out = a->dr_out; p.dx = a->dx; p.dr = a->dr;
  p.part = reinterpret_cast<float*>(a->workspace);
  p.rows = a->rows; p.cols = a->cols; p.eps = a->eps; p.scale = a->scale;
  return run(kAddBack, p, a->dtype, at, a->dw, dw_post, stream) == cudaSuccess ? HA_LA_OK : HA_LA_ERR_CUDA;
}

}  // extern "C"

"""The chunk table's kernel (csrc/plan.cu), compiled for the host with a thread for each of its threads: whatever the offsets of a packed batch
are, the table that the other kernels read and write by stays within the tokens and the slots, and offsets that do not fit are reported."""
import ctypes
import os
import random
import re
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_32114_b200", "csrc")

# One host thread per device thread; a shared variable is a static one.
SHIM = r"""
#include <algorithm>
#include <barrier>
#include <cstdint>
#include <thread>
#include <vector>
using std::min;
enum { HA_LA_ERR_DEVICE_CHECK = 6 };
struct Dim { int x; };
static thread_local Dim threadIdx;
static Dim blockDim;
constexpr int kMost = 512;
static std::barrier<> block(kMost);
static std::vector<std::barrier<>*> warps;
static long long given[kMost];
static int any[2];
static void __syncthreads() { block.arrive_and_wait(); }
static int __syncthreads_or(int x) {
  if (threadIdx.x == 0) any[0] = 0;
  block.arrive_and_wait();
  if (x) __atomic_store_n(&any[0], 1, __ATOMIC_RELAXED);
  block.arrive_and_wait();
  const int r = any[0];
  block.arrive_and_wait();
  return r;
}
template <typename T> static T __shfl_up_sync(unsigned, T x, int o) {
  given[threadIdx.x] = x;
  warps[threadIdx.x / 32]->arrive_and_wait();
  const int lane = threadIdx.x & 31;
  const T r = lane >= o ? (T)given[threadIdx.x - o] : x;
  warps[threadIdx.x / 32]->arrive_and_wait();
  return r;
}
template <typename T, typename U> static T atomicAdd(T* p, U x) { return __atomic_fetch_add(p, (T)x, __ATOMIC_RELAXED); }
static void report_status(int32_t* status, int code) { int none = 0; __atomic_compare_exchange_n(status, &none, code, false, __ATOMIC_RELAXED, __ATOMIC_RELAXED); }
"""
CALL = r"""
extern "C" void plan(int N, int T_total, int T_row, int max_len, int max_chunks, int step, const int32_t* cu, int32_t* tok0, int32_t* len, int32_t* chunk0,
                     int32_t* order, int32_t* chunk_seq, int32_t* chunk_tok0, int32_t* chunk_len, int32_t* hdr, int32_t* status) {
  static_assert(kThreads == kMost, "threads");
  blockDim.x = kThreads;
  if (warps.empty()) for (int i = 0; i < kThreads / 32; ++i) warps.push_back(new std::barrier<>(32));
  std::vector<std::thread> ts;
  for (int t = 0; t < kThreads; ++t)
    ts.emplace_back([=] {
      threadIdx.x = t;
      plan_kernel(PlanParams{N, T_total, T_row, max_len, max_chunks, step}, cu, PlanView{hdr, tok0, len, chunk0, order, chunk_seq, chunk_tok0, chunk_len}, status);
    });
  for (auto& t : ts) t.join();
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    view = re.search(r"struct PlanView \{.*?\n\};", open(os.path.join(CSRC, "common.cuh")).read(), re.S).group(0)
    src = open(os.path.join(CSRC, "plan.cu")).read()
    body = src[src.index("struct PlanParams"):src.index("}  // namespace\n")]
    body = re.sub(r"asm volatile\(.*", "", body)
    body = re.sub(r"__global__ void __launch_bounds__\(\w+\)", "static void", body).replace("__shared__", "static").replace("__restrict__", "")
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SHIM + view + body + CALL)
    r = subprocess.run(["g++", "-std=c++20", "-O1", "-shared", "-fPIC", "-pthread", "-o", str(d / "plan.so"), str(d / "plan.cpp")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    lib = ctypes.CDLL(str(d / "plan.so"))

    def run(cu, T, step, max_len=None, N=None, T_row=0):
        N = len(cu) - 1 if cu is not None else N
        # the bound on the slots that every caller takes (a packed batch: each sequence may end inside a chunk)
        most = (T + (step - 1) * N) // step if cu is not None else N * (-(-T_row // step))
        z = lambda n: np.full(max(n, 1), -77, np.int32)
        t = dict(tok0=z(N), len=z(N), chunk0=z(N + 1), order=z(N), chunk_seq=z(most), chunk_tok0=z(most), chunk_len=z(most), hdr=z(8), status=np.zeros(1, np.int32))
        arr = None if cu is None else np.asarray(cu, np.int32)
        p = lambda a: None if a is None else a.ctypes.data_as(ctypes.c_void_p)
        lib.plan(N, T, T_row, T if max_len is None else max_len, most, step, p(arr), *(p(a) for a in t.values()))
        return t, most

    return run


def fits(cu, T, max_len):
    return cu[0] == 0 and cu[-1] == T and all(a <= b and b - a <= max_len for a, b in zip(cu, cu[1:]))


def check(t, most, cu, T, step, max_len):
    """Everything that another kernel may take from the table is in bounds, and the parts agree."""
    N = len(cu) - 1
    tok0, length, chunk0 = (t[n].astype(np.int64) for n in ("tok0", "len", "chunk0"))
    assert (tok0[:N] >= 0).all() and (length[:N] >= 0).all() and (tok0[:N] + length[:N] <= T).all() and (length[:N] <= max_len).all()
    counts = -(-length[:N] // step)
    assert chunk0[0] == 0 and (np.diff(chunk0[:N + 1]) == counts).all() and chunk0[N] <= most
    assert sorted(t["order"][:N]) == list(range(N)) and t["hdr"][0] == chunk0[N] and t["hdr"][1] == N
    used = int(chunk0[N])
    seq = np.repeat(np.arange(N), counts)
    at = np.arange(used) - chunk0[seq]
    assert (t["chunk_seq"][:used] == seq).all() and (t["chunk_tok0"][:used] == tok0[seq] + at * step).all()
    assert (t["chunk_len"][:used] == np.minimum(step, length[seq] - at * step)).all()
    assert (t["chunk_len"][used:most] == 0).all()
    assert int(t["status"][0]) == (0 if fits(cu, T, max_len) else 6)
    if fits(cu, T, max_len):
        assert (tok0[:N] == np.asarray(cu)[:-1]).all() and (length[:N] == np.diff(cu)).all()


@pytest.mark.parametrize("step", [64, 128])
@pytest.mark.parametrize("N", [1, 2, 3, 24, 700, 1500])
def test_lengths_that_fit(plan, N, step):
    rng = random.Random(N)
    cu = [0]
    for _ in range(N):
        cu.append(cu[-1] + rng.choice([0, 1, step - 1, step, step + 1, rng.randint(0, 700)]))
    t, most = plan(cu, cu[-1], step)
    check(t, most, cu, cu[-1], step, cu[-1])
    longest_first = t["len"][t["order"][:N]]
    assert (np.diff(longest_first) <= 0).all()


def test_equal_rows(plan):
    t, most = plan(None, 5 * 300, 128, N=5, T_row=300)
    check(t, most, [300 * i for i in range(6)], 1500, 128, 300)


# One checked sequence goes from 0 to the end again and again: more chunks than slots, in the last case more than 31 bits count.
OVERLAPPING = {"three": ([0, 1000] * 3, 1000), "many": ([0, 5000] * 40, 5000), "pieces": ([0, 900, 100, 1000, 200, 1000], 1000), "long": ([0, 1 << 30] * 301, 1 << 30)}


@pytest.mark.parametrize("step", [64, 128])
@pytest.mark.parametrize("name", list(OVERLAPPING))
def test_sequences_that_overlap(plan, name, step):
    cu, T = OVERLAPPING[name]
    t, most = plan(cu, T, step)
    check(t, most, cu, T, step, T)


@pytest.mark.parametrize("seed", range(40))
def test_offsets_of_any_kind(plan, seed):
    rng = random.Random(seed)
    T, step = rng.choice([0, 1, 100, 1000, 5000]), rng.choice([64, 128])
    N = rng.choice([1, 2, 3, 7, 30, 1100])
    cu = [rng.choice([0, T, rng.randint(0, T), rng.randint(0, T), rng.randint(-50, T + 50), -2 ** 31, 2 ** 31 - 1]) for _ in range(N + 1)]
    if rng.random() < 0.7:
        cu[0], cu[-1] = 0, T
    max_len = rng.choice([T, T, max(1, T // 2)])
    t, most = plan(cu, T, step, max_len)
    check(t, most, cu, T, step, max_len)

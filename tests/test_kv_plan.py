"""Launches of the cached attention and the rows of its join, as the library plans them (CPU only).

kv_plan.h is compiled for the host as it stands. Checked over many sizes: every wave of the joining launch, the spare ones
of its last work-group included, touches only chunk results that lie inside the workspace, every row that may be split is
joined by exactly one wave, and every chunk of every work-group has a place.
"""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_09142_amd", "csrc")

HARNESS = r"""
#define __host__
#define __device__
#include "kv_plan.h"
using namespace elis;

static int floor_div(long long a, long long b) { return static_cast<int>(a / b); }

// Joins of one call. out: rows joined, chunk results of a row, results in the workspace. 0, or what is wrong.
extern "C" int joins(int n, int total_q, int max_q, int max_kv, int heads, int kv_heads, int d, int window, long long* out) {
    const KvAttnPlan most = plan_kv_attention(n, total_q, max_q, max_kv, heads, kv_heads, d, 0);  // sizes the workspace
    const KvAttnPlan p = plan_kv_attention(n, total_q, max_q, max_kv, heads, kv_heads, d, window >= max_kv ? 0 : window);
    const long long parts = most.small_parts + most.many_parts;
    if (p.small_parts != most.small_parts || p.many_parts != most.many_parts) return 1;
    const KvJoins j = kv_joins(p, n, total_q, heads, kv_heads);
    out[0] = j.all;
    out[1] = j.small;
    out[2] = parts;
    const int a_row = j.wide ? 4 : 1;  // waves that join a row
    const long long grid = j.wide ? j.all : (j.all + 3) / 4;
    long long small = 0, many = 0;
    for (long long wave = 0; wave < 4 * grid; wave += a_row) {
        const KvJoinRow x = kv_join_row(wave / a_row, j, p.small_rows, heads, kv_heads);
        if (!x.any) continue;
        const long long chunks = x.many ? p.many_chunks : p.small_chunks;
        const long long first = (x.many ? static_cast<long long>(p.small_parts) : 0) +
            static_cast<long long>(kv_part_row(x.many, x.req, x.h, x.tok, x.head, x.r, heads, kv_heads, p.small_rows)) * chunks;
        // the wave reads the results first .. first + chunks - 1 before it knows the lengths
        if (first < 0 || first + chunks > parts) return 2;
        if (!x.many && first + chunks > static_cast<long long>(p.small_parts)) return 3;
        if (x.many ? x.tok >= total_q || x.head >= heads : x.req >= n || x.h >= kv_heads || x.r >= p.small_rows) return 4;
        (x.many ? many : small) += 1;
    }
    if (small != j.small || many != j.all - j.small) return 5;
    // a chunk number of any work-group has a place among its row's results
    const int g = heads / kv_heads;
    for (int i = 0; i < 2; ++i) {
        const long long chunk = i ? p.many_chunk : p.small_chunk, chunks = i ? p.many_chunks : p.small_chunks;
        if (i ? !p.many : p.small_rows == 0) continue;
        const long long tokens = i ? floor_div(16LL * p.many_nb - 1, g) + 2 : max_q < 32 ? max_q : 32;
        long long keys = window > 0 && window < max_kv ? window + (tokens < max_q ? tokens : max_q) - 1 + kRecTokens - 1 : max_kv;
        if (keys > max_kv) keys = max_kv;
        if (chunk % kRecTokens || chunk * chunks < keys) return 6;
        if (chunks > 1 && static_cast<long long>(i ? p.many_parts : p.small_parts) == 0) return 7;
        if (!i && chunk > 4096) return 8;  // the pages that a work-group's lanes hold
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def joins(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    tmp = tmp_path_factory.mktemp("kv_plan")
    (tmp / "plan.cpp").write_text(HARNESS)
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I", CSRC, "-o", str(tmp / "plan.so"), str(tmp / "plan.cpp")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    fn = ctypes.CDLL(str(tmp / "plan.so")).joins

    def call(*sizes):
        out = (ctypes.c_longlong * 3)()
        return fn(*sizes, out), tuple(out)

    return call


@pytest.mark.parametrize("heads,kv_heads,d,n,kv", [(5, 1, 128, 1, 2000), (7, 1, 64, 1, 5000), (5, 5, 128, 1, 1100), (3, 1, 64, 3, 9000), (6, 2, 128, 3, 2100)])
def test_spare_waves_of_the_join(joins, heads, kv_heads, d, n, kv):
    """Single tokens whose rows are no multiple of four: the last work-group has waves without a row."""
    status, (rows, small, parts) = joins(n, n, 1, kv, heads, kv_heads, d, 0)
    assert status == 0 and rows == small == n * heads and parts > 0


@pytest.mark.parametrize("seed", range(8))
def test_joins_stay_inside_the_workspace(joins, seed):
    rng = np.random.default_rng(seed)
    split = 0
    for _ in range(3000):
        log = lambda lo, hi: int(round(np.exp(rng.uniform(np.log(lo), np.log(hi)))))  # noqa: E731
        kv_heads, n, max_q = log(1, 130), log(1, 300), log(1, 300)
        heads = kv_heads * log(1, 70)
        total = int(rng.integers(1, n * max_q + 1)) if rng.random() < 0.7 else n * max_q
        max_kv = log(1, 1 << 20)
        if total * heads > 1 << 19:
            continue
        sizes = (n, total, max_q, max_kv, heads, kv_heads, int(rng.choice([64, 128])), 0 if rng.random() < 0.5 else log(1, 1 << 20))
        status, (rows, _, parts) = joins(*sizes)
        assert status == 0, (status, sizes)
        split += rows > 0
    assert split > 100

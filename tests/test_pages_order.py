"""The page kernels on the CPU, threads and work-groups in several orders (pages.hip compiled for the host as it stands).

Between two barriers the hardware may run a work-group's waves in any order. tests/simt.h runs its threads one at a time, in
ascending, descending and shuffled orders; in every one of them the pages, block tables and slot maps have to be the oracle's.
"""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from oracle import batch as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_09142_amd", "csrc")
CLANG = "/opt/rocm/llvm/bin/clang++"

HARNESS = r"""
#include "simt.h"
#include "pages.hip"

static elis::PagePoolView view(int32_t* state, int32_t* free_pages, int32_t* held, int32_t* table, int32_t* scratch, const int32_t* size) {
    int shift = 0;
    while ((1 << shift) < size[1]) ++shift;
    return elis::PagePoolView{state, free_pages, held, table, scratch, (reinterpret_cast<uintptr_t>(scratch) & 15) == 0, size[0], size[1], shift, size[2], size[3]};
}
extern "C" void grow(unsigned order, int32_t* st, int32_t* fr, int32_t* held, int32_t* table, int32_t* scratch, const int32_t* size, const int32_t* slots,
                     const int32_t* lens, const int32_t* cu, int n, int total, int width, int32_t* blocks, int32_t* map) {
    simt::order_seed = order;
    elis::launch_pages_grow(view(st, fr, held, table, scratch, size), slots, lens, cu, n, total, width, blocks, map, nullptr);
}
// Threads in a row of the largest launch of a grow of n entries; 0 if there are too many rows.
extern "C" unsigned long long threads_of(const int32_t* size, int n, int total, int width) {
    static int32_t some[4];
    simt::dry = true;
    simt::most = 1;
    elis::launch_pages_grow(view(some, some, some, some, some, size), some, some, some, n, total, width, some, some, nullptr);
    simt::dry = false;
    return simt::most;
}
extern "C" void trim(unsigned order, int32_t* st, int32_t* fr, int32_t* held, int32_t* table, int32_t* scratch, const int32_t* size, const int32_t* slots,
                     const int32_t* lens, int n) {
    simt::order_seed = order;
    elis::launch_pages_trim(view(st, fr, held, table, scratch, size), slots, lens, n, nullptr);
}
"""


def compiled(tmp, name, text):
    if not os.path.exists(CLANG):
        pytest.skip("clang++ not available")
    (tmp / "hip").mkdir()
    for h in ("hip_runtime.h", "hip_ext.h"):
        (tmp / "hip" / h).write_text('#include "simt.h"\n')
    (tmp / f"{name}.cpp").write_text(text)
    r = subprocess.run([CLANG, "-std=c++17", "-O1", "-shared", "-fPIC", "-w", "-I", str(tmp), "-I", os.path.dirname(os.path.abspath(__file__)), "-I", CSRC,
                        "-I", os.path.join(ROOT, "include"), "-o", str(tmp / f"{name}.so"), str(tmp / f"{name}.cpp")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return ctypes.CDLL(str(tmp / f"{name}.so"))


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return compiled(tmp_path_factory.mktemp("pages"), "pages", HARNESS)


def i32(a):
    return np.ascontiguousarray(a, dtype=np.int32)


class Pool:
    def __init__(self, lib, order, n_pages, page, jobs, width):
        self.lib, self.order, self.size = lib, order, i32([n_pages, page, jobs, width])
        self.state, self.free = i32([0, n_pages]), i32(np.arange(n_pages)[::-1])
        self.held, self.table, self.scratch = i32(np.zeros(jobs)), i32(np.full((jobs, width), -7)), i32(np.full(4 * jobs + 4, 0x5A5A5A5A))

    def call(self, fn, *args):
        arrays = (self.state, self.free, self.held, self.table, self.scratch, self.size)
        fn(self.order, *(ctypes.c_void_p(a.ctypes.data) for a in arrays),
           *(ctypes.c_void_p(a.ctypes.data) if isinstance(a, np.ndarray) else a for a in args))


@pytest.mark.parametrize("order", [0, 1, 2, 3])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 127, 128, 129, 300])
def test_pages_in_any_order(lib, n, order):
    rng = np.random.default_rng(n)
    page, W = 16, 8
    n_pages = int(3.5 * n) + 2
    pool, ref = Pool(lib, order, n_pages, page, n + 3, W), O.Pages(n_pages, page, n + 3, W)
    lens = np.zeros(n + 3, np.int64)
    for step in range(3):
        slots = rng.permutation(n + 3)[:n]
        new = rng.integers(1, 60 if step == 0 else 3, n)
        want = np.minimum(lens[slots] + new, W * page)
        new = want - lens[slots]
        cu = i32(np.concatenate([[0], np.cumsum(new)]))
        blocks, smap = i32(np.full((n, W), -9)), i32(np.full(int(cu[-1]) + 1, -9))
        pool.call(lib.grow, i32(slots), i32(want), cu, n, int(cu[-1]), W, blocks, smap)
        rb, rm = ref.grow(slots.tolist(), want.tolist(), new.tolist())
        assert blocks.tolist() == [r + [-1] * (W - len(r)) for r in rb]
        assert smap.tolist() == [x for r in rm for x in r] + [-9]
        assert pool.held.tolist() == [len(h) for h in ref.held] and pool.state[1] == len(ref.free)
        held = np.array([len(h) for h in ref.held])
        lens[slots] = np.minimum(want, held[slots] * page)
        gone = rng.permutation(n + 3)[:n]
        keep = np.where(rng.random(n) < 0.3, 0, np.maximum(lens[gone] - rng.integers(0, 20, n), 0))
        pool.call(lib.trim, i32(gone), i32(keep), n)
        ref.trim(gone.tolist(), keep.tolist())
        lens[gone] = np.minimum(lens[gone], keep)
        assert pool.free[:len(ref.free)].tolist() == ref.free
        assert pool.held.tolist() == [len(h) for h in ref.held] and pool.state[1] == len(ref.free)


@pytest.mark.parametrize("n", [129, 1 << 16, (1 << 16) + 1, (1 << 24) - 1, 1 << 24, (1 << 24) + 1, 1 << 27])
def test_launches_of_many_entries(lib, n):
    """A row of a launch's grid has fewer than 2^32 threads, however many jobs a call names."""
    lib.threads_of.restype = ctypes.c_ulonglong
    size = i32([1 << 20, 16, n, 4])
    for total, width in ((0, 0), (n, 0), (n, 4), (2 ** 31 - 1, 4)):
        assert 0 < lib.threads_of(ctypes.c_void_p(size.ctypes.data), n, total, width) < 1 << 32

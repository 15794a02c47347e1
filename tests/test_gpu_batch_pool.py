"""Page pools at their ends, on the device: a schedule whose pool is too small for its batches, calls of very many jobs."""
import numpy as np
import pytest
import torch

from paper_2505_09142_amd import _elis as E
from paper_2505_09142_amd.device import PagePool
from paper_2505_09142_amd.driver import DeviceRoundDriver
from paper_2505_09142_amd.scheduler import run_schedule
from tests.gpu_util import note
from tests.test_gpu_batch_driver import Watched

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_pages", [14, 25])
def test_jobs_run_only_with_their_pages(n_pages):
    rng = np.random.default_rng(2)
    n = 40
    arrival = np.sort(rng.uniform(0, 3, n))
    prompts = [rng.integers(1, 99, int(m)).astype(np.int32) for m in rng.integers(1, 60, n)]
    responses = [rng.integers(1, 99, int(m)).astype(np.int32) for m in rng.integers(1, 150, n)]
    note(f"schedule of 40 jobs with {n_pages} pages")
    drv = Watched(None, 64, 8, pages=PagePool(n_pages, 16, 64, 14))
    kw = dict(window=20, step_cost=0.01, batch_cap=6, policy="sjf", end_rule="all")
    res = run_schedule(arrival, prompts, responses, drv, **kw)
    assert drv.checked == len(res.rounds) and np.isfinite(res.finish_t).all()
    assert any(len(r.chosen) < min(6, len(r.candidates)) for r in res.rounds)
    assert int(drv.pages.state[1]) == n_pages and drv.pages.status() == (E.ELIS_OK, 0)
    with pytest.raises(ValueError, match="pool"):
        run_schedule(arrival, prompts, responses, DeviceRoundDriver(None, 64, 8, pages=PagePool(600, 16, 64, 3)), **kw)


@pytest.mark.parametrize("n", [70_000, (1 << 24) + 77])
def test_pages_of_very_many_jobs(n):
    """More entries than the second launch has work-groups, and more than it could have. A page each, and back."""
    note(f"pages of {n} jobs")
    pool = PagePool(n, 16, n, 1)
    slots = torch.randperm(n, device="cuda").to(torch.int32)
    lens = torch.ones(n, dtype=torch.int32, device="cuda")
    cu = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    smap = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    blocks = torch.full((n, 1), -9, dtype=torch.int32, device="cuda")
    pool.grow(slots, lens, cu, n, smap, out_blocks=blocks)
    assert pool.status() == (E.ELIS_OK, 0) and int(pool.state[1]) == 0
    assert torch.equal(blocks[:, 0], cu[:n]) and torch.equal(smap, 16 * cu[:n])          # entry i takes page i
    assert torch.equal(pool.table[slots.long(), 0], cu[:n]) and int(pool.held.min()) == int(pool.held.max()) == 1
    pool.grow(slots, lens, None, 0, None)                                                # nothing to do, and no claim is left
    assert pool.status() == (E.ELIS_OK, 0) and int(pool.held.min()) == int(pool.held.max()) == 1
    pool.trim(slots, lens - 1)
    assert pool.status() == (E.ELIS_OK, 0) and int(pool.state[1]) == n and int(pool.held.max()) == 0
    assert torch.equal(pool.free_pages, cu[:n].flip(0))

"""A schedule whose page pool is too small for its batches, on the device."""
import numpy as np
import pytest

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

"""The round driver's page pool and logits: pages follow the batch through a whole schedule (preemptions and ends give
theirs back, the first of the batch are served first), and logits are adjusted with the histories the table holds."""
import numpy as np
import pytest
import torch

from oracle import batch as O
from oracle.simulate import job_input
from paper_2505_09142_amd import _elis as E
from paper_2505_09142_amd.device import PagePool
from paper_2505_09142_amd.driver import DeviceRoundDriver
from paper_2505_09142_amd.scheduler import run_schedule
from tests.gpu_util import note

pytestmark = pytest.mark.gpu


class Watched(DeviceRoundDriver):
    """Checks the pool after every window's reservation against the batch's lengths."""

    def reserve(self, jobs, lens, *args, **kw):
        out = super().reserve(jobs, lens, *args, **kw)
        held = self.pages.held.cpu().numpy()
        want = np.zeros_like(held)
        for j, n in zip(jobs, lens):
            want[self.slot_of[j]] = -(-n // self.pages.page_tokens)
        assert np.array_equal(held, want)
        table = self.pages.table.cpu().numpy()
        ids = np.concatenate([table[s, :held[s]] for s in range(len(held))])
        assert len(set(ids.tolist())) == len(ids) and int(self.pages.state[1]) == self.pages.n_pages - len(ids)
        self.checked = getattr(self, "checked", 0) + 1
        return out


def test_pages_follow_the_schedule():
    rng = np.random.default_rng(2)
    n = 40
    arrival = np.sort(rng.uniform(0, 3, n))
    prompts = [rng.integers(1, 99, int(m)).astype(np.int32) for m in rng.integers(1, 60, n)]
    responses = [rng.integers(1, 99, int(m)).astype(np.int32) for m in rng.integers(1, 150, n)]
    note("schedule of 40 jobs with a page pool")
    drv = Watched(None, 64, 8, pages=PagePool(600, 16, 64, 16))
    plain = DeviceRoundDriver(None, 64, 8)
    kw = dict(window=20, step_cost=0.01, batch_cap=6, policy="sjf", end_rule="first")
    a, b = (run_schedule(arrival, prompts, responses, d, **kw) for d in (drv, plain))
    assert np.array_equal(a.finish_t, b.finish_t) and [r.chosen for r in a.rounds] == [r.chosen for r in b.rounds]
    assert drv.checked == len(a.rounds) and a.preemptions.sum() > 0
    assert int(drv.pages.state[1]) == 600 and drv.pages.status() == (E.ELIS_OK, 0)
    with pytest.raises(ValueError):
        DeviceRoundDriver(None, 65, 8, pages=drv.pages)


def test_slot_maps_and_logits_of_a_batch():
    rng = np.random.default_rng(3)
    max_pos, vocab = 16, 200
    drv = DeviceRoundDriver(None, 32, max_pos, pages=PagePool(64, 16, 32, 8))
    jobs = [3, 11, 5, 8]
    prompts = {j: rng.integers(0, vocab, m).astype(np.int32) for j, m in zip(jobs, (4, 20, 15, 16))}
    responses = {j: rng.integers(0, vocab, 40).astype(np.int32) for j in jobs}
    gen = {3: 5, 11: 9, 5: 30, 8: 0}
    drv.start(jobs, [0, 1, 2, 3])
    drv.sync_tokens(jobs, prompts, responses, gen)
    lens = [len(prompts[j]) + gen[j] for j in jobs]
    new = [2, 1, 3, 16]
    note("driver: slot map of a batch")
    slot_map = torch.full((sum(new),), -9, dtype=torch.int32, device="cuda")
    rows = drv.reserve(jobs, lens, new, slot_map)
    table, rows = drv.pages.table.cpu().numpy(), rows.cpu().numpy()
    want = [table[r, p // 16] * 16 + p % 16 for r, n, m in zip(rows, lens, new) for p in range(n - m, n)]
    assert slot_map.cpu().tolist() == want
    note("driver: logits with the table's histories")
    logits = torch.from_numpy(rng.standard_normal((4, vocab)).astype(np.float32)).cuda()
    one = lambda v: torch.full((4,), v, dtype=torch.float32, device="cuda")  # noqa: E731
    out = drv.adjust_logits(jobs, logits, [len(prompts[j]) for j in jobs], repetition=one(1.5), frequency=one(0.25), presence=one(0.5))
    for i, j in enumerate(jobs):
        history = job_input(prompts[j], responses[j], gen[j], max_pos).tolist()
        # which of them are the prompt's: the first token, and those of the recent ones that lie in it
        n, plen = lens[i], len(prompts[j])
        at = list(range(n)) if n <= max_pos else [0] + list(range(n - max_pos + 1, n))
        x = logits[i].double().cpu().numpy()
        y = O.logits_adjust(x, history, sum(p < plen for p in at), 1.5, 0.25, 0.5)
        assert (np.abs(out[i].double().cpu().numpy() - y) <= 5 * 2.0 ** -24 * (np.abs(x) * 1.5 + 0.25 * max_pos + 0.5)).all()
    assert drv.adjust_logits([], logits[:0], []).shape == (0, vocab)
    with pytest.raises(ValueError):
        drv.adjust_logits(jobs, logits[:2], [1, 1, 1, 1])
    drv.drop([5])
    drv.release([3, 11, 8])
    assert int(drv.pages.state[1]) == 64 and drv.table.status() == (E.ELIS_OK, 0)


def test_batches_that_are_refused_or_empty():
    drv = DeviceRoundDriver(None, 8, 16, pages=PagePool(8, 16, 8, 4))
    drv.start([1, 2], [0, 1])
    note("driver: empty and refused batches")
    drv.sync_tokens([1], {1: np.array([4, 5], dtype=np.int32)}, {1: np.zeros(0, np.int32)}, {1: 0})
    logits = torch.zeros((2, 9), dtype=torch.float32, device="cuda")
    for jobs, prompts in (([1, 2], [2, 1]), ([1], [2]), ([1, 1], [2])):  # a job without tokens; rows or lengths that do not fit
        with pytest.raises(ValueError):
            drv.adjust_logits(jobs, logits, prompts)
    assert drv.table.status() == (E.ELIS_OK, 0)
    with pytest.raises(ValueError):
        drv.reserve([1, 2], [5])
    assert drv.reserve([], []).numel() == 0
    drv.reserve([2], [33])
    drv.drop([])
    assert int(drv.pages.state[1]) == 5 and drv.pages.status() == (E.ELIS_OK, 0)

"""The round driver's calls for the selected batch, host side (no kernel is launched here)."""
import numpy as np
import pytest
import torch

from oracle import batch as O
from paper_2505_09142_amd import _elis as E
from paper_2505_09142_amd.driver import DeviceRoundDriver
from paper_2505_09142_amd.scheduler import run_schedule


def test_logits_take_no_stream():
    """The histories are packed on the current stream: an adjustment on another one would read them too early."""
    drv = DeviceRoundDriver.__new__(DeviceRoundDriver)
    drv.appended, drv.slot_of = {1: 3}, {1: 0}
    with pytest.raises(TypeError, match="stream"):
        drv.adjust_logits([1], torch.zeros((1, 9)), [1], stream=object())
    with pytest.raises(TypeError):
        drv.adjust_logits([1], torch.zeros((1, 9)), [1], cu_seqlens=torch.zeros(2))


class Pool(O.Pages):
    """The oracle's pages behind the attributes of a page pool; bits as the library's."""

    def __init__(self, n_pages, page_tokens, max_jobs, max_pages):
        super().__init__(n_pages, page_tokens, max_jobs, max_pages)
        self.page_tokens, self.n_pages, self.bits = page_tokens, n_pages, 0

    @property
    def state(self):
        return [self.bits, len(self.free)]

    def status(self):
        return (E.ELIS_EDEVICE if self.bits else E.ELIS_OK), self.bits


class Driver:
    """A round driver on the host: keys in a dict, pages of the oracle. Checks every window's reservation."""

    def __init__(self, pages=None):
        self.pages, self.slot_of, self.key, self.windows = pages, {}, {}, 0

    def start(self, jobs, arrival):
        self.slot_of.update((j, j) for j in jobs)

    def store_keys(self, jobs, keys):
        self.key.update(zip(jobs, keys))

    def select(self, candidates, cap, wait=None, aging=0.0):
        return sorted(candidates, key=lambda j: (self.key[j], j))[:cap]

    def reserve(self, jobs, lens):
        self.windows += 1
        self.pages.grow([self.slot_of[j] for j in jobs], lens, [0] * len(jobs))
        if self.pages.short:
            self.pages.bits |= E.ELIS_DEV_NO_PAGES
        for j, n in zip(jobs, lens):
            assert len(self.pages.held[self.slot_of[j]]) == -(-n // self.pages.P), f"job {j} runs without its pages"
        assert sum(map(len, self.pages.held)) == sum(-(-n // self.pages.P) for n in lens)  # and nobody else holds any

    def drop(self, jobs):
        self.pages.trim([self.slot_of[j] for j in jobs], [0] * len(jobs))

    def release(self, jobs):
        if self.pages is not None:
            self.drop(jobs)


def requests(seed, n=30):
    rng = np.random.default_rng(seed)
    some = lambda hi: [np.zeros(int(m), np.int32) for m in rng.integers(1, hi, n)]  # noqa: E731
    return np.sort(rng.uniform(0, 2, n)), some(60), some(150)


KW = dict(window=20, step_cost=0.01, batch_cap=6)


@pytest.mark.parametrize("end_rule", ["all", "first"])
@pytest.mark.parametrize("policy", ["sjf", "fcfs"])
@pytest.mark.parametrize("n_pages", [14, 20, 31, 45, 600])
def test_jobs_run_only_with_their_pages(n_pages, policy, end_rule):
    """Pools from one that the longest job alone fills to an ample one."""
    arrival, prompts, responses = requests(2)
    drv = Driver(Pool(n_pages, 16, 30, 14))
    res = run_schedule(arrival, prompts, responses, drv, policy=policy, end_rule=end_rule, **KW)
    assert not drv.pages.short and drv.windows == len(res.rounds) and len(drv.pages.free) == n_pages
    assert np.isfinite(res.finish_t).all() and res.generated.tolist() == [len(r) for r in responses]
    plain = run_schedule(arrival, prompts, responses, Driver(), policy=policy, end_rule=end_rule, **KW)
    same = [r.chosen for r in res.rounds] == [r.chosen for r in plain.rounds]
    assert same == (n_pages == 600)
    if same:
        assert np.array_equal(res.finish_t, plain.finish_t) and np.array_equal(res.preemptions, plain.preemptions)
    else:
        assert any(len(r.chosen) < min(6, len(r.candidates)) for r in res.rounds)


def test_a_job_that_is_cut_off_is_preempted():
    """Two jobs of two pages each in a pool of three: the second one gives its first page back while the first grows."""
    prompts, responses = [np.zeros(10, np.int32), np.zeros(10, np.int32)], [np.zeros(20, np.int32)] * 2
    drv = Driver(Pool(3, 16, 2, 2))
    res = run_schedule([0.0, 0.0], prompts, responses, drv, window=6, step_cost=1.0, batch_cap=2, policy="fcfs", prefill_cost=0.5)
    assert [r.chosen for r in res.rounds] == [[0, 1], [0], [0], [0], [1], [1], [1]]
    assert res.preemptions.tolist() == [0, 1] and res.rounds[4].resumed == [1] and res.rounds[4].prefill_s == 0.5 * 16
    assert res.finish_t.tolist() == [20.0, 20.0 + 8.0 + 14.0]


def test_what_the_pool_can_never_hold_is_refused():
    arrival, prompts, responses = requests(3)
    most = max(-(-(len(p) + len(r)) // 16) for p, r in zip(prompts, responses))
    for n_pages, max_pages in ((600, most - 1), (most - 1, 100)):
        drv = Driver(Pool(n_pages, 16, 30, max_pages))
        with pytest.raises(ValueError, match="pool"):
            run_schedule(arrival, prompts, responses, drv, policy="sjf", **KW)
        assert not drv.slot_of and len(drv.pages.free) == n_pages
    drv = Driver(Pool(600, 16, 30, most))
    drv.pages.bits = E.ELIS_DEV_BAD_SLOT                       # of an earlier call
    with pytest.raises(E.ElisError):
        run_schedule(arrival, prompts, responses, drv, policy="sjf", **KW)


def test_pages_that_somebody_else_takes_are_noticed():
    class Shared(Driver):
        def reserve(self, jobs, lens):
            self.windows += 1
            if self.windows == 3:
                self.pages.bits |= E.ELIS_DEV_NO_PAGES         # as a grow of somebody else's would leave it

    arrival, prompts, responses = requests(4)
    with pytest.raises(E.ElisError):
        run_schedule(arrival, prompts, responses, Shared(Pool(600, 16, 30, 14)), policy="sjf", **KW)

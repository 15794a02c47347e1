"""Cached attention whose scores jump, in every kernel: the running maximum has to follow at once.

Queries are +-2 u and the high keys c u for a sign vector u, so their scores are exact: +-2 c sqrt(d) times log2(e), 16 to
1,100 powers of two. Queries of both signs lie in one block of rows: for one the high keys take all the weight, for the
other none. The high keys come in growing order, at places that every row of the request sees, in turn at each of the four
keys that a lane holds. The tolerance is that of the other attention tests: the exponent's argument is one rounding of a
fused product and sum, so keys whose weights count (within 2^-24 of the largest) have it as exact as with flat scores.
"""
import numpy as np
import pytest
import torch

from paper_2505_09142_amd import _elis as E
from tests.gpu_util import note
from tests.test_gpu_batch import BF, check_attention, host, i32, paged

pytestmark = pytest.mark.gpu
HEIGHTS = (0.5, 1.0, 1.5, 8.0, 24.0)

KERNELS = [  # heads, kv heads, d, q lens, kv lens, heads to compare
    (4, 2, 64, [1], [700], None), (8, 2, 128, [1], [700], None),                        # 16 rows
    (8, 2, 128, [1, 1], [3000, 500], None),                                             # and split
    (20, 1, 64, [1], [700], None), (34, 2, 128, [1], [700], None), (32, 1, 128, [1], [2500], None),  # 17 to 32 rows
    (8, 2, 64, [40], [500], None), (8, 2, 128, [70], [500], None),                      # prompts in tiles of 32 rows
    (8, 2, 64, [40, 1, 1], [500, 700, 450], None), (8, 2, 128, [70, 1, 1], [500, 700, 450], None),      # beside single tokens
    (20, 1, 64, [30, 1], [500, 700], None), (20, 1, 128, [30, 1], [500, 700], None),    # of 20 rows
    (128, 128, 128, [200], [450], [0, 77]), (64, 64, 128, [448, 1], [1000, 500], [3, 63]),  # tiles of 64 rows, alone and beside one
]


def climbing(rng, kv_lens, q_lens, kv_heads, d, key):
    """The cache, blocks, what it keeps, and the sign vectors [kv heads, d]; the high keys at lane key `key`."""
    cache, blocks, k, v, slots = paged(rng, kv_lens, kv_heads, d, 16)
    u = np.sign(rng.standard_normal((kv_heads, d)))
    at = 0
    for q, n in zip(q_lens, kv_lens):
        seen = n - q + 1                                     # keys that every query sees
        recs = np.sort(rng.permutation(seen // 16 - 1)[:len(HEIGHTS)])
        where = at + 16 * recs + 4 * rng.integers(0, 4, len(recs)) + key
        high = torch.from_numpy(np.array(HEIGHTS)[:, None, None] * u).to("cuda").to(BF)
        vals = torch.from_numpy(v[where]).to("cuda").to(BF)
        cache.append(high, vals, slots[torch.from_numpy(where).to("cuda")])
        k[where] = host(high)
        at += n
    return cache, blocks, k, v, u


def queries(rng, tokens, heads, kv_heads, u):
    sign = np.where(rng.random((tokens, heads, 1)) < 0.5, -1.0, 1.0)
    return torch.from_numpy(2.0 * sign * np.repeat(u, heads // kv_heads, axis=0)).to("cuda").to(BF)


def compare(out, q, q_lens, kv_lens, k, v, heads, kv_heads, d, few):
    few = range(kv_heads) if few is None else few
    g = heads // kv_heads
    qh = [h * g + i for h in few for i in range(g)]
    check_attention(out[:, qh], q[:, qh], q_lens, kv_lens, k[:, list(few)], v[:, list(few)], d ** -0.5)


@pytest.mark.parametrize("key", range(4))
@pytest.mark.parametrize("heads,kv_heads,d,q_lens,kv_lens,few", KERNELS)
def test_scores_that_jump(heads, kv_heads, d, q_lens, kv_lens, few, key):
    note(f"kv attention, jumping scores: q={q_lens} kv={kv_lens} heads={heads}/{kv_heads} d={d} key {key}")
    rng = np.random.default_rng(heads + d + key)
    cache, blocks, k, v, u = climbing(rng, kv_lens, q_lens, kv_heads, d, key)
    q = queries(rng, sum(q_lens), heads, kv_heads, u)
    cu = i32(np.concatenate([[0], np.cumsum(q_lens)]))
    out = cache.attention(q, cu, i32(kv_lens), i32(blocks), max(q_lens), max(kv_lens))
    assert cache.status() == (E.ELIS_OK, 0) and bool(torch.isfinite(out).all())
    compare(out, q, q_lens, kv_lens, k, v, heads, kv_heads, d, few)
    again = cache.attention(q, cu, i32(kv_lens), i32(blocks), max(q_lens), max(kv_lens))
    assert torch.equal(out, again)


@pytest.mark.parametrize("heads,kv_heads,d", [(8, 2, 128), (4, 2, 64), (34, 2, 64), (32, 1, 128)])
def test_scores_that_jump_past_the_caches(heads, kv_heads, d):
    """As above under a bound on the lengths by which the batch may hold more than the caches."""
    rng = np.random.default_rng(d)
    q_lens, kv_lens = [1] * 4, [700, 300, 1500, 450]
    width = -(-420_000_000 // (4 * kv_heads * 17 * d // 16 * 16))
    note(f"kv attention, jumping scores past the caches: heads={heads}/{kv_heads} d={d}")
    cache, blocks, k, v, u = climbing(rng, kv_lens, q_lens, kv_heads, d, 2)
    table = np.full((4, width), -1)
    table[:, :blocks.shape[1]] = blocks
    q = queries(rng, 4, heads, kv_heads, u)
    out = cache.attention(q, i32(range(5)), i32(kv_lens), i32(table), 1, width * 16)
    compare(out, q, q_lens, kv_lens, k, v, heads, kv_heads, d, None)


@pytest.mark.parametrize("heads,kv_heads,d,q_lens,kv_lens,few", KERNELS)
def test_a_query_of_nan_is_its_own_rows(heads, kv_heads, d, q_lens, kv_lens, few):
    """NaN in one query head: its row is NaN, and the jumps of the rows beside it are followed all the same."""
    note(f"kv attention, a query of NaN: q={q_lens} kv={kv_lens} heads={heads}/{kv_heads} d={d}")
    rng = np.random.default_rng(heads + d)
    cache, blocks, k, v, u = climbing(rng, kv_lens, q_lens, kv_heads, d, 1)
    T = sum(q_lens)
    q = queries(rng, T, heads, kv_heads, u)
    bad = [(int(rng.integers(T)), h) for h in range(0, heads, 3)]
    args = i32(np.concatenate([[0], np.cumsum(q_lens)])), i32(kv_lens), i32(blocks), max(q_lens), max(kv_lens)
    clean = cache.attention(q, *args)
    compare(clean, q, q_lens, kv_lens, k, v, heads, kv_heads, d, few)
    with_nan = q.clone()
    for t, h in bad:
        with_nan[t, h, int(rng.integers(d))] = float("nan")
    out = cache.attention(with_nan, *args)
    nan = torch.zeros((T, heads, d), dtype=torch.bool, device="cuda")
    for t, h in bad:
        nan[t, h] = True
    assert torch.equal(torch.isnan(out), nan)
    compare(torch.where(nan, clean, out), q, q_lens, kv_lens, k, v, heads, kv_heads, d, few)

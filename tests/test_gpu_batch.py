"""The batch operators on the GPU against the 64-bit oracle: pages, 4-bit cache, cached attention, logits, and a decode
loop of all of them over the job table.

Tolerances. Integers, 4-bit values and what the cache reads back: equal. Attention: a weight is rounded to bf16 once
(half a step, 2^-8 of it) and the same rounded weights are summed for the denominator, so numerator and denominator are
each off by at most 2^-8 of sum w|v|, and the result is rounded to bf16, 2^-8 of it again: 3 * 2^-8 * sum w|v|, and a
hundredth of that for the fp32 sums and exponentials. Logits: five fp32 operations, 2^-24 each of the largest
intermediate value (|x| max(r, 1/r) + |f| c + |p| + sum |b|), times (5 + biases).
"""
import numpy as np
import pytest
import torch

from oracle import batch as O
from oracle.select import oracle_select
from paper_2505_09142_amd import _elis as E
from paper_2505_09142_amd.device import JobTable, KVCache, PagePool, adjust_logits
from tests.gpu_util import dev, note

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def i32(a):
    return dev(np.asarray(a, dtype=np.int32))


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64) if t.is_floating_point() else t.cpu().numpy()


# ------------------------------------------------------------------ pages

@pytest.mark.parametrize("n,page,longest", [(1, 16, 5000), (3, 16, 40), (64, 16, 700), (128, 64, 300), (129, 16, 60), (700, 32, 90), (2500, 16, 70)])
def test_pages_follow_the_oracle(n, page, longest):
    rng = np.random.default_rng(n)
    J, W = n + 7, -(-longest // page) + 2
    n_pages = int(n * longest / page * 0.45) + 3          # runs out now and then
    pool, ref = PagePool(n_pages, page, J, W), O.Pages(n_pages, page, J, W)
    lens = np.zeros(J, np.int64)
    for step in range(6):
        m = int(rng.integers(1, n + 1))
        slots = rng.permutation(J)[:m]
        new = rng.integers(0, longest // 3 + 2, m) if step % 2 else rng.integers(0, 2, m)
        want = np.minimum(lens[slots] + new, W * page)
        new = want - lens[slots]
        width, total = int(rng.integers(1, W + 1)), int(new.sum())
        note(f"pages grow n={m} page={page} step={step} new={total}")
        blocks = torch.full((m + 1, width), -9, dtype=torch.int32, device="cuda")
        slot_map = torch.full((total + 5,), -9, dtype=torch.int32, device="cuda")
        pool.grow(i32(slots), i32(want), i32(np.concatenate([[0], np.cumsum(new)])), total, slot_map, out_blocks=blocks[:m])
        rb, rm = ref.grow(slots.tolist(), want.tolist(), new.tolist())
        assert host(blocks)[:m].tolist() == [(r + [-1] * width)[:width] for r in rb]
        assert (host(blocks)[m] == -9).all() and (host(slot_map)[total:] == -9).all()
        assert host(slot_map)[:total].tolist() == [x for r in rm for x in r]
        held = np.array([len(h) for h in ref.held])
        assert host(pool.held).tolist() == held.tolist() and int(pool.state[1]) == len(ref.free)
        assert host(pool.free_pages)[:len(ref.free)].tolist() == ref.free
        status, bits = pool.status()
        assert bits == (E.ELIS_DEV_NO_PAGES if ref.short else 0) and status == (E.ELIS_EDEVICE if ref.short else E.ELIS_OK)
        lens[slots] = np.minimum(want, held[slots] * page)
        gone = rng.permutation(J)[:max(1, J // 3)]
        keep = np.where(rng.random(len(gone)) < 0.5, 0, lens[gone] * rng.random(len(gone))).astype(np.int64)
        note(f"pages trim n={len(gone)}")
        for a in range(0, len(gone), n):
            pool.trim(i32(gone[a:a + n]), i32(keep[a:a + n]))
            ref.trim(gone[a:a + n].tolist(), keep[a:a + n].tolist())
        lens[gone] = np.minimum(lens[gone], keep)
        assert host(pool.free_pages)[:len(ref.free)].tolist() == ref.free
        assert host(pool.held).tolist() == [len(h) for h in ref.held] and int(pool.state[1]) == len(ref.free)
        table = host(pool.table)
        assert all(table[s, :len(h)].tolist() == h for s, h in enumerate(ref.held))
    every = sorted(ref.free + [p for h in ref.held for p in h])
    assert every == list(range(n_pages))


def test_pages_content_errors():
    pool = PagePool(40, 16, 8, 3)
    out = torch.full((4,), -9, dtype=torch.int32, device="cuda")
    note("pages: slots outside, a slot twice, a length past the table, a negative one")
    pool.grow(i32([1, 99, -1, 1]), i32([20, 20, 20, 20]), i32([0, 1, 2, 3, 4]), 4, out)
    assert pool.status()[1] == E.ELIS_DEV_BAD_SLOT
    assert int(pool.state[1]) == 38 and host(pool.held).tolist() == [0, 2, 0, 0, 0, 0, 0, 0]
    assert sorted(host(out).tolist()) == [-1, -1, -1, 19] and host(out)[1:3].tolist() == [-1, -1]  # one of the two is served
    pool = PagePool(40, 16, 8, 3)
    pool.grow(i32([2, 3, 4]), i32([49, -5, 48]), i32([0, 1, 2, 3]), 3, out[:3])
    assert pool.status()[1] & E.ELIS_DEV_LONG_SEQ and pool.status()[1] & E.ELIS_DEV_BAD_SLOT
    assert host(pool.held).tolist() == [0, 0, 0, 0, 3, 0, 0, 0] and host(out)[:3].tolist() == [-1, -1, 2 * 16 + 15]
    pool = PagePool(40, 16, 8, 3)
    pool.grow(i32([2, 3]), i32([5, 5]), i32([0, 9, 2]), 2, out[:2])
    assert pool.status()[1] & E.ELIS_DEV_BAD_CU
    pool.trim(i32([2, 2, 77]), i32([0, 0, 0]))
    assert int(pool.state[1]) + int(pool.held.sum()) == 40


@pytest.mark.parametrize("n,page,longest", [(100, 16, 9000), (5, 1024, 70000)])
def test_pages_wide_tables_and_again(n, page, longest):
    """Tables of many cells (two launches for few jobs); a call served again changes nothing; pages back by a trim."""
    rng = np.random.default_rng(page)
    W = -(-longest // page)
    lens = rng.integers(1, longest + 1, n)
    need = -(-lens // page)
    pool, ref = PagePool(int(need.sum()), page, n, W), O.Pages(int(need.sum()), page, n, W)
    slots, total = rng.permutation(n), int(lens.sum())
    rb, rm = ref.grow(slots.tolist(), lens.tolist(), lens.tolist())
    for turn in range(3):
        note(f"pages wide n={n} page={page} turn={turn}")
        blocks = torch.full((n, W), -9, dtype=torch.int32, device="cuda")
        smap = torch.full((total,), -9, dtype=torch.int32, device="cuda")
        pool.grow(i32(slots), i32(lens), i32(np.concatenate([[0], np.cumsum(lens)])), total, smap, out_blocks=blocks)
        assert host(blocks).tolist() == [r + [-1] * (W - len(r)) for r in rb] and host(smap).tolist() == [x for r in rm for x in r]
        assert int(pool.state[1]) == 0 and pool.status() == (E.ELIS_OK, 0)
    pool.trim(i32(slots), i32(np.zeros(n)))
    assert host(pool.free_pages).tolist() == list(range(int(need.sum())))[::-1] and int(pool.held.sum()) == 0


# ------------------------------------------------------------------ the cache

def filled(rng, T, heads, d, extra=0):
    """k, v as views of a wider matrix, with a spread of magnitudes, zero groups and huge and tiny ones."""
    x = rng.standard_normal((T, 2 * heads * d + extra)) * np.exp(rng.standard_normal((T, 1)))
    x[rng.random(x.shape) < 0.02] = 0
    x[0, :32] = 0
    if T > 2:
        x[1, :64] *= 2.0 ** 120
        x[2, :64] *= 2.0 ** -120
    t = torch.from_numpy(x).to("cuda").to(BF)
    return t[:, :heads * d].unflatten(1, (heads, d)), t[:, heads * d:2 * heads * d].unflatten(1, (heads, d))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,heads,page,extra", [(1, 1, 16, 0), (5, 3, 16, 8), (37, 2, 32, 1), (130, 1, 64, 0)])
def test_append_then_read(T, heads, page, extra, d):
    rng = np.random.default_rng(T + d)
    note(f"kv append + read T={T} heads={heads} d={d} page={page} extra={extra}")
    k, v = filled(rng, T, heads, d, extra)
    n_pages = -(-T // page) + 2
    cache = KVCache(n_pages, page, heads, d)
    base = cache.c.base - cache.buf.data_ptr() + 256
    cache.buf[base:].fill_(0xEE)
    slots = rng.permutation(n_pages * page)[:T].astype(np.int32)
    if T > 4:
        slots[3] = -1
    cache.append(k, v, i32(slots))
    out_k, out_v = (torch.full((T + 1, heads, d), 7.0, dtype=BF, device="cuda") for _ in range(2))
    cache.read(i32(slots), out_k[:T], out_v[:T])
    for x, out in ((k, out_k), (v, out_v)):
        want = O.kv_round(host(x))
        want[slots < 0] = 0
        assert np.array_equal(host(out)[:T], want)
        assert (host(out)[T] == 7).all()
    assert cache.status() == (E.ELIS_OK, 0)
    # slots that no token took are left as they were
    rec = host(cache.buf)[base:base + n_pages * heads * page * 17 * d // 16].reshape(n_pages, heads, page // 16, 17 * d)
    used = set(slots[slots >= 0].tolist())
    for s in set(range(n_pages * page)) - used:
        r = rec[s // page, :, s % page // 16]
        b = s % 16
        assert (r[:, b * d // 2:(b + 1) * d // 2] == 0xEE).all()
        assert (r[:, 8 * d:16 * d].reshape(heads, 4, 16, 4, d // 32)[:, b // 4, :, b % 4] == 0xEE).all()
        assert (r[:, 16 * d:16 * d + d // 2].reshape(heads, 16, d // 32)[:, b] == 0xEE).all()
        assert (r[:, 16 * d + d // 2:].reshape(heads, 4, d // 32, 4)[:, b // 4, :, b % 4] == 0xEE).all()


def test_append_ties_and_non_finite():
    d = 64
    x = np.zeros((3, 1, d))
    x[0, 0, :16] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5, 5.03125]
    x[1, 0, :3] = [np.inf, 1, 2]
    x[1, 0, 40] = -3e38
    x[2, 0, 33] = np.nan
    x[2, 0, :2] = [2.0 ** -126, 1e-39]
    t = torch.from_numpy(x).to("cuda").to(BF)
    note("kv append: ties, infinity, NaN, the ends of the exponent range")
    cache = KVCache(1, 16, 1, d)
    out = [torch.empty_like(t) for _ in range(2)]
    cache.append(t, t, i32([3, 4, 5]))
    cache.read(i32([3, 4, 5]), *out)
    for o in out:
        assert np.array_equal(host(o), O.kv_round(host(t)), equal_nan=True)
    note("kv append / read: a slot outside the cache")
    cache.append(t, t, i32([16, -1, 2 ** 31 - 1]))
    assert cache.status() == (E.ELIS_EDEVICE, E.ELIS_DEV_BAD_PAGE)
    E.check(E.elis_kv_init(cache.c, None))
    cache.append(t, t, i32([-1, -7, -1]))
    assert cache.status() == (E.ELIS_EDEVICE, E.ELIS_DEV_BAD_PAGE)
    cache.read(i32([99, -1, 3]), *out)
    assert (host(out[0])[:2] == 0).all() and np.array_equal(host(out[0])[2], O.kv_round(host(t[0])))


# ------------------------------------------------------------------ attention

def paged(rng, kv_lens, heads, d, page, spare=3):
    """A cache holding kv_lens[i] random tokens of each request on scattered pages; stale bytes everywhere else."""
    need = [-(-n // page) for n in kv_lens]
    n_pages = sum(need) + spare
    cache = KVCache(n_pages, page, heads, d)
    cache.buf.fill_(0xFF)  # every scale NaN
    E.check(E.elis_kv_init(cache.c, None))
    ids = rng.permutation(n_pages)
    width = max(max(need), 1) + 1
    blocks = np.full((len(kv_lens), width), -1)
    at, slots = 0, []
    for i, (m, n) in enumerate(zip(need, kv_lens)):
        blocks[i, :m] = ids[at:at + m]
        slots.append(blocks[i, np.arange(n) // page] * page + np.arange(n) % page)
        at += m
    T = sum(kv_lens)
    slots = i32(np.concatenate(slots))
    k = torch.from_numpy(rng.standard_normal((T, heads, d))).to("cuda").to(BF)
    v = torch.from_numpy(rng.standard_normal((T, heads, d))).to("cuda").to(BF)
    cache.append(k, v, slots)
    cache.read(slots, k, v)
    return cache, blocks, host(k), host(v), slots


def check_attention(out, q, q_lens, kv_lens, k, v, scale, window=0, seen=None):
    at_q = at_k = 0
    for i, (a, b) in enumerate(zip(q_lens, kv_lens)):
        args = host(q)[at_q:at_q + a], k[at_k:at_k + b]
        s = None if seen is None else seen[i]
        want = O.kv_attention(*args, v[at_k:at_k + b], b, scale, window, s)
        size = O.kv_attention(*args, np.abs(v[at_k:at_k + b]), b, scale, window, s)
        got = host(out)[at_q:at_q + a]
        assert np.isfinite(got).all() and (np.abs(got - want) <= 3 * 2.0 ** -8 * 1.01 * size + 1e-30).all(), \
            (i, a, b, np.abs(got - want).max(), (np.abs(got - want) / (size + 1e-30)).max())
        at_q += a
        at_k += b


SHAPES = [  # q lens, kv lens
    ([1], [1]), ([1], [193]), ([1, 1, 1], [15, 16, 17]), ([1] * 5, [31, 32, 33, 1, 700]), ([1], [9001]),
    ([3, 0, 1, 2], [5, 40, 0, 130]), ([4], [2]), ([16, 1, 7], [16, 50, 400]), ([70, 1, 1], [70, 300, 2]), ([200, 130], [200, 517]), ([33], [4500]),
]


@pytest.mark.parametrize("heads,kv_heads,d,page,window", [
    (2, 2, 64, 16, 0), (8, 2, 128, 16, 0), (5, 1, 128, 32, 0), (4, 1, 64, 64, 0), (8, 2, 128, 16, 40), (2, 2, 64, 32, 1), (34, 2, 64, 16, 0), (40, 1, 128, 128, 100),
    (66, 1, 64, 16, 0)])
@pytest.mark.parametrize("q_lens,kv_lens", SHAPES)
def test_attention(q_lens, kv_lens, heads, kv_heads, d, page, window):
    if heads > 8 and max(kv_lens) > 1000:
        kv_lens, q_lens = [min(n, 1200) for n in kv_lens], [min(n, 9) for n in q_lens]
    note(f"kv attention q={q_lens} kv={kv_lens} heads={heads}/{kv_heads} d={d} page={page} window={window}")
    rng = np.random.default_rng(sum(kv_lens) + heads)
    cache, blocks, k, v, _ = paged(rng, kv_lens, kv_heads, d, page)
    T = sum(q_lens)
    q = torch.from_numpy(rng.standard_normal((T + 2, heads, d)) * 2).to("cuda").to(BF)
    out = torch.full((T + 2, heads, d), 5.0, dtype=BF, device="cuda")
    cu = i32(np.concatenate([[0], np.cumsum(q_lens)]))
    cache.attention(q, cu, i32(kv_lens), i32(blocks), max(q_lens), max(kv_lens), window=window, out=out)
    assert cache.status() == (E.ELIS_OK, 0)
    check_attention(out, q, q_lens, kv_lens, k, v, d ** -0.5, window)
    assert (host(out)[T:] == 5).all()  # rows behind the last request are left as they were
    # larger bounds, block tables by slot, strided and unaligned rows: the same request, other launches
    table = np.full((len(kv_lens) + 4, blocks.shape[1] + 30), -1)
    rows = rng.permutation(len(table))[:len(kv_lens)]
    table[rows, :blocks.shape[1]] = blocks
    wide = torch.zeros((T + 2, heads * d + 3), dtype=BF, device="cuda")
    wide[:, 1:1 + heads * d] = q.flatten(1)
    wide_out = torch.full((T + 2, heads * d + 5), 5.0, dtype=BF, device="cuda")
    view = lambda w: w[:, 1:1 + heads * d].unflatten(1, (heads, d))  # noqa: E731
    cache.attention(view(wide), cu, i32(kv_lens), i32(table), max(q_lens) + 30, max(kv_lens) + 16 * page, rows=i32(rows), window=window,
                    out=view(wide_out))
    check_attention(view(wide_out), q, q_lens, kv_lens, k, v, d ** -0.5, window)
    assert (host(wide_out)[T:] == 5).all() and (host(wide_out)[:, 0] == 5).all() and (host(wide_out)[:, 1 + heads * d:] == 5).all()


@pytest.mark.parametrize("heads,kv_heads,d,window,q_lens,kv_lens", [
    (128, 128, 64, 0, [300, 0, 250], [300, 7, 400]),           # tiles of 64 rows
    (128, 128, 128, 90, [300, 1, 250, 1], [300, 700, 310, 30]),  # beside single tokens
    (160, 8, 64, 0, [2, 1, 230, 1], [50, 70, 230, 1]),         # groups of 20: tiles of 32 for single tokens, beside them
    (128, 128, 64, 0, [20], [4500]),                           # keys past what the lanes hold pages for
    (128, 64, 64, 0, [450, 1, 12], [450, 900, 4200])])
def test_attention_of_many_rows(heads, kv_heads, d, window, q_lens, kv_lens):
    note(f"kv attention q={q_lens} kv={kv_lens} heads={heads}/{kv_heads} d={d} window={window}")
    rng = np.random.default_rng(heads + d)
    cache, blocks, k, v, _ = paged(rng, kv_lens, kv_heads, d, 16)
    q = torch.from_numpy(rng.standard_normal((sum(q_lens), heads, d))).to("cuda").to(BF)
    out = cache.attention(q, i32(np.concatenate([[0], np.cumsum(q_lens)])), i32(kv_lens), i32(blocks), max(q_lens), max(kv_lens), window=window)
    assert cache.status() == (E.ELIS_OK, 0)
    check_attention(out, q, q_lens, kv_lens, k, v, d ** -0.5, window)


@pytest.mark.parametrize("q_lens,room", [([40, 1], 40), ([0, 40, 3], 27), ([1, 40, 0, 12], 67)])
def test_attention_of_padded_rows(q_lens, room):
    """As many rows as if every request had max_q tokens, though some are shorter and the last rows are nobody's."""
    rng = np.random.default_rng(len(q_lens))
    T, kv_lens = sum(q_lens), [n + 20 for n in q_lens]
    note(f"kv attention padded q={q_lens} rows {T + room}")
    cache, blocks, k, v, _ = paged(rng, kv_lens, 2, 64, 16)
    for n in (len(q_lens) * 40, T + room):
        q = torch.from_numpy(rng.standard_normal((n, 4, 64))).to("cuda").to(BF)
        out = torch.full_like(q, 5.0)
        cache.attention(q, i32(np.concatenate([[0], np.cumsum(q_lens)])), i32(kv_lens), i32(blocks), 40, max(kv_lens), out=out)
        check_attention(out, q, q_lens, kv_lens, k, v, 64 ** -0.5)
        assert (host(out)[T:] == 5).all()


@pytest.mark.parametrize("q_lens,kv_lens", [([1], [9001]), ([1, 1, 3, 1], [9001, 20, 5300, 2000]), ([80, 1, 2], [7000, 9001, 1])])
@pytest.mark.parametrize("window", [1500, 5000, 9000, 2 ** 31 - 1])
def test_attention_of_long_windows(q_lens, kv_lens, window):
    rng = np.random.default_rng(window % 1000)
    note(f"kv attention q={q_lens} kv={kv_lens} window={window}")
    cache, blocks, k, v, _ = paged(rng, kv_lens, 1, 64, 32)
    q = torch.from_numpy(rng.standard_normal((sum(q_lens), 4, 64))).to("cuda").to(BF)
    out = cache.attention(q, i32(np.concatenate([[0], np.cumsum(q_lens)])), i32(kv_lens), i32(blocks), max(q_lens), max(kv_lens), window=window)
    check_attention(out, q, q_lens, kv_lens, k, v, 64 ** -0.5, window)


def test_attention_of_no_tokens_and_of_more_than_there_are_keys():
    rng = np.random.default_rng(6)
    cache, blocks, k, v, _ = paged(rng, [2, 5], 1, 64, 16)
    note("kv attention of no tokens")
    assert cache.attention(torch.empty((0, 2, 64), dtype=BF, device="cuda"), i32([0, 0, 0]), i32([2, 5]), i32(blocks), 1, 5).shape == (0, 2, 64)
    for window in (0, 1, 3, 2 ** 31 - 1):
        note(f"kv attention of more tokens than keys, window {window}")
        q = torch.from_numpy(rng.standard_normal((13, 2, 64))).to("cuda").to(BF)
        out = cache.attention(q, i32([0, 4, 13]), i32([2, 5]), i32(blocks), 9, 5, window=window)
        check_attention(out, q, [4, 9], [2, 5], k, v, 64 ** -0.5, window)


def test_attention_on_two_streams_and_in_two_graphs():
    """One cache, calls that split their keys: on two streams at once, and in two graphs replayed in turn with eager calls
    of other sizes between them."""
    rng = np.random.default_rng(12)
    kv = [9001, 4000, 5200]
    cache, blocks, k, v, _ = paged(rng, kv, 2, 64, 16)
    blocks, at = i32(blocks), np.concatenate([[0], np.cumsum(kv)])

    def check(out, q, which):
        pick = np.concatenate([np.arange(at[i], at[i + 1]) for i in which])
        check_attention(out, q, [1] * len(which), [kv[i] for i in which], k[pick], v[pick], 64 ** -0.5)

    sets = ([0], [1, 2], [2, 0, 1])
    q = [torch.from_numpy(rng.standard_normal((len(w), 4, 64))).to("cuda").to(BF) for w in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    note("kv attention on three streams")
    args = [(i32(np.arange(len(w) + 1)), i32([kv[i] for i in w]), blocks[w].contiguous(), 1, max(kv[i] for i in w)) for w in sets]
    torch.cuda.synchronize()
    outs = []
    for turn in range(5):
        for s, x, a in zip(streams, q, args):
            outs.append(cache.attention(x, *a, stream=s if turn % 2 else s.cuda_stream))
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        check(out, q[i % 3], sets[i % 3])
    note("kv attention in two graphs")
    graphs, held = [], [torch.zeros_like(x) for x in q[:2]]
    for x, a, o in zip(q, args, held):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cache.attention(x, *a, out=o)
        graphs.append(g)
    for replay in range(4):
        for x in q:
            x.copy_(torch.from_numpy(rng.standard_normal(tuple(x.shape))).to("cuda"))
        for o in held:
            o.fill_(9)
        graphs[replay % 2].replay()
        eager = cache.attention(q[2], *args[2])
        graphs[1 - replay % 2].replay()
        torch.cuda.synchronize()
        for o, x, w in zip((*held, eager), q, sets):
            check(o, x, w)


@pytest.mark.parametrize("heads,kv_heads,q_lens,kv_lens,window", [
    (128, 128, [200], [450], 0), (128, 128, [200], [450], 70),       # tiles of 64 rows, alone
    (64, 64, [448, 1], [1000, 300], 0), (64, 64, [448, 1], [1000, 300], 129),  # beside a single token
    (160, 8, [158, 1, 1], [400, 50, 70], 0),                          # beside single tokens of 20 rows
    (128, 128, [230], [4700], 0)])                                    # keys past what the lanes hold pages for
def test_attention_in_tall_tiles(heads, kv_heads, q_lens, kv_lens, window):
    """Few enough tiles of 64 rows for one fill of the machine, too many of 32."""
    note(f"kv attention q={q_lens} kv={kv_lens} heads={heads}/{kv_heads} window={window}")
    rng = np.random.default_rng(heads + len(q_lens))
    cache, blocks, k, v, _ = paged(rng, kv_lens, kv_heads, 128, 16)
    T = sum(q_lens)
    q = torch.from_numpy(rng.standard_normal((T + 1, heads, 128))).to("cuda").to(BF)
    out = torch.full_like(q, 5.0)
    cu = i32(np.concatenate([[0], np.cumsum(q_lens)]))
    for rows in (T, T + 1):
        cache.attention(q[:rows], cu, i32(kv_lens), i32(blocks), max(q_lens), max(kv_lens), window=window, out=out[:rows])
        assert cache.status() == (E.ELIS_OK, 0)
        few = [0, 5, kv_heads - 1] if heads == kv_heads else range(kv_heads)  # the oracle takes a minute for all of 128
        qh = [h * heads // kv_heads + i for h in few for i in range(heads // kv_heads)]
        check_attention(out[:, qh], q[:, qh], q_lens, kv_lens, k[:, list(few)], v[:, list(few)], 128 ** -0.5, window)
        assert (host(out)[T:] == 5).all() and np.isfinite(host(out)).all()


@pytest.mark.parametrize("longest", [1, 40])
@pytest.mark.parametrize("window", [0, 9])
def test_attention_of_many_requests(longest, window):
    """More requests than a work-group has threads, some of them empty, with lengths in no order."""
    rng = np.random.default_rng(longest)
    n = 700
    q_lens = rng.integers(0, longest + 1, n)
    kv_lens = (q_lens + rng.integers(0, 30, n)).tolist()
    q_lens[[0, 300, n - 1]], kv_lens[5] = [0, longest, longest], 2000
    kv_lens = np.maximum(kv_lens, q_lens).tolist()
    note(f"kv attention of {n} requests of up to {longest} tokens, window {window}")
    cache, blocks, k, v, _ = paged(rng, kv_lens, 1, 64, 16)
    q = torch.from_numpy(rng.standard_normal((int(q_lens.sum()), 2, 64))).to("cuda").to(BF)
    out = cache.attention(q, i32(np.concatenate([[0], np.cumsum(q_lens)])), i32(kv_lens), i32(blocks), longest, max(kv_lens), window=window)
    assert cache.status() == (E.ELIS_OK, 0)
    check_attention(out, q, q_lens.tolist(), kv_lens, k, v, 64 ** -0.5, window)


def test_wrappers_refuse_what_does_not_fit():
    """Tensors of another device, type, shape or layout never reach a kernel."""
    note("refusals of the wrappers")
    pool, cache = PagePool(8, 16, 4, 3), KVCache(8, 16, 2, 64)
    s, cu, m = i32([0, 1]), i32([0, 3, 5]), i32([0] * 5)
    kv, q = torch.zeros((5, 2, 64), dtype=BF, device="cuda"), torch.zeros((5, 4, 64), dtype=BF, device="cuda")
    lens, blocks = i32([3, 2]), i32([[0], [1]])
    x, ids = torch.zeros((2, 50), dtype=torch.float32, device="cuda"), i32([1, 2, 3, 4, 5])
    calls = [
        lambda: pool.grow(s.cpu(), lens, cu, 5, m), lambda: pool.grow(s.long(), lens, cu, 5, m), lambda: pool.grow(s, lens[:1], cu, 5, m),
        lambda: pool.grow(s, lens, cu[:2], 5, m), lambda: pool.grow(s, lens, cu, 6, m), lambda: pool.grow(s, lens, cu, 5, m, out_blocks=blocks[:1]),
        lambda: pool.grow(s, lens, cu, 5, i32([[0, 0]] * 5)[:, 0]), lambda: pool.grow(i32([0, 1, 2, 3, 0]), i32([1] * 5), i32(range(6)), 5, m),
        lambda: pool.grow(s, lens, None, 5, m), lambda: pool.grow(s, lens, cu, 5, m, out_blocks=i32([[0] * 4] * 2)),
        lambda: pool.trim(s, lens.cpu()), lambda: pool.trim(s, lens[:1]),
        lambda: cache.append(kv.float(), kv, m), lambda: cache.append(kv[:4], kv, m), lambda: cache.append(kv, kv.cpu(), m),
        lambda: cache.append(kv[:, :1], kv, m), lambda: cache.append(kv.transpose(1, 2).contiguous().transpose(1, 2), kv, m),
        lambda: cache.append(kv[:1].expand(5, 2, 64), kv, m), lambda: cache.append(kv, kv, m.long()), lambda: cache.read(m, kv, kv.half()),
        lambda: cache.attention(q.half(), cu, lens, blocks, 3, 3), lambda: cache.attention(q[:, :3], cu, lens, blocks, 3, 3),
        lambda: cache.attention(q, cu[:2], lens, blocks, 3, 3), lambda: cache.attention(q, cu, lens, blocks[0], 3, 3),
        lambda: cache.attention(q, cu, lens, blocks.cpu(), 3, 3), lambda: cache.attention(q, cu, lens, blocks, 3, 17),
        lambda: cache.attention(q, cu, lens, blocks[:1], 3, 3), lambda: cache.attention(q, cu, lens, blocks, 3, 3, rows=s[:1]),
        lambda: cache.attention(q, cu, lens, blocks, 3, 3, out=q[:3]), lambda: cache.attention(q, cu, lens, blocks, 3, 3, scale=-1.0),
        lambda: cache.attention(q, cu, lens, blocks, 0, 3), lambda: cache.attention(q, cu, lens, i32([[0, 9], [1, 9]])[:, :1], 3, 3),
        lambda: adjust_logits(x.cpu(), ids, cu), lambda: adjust_logits(x.half(), ids, cu), lambda: adjust_logits(x.t(), ids, cu),
        lambda: adjust_logits(x, ids, cu[:2]), lambda: adjust_logits(x, ids.cpu(), cu), lambda: adjust_logits(x, ids, cu, prompt_lens=lens[:1]),
        lambda: adjust_logits(x, ids, None), lambda: adjust_logits(x, ids, cu, repetition=dev(np.ones(1, np.float32))),
        lambda: adjust_logits(x, ids, cu, frequency=torch.ones(2, dtype=torch.float64, device="cuda")),
        lambda: adjust_logits(x, ids, cu, bias=(cu, ids, dev(np.ones(4, np.float32)))), lambda: adjust_logits(x, ids, cu, mask=i32([[1]])),
        lambda: adjust_logits(x, ids, cu, mask=i32([[1, 1]])), lambda: adjust_logits(x, ids, cu, mask=i32([[1, 1]]), mask_rows=s[:1]),
        lambda: adjust_logits(x, ids, cu, out=x[:1]), lambda: adjust_logits(x[:1].expand(2, 50), ids, cu), lambda: adjust_logits(x.bfloat16(), ids, cu, out=x.bfloat16()),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(E.ElisError):
            call()
            pytest.fail(f"call {i} was served")
    assert pool.status() == (E.ELIS_OK, 0) and cache.status() == (E.ELIS_OK, 0) and int(pool.held.sum()) == 0


@pytest.mark.parametrize("heads,kv_heads,d", [(8, 8, 128), (40, 2, 128), (12, 12, 64), (20, 1, 64)])
@pytest.mark.parametrize("q_lens", [[1] * 6, [1, 60, 1, 0, 2, 1]])
def test_attention_of_batches_that_may_be_long(heads, kv_heads, d, q_lens):
    """Bounds on the lengths by which the batch may hold more than the caches."""
    rng = np.random.default_rng(d + heads)
    kv_lens = [700, 130, 1, 64, 300, 2500]
    width = -(-420_000_000 // (6 * kv_heads * 17 * d // 16 * 128))
    note(f"kv attention q={q_lens} heads={heads}/{kv_heads} d={d} of up to {width * 128} keys")
    cache, blocks, k, v, _ = paged(rng, kv_lens, kv_heads, d, 128)
    table = np.full((6, width), -1)
    table[:, :blocks.shape[1]] = blocks
    q = torch.from_numpy(rng.standard_normal((sum(q_lens), heads, d))).to("cuda").to(BF)
    out = cache.attention(q, i32(np.concatenate([[0], np.cumsum(q_lens)])), i32(kv_lens), i32(table), max(q_lens), width * 128)
    assert cache.status() == (E.ELIS_OK, 0)
    check_attention(out, q, q_lens, kv_lens, k, v, d ** -0.5)


def test_cache_past_four_gib():
    """Records whose places pass 32 bits: append, read and attention on the last pages of a large cache."""
    rng = np.random.default_rng(4)
    d, heads, page, kv = 128, 16, 64, 150
    n_pages = 5 * 2 ** 30 // (heads * page // 16 * 17 * d) + 1
    note(f"kv cache of {n_pages} pages, {E.elis_kv_cache_bytes(n_pages, page, heads, d) / 2 ** 30:.1f} GiB")
    cache = KVCache(n_pages, page, heads, d)
    blocks = np.array([[n_pages - 1, 3, n_pages - 2]])
    slots = i32(blocks[0, np.arange(kv) // page] * page + np.arange(kv) % page)
    k, v = (torch.from_numpy(rng.standard_normal((kv, heads, d))).to("cuda").to(BF) for _ in range(2))
    cache.append(k, v, slots)
    rk, rv = torch.empty_like(k), torch.empty_like(v)
    cache.read(slots, rk, rv)
    assert np.array_equal(host(rk)[[0, 70, 149]], O.kv_round(host(k)[[0, 70, 149]])) and np.array_equal(host(rv)[[63, 64]], O.kv_round(host(v)[[63, 64]]))
    for n in (1, 40):
        q = torch.from_numpy(rng.standard_normal((n, heads, d))).to("cuda").to(BF)
        out = cache.attention(q, i32([0, n]), i32([kv]), i32(blocks), n, kv)
        check_attention(out, q, [n], [kv], host(rk), host(rv), d ** -0.5)


@pytest.mark.parametrize("q_len", [1, 40, 300])
def test_attention_masked_pages_and_nan(q_len):
    """Keys on bad pages are not seen; NaN in a key or a value reaches the rows that see it, and no other."""
    rng = np.random.default_rng(3)
    d, page, kv, heads = 128, 16, 420, 4
    for bad_key, bad_value in ((None, None), (350, None), (None, 200), (None, 419)):
        cache, blocks, k, v, slots = paged(rng, [kv], 2, d, page)
        note(f"kv attention q_len={q_len} NaN key {bad_key} value {bad_value}")
        T = 1
        for at, which in ((bad_key, 0), (bad_value, 1)):
            if at is not None:
                pair = [torch.from_numpy(x[at:at + 1]).to("cuda").to(BF) for x in (k, v)]
                pair[which][0, 1, 70] = float("nan")
                cache.append(*pair, slots[at:at + 1])
        q = torch.from_numpy(rng.standard_normal((q_len, heads, d))).to("cuda").to(BF)
        out = cache.attention(q, i32([0, q_len]), i32([kv]), i32(blocks), q_len, kv)
        got = host(out)
        pos = np.arange(kv - q_len, kv)
        nan = np.zeros(got.shape, bool)
        if bad_key is not None:
            nan[pos >= bad_key, 2:] = True                     # every value of the rows that see the key
        if bad_value is not None:
            nan[np.ix_(pos >= bad_value, [2, 3], range(64, 96))] = True  # the 32 columns of its scale
        assert np.array_equal(np.isnan(got), nan)
        want = O.kv_attention(host(q), k, v, kv, d ** -0.5)
        size = O.kv_attention(host(q), k, np.abs(v), kv, d ** -0.5)
        assert (np.abs(got - want) <= 3 * 2.0 ** -8 * 1.01 * size)[~nan].all()
        del T
    note(f"kv attention q_len={q_len} bad pages")
    cache, blocks, k, v, _ = paged(rng, [kv], 2, d, page)
    seen = np.ones(kv, bool)
    for b, bad in ((2, -1), (7, 1 << 20), (26, -5)):
        blocks[0, b] = bad
        seen[b * page:(b + 1) * page] = False
    out = cache.attention(q, i32([0, q_len]), i32([kv]), i32(blocks), q_len, kv)
    assert cache.status() == (E.ELIS_EDEVICE, E.ELIS_DEV_BAD_PAGE)
    check_attention(out, q, [q_len], [kv], k, v, d ** -0.5, seen=[seen])


def test_attention_content_errors():
    rng = np.random.default_rng(5)
    cache, blocks, k, v, _ = paged(rng, [50, 60, 70], 1, 64, 16)
    q = torch.from_numpy(rng.standard_normal((6, 2, 64))).to("cuda").to(BF)
    for cu, lens, rows, bit in (([0, 2, 9, 6], [50, 60, 70], None, E.ELIS_DEV_BAD_CU), ([0, 2, 1, 3], [50, 60, 70], None, E.ELIS_DEV_BAD_CU),
                                ([0, 1, 6, 6], [50, 60, 70], None, E.ELIS_DEV_LONG_SEQ), ([0, 2, 4, 6], [50, 71, 70], None, E.ELIS_DEV_LONG_SEQ),
                                ([0, 2, 4, 6], [50, -1, 70], None, E.ELIS_DEV_LONG_SEQ), ([0, 2, 4, 6], [50, 60, 70], [0, 3, 2], E.ELIS_DEV_BAD_PAGE),
                                ([0, 2, 4, 6], [50, 60, 70], [0, -1, 2], E.ELIS_DEV_BAD_PAGE)):
        note(f"kv attention content error cu={cu} lens={lens} rows={rows}")
        E.check(E.elis_kv_init(cache.c, None))
        out = cache.attention(q, i32(cu), i32(lens), i32(blocks), 4, 70, rows=None if rows is None else i32(rows))
        assert cache.status() == (E.ELIS_EDEVICE, bit)
        # the other requests are served: request 0 owns the rows that no other range names ([0, 2, 1, 3] gives row 1 to
        # request 2 as well, which may write it first or last), at their place in its two or one queries
        m = min(cu[1], cu[2])
        want = O.kv_attention(host(q)[:cu[1]], k[:50], v[:50], 50, 64 ** -0.5)[:m]
        size = O.kv_attention(host(q)[:cu[1]], k[:50], np.abs(v[:50]), 50, 64 ** -0.5)[:m]
        assert (np.abs(host(out)[:m] - want) <= 3 * 2.0 ** -8 * 1.01 * size).all()


def test_attention_scores_far_apart():
    """A running maximum that climbs with the keys, weights that vanish, and scores near the top of the range."""
    rng = np.random.default_rng(9)
    d, kv = 64, 700
    cache, blocks, k, v, slots = paged(rng, [kv], 1, d, 16)
    for spread in (1.0, 40.0, 3000.0):
        ramp = (np.linspace(-1, 1, kv) * spread)[:, None, None] * np.sign(rng.standard_normal((1, 1, d)))
        kk = torch.from_numpy(ramp).to("cuda").to(BF)
        cache.append(kk, torch.from_numpy(v).to("cuda").to(BF), slots)
        rk, rv = torch.empty_like(kk), torch.empty_like(kk)
        cache.read(slots, rk, rv)
        q = torch.from_numpy(np.sign(host(kk)[-1:]).repeat(3, 0)).to("cuda").to(BF)
        q[1] = -q[1]
        note(f"kv attention spread {spread}")
        for n in (1, 3):
            out = cache.attention(q[:n], i32([0, n]), i32([kv]), i32(blocks), n, kv)
            check_attention(out, q[:n], [n], [kv], host(rk), host(rv), d ** -0.5)


# ------------------------------------------------------------------ logits

@pytest.mark.parametrize("dtype", [torch.float32, BF])
@pytest.mark.parametrize("n,vocab,hist,pad", [(1, 1, 3, 0), (2, 31, 0, 0), (3, 33, 40, 1), (2, 8192, 100, 0), (3, 8195, 900, 3), (2, 30522, 3000, 2), (4, 16389, 17, 0)])
def test_logits(n, vocab, hist, pad, dtype):
    rng = np.random.default_rng(vocab + n)
    note(f"logits n={n} vocab={vocab} hist={hist} pad={pad} {dtype}")
    wide = torch.from_numpy(rng.standard_normal((n, vocab + pad)) * 4).to("cuda").to(dtype)
    x = wide[:, pad:]
    x[0, 0] = -np.inf
    lens = rng.integers(0, hist + 1, n)
    ids = rng.integers(-1, min(vocab, 50) + 1, int(lens.sum()) + 3)
    ids[rng.random(len(ids)) < 0.5] = vocab - 1
    cu = np.concatenate([[0], np.cumsum(lens)])
    prompt = rng.integers(0, hist + 2, n)
    rep, freq, pres = rng.uniform(0.5, 2, n), rng.uniform(-1, 1, n), rng.uniform(-1, 1, n)
    b_lens = rng.integers(0, 9, n)
    b_tok = rng.integers(-1, vocab + 1, int(b_lens.sum()))
    b_tok[rng.random(len(b_tok)) < 0.5] = min(7, vocab - 1)
    b_val = rng.standard_normal(len(b_tok)).astype(np.float32)
    b_cu = np.concatenate([[0], np.cumsum(b_lens)])
    words = (vocab + 31) // 32 + 1
    mask = rng.integers(0, 2 ** 32, (3, words), dtype=np.uint32)
    mask[1] = 0
    rows = rng.integers(-1, 4, n)
    f32 = lambda a: dev(np.asarray(a, np.float32))  # noqa: E731
    bias = (i32(b_cu), i32(b_tok), f32(b_val)) if len(b_tok) else None
    full = torch.full((n + 1, vocab + 3), 77.0, dtype=torch.float32, device="cuda")
    out = full[:n, 3:]
    for use_mask, use_rest in ((True, True), (False, True), (False, False)):
        kw = dict(repetition=f32(rep), frequency=f32(freq), presence=f32(pres), bias=bias, prompt_lens=i32(prompt)) if use_rest else {}
        if use_mask:
            kw |= dict(mask=dev(mask.view(np.int32)), mask_rows=i32(rows))
        tokens = (i32(ids), i32(cu)) if use_rest else (None, None)
        adjust_logits(x, *tokens, out=out, **kw)
        got = host(out)
        for i in range(n):
            h = ids[cu[i]:cu[i + 1]].tolist() if use_rest else []
            bl = list(zip(b_tok[b_cu[i]:b_cu[i + 1]].tolist(), b_val[b_cu[i]:b_cu[i + 1]].tolist())) if use_rest else []
            allowed = None
            if use_mask and 0 <= rows[i] < 3:
                allowed = (mask[rows[i]][np.arange(vocab) // 32] >> (np.arange(vocab) % 32)) & 1 == 1
            r, f, p = np.float32([rep[i], freq[i], pres[i]]).astype(np.float64) if use_rest else (1, 0, 0)
            xi = host(x)[i]
            want = O.logits_adjust(xi, h, int(prompt[i]), r, f, p, bl, allowed)
            assert np.array_equal(np.isneginf(got[i]), np.isneginf(want))
            fin = np.isfinite(want)
            size = np.abs(np.where(fin, xi, 0)) * max(r, 1 / r) + abs(f) * len(h) + abs(p) + sum(abs(b) for _, b in bl)
            assert (np.abs(got[i] - want)[fin] <= ((5 + len(bl)) * 2.0 ** -24 * size)[fin]).all()
        assert (host(full)[n] == 77).all() and (host(full)[:, :3] == 77).all()
    if dtype == torch.float32:
        y = x.clone()
        adjust_logits(x, i32(ids), i32(cu), out=full[:n, 3:], **kw)
        adjust_logits(y, i32(ids), i32(cu), out=y, **kw)
        assert torch.equal(y, full[:n, 3:])


def test_logits_of_crowded_rows():
    """One token over and over, as many biases as tokens and every one twice, prompts as long as the history, no mask bit set."""
    rng = np.random.default_rng(8)
    n, vocab = 3, 5000
    x = torch.from_numpy(rng.standard_normal((n, vocab)).astype(np.float32)).cuda()
    ids = np.concatenate([np.full(20000, 4321), rng.integers(0, vocab, 3000), [7]])
    cu = np.array([0, 20000, 23000, 23001])
    tok = np.concatenate([rng.permutation(vocab)] * 2)
    val = rng.standard_normal(len(tok)).astype(np.float32)
    note("logits: crowded rows")
    out = adjust_logits(x, i32(ids), i32(cu), prompt_lens=i32([5, 3000, 9]), frequency=dev(np.full(n, 0.01, np.float32)),
                        presence=dev(np.full(n, 0.5, np.float32)), repetition=dev(np.full(n, 2.0, np.float32)),
                        bias=(i32([0, 2 * vocab, 2 * vocab, 2 * vocab]), i32(tok), dev(val)),
                        mask=dev(np.zeros((1, 157), np.int32)), mask_rows=i32([-1, -1, 0]))
    total = np.zeros(vocab)
    np.add.at(total, tok, val.astype(np.float64))
    for i, (h, p) in enumerate(((ids[:20000], 5), (ids[20000:23000], 3000), (ids[23000:], 9))):
        f = float(np.float32(0.01))
        y = O.logits_adjust(host(x)[i], h.tolist()[:p] + h.tolist()[p:p + 1], p, 2.0, f, 0.5, [], None)
        count = max(0, len(h) - p)
        if i == 0:
            y[4321] -= f * (count - 1)       # the oracle has seen it once
            y += total
        if i == 2:
            y[:] = -np.inf
        got = host(out)[i]
        assert np.array_equal(np.isneginf(got), np.isneginf(y))
        size = np.abs(host(x)[i]) * 2 + f * count + 0.5 + (np.abs(val).max() * 2 if i == 0 else 0)
        fin = np.isfinite(y)
        assert (np.abs(got[fin] - y[fin]) <= 7 * 2.0 ** -24 * size[fin]).all()


# ------------------------------------------------------------------ together

def decode(heads=4, kv_heads=2, d=64, page=16, vocab=500, steps=20):
    """Eight jobs of a job table: each step selects five by predicted length, gives them pages, keeps their keys and
    values, attends, adjusts the logits and appends the best token. Returns what each job wrote, and the device's log."""
    rng = np.random.default_rng(11)
    J, max_pos = 8, 512
    table = JobTable(J, max_pos)
    pool = PagePool(60, page, J, 8)
    cache = KVCache(60, page, kv_heads, d)
    emb = torch.from_numpy(rng.standard_normal((vocab, (heads + 2 * kv_heads) * d))).to("cuda").to(BF)
    head = torch.from_numpy(rng.standard_normal((heads * d, vocab)) * 0.3).to("cuda").to(BF)
    slots = np.arange(J, dtype=np.int32)
    table.start(i32(slots), dev(np.arange(J, dtype=np.int64)))
    tokens = [rng.integers(0, vocab, int(m)).tolist() for m in rng.integers(1, 40, J)]
    prompt = np.array([len(t) for t in tokens])
    table.append(i32(slots), i32(np.concatenate([[0], np.cumsum(prompt)])), i32(np.concatenate(tokens)), int(prompt.sum()))
    cached = np.zeros(J, np.int64)
    log = []
    for step in range(steps):
        pred = rng.uniform(0, 100, J).astype(np.float32)
        table.store_pred(i32(slots), dev(pred))
        chosen = torch.zeros(5, dtype=torch.int32, device="cuda")
        table.select(i32(slots), 5, chosen, torch.zeros(1, dtype=torch.int32, device="cuda"))
        picked = oracle_select(pred, np.arange(J), 5)
        lens = np.array([len(tokens[j]) for j in picked])
        new = lens - cached[picked]                       # the whole prompt at first, then one token
        cu = np.concatenate([[0], np.cumsum(new)])
        total = int(cu[-1])
        note(f"decode step {step}: jobs {picked.tolist()}, {total} new tokens")
        slot_map = torch.empty(total, dtype=torch.int32, device="cuda")
        pool.grow(chosen, i32(lens), i32(cu), total, slot_map)
        ids = np.concatenate([tokens[j][cached[j]:] for j in picked])
        qkv = emb[torch.from_numpy(ids).to("cuda")]
        q, kv = qkv[:, :heads * d].unflatten(1, (heads, d)), qkv[:, heads * d:].unflatten(1, (2 * kv_heads, d))
        cache.append(kv[:, :kv_heads], kv[:, kv_heads:], slot_map)
        o = cache.attention(q, i32(cu), i32(lens), pool.table, int(new.max()), int(lens.max()), rows=chosen)
        last = o[torch.from_numpy(cu[1:] - 1).to("cuda")].flatten(1)
        logits = (last.float() @ head.float())
        packed, pcu = torch.empty(int(lens.sum()), dtype=torch.int32, device="cuda"), torch.empty(6, dtype=torch.int32, device="cuda")
        table.pack(chosen, int(lens.sum()), int(lens.max()), packed, pcu)
        out = adjust_logits(logits, packed, pcu, prompt_lens=i32(prompt[picked]), repetition=dev(np.full(5, 1.2, np.float32)),
                            frequency=dev(np.full(5, 0.3, np.float32)))
        best = out.argmax(1)
        table.append(chosen, i32(np.arange(6)), best.to(torch.int32), 5)
        log.append((picked, cu, lens, host(q), host(o), host(logits), host(out), [list(tokens[j]) for j in picked]))
        for j, t in zip(picked, best.tolist()):
            cached[j] = len(tokens[j])
            tokens[j].append(t)
        assert int(pool.state[1]) == 60 - sum(-(-c // page) for c in cached.tolist())
    assert pool.status() == (E.ELIS_OK, 0) and cache.status() == (E.ELIS_OK, 0) and table.status() == (E.ELIS_OK, 0)
    return log, emb, prompt


def test_decode_loop_over_the_job_table():
    heads, kv_heads, d = 4, 2, 64
    log, emb, prompt = decode(heads, kv_heads, d)
    rounded = O.kv_round(host(emb)[:, heads * d:]).reshape(-1, 2 * kv_heads, d)
    for picked, cu, lens, q, o, logits, out, tokens in log:
        for i, j in enumerate(picked):
            kv = rounded[tokens[i]]
            a, b = int(cu[i]), int(cu[i + 1])
            want = O.kv_attention(q[a:b], kv[:, :kv_heads], kv[:, kv_heads:], int(lens[i]), d ** -0.5)
            size = O.kv_attention(q[a:b], kv[:, :kv_heads], np.abs(kv[:, kv_heads:]), int(lens[i]), d ** -0.5)
            assert (np.abs(o[a:b] - want) <= 3 * 2.0 ** -8 * 1.01 * size).all()
            y = O.logits_adjust(logits[i], tokens[i], int(prompt[j]), float(np.float32(1.2)), float(np.float32(0.3)))
            assert (np.abs(out[i] - y) <= 8 * 2.0 ** -24 * (np.abs(logits[i]) * 1.2 + 0.3 * len(tokens[i]))).all()


@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1, 1], [600, 33, 5000]), ([60, 1, 1], [100, 33, 5000])])
def test_captured_step(q_lens, kv_lens):
    """A captured step (pages, append, attention, logits, pages back) replays with the program's own work in between,
    for contents and lengths that change under it, on a stream that is not the default one."""
    rng = np.random.default_rng(1)
    n, heads, kv_heads, d, page, vocab = len(q_lens), 8, 2, 128, 16, 3000
    pool, cache = PagePool(500, page, n + 2, 400), KVCache(500, page, kv_heads, d)
    slots = i32([3, 0, 2])
    before = np.array(kv_lens) - np.array(q_lens)
    pool.grow(slots, i32(before), None, 0, None)
    T = sum(q_lens)
    fill = torch.empty(int(before.sum()), dtype=torch.int32, device="cuda")
    pool.grow(slots, i32(before), i32(np.concatenate([[0], np.cumsum(before)])), int(before.sum()), fill)
    hist = [torch.from_numpy(rng.standard_normal((int(before.sum()), kv_heads, d))).to("cuda").to(BF) for _ in range(2)]
    cache.append(*hist, fill)
    lens, old, cu = i32(kv_lens), i32(before), i32(np.concatenate([[0], np.cumsum(q_lens)]))
    smap = torch.zeros(T, dtype=torch.int32, device="cuda")
    blocks = torch.zeros((n, 400), dtype=torch.int32, device="cuda")
    q, k, v = (torch.zeros((T, h, d), dtype=BF, device="cuda") for h in (heads, kv_heads, kv_heads))
    logits, ids, hcu = torch.zeros((n, vocab), dtype=torch.float32, device="cuda"), i32(rng.integers(0, vocab, 90)), i32([0, 10, 50, 90])
    o, y = torch.zeros_like(q), torch.zeros_like(logits)
    rep = dev(np.full(n, 1.3, np.float32))
    stream = torch.cuda.Stream()

    def step(o, y):
        pool.grow(slots, lens, cu, T, smap, out_blocks=blocks)
        cache.append(k, v, smap)
        cache.attention(q, cu, lens, blocks, max(q_lens), 6000, out=o)
        adjust_logits(logits, ids, hcu, out=y, repetition=rep)
        pool.trim(slots, old)

    note("capture of a step")
    with torch.cuda.stream(stream):
        step(o, y)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(o, y)
    for replay in range(4):
        for t in (q, k, v, logits):
            t.copy_(torch.from_numpy(rng.standard_normal(tuple(t.shape))).to("cuda"))
        lens.copy_(i32(np.array(kv_lens) + [0, 0, -replay]))   # a shorter history under the same graph
        old.copy_(i32(before + [0, 0, -replay]))
        o.fill_(9)
        note(f"replay {replay}")
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = (o.clone(), y.clone(), smap.clone(), blocks.clone(), pool.state.clone())
        torch.mm(*(torch.randn((512, 512), dtype=torch.float32, device="cuda") for _ in range(2))).sum().item()
        o2, y2 = torch.zeros_like(o), torch.zeros_like(y)
        step(o2, y2)
        torch.cuda.synchronize()
        for a, b in zip(got, (o2, y2, smap, blocks, pool.state)):
            assert torch.equal(a, b)
    assert cache.status() == (E.ELIS_OK, 0) and pool.status() == (E.ELIS_OK, 0)

"""The batch operators' oracle against hand-computed values, and the library's refusals (no kernel is launched here)."""
import numpy as np
import pytest

from oracle import batch as O
from paper_2505_09142_amd import _elis as E

FAKE, FAKE_WS, NAN, INF = 0x1000, 0x100000, float("nan"), float("inf")


def test_kv_round_by_hand():
    x = np.zeros(32)
    x[:12] = [6.0, 0.24, 0.25, 0.26, 0.75, -1.25, 1.75, 2.5, -3.5, 5.0, 5.1, -0.1]  # scale 1: 6 < 7
    assert O.kv_round(x)[:12].tolist() == [6.0, 0.0, 0.0, 0.5, 1.0, -1.0, 2.0, 2.0, -4.0, 4.0, 6.0, 0.0]
    x[0] = 6.99                                                   # still scale 1, saturates
    assert O.kv_round(x)[0] == 6.0 and O.kv_round(x)[3] == 0.5
    x[0] = 7.0                                                    # scale 2: 3.5 is a tie, to 4
    assert O.kv_round(x)[0] == 8.0 and O.kv_round(x)[9] == 4.0    # 5 / 2 = 2.5, to 2
    assert np.isnan(O.kv_round(np.where(np.arange(64) == 40, INF, 1.0))[32:]).all()
    assert O.kv_round(np.where(np.arange(64) == 40, NAN, 1.0))[:32].tolist() == [1.0] * 32
    assert (O.kv_round(O.kv_round(x)) == O.kv_round(x)).all()


def test_pages_by_hand():
    p = O.Pages(6, 16, 4, 4)
    blocks, maps = p.grow([2, 0], [17, 16], [17, 2])
    assert blocks == [[0, 1], [2]] and maps[0][15:] == [15, 16] and maps[1] == [46, 47]
    blocks, maps = p.grow([2, 1, 3], [64, 33, 1], [1, 1, 1])      # two pages for slot 2, one left: slot 1 and 3 go without
    assert blocks == [[0, 1, 3, 4], [], []] and maps == [[4 * 16 + 15], [-1], [-1]] and p.short
    p.trim([2, 0], [17, 0])
    assert p.free == [5, 2, 4, 3] and p.held[2] == [0, 1] and p.held[0] == []


def test_attention_and_logits_by_hand():
    k = np.array([[[0.0]], [[np.log(3.0)]], [[9.0]]])
    v = np.array([[[4.0]], [[8.0]], [[1.0]]])
    q = np.ones((2, 1, 1))
    out = O.kv_attention(q, k, v, 2, 1.0)
    assert out[:, 0, 0].tolist() == [4.0, pytest.approx(7.0)]
    assert O.kv_attention(q, k, v, 2, 1.0, window=1)[1, 0, 0] == 8.0
    assert O.kv_attention(q, k, v, 1, 1.0)[:, 0, 0].tolist() == [0.0, 4.0]      # a query before the first key
    assert O.kv_attention(q, k, v, 2, 1.0, seen=[False, True])[:, 0, 0].tolist() == [0.0, 8.0]
    y = O.logits_adjust([2.0, -2.0, 1.0, 5.0, 5.0], [0, 1, 1, 1, 7, -1], 2, 2.0, 0.5, 0.25, [(3, 1.0), (3, -2.0)], np.array([1, 1, 1, 1, 0], bool))
    assert y.tolist() == [1.0, -4.0 - 1.0 - 0.25, 1.0, 4.0, -INF]


def pool(**kw):
    a = dict(state=FAKE, free_pages=FAKE, held=FAKE, table=FAKE, scratch=FAKE, n_pages=8, page_tokens=16, max_jobs=4, max_pages=2) | kw
    return E.elis_page_pool(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(state=None), E.ELIS_EINVAL), (dict(free_pages=None), E.ELIS_EINVAL), (dict(held=None), E.ELIS_EINVAL),
    (dict(table=None), E.ELIS_EINVAL), (dict(scratch=None), E.ELIS_EINVAL), (dict(n_pages=0), E.ELIS_EINVAL),
    (dict(max_jobs=0), E.ELIS_EINVAL), (dict(max_pages=-1), E.ELIS_EINVAL), (dict(page_tokens=8), E.ELIS_EUNSUPPORTED),
    (dict(page_tokens=48), E.ELIS_EUNSUPPORTED), (dict(page_tokens=2048), E.ELIS_EUNSUPPORTED),
    (dict(n_pages=1 << 27), E.ELIS_EUNSUPPORTED), (dict(max_jobs=1 << 20, max_pages=1 << 12), E.ELIS_EUNSUPPORTED)])
def test_pool_refusals(kw, status):
    p = pool(**kw)
    assert E.elis_pages_init(p, None) == status
    assert E.elis_pages_grow(p, FAKE, FAKE, FAKE, 1, 1, 1, FAKE, FAKE, None) == status
    assert E.elis_pages_trim(p, FAKE, FAKE, 1, None) == status


def test_pages_call_refusals():
    p = pool()
    grow = lambda s=FAKE, l=FAKE, c=FAKE, n=2, t=3, w=2, b=FAKE, m=FAKE: E.elis_pages_grow(p, s, l, c, n, t, w, b, m, None)  # noqa: E731
    assert E.elis_pages_init(None, None) == E.ELIS_EINVAL
    assert grow(n=0) == E.ELIS_OK and E.elis_pages_trim(p, None, None, 0, None) == E.ELIS_OK
    assert grow(s=None) == E.ELIS_EINVAL and grow(l=None) == E.ELIS_EINVAL and grow(c=None) == E.ELIS_EINVAL
    assert grow(n=-1) == E.ELIS_EINVAL and grow(t=-1) == E.ELIS_EINVAL and grow(w=-1) == E.ELIS_EINVAL
    assert grow(n=5) == E.ELIS_ESHAPE and grow(w=3) == E.ELIS_ESHAPE
    assert E.elis_pages_trim(p, FAKE, None, 1, None) == E.ELIS_EINVAL
    assert E.elis_pages_trim(p, FAKE, FAKE, 5, None) == E.ELIS_ESHAPE


def test_cache_refusals():
    assert E.elis_kv_cache_bytes(3, 32, 2, 128) == 256 + 3 * 2 * 2 * 17 * 128
    for bad in ((0, 16, 1, 64), (1, 16, 0, 64), (1, 24, 1, 64), (1, 16, 1, 96), (1, 16, 1025, 64), (1 << 27, 16, 1, 64)):
        assert E.elis_kv_cache_bytes(*bad) == 0
    good = E.elis_kv_cache(FAKE_WS, 4, 16, 2, 64)
    for c, st in ((None, E.ELIS_EINVAL), (E.elis_kv_cache(None, 4, 16, 2, 64), E.ELIS_EINVAL), (E.elis_kv_cache(FAKE_WS + 16, 4, 16, 2, 64), E.ELIS_EINVAL),
                  (E.elis_kv_cache(FAKE_WS, 4, 16, 2, 32), E.ELIS_EUNSUPPORTED), (E.elis_kv_cache(FAKE_WS, 4, 20, 2, 64), E.ELIS_EUNSUPPORTED)):
        assert E.elis_kv_init(c, None) == st
        assert E.elis_kv_append(c, FAKE, FAKE, 128, 128, FAKE, 1, None) == st
        assert E.elis_kv_read(c, FAKE, 1, FAKE, FAKE, 128, 128, None) == st
    for f in (lambda k=FAKE, v=FAKE, ks=128, vs=128, m=FAKE, n=1: E.elis_kv_append(good, k, v, ks, vs, m, n, None),
              lambda k=FAKE, v=FAKE, ks=128, vs=128, m=FAKE, n=1: E.elis_kv_read(good, m, n, k, v, ks, vs, None)):
        assert f(n=0, k=None, v=None, m=None) == E.ELIS_OK
        assert f(k=None) == f(v=None) == f(m=None) == f(n=-1) == E.ELIS_EINVAL
        assert f(ks=127) == f(vs=100) == f(n=1 << 30) == E.ELIS_ESHAPE


def test_attention_refusals():
    good = E.elis_kv_cache(FAKE_WS, 64, 16, 2, 64)
    ok = dict(c=good, q=FAKE, qs=256, cu=FAKE, n=2, total=5, max_q=4, blocks=FAKE, rows_n=2, bs=8, rows=None, lens=FAKE, max_kv=100, heads=4,
              scale=0.1, window=0, out=FAKE, os=256, ws=FAKE_WS, wsb=1 << 30)

    def call(**kw):
        return E.elis_kv_attention(*(ok | kw).values(), None)

    for kw in (dict(c=None), dict(q=None), dict(cu=None), dict(blocks=None), dict(lens=None), dict(out=None), dict(ws=None), dict(ws=FAKE_WS + 8),
               dict(n=0), dict(total=-1), dict(max_q=0), dict(max_kv=-1), dict(heads=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN),
               dict(scale=INF), dict(window=-1), dict(rows_n=0), dict(bs=0)):
        assert call(**kw) == E.ELIS_EINVAL, kw
    for kw in (dict(qs=255), dict(os=100), dict(max_kv=129), dict(rows_n=1), dict(n=65536, rows_n=65536), dict(max_q=1 << 30), dict(total=1 << 30)):
        assert call(**kw) == E.ELIS_ESHAPE, kw
    assert call(heads=5, qs=320, os=320) == E.ELIS_EUNSUPPORTED
    assert call(wsb=0) == E.ELIS_EWORKSPACE
    assert call(total=0) == E.ELIS_OK
    size = E.elis_kv_attention_workspace_bytes
    assert size(2, 5, 4, 100, 4, 2, 64) >= 256 and size(0, 5, 4, 100, 4, 2, 64) == 0 and size(2, 5, 4, 100, 5, 2, 64) == 0
    assert size(1, 1, 1, 30000, 32, 8, 128) >= 32 * 8 * 128 * 4        # one long request is split
    assert size(1, 1, 1, 1 << 30, 32, 8, 128) > 0


def test_logits_refusals():
    ok = dict(x=FAKE, dt=0, xs=100, n=2, vocab=100, ids=FAKE, cu=FAKE, total=10, pl=None, r=None, f=None, p=None, bc=None, bt=None, bv=None, bn=0,
              mask=None, nm=0, ms=0, mr=None, out=0x2000, os=100)

    def call(**kw):
        return E.elis_logits_adjust(*(ok | kw).values(), None)

    assert call(n=0) == E.ELIS_OK
    for kw in (dict(x=None), dict(dt=2), dict(n=-1), dict(vocab=0), dict(cu=None), dict(total=-1), dict(out=None), dict(bn=-1),
               dict(bc=FAKE, bn=3, bt=None, bv=FAKE), dict(bc=FAKE, bn=3, bt=FAKE), dict(mask=FAKE, nm=0, ms=4), dict(out=FAKE, os=101),
               dict(out=FAKE, dt=1)):
        assert call(**kw) == E.ELIS_EINVAL, kw
    for kw in (dict(xs=99), dict(os=99), dict(mask=FAKE, nm=2, ms=3), dict(mask=FAKE, nm=1, ms=4), dict(n=65536)):
        assert call(**kw) == E.ELIS_ESHAPE, kw
    assert call(total=2 ** 29 + 1) == E.ELIS_ESHAPE


def test_attention_of_nothing_and_scales_at_the_end():
    c = E.elis_kv_cache(FAKE_WS, 64, 16, 2, 64)
    call = lambda total, q, scale=0.1: E.elis_kv_attention(c, q, 256, FAKE, 2, total, 4, FAKE, 2, 8, None, FAKE, 100, 4, scale, 0, q, 256, FAKE_WS,  # noqa: E731
                                                           1 << 20, None)
    assert call(0, None) == E.ELIS_OK and call(1, None) == E.ELIS_EINVAL
    assert call(0, FAKE, 2.0e38) == E.ELIS_OK and call(0, FAKE, 3.0e38) == E.ELIS_EINVAL  # times log2(e): past the range


def test_state_off_the_device_is_refused():
    """What a constructor would set up with a kernel has to lie on the current device."""
    from paper_2505_09142_amd.device import KVCache, PagePool
    with pytest.raises(E.ElisError):
        PagePool(4, 16, 2, 2, device="cpu")
    with pytest.raises(E.ElisError):
        KVCache(4, 16, 2, 64, device="cpu")

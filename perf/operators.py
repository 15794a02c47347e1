"""What the jobs that a round has selected need next: cases, inputs, one pass and its plain form.

A case is a dict of plain values; "op" says which operator a pass goes through:

  pages      the block tables and slot maps of a batch out of its lengths (grow), and the pages given back (trim)
  append     keys and values of new tokens into the 4-bit cache, and the same tokens read back as what was kept
  attention  new tokens of every job against its cached keys: one token each, long prompts, or both in one batch
  logits     penalties for repeated tokens, biases and grammar masks on the next token's logits

Lengths follow from the case alone ("lens": a seed of their own), so a case's work is fixed; the contents follow from the
seed that prepare() is given. The cache holds, for every page, head and 16 tokens, one record of 17 * d_head bytes:

  keys     [16 tokens][d_head / 2]         two E2M1 values a byte, the lower value in the lower half
  values   [4][16][4][d_head / 32]         token 4 a + b, values (d_head / 16) c ... of column c at [a][c][b]
  scales   keys [16][groups], values [4][groups][4]   E8M0, one for 32 values; groups = d_head / 32
"""
import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

DEV = "cuda"
HEADER = 256  # bytes before a cache's first page
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # A decode step of 64 running jobs: every job gains one token, few need a page. Latency is all.
        {"name": "pages_step_64", "op": "pages", "jobs": 64, "lens": 1, "median": 900, "max_len": 4096, "page": 16, "fresh": False},
        # A burst of 2048 new requests: every prompt gets its pages and a slot for each of its tokens.
        {"name": "pages_admit_2048", "op": "pages", "jobs": 2048, "lens": 2, "median": 200, "max_len": 2048, "page": 16, "fresh": True},
        # The keys and values of one new token of each of 64 jobs, out of the fused projection's rows.
        {"name": "append_64", "op": "append", "tokens": 64, "page": 16, "kv_heads": 8, "heads": 32, "d_head": 128, "runs": 64},
        # A prefill step of 32768 prompt tokens.
        {"name": "append_32k", "op": "append", "tokens": 32768, "page": 64, "kv_heads": 8, "heads": 32, "d_head": 128, "runs": 37},
        # One job at its first tokens: twelve heads of 64, the framework's own head layout.
        {"name": "decode_1_short", "op": "attention", "seqs": 1, "lens": 3, "median": 193, "max_kv": 256, "new": 1, "chunks": 0, "heads": 12, "kv_heads": 12, "d_head": 64, "page": 16, "window": 0},
        # One long conversation alone: the work has to be split over its length.
        {"name": "decode_1_long", "op": "attention", "seqs": 1, "lens": 4, "median": 30001, "max_kv": 32768, "new": 1, "chunks": 0, "heads": 32, "kv_heads": 8, "d_head": 128, "page": 16, "window": 0},
        # The selected batch of 64 jobs with lengths as the request stream has them, up to 4096.
        {"name": "decode_64", "op": "attention", "seqs": 64, "lens": 5, "median": 900, "max_kv": 4096, "new": 1, "chunks": 0, "heads": 32, "kv_heads": 8, "d_head": 128, "page": 16, "window": 0},
        # Long contexts in a full batch: the cache's bytes are what counts.
        {"name": "decode_48_long", "op": "attention", "seqs": 48, "lens": 6, "median": 16000, "max_kv": 32768, "new": 1, "chunks": 0, "heads": 32, "kv_heads": 8, "d_head": 128, "page": 64, "window": 0},
        # A step that takes two prompt chunks of up to 512 tokens along with 30 running jobs.
        {"name": "mixed_32", "op": "attention", "seqs": 32, "lens": 7, "median": 1500, "max_kv": 4096, "new": 512, "chunks": 2, "heads": 32, "kv_heads": 8, "d_head": 128, "page": 16, "window": 0},
        # A prompt chunk of 2048 tokens deep in a long document.
        {"name": "prefill_2k_16k", "op": "attention", "seqs": 1, "lens": 8, "median": 16000, "max_kv": 16384, "new": 2048, "chunks": 1, "heads": 32, "kv_heads": 8, "d_head": 128, "page": 64, "window": 0},
        # The next token of 32 jobs, bf16 logits over the framework's smaller vocabulary, short histories.
        {"name": "logits_32_30k", "op": "logits", "rows": 32, "lens": 9, "vocab": 30522, "median": 300, "max_len": 512, "bf16": True, "bias": 16, "mask": True},
        # 128 jobs over the large multilingual vocabulary, long histories, fp32 logits.
        {"name": "logits_128_250k", "op": "logits", "rows": 128, "lens": 10, "vocab": 250002, "median": 2000, "max_len": 8192, "bf16": False, "bias": 64, "mask": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["pages", "append", "attention", "attention", "attention", "attention", "logits", "logits"])
    lens = rng.randrange(1 << 20)
    if op == "pages":
        fresh = rng.random() < 0.5
        return {"op": op, "jobs": _log(rng, 1, 2048), "lens": lens, "median": _log(rng, 20, 400 if fresh else 4000), "max_len": 2048 if fresh else 8192,
                "page": rng.choice([16, 32, 64, 128]), "fresh": fresh}
    if op == "append":
        kv, tokens = rng.choice([1, 2, 4, 8, 12]), _log(rng, 1, 20000)
        return {"op": op, "tokens": tokens, "page": rng.choice([16, 32, 64, 128]), "kv_heads": kv, "heads": kv * rng.choice([1, 3, 4]),
                "d_head": rng.choice([64, 128]), "runs": _log(rng, 1, min(tokens, 256))}
    if op == "attention":
        kv = rng.choice([1, 2, 4, 8, 12])
        heads = kv * rng.choice([1, 2, 4, 5, 8] if kv < 12 else [1, 2])
        kind = rng.choice(["decode", "decode", "mixed", "prefill"])
        seqs = _log(rng, 1, 96) if kind == "decode" else _log(rng, 1, 12)
        max_kv = min(32768, _log(rng, 64, 1 << 20) // seqs + 16) if kind == "decode" else _log(rng, 64, 12000)
        new = 1 if kind == "decode" else min(max_kv, _log(rng, 2, 2000), max(1, int(2e9) // (seqs * heads * max_kv)))
        chunks = 0 if kind == "decode" else seqs if kind == "prefill" else max(1, seqs // 3)
        return {"op": op, "seqs": seqs, "lens": lens, "median": max(1, max_kv // rng.choice([1, 2, 3])), "max_kv": max_kv, "new": new, "chunks": chunks,
                "heads": heads, "kv_heads": kv, "d_head": rng.choice([64, 128, 128]), "page": rng.choice([16, 16, 32, 64, 128]),
                "window": rng.choice([0, 0, 0, _log(rng, 16, 2000)])}
    return {"op": op, "rows": _log(rng, 1, 128), "lens": lens, "vocab": rng.choice([1000, 30522, 50257, 128000, 250002]), "median": _log(rng, 20, 3000),
            "max_len": 8192, "bf16": rng.random() < 0.5, "bias": rng.choice([0, 1, 16, 200]), "mask": rng.random() < 0.5}


# ------------------------------------------------------------------ sizes that follow from a case

def _lengths(case, n, longest):
    r = np.random.default_rng(case["lens"])
    v = np.exp(np.log(case["median"]) + 0.6 * r.standard_normal(n))
    if n == 1:
        v[:] = case["median"]
    return np.clip(np.rint(v), 1, longest).astype(np.int64), r


def _pages_sizes(case):
    after, _ = _lengths(case, case["jobs"], case["max_len"])
    before = np.zeros_like(after) if case["fresh"] else after - 1
    return before, after


def _attention_sizes(case):
    kv, r = _lengths(case, case["seqs"], case["max_kv"])
    q = np.ones_like(kv)
    at = r.permutation(case["seqs"])[:case["chunks"]]
    q[at] = np.minimum(kv[at], np.rint(case["new"] * r.uniform(0.5, 1.0, len(at)) if case["seqs"] > 1 else case["new"]).astype(np.int64))
    return np.maximum(q, 1), kv


def _history_sizes(case):
    total, r = _lengths(case, case["rows"], case["max_len"])
    return np.rint(total * r.uniform(0.2, 0.9, len(total))).astype(np.int64), total


def _visible(q, kv, window):
    """Sum over the query tokens of the keys that each one sees, and the keys that any of a job's tokens sees."""
    pairs = keys = 0
    for a, b in zip(q.tolist(), kv.tolist()):
        p = np.arange(b - a, b)
        n = p + 1 if window == 0 else np.minimum(p + 1, window)
        pairs += int(n.sum())
        keys += int(n[0] + a - 1)
    return pairs, keys


def work(case):
    op = case["op"]
    if op == "pages":
        before, after = _pages_sizes(case)
        pages = -(-after // case["page"])
        moved = int((pages - -(-before // case["page"])).sum())
        n, t = len(after), int((after - before).sum())
        # slots, lengths, offsets and counts; a slot for each token; the batch's tables; pages that move there and back
        return {"bytes": 24 * n + 4 * t + 4 * n * int(pages.max()) + 4 * int(pages.sum()) + 16 * moved, "flops": 0}
    if op == "append":
        values = 2 * case["tokens"] * case["kv_heads"] * case["d_head"]
        return {"bytes": values * 2 + values * 17 / 32 * 2 + values * 2 + 8 * case["tokens"], "flops": 0}
    if op == "attention":
        q, kv = _attention_sizes(case)
        pairs, keys = _visible(q, kv, case["window"])
        d = case["d_head"]
        return {"bytes": keys * case["kv_heads"] * 2 * d * 17 / 32 + 4 * int(q.sum()) * case["heads"] * d + 4 * int((-(-kv // case["page"])).sum()) + 8 * len(q),
                "flops": 4.0 * pairs * case["heads"] * d}
    _, total = _history_sizes(case)
    n = case["rows"]
    return {"bytes": n * case["vocab"] * ((2 if case["bf16"] else 4) + 4) + 4 * int(total.sum()) + 8 * n * case["bias"] + (n * case["vocab"] / 8 if case["mask"] else 0), "flops": 0}


# ------------------------------------------------------------------ inputs

def _int(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _cu(lens):
    return np.concatenate([[0], np.cumsum(lens)])


def _cache_bytes(case, n_pages):
    return HEADER + n_pages * case["kv_heads"] * (case["page"] // 16) * 17 * case["d_head"]


def _filled_cache(case, n_pages, gen):
    """A cache whose pages hold keys and values of random tokens: some channels of the keys are larger than others, as in trained models."""
    d, heads, page = case["d_head"], case["kv_heads"], case["page"]
    buf = torch.zeros(_cache_bytes(case, n_pages), dtype=torch.uint8, device=DEV)
    channel = torch.exp(0.5 * torch.randn((heads, 1, d), generator=gen, device=DEV))
    step = max(1, (1 << 26) // (heads * page * d))
    for at in range(0, n_pages, step):
        m = min(step, n_pages - at)
        k = torch.randn((m, heads, page, d), generator=gen, device=DEV) * channel
        v = torch.randn((m, heads, page, d), generator=gen, device=DEV)
        _pages_of(buf, case)[at:at + m] = _records(*_quantise(k), *_quantise(v))
    return buf


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    r = np.random.default_rng(seed)
    op = case["op"]
    s = SimpleNamespace(case=case, op=op)
    if op == "pages":
        before, after = _pages_sizes(case)
        n, P = len(after), case["page"]
        held = -(-before // P)
        need = -(-after // P)
        s.width = int(need.max())
        n_pages, max_jobs, max_pages = int(1.25 * need.sum()) + 8, 2 * n, s.width + 3
        ids = r.permutation(n_pages)
        slots = r.permutation(max_jobs)[:n]
        table = np.full((max_jobs, max_pages), -1)
        at = _cu(held)
        for i, slot in enumerate(slots):
            table[slot, :held[i]] = ids[at[i]:at[i + 1]]
        count = n_pages - int(at[-1])
        free = np.full(n_pages, -1)
        free[:count] = ids[at[-1]:]
        of_slot = np.zeros(max_jobs, np.int64)
        of_slot[slots] = held
        s.state, s.free, s.held, s.table = _int([0, count]), _int(free), _int(of_slot), _int(table)
        s.slots, s.before, s.after, s.cu = _int(slots), _int(before), _int(after), _int(_cu(after - before))
        s.total = int((after - before).sum())
        s.blocks = torch.empty((n, s.width), dtype=torch.int32, device=DEV)
        s.map = torch.empty(s.total, dtype=torch.int32, device=DEV)
        if own:
            from paper_2505_09142_amd.device import PagePool
            s.pool = PagePool(n_pages, P, max_jobs, max_pages, tensors=(s.state, s.free, s.held, s.table))
    elif op == "append":
        T, P, d, kv, runs = case["tokens"], case["page"], case["d_head"], case["kv_heads"], case["runs"]
        rows = torch.randn((T, (case["heads"] + 2 * kv) * d), generator=gen, device=DEV).to(torch.bfloat16)
        s.k = rows[:, case["heads"] * d:(case["heads"] + kv) * d].unflatten(1, (kv, d))
        s.v = rows[:, (case["heads"] + kv) * d:].unflatten(1, (kv, d))
        # `runs` jobs share the tokens; each starts somewhere in its first page
        cuts = np.sort(r.choice(np.arange(1, T), runs - 1, replace=False)) if runs > 1 else np.zeros(0, np.int64)
        lens = np.diff(np.concatenate([[0], cuts, [T]]))
        first = r.integers(0, P, runs)
        need = -(-(first + lens) // P)
        n_pages = int(need.sum()) + 5
        ids, at = r.permutation(n_pages), _cu(need)
        pos = np.concatenate([f + np.arange(m) for f, m in zip(first, lens)])
        s.map = _int(ids[np.repeat(at[:-1], lens) + pos // P] * P + pos % P)
        s.buf = torch.zeros(_cache_bytes(case, n_pages), dtype=torch.uint8, device=DEV)
        s.out_k = torch.empty((T, kv, d), dtype=torch.bfloat16, device=DEV)
        s.out_v = torch.empty((T, kv, d), dtype=torch.bfloat16, device=DEV)
        if own:
            from paper_2505_09142_amd.device import KVCache
            s.cache = KVCache(n_pages, P, kv, d, buf=s.buf)
    elif op == "attention":
        q, kv = _attention_sizes(case)
        P, d = case["page"], case["d_head"]
        need = -(-kv // P)
        s.width, s.max_q, s.max_kv = int(need.max()), int(q.max()), int(kv.max())
        n_pages = int(need.sum()) + 3
        ids, at = r.permutation(n_pages), _cu(need)
        blocks = np.full((len(q), s.width), -1)
        for i in range(len(q)):
            blocks[i, :need[i]] = ids[at[i]:at[i + 1]]
        s.blocks, s.lens, s.cu = _int(blocks), _int(kv), _int(_cu(q))
        s.buf = _filled_cache(case, n_pages, gen)
        s.q = torch.randn((int(q.sum()), case["heads"], d), generator=gen, device=DEV).to(torch.bfloat16)
        s.out = torch.empty_like(s.q)
        if own:
            from paper_2505_09142_amd.device import KVCache
            s.cache = KVCache(n_pages, P, case["kv_heads"], d, buf=s.buf)
    else:
        prompt, total = _history_sizes(case)
        n, V = case["rows"], case["vocab"]
        s.logits = torch.randn((n, V), generator=gen, device=DEV).mul_(3).to(torch.bfloat16 if case["bf16"] else torch.float32)
        T = int(total.sum())
        # token frequencies fall like natural text's: a few tokens come again and again
        u = torch.rand(T, generator=gen, device=DEV, dtype=torch.float64)
        s.ids = (torch.exp(u * math.log(V)) - 1).to(torch.int32).clamp_(0, V - 1)
        s.cu, s.prompt = _int(_cu(total)), _int(prompt)
        s.total = T
        draw_ = lambda lo, hi: torch.from_numpy(r.uniform(lo, hi, n).astype(np.float32)).to(DEV)  # noqa: E731
        s.rep, s.freq, s.pres = draw_(1.0, 1.5), draw_(-0.2, 0.8), draw_(-0.2, 0.8)
        b = min(case["bias"], V)
        s.bias = None
        if b:
            tokens = torch.rand((n, V), generator=gen, device=DEV).topk(b, dim=1).indices.to(torch.int32)
            s.bias = (_int(np.arange(n + 1) * b), tokens.reshape(-1).contiguous(), torch.randn(n * b, generator=gen, device=DEV) * 2)
        s.mask = s.mask_rows = None
        if case["mask"]:
            # half of the jobs write under one of a few grammars; the others freely
            words = -(-V // 32)
            s.mask = torch.randint(-2**31, 2**31 - 1, (5, words), generator=gen, device=DEV, dtype=torch.int64).to(torch.int32)
            s.mask_rows = _int(np.where(r.random(n) < 0.5, -1, r.integers(0, 5, n)))
        s.out = torch.empty((n, V), dtype=torch.float32, device=DEV)
    return s


# ------------------------------------------------------------------ the 4-bit form

def _quantise(x):
    """E2M1 codes and E8M0 scales (one for 32 values along the last axis) of x: the scale is the least 2^e with max|x| < 7 * 2^e."""
    g = x.float().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)
    e = (e - 3 + (m >= 0.875) + 127).clamp(2, 252)
    y = torch.ldexp(g.abs(), 127 - e)
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0) + 8 * (g < 0)).to(torch.uint8)
    return code.flatten(-2), e.squeeze(-1).to(torch.uint8)


def _halves(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _records(kc, ks, vc, vs):
    """The pages' bytes [pages, heads, page / 16, 17 d] of codes [pages, heads, page, d] and scales [pages, heads, page, d / 32]."""
    d = kc.shape[-1]
    lead = kc.shape[:2] + (kc.shape[2] // 16,)
    k = _halves(kc).reshape(*lead, 8 * d)
    v = _halves(vc).reshape(*lead, 4, 4, 16, d // 32).transpose(-3, -2).reshape(*lead, 8 * d)
    return torch.cat([k, v, ks.reshape(*lead, d // 2), vs.reshape(*lead, 4, 4, d // 32).transpose(-2, -1).reshape(*lead, d // 2)], dim=-1)


def _pages_of(buf, case):
    return buf[HEADER:].view(-1, case["kv_heads"], case["page"] // 16, 17 * case["d_head"])


def _values(pages, d):
    """Keys and values [..., heads, tokens, d] in fp32 of pages [..., heads, page / 16, 17 d]."""
    lead = pages.shape[:-1]
    pair = torch.tensor([[E2M1[n & 7] * (1 - 2 * (n >> 3)) for n in (b & 15, b >> 4)] for b in range(256)], device=DEV)
    k = pair[pages[..., :8 * d].int()].reshape(*lead, 16, d // 32, 32)
    v = pages[..., 8 * d:16 * d].reshape(*lead, 4, 16, 4, d // 32).transpose(-3, -2)
    v = pair[v.int()].reshape(*lead, 16, d // 32, 32)
    ks = pages[..., 16 * d:16 * d + d // 2].reshape(*lead, 16, d // 32)
    vs = pages[..., 16 * d + d // 2:].reshape(*lead, 4, d // 32, 4).transpose(-2, -1).reshape(*lead, 16, d // 32)
    one = torch.ones((), device=DEV)
    k.mul_(torch.ldexp(one, ks.int() - 127).unsqueeze(-1))
    v.mul_(torch.ldexp(one, vs.int() - 127).unsqueeze(-1))
    return k.reshape(*lead[:-1], -1, d), v.reshape(*lead[:-1], -1, d)


# ------------------------------------------------------------------ one pass

def _plain_pages(s):
    P = s.case["page"]
    slots = s.slots.long()
    j = torch.arange(s.width, device=DEV)
    held = s.held[slots].unsqueeze(1)
    need = (-(-s.after.unsqueeze(1) // P) - held).clamp(min=0)
    off = need.cumsum(0) - need
    fits = (need == 0) | (off + need <= s.state[1])
    new = (j >= held) & (j < held + need) & fits
    at = (s.state[1] - 1 - (off + j - held)).clamp(0, len(s.free) - 1)
    rows = torch.where(new, s.free[at], s.table[slots, :s.width])
    s.table[slots, :s.width] = rows
    held = held + need * fits
    s.held[slots] = held.squeeze(1).int()
    s.state[1] -= (need * fits).sum()
    s.blocks.copy_(torch.where(j < held, rows, -1))
    t = torch.arange(s.total, device=DEV)
    i = torch.searchsorted(s.cu[1:].contiguous(), t, right=True)
    p = s.before[i] + t - s.cu[i]
    s.map.copy_(rows[i, p // P] * P + p % P)
    # and back: the pages past each job's former length return in the order that undoes the above
    keep = -(-s.before.unsqueeze(1) // P)
    give = held - keep
    off = give.cumsum(0) - give
    back = (j >= keep) & (j < held)
    to = torch.where(back, s.state[1] + give.sum() - 1 - (off + j - keep), len(s.free))
    free = torch.cat([s.free, s.free[:1]])
    free[to.reshape(-1)] = rows.reshape(-1)
    s.free.copy_(free[:-1])
    s.held[slots] = keep.squeeze(1).int()
    s.state[1] += give.sum()
    return {"blocks": s.blocks, "map": s.map, "state": s.state, "free": s.free, "held": s.held}


def _plain_append(s):
    d, P = s.case["d_head"], s.case["page"]
    pages = _pages_of(s.buf, s.case)
    page, tile, b = s.map.long() // P, s.map.long() % P // 16, s.map.long() % 16
    h = torch.arange(s.case["kv_heads"], device=DEV)
    at = (((page * s.case["kv_heads"]).unsqueeze(1) + h) * (P // 16) + tile.unsqueeze(1)) * (17 * d)  # [tokens, heads]
    at, b = at.unsqueeze(2), b.view(-1, 1, 1)
    kc, ks = _quantise(s.k)
    vc, vs = _quantise(s.v)
    flat = pages.view(-1)
    m, g = torch.arange(d // 2, device=DEV), torch.arange(d // 32, device=DEV)
    places = [at + b * (d // 2) + m,
              at + 8 * d + (((b // 4 * 16 + m // (d // 32)) * 4 + b % 4) * (d // 32)) + m % (d // 32),
              at + 16 * d + b * (d // 32) + g,
              at + 16 * d + d // 2 + (b // 4 * (d // 32) + g) * 4 + b % 4]
    flat[places[0]] = _halves(kc)
    flat[places[1]] = _halves(vc)
    flat[places[2]] = ks
    flat[places[3]] = vs
    # read back
    pair = torch.tensor([[E2M1[n & 7] * (1 - 2 * (n >> 3)) for n in (c & 15, c >> 4)] for c in range(256)], device=DEV)
    one = torch.ones((), device=DEV)
    scale = lambda p: torch.ldexp(one, flat[p].int() - 127).unsqueeze(-1)  # noqa: E731
    s.out_k.copy_((pair[flat[places[0]].int()].reshape(*s.k.shape[:2], -1, 32) * scale(places[2])).reshape(s.k.shape))
    s.out_v.copy_((pair[flat[places[1]].int()].reshape(*s.v.shape[:2], -1, 32) * scale(places[3])).reshape(s.v.shape))
    return {"k": s.out_k, "v": s.out_v}


def _plain_attention(s):
    c = s.case
    d, kv, G, n = c["d_head"], c["kv_heads"], c["heads"] // c["kv_heads"], len(s.lens)
    pages = _pages_of(s.buf, c)[s.blocks.clamp(min=0).reshape(-1).long()]             # [n * width, heads, page / 16, 17 d]
    k, v = _values(pages, d)
    k, v = (x.unflatten(0, (n, -1)).transpose(1, 2).reshape(n * kv, -1, d) for x in (k, v))  # [n * heads, width * page, d]
    # the queries of every job, padded to the longest
    length = (s.cu[1:] - s.cu[:-1]).long()
    t = torch.arange(s.max_q, device=DEV)
    real = t < length.unsqueeze(1)                                                     # [n, max_q]
    at = (s.cu[:-1].long().unsqueeze(1) + t).clamp(max=len(s.q) - 1)
    q = s.q[at].float().view(n, s.max_q, kv, G, d).permute(0, 2, 1, 3, 4).reshape(n * kv, s.max_q * G, d)
    score = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(d ** -0.5).view(n, kv, s.max_q, G, -1)
    key = torch.arange(score.shape[-1], device=DEV)
    pos = (s.lens.long() - length).unsqueeze(1) + t
    sees = key <= pos.unsqueeze(-1)
    if c["window"]:
        sees &= key > pos.unsqueeze(-1) - c["window"]
    score.masked_fill_(~sees.view(n, 1, s.max_q, 1, -1), -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.bmm(p.view(n * kv, s.max_q * G, -1), v).view(n, kv, s.max_q, G, d) / torch.where(total == 0, 1.0, total)
    out = out.permute(0, 2, 1, 3, 4).reshape(n * s.max_q, c["heads"], d)
    spare = torch.empty((len(s.q) + 1, c["heads"], d), dtype=torch.bfloat16, device=DEV)  # padding goes to the last row
    spare[torch.where(real, at, len(s.q)).reshape(-1)] = out.to(torch.bfloat16)
    s.out.copy_(spare[:-1])
    return s.out


def _plain_logits(s):
    n, V = s.logits.shape
    t = torch.arange(s.total, device=DEV)
    row = torch.searchsorted(s.cu[1:].contiguous(), t, right=True)
    written = t - s.cu[row] >= s.prompt[row]
    cell = row * V + s.ids
    count = torch.zeros(n * V, device=DEV).index_add_(0, cell, written.float()).view(n, V)
    seen = torch.zeros(n * V, dtype=torch.bool, device=DEV).index_fill_(0, cell, True).view(n, V)
    x = s.logits.float()
    x = torch.where(seen, torch.where(x > 0, x / s.rep.unsqueeze(1), x * s.rep.unsqueeze(1)), x)
    x = x - s.freq.unsqueeze(1) * count - s.pres.unsqueeze(1) * (count > 0)
    if s.bias is not None:
        cu, tokens, values = s.bias
        i = torch.searchsorted(cu[1:].contiguous(), torch.arange(len(tokens), device=DEV), right=True)
        x.view(-1).index_add_(0, i * V + tokens, values)
    if s.mask is not None:
        v = torch.arange(V, device=DEV)
        allowed = (s.mask[:, v // 32] >> (v % 32).int()) & 1 == 1
        x.masked_fill_((s.mask_rows >= 0).unsqueeze(1) & ~allowed[s.mask_rows.clamp(min=0).long()], -math.inf)
    s.out.copy_(x)
    return s.out


def run(s):
    if not own:
        return {"pages": _plain_pages, "append": _plain_append, "attention": _plain_attention, "logits": _plain_logits}[s.op](s)
    if s.op == "pages":
        s.pool.grow(s.slots, s.after, s.cu, s.total, s.map, out_blocks=s.blocks)
        s.pool.trim(s.slots, s.before)
        return {"blocks": s.blocks, "map": s.map, "state": s.state, "free": s.free, "held": s.held}
    if s.op == "append":
        s.cache.append(s.k, s.v, s.map)
        s.cache.read(s.map, s.out_k, s.out_v)
        return {"k": s.out_k, "v": s.out_v}
    if s.op == "attention":
        s.cache.attention(s.q, s.cu, s.lens, s.blocks, s.max_q, s.max_kv, window=s.case["window"], out=s.out)
        return s.out
    from paper_2505_09142_amd.device import adjust_logits
    adjust_logits(s.logits, s.ids, s.cu, s.out, prompt_lens=s.prompt, repetition=s.rep, frequency=s.freq, presence=s.pres,
                  bias=s.bias, mask=s.mask, mask_rows=s.mask_rows)
    return s.out


# ------------------------------------------------------------------ the same in 64 bits, from the definitions

def _rounded64(x):
    """What 4 bits keep of x: groups of 32, a power of two each, the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times it, ties to the even code."""
    g = x.double().reshape(*x.shape[:-1], -1, 32)
    top = g.abs().amax(-1, keepdim=True)
    unit = torch.exp2(torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 2)
    unit = torch.where(top >= 7 * unit, 2 * unit, unit)
    y = g.abs() / unit
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0)).double()
    return (torch.sign(g) * torch.clamp(torch.round(y / step) * step, max=6.0) * unit).reshape(x.shape)


def _token64(buf, case, page, i, value):
    """Row i of a page (or rows, as tensors) for every head, in 64 bits, out of the record's definition."""
    d = case["d_head"]
    rec = buf[HEADER:].view(-1, case["kv_heads"], case["page"] // 16, 17 * d)
    h = torch.arange(case["kv_heads"], device=DEV).view(1, -1, 1)
    e = torch.arange(d, device=DEV).view(1, 1, -1)
    page, i = page.view(-1, 1, 1), i.view(-1, 1, 1)
    tile, b = i // 16, i % 16
    if value:
        per = d // 16
        byte = rec[page, h, tile, 8 * d + ((b // 4 * 16 + e // per) * 4 + b % 4) * (d // 32) + e % per // 2]
        scale = rec[page, h, tile, 16 * d + d // 2 + (b // 4 * (d // 32) + e // 32) * 4 + b % 4]
    else:
        byte = rec[page, h, tile, b * (d // 2) + e // 2]
        scale = rec[page, h, tile, 16 * d + b * (d // 32) + e // 32]
    code = (byte.int() >> (4 * (e % 2)).int()) & 15
    size, half = (code >> 1 & 3).double(), (code & 1).double()
    x = torch.where(size == 0, 0.5 * half, torch.exp2(size - 1) * (1 + 0.5 * half))
    return torch.where(code >= 8, -x, x) * torch.exp2(scale.double() - 127)


def exact(case, seed):
    op = case["op"]
    if op == "pages":
        return None
    s = prepare(case, seed)
    if op == "append":
        return {"k": _rounded64(s.k), "v": _rounded64(s.v)}
    if op == "attention":
        q_lens, kv_lens = _attention_sizes(case)
        G, P = case["heads"] // case["kv_heads"], case["page"]
        at, outs = 0, []
        for i, (a, b) in enumerate(zip(q_lens.tolist(), kv_lens.tolist())):
            j = torch.arange(b, device=DEV)
            page = s.blocks[i].long()[j // P]
            parts = []
            k = torch.cat([_token64(s.buf, case, page[u:u + 4096], j[u:u + 4096] % P, False) for u in range(0, b, 4096)])
            v = torch.cat([_token64(s.buf, case, page[u:u + 4096], j[u:u + 4096] % P, True) for u in range(0, b, 4096)])
            pos = torch.arange(b - a, b, device=DEV)
            sees = (j <= pos[:, None]) & ((j > pos[:, None] - case["window"]) if case["window"] else True)
            for head in range(case["heads"]):
                w = s.q[at:at + a, head].double() @ k[:, head // G].t().contiguous() / math.sqrt(case["d_head"])
                parts.append(torch.softmax(torch.where(sees, w, -math.inf), dim=-1) @ v[:, head // G])
            outs.append(torch.stack(parts, 1))
            at += a
        return torch.cat(outs)
    n, V = s.logits.shape
    out = s.logits.double()
    prompt, total = _history_sizes(case)
    at = _cu(total)
    bit = torch.arange(V, device=DEV)
    for i in range(n):
        ids = s.ids[at[i]:at[i + 1]].long()
        x = out[i]
        rep, freq, pres = (float(t[i]) for t in (s.rep, s.freq, s.pres))
        h = torch.bincount(ids, minlength=V)
        c = torch.bincount(ids[int(prompt[i]):], minlength=V)
        x = torch.where(h > 0, torch.where(x > 0, x / rep, x * rep), x) - freq * c - pres * (c > 0)
        if s.bias is not None:
            b = case["bias"] if case["bias"] < V else V
            x = x.index_add(0, s.bias[1][i * b:(i + 1) * b].long(), s.bias[2][i * b:(i + 1) * b].double())
        if s.mask is not None and int(s.mask_rows[i]) >= 0:
            word = s.mask[int(s.mask_rows[i])].long() & 0xFFFFFFFF
            x = torch.where((word[bit // 32] >> (bit % 32)) & 1 == 1, x, -math.inf)
        out[i] = x
    return out

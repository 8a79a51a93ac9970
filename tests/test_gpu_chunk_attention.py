"""Attention of chunks of new tokens over a paged cache, and differential attention, against softmax in 64 bits."""
import math

import numpy as np
import pytest

import paper_2607_27952_gb300 as last

pytestmark = pytest.mark.gpu

DTYPES = ["float32", "bfloat16"]


def _chunk(cache, seqs, q, cu_new, causal=True, window=0, scale=0.0, stream=None, poll=True):
    import torch
    import chunk_util as ch
    out = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:2], float("nan"), dtype=torch.float32, device="cuda")
    ws = ch.workspace(cache, q.shape[1])
    last.last_cache_chunk_attention(cache, 0, seqs, q, out, ws, cu_new=cu_new, lse=lse, causal=causal, window=window,
                                    softmax_scale=scale, stream=stream)
    if poll:
        last.last_poll(ws, stream)
    return out, lse, ws


def _params(pairs, d, seed, norm=True):
    import torch
    import cache_util as cu
    lam = 0.5 + 0.3 * torch.tanh(cu.randn((pairs,), "float32", seed))
    return lam, 1 + 0.2 * cu.randn((2 * d,), "float32", seed + 1) if norm else None


def _diff(cache, seqs, q, cu_new, lam, weight=None, eps=1e-5, out_scale=1.0, causal=True, window=0, scale=0.0, stream=None, poll=True):
    import torch
    import chunk_util as ch
    out = torch.full((q.shape[0], q.shape[1] // 2, 2 * q.shape[2]), float("nan"), dtype=q.dtype, device="cuda")
    ws = ch.workspace(cache, q.shape[1])
    last.last_cache_diff_attention(cache, 0, seqs, q, out, ws, lam, cu_new=cu_new, norm_weight=weight, norm_eps=eps, out_scale=out_scale,
                                   causal=causal, window=window, softmax_scale=scale, stream=stream)
    if poll:
        last.last_poll(ws, stream)
    return out, ws


NEW = [1, 0, 7, 64, 65, 130, 1, 33, 0, 300]
OLD = [0, 5, 0, 0, 63, 1, 500, 127, 0, 17]
LENS = [a + b for a, b in zip(NEW, OLD)]
MASKS = [(True, 0), (False, 0), (True, 1), (True, 50), (True, 129)]
SHAPES = [(1, 1, 64, 16), (4, 4, 128, 16), (12, 2, 128, 32), (14, 2, 64, 8), (16, 2, 80, 24), (9, 1, 128, 64),
          (32, 2, 64, 96), (34, 2, 72, 16), (6, 2, 256, 16), (20, 2, 192, 40), (3, 1, 8, 256), (10, 5, 16, 16), (5, 1, 136, 72),
          (200, 1, 64, 48)]


@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hq,hkv,d,size", SHAPES)
def test_lengths_heads_and_pages(hq, hkv, d, size, dtype, order):
    import chunk_util as ch
    cache, seqs, q, cu_new = ch.setup(NEW, OLD, hq, hkv, d, dtype, size, order, stale=float("nan"))
    out, lse, _ = _chunk(cache, seqs, q, cu_new)
    ch.check_chunk(cache, seqs, q, cu_new, out, lse, NEW, LENS)


@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hq,hkv,d,size", [(2, 2, 64, 16), (4, 4, 128, 16), (12, 2, 128, 32), (14, 2, 64, 8), (16, 4, 80, 24),
                                           (30, 2, 72, 16), (4, 2, 8, 256), (20, 10, 16, 16), (260, 2, 104, 48)])
@pytest.mark.parametrize("norm", [True, False])
def test_differences_of_lengths_heads_and_pages(hq, hkv, d, size, dtype, order, norm):
    import chunk_util as ch
    cache, seqs, q, cu_new = ch.setup(NEW, OLD, hq, hkv, d, dtype, size, order, stale=float("nan"))
    lam, weight = _params(hq // 2, d, 5, norm)
    out, _ = _diff(cache, seqs, q, cu_new, lam, weight, out_scale=0.7)
    ch.check_diff(cache, seqs, q, cu_new, out, lam, NEW, LENS, weight=weight, out_scale=0.7)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("causal,window", MASKS)
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (2, 2, 80), (6, 2, 192)])
def test_masks(hq, hkv, d, causal, window, dtype):
    import chunk_util as ch
    cache, seqs, q, cu_new = ch.setup(NEW, OLD, hq, hkv, d, dtype, 16, stale=float("inf"), seed=7)
    out, lse, _ = _chunk(cache, seqs, q, cu_new, causal, window, 0.2)
    ch.check_chunk(cache, seqs, q, cu_new, out, lse, NEW, LENS, None, causal, window, 0.2)
    if d > 128:
        return
    lam, weight = _params(hq // 2, d, 3)
    out, _ = _diff(cache, seqs, q, cu_new, lam, weight, causal=causal, window=window, scale=0.2)
    ch.check_diff(cache, seqs, q, cu_new, out, lam, NEW, LENS, None, causal, window, 0.2, weight)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [8, 16, 64, 80])
def test_key_begin(size, dtype):
    """First keys before, inside and behind the new tokens: rows without a key are empty; pages before it are not read."""
    import torch
    import chunk_util as ch
    new, old = [30, 30, 30, 5, 200, 1, 1], [70, 70, 70, 0, 300, 64, 64]
    begin = [0, 33, 85, 9, 260, 64, 65]
    lens = [a + b for a, b in zip(new, old)]
    cache, seqs, q, cu_new = ch.setup(new, old, 8, 2, 64, dtype, size, begin=begin, stale=float("inf"))
    for b, f in enumerate(begin):
        seqs.page_table[b, :min(f, lens[b]) // size] = -7
    lam, weight = _params(4, 64, 3)
    for causal, window in ((True, 0), (False, 0), (True, 40)):
        out, lse, _ = _chunk(cache, seqs, q, cu_new, causal, window)
        diff, _ = _diff(cache, seqs, q, cu_new, lam, weight, causal=causal, window=window)
        assert torch.isfinite(out).all() and torch.isfinite(diff).all()
        seqs.page_table.clamp_(min=0)      # for the plain form, which gathers them and leaves them out
        ch.check_chunk(cache, seqs, q, cu_new, out, lse, new, lens, begin, causal, window)
        ch.check_diff(cache, seqs, q, cu_new, diff, lam, new, lens, begin, causal, window, weight=weight)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,old,hq,hkv,d", [([3], [40000], 16, 4, 128), ([1, 17, 2], [9000, 20011, 100], 8, 2, 64),
                                              ([1] * 40, list(range(10, 4000, 100)), 4, 2, 80), ([140], [12000], 4, 2, 128),
                                              ([700, 1100], [3000, 0], 6, 2, 64)])
def test_keys_spread_over_the_gpu(new, old, hq, hkv, d, dtype):
    """Few rows over many keys: a block's keys are cut between CTAs."""
    import torch
    import chunk_util as ch
    lens = [a + b for a, b in zip(new, old)]
    cache, seqs, q, cu_new = ch.setup(new, old, hq, hkv, d, dtype, 32, seed=2)
    out, lse, _ = _chunk(cache, seqs, q, cu_new)
    ch.check_chunk(cache, seqs, q, cu_new, out, lse, new, lens)
    lam, weight = _params(hq // 2, d, 3)
    diff, _ = _diff(cache, seqs, q, cu_new, lam, weight)
    ch.check_diff(cache, seqs, q, cu_new, diff, lam, new, lens, weight=weight)
    again = _chunk(cache, seqs, q, cu_new)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    assert torch.equal(_diff(cache, seqs, q, cu_new, lam, weight)[0], diff)


@pytest.mark.parametrize("dtype", DTYPES)
def test_single_tokens_without_cu_new(dtype):
    """One token per sequence: the same as with cu_new, and for chunks as the attention of single tokens."""
    import torch
    import cache_util as cu
    import chunk_util as ch
    old = [0, 15, 16, 700, 64, 3000]
    lens = [n + 1 for n in old]
    cache, seqs, q, cu_new = ch.setup([1] * 6, old, 8, 4, 64, dtype, 16)
    a, b = _chunk(cache, seqs, q, cu_new), _chunk(cache, seqs, q, None)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    ch.check_chunk(cache, seqs, q, cu_new, b[0], b[1], [1] * 6, lens)
    one = torch.empty_like(q)
    last.last_cache_attention(cache, 0, seqs, q, one, cu.workspace(cache, 6, 8))
    assert float((one.double() - b[0].double()).norm() / one.double().norm()) < 3 * ch.UNIT[dtype] + 2.0 ** -18
    lam, weight = _params(4, 64, 1)
    d1, d2 = _diff(cache, seqs, q, cu_new, lam, weight)[0], _diff(cache, seqs, q, None, lam, weight)[0]
    assert torch.equal(d1, d2)
    ch.check_diff(cache, seqs, q, cu_new, d2, lam, [1] * 6, lens, weight=weight)


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_and_rising_logits(dtype):
    """Logits of hundreds that rise or fall along the keys: the maximum moves at every tile, or never again."""
    import torch
    import chunk_util as ch
    new, old = [40, 40], [300, 300]
    cache, seqs, q, cu_new = ch.setup(new, old, 4, 2, 64, dtype, 16, qscale=4.0)
    i = torch.arange(340, device="cuda")
    for b, w in ((0, i / 30.0), (1, (339 - i) / 30.0)):
        p = seqs.page_table[b].long()[i // 16]
        for h in range(2):
            cache.k[0, p, h, i % 16] = (q[40 * b, 2 * h].float()[None] * w[:, None].float()).to(q.dtype)
    lam, weight = _params(2, 64, 2)
    for scale in (0.0, 0.75):
        out, lse, _ = _chunk(cache, seqs, q, cu_new, scale=scale)
        ch.check_chunk(cache, seqs, q, cu_new, out, lse, new, [340, 340], scale=scale or None)
        diff, _ = _diff(cache, seqs, q, cu_new, lam, None, scale=scale)
        ch.check_diff(cache, seqs, q, cu_new, diff, lam, new, [340, 340], scale=scale or None)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 192])
@pytest.mark.parametrize("hkv", [2])
def test_what_a_row_does_not_see_has_no_part(d, hkv, dtype):
    """Infinities and NaN in K and V of keys that only later rows see: earlier rows are as without them, later ones show them."""
    import torch
    import chunk_util as ch
    new, old = [200, 90], [20, 100]
    cache, seqs, q, cu_new = ch.setup(new, old, 4, hkv, d, dtype, 16, seed=4)
    want = _chunk(cache, seqs, q, cu_new)
    lam, weight = _params(2, d, 2)
    at = {0: 150, 1: 130}                       # positions of the keys that are not finite
    early, total = [p - o for p, o in zip(at.values(), old)], list(at.values())
    for what in ("k", "v"):
        for x in (float("nan"), float("inf")):
            t = cache.k.clone(), cache.v.clone()
            for b, p in at.items():
                page = int(seqs.page_table[b, p // 16])
                t["kv".index(what)][0, page, :, p % 16, 3] = x
            bad = last.Cache(*t)
            out, lse, _ = _chunk(bad, seqs, q, cu_new)
            ch.check_chunk(cache, seqs, q, cu_new, out, lse, early, total)     # the rows before, over the keys before
            for b in at:
                t0, first = int(cu_new[b]), early[b]
                assert torch.equal(lse[t0:t0 + first], want[1][t0:t0 + first])
                late = out[t0 + first:t0 + new[b]]
                if what == "v":
                    assert not torch.isfinite(late[..., 3]).any() and torch.isfinite(late[..., 4:]).all()
                elif x != x:
                    assert late.isnan().all()
            if d > 128:
                continue
            got, _ = _diff(bad, seqs, q, cu_new, lam, weight)
            ch.check_diff(cache, seqs, q, cu_new, got, lam, early, total, weight=weight)
            plain, _ = _diff(bad, seqs, q, cu_new, lam)
            ch.check_diff(cache, seqs, q, cu_new, plain, lam, early, total)
            if what == "v":
                for b in at:
                    late = plain[int(cu_new[b]) + early[b]:int(cu_new[b]) + new[b]]
                    assert not torch.isfinite(late[..., 3]).any() and torch.isfinite(late[..., 4:d]).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinite_logits(dtype):
    """Keys whose logits are -inf take no part, a row of nothing else is empty."""
    import torch
    import chunk_util as ch
    new, old = [50, 50], [150, 100]
    cache, seqs, q, cu_new = ch.setup(new, old, 2, 2, 64, dtype, 16)
    q[:] = q.abs() + 0.01
    def put(b, at):
        at = torch.as_tensor(at, device="cuda")
        cache.k[0, seqs.page_table[b].long()[at // 16], :, at % 16] = -float("inf")
    put(0, [*range(0, 64), *range(70, 90), 199])
    put(1, list(range(150)))
    out, lse, _ = _chunk(cache, seqs, q, cu_new)
    assert (out[50:] == 0).all() and (lse[50:] == -math.inf).all()
    live = torch.ones(200, dtype=torch.bool, device="cuda")
    live[[*range(0, 64), *range(70, 90), 199]] = False
    for h in range(2):
        k, v = ch.keys_of(cache, seqs.page_table[0], 200, h)
        see = ch.seen(50, 200, 0, True, 0) & live
        want, want_lse, size, ez = ch.one_map(q[:50, h], torch.where(live[:, None], k, 0), v, see, 0.125)
        assert ((out[:50, h].double() - want).abs() <= ch.relative(ez, 200, dtype) * size + ch.UNIT[dtype] * want.abs()).all()
    lam, weight = _params(1, 64, 2)
    diff, _ = _diff(cache, seqs, q, cu_new, lam, weight)
    assert (diff[50:] == 0).all() and torch.isfinite(diff).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_views_layers_and_rows_of_no_sequence(dtype):
    """q inside a fused projection, out inside a wider row, K and V of one tensor, a layer of several, rows behind the last sequence."""
    import torch
    import cache_util as cu
    import chunk_util as ch
    new, lens, hq, hkv, d, size = [33, 0, 50], [33, 4, 150], 6, 2, 64, 16
    kv = cu.randn((3, 20, 2, size, hkv, d), dtype, 1)
    cache = last.Cache(kv[:, :, 0].transpose(2, 3), kv[:, :, 1].transpose(2, 3))
    table, _ = cu.table(lens, size, 20, 2)
    seqs = last.Sequences(table, cu.ints(lens))
    cu_new = cu.ints([0, 33, 33, 83])
    fused = cu.randn((90, (hq + 2 * hkv) * d), dtype, 3)
    q = fused[:, :hq * d].unflatten(1, (hq, d))
    lam, weight = _params(hq // 2, d, 4)
    ws = ch.workspace(cache, hq)
    for layer in range(3):
        part = last.Cache(cache.k[layer:layer + 1], cache.v[layer:layer + 1])
        out = torch.full((90, hq * d + 64), 7.0, dtype=q.dtype, device="cuda")
        lse = torch.full((90, hq), 7.0, device="cuda")
        o = out[:, 64:].unflatten(1, (hq, d))
        last.last_cache_chunk_attention(cache, layer, seqs, q, o, ws, cu_new=cu_new, lse=lse)
        last.last_poll(ws)
        ch.check_chunk(part, seqs, q, cu_new, o, lse, new, lens)
        assert (out[:, :64] == 7).all() and (out[83:] == 7).all() and (lse[83:] == 7).all()
        out.fill_(7.0)
        o = out[:, 64:].unflatten(1, (hq // 2, 2 * d))
        last.last_cache_diff_attention(cache, layer, seqs, q, o, ws, lam, cu_new=cu_new, norm_weight=weight)
        last.last_poll(ws)
        ch.check_diff(part, seqs, q, cu_new, o, lam, new, lens, weight=weight)
        assert (out[:, :64] == 7).all() and (out[83:] == 7).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_offsets_past_32_bits(dtype):
    """Pages 5 GB apart, tokens of q and out 3 GB apart."""
    import torch
    import cache_util as cu
    import chunk_util as ch
    e = 4 if dtype == "float32" else 2
    far, row = 5 * 2**30 // e, 3 * 2**30 // e
    base = [torch.empty(2 * far + 4096, dtype=getattr(torch, dtype), device="cuda") for _ in range(2)]
    k, v = (b.as_strided((1, 3, 2, 16, 64), (0, far, 1024, 64, 1)) for b in base)
    for i, t in enumerate((k, v)):
        t.copy_(cu.randn((1, 3, 2, 16, 64), dtype, i))
    cache, seqs = last.Cache(k, v), last.Sequences(cu.ints([[2, 0, 1]]), cu.ints([47]))
    wide = [torch.empty(4 * row + 4096, dtype=k.dtype, device="cuda") for _ in range(2)]
    q, out = wide[0].as_strided((5, 4, 64), (row, 64, 1)), wide[1].as_strided((5, 4, 64), (row, 64, 1))
    q.copy_(cu.randn((5, 4, 64), dtype, 5))
    ws, cu_new = ch.workspace(cache, 4), cu.ints([0, 5])
    last.last_cache_chunk_attention(cache, 0, seqs, q, out, ws, cu_new=cu_new)
    last.last_poll(ws)
    ch.check_chunk(cache, seqs, q, cu_new, out, None, [5], [47])
    lam, weight = _params(2, 64, 4)
    out = wide[1].as_strided((5, 2, 128), (row, 128, 1))
    last.last_cache_diff_attention(cache, 0, seqs, q, out, ws, lam, cu_new=cu_new, norm_weight=weight)
    last.last_poll(ws)
    ch.check_diff(cache, seqs, q, cu_new, out, lam, [5], [47], weight=weight)


@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hq,hkv,d,size", [(4, 2, 64, 16), (6, 2, 80, 24), (2, 2, 128, 8), (16, 2, 64, 64), (6, 2, 256, 40), (20, 2, 128, 128)])
def test_keys_of_bad_pages_are_left_out(hq, hkv, d, size, dtype, order):
    import torch
    import cache_util as cu
    import chunk_util as ch
    new, lens = [300, 31, 64, 1, 30, 7], [300, 301, 64, 257, 30, 2000]
    pool = sum(-(-n // size) for n in lens) + 1
    k, v = cu.pages(1, pool, hkv, size, d, dtype, order, 1)
    table, _ = cu.table(lens, size, pool - 1, 2)
    table = torch.where(table >= 0, table + 1, table)
    for t in (k, v):
        t[0, 0] = float("nan")                                    # page 0 is nobody's
    pages = [-(-n // size) for n in lens]
    bad = {1: [0], 2: list(range(pages[2])), 3: [pages[3] - 1, pages[3] // 2], 5: list(range(1, pages[5], 2))}
    broken = table.clone()
    for b, at in bad.items():
        for i, p in enumerate(at):
            broken[b, p] = (-1, pool, 2**31 - 1, -2**31)[i % 4]
    cache, q = last.Cache(k, v), cu.randn((sum(new), hq, d), dtype, 3)
    cu_new = cu.ints(np.concatenate([[0], np.cumsum(new)]))
    out, lse, ws = _chunk(cache, last.Sequences(broken, cu.ints(lens)), q, cu_new, poll=False)
    with pytest.raises(last.LastError) as e:
        last.last_poll(ws)
    assert e.value.status == last.LAST_ERR_DEVICE_INDEX
    seqs = last.Sequences(table, cu.ints(lens))
    ch.check_chunk(cache, seqs, q, cu_new, out, lse, new, lens, bad=bad)
    if d > 128:
        return
    lam, weight = _params(hq // 2, d, 4)
    out, ws = _diff(cache, last.Sequences(broken, cu.ints(lens)), q, cu_new, lam, weight, poll=False)
    with pytest.raises(last.LastError):
        last.last_poll(ws)
    ch.check_diff(cache, seqs, q, cu_new, out, lam, new, lens, weight=weight, bad=bad)


@pytest.mark.parametrize("dtype", DTYPES)
def test_sequences_of_bad_lengths_and_offsets(dtype):
    """A length or first key out of range: rows without a key.  Offsets out of range: rows left as they were.  The others get theirs."""
    import torch
    import cache_util as cu
    import chunk_util as ch
    new, old = [10, 40, 5, 70, 5], [90, 260, 45, 630, 0]
    lens = [a + b for a, b in zip(new, old)]
    cache, seqs, q, cu_new = ch.setup(new, old, 4, 2, 64, dtype, 16)
    room, others = seqs.page_table.shape[1] * 16, [0, 2, 3, 4]
    lam, weight = _params(2, 64, 4)
    for n, begin in ((room + 1, 0), (2**31 - 1, 0), (-1, 0), (39, 0), (-2**31, 0), (300, -1), (300, -2**31)):
        lens_dev, first = cu.ints(lens), cu.ints([0] * 5)
        lens_dev[1], first[1] = n, begin
        s = last.Sequences(seqs.page_table, lens_dev, first)
        out, lse, ws = _chunk(cache, s, q, cu_new, poll=False)
        with pytest.raises(last.LastError) as e:
            last.last_poll(ws)
        assert e.value.status == last.LAST_ERR_DEVICE_INDEX
        assert (out[10:50] == 0).all() and (lse[10:50] == -math.inf).all(), (n, begin)
        ch.check_chunk(cache, seqs, q, cu_new, out, lse, new, lens, only=others)
        diff, ws = _diff(cache, s, q, cu_new, lam, weight, poll=False)
        with pytest.raises(last.LastError):
            last.last_poll(ws)
        assert (diff[10:50] == 0).all()
        ch.check_diff(cache, seqs, q, cu_new, diff, lam, new, lens, weight=weight, only=others)
    # the rows that no valid pair of offsets covers any more
    for at, value, rows in ((1, 51, None), (1, -1, slice(0, 50)), (2, 2**31 - 1, slice(10, 55)), (2, 5, None)):
        broken = cu_new.clone()
        broken[at] = value
        out, lse, ws = _chunk(cache, seqs, q, broken, poll=False)
        with pytest.raises(last.LastError) as e:
            last.last_poll(ws)
        assert e.value.status == last.LAST_ERR_DEVICE_INDEX
        ch.check_chunk(cache, seqs, q, cu_new, out, lse, new, lens, only=[3, 4])
        assert rows is None or (out[rows].isnan().all() and lse[rows].isnan().all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_sequences(dtype):
    """More sequences than threads, most of them without a new token or with a few."""
    import chunk_util as ch
    rng = np.random.default_rng(3)
    new = rng.integers(0, 4, 900)
    new[rng.random(900) < 0.5] = 0
    new[[7, 500]] = [90, 260]
    old = rng.integers(0, 60, 900)
    cache, seqs, q, cu_new = ch.setup(new, old, 4, 2, 64, dtype, 16, "token", seed=9)
    out, lse, _ = _chunk(cache, seqs, q, cu_new)
    picked = [7, 500, *np.flatnonzero(new)[::9].tolist()]
    ch.check_chunk(cache, seqs, q, cu_new, out, lse, new, new + old, only=picked)
    assert not out.isnan().any() and not lse.isnan().any()
    lam, weight = _params(2, 64, 4)
    diff, _ = _diff(cache, seqs, q, cu_new, lam, weight)
    ch.check_diff(cache, seqs, q, cu_new, diff, lam, new, new + old, weight=weight, only=picked)
    assert not diff.isnan().any()


@pytest.mark.parametrize("dtype,d", [("float32", 8), ("bfloat16", 64)])
def test_the_last_keys_of_the_longest_sequence(dtype, d):
    """A window at the end of the longest sequence; its pages are one page over and over."""
    import torch
    import cache_util as cu
    import chunk_util as ch
    n, keys, new, size = 2**31 - 256, 90, 20, 1 << 20
    k, v = cu.pages(1, 1, 2, size, d, dtype, "head", 1)
    table = torch.zeros((1, -(-n // size)), dtype=torch.int32, device="cuda")
    cache, q = last.Cache(k, v), cu.randn((new, 2, d), dtype, 3)
    seqs, cu_new = last.Sequences(table, cu.ints([n]), cu.ints([n - keys])), cu.ints([0, new])
    out, lse, _ = _chunk(cache, seqs, q, cu_new)
    at = (torch.arange(n - keys, n, device="cuda") % size).long()
    see = ch.seen(new, keys, 0, True, 0)
    for h in range(2):
        want, _, mass, ez = ch.one_map(q[:, h], k[0, 0, h, at], v[0, 0, h, at], see, 1 / math.sqrt(d))
        assert ((out[:, h].double() - want).abs() <= ch.relative(ez, keys, dtype) * mass + ch.UNIT[dtype] * want.abs()).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_repeats_streams_and_graphs_give_the_same_bits(dtype):
    """A captured call replayed while lengths, tables and queries change in place; two graphs by turns on one workspace."""
    import torch
    import chunk_util as ch
    new, old = [5, 1, 130, 40], [700, 33, 0, 2000]
    cache, seqs, q, cu_new = ch.setup(new, old, 8, 2, 128, dtype, 16, "token", seed=4)
    lam, weight = _params(4, 128, 2)
    want, lse, _ = _chunk(cache, seqs, q, cu_new)
    diff, _ = _diff(cache, seqs, q, cu_new, lam, weight)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for stream in (None, s):
        with torch.cuda.stream(stream):
            got = _chunk(cache, seqs, q, cu_new, stream=stream)
            d2, _ = _diff(cache, seqs, q, cu_new, lam, weight, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want) and torch.equal(got[1], lse) and torch.equal(d2, diff)
    ws, out, dout = ch.workspace(cache, 8), torch.empty_like(q), torch.empty_like(diff)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0]):
        last.last_cache_chunk_attention(cache, 0, seqs, q, out, ws, cu_new=cu_new)
    with torch.cuda.graph(graphs[1]):
        last.last_cache_diff_attention(cache, 0, seqs, q, dout, ws, lam, cu_new=cu_new, norm_weight=weight)
    for step in range(3):
        out.fill_(float("nan"))
        dout.fill_(float("nan"))
        graphs[step & 1].replay()
        graphs[1 - (step & 1)].replay()
        last.last_poll(ws)
        eager, eager_diff = _chunk(cache, seqs, q, cu_new)[0], _diff(cache, seqs, q, cu_new, lam, weight)[0]
        assert torch.equal(out, eager) and torch.equal(dout, eager_diff)
        seqs.lens.sub_(1).clamp_(min=130)     # other lengths, in place
        seqs.lens[1] = 34 - step
        q.mul_(-0.5)


def test_host_threads():
    """Threads with problems of other sizes, head widths and types, each on its own stream and workspace."""
    import threading
    import torch
    import chunk_util as ch
    calls = []
    for i, (new, old, hq, hkv, d, dtype) in enumerate([([70, 3], [500, 9], 4, 2, 128, "bfloat16"), ([9] * 40, [50] * 40, 8, 8, 64, "float32"),
                                                       ([500], [0], 16, 2, 256, "bfloat16"), ([33, 0, 200], [1, 1, 1], 12, 2, 80, "bfloat16")]):
        cache, seqs, q, cu_new = ch.setup(new, old, hq, hkv, d, dtype, 16, seed=20 + i)
        calls.append((cache, seqs, q, cu_new, torch.empty_like(q), ch.workspace(cache, hq), torch.cuda.Stream()))
    torch.cuda.synchronize()
    want = []
    for cache, seqs, q, cu_new, out, ws, _ in calls:
        last.last_cache_chunk_attention(cache, 0, seqs, q, out, ws, cu_new=cu_new)
        want.append(out.clone())
    torch.cuda.synchronize()
    errors, start = [], threading.Barrier(len(calls))

    def work(i):
        cache, seqs, q, cu_new, out, ws, s = calls[i]
        start.wait()
        try:
            for r in range(100):
                last.last_cache_chunk_attention(cache, 0, seqs, q, out, ws, cu_new=cu_new, stream=s)
                if r % 50 == 49:
                    s.synchronize()
        except Exception as e:   # reported by the main thread
            errors.append(f"thread {i}: {e}")
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    assert all(torch.equal(c[4], w) for c, w in zip(calls, want))


@pytest.mark.parametrize("dtype", DTYPES)
def test_empty_calls_and_refusals(dtype):
    import torch
    import cache_util as cu
    import chunk_util as ch
    cache, seqs, q, cu_new = ch.setup([10, 20], [0, 3], 4, 2, 64, dtype, 16)
    out, ws = torch.empty_like(q), ch.workspace(cache, 4)
    lam, weight = _params(2, 64, 1)
    wide = out.view(30, 2, 128)
    none = last.Sequences(seqs.page_table[:0], seqs.lens[:0])
    last.last_cache_chunk_attention(cache, 0, none, q[:0], out[:0], ws)
    last.last_cache_chunk_attention(cache, 0, none, q[:0], out[:0], ws, cu_new=cu_new[:1])
    last.last_cache_chunk_attention(cache, 0, seqs, q[:0], out[:0], ws, cu_new=cu.ints([0, 0, 0]))
    last.last_cache_diff_attention(cache, 0, none, q[:0], wide[:0], ws, lam)
    last.last_poll(ws)
    for args in ((q[:1], out), (q, out[:29]), (q.double(), out.double()), (q[:, :, :32], out[:, :, :32]), (q, out[:, ::2]),
                 (q.cpu(), out.cpu()), (q.transpose(0, 1), out)):
        with pytest.raises(ValueError):
            last.last_cache_chunk_attention(cache, 0, seqs, *args, ws, cu_new=cu_new)
    for kw in (dict(cu_new=cu_new[:2]), dict(cu_new=cu_new.long()), dict(lse=torch.empty(30, 4, dtype=torch.float64, device="cuda")),
               dict(lse=torch.empty(29, 4, device="cuda"))):
        with pytest.raises(ValueError):
            last.last_cache_chunk_attention(cache, 0, seqs, q, out, ws, **{"cu_new": cu_new, **kw})
    for args, kw in (((q, out, ws, lam), {}), ((q, wide, ws, None), {}), ((q, wide, ws, lam[:1]), {}), ((q, wide, ws, lam.double()), {}),
                     ((q, wide, ws, lam), dict(norm_weight=weight[:64]))):
        with pytest.raises(ValueError):
            last.last_cache_diff_attention(cache, 0, seqs, *args, cu_new=cu_new, **kw)
    for kw, status in ((dict(window=-1), last.LAST_ERR_INVALID_ARG), (dict(window=3, causal=False), last.LAST_ERR_INVALID_ARG),
                       (dict(cu_new=None), last.LAST_ERR_INVALID_ARG)):
        with pytest.raises(last.LastError) as e:
            last.last_cache_chunk_attention(cache, 0, seqs, q, out, ws, **{"cu_new": cu_new, **kw})
        assert e.value.status == status
    for kw in (dict(norm_eps=-1.0), dict(norm_eps=float("nan")), dict(out_scale=float("inf"))):
        with pytest.raises(last.LastError) as e:
            last.last_cache_diff_attention(cache, 0, seqs, q, wide, ws, lam, cu_new=cu_new, norm_weight=weight, **kw)
        assert e.value.status == last.LAST_ERR_INVALID_ARG
    with pytest.raises(last.LastError) as e:
        last.last_cache_chunk_attention(cache, 0, seqs, q, out, ws[:1024], cu_new=cu_new)
    assert e.value.status == last.LAST_ERR_WORKSPACE_TOO_SMALL
    with pytest.raises(last.LastError) as e:
        last.last_cache_chunk_attention(cache, 1, seqs, q, out, ws, cu_new=cu_new)
    assert e.value.status == last.LAST_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_prompt_in_chunks_is_the_prompt_at_once(dtype):
    """Appended and attended chunk by chunk, then token by token, over one cache: what one call over the whole prompt gives."""
    import torch
    import cache_util as cu
    import chunk_util as ch
    n, hq, hkv, d, size = 333, 8, 4, 64, 16
    k, v = cu.pages(1, 30, hkv, size, d, dtype, "head", 1, fill=float("nan"))
    cache = last.Cache(k, v)
    table, _ = cu.table([n], size, 30, 3)
    q, kn, vn = cu.randn((n, hq, d), dtype, 4), cu.randn((n, hkv, d), dtype, 5), cu.randn((n, hkv, d), dtype, 6)
    lens = cu.ints([0])
    seqs = last.Sequences(table, lens)
    cws, ws = cu.workspace(cache, 1, hq), ch.workspace(cache, hq)
    lam, weight = _params(hq // 2, d, 2)
    rope = last.Rope.sections([32])
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    q_rot, out, diff = torch.empty_like(q), torch.empty_like(q), torch.empty((n, hq // 2, 2 * d), dtype=q.dtype, device="cuda")
    at = 0
    for m in (128, 100, 64, 37, 1, 1, 1, 1):
        part, one = slice(at, at + m), m == 1
        lens += m
        cu_new = None if one else cu.ints([0, m])
        last.last_cache_append(cache, 0, seqs, kn[part], vn[part], cws, cu_new=cu_new, rope=rope, positions=pos[part], q=q[part],
                               q_out=q_rot[part])
        last.last_cache_chunk_attention(cache, 0, seqs, q_rot[part], out[part], ws, cu_new=cu_new)
        last.last_cache_diff_attention(cache, 0, seqs, q_rot[part], diff[part], ws, lam, cu_new=cu_new, norm_weight=weight)
        last.last_poll(cws)
        last.last_poll(ws)
        at += m
    assert at == n
    cu_new = cu.ints([0, n])
    ch.check_chunk(cache, seqs, q_rot, cu_new, out, None, [n], [n])
    ch.check_diff(cache, seqs, q_rot, cu_new, diff, lam, [n], [n], weight=weight)

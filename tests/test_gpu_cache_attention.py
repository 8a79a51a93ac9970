"""Attention of one new token over a paged cache against softmax in 64 bits."""
import math

import numpy as np
import pytest

import paper_2607_27952_gb300 as last

pytestmark = pytest.mark.gpu


def _setup(lens, hq, hkv, d, dtype, size, order, seed=0, begin=None, stale=None, qscale=1.0):
    import torch
    import cache_util as cu
    pool = sum(-(-int(n) // size) for n in lens) + 2
    k, v = cu.pages(1, pool, hkv, size, d, dtype, order, seed + 1)
    table, rest = cu.table(lens, size, pool, seed)
    if stale is not None:      # what no sequence's keys are
        used = torch.zeros((pool, size), dtype=torch.bool, device="cuda")
        for b, n in enumerate(lens):
            i = torch.arange(0 if begin is None else min(int(begin[b]), int(n)), int(n), device="cuda")
            used[table[b].long()[i // size], i % size] = True
        for t in (k, v):
            t[0].transpose(1, 2)[~used] = stale
    q = cu.randn((len(lens), hq, d), dtype, seed + 3, qscale)
    cache = last.Cache(k, v)
    seqs = last.Sequences(table, cu.ints(lens), None if begin is None else cu.ints(begin))
    return cache, seqs, q


def _run(cache, seqs, q, scale=0.0, stream=None):
    import torch
    import cache_util as cu
    out = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:2], float("nan"), dtype=torch.float32, device="cuda")
    ws = cu.workspace(cache, seqs.batch, q.shape[1])
    last.last_cache_attention(cache, 0, seqs, q, out, ws, lse=lse, softmax_scale=scale, stream=stream)
    last.last_poll(ws, stream)
    return out, lse


def _check(cache, seqs, q, out, lse, lens, begin=None, scale=None):
    import torch
    import cache_util as cu
    scale = 1 / math.sqrt(cache.head_dim) if scale is None else scale
    dtype = str(q.dtype).rpartition(".")[2]
    for b, n in enumerate(lens):
        first = 0 if begin is None else min(int(begin[b]), int(n))
        k, v = (cu.rows(t, seqs.page_table[b], int(n), cache.page_size)[0][:, first:] for t in (cache.k, cache.v))
        want, want_lse, size = cu.attention(q[b], k, v, scale)
        ez, rel, u = cu.attention_bounds(q[b], k, scale, int(n) - first, dtype)
        err = (out[b].double() - want).abs()
        tol = rel * size + u * want.abs()
        assert (err <= tol).all(), f"sequence {b} ({n} keys): worst {(err - tol).max():.3e} past the bound"
        if n == first:
            assert (lse[b] == -math.inf).all()
        else:
            assert ((lse[b].double() - want_lse).abs() <= 2 * ez + 2.0 ** -20 * (1 + want_lse.abs())
                    + (n / 8 + 64) * 2.0 ** -24).all()


LENS = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 129, 500]


@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("hq,hkv,d,size", [
    (1, 1, 64, 16), (4, 4, 128, 16), (12, 2, 128, 32), (14, 2, 64, 8), (16, 2, 80, 24), (9, 1, 128, 64),
    (16, 1, 128, 48), (32, 2, 64, 96), (34, 2, 72, 16), (40, 1, 128, 128), (6, 2, 256, 16), (20, 2, 192, 40),
    (3, 1, 8, 256), (10, 5, 16, 16), (5, 1, 136, 72), (48, 1, 256, 56),
])
def test_lengths_heads_and_pages(hq, hkv, d, size, dtype, order):
    cache, seqs, q = _setup(LENS, hq, hkv, d, dtype, size, order, stale=float("nan"))
    out, lse = _run(cache, seqs, q)
    _check(cache, seqs, q, out, lse, LENS)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size", [8, 16, 64, 80])
def test_key_begin(size, dtype):
    """Windows that start anywhere, end anywhere, hold one key or none; what lies before them is never used."""
    import torch
    lens = [100, 100, 100, 100, 700, 700, 700, 64, 64, 65, 5]
    begin = [0, 1, 99, 100, 64, 65, 640, 63, 64, 64, 9]
    cache, seqs, q = _setup(lens, 8, 2, 128, dtype, size, "head", begin=begin, stale=float("inf"))
    table = seqs.page_table
    for b, f in enumerate(begin):      # pages before the window have been given back
        table[b, :min(f, lens[b]) // size] = -7
    out, lse = _run(cache, seqs, q)
    table.clamp_(min=0)                # for the plain form, which gathers them and leaves them out
    _check(cache, seqs, q, out, lse, lens, begin)
    assert (out[3] == 0).all() and (out[10] == 0).all() and torch.isfinite(out).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_many_sequences_and_long_ones(dtype):
    rng = np.random.default_rng(5)
    for lens in (rng.integers(0, 40, 700), [20011, 1, 0, 9000, 30000], [70001]):
        cache, seqs, q = _setup(lens, 4, 2, 64, dtype, 16, "head", seed=9)
        out, lse = _run(cache, seqs, q)
        _check(cache, seqs, q, out, lse, lens)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_large_and_rising_logits(dtype):
    """Logits of hundreds, the largest last or first, and an explicit scale."""
    import torch
    lens = [300, 300]
    cache, seqs, q = _setup(lens, 4, 1, 64, dtype, 16, "head", qscale=4.0)
    i = torch.arange(300, device="cuda")
    for b, w in ((0, i / 30.0), (1, (299 - i) / 30.0)):
        p = seqs.page_table[b].long()[i // 16]
        cache.k[0, p, 0, i % 16] = (q[b, 0].float()[None] * w[:, None].float()).to(q.dtype)
    for scale in (0.0, 0.75):
        out, lse = _run(cache, seqs, q, scale)
        _check(cache, seqs, q, out, lse, lens, scale=scale or None)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_infinite_logits(dtype):
    """Keys whose logits are -inf take no part, a sequence of nothing else is empty; NaN and +inf show."""
    import torch
    lens = [200, 200, 70, 130]
    cache, seqs, q = _setup(lens, 2, 1, 64, dtype, 16, "head")
    q[:] = q.abs() + 0.01
    def put(b, at, x):
        at = torch.as_tensor(at, device="cuda")
        cache.k[0, seqs.page_table[b].long()[at // 16], 0, at % 16] = x
    dead = [*range(0, 64), *range(70, 90), 199]
    put(0, dead, -float("inf"))
    put(1, list(range(200)), -float("inf"))
    put(2, [69], float("nan"))
    put(3, [3], float("inf"))
    out, lse = _run(cache, seqs, q)
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all()
    assert out[2].isnan().all() and lse[2].isnan().all()
    assert out[3].isnan().all() and not torch.isfinite(lse[3]).any()
    import cache_util as cu
    live = [i for i in range(200) if i not in dead]
    k, v = (cu.rows(t, seqs.page_table[0], 200, 16)[0][:, live] for t in (cache.k, cache.v))
    want, want_lse, size = cu.attention(q[0], k, v, 0.125)
    ez, rel, u = cu.attention_bounds(q[0], k, 0.125, len(live), dtype)
    assert ((out[0].double() - want).abs() <= rel * size + u * want.abs()).all()
    assert ((lse[0].double() - want_lse).abs() <= 2 * ez + 2.0 ** -18).all()


def test_infinite_values_of_live_keys_show():
    import torch
    cache, seqs, q = _setup([40], 2, 1, 64, "bfloat16", 16, "head")
    cache.v[0, seqs.page_table[0, 1].long(), 0, 3, 5] = float("inf")
    out, lse = _run(cache, seqs, q)
    assert (out[0, :, 5] == math.inf).all() and torch.isfinite(out[0, :, 6:]).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_views_and_layers(dtype):
    """q inside a fused projection, out inside a wider row, K and V of one tensor, a layer of several."""
    import torch
    import cache_util as cu
    lens, hq, hkv, d, size = [33, 0, 150], 6, 2, 64, 16
    kv = cu.randn((3, 20, 2, size, hkv, d), dtype, 1)
    cache = last.Cache(kv[:, :, 0].transpose(2, 3), kv[:, :, 1].transpose(2, 3))
    table, _ = cu.table(lens, size, 20, 2)
    wide = torch.nn.functional.pad(table, (0, 5), value=-1)[:, :table.shape[1]]
    seqs = last.Sequences(wide, cu.ints(lens))
    fused = cu.randn((3, (hq + 2 * hkv) * d), dtype, 3)
    q = fused[:, :hq * d].unflatten(1, (hq, d))
    out = torch.zeros((3, hq * d + 64), dtype=q.dtype, device="cuda")
    ws = cu.workspace(cache, 3, hq)
    for layer in range(3):
        o = out[:, 64:].unflatten(1, (hq, d))
        lse = torch.zeros((3, hq), device="cuda")
        last.last_cache_attention(cache, layer, seqs, q, o, ws, lse=lse)
        last.last_poll(ws)
        part = last.Cache(cache.k[layer:layer + 1], cache.v[layer:layer + 1])
        _check(part, seqs, q, o, lse, lens)
    assert (out[:, :64] == 0).all()
    last.last_cache_attention(cache, 0, seqs, q, o, ws)      # without lse


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_offsets_past_32_bits(dtype):
    """Pages 5 GB apart (3 of them, most of the storage never touched)."""
    import torch
    import cache_util as cu
    e = 4 if dtype == "float32" else 2
    far = 5 * 2**30 // e
    base = [torch.empty(2 * far + 4096, dtype=getattr(torch, dtype), device="cuda") for _ in range(2)]
    k, v = (b.as_strided((1, 3, 2, 16, 64), (0, far, 1024, 64, 1)) for b in base)
    for i, t in enumerate((k, v)):
        t.copy_(cu.randn((1, 3, 2, 16, 64), dtype, i))
    cache, seqs = last.Cache(k, v), last.Sequences(cu.ints([[2, 0, 1]]), cu.ints([47]))
    q = cu.randn((1, 4, 64), dtype, 5)
    out, lse = _run(cache, seqs, q)
    _check(cache, seqs, q, out, lse, [47])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_repeats_and_streams_give_the_same_bits(dtype):
    import torch
    rng = np.random.default_rng(1)
    lens = rng.integers(1, 3000, 20)
    cache, seqs, q = _setup(lens, 8, 2, 128, dtype, 16, "token", seed=4)
    want = _run(cache, seqs, q)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for stream in (None, s, None):
        with torch.cuda.stream(stream):
            got = _run(cache, seqs, q, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_empty_batch_and_refusals():
    import torch
    import cache_util as cu
    cache, seqs, q = _setup([10, 20], 4, 2, 64, "bfloat16", 16, "head")
    out, ws = torch.empty_like(q), cu.workspace(cache, 2, 4)
    none = last.Sequences(seqs.page_table[:0], seqs.lens[:0])
    last.last_cache_attention(cache, 0, none, q[:0], out[:0], ws)
    last.last_poll(ws)
    for args in ((q[:1], out), (q.float(), out.float()), (q[:, :, :32], out[:, :, :32]), (q, out[:, ::2]),
                 (q.cpu(), out.cpu()), (q.transpose(0, 1), out)):
        with pytest.raises(ValueError):
            last.last_cache_attention(cache, 0, seqs, *args, ws)
    with pytest.raises(ValueError):
        last.last_cache_attention(cache, 0, seqs, q, out, ws, lse=torch.empty(2, 4, dtype=torch.float64, device="cuda"))
    with pytest.raises(ValueError):
        last.Sequences(seqs.page_table.long(), seqs.lens)
    with pytest.raises(ValueError):
        last.Sequences(seqs.page_table, seqs.lens[:1])
    with pytest.raises(ValueError):
        last.Cache(cache.k, cache.v.float())
    with pytest.raises(ValueError):
        last.Cache(cache.k, cache.v[:, :-1])
    with pytest.raises(last.LastError) as e:
        last.last_cache_attention(cache, 1, seqs, q, out, ws)
    assert e.value.status == last.LAST_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_bad_pages_and_lengths_are_reported(dtype):
    """The call flags them, leaves the other sequences right, and the next good call on the workspace is clean."""
    import torch
    import cache_util as cu
    lens = [100, 300, 50]
    cache, seqs, q = _setup(lens, 4, 2, 64, dtype, 16, "head")
    out, ws = torch.zeros_like(q), cu.workspace(cache, 3, 4)
    good = torch.zeros_like(q)
    last.last_cache_attention(cache, 0, seqs, q, good, ws)
    last.last_poll(ws)
    pool = cache.k.shape[1]
    for where, value in (("table", -1), ("table", pool), ("table", 2**31 - 1), ("lens", 10**6), ("lens", -3),
                         ("begin", -1)):
        t, n = seqs.page_table.clone(), seqs.lens.clone()
        begin = torch.zeros_like(n) if where == "begin" else None
        {"table": t[1, 7:8], "lens": n[1:2], "begin": begin[1:2] if begin is not None else None}[where].fill_(value)
        last.last_cache_attention(cache, 0, last.Sequences(t, n, begin), q, out, ws)
        with pytest.raises(last.LastError) as e:
            last.last_poll(ws)
        assert e.value.status == last.LAST_ERR_DEVICE_INDEX
        assert torch.equal(out[0], good[0]) and torch.equal(out[2], good[2])
        last.last_cache_attention(cache, 0, seqs, q, out, ws)
        last.last_poll(ws)
        assert torch.equal(out, good)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("hq,hkv,d,lens", [(16, 1, 128, [40000]), (40, 1, 64, [25000]), (9, 3, 256, [6000, 9000]), (32, 2, 128, [3000, 0, 777])])
def test_long_sequences_of_many_heads(hq, hkv, d, lens, dtype):
    """A (sequence, kv-head) spread over a few CTAs or over all of them, several passes of heads."""
    cache, seqs, q = _setup(lens, hq, hkv, d, dtype, 32, "head", seed=3)
    out, lse = _run(cache, seqs, q)
    _check(cache, seqs, q, out, lse, lens)


def test_host_threads():
    """Threads with problems of other sizes, head widths and types, each on its own stream and workspace."""
    import threading
    import torch
    import cache_util as cu
    calls = []
    for i, (lens, hq, hkv, d, dtype) in enumerate([([700, 3], 4, 2, 128, "bfloat16"), ([90] * 40, 8, 8, 64, "float32"), ([5000], 16, 1, 256, "bfloat16"),
                                                   ([33, 0, 2000], 12, 2, 80, "float32")]):
        cache, seqs, q = _setup(lens, hq, hkv, d, dtype, 16, "head", seed=20 + i)
        calls.append((cache, seqs, q, torch.empty_like(q), cu.workspace(cache, len(lens), hq), torch.cuda.Stream()))
    torch.cuda.synchronize()
    want = []
    for cache, seqs, q, out, ws, _ in calls:
        last.last_cache_attention(cache, 0, seqs, q, out, ws)
        want.append(out.clone())
    torch.cuda.synchronize()
    errors, start = [], threading.Barrier(len(calls))

    def work(i):
        cache, seqs, q, out, ws, s = calls[i]
        start.wait()
        try:
            for r in range(200):
                last.last_cache_attention(cache, 0, seqs, q, out, ws, stream=s)
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
    assert all(torch.equal(c[3], w) for c, w in zip(calls, want))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_mostly_empty_batches(dtype):
    """Long runs of sequences without a key between those that have some."""
    lens = np.zeros(2000, int)
    lens[[3, 40, 41, 700, 1290, 1999]] = [5, 300, 1, 64, 2000, 130]
    cache, seqs, q = _setup(lens, 4, 2, 64, dtype, 16, "token", seed=12)
    out, lse = _run(cache, seqs, q)
    live = np.flatnonzero(lens)
    import torch
    empty = torch.ones(2000, dtype=torch.bool, device="cuda")
    empty[torch.as_tensor(live).cuda()] = False
    assert (out[empty] == 0).all() and (lse[empty] == -math.inf).all()
    part = last.Sequences(seqs.page_table[live.tolist()].contiguous(), seqs.lens[live.tolist()].contiguous())
    _check(cache, part, q[live.tolist()], out[live.tolist()], lse[live.tolist()], lens[live])


# ---- what a call may not depend on ----

@pytest.mark.parametrize("hq,hkv,d,dtype", [
    (4, 2, 64, "float32"), (6, 2, 128, "float32"), (3, 1, 80, "float32"), (12, 2, 64, "float32"), (14, 2, 128, "float32"),
    (5, 1, 256, "float32"), (20, 2, 64, "float32"), (20, 1, 128, "float32"), (9, 1, 256, "float32"),
    (12, 2, 64, "bfloat16"), (20, 1, 128, "bfloat16"), (9, 1, 256, "bfloat16"),
])
def test_what_shared_memory_held_decides_no_bits(hq, hkv, d, dtype):
    """Groups that leave some of the heads a kernel holds without a query: calls of full groups with queries of no, of
    common and of huge size in between change nothing."""
    import torch
    import cache_util as cu
    rng = np.random.default_rng(2)
    lens = rng.integers(1, 2500, 24)
    cache, seqs, q = _setup(lens, hq, hkv, d, dtype, 16, "head", seed=6)
    want = _run(cache, seqs, q)
    _check(cache, seqs, q, *want, lens)
    for full in (4, 8, 16):
        for scale in (0.0, 3.0, 1e4):
            _run(cache, seqs, cu.randn((len(lens), full * hkv, d), dtype, 30 + full, scale))
            got = _run(cache, seqs, q)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (full, scale)


@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("hq,hkv,d,size", [(4, 2, 64, 16), (6, 2, 80, 24), (1, 1, 128, 8), (16, 1, 64, 64), (3, 1, 256, 40), (20, 1, 128, 128)])
def test_keys_of_bad_pages_are_left_out(hq, hkv, d, size, dtype, order):
    """A sequence with pages out of range attends over its other keys alone, and is empty without any; no
    page that it does not name (page 0 among them) is used in their place."""
    import torch
    import cache_util as cu
    lens = [300, 301, 64, 257, 30, 2000]
    pool = sum(-(-n // size) for n in lens) + 1
    k, v = cu.pages(1, pool, hkv, size, d, dtype, order, 1)
    table, _ = cu.table(lens, size, pool - 1, 2)
    table = torch.where(table >= 0, table + 1, table)
    for t in (k, v):
        t[0, 0] = float("nan")                                    # page 0 is nobody's
    cache, q = last.Cache(k, v), cu.randn((len(lens), hq, d), dtype, 3)
    pages = [-(-n // size) for n in lens]
    bad = {1: [0], 2: list(range(pages[2])), 3: [pages[3] - 1, pages[3] // 2], 5: list(range(1, pages[5], 2))}
    broken = table.clone()
    for b, at in bad.items():
        for i, p in enumerate(at):
            broken[b, p] = (-1, pool, 2**31 - 1, -2**31)[i % 4]
    out, lse = torch.full_like(q, float("nan")), torch.full((len(lens), hq), float("nan"), device="cuda")
    ws, scale = cu.workspace(cache, len(lens), hq), 1 / math.sqrt(d)
    last.last_cache_attention(cache, 0, last.Sequences(broken, cu.ints(lens)), q, out, ws, lse=lse)
    with pytest.raises(last.LastError) as e:
        last.last_poll(ws)
    assert e.value.status == last.LAST_ERR_DEVICE_INDEX
    for b, n in enumerate(lens):
        live = [i for i in range(n) if i // size not in bad.get(b, [])]
        kb, vb = (cu.rows(t, table[b], n, size)[0][:, live] for t in (k, v))
        want, want_lse, mass = cu.attention(q[b], kb, vb, scale)
        if not live:
            assert (out[b] == 0).all() and (lse[b] == -math.inf).all()
            continue
        ez, rel, u = cu.attention_bounds(q[b], kb, scale, len(live), dtype)
        assert ((out[b].double() - want).abs() <= rel * mass + u * want.abs()).all(), b
        assert ((lse[b].double() - want_lse).abs() <= 2 * ez + 2.0 ** -20 * (1 + want_lse.abs()) + (n / 8 + 64) * 2.0 ** -24).all(), b


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_sequences_of_bad_length_are_empty(dtype):
    """A length or first key out of range: the sequence gets what one without a key gets, the others theirs."""
    import torch
    import cache_util as cu
    lens = [100, 300, 50, 700, 5]
    cache, seqs, q = _setup(lens, 4, 2, 64, dtype, 16, "head")
    room = seqs.page_table.shape[1] * 16
    for n, begin in ((room + 1, 0), (2**31 - 1, 0), (-1, 0), (-2**31, 0), (300, -1), (300, -2**31), (room + 1, 290)):
        lens_dev, first = cu.ints(lens), cu.ints([0] * 5)
        lens_dev[1], first[1] = n, begin
        out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
        ws = cu.workspace(cache, 5, 4)
        last.last_cache_attention(cache, 0, last.Sequences(seqs.page_table, lens_dev, first), q, out, ws, lse=lse)
        with pytest.raises(last.LastError) as e:
            last.last_poll(ws)
        assert e.value.status == last.LAST_ERR_DEVICE_INDEX
        assert (out[1] == 0).all() and (lse[1] == -math.inf).all(), (n, begin)
        others = [0, 2, 3, 4]
        part = last.Sequences(seqs.page_table[others], seqs.lens[others])
        _check(cache, part, q[others], out[others], lse[others], [lens[b] for b in others])


@pytest.mark.parametrize("size", [8, 24, 1 << 20])
@pytest.mark.parametrize("dtype,d", [("float32", 8), ("bfloat16", 16), ("bfloat16", 64)])
def test_the_last_keys_that_32_bits_count(size, dtype, d):
    """A window at the end of the longest sequence that a length can say; its pages are one page over and over."""
    import torch
    import cache_util as cu
    n, keys = 2**31 - 1, 90
    k, v = cu.pages(1, 1, 1, size, d, dtype, "head", 1)
    table = torch.zeros((1, -(-n // size)), dtype=torch.int32, device="cuda")
    cache, q = last.Cache(k, v), cu.randn((1, 2, d), dtype, 3)
    seqs = last.Sequences(table, cu.ints([n]), cu.ints([n - keys]))
    out, lse = _run(cache, seqs, q)
    at = (torch.arange(n - keys, n, device="cuda") % size).long()
    want, want_lse, mass = cu.attention(q[0], k[0, 0][:, at], v[0, 0][:, at], 1 / math.sqrt(d))
    ez, rel, u = cu.attention_bounds(q[0], k[0, 0][:, at], 1 / math.sqrt(d), keys, dtype)
    assert ((out[0].double() - want).abs() <= rel * mass + u * want.abs()).all()
    assert ((lse[0].double() - want_lse).abs() <= 2 * ez + 2.0 ** -18).all()

"""Chunk and differential attention with few new tokens per sequence (bf16 has kernels of its own for them)."""
import numpy as np
import pytest

import paper_2607_27952_gb300 as last
from test_gpu_chunk_attention import DTYPES, _chunk, _diff, _params

pytestmark = pytest.mark.gpu

NEW = [1, 0, 3, 2, 1, 5, 0, 1]
OLD = [0, 5, 0, 63, 500, 130, 0, 64]
LENS = [a + b for a, b in zip(NEW, OLD)]
SHAPES = [(2, 2, 64, 16), (4, 2, 128, 8), (8, 2, 128, 32), (16, 2, 64, 24), (6, 2, 80, 24), (4, 2, 256, 16), (2, 1, 192, 40), (3, 1, 8, 256),
          (4, 2, 136, 72), (8, 2, 16, 16), (8, 4, 72, 8)]


@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 2), (True, 70)])
@pytest.mark.parametrize("hq,hkv,d,size", SHAPES)
def test_few_rows(hq, hkv, d, size, causal, window, order):
    import chunk_util as ch
    cache, seqs, q, cu_new = ch.setup(NEW, OLD, hq, hkv, d, "bfloat16", size, order, stale=float("nan"))
    out, lse, _ = _chunk(cache, seqs, q, cu_new, causal, window)
    ch.check_chunk(cache, seqs, q, cu_new, out, lse, NEW, LENS, None, causal, window)
    if d > 128 or hkv % 2:
        return
    for norm in (True, False):
        lam, weight = _params(hq // 2, d, 5, norm)
        out, _ = _diff(cache, seqs, q, cu_new, lam, weight, out_scale=0.7, causal=causal, window=window)
        ch.check_diff(cache, seqs, q, cu_new, out, lam, NEW, LENS, None, causal, window, weight=weight, out_scale=0.7)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [8, 16, 64])
def test_first_keys(size, dtype):
    """First keys before, inside and behind the new tokens."""
    import torch
    import chunk_util as ch
    new, old, begin = [3, 1, 2, 4, 1], [70, 64, 0, 300, 20], [0, 65, 1, 260, 20]
    lens = [a + b for a, b in zip(new, old)]
    cache, seqs, q, cu_new = ch.setup(new, old, 4, 2, 64, dtype, size, begin=begin, stale=float("inf"))
    for b, f in enumerate(begin):
        seqs.page_table[b, :min(f, lens[b]) // size] = -7
    lam, weight = _params(2, 64, 3)
    for causal, window in ((True, 0), (False, 0), (True, 40)):
        out, lse, _ = _chunk(cache, seqs, q, cu_new, causal, window)
        diff, _ = _diff(cache, seqs, q, cu_new, lam, weight, causal=causal, window=window)
        assert torch.isfinite(out).all() and torch.isfinite(diff).all()
        seqs.page_table.clamp_(min=0)      # for the plain form, which gathers them and leaves them out
        ch.check_chunk(cache, seqs, q, cu_new, out, lse, new, lens, begin, causal, window)
        ch.check_diff(cache, seqs, q, cu_new, diff, lam, new, lens, begin, causal, window, weight=weight)


@pytest.mark.parametrize("d", [64, 80, 128, 256])
def test_what_a_row_does_not_see_has_no_part(d):
    """Infinities and NaN in K and V of keys that only later rows see."""
    import torch
    import chunk_util as ch
    new, old, at = [4, 3], [100, 61], {0: 102, 1: 62}
    cache, seqs, q, cu_new = ch.setup(new, old, 4, 2, d, "bfloat16", 16, seed=4)
    want = _chunk(cache, seqs, q, cu_new)
    lam, weight = _params(2, d, 2)
    early, total = [p - o for p, o in zip(at.values(), old)], list(at.values())
    for what in ("k", "v"):
        for x in (float("nan"), float("inf")):
            t = cache.k.clone(), cache.v.clone()
            for b, p in at.items():
                t["kv".index(what)][0, int(seqs.page_table[b, p // 16]), :, p % 16, 3] = x
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


@pytest.mark.parametrize("hq,hkv,d,size", [(4, 2, 64, 16), (6, 2, 80, 24), (2, 2, 128, 8), (4, 2, 128, 64), (2, 2, 256, 40)])
def test_keys_of_bad_pages_are_left_out(hq, hkv, d, size):
    import torch
    import cache_util as cu
    import chunk_util as ch
    new, lens = [3, 1, 4, 1, 2, 1], [300, 301, 64, 257, 30, 2000]
    pool = sum(-(-n // size) for n in lens) + 1
    k, v = cu.pages(1, pool, hkv, size, d, "bfloat16", "head", 1)
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
    cache, q = last.Cache(k, v), cu.randn((sum(new), hq, d), "bfloat16", 3)
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
def test_one_long_prompt_among_single_tokens(dtype):
    """Few rows on average, many in one sequence; captured, with offsets that change in place."""
    import torch
    import chunk_util as ch
    new, old = [1] * 60 + [150] + [1] * 40, [40 + 3 * i for i in range(101)]
    lens = [a + b for a, b in zip(new, old)]
    cache, seqs, q, cu_new = ch.setup(new, old, 4, 2, 64, dtype, 16, seed=3)
    out, lse, _ = _chunk(cache, seqs, q, cu_new)
    picked = [0, 59, 60, 61, 100]
    ch.check_chunk(cache, seqs, q, cu_new, out, lse, new, lens, only=picked)
    lam, weight = _params(2, 64, 4)
    diff, _ = _diff(cache, seqs, q, cu_new, lam, weight)
    ch.check_diff(cache, seqs, q, cu_new, diff, lam, new, lens, weight=weight, only=picked)
    ws, again, graph = ch.workspace(cache, 4), torch.empty_like(q), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        last.last_cache_chunk_attention(cache, 0, seqs, q, again, ws, cu_new=cu_new)
    # the long prompt's tokens go to the first sequence
    moved = [150] + [1] * 59 + [1] + [1] * 40
    cu_new.copy_(torch.tensor(np.concatenate([[0], np.cumsum(moved)]), dtype=torch.int32))
    for _ in range(2):
        again.fill_(float("nan"))
        graph.replay()
    eager = _chunk(cache, seqs, q, cu_new, poll=False)[0]   # the first sequence is shorter than its new tokens: rows without a key
    assert torch.equal(again, eager) and not again.isnan().any()

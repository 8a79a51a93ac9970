"""Appending to a paged cache, cutting it to kept tokens and copying its pages: bit for bit against plain
indexing, and the operators together as a decode loop uses them."""
import math

import numpy as np
import pytest

import paper_2607_27952_gb300 as last

pytestmark = pytest.mark.gpu


def _bits(t):
    import torch
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


def _same(a, b):
    import torch
    return torch.equal(_bits(a), _bits(b))


# ---- append ----

@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("hq,hkv,d,size,new,old,sections,pairs", [
    (16, 2, 128, 16, [1] * 5, [0, 15, 16, 700, 3], [16, 24, 24], "half"),
    (4, 4, 64, 8, [0, 1, 33, 0, 64, 100], [5, 0, 7, 1, 0, 64], [32], "adjacent"),
    (6, 3, 80, 24, [300, 2], [0, 23], [6, 7, 7], "half"),
    (2, 1, 256, 40, [17], [0], [5, 4], "half"),            # 9 pairs, 238 elements copied
    (12, 2, 16, 16, [3, 3], [2, 2], None, "half"),         # no rotation
])
def test_append(hq, hkv, d, size, new, old, sections, pairs, dtype, order):
    import torch
    import cache_util as cu
    lens = [a + b for a, b in zip(new, old)]
    pool, t = sum(-(-n // size) for n in lens) + 2, sum(new)
    k, v = cu.pages(2, pool, hkv, size, d, dtype, order, 1)
    table, _ = cu.table(lens, size, pool, 3)
    cache, seqs = last.Cache(k, v), last.Sequences(table, cu.ints(lens))
    fused = cu.randn((t, hq + 2 * hkv, d), dtype, 4)
    q, kn, vn = fused.split([hq, hkv, hkv], dim=1)
    ws = cu.workspace(cache, len(lens), hq)
    want_k, want_v, kr = k.clone(), v.clone(), kn.clone()
    kw = {}
    if sections is not None:
        rope = last.Rope.sections(sections, pairs=pairs)
        pos = torch.randint(0, 5000, (len(sections), t), dtype=torch.int32, device="cuda")
        qo, want_q = torch.zeros((t, hq, d), dtype=q.dtype, device="cuda"), torch.empty((t, hq, d), dtype=q.dtype, device="cuda")
        last.last_rope(rope, pos, q, want_q, k=kn, k_out=kr)       # its own tests check it
        kw = dict(rope=rope, positions=pos, q=q, q_out=qo)
    cu_new = None if new == [1] * len(new) else cu.ints(np.concatenate([[0], np.cumsum(new)]))
    i = 0
    for b, n in enumerate(lens):
        for at in range(old[b], n):
            page, slot = int(table[b, at // size]), at % size
            want_k[1, page, :, slot], want_v[1, page, :, slot] = kr[i], vn[i]
            i += 1
    last.last_cache_append(cache, 1, seqs, kn, vn, ws, cu_new=cu_new, **kw)
    last.last_poll(ws)
    assert _same(k, want_k) and _same(v, want_v)
    if sections is not None:
        assert _same(qo, want_q)


def test_append_of_unaligned_heads():
    """Heads at odd element offsets: the copies go element by element."""
    import torch
    import cache_util as cu
    k, v = cu.pages(1, 4, 2, 16, 64, "bfloat16", "head", 1)
    cache, seqs = last.Cache(k, v), last.Sequences(cu.ints([[2, 0], [3, 1]]), cu.ints([17, 5]))
    x = cu.randn((2, 300), "bfloat16", 2)
    kn, vn = x[:, 1:129].unflatten(1, (2, 64)), x[:, 131:259].unflatten(1, (2, 64))
    ws = cu.workspace(cache, 2, 2)
    last.last_cache_append(cache, 0, seqs, kn, vn, ws)
    last.last_poll(ws)
    assert _same(k[0, 0, :, 0], kn[0]) and _same(v[0, 0, :, 0], vn[0])
    assert _same(k[0, 3, :, 4], kn[1]) and _same(v[0, 3, :, 4], vn[1])


def test_append_of_many_tokens():
    """More token groups than the kernel has CTAs."""
    import torch
    import cache_util as cu
    n, size = 70000, 64
    k, v = cu.pages(1, -(-n // size), 1, size, 16, "bfloat16", "head", 1)
    cache = last.Cache(k, v)
    table, _ = cu.table([n], size, k.shape[1], 2, extra=0)
    kn, vn = cu.randn((n, 1, 16), "bfloat16", 3), cu.randn((n, 1, 16), "bfloat16", 4)
    q = cu.randn((n, 16, 16), "bfloat16", 5)
    rope, pos = last.Rope.sections([8]), torch.arange(n, dtype=torch.int32, device="cuda")
    qo, want_q, want_k = torch.empty_like(q), torch.empty_like(q), torch.empty_like(kn)
    ws = cu.workspace(cache, 1, 16)
    last.last_cache_append(cache, 0, last.Sequences(table, cu.ints([n])), kn, vn, ws, cu_new=cu.ints([0, n]), rope=rope,
                           positions=pos, q=q, q_out=qo)
    last.last_poll(ws)
    last.last_rope(rope, pos, q, want_q, k=kn, k_out=want_k)
    assert _same(qo, want_q)
    assert _same(cu.rows(k, table[0], n, size)[0, 0], want_k[:, 0]) and _same(cu.rows(v, table[0], n, size)[0, 0], vn[:, 0])


def test_append_reports_what_has_no_slot():
    import torch
    import cache_util as cu
    for table, lens, cu_new in (([[9, 9]], [3], [0, 3]), ([[-1, 0]], [2], [0, 3]), ([[0, 1]], [40], [0, 3]),
                                ([[0, 1]], [2], [0, 3]), ([[0, 1]], [3], [0, 2])):
        k, v = cu.pages(1, 3, 1, 16, 64, "float32", "head", 1)
        k0 = k.clone()
        cache, seqs = last.Cache(k, v), last.Sequences(cu.ints(table), cu.ints(lens))
        x = cu.randn((3, 1, 64), "float32", 2)
        ws = cu.workspace(cache, 1, 1)
        last.last_cache_append(cache, 0, seqs, x, x, ws, cu_new=cu.ints(cu_new))
        with pytest.raises(last.LastError) as e:
            last.last_poll(ws)
        assert e.value.status == last.LAST_ERR_DEVICE_INDEX
        assert _same(k[0, 2], k0[0, 2])
        last.last_cache_append(cache, 0, last.Sequences(cu.ints([[0, 1]]), cu.ints([3])), x, x, ws, cu_new=cu.ints([0, 3]))
        last.last_poll(ws)
        assert _same(k[0, 0, 0, :3], x[:, 0])


def test_append_refuses_tensors():
    import torch
    import cache_util as cu
    k, v = cu.pages(1, 3, 2, 16, 64, "bfloat16", "head", 1)
    cache, seqs = last.Cache(k, v), last.Sequences(cu.ints([[0], [1]]), cu.ints([1, 1]))
    x, ws = cu.randn((2, 2, 64), "bfloat16", 2), cu.workspace(cache, 2, 2)
    rope, pos = last.Rope.sections([32]), cu.ints([0, 0])
    for args, kw in (((x, x[:1], ws), {}), ((x.float(), x, ws), {}), ((x[..., :32], x, ws), {}),
                     ((x, x, ws), dict(q=x, rope=rope, positions=pos)), ((x, x, ws), dict(rope=rope)),
                     ((x, x, ws), dict(cu_new=cu.ints([0, 2])))):
        with pytest.raises(ValueError):
            last.last_cache_append(cache, 0, seqs, *args, **kw)
    with pytest.raises(last.LastError):
        last.last_cache_append(cache, 0, seqs, x[:1], x[:1], ws)       # one token, two sequences
    last.last_cache_append(cache, 0, seqs, x[:0], x[:0], ws, cu_new=cu.ints([0, 0, 0]))
    last.last_poll(ws)


# ---- compaction ----

def _compact(layers, lens, begin, span, kept, hkv, d, size, dtype, order, seed=0, whole=False):
    import torch
    import cache_util as cu
    rng = np.random.default_rng(seed)
    idx = [np.sort(rng.choice(int(s), int(k), replace=False)) for s, k in zip(span, kept)]
    short = [n - s + k for n, s, k in zip(lens, span, kept)]
    pool = sum(-(-n // size) for n in lens) + sum(-(-n // size) for n in short) + 2
    k, v = cu.pages(layers, pool, hkv, size, d, dtype, order, seed + 1)
    table, rest = cu.table(lens, size, pool, seed)
    dst = np.full((len(lens), max(-(-n // size) for n in short) + 2), -1)
    at = 0
    for b, n in enumerate(short):
        m = -(-n // size)
        dst[b, :m] = rest[at:at + m]
        at += m
    cache, seqs, dst = last.Cache(k, v), last.Sequences(table, cu.ints(lens)), cu.ints(dst)
    k0, v0 = k.clone(), v.clone()
    out, ws = cu.ints([-5] * len(lens)), cu.workspace(cache, len(lens), hkv)
    kw = {} if whole else dict(span_begin=cu.ints(begin), span_len=cu.ints(span))
    flat = cu.ints(np.concatenate(idx)) if idx else cu.ints([])
    last.last_cache_compact(cache, seqs, dst, cu.ints(np.concatenate([[0], np.cumsum(kept)])), flat, out, ws, **kw)
    last.last_poll(ws)
    assert out.tolist() == short
    touched = torch.zeros(pool, size, dtype=torch.bool, device="cuda")
    for b, n in enumerate(lens):
        keep = np.concatenate([np.arange(begin[b]), begin[b] + idx[b], np.arange(begin[b] + span[b], n)]).astype(int)
        for new, old in ((k, k0), (v, v0)):
            assert _same(cu.rows(new, dst[b], len(keep), size), cu.rows(old, table[b], n, size)[:, :, keep])
        i = torch.arange(len(keep), device="cuda")
        touched[dst[b].long()[i // size], i % size] = True
    for new, old in ((k, k0), (v, v0)):      # and nothing else is written
        assert _same(new.transpose(2, 3)[:, ~touched], old.transpose(2, 3)[:, ~touched])


@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("layers,hkv,d,size", [(1, 1, 64, 16), (3, 2, 128, 16), (2, 5, 80, 24), (1, 4, 8, 8), (2, 2, 256, 64)])
def test_compaction(layers, hkv, d, size, dtype, order):
    lens = [100, 1, 0, 64, 333, 90, 17]
    begin = [5, 0, 0, 0, 16, 90, 3]
    span = [80, 1, 0, 64, 300, 0, 14]
    kept = [11, 1, 0, 0, 300, 0, 13]
    _compact(layers, lens, begin, span, kept, hkv, d, size, dtype, order)


def test_compaction_of_whole_sequences_and_long_ones():
    _compact(1, [50, 200], [0, 0], [50, 200], [7, 199], 2, 64, 16, "bfloat16", "head", whole=True)
    _compact(2, [9000, 3, 20000], [700, 1, 0], [8000, 2, 20000], [1000, 1, 19999], 2, 64, 16, "float32", "token", seed=5)
    _compact(1, [40] * 600, [3] * 600, [30] * 600, [4] * 600, 1, 64, 8, "bfloat16", "head", seed=6)


def test_compaction_keeps_shared_leading_pages():
    """A page in both tables whose tokens keep their slots is left alone, wherever the span begins."""
    import torch
    import cache_util as cu
    k, v = cu.pages(2, 12, 2, 16, 64, "bfloat16", "head", 1)
    table = cu.ints([[4, 9, 1, 7, 3]])
    dst = cu.ints([[4, 9, 2, 0]])            # the first 32 tokens stay where they are
    cache, seqs = last.Cache(k, v), last.Sequences(table, cu.ints([75]))
    k0, out, ws = k.clone(), cu.ints([0]), cu.workspace(cache, 1, 2)
    idx = [0, 2, 5, 20]
    last.last_cache_compact(cache, seqs, dst, cu.ints([0, 4]), cu.ints(idx), out, ws, span_begin=cu.ints([32]),
                            span_len=cu.ints([30]))
    last.last_poll(ws)
    keep = [*range(32), *[32 + i for i in idx], *range(62, 75)]
    assert out.tolist() == [len(keep)]
    assert _same(cu.rows(k, dst[0], len(keep), 16), cu.rows(k0, table[0], 75, 16)[:, :, keep])
    assert _same(k[:, [4, 9]], k0[:, [4, 9]])


def test_compaction_reports_and_skips():
    import torch
    import cache_util as cu
    ok = dict(lens=[40, 40], begin=[4, 4], span=[30, 30], cu_keep=[0, 2, 4], idx=[1, 7, 0, 29], table=None, dst=None)
    for bad, kept_idx in ((dict(lens=[40, -1]), 0), (dict(lens=[40, 1000]), 0), (dict(begin=[4, 12]), 0), (dict(begin=[4, -1]), 0),
                          (dict(span=[30, 41]), 0), (dict(span=[30, -2]), 0), (dict(cu_keep=[0, 2, 5]), 0),
                          (dict(cu_keep=[0, 2, 1]), 0), (dict(idx=[1, 7, 0, 30]), 1), (dict(idx=[1, 7, -1, 29]), 1),
                          (dict(table=(1, 0, 99)), 1), (dict(dst=(1, 0, -4)), 1)):
        a = {**ok, **bad}
        k, v = cu.pages(1, 12, 1, 16, 64, "float32", "head", 1)
        table, dst = cu.ints([[0, 1, 2], [3, 4, 5]]), cu.ints([[6, 7], [8, 9]])
        if a["table"]:
            table[a["table"][0], a["table"][1]] = a["table"][2]
        if a["dst"]:
            dst[a["dst"][0], a["dst"][1]] = a["dst"][2]
        cache, seqs = last.Cache(k, v), last.Sequences(table, cu.ints(a["lens"]))
        k0, out, ws = k.clone(), cu.ints([-5, -5]), cu.workspace(cache, 2, 1)
        last.last_cache_compact(cache, seqs, dst, cu.ints(a["cu_keep"]), cu.ints(a["idx"]), out, ws,
                                span_begin=cu.ints(a["begin"]), span_len=cu.ints(a["span"]))
        with pytest.raises(last.LastError) as e:
            last.last_poll(ws)
        assert e.value.status == last.LAST_ERR_DEVICE_INDEX, bad
        assert out.tolist() == [12, 12 if kept_idx else -5], bad
        keep = [0, 1, 2, 3, 5, 11, *range(34, 40)]
        assert _same(cu.rows(k, dst[0], 12, 16), cu.rows(k0, table[0], 40, 16)[:, :, keep])
        assert _same(k[:, 10:], k0[:, 10:]) and _same(k[:, :6], k0[:, :6])


def test_compaction_refuses_tensors():
    import cache_util as cu
    k, v = cu.pages(1, 6, 1, 16, 64, "float32", "head", 1)
    cache, seqs, ws = last.Cache(k, v), last.Sequences(cu.ints([[0, 1]]), cu.ints([20])), None
    ws = cu.workspace(cache, 1, 1)
    dst, keep, idx, out = cu.ints([[2, 3]]), cu.ints([0, 1]), cu.ints([0]), cu.ints([0])
    for args in ((dst[0], keep, idx, out), (dst, keep[:1], idx, out), (dst, keep, idx.long(), out), (dst, keep, idx, out[:0])):
        with pytest.raises(ValueError):
            last.last_cache_compact(cache, seqs, *args, ws)
    with pytest.raises(last.LastError):
        last.last_cache_compact(cache, seqs, dst, keep, idx, seqs.lens, ws)
    with pytest.raises(last.LastError):
        last.last_cache_compact(cache, seqs, dst, keep, idx, out, ws, span_begin=cu.ints([0]))


# ---- page copies ----

@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("layers,hkv,d,size,n", [(1, 1, 8, 8, 1), (4, 4, 128, 16, 9), (2, 3, 80, 24, 30), (1, 2, 256, 128, 5), (3, 2, 64, 16, 2000)])
def test_copies(layers, hkv, d, size, n, dtype, order):
    import torch
    import cache_util as cu
    pool = 2 * n + 3
    k, v = cu.pages(layers, pool, hkv, size, d, dtype, order, 1)
    cache, ws = last.Cache(k, v), None
    ws = cu.workspace(cache, 1, hkv)
    perm = torch.as_tensor(np.random.default_rng(2).permutation(pool)).cuda()
    src, dst = perm[:n].int(), perm[n:2 * n].int()
    dst[n // 2] = src[n // 2]                      # onto itself: nothing
    want = [t.clone() for t in (k, v)]
    for t in want:
        t[:, dst.long()] = t[:, src.long()]
    last.last_cache_copy(cache, src, dst, ws)
    last.last_poll(ws)
    assert _same(k, want[0]) and _same(v, want[1])


def test_copies_of_part_of_a_cache():
    """A cache whose pages, heads and tokens lie apart: what is between them is not touched."""
    import torch
    import cache_util as cu
    base = [cu.randn((2, 7, 3, 24, 96), "bfloat16", i) for i in range(2)]
    k, v = (t[:, :, :2, :16, 16:80] for t in base)
    want = [t.clone() for t in base]
    for t in want:
        t[:, 5, :2, :16, 16:80] = t[:, 1, :2, :16, 16:80]
    cache = last.Cache(k, v)
    ws = cu.workspace(cache, 1, 2)
    last.last_cache_copy(cache, cu.ints([1]), cu.ints([5]), ws)
    last.last_poll(ws)
    assert _same(base[0], want[0]) and _same(base[1], want[1])


def test_copies_report_bad_pages():
    import cache_util as cu
    k, v = cu.pages(1, 6, 1, 16, 64, "float32", "head", 1)
    cache = last.Cache(k, v)
    ws = cu.workspace(cache, 1, 1)
    for src, dst in (([0, 6], [3, 4]), ([0, -1], [3, 4]), ([0, 1], [3, 6]), ([0, 1], [3, -2])):
        k0 = k.clone()
        last.last_cache_copy(cache, cu.ints(src), cu.ints(dst), ws)
        with pytest.raises(last.LastError) as e:
            last.last_poll(ws)
        assert e.value.status == last.LAST_ERR_DEVICE_INDEX
        assert _same(k[0, 3], k0[0, 0]) and _same(k[0, 4:], k0[0, 4:])
        last.last_cache_copy(cache, cu.ints([0]), cu.ints([3]), ws)
        last.last_poll(ws)
    last.last_cache_copy(cache, cu.ints([]), cu.ints([]), ws)
    last.last_poll(ws)
    with pytest.raises(ValueError):
        last.last_cache_copy(cache, cu.ints([0]), cu.ints([1, 2]), ws)


# ---- together ----

def test_decode_loop_in_a_graph():
    """Append and attention captured once and replayed while lengths and positions grow in place give what
    the calls give one by one."""
    import torch
    import cache_util as cu
    hq, hkv, d, size, old, steps = 8, 2, 128, 16, [30, 0, 95], 40
    rope = last.Rope.sections([16, 24, 24])
    k, v = cu.pages(1, 40, hkv, size, d, "bfloat16", "head", 1)
    table, _ = cu.table([n + steps for n in old], size, 40, 2)
    x = cu.randn((steps, 3, hq + 2 * hkv, d), "bfloat16", 3)

    def program(kk, vv):
        cache, lens = last.Cache(kk, vv), cu.ints(old)
        seqs, ws = last.Sequences(table, lens), cu.workspace(last.Cache(kk, vv), 3, hq)
        inp, pos = x[0].clone(), cu.ints([old] * 3)
        q = torch.empty((3, hq, d), dtype=x.dtype, device="cuda")
        out = torch.empty_like(q)

        def step():
            lens.add_(1)
            last.last_cache_append(cache, 0, seqs, inp[:, hq:hq + hkv], inp[:, hq + hkv:], ws, rope=rope, positions=pos,
                                   q=inp[:, :hq], q_out=q)
            last.last_cache_attention(cache, 0, seqs, q, out, ws)
            pos.add_(1)
        return inp, out, step, ws, lens, pos, seqs, cache, q

    plain = program(k.clone(), v.clone())
    want = []
    for i in range(steps):
        plain[0].copy_(x[i])
        plain[2]()
        last.last_poll(plain[3])
        want.append(plain[1].clone())
    g = program(k.clone(), v.clone())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):      # a first step outside the graph, then undone
        g[0].copy_(x[0])
        g[2]()
    torch.cuda.synchronize()
    g[4].sub_(1)
    g[5].sub_(1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g[2]()
    for i in range(steps):
        g[0].copy_(x[i])
        graph.replay()
        assert _same(g[1], want[i]), i
    last.last_poll(g[3])


@pytest.mark.parametrize("dtype,d,rot", [("bfloat16", 8, 0), ("bfloat16", 8, 2), ("bfloat16", 24, 0), ("float32", 4, 0), ("float32", 12, 4),
                                         ("bfloat16", 128, 40), ("float32", 128, 40), ("bfloat16", 80, 64), ("float32", 256, 250)])
@pytest.mark.parametrize("pairs", ["half", "adjacent"])
def test_append_of_narrow_and_partly_rotated_rows(dtype, d, rot, pairs):
    """Rows of one or three pieces, and rows of which a part is copied."""
    import torch
    import cache_util as cu
    k, v = cu.pages(1, 5, 3, 8, d, dtype, "token", 1)
    cache, seqs = last.Cache(k, v), last.Sequences(cu.ints([[4, 2], [1, 0]]), cu.ints([11, 6]))
    q, kn, vn = cu.randn((5, 6, d), dtype, 2), cu.randn((5, 3, d), dtype, 3), cu.randn((5, 3, d), dtype, 4)
    kn[..., rot:] = float("inf")                    # what is copied is only copied
    kr, qo, want_q, kw = kn.clone(), torch.zeros_like(q), torch.zeros_like(q), {}
    if rot:
        rope, pos = last.Rope.sections([rot // 2], pairs=pairs), torch.arange(5, dtype=torch.int32, device="cuda")
        last.last_rope(rope, pos, q, want_q, k=kn, k_out=kr)
        kw = dict(rope=rope, positions=pos, q=q, q_out=qo)
    assert _same(kr[..., rot:], kn[..., rot:])
    k0, v0, ws = k.clone(), v.clone(), cu.workspace(cache, 2, 6)
    last.last_cache_append(cache, 0, seqs, kn, vn, ws, cu_new=cu.ints([0, 3, 5]), **kw)
    last.last_poll(ws)
    for i, (page, slot) in enumerate([(2, 0), (2, 1), (2, 2), (1, 4), (1, 5)]):
        k0[0, page, :, slot], v0[0, page, :, slot] = kr[i], vn[i]
    assert _same(k, k0) and _same(v, v0) and _same(qo, want_q)


def test_compaction_of_many_layers():
    """More rows a token than a CTA keeps addresses of."""
    _compact(24, [40, 9], [3, 0], [30, 9], [7, 2], 88, 8, 8, "bfloat16", "head", seed=7)


def test_calls_behind_copies_and_joined_streams():
    """The calls behind memory copies, memory sets and another stream's work, at once and in a graph."""
    import torch
    import cache_util as cu
    hq, hkv, d, n = 8, 2, 128, 700
    k, v = cu.pages(2, 120, hkv, 16, d, "bfloat16", "head", 1)
    table, rest = cu.table([n], 16, 60, 2)
    cache, lens = last.Cache(k, v), cu.ints([n])
    seqs, ws, ws2 = last.Sequences(table, lens), cu.workspace(cache, 1, hq), cu.workspace(cache, 1, hq)
    src_q, src_kv = cu.randn((40, hq, d), "bfloat16", 3), cu.randn((40, 2, hkv, d), "bfloat16", 4)
    q, kv, out, out2 = torch.zeros_like(src_q[:1]), torch.zeros_like(src_kv[:1]), torch.zeros_like(src_q[:1]), torch.zeros_like(src_q[:1])
    big, other = torch.empty(1 << 24, device="cuda"), torch.empty(1 << 24, device="cuda")
    copied = cu.ints([100])
    one = table[0, 43:44].clone()           # the last, partly filled page
    side = torch.cuda.Stream()

    def program():
        main = torch.cuda.current_stream()
        q.copy_(src_q[7:8])
        kv.copy_(src_kv[7:8])               # memory copies
        last.last_cache_append(cache, 0, seqs, kv[:, 0], kv[:, 1], ws)
        big.zero_()                         # a memory set, or a kernel of torch
        last.last_cache_attention(cache, 0, seqs, q, out, ws)
        side.wait_stream(main)
        with torch.cuda.stream(side):
            other.copy_(big)
            last.last_cache_copy(cache, one, copied, ws2)
        main.wait_stream(side)
        last.last_cache_attention(cache, 1, seqs, q, out2, ws)

    torch.cuda.synchronize()
    program()
    torch.cuda.synchronize()
    last.last_poll(ws)
    last.last_poll(ws2)
    want, want2, want_k = out.clone(), out2.clone(), k.clone()
    assert _same(k[:, 100], k[:, int(one)]) and want.abs().sum() > 0
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        program()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        program()
    for t in (q, kv, out, out2):
        t.zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    last.last_poll(ws)
    assert _same(out, want) and _same(out2, want2) and _same(k, want_k)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_offsets_past_32_bits(dtype):
    """Appending, cutting and copying in pages 5 GB apart (most of the storage is never touched)."""
    import torch
    import cache_util as cu
    e = 4 if dtype == "float32" else 2
    far = 5 * 2**30 // e
    base = [torch.empty(3 * far + 8192, dtype=getattr(torch, dtype), device="cuda") for _ in range(2)]
    k, v = (b.as_strided((1, 4, 2, 16, 64), (0, far, 1024, 64, 1)) for b in base)
    for i, t in enumerate((k, v)):
        t.copy_(cu.randn((1, 4, 2, 16, 64), dtype, i))
    cache = last.Cache(k, v)
    ws = cu.workspace(cache, 1, 2)
    seqs = last.Sequences(cu.ints([[2, 0]]), cu.ints([20]))
    x = cu.randn((6, 2, 64), dtype, 5)
    last.last_cache_append(cache, 0, seqs, x, -x, ws, cu_new=cu.ints([0, 6]))
    last.last_poll(ws)
    assert _same(k[0, 2, :, 14:].transpose(0, 1), x[:2]) and _same(v[0, 0, :, :4].transpose(0, 1), -x[2:])
    k0, v0, out = k.clone(), v.clone(), cu.ints([0])
    idx = [0, 3, 15, 19]
    last.last_cache_compact(cache, seqs, cu.ints([[3]]), cu.ints([0, 4]), cu.ints(idx), out, ws)
    last.last_poll(ws)
    for t, t0 in ((k, k0), (v, v0)):
        assert _same(cu.rows(t, cu.ints([3]), 4, 16), cu.rows(t0, seqs.page_table[0], 20, 16)[:, :, idx])
    last.last_cache_copy(cache, cu.ints([3]), cu.ints([1]), ws)
    last.last_poll(ws)
    assert _same(k[:, 1], k[:, 3]) and _same(v[:, 1], v[:, 3]) and _same(k[:, 0], k0[:, 0])


def test_calls_allocate_nothing():
    import torch
    import cache_util as cu
    k, v = cu.pages(2, 300, 2, 16, 128, "bfloat16", "head", 1)
    table, rest = cu.table([900, 70], 16, 300, 2)
    cache, seqs = last.Cache(k, v), last.Sequences(table, cu.ints([900, 70]))
    ws = cu.workspace(cache, 2, 8)
    q, x = cu.randn((2, 8, 128), "bfloat16", 3), cu.randn((2, 2, 128), "bfloat16", 4)
    qo, out, rope, pos = torch.empty_like(q), torch.empty_like(q), last.Rope.sections([64]), cu.ints([5, 6])
    dst, lens_out = cu.ints([rest[:60], rest[60:120]]), cu.ints([0, 0])
    keep, idx, a, b = cu.ints([0, 10, 20]), cu.ints([*range(10)] * 2), cu.ints(rest[:3]), cu.ints(rest[120:123])

    def calls():
        last.last_rope(rope, pos, q, qo)
        last.last_cache_append(cache, 0, seqs, x, x, ws, rope=rope, positions=pos, q=q, q_out=qo)
        last.last_cache_attention(cache, 0, seqs, q, out, ws)
        last.last_cache_compact(cache, seqs, dst, keep, idx, lens_out, ws)
        last.last_cache_copy(cache, a, b, ws)
        torch.cuda.synchronize()
    calls()
    free = torch.cuda.mem_get_info()[0]
    for _ in range(3):
        calls()
    assert torch.cuda.mem_get_info()[0] == free


def test_both_ways_of_the_binding(monkeypatch):
    """The marshalling module and ctypes hand the library the same arguments and refuse the same tensors."""
    import torch
    import cache_util as cu
    assert last.load_library() and last._fast is not None, "the marshalling module has not been built"

    def everything():
        k, v = cu.pages(2, 60, 2, 16, 64, "bfloat16", "token", 1)
        table, rest = cu.table([90, 33], 16, 60, 2)
        cache, seqs = last.Cache(k, v), last.Sequences(table, cu.ints([90, 33]), cu.ints([3, 0]))
        ws = cu.workspace(cache, 2, 6)
        fused = cu.randn((5, 10, 64), "bfloat16", 3)
        q, kn, vn = fused.split([6, 2, 2], dim=1)
        qo, ko, out = torch.zeros_like(q), torch.zeros_like(kn), torch.zeros((2, 6, 64), dtype=q.dtype, device="cuda")
        lse, rope, pos = torch.zeros((2, 6), device="cuda"), last.Rope.sections([8, 12, 12]), cu.ints(np.arange(15).reshape(3, 5))
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        last.last_rope(rope, pos, q, qo, k=kn, k_out=ko, stream=s)
        last.last_rope_backward(rope, pos, qo, qo, stream=s.cuda_stream)
        torch.cuda.current_stream().wait_stream(s)
        got = [qo.clone(), ko]
        last.last_cache_append(cache, 1, seqs, kn, vn, ws, cu_new=cu.ints([0, 3, 5]), rope=rope, positions=pos, q=q, q_out=qo)
        last.last_cache_append(cache, 0, seqs, kn[:2], vn[:2], ws)
        last.last_cache_attention(cache, 1, seqs, qo[[2, 4]], out, ws, lse=lse, softmax_scale=0.2)
        lens_out, dst = cu.ints([0, 0]), cu.ints(np.stack([rest[:6], rest[6:12]]))
        last.last_cache_compact(cache, seqs, dst, cu.ints([0, 2, 3]), cu.ints([0, 7, 1]), lens_out, ws, span_begin=cu.ints([4, 0]),
                                span_len=cu.ints([60, 20]))
        last.last_cache_copy(cache, dst[:, 0].contiguous(), cu.ints(rest[12:14]), ws)
        last.last_poll(ws)
        for call in (lambda: last.last_rope(rope, pos[:2], q, qo), lambda: last.last_rope(rope, pos, q, qo, k=kn),
                     lambda: last.last_cache_append(cache, 0, seqs, kn[:2], vn, ws),
                     lambda: last.last_cache_append(cache, 0, seqs, kn[:2].float(), vn[:2], ws),
                     lambda: last.last_cache_attention(cache, 0, seqs, qo[:2].cpu(), out, ws),
                     lambda: last.last_cache_attention(cache, 0, seqs, qo[:2], out, ws, lse=lse[:, :3]),
                     lambda: last.last_cache_attention(cache, 0, seqs, qo[:2], out, ws.cpu()),
                     lambda: last.last_cache_compact(cache, seqs, dst, cu.ints([0, 2]), cu.ints([0, 7, 1]), lens_out, ws),
                     lambda: last.last_cache_copy(cache, cu.ints([1]), torch.zeros(1, dtype=torch.int64, device="cuda"), ws)):
            with pytest.raises(ValueError):
                call()
        with pytest.raises(last.LastError):
            last.last_cache_attention(cache, 2, seqs, qo[:2], out, ws)
        with pytest.raises(last.LastError):
            last.last_cache_copy(cache, cu.ints([1]), cu.ints([2]), ws[:512])
        return [*got, qo, k, v, out, lse, lens_out]

    want = everything()
    monkeypatch.setattr(last, "_fast", None)
    assert all(_same(a, b) for a, b in zip(everything(), want))


def test_a_failed_launch_leaves_no_error_behind():
    """The calls' launches refused by the runtime (the stream's capture is broken): each says so once, and later
    calls of the path start clean."""
    import ctypes
    import torch
    import cache_util as cu
    rt = ctypes.CDLL("libcudart.so.13")
    rt.cudaStreamBeginCapture.argtypes = [ctypes.c_void_p, ctypes.c_int]
    rt.cudaStreamEndCapture.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
    rt.cudaStreamSynchronize.argtypes = [ctypes.c_void_p]
    k, v = cu.pages(1, 8, 2, 16, 64, "bfloat16", "head", 1)
    cache, seqs = last.Cache(k, v), last.Sequences(cu.ints([[0, 1]]), cu.ints([20]))
    ws, ints, out = cu.workspace(cache, 1, 2), cu.ints([2]), cu.ints([0])
    x, rope, pos, y = cu.randn((1, 2, 64), "bfloat16", 2), last.Rope.sections([32]), cu.ints([3]), cu.randn((1, 2, 64), "bfloat16", 3)
    keep, idx, dst = cu.ints([0, 1]), cu.ints([0]), cu.ints([[4]])
    calls = (lambda s: last.last_cache_copy(cache, ints, ints, ws, stream=s), lambda s: last.last_rope(rope, pos, x, y, stream=s),
             lambda s: last.last_cache_append(cache, 0, seqs, x, x, ws, stream=s),
             lambda s: last.last_cache_attention(cache, 0, seqs, x, y, ws, stream=s),
             lambda s: last.last_cache_compact(cache, seqs, dst, keep, idx, out, ws, stream=s))
    for call in calls:
        call(None)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for call in calls:
        assert rt.cudaStreamBeginCapture(s.cuda_stream, 2) == 0
        graph = ctypes.c_void_p()
        try:
            assert rt.cudaStreamSynchronize(s.cuda_stream) != 0      # not allowed: breaks the capture
            rt.cudaGetLastError()
            with pytest.raises(last.LastError) as e:
                call(s)
            left = rt.cudaGetLastError()
        finally:
            rt.cudaStreamEndCapture(s.cuda_stream, ctypes.byref(graph))
            rt.cudaGetLastError()
        assert e.value.status == last.LAST_ERR_CUDA and left == 0
    for call in calls:
        call(s)
    s.synchronize()
    last.last_poll(ws, s)

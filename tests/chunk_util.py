"""Chunk and differential attention in 64 bits, with bounds of what the kernels may differ by."""
import math

import numpy as np
import torch

import cache_util as cu
import paper_2607_27952_gb300 as last

# One rounding to the type, relative.
UNIT = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8}


def setup(new, old, hq, hkv, d, dtype, size, order="head", seed=0, begin=None, stale=None, qscale=1.0, extra=0):
    """Sequences with new[b] new tokens behind old[b] cached ones.  stale: what slots of no sequence's visible keys hold;
    extra: rows of q that belong to no sequence."""
    new, old = np.asarray(new, int), np.asarray(old, int)
    lens = new + old
    pool = int(sum(-(-int(n) // size) for n in lens)) + 2
    k, v = cu.pages(1, pool, hkv, size, d, dtype, order, seed + 1)
    table, _ = cu.table(lens, size, pool, seed)
    if stale is not None:
        used = torch.zeros((pool, size), dtype=torch.bool, device="cuda")
        for b, n in enumerate(lens):
            i = torch.arange(0 if begin is None else min(int(begin[b]), int(n)), int(n), device="cuda")
            used[table[b].long()[i // size], i % size] = True
        for t in (k, v):
            t[0].transpose(1, 2)[~used] = stale
    q = cu.randn((int(new.sum()) + extra, hq, d), dtype, seed + 3, qscale)
    cu_new = cu.ints(np.concatenate([[0], np.cumsum(new)]))
    seqs = last.Sequences(table, cu.ints(lens), None if begin is None else cu.ints(begin))
    return last.Cache(k, v), seqs, q, cu_new


def workspace(cache, heads):
    return last.chunk_workspace(cache, heads).fill_(0xA5)   # its contents may be anything


def seen(n, lens, begin, causal, window):
    """[n][lens]: keys that new tokens see."""
    p = torch.arange(lens - n, lens, device="cuda")[:, None]
    j = torch.arange(lens, device="cuda")
    s = (j >= begin).expand(n, lens)
    if causal:
        s = s & (j <= p)
    if window:
        s = s & (j > p - window)
    return s


def one_map(q, k, v, see, scale):
    """q [n][d] over k [keys][d], v [keys][w]: outputs, log of the denominator, sum p |v|, and the error of a logit."""
    q, k, v = q.double(), k.double(), v.double()
    v = torch.where(see.any(0)[:, None], v, 0.0)
    z = torch.where(see, (q @ k.T) * scale, -math.inf)
    lse = torch.logsumexp(z, 1)
    p = torch.where(see & (z > -math.inf), torch.exp(z - lse[:, None]), 0.0)
    size = torch.where(see, (q.abs() @ k.abs().T) * scale, 0.0)
    # a logit: a sum of d products in fp32, each term within (d + 8) 2^-24 of sum |q k|
    ez = float(size.max()) * (q.shape[1] + 8) * 2.0 ** -24 if see.any() else 0.0
    return p @ v, lse, p @ v.abs(), ez


def relative(ez, n, dtype, parts=1):
    """Of the weighted sums, times sum p |v|: the exponentials' and the sums' errors as for single tokens, and for bf16 a
    weight rounded once (2^-8), or held in two parts (2^-16)."""
    return 4 * ez + 2.0 ** -20 + (n / 8 + 64) * 2.0 ** -24 + (2.0 ** (-8 * parts) if dtype == "bfloat16" else 0.0)


def keys_of(cache, table_row, lens, head, live=None):
    k, v = (cu.rows(t, table_row, lens, cache.page_size)[0] for t in (cache.k, cache.v))
    return k[head], v[head]


def check_chunk(cache, seqs, q, cu_new, out, lse, new, lens, begin=None, causal=True, window=0, scale=None, bad=None, only=None):
    """bad: {sequence: table indices that are out of range}."""
    hq, d = q.shape[1:]
    g = hq // cache.kv_heads
    dtype, scale = str(q.dtype).rpartition(".")[2], scale or 1 / math.sqrt(d)
    for b, (n, total) in enumerate(zip(new, lens)):
        if n == 0 or (only is not None and b not in only):
            continue
        t0 = int(cu_new[b])
        see = seen(int(n), int(total), 0 if begin is None else int(begin[b]), causal, window)
        if bad and b in bad:
            gone = torch.isin(torch.arange(int(total), device="cuda") // cache.page_size, torch.as_tensor(bad[b], device="cuda"))
            see = see & ~gone
        for h in range(hq):
            k, v = keys_of(cache, seqs.page_table[b].clamp(0, cache.k.shape[1] - 1), int(total), h // g)
            k = torch.where(see.any(0)[:, None], k, 0)
            want, want_lse, size, ez = one_map(q[t0:t0 + n, h], k, v, see, scale)
            err = (out[t0:t0 + n, h].double() - want).abs()
            tol = relative(ez, total, dtype) * size + UNIT[dtype] * want.abs()
            assert (err <= tol).all(), f"sequence {b} ({n} of {total}), head {h}: {(err - tol).max():.3e} past the bound"
            if lse is None:
                continue
            got, none = lse[t0:t0 + n, h].double(), ~see.any(1)
            assert (got[none] == -math.inf).all() and (out[t0:t0 + n, h][none] == 0).all()
            tol = 2 * ez + 2.0 ** -20 * (1 + want_lse.abs()) + (total / 8 + 64) * 2.0 ** -24
            assert ((got - want_lse).abs() <= tol)[~none].all(), f"sequence {b}, head {h}: lse"


def check_diff(cache, seqs, q, cu_new, out, lam, new, lens, begin=None, causal=True, window=0, scale=None, weight=None, eps=1e-5,
               out_scale=1.0, bad=None, only=None):
    hq, d = q.shape[1:]
    g = hq // cache.kv_heads
    dtype, scale = str(q.dtype).rpartition(".")[2], scale or 1 / math.sqrt(d)
    for b, (n, total) in enumerate(zip(new, lens)):
        if n == 0 or (only is not None and b not in only):
            continue
        t0 = int(cu_new[b])
        see = seen(int(n), int(total), 0 if begin is None else int(begin[b]), causal, window)
        if bad and b in bad:
            gone = torch.isin(torch.arange(int(total), device="cuda") // cache.page_size, torch.as_tensor(bad[b], device="cuda"))
            see = see & ~gone
        row = seqs.page_table[b].clamp(0, cache.k.shape[1] - 1)
        for j in range(hq // 2):
            u = j // g
            v = torch.cat([keys_of(cache, row, int(total), 2 * u + e)[1] for e in range(2)], 1)
            x = e = 0.0
            for m in range(2):
                k = torch.where(see.any(0)[:, None], keys_of(cache, row, int(total), 2 * u + m)[0], 0)
                o, _, size, ez = one_map(q[t0:t0 + n, 2 * j + m], k, v, see, scale)
                f = 1.0 if m == 0 else -float(lam[j])
                x = x + f * o
                e = e + abs(f) * relative(ez, total, dtype, 2) * size
            e = e + 2.0 ** -22 * x.abs()
            if weight is None:
                want, tol = x * out_scale, e * abs(out_scale)
            else:
                # r = sqrt(mean x^2 + eps) moves by no more than the root mean square of e
                r, w = torch.sqrt(x.square().mean(1, keepdim=True) + eps), weight.double() * out_scale
                moved = e.square().mean(1, keepdim=True).sqrt()
                want = torch.where(r > 0, x / r, 0.0) * w
                low = r - moved
                tol = torch.where(low > 0, (e / low + x.abs() * moved / (r * low)), math.inf) * w.abs()
                tol = torch.where(r > 0, tol, 0.0)
            err = (out[t0:t0 + n, j].double() - want).abs()
            tol = tol + (UNIT[dtype] + 2.0 ** -20) * want.abs()
            assert (err <= tol).all(), f"sequence {b} ({n} of {total}), pair {j}: {(err - tol).max():.3e} past the bound"
            none = ~see.any(1)
            assert (out[t0:t0 + n, j][none] == 0).all()

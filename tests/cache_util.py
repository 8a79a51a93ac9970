"""Paged caches for the tests: random pages in either order, shuffled tables, and plain definitions in 64 bits."""
import numpy as np
import torch

import paper_2607_27952_gb300 as last


def randn(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(getattr(torch, dtype))


def ints(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()


def pages(layers, n, heads, size, dim, dtype, order, seed, fill=None):
    """K, V [layers][n][heads][size][dim]; order "token": heads inside tokens, as a transposed view."""
    shape = (layers, n, heads, size, dim) if order == "head" else (layers, n, size, heads, dim)
    kv = [randn(shape, dtype, seed + i) for i in range(2)]
    if fill is not None:
        for t in kv:
            t.fill_(fill)
    return [t if order == "head" else t.transpose(2, 3) for t in kv]


def table(lens, size, pool, seed, extra=1, unused=-1):
    """Shuffled pages for sequences of these lengths: the table, `unused` past their last pages."""
    order = np.random.default_rng(seed).permutation(pool)
    need = [-(-int(n) // size) for n in lens]
    t = np.full((len(lens), max(need + [0]) + extra), unused, np.int64)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = order[at:at + n]
        at += n
    assert at <= pool
    return ints(t), order[at:]


def rows(x, row, n, size):
    """[layers][heads][n][dim] of the first n tokens of one table row."""
    i = torch.arange(n, device=x.device)
    return x[:, row.long()[i // size], :, i % size].permute(1, 2, 0, 3)


def attention(q, k, v, scale):
    """q [heads][d], k, v [kv_heads][n][d] -> out, lse, and per element sum p |v| (64 bits)."""
    q, k, v = q.double(), k.double(), v.double()
    g = q.shape[0] // k.shape[0]
    k, v = k.repeat_interleave(g, 0), v.repeat_interleave(g, 0)
    if k.shape[1] == 0:
        z = torch.zeros_like(q)
        return z, torch.full((q.shape[0],), -np.inf, dtype=torch.float64, device=q.device), z
    z = torch.einsum("hd,hnd->hn", q, k) * scale
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None]).nan_to_num(0.0)
    return torch.einsum("hn,hnd->hd", p, v), lse, torch.einsum("hn,hnd->hd", p, v.abs())


def attention_bounds(q, k, scale, n, dtype):
    """Relative error of the probabilities (times sum p |v|) and of one rounding of the result.
    A logit is a sum of d products, each term's error at most (d + 4) 2^-24 of sum |q k|, and its exponential two
    more units of |z|; the sums over n keys add at most (n / 8 + 64) 2^-24 in any grouping used, and bf16 weights
    split in two leave 2^-16."""
    g = q.shape[0] // k.shape[0]
    size = torch.einsum("hd,hnd->hn", q.double().abs(), k.double().repeat_interleave(g, 0).abs()) * scale
    ez = float(size.max()) * (q.shape[1] + 8) * 2.0 ** -24 if n else 0.0
    rel = 4 * ez + 2.0 ** -20 + (n / 8 + 64) * 2.0 ** -24 + (2.0 ** -16 if dtype == "bfloat16" else 0.0)
    return ez, rel, {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8}[dtype]


def workspace(cache, batch, heads):
    return last.cache_workspace(cache, batch, heads).fill_(0xA5)   # its contents may be anything

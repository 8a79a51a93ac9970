"""Attention of chunks of new tokens over the paged key-value cache, as measurable cases.

  chunk     softmax attention of several new tokens per sequence over its pages
            (`last_cache_chunk_attention`), causal, full or in a window, with the log of the
            softmax's denominator: prompts, prompts behind a cached part, drafted tokens
  diff      differential attention (`last_cache_diff_attention`) of single tokens and of chunks:
            the difference of two softmax maps, weighted by a learned lambda per pair of
            heads, over values twice as wide, with the RMS norm behind it

Sizes are those of the benchmark presets (one image in fp32, a batch of 576-token images,
dynamic resolution, tiled images, video) and odd ones like the tests'.  q, K and V are N(0, 1),
so that logits are N(0, 1) and the two maps of a pair differ; lambda lies between 0.2 and 0.8.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_EPS = 1e-5                      # of the RMS norm
_MOST_FLOPS = 0.5e12             # a drawn case's, at most
_MOST_KEYS = 6 * 115536 * 4      # (token, kv-head) pairs of the largest listed cache


def _case(name, op, batch, new_lo, new_hi, old_lo, old_hi, hq, hkv, d, dtype, page, order, mask="causal",
          window=0, empty=0, norm=True):
    """new_lo..new_hi new tokens per sequence behind old_lo..old_hi cached ones; order: which of a page's
    heads and tokens is outer; window > 0: only the last so many keys; empty: so many
    sequences without a new token; norm: diff with its RMS norm."""
    c = dict(op=op, batch=batch, new_lo=new_lo, new_hi=new_hi, old_lo=old_lo, old_hi=old_hi, hq=hq, hkv=hkv, d=d,
             dtype=dtype, page=page, order=order, mask=mask, window=window, empty=empty, norm=norm)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a short question behind one image, fp32: the smallest call, latency
        _case("chunk-image-f32", "chunk", 1, 32, 32, 576, 576, 16, 16, 64, "f32", 16, "head"),
        # five drafted tokens per sequence verified over 576-token images
        _case("chunk-drafts", "chunk", 64, 5, 5, 592, 704, 16, 16, 128, "bf16", 16, "head"),
        # whole prompts of dynamic resolution: ragged, 6 query heads share a K head, token-major pages
        _case("chunk-ragged", "chunk", 24, 264, 4352, 0, 0, 12, 2, 128, "bf16", 32, "token", empty=2),
        # prefill of tiled images
        _case("chunk-tiles", "chunk", 16, 2944, 2944, 0, 0, 16, 4, 128, "bf16", 16, "head"),
        # the next question in a long video session: many keys, few rows
        _case("chunk-video", "chunk", 1, 301, 301, 115235, 115235, 16, 4, 128, "bf16", 64, "head"),
        # image tokens that see each other both ways, head width 80
        _case("chunk-full", "chunk", 8, 1201, 1201, 35, 35, 16, 2, 80, "bf16", 24, "head", mask="full"),
        # a sliding window over a long prompt, in two halves
        _case("chunk-window", "chunk", 2, 8191, 8192, 8000, 8400, 14, 2, 64, "bf16", 16, "token", window=1024),
        # one decode step over 576-token images
        _case("diff-token", "diff", 64, 1, 1, 592, 704, 16, 16, 128, "bf16", 16, "head"),
        # the next token after one image, fp32, without the norm: the smallest call of its kind
        _case("diff-token-f32", "diff", 1, 1, 1, 607, 607, 16, 16, 64, "f32", 16, "head", norm=False),
        # a few long video sessions, odd lengths
        _case("diff-long", "diff", 6, 1, 1, 99998, 131072, 16, 4, 128, "bf16", 64, "head"),
        # prefill of tiled images: the largest of its kind
        _case("diff-tiles", "diff", 4, 2944, 2944, 0, 0, 16, 4, 128, "bf16", 16, "head"),
        # prompts behind a cached part, narrow heads, ragged
        _case("diff-ragged", "diff", 12, 33, 1500, 264, 704, 12, 4, 64, "bf16", 32, "token"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["chunk", "chunk", "diff"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    heads = [(16, 16), (16, 4), (12, 2), (14, 2), (16, 2), (8, 8), (12, 4)]
    hq, hkv = rng.choice(heads + [(16, 1), (6, 3)] if op == "chunk" else heads)
    d = rng.choice([64, 80, 128, 128])
    page = rng.choice([8, 16, 16, 24, 32, 64])
    order = rng.choice(["head", "token"])
    most = _MOST_FLOPS / (20 if dtype == "f32" else 1)
    kind = rng.choice(["token", "few", "prompt", "prompt", "behind"])
    if kind == "token" and op == "chunk":
        kind = "few"
    if kind in ("token", "few"):          # decode or drafts: a cache and few new tokens
        new = 1 if kind == "token" else _log_int(rng, 1, 16)
        old = _log_int(rng, 1, 131072)
        batch = _log_int(rng, 1, max(1, min(128, _MOST_KEYS // (2 * hkv * (old + new)))))
        new_lo, old_lo = max(1, new // rng.randint(1, 4)), old // rng.randint(1, 8)
    else:
        new = _log_int(rng, 17, 9000)
        old = 0 if kind == "prompt" else _log_int(rng, 1, 60000)
        per = 12 * hq * d * new * (old + new / 2)
        while per > most:
            new, old = max(1, new // 2), old // 2
            per = 12 * hq * d * new * (old + new / 2)
        batch = _log_int(rng, 1, max(1, min(32, int(most / per), _MOST_KEYS // (2 * hkv * (old + new)))))
        new_lo, old_lo = max(1, new // rng.randint(1, 8)), old // rng.randint(1, 4)
    mask, window = "causal", 0
    if rng.random() < 0.2:
        mask = "full"
    elif rng.random() < 0.25:
        window = _log_int(rng, 1, old + new)
    return _case(None, op, batch, new_lo, new, old_lo, old, hq, hkv, d, dtype, page, order, mask, window,
                 rng.randint(1, 2) if batch > 2 and rng.random() < 0.3 else 0, rng.random() < 0.8)


# ---- shapes: host arithmetic ----

def _spread(lo, hi, n, seed):
    """n sizes spread evenly over lo..hi, in a seeded order."""
    v = np.rint(np.linspace(lo, hi, n) if n > 1 else np.array([hi])).astype(np.int64)
    return v[np.random.default_rng([seed, 11]).permutation(n)]


def _lengths(case, seed):
    """New and cached tokens (the new ones among them) by sequence."""
    new = _spread(case["new_lo"], case["new_hi"], case["batch"], seed)
    old = _spread(case["old_lo"], case["old_hi"], case["batch"], seed + 1)
    if case["empty"]:
        new[np.argsort(new, kind="stable")[: case["empty"]]] = 0
    return new, new + old


def _seen(case, n, total):
    """First visible key and the one behind the last, by new token."""
    p = total - n + np.arange(n)
    hi = p + 1 if case["mask"] == "causal" else np.full(n, total)
    lo = np.maximum(0, p - case["window"] + 1) if case["window"] else np.zeros(n, dtype=np.int64)
    return lo, hi


def _elem(case):
    return 4 if case["dtype"] == "f32" else 2


def _torch_dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def work(case):
    """K and V of the keys that some new token sees, once per sequence; the products of visible pairs alone."""
    keys = pairs = 0
    new, total = _lengths(case, 0)
    for n, t in zip(new.tolist(), total.tolist()):
        if n:
            lo, hi = _seen(case, n, t)
            keys += int(hi.max() - lo.min())
            pairs += int((hi - lo).sum())
    tokens, d, e = int(new.sum()), case["d"], _elem(case)
    io = 2 * tokens * case["hq"] * d * e
    kv = 2 * keys * case["hkv"] * d * e
    if case["op"] == "chunk":
        return {"bytes": kv + io + 4 * tokens * case["hq"], "flops": 4 * pairs * case["hq"] * d}
    return {"bytes": kv + io, "flops": 6 * pairs * case["hq"] * d}


# ---- inputs ----

def _pages(case, pages, g):
    """K and V pages [1][pages][hkv][page][d]; token-major pages are a transposed view."""
    hkv, page, d = case["hkv"], case["page"], case["d"]
    inner = (hkv, page) if case["order"] == "head" else (page, hkv)
    kv = []
    for _ in range(2):
        t = torch.empty((1, pages, *inner, d), dtype=_torch_dtype(case), device="cuda").normal_(0.0, 1.0, generator=g)
        kv.append(t if case["order"] == "head" else t.transpose(2, 3))
    return kv


def _table(total, page, pool, g):
    """Page table over a shuffled pool of pages; -1 past a sequence's last page."""
    need = -(-total // page)
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    at = np.full((len(total), max(1, int(need.max()))), -1, dtype=np.int64)
    first = 0
    for b, n in enumerate(need.tolist()):
        at[b, :n] = np.arange(first, first + n)
        first += n
    t = torch.from_numpy(at).cuda()
    return torch.where(t < 0, -1, order[t.clamp_min(0)].long()).to(torch.int32).contiguous()


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new, total = _lengths(case, seed)
    pool = int((-(-total // case["page"])).sum()) + 3
    s = {"new_host": new.tolist(), "lens_host": total.tolist()}
    s["k"], s["v"] = _pages(case, pool, g)
    s["table"] = _table(total, case["page"], pool, g)
    s["lens"] = torch.from_numpy(total.astype(np.int32)).cuda()
    s["cu_new"] = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
    tokens, hq, d = int(new.sum()), case["hq"], case["d"]
    s["q"] = torch.empty((tokens, hq, d), dtype=_torch_dtype(case), device="cuda").normal_(0.0, 1.0, generator=g)
    if case["op"] == "chunk":
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((tokens, hq), dtype=torch.float32, device="cuda")
    else:
        s["out"] = torch.zeros((tokens, hq // 2, 2 * d), dtype=s["q"].dtype, device="cuda")
        s["lam"] = torch.empty(hq // 2, device="cuda").uniform_(0.2, 0.8, generator=g)
        s["weight"] = torch.empty(2 * d, device="cuda").normal_(1.0, 0.1, generator=g) if case["norm"] else None
        s["out_scale"] = 0.5
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:   # the handles and the workspace that a program keeps beside its cache
        import paper_2607_27952_gb300 as last
        s["last"] = last
        s["cache"] = last.Cache(s["k"], s["v"])
        s["seqs"] = last.Sequences(s["table"], s["lens"])
        s["ws"] = last.chunk_workspace(s["cache"], case["hq"])
    return s


# ---- one pass ----

def _run_own(s):
    last, c = s["last"], s["case"]
    cu = None if c["new_lo"] == c["new_hi"] == 1 and not c["empty"] else s["cu_new"]   # one token per sequence
    if c["op"] == "chunk":
        last.last_cache_chunk_attention(s["cache"], 0, s["seqs"], s["q"], s["out"], s["ws"], cu_new=cu, lse=s["lse"],
                                        causal=c["mask"] == "causal", window=c["window"])
        return {"out": s["out"], "lse": s["lse"]}
    last.last_cache_diff_attention(s["cache"], 0, s["seqs"], s["q"], s["out"], s["ws"], s["lam"], cu_new=cu,
                                   norm_weight=s["weight"], norm_eps=_EPS, out_scale=s["out_scale"],
                                   causal=c["mask"] == "causal", window=c["window"])
    return {"out": s["out"]}


def _hidden(case, n, total):
    """[n][total]: keys that a new token does not see."""
    p = torch.arange(total - n, total, device="cuda")[:, None]
    j = torch.arange(total, device="cuda")
    h = j > p if case["mask"] == "causal" else torch.zeros((n, total), dtype=torch.bool, device="cuda")
    return h | (j <= p - case["window"]) if case["window"] else h


def _softmax(q, k, hidden, scale):
    """Weights [kv][group][n][keys] of q [n][kv][group][d] over k [kv][keys][d], and the log of their denominator."""
    z = torch.matmul(q.permute(1, 2, 0, 3), k.transpose(1, 2)[:, None]) * scale
    z.masked_fill_(hidden, -math.inf)
    top = z.amax(-1, keepdim=True)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    return p.div_(total), (total.log() + top)[..., 0]


def _run_plain(s):
    c = s["case"]
    hkv, page, scale = c["hkv"], c["page"], 1.0 / math.sqrt(c["d"])
    units, group = (hkv, c["hq"] // hkv) if c["op"] == "chunk" else (hkv // 2, c["hq"] // hkv)
    t0 = 0
    for b, (n, total) in enumerate(zip(s["new_host"], s["lens_host"])):
        if n == 0:
            continue
        pages = s["table"][b, : -(-total // page)].long()
        k, v = (x[0, pages].transpose(0, 1).flatten(1, 2)[:, :total].float() for x in (s["k"], s["v"]))   # [hkv][keys][d]
        hidden, rows = _hidden(c, n, total), slice(t0, t0 + n)
        q, out = s["q"][rows].float(), s["out"][rows].unflatten(1, (units, group))
        step = max(1, (1 << 28) // (group * n * total))    # units at a time: the weights fill a GB
        for u in range(0, units, step):
            some = slice(u, min(units, u + step))
            if c["op"] == "chunk":
                p, lse = _softmax(q.unflatten(1, (units, group))[:, some], k[some], hidden, scale)
                out[:, some] = torch.matmul(p, v[some, None]).permute(2, 0, 1, 3).to(out.dtype)
                s["lse"][rows].unflatten(1, (units, group))[:, some] = lse.permute(2, 0, 1)
                continue
            maps = q.unflatten(1, (units, group, 2))[:, some]                          # [n][units][group][map][d]
            wide = v.unflatten(0, (units, 2))[some].transpose(1, 2).flatten(2, 3)      # [units][keys][2 d]
            first, second = (torch.matmul(_softmax(maps[..., m, :], k[m::2][some], hidden, scale)[0], wide[:, None])
                             for m in range(2))
            x = first - s["lam"].unflatten(0, (units, group))[some, :, None, None] * second
            if s["weight"] is not None:
                x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + _EPS) * s["weight"]
            out[:, some] = (x * s["out_scale"]).permute(2, 0, 1, 3).to(out.dtype)
        t0 += n
    return {"out": s["out"], "lse": s["lse"]} if c["op"] == "chunk" else {"out": s["out"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the definitions in 64 bits ----

def _exact_rows(q, k, v, lo, hi, scale):
    """q [rows][d], rows' visible keys lo..hi-1 of k and v: outputs and the log of the denominator."""
    a, e = int(lo.min()), int(hi.max())
    j = torch.arange(a, e, device="cuda")
    z = torch.einsum("rd,jd->rj", q, k[a:e]) * scale
    z[(j < lo[:, None]) | (j >= hi[:, None])] = -math.inf
    lse = torch.logsumexp(z, 1)
    return torch.einsum("rj,jd->rd", torch.exp(z - lse[:, None]), v[a:e]), lse


def exact(case, seed):
    if work(case)["flops"] > 1.5e12:
        return None
    s = _inputs(case, seed)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    scale = d ** -0.5
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    t0 = 0
    for b, (n, total) in enumerate(zip(s["new_host"], s["lens_host"])):
        if n == 0:
            continue
        i = torch.arange(total, device="cuda")
        at = s["table"][b].long()[i // case["page"]], i % case["page"]
        lo, hi = (torch.from_numpy(x).cuda() for x in _seen(case, n, total))
        step = max(1, (1 << 26) // total)
        for h in range(hq):
            g = h // (hq // hkv) if case["op"] == "chunk" else (h // 2) // (hq // hkv) * 2 + h % 2
            k = s["k"][0][at[0], g, at[1]].double()
            if case["op"] == "chunk":
                v = s["v"][0][at[0], g, at[1]].double()
            else:
                v = torch.cat([s["v"][0][at[0], g // 2 * 2 + e, at[1]].double() for e in range(2)], dim=1)
            for r in range(0, n, step):
                rows = slice(r, min(n, r + step))
                to = slice(t0 + rows.start, t0 + rows.stop)
                o, l = _exact_rows(s["q"][to, h].double(), k, v, lo[rows], hi[rows], scale)
                if case["op"] == "chunk":
                    out[to, h], lse[to, h] = o, l
                else:
                    out[to, h // 2] += o if h % 2 == 0 else -s["lam"][h // 2].double() * o
        t0 += n
    if case["op"] == "chunk":
        return {"out": out, "lse": lse}
    if s["weight"] is not None:
        out = out * s["weight"].double() * (out.square().mean(-1, keepdim=True) + _EPS).rsqrt()
    return {"out": out * s["out_scale"]}

"""The operators of the key-value cache around the pruning path, as measurable cases.

  rope      rotary positions with several axes on q and K (`last_rope`), and its backward pass
            (`last_rope_backward`)
  append    new tokens' q rotated, their K rotated and written with V into a paged cache
            (`last_cache_append`): single tokens and whole prompts
  attend    attention of one new token per sequence over a paged cache
            (`last_cache_attention`), with the log of the softmax's denominator
  compact   the pruning applied to a cache: of each sequence the text and the kept visual
            tokens, moved into other pages (`last_cache_compact`), every layer, K and V
  copy      pages copied for sequences that part (`last_cache_copy`), every layer, K and V

Sizes are those of the benchmark presets (one image in fp32, a batch of 576-token images,
dynamic resolution, tiled images, video) and odd ones like the tests'.  q and K are
N(0, 1)/sqrt(D) as in `workloads/`; V is N(0, 1).  Visual tokens have the positions of
a (frame, row, column) grid, text tokens the same position on every axis.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_BIG_KEYS = 6 * 115536 * 4      # (token, kv-head) pairs of the largest listed attention
_BIG_ROWS = 32 * 2944           # tokens of the largest listed append


def _attend(name, batch, lo, hi, hq, hkv, d, dtype, page, order, window=0, empty=0):
    """Cached tokens per sequence lo..hi; order: which of a page's heads and tokens is outer;
    window > 0: only the last so many keys; empty: so many sequences without a key."""
    c = dict(op="attend", batch=batch, lo=lo, hi=hi, hq=hq, hkv=hkv, d=d, dtype=dtype, page=page,
             order=order, window=window, empty=empty)
    return dict(c, name=name) if name else c


def _rope(name, tokens, hq, hkv, d, rot, sections, pairs, dtype, backward):
    """sections: frequencies per axis; pairs: "half" (i, i + rot/2) or "adjacent" (2i, 2i + 1)."""
    c = dict(op="rope", tokens=tokens, hq=hq, hkv=hkv, d=d, rot=rot, sections=sections,
             pairs=pairs, dtype=dtype, backward=backward)
    return dict(c, name=name) if name else c


def _append(name, batch, old, lo, hi, hq, hkv, d, rot, sections, pairs, dtype, page, order):
    """lo..hi new tokens per sequence behind `old` cached ones."""
    c = dict(op="append", batch=batch, old=old, lo=lo, hi=hi, hq=hq, hkv=hkv, d=d, rot=rot,
             sections=sections, pairs=pairs, dtype=dtype, page=page, order=order)
    return dict(c, name=name) if name else c


def _compact(name, batch, before, lo, hi, after, den, layers, hkv, d, dtype, page, order):
    """`before` text tokens, lo..hi visual ones of which one in `den` is kept, `after` text tokens."""
    c = dict(op="compact", batch=batch, before=before, lo=lo, hi=hi, after=after, den=den,
             layers=layers, hkv=hkv, d=d, dtype=dtype, page=page, order=order)
    return dict(c, name=name) if name else c


def _copy(name, pages, layers, hkv, d, dtype, page, order):
    c = dict(op="copy", pages=pages, layers=layers, hkv=hkv, d=d, dtype=dtype, page=page, order=order)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the next token after one image and its prompt, fp32: the smallest call, latency
        _attend("attend-image-f32", 1, 608, 608, 16, 16, 64, "f32", 16, "head"),
        # a server's decode step over 576-token images, a K and V head for every query head
        _attend("attend-images", 64, 592, 704, 16, 16, 128, "bf16", 16, "head"),
        # dynamic resolution: ragged lengths, 6 query heads share a K head, token-major pages
        _attend("attend-ragged", 128, 264, 4352, 12, 2, 128, "bf16", 32, "token"),
        # a few long video sessions, odd lengths: the largest
        _attend("attend-long", 6, 99999, 131073, 16, 4, 128, "bf16", 64, "head"),
        # q and K of one video prompt's prefill
        _rope("rope-video", 16512, 16, 4, 128, 128, "16,24,24", "half", "bf16", False),
        # gradients through the rotation, fp32, odd token count, head width 80
        _rope("rope-backward", 1201, 16, 2, 80, 80, "12,14,14", "adjacent", "f32", True),
        # one decode step of 64 sequences
        _append("append-token", 64, 640, 1, 1, 16, 16, 128, 128, "16,24,24", "half", "bf16", 16, "head"),
        # prefill of tiled images: the largest append
        _append("append-tiles", 32, 0, 2944, 2944, 16, 4, 128, 128, "16,24,24", "half", "bf16", 16, "head"),
        # one image's cache cut to 72 of 576 visual tokens, fp32
        _compact("compact-image-f32", 1, 0, 576, 576, 32, 8, 1, 16, 64, "f32", 16, "head"),
        # video caches of 4 layers cut to an eighth
        _compact("compact-video", 8, 5, 16384, 16384, 128, 8, 4, 4, 128, "bf16", 16, "head"),
        # 64 sequences fork: each copies its last, partly filled page
        _copy("copy-tails", 64, 4, 4, 128, "bf16", 16, "head"),
        # a session's whole cache copied, token-major pages
        _copy("copy-session", 2048, 4, 4, 128, "bf16", 16, "token"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend"] * 5 + ["rope"] * 2 + ["append"] * 2 + ["compact"] * 2 + ["copy"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    hq, hkv = rng.choice([(16, 16), (16, 4), (12, 2), (14, 2), (16, 2), (8, 8), (16, 1)])
    d = rng.choice([64, 80, 128, 128])
    page = rng.choice([8, 16, 16, 24, 32, 64])
    order = rng.choice(["head", "token"])
    half = d // 2
    rot = d if rng.random() < 0.8 else 2 * rng.randint(8, half)
    if rng.random() < 0.3:
        sections = str(rot // 2)
    else:
        s0, s1 = rot // 8, 3 * rot // 16
        sections = f"{s0},{s1},{rot // 2 - s0 - s1}"
    pairs = rng.choice(["half", "half", "adjacent"])
    if op == "attend":
        hi = _log_int(rng, 1, 131073)
        batch = _log_int(rng, 1, max(1, min(128, _BIG_KEYS // (2 * hkv * hi))))
        lo = hi if rng.random() < 0.3 else max(1, hi // rng.randint(2, 16))
        window = _log_int(rng, 1, hi) if rng.random() < 0.25 else 0
        return _attend(None, batch, lo, hi, hq, hkv, d, dtype, page, order, window,
                       rng.randint(1, 2) if batch > 2 and rng.random() < 0.3 else 0)
    if op == "rope":
        return _rope(None, _log_int(rng, 1, 40000), hq, hkv, d, rot, sections, pairs, dtype, rng.random() < 0.5)
    if op == "append":
        if rng.random() < 0.5:
            lo = hi = 1
            batch = _log_int(rng, 1, 256)
        else:
            hi = _log_int(rng, 2, 16512)
            batch = _log_int(rng, 1, max(1, min(64, _BIG_ROWS * 5 // (2 * (hq + 2 * hkv) * hi))))
            lo = max(1, hi // rng.randint(1, 4))
        return _append(None, batch, rng.randint(0, 700), lo, hi, hq, hkv, d, rot, sections, pairs,
                       dtype, page, order)
    layers = rng.randint(1, 4)
    if op == "compact":
        hi = _log_int(rng, 16, 16384)
        batch = _log_int(rng, 1, max(1, min(64, 8 * 16384 * 4 // (2 * hi * hkv))))
        return _compact(None, batch, rng.randint(0, 40), max(8, hi // rng.randint(1, 4)), hi, rng.randint(1, 200),
                        rng.choice([2, 4, 5, 8, 10, 20]), layers, hkv, d, dtype, page, order)
    most = max(1, 2048 * 16 * 4 // (2 * page * hkv))
    return _copy(None, _log_int(rng, 1, most), layers, hkv, d, dtype, page, order)


# ---- shapes: host arithmetic ----

def _spread(lo, hi, n, seed):
    """n sizes spread evenly over lo..hi, in a seeded order."""
    v = np.rint(np.linspace(lo, hi, n) if n > 1 else np.array([hi])).astype(np.int64)
    return v[np.random.default_rng([seed, 7]).permutation(n)]


def _cu(v):
    return np.concatenate([[0], np.cumsum(v)]).astype(np.int32)


def _elem(case):
    return 4 if case["dtype"] == "f32" else 2


def _torch_dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _axis_of(case):
    """Axis of each frequency: sections of consecutive frequencies."""
    s = [int(v) for v in case["sections"].split(",")]
    return np.repeat(np.arange(len(s)), s).astype(np.int64)


def _inv_freq(case):
    n = case["rot"] // 2
    return (10000.0 ** (-np.arange(n, dtype=np.float64) / n)).astype(np.float32)


def _kept(case, n):
    return -(-n // case["den"])


def _keys(case):
    """Attended keys over all sequences."""
    n = _spread(case["lo"], case["hi"], case["batch"], 0)
    n = np.minimum(n, case["window"]) if case["window"] else n
    return int(np.sort(n)[: case["batch"] - case["empty"]].sum()) if case["empty"] else int(n.sum())


def work(case):
    e, op, d = _elem(case), case["op"], case["d"]
    if op == "attend":
        keys = _keys(case)
        io = 2 * case["batch"] * case["hq"] * d * e + 4 * case["batch"] * case["hq"]
        return {"bytes": 2 * keys * case["hkv"] * d * e + io, "flops": 4 * keys * case["hq"] * d}
    if op == "rope":
        n = case["tokens"] * (case["hq"] + case["hkv"])
        return {"bytes": 2 * n * d * e + 4 * case["tokens"] * (1 + case["sections"].count(",")),
                "flops": 3 * n * case["rot"]}
    if op == "append":
        t = int(_spread(case["lo"], case["hi"], case["batch"], 0).sum())
        return {"bytes": 2 * t * (case["hq"] + 2 * case["hkv"]) * d * e + 4 * t * (1 + case["sections"].count(",")),
                "flops": 3 * t * (case["hq"] + case["hkv"]) * case["rot"]}
    if op == "compact":
        n = _spread(case["lo"], case["hi"], case["batch"], 0)
        rows = int((_kept(case, n) + case["before"] + case["after"]).sum())
        return {"bytes": 4 * rows * case["layers"] * case["hkv"] * d * e + 4 * rows, "flops": 0}
    return {"bytes": 4 * case["pages"] * case["page"] * case["layers"] * case["hkv"] * d * e, "flops": 0}


# ---- inputs ----

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _pages(case, layers, pages, gen):
    """K and V pages [layers][pages][hkv][page][d]; token-major pages are a transposed view."""
    hkv, page, d = case["hkv"], case["page"], case["d"]
    inner = (hkv, page) if case["order"] == "head" else (page, hkv)
    kv = []
    for scale in (1.0 / math.sqrt(d), 1.0):
        t = torch.empty((layers, pages, *inner, d), dtype=_torch_dtype(case), device="cuda")
        t.normal_(0.0, scale, generator=gen)
        kv.append(t if case["order"] == "head" else t.transpose(2, 3))
    return kv


def _tables(lens, page, pool, gen):
    """Page table over a shuffled pool of pages; -1 past a sequence's last page."""
    need = -(-lens // page)
    order = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32)
    table = np.full((len(lens), max(1, int(need.max()))), -1, dtype=np.int64)
    cu = _cu(need)
    for b, n in enumerate(need):
        table[b, :n] = np.arange(cu[b], cu[b] + n)
    t = torch.from_numpy(table).cuda()
    return torch.where(t < 0, -1, order[t.clamp_min(0)].to(torch.int64)).to(torch.int32).contiguous(), order[int(cu[-1]):]


def _positions(case, tokens, first):
    """[axes][tokens] int32: visual tokens on a (frame, row, column) grid of 16 x 32 tokens a frame
    up to the last 32 tokens, which are text."""
    axes = 1 + case["sections"].count(",")
    i = np.arange(tokens)
    vis = max(0, tokens - 32)
    p = np.stack([first + i] * axes)
    if axes == 3 and vis > 0:
        j = i[:vis]
        p[0, :vis], p[1, :vis], p[2, :vis] = first + j // 512, first + j // 32 % 16, first + j % 32
        p[:, vis:] = first + vis // 512 + 32 + np.arange(tokens - vis)
    return p.astype(np.int32)


def _device(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dtype)


def _attend_inputs(case, seed):
    g = _gen(seed)
    lens = _spread(case["lo"], case["hi"], case["batch"], seed)
    if case["empty"]:
        lens[np.argsort(lens)[len(lens) - case["empty"]:]] = 0
    s = {"lens_host": lens}
    pool = int((-(-lens // case["page"])).sum()) + 3
    s["k"], s["v"] = _pages(case, 1, pool, g)
    s["table"], _ = _tables(lens, case["page"], pool, g)
    s["lens"] = _device(lens)
    s["begin"] = _device(np.maximum(0, lens - case["window"])) if case["window"] else None
    q = torch.empty((case["batch"], case["hq"], case["d"]), dtype=_torch_dtype(case), device="cuda")
    s["q"] = q.normal_(0.0, 1.0, generator=g)
    s["out"] = torch.zeros_like(q)
    s["lse"] = torch.zeros((case["batch"], case["hq"]), dtype=torch.float32, device="cuda")
    return s


def _heads(shape, scale, case, g):
    return torch.empty(shape, dtype=_torch_dtype(case), device="cuda").normal_(0.0, scale, generator=g)


def _rope_inputs(case, seed):
    g, t, d = _gen(seed), case["tokens"], case["d"]
    s = {"pos": _device(_positions(case, t, seed % 50))}
    s["q"] = _heads((t, case["hq"], d), 1.0, case, g)
    s["k"] = _heads((t, case["hkv"], d), 1.0, case, g)
    s["q_out"], s["k_out"] = torch.zeros_like(s["q"]), torch.zeros_like(s["k"])
    return s


def _append_inputs(case, seed):
    g, d = _gen(seed), case["d"]
    new = _spread(case["lo"], case["hi"], case["batch"], seed)
    lens = case["old"] + new
    pool = int((-(-lens // case["page"])).sum()) + 3
    s = {"new_host": new, "lens_host": lens, "lens": _device(lens), "cu_new": _device(_cu(new))}
    s["k"], s["v"] = _pages(case, 1, pool, g)
    s["table"], _ = _tables(lens, case["page"], pool, g)
    one = new.max() == 1
    s["pos"] = _device(np.full((1 + case["sections"].count(","), len(new)), case["old"] + seed % 50) if one else
                       np.concatenate([_positions(case, int(n), case["old"]) for n in new], axis=1))
    t = int(new.sum())
    s["q"] = _heads((t, case["hq"], d), 1.0, case, g)
    # k and v of a token lie side by side, as a fused projection leaves them
    s["k_new"], s["v_new"] = _heads((t, 2 * case["hkv"], d), 1.0, case, g).chunk(2, dim=1)
    s["q_out"] = torch.zeros_like(s["q"])
    return s


def _compact_inputs(case, seed):
    g, rng = _gen(seed), np.random.default_rng([seed, 3])
    n = _spread(case["lo"], case["hi"], case["batch"], seed)
    lens = n + case["before"] + case["after"]
    kept = _kept(case, n)
    short = kept + case["before"] + case["after"]
    pool = int((-(-lens // case["page"])).sum() + (-(-short // case["page"])).sum()) + 3
    s = {"lens_host": lens, "kept_host": kept, "rows": int(short.sum()), "lens": _device(lens)}
    s["k"], s["v"] = _pages(case, case["layers"], pool, g)
    s["table"], rest = _tables(lens, case["page"], pool, g)
    need = -(-short // case["page"])
    dst = np.full((len(n), int(need.max())), -1, dtype=np.int32)
    cu, rest = _cu(need), rest.cpu().numpy()
    for b, m in enumerate(need):
        dst[b, :m] = rest[cu[b]:cu[b] + m]
    s["dst"] = _device(dst)
    s["cu_keep"] = _device(_cu(kept))
    s["idx_host"] = [np.sort(rng.choice(int(v), size=int(k), replace=False)) for v, k in zip(n, kept)]
    s["idx"] = _device(np.concatenate(s["idx_host"]))
    s["span_begin"] = _device(np.full(len(n), case["before"]))
    s["span_len"] = _device(n)
    s["lens_out"] = torch.zeros(len(n), dtype=torch.int32, device="cuda")
    return s


def _copy_inputs(case, seed):
    g, n = _gen(seed), case["pages"]
    s = {}
    s["k"], s["v"] = _pages(case, case["layers"], 2 * n + 3, g)
    order = torch.randperm(2 * n + 3, generator=g, device="cuda").to(torch.int32)
    s["src"], s["dst"] = order[:n].clone(), order[n:2 * n].clone()
    return s


_INPUTS = {"attend": _attend_inputs, "rope": _rope_inputs, "append": _append_inputs,
           "compact": _compact_inputs, "copy": _copy_inputs}


def prepare(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    s["case"] = case
    if case["op"] in ("rope", "append"):
        s["inv_freq"], s["axis"] = _device(_inv_freq(case), torch.float32), _device(_axis_of(case), torch.int64)
    if own:   # the handles and the workspace that a program keeps beside its cache
        import paper_2607_27952_gb300 as last
        s["last"] = last
        if case["op"] in ("rope", "append"):
            s["rope"] = last.Rope(_inv_freq(case), axis=_axis_of(case), pairs=case["pairs"],
                                  num_axes=1 + case["sections"].count(","))
        if case["op"] != "rope":
            s["cache"] = last.Cache(s["k"], s["v"])
            s["ws"] = last.cache_workspace(s["cache"], case.get("batch", 1), case.get("hq", case["hkv"]))
        if case["op"] not in ("rope", "copy"):
            s["seqs"] = last.Sequences(s["table"], s["lens"], key_begin=s.get("begin"))
    return s


# ---- one pass ----

def _run_own(s):
    last, op = s["last"], s["case"]["op"]
    if op == "attend":
        last.last_cache_attention(s["cache"], 0, s["seqs"], s["q"], s["out"], s["ws"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "rope":
        call = last.last_rope_backward if s["case"]["backward"] else last.last_rope
        call(s["rope"], s["pos"], s["q"], s["q_out"], k=s["k"], k_out=s["k_out"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "append":
        last.last_cache_append(s["cache"], 0, s["seqs"], s["k_new"], s["v_new"], s["ws"], cu_new=s["cu_new"],
                               rope=s["rope"], positions=s["pos"], q=s["q"], q_out=s["q_out"])
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    if op == "compact":
        last.last_cache_compact(s["cache"], s["seqs"], s["dst"], s["cu_keep"], s["idx"], s["lens_out"], s["ws"],
                                span_begin=s["span_begin"], span_len=s["span_len"])
        return {"k": s["k"], "v": s["v"], "lens": s["lens_out"]}
    last.last_cache_copy(s["cache"], s["src"], s["dst"], s["ws"])
    return {"k": s["k"], "v": s["v"]}


def _turn(x, pos, s, back):
    """The rotation in fp32, rounded once."""
    rot, n = s["case"]["rot"], s["case"]["rot"] // 2
    phi = pos[s["axis"]].t().float() * s["inv_freq"]            # [tokens][rot/2]
    cos, sin = phi.cos()[:, None], phi.sin()[:, None]
    sin = -sin if back else sin
    y = x.float()
    if s["case"]["pairs"] == "half":
        a, b = y[..., :n], y[..., n:rot]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], dim=-1).to(x.dtype)


def _attend_plain(s):
    c = s["case"]
    B, hkv, d, page = c["batch"], c["hkv"], c["d"], c["page"]
    table = s["table"].long().clamp_min(0)
    n = table.shape[1] * page
    k = s["k"][0][table].transpose(2, 3).reshape(B, n, hkv, d)   # [B][pages][hkv][page][d] by token
    v = s["v"][0][table].transpose(2, 3).reshape(B, n, hkv, d)
    q = s["q"].float().view(B, hkv, -1, d)
    z = torch.matmul(q, k.permute(0, 2, 3, 1).float()) * (1.0 / math.sqrt(d))   # [B][hkv][group][n]
    at = torch.arange(n, device="cuda")
    seen = at < s["lens"][:, None]
    if s["begin"] is not None:
        seen = seen & (at >= s["begin"][:, None])
    z = torch.where(seen[:, None, None], z, -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = (z - top).exp()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v.permute(0, 2, 1, 3).float()) / torch.where(total == 0, 1.0, total)
    s["out"].copy_(o.view(B, -1, d))
    s["lse"].copy_((total.log() + top).view(B, -1))
    return {"out": s["out"], "lse": s["lse"]}


def _append_plain(s):
    c = s["case"]
    t = s["q"].shape[0]
    i = torch.arange(t, device="cuda")
    b = torch.searchsorted(s["cu_new"][1:].long(), i, right=True)
    at = s["lens"].long()[b] - (s["cu_new"].long()[b + 1] - i)
    page, slot = s["table"].long()[b, at // c["page"]], at % c["page"]
    s["q_out"].copy_(_turn(s["q"], s["pos"], s, False))
    s["k"][0][page, :, slot] = _turn(s["k_new"], s["pos"], s, False)
    s["v"][0][page, :, slot] = s["v_new"]
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


def _compact_plain(s):
    page = s["case"]["page"]
    kept = (s["cu_keep"][1:] - s["cu_keep"][:-1]).long()
    lens, first, span = s["lens"].long(), s["span_begin"].long(), s["span_len"].long()
    short = lens - span + kept
    cu = torch.cumsum(short, 0)
    i = torch.arange(s["rows"], device="cuda")
    b = torch.searchsorted(cu, i, right=True)
    at = i - (cu - short)[b]                                     # row of the new sequence
    j = at - first[b]                                            # which kept token it is
    chosen = (s["cu_keep"].long()[b] + j).clamp(0, max(0, s["idx"].numel() - 1))
    src = torch.where(j < 0, at, torch.where(j < kept[b], first[b] + s["idx"].long()[chosen], at + (span - kept)[b]))
    sp, so = s["table"].long()[b, src // page], src % page
    dp, do = s["dst"].long()[b, at // page], at % page
    for t in (s["k"], s["v"]):
        t[:, dp, :, do] = t[:, sp, :, so]
    s["lens_out"].copy_(short)
    return {"k": s["k"], "v": s["v"], "lens": s["lens_out"]}


def run(state):
    s = state
    if own:
        return _run_own(s)
    op = s["case"]["op"]
    if op == "attend":
        return _attend_plain(s)
    if op == "rope":
        back = s["case"]["backward"]
        s["q_out"].copy_(_turn(s["q"], s["pos"], s, back))
        s["k_out"].copy_(_turn(s["k"], s["pos"], s, back))
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "append":
        return _append_plain(s)
    if op == "compact":
        return _compact_plain(s)
    src, dst = s["src"].long(), s["dst"].long()
    s["k"][:, dst] = s["k"][:, src]
    s["v"][:, dst] = s["v"][:, src]
    return {"k": s["k"], "v": s["v"]}


# ---- the definitions in 64 bits ----

def _exact_turn(x, pos, case, sign):
    """Frequency by frequency: one complex product per pair."""
    y = x.double().clone()
    f, axis, n = _inv_freq(case).astype(np.float64), _axis_of(case), case["rot"] // 2
    p = pos.double()
    for i in range(n):
        a, b = (i, i + n) if case["pairs"] == "half" else (2 * i, 2 * i + 1)
        w = torch.polar(torch.ones_like(p[0]), sign * p[int(axis[i])] * float(f[i]))[:, None]
        z = torch.complex(x[..., a].double(), x[..., b].double()) * w
        y[..., a], y[..., b] = z.real, z.imag
    return y


def _token_slots(table_row, n, page):
    i = torch.arange(n, device="cuda")
    return table_row.long()[i // page], i % page


def exact(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    op = case["op"]
    if op == "attend":
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
        group = case["hq"] // case["hkv"]
        for b, n in enumerate(s["lens_host"]):
            first = max(0, int(n) - case["window"]) if case["window"] else 0
            if n <= first:
                continue
            p, o = _token_slots(s["table"][b], int(n), case["page"])
            p, o = p[first:], o[first:]
            for h in range(case["hq"]):
                k, v = s["k"][0][p, h // group, o].double(), s["v"][0][p, h // group, o].double()
                z = (k * s["q"][b, h].double()).sum(1) / math.sqrt(case["d"])
                lse[b, h] = torch.logsumexp(z, 0)
                out[b, h] = (torch.exp(z - lse[b, h])[:, None] * v).sum(0)
        return {"out": out, "lse": lse}
    if op == "rope":
        sign = -1.0 if case["backward"] else 1.0
        return {"q": _exact_turn(s["q"], s["pos"], case, sign), "k": _exact_turn(s["k"], s["pos"], case, sign)}
    k, v = s["k"].double(), s["v"].double()
    if op == "append":
        q = _exact_turn(s["q"], s["pos"], case, 1.0)
        kr, t = _exact_turn(s["k_new"], s["pos"], case, 1.0), 0
        for b, (m, n) in enumerate(zip(s["new_host"], s["lens_host"])):
            p, o = _token_slots(s["table"][b], int(n), case["page"])
            p, o = p[int(n - m):], o[int(n - m):]
            k[0][p, :, o], v[0][p, :, o] = kr[t:t + int(m)], s["v_new"][t:t + int(m)].double()
            t += int(m)
        return {"q": q, "k": k, "v": v}
    if op == "compact":
        k0, v0 = s["k"], s["v"]
        for b, n in enumerate(s["lens_host"]):
            a, m = case["before"], int(n) - case["after"]
            keep = np.concatenate([np.arange(a), a + s["idx_host"][b], np.arange(m, int(n))])
            p, o = _token_slots(s["table"][b], int(n), case["page"])
            at = torch.from_numpy(keep).cuda()
            p, o = p[at], o[at]
            dp, do = _token_slots(s["dst"][b], len(keep), case["page"])
            k[:, dp, :, do], v[:, dp, :, do] = k0[:, p, :, o].double(), v0[:, p, :, o].double()
        return {"k": k, "v": v, "lens": None}
    for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
        k[:, b], v[:, b] = s["k"][:, a].double(), s["v"][:, a].double()
    return {"k": k, "v": v}

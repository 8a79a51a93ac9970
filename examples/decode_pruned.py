"""The pruning path inside a model's attention: prefill, prune, shorten the cache, fork, decode.

A model's layers are stood in for by random q, K and V; everything else is what a serving
program does with liblast around them:

  1. last_rope turns the guidance layer's last query and keys by their (frame, row, column)
     positions, last_cache_append does the same for every layer and fills the paged cache;
  2. last_prune scores and selects the visual tokens to keep;
  3. last_cache_compact moves the text and the kept tokens into new pages of every layer, and
     the old pages go back to the pool;
  4. a second continuation of the first request shares its full pages and copies the last,
     partly filled one (last_cache_copy);
  5. every decoding step appends one token per sequence and attends over what the cache holds.

  python examples/decode_pruned.py [--requests 4 --visual 576 --steps 16 --check]

--check compares every attention output with a dense softmax in 64 bits.
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import numpy as np  # noqa: E402
import torch  # noqa: E402

import paper_2607_27952_gb300 as last  # noqa: E402


def positions(n_before: int, n_vis: int, n_text: int, width: int = 24) -> np.ndarray:
    """[3][tokens]: text advances on all axes together, visual tokens lie on a grid of one frame."""
    before = np.tile(np.arange(n_before), (3, 1))
    i = np.arange(n_vis)
    vis = np.stack([np.zeros(n_vis, int), i // width, i % width]) + n_before
    at = n_before + max(1, -(-n_vis // width), min(n_vis, width))
    return np.concatenate([before, vis, np.tile(at + np.arange(n_text), (3, 1))], axis=1).astype(np.int32)


class Session:
    """A paged cache, its pages and its sequences' tables."""

    def __init__(self, layers, pages, kv_heads, page_size, head_dim, dtype, max_seqs, max_pages):
        shape = (layers, pages, kv_heads, page_size, head_dim)
        self.cache = last.Cache(torch.empty(shape, dtype=dtype, device="cuda"), torch.empty(shape, dtype=dtype, device="cuda"))
        self.pool, self.size = last.PagePool(pages), page_size
        self.pages = [np.zeros(0, np.int32) for _ in range(max_seqs)]     # by sequence, host
        self.host_lens = np.zeros(max_seqs, np.int64)
        self.table = torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(max_seqs, dtype=torch.int32, device="cuda")

    def hold(self, b: int, pages: np.ndarray):
        self.pages[b] = pages
        self.table[b, :len(pages)] = torch.from_numpy(pages).cuda()

    def room(self, b: int, tokens: int):
        """Takes the pages that sequence b needs to hold so many tokens."""
        more = -(-tokens // self.size) - len(self.pages[b])
        if more > 0:
            self.hold(b, np.concatenate([self.pages[b], last.last_pages_take(self.pool, more)]))
        self.host_lens[b] = tokens
        self.lens[b] = tokens

    def sequences(self, n: int) -> last.Sequences:
        return last.Sequences(self.table[:n], self.lens[:n])


def dense(cache, pages, n, layer, q, size):
    """Attention of one query over the cache's first n tokens, in 64 bits."""
    p = torch.from_numpy(pages.astype(np.int64)).cuda()
    k, v = (t[layer, p].transpose(1, 2).flatten(0, 1)[:n].double() for t in (cache.k, cache.v))   # [n][heads][d]
    g = q.shape[0] // k.shape[1]
    z = torch.einsum("hd,nhd->hn", q.double(), k.repeat_interleave(g, 1)) / q.shape[1] ** 0.5
    return torch.einsum("hn,nhd->hd", torch.softmax(z, 1), v.repeat_interleave(g, 1))


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--visual", type=int, default=576)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--page", type=int, default=16)
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args(argv)
    B, N, L, hq, hkv, d, dv, before = a.requests, a.visual, a.layers, 16, 4, 128, 1024, 5
    text = [24 + 3 * b for b in range(B)]
    lens = np.array([before + N + t for t in text])
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    T, keep = int(cu[-1]), [last.last_budget(N, 1, 8)] * B
    gen = torch.Generator(device="cuda").manual_seed(1)

    def rand(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * scale).bfloat16()

    rope = last.Rope.sections([16, 24, 24])
    pos_host = [positions(before, N, t) for t in text]
    pos = torch.from_numpy(np.concatenate(pos_host, axis=1)).cuda()
    need = sum(-(-int(n) // a.page) for n in lens) * 2 + (B + 1) * (a.steps // a.page + 2)
    s = Session(L, need, hkv, a.page, d, torch.bfloat16, B + 1, int(lens.max()) // a.page + a.steps + 2)
    ws = last.cache_workspace(s.cache, B + 1, hq)

    # 1. prefill: every layer's q and K turned by their positions, K and V into the cache
    for b in range(B):
        s.room(b, int(lens[b]))
    q, k, v = rand(L, T, hq, d, scale=d ** -0.25), rand(L, T, hkv, d, scale=d ** -0.25), rand(L, T, hkv, d)
    q_rot, cu_dev = torch.empty_like(q), torch.from_numpy(cu).cuda()
    for layer in range(L):
        last.last_cache_append(s.cache, layer, s.sequences(B), k[layer], v[layer], ws, cu_new=cu_dev, rope=rope,
                               positions=pos, q=q[layer], q_out=q_rot[layer])

    # 2. the pruning, guided by the first layer: its last query row and its keys
    k_rot = torch.empty_like(k[:1])
    at_last = torch.from_numpy(cu[1:].astype(np.int64) - 1).cuda()
    last.last_rope(rope, pos, k[0], k_rot[0])
    problem = last.Problem(batch=B, num_layers=1, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, feat_dim=dv, dtype="bf16",
                           cu_seqlens=cu, vis_start=[before] * B, cu_vis=np.arange(B + 1) * N,
                           cu_keep=np.concatenate([[0], np.cumsum(keep)]))
    x, w = rand(B * N, dv), torch.empty(B * N, device="cuda")
    idx = torch.empty(problem.total_keep, dtype=torch.int32, device="cuda")
    x_kept = torch.empty((problem.total_keep, dv), dtype=x.dtype, device="cuda")
    prune_ws = last.workspace(problem)
    last.last_prune(problem, q_rot[0, at_last][:, None].contiguous(), k_rot, x, w, idx, x_kept, prune_ws)
    last.last_poll(prune_ws)

    # 3. the cache shortened to the text and the kept tokens, the old pages given back
    old = s.pages[:B]
    short = lens - N + np.array(keep)
    new = [last.last_pages_take(s.pool, -(-int(n) // a.page)) for n in short]
    dst = torch.full((B, max(len(p) for p in new)), -1, dtype=torch.int32)
    for b in range(B):
        dst[b, :len(new[b])] = torch.from_numpy(new[b])
    lens_out = torch.empty(B, dtype=torch.int32, device="cuda")
    last.last_cache_compact(s.cache, s.sequences(B), dst.cuda(), torch.from_numpy(problem.arrays["cu_keep"]).cuda(), idx, lens_out, ws,
                            span_begin=torch.full_like(lens_out, before), span_len=torch.full_like(lens_out, N))
    last.last_poll(ws)
    assert lens_out.tolist() == short.tolist()
    for b in range(B):
        last.last_pages_release(s.pool, old[b])
        s.table[b] = -1
        s.hold(b, new[b])
        s.room(b, int(short[b]))

    # 4. a second continuation of request 0: full pages shared, the last one copied
    full = int(short[0]) // a.page
    last.last_pages_share(s.pool, s.pages[0][:full])
    s.hold(B, s.pages[0][:full])
    s.room(B, int(short[0]))
    if short[0] % a.page:
        last.last_cache_copy(s.cache, torch.from_numpy(s.pages[0][full:full + 1]).cuda(),
                             torch.from_numpy(s.pages[B][full:full + 1]).cuda(), ws)
        last.last_poll(ws)

    # 5. decoding: one token per sequence and step
    worst, out = 0.0, torch.empty((B + 1, hq, d), dtype=torch.bfloat16, device="cuda")
    next_pos = np.array([p[0, -1] + 1 for p in pos_host] + [pos_host[0][0, -1] + 1])
    q_new = torch.empty_like(out)
    for step in range(a.steps):
        for b in range(B + 1):
            s.room(b, int(s.host_lens[b]) + 1)
        p = torch.from_numpy(np.tile(next_pos + step, (3, 1)).astype(np.int32)).cuda()
        for layer in range(L):
            qkv = rand(B + 1, hq + 2 * hkv, d, scale=d ** -0.25)
            last.last_cache_append(s.cache, layer, s.sequences(B + 1), qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], ws, rope=rope,
                                   positions=p, q=qkv[:, :hq], q_out=q_new)
            last.last_cache_attention(s.cache, layer, s.sequences(B + 1), q_new, out, ws)
            if a.check:
                last.last_poll(ws)
                for b in range(B + 1):
                    want = dense(s.cache, s.pages[b], int(s.host_lens[b]), layer, q_new[b], a.page)
                    worst = max(worst, float((out[b].double() - want).norm() / want.norm()))
    last.last_poll(ws)
    got = {"prompt_tokens": lens.tolist(), "cached_after_pruning": short.tolist(), "cached_at_the_end": s.host_lens.tolist(),
           "pages_free": s.pool.num_free, "pages": need, "worst_relative_error": worst if a.check else None}
    for b in range(B + 1):
        last.last_pages_release(s.pool, s.pages[b])
    assert s.pool.num_free == need
    return got


if __name__ == "__main__":
    print(main())

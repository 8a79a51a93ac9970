"""CPU-side checks of the rotary positions and the key-value cache: arguments are refused on
the host before any launch, and the page pool is host code (no compute call runs here)."""
import ctypes

import numpy as np
import pytest

import paper_2607_27952_gb300 as last

ONE_PAIR = (ctypes.c_float * 4)(1.0, 0.5, 0.25, 0.125)
AXES = (ctypes.c_int32 * 4)(0, 1, 2, 0)


@pytest.fixture(scope="module")
def lib():
    from paper_2607_27952_gb300.build import build
    build()
    return last.load_library()


def _rotary(**kw):
    f = dict(rot_dim=8, num_axes=3, pairs=0, inv_freq=ONE_PAIR, axis=AXES)
    f.update(kw)
    return last._Rotary(f["rot_dim"], f["num_axes"], f["pairs"],
                        ctypes.cast(f["inv_freq"], ctypes.POINTER(ctypes.c_float)),
                        ctypes.cast(f["axis"], ctypes.POINTER(ctypes.c_int32)))


def _heads(**kw):
    f = dict(in_=16, out=16, heads=2, in_token=128, in_head=64, out_token=128, out_head=64)
    f.update(kw)
    return last._Heads(*f.values())


def _cache(**kw):
    f = dict(k=4096, v=8192, num_layers=2, num_pages=10, page_size=16, num_kv_heads=2, head_dim=64, dtype=1,
             layer_stride=20480, page_stride=2048, head_stride=1024, token_stride=64)
    f.update(kw)
    return last._Cache(*f.values())


def _seqs(**kw):
    f = dict(batch=3, max_pages=4, table_stride=4, page_table=512, lens=256, key_begin=None)
    f.update(kw)
    return last._Sequences(*f.values())


def _status(st):
    return st, last.load_library().last_error_message().decode()


def _rope(lib, r=None, h=None, k=None, dtype=1, tokens=5, dim=64, pos=16, stride=5, back=False):
    r, h = r or _rotary(), h or _heads()
    call = lib.last_rope_backward if back else lib.last_rope
    return call(ctypes.byref(r), dtype, tokens, dim, pos, stride, ctypes.byref(h),
                ctypes.byref(k) if k else None, 0)


BAD_AXES = (ctypes.c_int32 * 4)(0, 3, 0, 0)
BAD_FREQ = (ctypes.c_float * 4)(1.0, float("nan"), 0, 0)
BIG_FREQ = (ctypes.c_float * 4)(1.0, 65537.0, 0, 0)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), last.LAST_ERR_INVALID_ARG),
    (dict(tokens=-1), last.LAST_ERR_INVALID_ARG),
    (dict(dim=264), last.LAST_ERR_UNSUPPORTED),
    (dict(dim=1), last.LAST_ERR_INVALID_ARG),
    (dict(dim=6), last.LAST_ERR_INVALID_ARG),                        # rot_dim > head_dim
    (dict(pos=None), last.LAST_ERR_INVALID_ARG),
    (dict(stride=4), last.LAST_ERR_INVALID_ARG),                     # axes overlap
    (dict(r=_rotary(rot_dim=7)), last.LAST_ERR_INVALID_ARG),
    (dict(r=_rotary(rot_dim=0)), last.LAST_ERR_INVALID_ARG),
    (dict(r=_rotary(num_axes=0)), last.LAST_ERR_INVALID_ARG),
    (dict(r=_rotary(num_axes=5)), last.LAST_ERR_INVALID_ARG),
    (dict(r=_rotary(pairs=2)), last.LAST_ERR_INVALID_ARG),
    (dict(r=_rotary(axis=BAD_AXES)), last.LAST_ERR_INVALID_ARG),
    (dict(r=_rotary(inv_freq=BAD_FREQ)), last.LAST_ERR_INVALID_ARG),
    (dict(r=_rotary(inv_freq=BIG_FREQ)), last.LAST_ERR_INVALID_ARG),
    (dict(h=_heads(in_=None)), last.LAST_ERR_INVALID_ARG),
    (dict(h=_heads(out=None)), last.LAST_ERR_INVALID_ARG),
    (dict(h=_heads(heads=0)), last.LAST_ERR_INVALID_ARG),
    (dict(h=_heads(in_=17)), last.LAST_ERR_INVALID_ARG),             # not a whole element
    (dict(k=_heads(heads=-1)), last.LAST_ERR_INVALID_ARG),
])
def test_rope_refuses(lib, kw, status, back):
    st, msg = _status(_rope(lib, back=back, **kw))
    assert st == status and msg


def test_rope_of_no_tokens_is_nothing(lib):
    assert _rope(lib, tokens=0, pos=None, h=_heads(in_=None, out=None)) == last.LAST_OK


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), last.LAST_ERR_INVALID_ARG),
    (dict(num_layers=0), last.LAST_ERR_INVALID_ARG),
    (dict(num_pages=0), last.LAST_ERR_INVALID_ARG),
    (dict(num_kv_heads=0), last.LAST_ERR_INVALID_ARG),
    (dict(page_size=0), last.LAST_ERR_INVALID_ARG),
    (dict(page_size=12), last.LAST_ERR_INVALID_ARG),
    (dict(head_dim=0), last.LAST_ERR_INVALID_ARG),
    (dict(head_dim=60), last.LAST_ERR_UNSUPPORTED),                  # 120-byte rows
    (dict(head_dim=320, token_stride=320), last.LAST_ERR_UNSUPPORTED),
    (dict(k=None), last.LAST_ERR_INVALID_ARG),
    (dict(v=8), last.LAST_ERR_INVALID_ARG),
    (dict(page_stride=2044), last.LAST_ERR_INVALID_ARG),             # 4088 bytes
    (dict(page_stride=-2048), last.LAST_ERR_INVALID_ARG),
    (dict(token_stride=56), last.LAST_ERR_INVALID_ARG),
])
def test_cache_calls_refuse_a_bad_cache(lib, kw, status):
    c, s, h = ctypes.byref(_cache(**kw)), ctypes.byref(_seqs()), ctypes.byref(_heads())
    n = ctypes.c_size_t(0)
    big = 1 << 30
    for st in (lib.last_cache_workspace_size(c, 3, 4, ctypes.byref(n)),
               lib.last_cache_append(c, 0, s, 3, None, None, None, 0, None, h, h, 256, big, 0),
               lib.last_cache_attention(c, 0, s, 4, 0.0, 256, 256, 256, 256, None, 256, big, 0),
               lib.last_cache_copy(c, 1, 256, 256, 256, big, 0),
               lib.last_cache_compact(c, s, 256, 4, 4, None, None, 256, 256, 5, 512, 256, big, 0)):
        assert st == status and last.load_library().last_error_message()


@pytest.mark.parametrize("kw", [dict(batch=-1), dict(page_table=None), dict(lens=None), dict(max_pages=-1),
                                dict(table_stride=3)])
def test_cache_calls_refuse_bad_sequences(lib, kw):
    c, s, h = ctypes.byref(_cache()), ctypes.byref(_seqs(**kw)), ctypes.byref(_heads())
    big = 1 << 30
    for st in (lib.last_cache_append(c, 0, s, 3, 256, None, None, 0, None, h, h, 256, big, 0),
               lib.last_cache_attention(c, 0, s, 4, 0.0, 256, 256, 256, 256, None, 256, big, 0),
               lib.last_cache_compact(c, s, 256, 4, 4, None, None, 256, 256, 5, 512, 256, big, 0)):
        assert st == last.LAST_ERR_INVALID_ARG


def _append(lib, layer=0, tokens=3, cu=None, r=None, pos=None, q=None, k=None, v=None, ws=256, ws_bytes=1 << 30, s=None):
    ref = lambda x: ctypes.byref(x) if x else None  # noqa: E731
    return lib.last_cache_append(ctypes.byref(_cache()), layer, ctypes.byref(s or _seqs()), tokens, cu, ref(r), pos, 3,
                                 ref(q), ref(k or _heads()), ref(v or _heads()), ws, ws_bytes, 0)


@pytest.mark.parametrize("kw,status", [
    (dict(layer=-1), last.LAST_ERR_INVALID_ARG),
    (dict(layer=2), last.LAST_ERR_INVALID_ARG),
    (dict(tokens=-1), last.LAST_ERR_INVALID_ARG),
    (dict(tokens=4), last.LAST_ERR_INVALID_ARG),                     # one per sequence without cu_new
    (dict(q=_heads()), last.LAST_ERR_INVALID_ARG),                   # q without a rotation
    (dict(r=_rotary(), q=_heads()), last.LAST_ERR_INVALID_ARG),      # no positions
    (dict(r=_rotary(rot_dim=66), pos=16), last.LAST_ERR_INVALID_ARG),
    (dict(k=_heads(heads=3)), last.LAST_ERR_INVALID_ARG),
    (dict(v=_heads(in_=None)), last.LAST_ERR_INVALID_ARG),
    (dict(ws=None), last.LAST_ERR_INVALID_ARG),
    (dict(ws=128), last.LAST_ERR_INVALID_ARG),
    (dict(ws_bytes=1024), last.LAST_ERR_WORKSPACE_TOO_SMALL),
])
def test_append_refuses(lib, kw, status):
    assert _append(lib, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(heads=3), last.LAST_ERR_INVALID_ARG),                      # not a multiple of the kv-heads
    (dict(heads=0), last.LAST_ERR_INVALID_ARG),
    (dict(heads=8194), last.LAST_ERR_UNSUPPORTED),
    (dict(q=None), last.LAST_ERR_INVALID_ARG),
    (dict(out=None), last.LAST_ERR_INVALID_ARG),
    (dict(q=264), last.LAST_ERR_INVALID_ARG),
    (dict(qs=257), last.LAST_ERR_INVALID_ARG),
    (dict(os=248), last.LAST_ERR_INVALID_ARG),                       # sequences overlap
    (dict(lse=2), last.LAST_ERR_INVALID_ARG),
    (dict(ws_bytes=1024), last.LAST_ERR_WORKSPACE_TOO_SMALL),
])
def test_attention_refuses(lib, kw, status):
    f = dict(heads=4, q=256, qs=256, out=256, os=256, lse=None, ws_bytes=1 << 40)
    f.update(kw)
    assert lib.last_cache_attention(ctypes.byref(_cache()), 0, ctypes.byref(_seqs()), f["heads"], 0.0, f["q"], f["qs"],
                                    f["out"], f["os"], f["lse"], 256, f["ws_bytes"], 0) == status


def test_copy_and_compact_refuse(lib):
    c, s = ctypes.byref(_cache()), ctypes.byref(_seqs())
    big = 1 << 30
    bad = last.LAST_ERR_INVALID_ARG
    assert lib.last_cache_copy(c, -1, 256, 256, 256, big, 0) == bad
    assert lib.last_cache_copy(c, 1, None, 256, 256, big, 0) == bad
    assert lib.last_cache_copy(c, 1, 256, None, 256, big, 0) == bad
    assert lib.last_cache_copy(c, 1, 256, 256, 256, 1024, 0) == last.LAST_ERR_WORKSPACE_TOO_SMALL
    ok = dict(dst=512, pages=4, stride=4, begin=256, span=256, cu=256, idx=256, n=5, out=512, ws=256, size=big)
    for kw in (dict(dst=None), dict(pages=0), dict(stride=3), dict(begin=None), dict(span=None), dict(cu=None),
               dict(idx=None), dict(n=-1), dict(out=None), dict(out=256), dict(ws=None), dict(ws=8)):
        a = {**ok, **kw}
        assert lib.last_cache_compact(c, s, a["dst"], a["pages"], a["stride"], a["begin"], a["span"], a["cu"], a["idx"],
                                      a["n"], a["out"], a["ws"], a["size"], 0) == bad, kw


def test_workspace_size_of_a_cache(lib):
    n, m = ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert lib.last_cache_workspace_size(ctypes.byref(_cache()), 3, 4, ctypes.byref(n)) == last.LAST_OK
    assert lib.last_cache_workspace_size(ctypes.byref(_cache()), 4000, 4, ctypes.byref(m)) == last.LAST_OK
    assert 0 < n.value <= m.value
    for batch, heads in ((-1, 4), (3, 0), (3, 3)):
        assert lib.last_cache_workspace_size(ctypes.byref(_cache()), batch, heads, ctypes.byref(n)) == last.LAST_ERR_INVALID_ARG
    assert lib.last_cache_workspace_size(ctypes.byref(_cache()), 3, 4, None) == last.LAST_ERR_INVALID_ARG


# ---- the page pool ----

def test_pool_against_counts(lib):
    """Random takes, forks and releases against a plain count per page."""
    rng = np.random.default_rng(3)
    pool, counts, lists = last.PagePool(37), np.zeros(37, int), []
    for _ in range(2000):
        what = rng.integers(3)
        if what == 0:
            n = int(rng.integers(0, 9))
            if n > pool.num_free:
                with pytest.raises(last.LastError) as e:
                    last.last_pages_take(pool, n)
                assert e.value.status == last.LAST_ERR_NO_PAGES
            else:
                pages = last.last_pages_take(pool, n)
                assert len(set(pages.tolist())) == n and (counts[pages] == 0).all()
                counts[pages] = 1
                lists.append(pages)
        elif lists and what == 1:
            pages = lists[int(rng.integers(len(lists)))]
            last.last_pages_share(pool, pages)
            counts[pages] += 1
            lists.append(pages)
        elif lists:
            pages = lists.pop(int(rng.integers(len(lists))))
            last.last_pages_release(pool, pages)
            counts[pages] -= 1
        assert (pool.holders == counts).all() and pool.num_free == (counts == 0).sum()
        assert sorted(pool.free_pages[:pool.num_free]) == np.flatnonzero(counts == 0).tolist()


def test_pool_changes_nothing_when_it_refuses(lib):
    pool = last.PagePool(4)
    a = last.last_pages_take(pool, 3)
    last.last_pages_share(pool, a[:1])
    before = pool.holders.copy(), pool.free_pages.copy(), pool.num_free
    free = int(np.flatnonzero(pool.holders == 0)[0])
    for call, pages in ((last.last_pages_share, [a[0], free]), (last.last_pages_share, [a[0], 4]),
                        (last.last_pages_release, [a[0], a[1], a[1]]),       # once too often
                        (last.last_pages_release, [a[0], free]), (last.last_pages_release, [-1])):
        with pytest.raises(last.LastError) as e:
            call(pool, pages)
        assert e.value.status == last.LAST_ERR_INVALID_ARG
        assert (pool.holders == before[0]).all() and (pool.free_pages == before[1]).all() and pool.num_free == before[2]
    last.last_pages_release(pool, [a[0], a[1], a[0]])      # both holders of one page at once
    assert pool.num_free == 3 and pool.holders[a[0]] == 0
    assert len(set(pool.free_pages[:3].tolist())) == 3


def test_pool_refuses_bad_structs(lib):
    bad = last.LAST_ERR_INVALID_ARG
    assert lib.last_pages_init(None) == bad
    p = last._PagePool(3, 0, None, None)
    assert lib.last_pages_init(ctypes.byref(p)) == bad
    pool = last.PagePool(3)
    assert lib.last_pages_take(ctypes.byref(pool.c), -1, None) == bad
    assert lib.last_pages_take(ctypes.byref(pool.c), 1, None) == bad
    empty = last.PagePool(0)
    assert empty.num_free == 0 and len(last.last_pages_take(empty, 0)) == 0


def test_rope_handle_of_sections():
    r = last.Rope.sections([2, 3, 3], base=10000.0, pairs="adjacent")
    assert r.num_axes == 3 and r.axis.tolist() == [0, 0, 1, 1, 1, 2, 2, 2]
    assert np.allclose(r.inv_freq, 10000.0 ** (-np.arange(8) / 8), rtol=1e-6)
    with pytest.raises(ValueError):
        last.Rope([1.0, 0.5], axis=[0])
    with pytest.raises(KeyError):
        last.Rope([1.0], pairs="other")


@pytest.mark.parametrize("kw", [dict(page_size=1 << 21), dict(num_layers=4097), dict(num_kv_heads=4097, head_dim=8, token_stride=8),
                                dict(page_size=1 << 20, num_kv_heads=64)])
def test_limits_of_a_cache(lib, kw):
    n = ctypes.c_size_t(0)
    assert lib.last_cache_workspace_size(ctypes.byref(_cache(**kw)), 3, 8194, ctypes.byref(n)) == last.LAST_ERR_UNSUPPORTED


def test_limits_of_tokens_and_tiles(lib):
    assert _rope(lib, tokens=(1 << 30) + 1, stride=1 << 31) == last.LAST_ERR_UNSUPPORTED
    assert _append(lib, tokens=(1 << 30) + 1, cu=256) == last.LAST_ERR_UNSUPPORTED
    s = _seqs(batch=1 << 20, max_pages=1 << 12, table_stride=1 << 12)
    assert lib.last_cache_attention(ctypes.byref(_cache()), 0, ctypes.byref(s), 4, 0.0, 256, 256, 256, 256, None, 256, 1 << 40,
                                    0) == last.LAST_ERR_UNSUPPORTED


def test_compact_refuses_lengths_over_what_it_reads(lib):
    """lens_out on any array that other blocks still read, whole or in part.  No call has a workspace, so that one
    whose arrays lie apart is refused too, but with another message."""
    c, big, bad = ctypes.byref(_cache()), 1 << 30, last.LAST_ERR_INVALID_ARG
    table, dst, lens, begin, span, keep, idx = (4096 * i for i in range(1, 8))
    rows, pages, stride, n = 3, 4, 6, 5

    def call(out, stride=stride, rows=rows):
        s = _seqs(batch=rows, max_pages=pages, table_stride=stride, page_table=table, lens=lens)
        st = lib.last_cache_compact(c, ctypes.byref(s), dst, pages, stride, begin, span, keep, idx, n, out, None, big, 0)
        assert st == bad
        return "lens_out may not overlap" in lib.last_error_message().decode()

    row, out_bytes = 4 * stride, 4 * rows
    sizes = {lens: 4 * rows, begin: 4 * rows, span: 4 * rows, keep: 4 * (rows + 1), idx: 4 * n}
    for at, size in sizes.items():
        for out in range(at - out_bytes - 8, at + size + 12, 4):
            assert call(out) == (at - out_bytes < out < at + size), (at, out)
    for at in (table, dst):
        for out in range(at - out_bytes - 8, at + rows * row + 12, 4):
            held = {at + i * row + 4 * j for i in range(rows) for j in range(pages)}
            assert call(out) == any(out + 4 * i in held for i in range(rows)), (at, out)
        # two sequences' lengths fit between the rows of a table
        assert not call(at + 4 * pages, stride=6, rows=2) and call(at + 4 * pages, stride=5, rows=2)
    assert not call(1 << 20)


def _overlap(tokens, token, heads, head, dim):
    at = [t * token + h * head for t in range(tokens) for h in range(heads)]
    at.sort()
    return any(b - a < dim for a, b in zip(at, at[1:]))


@pytest.mark.parametrize("back", [False, True])
def test_rotation_refuses_outputs_that_overlap(lib, back):
    """Against every element's place, tokens and heads any way round.  No call has positions or, for append, a workspace, so
    that one whose heads lie apart is refused too, but with another message."""
    rng = np.random.default_rng(4)
    shapes = [(3, 0, 2, 64, 64), (3, 128, 2, 0, 64), (3, 127, 2, 64, 64), (3, 128, 2, 63, 64), (1, 0, 2, 64, 64), (3, 64, 1, 0, 64),
              (2, 3 * 64, 2, 2 * 64, 64), (3, 3 * 64, 2, 2 * 64, 64), (4, 64, 2, 256, 64), (4, 64, 2, 192, 64), (3, -128, 2, 64, 64),
              (3, 128, 2, -64, 64), (1 << 20, 0, 8192, 0, 8), (1 << 20, 8192 * 8, 8192, 8, 8), (1 << 20, 8192 * 8 - 1, 8192, 8, 8)]
    for _ in range(3000):
        d = 8 * int(rng.integers(1, 4))
        shapes.append((int(rng.integers(1, 7)), int(rng.integers(0, 12)) * d + int(rng.integers(-2, 3)), int(rng.integers(1, 7)),
                       int(rng.integers(0, 12)) * d + int(rng.integers(-2, 3)), d))
    r, good = _rotary(rot_dim=8), _heads()
    seen = set()
    for tokens, token, heads, head, d in shapes:
        if tokens < 100:
            want = _overlap(tokens, token, heads, head, d)
        else:
            want = token != 8192 * 8
        seen.add(want)
        h = _heads(heads=heads, in_token=0, in_head=0, out_token=token, out_head=head)     # the input may be one head
        fine = _heads(in_=16, out=16, heads=heads, out_token=heads * d, out_head=d)
        messages = []
        for q, k in ((h, None), (fine, h)):
            st, msg = _status(_rope(lib, r=r, h=q, k=k, tokens=tokens, dim=d, pos=None, back=back))
            assert st == last.LAST_ERR_INVALID_ARG
            messages.append("overlap" in msg)
        assert messages == [want, want], (tokens, token, heads, head, d)
    assert seen == {False, True}
    x = _heads(out_token=0)
    assert _append(lib, r=r, pos=16, q=x, ws=None) == last.LAST_ERR_INVALID_ARG
    assert "overlap" in lib.last_error_message().decode()
    assert _append(lib, r=r, pos=16, q=good, k=_heads(out_token=0), ws=None) == last.LAST_ERR_INVALID_ARG     # k's out is not used
    assert "overlap" not in lib.last_error_message().decode()


@pytest.mark.parametrize("kw,reads,writes", [
    (dict(), True, True),
    (dict(head_stride=64, token_stride=128), True, True),                          # tokens outside heads
    (dict(page_stride=64, head_stride=640, token_stride=1280), True, True),        # pages innermost
    (dict(head_stride=64), True, False),                                           # heads on the tokens
    (dict(token_stride=1024), True, False),                                        # tokens on the heads
    (dict(page_stride=1024), True, False),                                         # pages on the heads
    (dict(page_stride=64, num_kv_heads=1), True, False),                           # pages on the tokens
    (dict(head_stride=960, num_pages=1), True, False),                             # heads by one token
    (dict(num_pages=1, page_stride=0), True, True),
    (dict(layer_stride=0), True, True),                                            # all layers are one
    (dict(layer_stride=2048), True, None),                                         # layers on pages: append writes one alone
])
def test_caches_that_overlap_themselves_are_not_written(lib, kw, reads, writes):
    """They may be read.  No call has a workspace: each is refused, the sound ones for that."""
    c, s, h = ctypes.byref(_cache(**kw)), ctypes.byref(_seqs()), ctypes.byref(_heads())

    def overlap(st):
        assert st == last.LAST_ERR_INVALID_ARG
        message = lib.last_error_message().decode()
        assert "overlap itself" in message or "workspace is NULL" in message
        return "overlap itself" in message

    big = 1 << 30
    assert overlap(lib.last_cache_attention(c, 0, s, 4, 0.0, 256, 256, 256, 256, None, None, big, 0)) is not reads
    assert overlap(lib.last_cache_append(c, 0, s, 3, None, None, None, 0, None, h, h, None, big, 0)) is (writes is False)
    assert overlap(lib.last_cache_copy(c, 1, 256, 256, None, big, 0)) is not bool(writes)
    assert overlap(lib.last_cache_compact(c, s, 4096, 4, 4, None, None, 8192, 12288, 5, 16384, None, big, 0)) is not bool(writes)


# ---- the marshalling module ----

def _build_marshal(monkeypatch, tmp_path):
    """build_marshal() into tmp_path: the files there, and the commands it ran."""
    import os
    import subprocess
    import sysconfig
    from paper_2607_27952_gb300 import build
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        pytest.skip("Python's headers are not installed")
    commands = []

    def compile_it(cmd):
        commands.append(cmd)
        subprocess.run(cmd, check=True, capture_output=True)
    monkeypatch.setattr(build, "MARSHAL", str(tmp_path / os.path.basename(build.MARSHAL)))
    build.build_marshal(compile_it)
    return sorted(f.name for f in tmp_path.iterdir()), commands


def test_marshalling_module_is_one_pythons(lib, monkeypatch, tmp_path):
    """Its name carries the interpreter's tag, so that no other imports it, and one without a tag is removed."""
    import sysconfig
    (tmp_path / "_marshal.so").write_bytes(b"")
    suffix = sysconfig.get_config_var("EXT_SUFFIX")
    assert suffix != ".so"
    files, commands = _build_marshal(monkeypatch, tmp_path)
    assert files == ["_marshal" + suffix] and len(commands) == 1
    assert last._fast is None or last._fast.__file__.endswith(suffix)


@pytest.mark.parametrize("error", [ImportError, AttributeError, TypeError])
def test_a_marshalling_module_that_does_not_fit_is_left_alone(lib, monkeypatch, error):
    """One of other sources may want other arguments: the calls then go through ctypes."""
    class Other:
        @staticmethod
        def bind(*args):
            raise error("bind")
    monkeypatch.setattr(last, "_marshal", Other, raising=False)
    assert last._load_fast(lib) is None


@pytest.mark.parametrize("cc", ["gcc -pipe", "", " "])
def test_marshalling_module_with_a_compiler_of_several_words(lib, monkeypatch, tmp_path, cc):
    """CC as make takes it; an empty one is none."""
    monkeypatch.setenv("CC", cc)
    files, commands = _build_marshal(monkeypatch, tmp_path)
    assert len(files) == 1 and commands[0][0] == "gcc"


def test_outputs_of_no_tokens_cannot_overlap(lib):
    for h in (_heads(out_token=0, out_head=0), _heads(out_head=0)):
        assert _rope(lib, tokens=0, pos=None, h=h, k=h) == last.LAST_OK

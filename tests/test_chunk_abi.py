"""CPU-side checks of the attention of chunks and of differential attention: arguments are refused on the
host before any launch (no compute call runs here)."""
import ctypes

import pytest

import paper_2607_27952_gb300 as last
from test_cache_abi import _cache, _seqs, _status

INVALID, UNSUPPORTED, SMALL = last.LAST_ERR_INVALID_ARG, last.LAST_ERR_UNSUPPORTED, last.LAST_ERR_WORKSPACE_TOO_SMALL


@pytest.fixture(scope="module")
def lib():
    from paper_2607_27952_gb300.build import build
    build()
    return last.load_library()


def _difference(**kw):
    f = dict(lambda_=1024, norm_weight=2048, norm_eps=1e-5, out_scale=1.0)
    f.update(kw)
    return last._Difference(*f.values())


def _need(lib, c, heads=8):
    n = ctypes.c_size_t(0)
    assert lib.last_chunk_workspace_size(ctypes.byref(c), heads, ctypes.byref(n)) == last.LAST_OK
    return n.value


def _call(lib, diff, c=None, s=None, d=None, layer=0, tokens=5, cu=768, heads=8, causal=1, window=0, q=4096, qs=512, out=8192, os=512, lse=None,
          ws=256, ws_bytes=1 << 40):
    c, s = c or _cache(), s or _seqs()
    head = (ctypes.byref(c), layer, ctypes.byref(s), tokens, cu, heads, 0.0, causal, window)
    if diff:
        return lib.last_cache_diff_attention(*head, ctypes.byref(d or _difference()), q, qs, out, os, ws, ws_bytes, 0)
    return lib.last_cache_chunk_attention(*head, q, qs, out, os, lse, ws, ws_bytes, 0)


@pytest.mark.parametrize("diff", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(c=_cache(dtype=2)), INVALID),
    (dict(c=_cache(page_size=12)), INVALID),
    (dict(c=_cache(head_dim=260, token_stride=264, head_stride=8192, page_stride=32768, layer_stride=1 << 20)), UNSUPPORTED),
    (dict(c=_cache(k=None)), INVALID),
    (dict(c=_cache(token_stride=60)), INVALID),
    (dict(layer=2), INVALID),
    (dict(layer=-1), INVALID),
    (dict(s=_seqs(batch=-1)), INVALID),
    (dict(s=_seqs(lens=None)), INVALID),
    (dict(s=_seqs(table_stride=3)), INVALID),
    (dict(s=_seqs(batch=0)), INVALID),                      # tokens without a sequence
    (dict(tokens=-1), INVALID),
    (dict(tokens=(1 << 30) + 1), UNSUPPORTED),
    (dict(cu=None), INVALID),                               # 5 tokens, 3 sequences
    (dict(heads=0), INVALID),
    (dict(heads=7), INVALID),
    (dict(heads=8194), UNSUPPORTED),
    (dict(heads=4096, tokens=1 << 20), UNSUPPORTED),        # rows past 31 bits
    (dict(heads=512, tokens=1 << 22, s=_seqs(max_pages=1 << 27, table_stride=1 << 27)), UNSUPPORTED),
    (dict(causal=2), INVALID),
    (dict(causal=-1), INVALID),
    (dict(window=-1), INVALID),
    (dict(window=4, causal=0), INVALID),
    (dict(q=None), INVALID),
    (dict(out=None), INVALID),
    (dict(q=4104), INVALID),
    (dict(out=8200), INVALID),
    (dict(qs=516), INVALID),
    (dict(os=516), INVALID),
    (dict(os=504), INVALID),                                # tokens overlap
    (dict(ws=None), INVALID),
    (dict(ws=128), INVALID),
    (dict(ws_bytes=1000), SMALL),
])
def test_refusals(lib, kw, status, diff):
    st, msg = _status(_call(lib, diff, **kw))
    assert st == status and msg


@pytest.mark.parametrize("kw,status", [
    (dict(c=_cache(num_kv_heads=1)), INVALID),
    (dict(c=_cache(head_dim=136, token_stride=136, head_stride=2176, page_stride=4352, layer_stride=43520)), UNSUPPORTED),
    (dict(d=_difference(lambda_=None)), INVALID),
    (dict(d=_difference(lambda_=1026)), INVALID),
    (dict(d=_difference(norm_weight=2050)), INVALID),
    (dict(d=_difference(norm_eps=-1e-9)), INVALID),
    (dict(d=_difference(norm_eps=float("inf"))), INVALID),
    (dict(d=_difference(norm_eps=float("nan"))), INVALID),
    (dict(d=_difference(out_scale=float("nan"))), INVALID),
    (dict(d=_difference(out_scale=-float("inf"))), INVALID),
])
def test_refusals_of_differences(lib, kw, status):
    st, msg = _status(_call(lib, True, **kw))
    assert st == status and msg


def test_lse_must_be_aligned(lib):
    assert _call(lib, False, lse=4098) == INVALID


def test_null_structs(lib):
    c, s, n = _cache(), _seqs(), ctypes.c_size_t(0)
    C, S = ctypes.byref(c), ctypes.byref(s)
    assert lib.last_chunk_workspace_size(None, 8, ctypes.byref(n)) == INVALID
    assert lib.last_chunk_workspace_size(C, 8, None) == INVALID
    assert lib.last_chunk_workspace_size(C, 7, ctypes.byref(n)) == INVALID
    assert lib.last_cache_chunk_attention(None, 0, S, 5, 768, 8, 0.0, 1, 0, 4096, 512, 8192, 512, None, 256, 1 << 40, 0) == INVALID
    assert lib.last_cache_chunk_attention(C, 0, None, 5, 768, 8, 0.0, 1, 0, 4096, 512, 8192, 512, None, 256, 1 << 40, 0) == INVALID
    assert lib.last_cache_diff_attention(C, 0, S, 5, 768, 8, 0.0, 1, 0, None, 4096, 512, 8192, 512, 256, 1 << 40, 0) == INVALID


def test_workspace_is_enough_and_no_more_is_asked(lib):
    for dtype in (0, 1):
        for dim in (8, 64, 128, 256):
            c = _cache(dtype=dtype, head_dim=dim, token_stride=dim, head_stride=16 * dim, page_stride=32 * dim, layer_stride=320 * dim)
            need = _need(lib, c)
            assert need % 256 == 0
            st, msg = _status(_call(lib, False, c=c, qs=8 * dim, os=8 * dim, ws_bytes=need - 1))
            assert st == SMALL and str(need) in msg

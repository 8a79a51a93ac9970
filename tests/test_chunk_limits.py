"""CPU-side checks of how much one call of the attention of chunks may ask for: what its shares' 64-bit sums could not count is refused
before any launch."""
import pytest

import paper_2607_27952_gb300 as last
from test_cache_abi import _cache, _seqs, _status
from test_chunk_abi import _call, lib  # noqa: F401  (the fixture)


def _asked(q_heads, kv_heads, tokens, batch, pages, page_size=16):
    """What the device would sum at most: blocks of eight rows, heads of a unit times keys and what an item costs, every unit."""
    group, keys = q_heads // kv_heads, min(pages * page_size, 2**31)
    return (tokens * group // 8 + batch) * q_heads * (keys + 1024)


@pytest.mark.parametrize("diff", [False, True])
@pytest.mark.parametrize("q_heads,kv_heads,tokens,batch,pages,page_size", [
    (8192, 2, 65536, 1, 1 << 26, 16),       # many heads to a kv-head: 2^64 and more, though tokens times heads times keys is below 2^60
    (8192, 2, 1 << 18, 1, 1 << 24, 16),
    (4096, 2, 1 << 18, 3, 1 << 27, 16),
    (8192, 2, 1 << 15, 1 << 20, 1 << 26, 16),
])
def test_sums_that_could_wrap_are_refused(lib, q_heads, kv_heads, tokens, batch, pages, page_size, diff):  # noqa: F811
    assert _asked(q_heads, kv_heads, tokens, batch, pages, page_size) >= 2**62
    assert tokens * (q_heads // kv_heads) < 2**31
    c = _cache(num_kv_heads=kv_heads, page_size=page_size)
    s = _seqs(batch=batch, max_pages=pages, table_stride=pages)
    stride = q_heads * 64
    st, msg = _status(_call(lib, diff, c=c, s=s, heads=q_heads, tokens=tokens, qs=stride, os=stride))
    assert st == last.LAST_ERR_UNSUPPORTED and "2^62" in msg


def test_long_sequences_are_not_refused(lib):  # noqa: F811
    """The longest sequences under ordinary head counts get as far as the workspace's check."""
    for q_heads, tokens, batch, pages in ((64, 1 << 20, 1, 1 << 27), (128, 1 << 16, 512, 1 << 20), (8, 512, 512, 1 << 27)):
        s = _seqs(batch=batch, max_pages=pages, table_stride=pages)
        st, _ = _status(_call(lib, False, s=s, heads=q_heads, tokens=tokens, qs=q_heads * 64, os=q_heads * 64, ws_bytes=1000))
        assert st == last.LAST_ERR_WORKSPACE_TOO_SMALL

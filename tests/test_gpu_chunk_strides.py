"""Tokens of q that overlap or coincide, rows that two sequences claim."""
import pytest

import paper_2607_27952_gb300 as last
from test_gpu_chunk_attention import DTYPES, _chunk, _diff, _params

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,old", [([40, 90], [300, 5]), ([1, 3], [70, 200])])
@pytest.mark.parametrize("step", [0, 16, 72])
def test_queries_that_overlap(step, new, old, dtype):
    """A token's queries begin `step` elements behind the token's before: 0 is one token for all."""
    import torch
    import cache_util as cu
    import chunk_util as ch
    hq, hkv, d, tokens = 4, 2, 64, sum(new)
    lens = [a + b for a, b in zip(new, old)]
    cache, seqs, _, cu_new = ch.setup(new, old, hq, hkv, d, dtype, 16, seed=3)
    q = cu.randn((tokens * step + hq * d,), dtype, 9).as_strided((tokens, hq, d), (step, d, 1))
    lam, weight = _params(hq // 2, d, 3)
    for x in (q, q.contiguous()):
        out = torch.full((tokens, hq, d), float("nan"), dtype=q.dtype, device="cuda")
        ws = ch.workspace(cache, hq)
        last.last_cache_chunk_attention(cache, 0, seqs, x, out, ws, cu_new=cu_new)
        last.last_poll(ws)
        ch.check_chunk(cache, seqs, x, cu_new, out, None, new, lens)
        diff, _ = _diff(cache, seqs, x, cu_new, lam, weight)
        ch.check_diff(cache, seqs, x, cu_new, diff, lam, new, lens, weight=weight)


@pytest.mark.parametrize("dtype", DTYPES)
def test_offsets_that_fall_leave_the_others_right(dtype):
    """Offsets 0, 50, 30, 80, 85: the second sequence is skipped, rows 30 .. 49 are two sequences', all others are their own's."""
    import cache_util as cu
    import chunk_util as ch
    new, lens = [50, 0, 50, 5], [300, 40, 120, 400]
    cache, seqs, q, _ = ch.setup([50, 0, 30, 5], [250, 40, 90, 395], 4, 2, 64, dtype, 16, seed=5)
    cu_new = cu.ints([0, 50, 30, 80, 85])
    out, lse, ws = _chunk(cache, seqs, q, cu_new, poll=False)
    with pytest.raises(last.LastError) as e:
        last.last_poll(ws)
    assert e.value.status == last.LAST_ERR_DEVICE_INDEX
    ch.check_chunk(cache, seqs, q, cu_new, out, lse, new, lens, only=[3])
    # the first sequence's first 30 rows alone, the third's last 30: as calls of their own, whose new tokens are fewer
    for b, rows, n, total in ((0, slice(0, 30), 30, 280), (2, slice(50, 80), 30, 120)):
        one = last.Sequences(seqs.page_table[b:b + 1].contiguous(), cu.ints([total]))
        ch.check_chunk(cache, one, q[rows], cu.ints([0, n]), out[rows], lse[rows], [n], [total])

"""Values that are not finite, under rows that see them and rows that do not: the rows that do not are as without them, other sequences
too, and the call takes no longer than its masks' edges ask for."""
import pytest

import paper_2607_27952_gb300 as last
from test_gpu_chunk_attention import DTYPES, MASKS, _chunk, _diff, _params

pytestmark = pytest.mark.gpu


def _with(cache, seqs, at, x, column=3):
    """The cache with x in one column of V at keys at[b] of sequence b, all heads."""
    import torch
    v = cache.v.clone()
    for b, keys in at.items():
        keys = torch.as_tensor(keys, device="cuda")
        v[0, seqs.page_table[b].long()[keys // cache.page_size], :, keys % cache.page_size, column] = x
    return last.Cache(cache.k, v)


def _sees(new, lens, begin, causal, window, at):
    """[tokens]: rows that see one of their sequence's keys at[b]."""
    import torch
    import chunk_util as ch
    rows = [ch.seen(n, m, 0 if begin is None else begin[b], causal, window)[:, at.get(b, [])].any(1) for b, (n, m) in enumerate(zip(new, lens))]
    return torch.cat(rows)


NEW, OLD = [300, 90, 150, 40], [20, 100, 0, 333]
LENS = [a + b for a, b in zip(NEW, OLD)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("begin", [None, [0, 117, 3, 350]])
@pytest.mark.parametrize("causal,window", MASKS)
@pytest.mark.parametrize("hq,hkv,d,size", [(8, 2, 128, 16), (6, 2, 64, 8), (2, 2, 80, 24), (12, 2, 72, 16), (6, 2, 192, 40), (4, 2, 256, 64),
                                           (130, 1, 64, 32)])
def test_each_row_shows_what_it_sees_and_nothing_else(hq, hkv, d, size, causal, window, begin, dtype):
    import torch
    import chunk_util as ch
    cache, seqs, q, cu_new = ch.setup(NEW, OLD, hq, hkv, d, dtype, size, begin=begin, seed=6, stale=float("nan"))
    clean, lse, _ = _chunk(cache, seqs, q, cu_new, causal, window)
    lam, _ = _params(hq // 2, d, 2, False)
    pairs = d <= 128 and hkv % 2 == 0
    if pairs:
        clean_diff, _ = _diff(cache, seqs, q, cu_new, lam, causal=causal, window=window)
    for at in ({0: [5, 150, 155, 290], 1: [118, 140], 3: [371]}, {2: list(range(0, 150, 7)), 3: [340]}):
        rows = _sees(NEW, LENS, begin, causal, window, at)
        for x in (float("nan"), float("inf")):
            bad = _with(cache, seqs, at, x)
            out, got, _ = _chunk(bad, seqs, q, cu_new, causal, window)
            assert torch.equal(got, lse)
            assert not torch.isfinite(out[rows][..., 3]).any()
            out[..., 3] = torch.where(rows[:, None], clean[..., 3], out[..., 3])
            ch.check_chunk(cache, seqs, q, cu_new, out, got, NEW, LENS, begin, causal, window)
            if not pairs:
                continue
            diff, _ = _diff(bad, seqs, q, cu_new, lam, causal=causal, window=window)
            for c in (3, d + 3):
                assert not torch.isfinite(diff[rows][..., c]).any()
                diff[..., c] = torch.where(rows[:, None], clean_diff[..., c], diff[..., c])
            ch.check_diff(cache, seqs, q, cu_new, diff, lam, NEW, LENS, begin, causal, window)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("keys", [[0], [0, 1, 20003, 39990], list(range(40000))])
def test_one_sequence_does_not_hold_up_the_others(d, keys):
    """A prompt of 40000 tokens with values that are not finite, next to clean ones: no wait runs out, and the others' bits stay."""
    import torch
    import chunk_util as ch
    new, old, hq, hkv = [40000, 700, 33, 1500], [0, 50, 4000, 0], 4, 1 if d > 128 else 2
    lens = [a + b for a, b in zip(new, old)]
    cache, seqs, q, cu_new = ch.setup(new, old, hq, hkv, d, "bfloat16", 32, seed=8)
    want, lse, _ = _chunk(cache, seqs, q, cu_new)
    lam, weight = _params(hq // 2, d, 2)
    clean = _diff(cache, seqs, q, cu_new, lam, weight)[0] if d <= 128 else None
    bad = _with(cache, seqs, {0: keys}, float("inf"))
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    out, got, _ = _chunk(bad, seqs, q, cu_new)                # raises where a wait has run out
    diff = _diff(bad, seqs, q, cu_new, lam, weight)[0] if d <= 128 else None
    end.record()
    torch.cuda.synchronize()
    assert begin.elapsed_time(end) < 500                      # some 10 ms without them
    rows = _sees(new, lens, None, True, 0, {0: keys})
    assert torch.equal(got, lse) and torch.equal(out[40000:], want[40000:])
    assert not torch.isfinite(out[rows][..., 3]).any()
    out[..., 3] = torch.where(rows[:, None], want[..., 3], out[..., 3])
    # weights of bf16 in one order of adding up and in another
    assert ((out.double() - want.double()).norm() / want.double().norm()) < 2.0 ** -8
    again = _chunk(bad, seqs, q, cu_new)[0]
    again[..., 3] = torch.where(rows[:, None], want[..., 3], again[..., 3])
    assert torch.equal(again, out)
    if diff is not None:
        assert torch.equal(diff[40000:], clean[40000:]) and not torch.isfinite(diff[rows][..., 3]).any()

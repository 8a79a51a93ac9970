"""Few rows per sequence, bf16: weights are held in two parts, so that an output is off by its own rounding and hardly more."""
import math

import pytest

import paper_2607_27952_gb300 as last  # noqa: F401
from test_gpu_chunk_attention import _chunk

pytestmark = pytest.mark.gpu


def _cut(p):
    """Weights cut to bf16, with nothing kept of the rest."""
    import torch
    return (p.float().view(torch.int32) & -65536).view(torch.float32).double()


@pytest.mark.parametrize("begin", [None, [3, 0, 40, 10]])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 70)])
@pytest.mark.parametrize("hq,hkv,d,size", [(2, 2, 64, 16), (8, 2, 64, 16), (4, 2, 128, 8), (8, 2, 128, 32), (2, 2, 80, 24), (2, 1, 192, 40),
                                           (2, 2, 256, 16), (4, 2, 16, 16)])
def test_weights_are_held_in_two_parts(hq, hkv, d, size, causal, window, begin):
    """Off by 2^-16 of sum p |v| for the weights' second part's rounding, the errors of exponentials and sums, and 2^-8 of the output.  One part
    would be off by more: the same bound does not hold for weights that are cut to bf16."""
    import torch
    import chunk_util as ch
    new, old = [1, 3, 2, 4], [70, 500, 130, 64]
    lens = [a + b for a, b in zip(new, old)]
    assert sum(new) / 4 * (hq // hkv) <= (16 if d in (64, 128) else 8)   # few rows on average
    cache, seqs, q, cu_new = ch.setup(new, old, hq, hkv, d, "bfloat16", size, begin=begin, seed=12)
    out, _, _ = _chunk(cache, seqs, q, cu_new, causal, window)
    found = False
    for b, (n, total) in enumerate(zip(new, lens)):
        t0 = int(cu_new[b])
        see = ch.seen(n, total, 0 if begin is None else begin[b], causal, window)
        for h in range(hq):
            k, v = ch.keys_of(cache, seqs.page_table[b].clamp(min=0), total, h // (hq // hkv))
            want, lse, mass, ez = ch.one_map(q[t0:t0 + n, h], k, v, see, 1 / math.sqrt(d))
            tol = ch.relative(ez, total, "bfloat16", 2) * mass + ch.UNIT["bfloat16"] * want.abs()
            err = (out[t0:t0 + n, h].double() - want).abs()
            assert (err <= tol).all(), f"sequence {b}, head {h}: {(err - tol).max():.3e} past the bound"
            z = torch.where(see, q[t0:t0 + n, h].double() @ k.double().T / math.sqrt(d), -math.inf)
            p = torch.where(see, torch.exp(z - lse[:, None]), 0.0)
            found |= bool(((_cut(p) @ v.double() - want).abs() > tol).any())
    assert found

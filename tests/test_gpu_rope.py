"""Rotary positions with several axes against their definition in extended precision."""
import numpy as np
import pytest

import paper_2607_27952_gb300 as last

pytestmark = pytest.mark.gpu

# One rounding of the result (u: 2^-8 bf16, 2^-24 fp32) on top of fp32 arithmetic: the sine
# and cosine carry 2 units in the last place and one for the conversion of the angle
# (pi 2^-24 of a radian), each product and the sum one more: below 2^-20 (|a| + |b|).
UNIT = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8}


def _definition(x, pos, rope, back=False):
    """x [t][h][d] float64, pos [axes][t] -> float64, and |a| + |b| of each element."""
    n, y, size = len(rope.inv_freq), x.astype(np.float64).copy(), np.abs(x.astype(np.float64))
    two_pi = 2 * np.longdouble("3.14159265358979323846264338327950288")
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if rope.c.pairs == last.LAST_ROPE_ADJACENT else (i, i + n)
        phi = np.remainder(pos[rope.axis[i]].astype(np.longdouble) * np.longdouble(rope.inv_freq[i]), two_pi)
        c, s = np.cos(phi).astype(np.float64)[:, None], np.sin(phi).astype(np.float64)[:, None]
        s = -s if back else s
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
        size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, size


def _check(got, x, pos, rope, back=False, dtype="bfloat16"):
    want, size = _definition(x.double().cpu().numpy(), pos.cpu().numpy(), rope, back)
    err = np.abs(got.double().cpu().numpy() - want)
    bad = err > UNIT[dtype] * np.abs(want) + 2.0 ** -20 * size
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, worst {err.max():.3e}"


def _randn(shape, dtype, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(getattr(torch, dtype))


def _pos(axes, tokens, seed, top=20000):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, top, (axes, tokens), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("t,hq,hk,d,sections,pairs", [
    (1, 1, 1, 2, [1], "half"),
    (1, 16, 2, 128, [16, 24, 24], "half"),
    (37, 12, 2, 80, [12, 14, 14], "adjacent"),
    (5, 3, 1, 72, [36], "half"),               # 36 pairs: half vectors
    (301, 4, 4, 64, [5, 6, 6], "half"),        # 17 pairs, the other 30 elements copied
    (64, 4, 4, 64, [5, 6, 6], "adjacent"),
    (9, 2, 1, 7, [1, 2], "half"),              # odd head width
    (1000, 7, 1, 256, [32, 32, 32, 32], "half"),
    (3, 130, 10, 256, [128], "adjacent"),
])
def test_rotation(t, hq, hk, d, sections, pairs, dtype, back):
    import torch
    rope = last.Rope.sections(sections, pairs=pairs)
    q, k, pos = _randn((t, hq, d), dtype, 1), _randn((t, hk, d), dtype, 2), _pos(len(sections), t, 3)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    call = last.last_rope_backward if back else last.last_rope
    call(rope, pos, q, qo, k=k, k_out=ko)
    _check(qo, q, pos, rope, back, dtype)
    _check(ko, k, pos, rope, back, dtype)
    call(rope, pos, q, q)                      # in place, q alone
    assert torch.equal(q, qo)


def test_positions_of_any_size():
    """Angles stay exact at the ends of 32-bit positions."""
    import torch
    rope = last.Rope(np.array([65536.0, 7.3, 1.0, 0.1, 1e-3, 1e-6, 1e-30, 0.0], np.float32), axis=[0, 1] * 4)
    ends = [0, 1, -1, 2**24 + 1, -2**24 - 3, 2**31 - 1, -2**31, 123456789]
    pos = torch.tensor([ends, ends[::-1]], dtype=torch.int32, device="cuda")
    q = _randn((len(ends), 3, 16), "float32", 5)
    out = torch.empty_like(q)
    last.last_rope(rope, pos, q, out)
    _check(out, q, pos, rope, dtype="float32")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_views(dtype):
    """A fused projection's heads, heads outside tokens, odd offsets, inputs shared by all tokens."""
    import torch
    rope, pos = last.Rope.sections([4, 6, 6]), _pos(3, 23, 1)
    fused = _randn((23, 5 * 32 + 3), dtype, 2)
    q, k = fused[:, 1:97].unflatten(1, (3, 32)), fused[:, 98:162].unflatten(1, (2, 32))
    qo = torch.empty((3, 23, 32), dtype=q.dtype, device="cuda").transpose(0, 1)
    ko = torch.empty((23, 2, 40), dtype=q.dtype, device="cuda")[..., 3:35]
    last.last_rope(rope, pos, q, qo, k=k, k_out=ko)
    _check(qo, q, pos, rope, dtype=dtype)
    _check(ko, k, pos, rope, dtype=dtype)
    one = _randn((1, 4, 32), dtype, 3).expand(23, 4, 32)
    out = torch.empty((23, 4, 32), dtype=q.dtype, device="cuda")
    last.last_rope(rope, pos, one, out)
    _check(out, one, pos, rope, dtype=dtype)


def test_backward_is_the_transposed_forward():
    """The rotation is linear: its Jacobian, taken column by column with differences (of exact step 1),
    transposed and applied to g, is the backward pass."""
    import torch
    d, t = 24, 6
    rope, pos = last.Rope.sections([3, 3, 4], pairs="adjacent"), _pos(3, t, 4)
    x, g = _randn((t, 1, d), "float32", 1), _randn((t, 1, d), "float32", 2)
    base, got = torch.empty_like(x), torch.empty_like(x)
    last.last_rope(rope, pos, x, base)
    want = torch.zeros((t, 1, d), dtype=torch.float64, device="cuda")
    for i in range(d):
        step, y = x.clone(), torch.empty_like(x)
        step[..., i] += 1.0
        last.last_rope(rope, pos, step, y)
        want[..., i] = ((y.double() - base.double()) * g.double()).sum(-1)
    last.last_rope_backward(rope, pos, g, got)
    # two evaluations, each within 2^-20 (|a| + |b|) <= 2^-20 * 8, and two components a sum
    assert (got.double() - want).abs().max() < 32 * 2.0 ** -20 * g.abs().max()


def test_stream_and_refused_tensors():
    import torch
    rope, pos, q = last.Rope.sections([8]), _pos(1, 50, 1), _randn((50, 2, 16), "bfloat16", 1)
    want, got = torch.empty_like(q), torch.zeros_like(q)
    last.last_rope(rope, pos, q, want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    last.last_rope(rope, pos[0], q, got, stream=s)      # one axis: positions [tokens]
    s.synchronize()
    assert torch.equal(got, want)
    for args in ((pos, q.cpu(), q), (pos, q, q[:, :1]), (pos.long(), q, q), (pos[:, :49], q, q),
                 (pos, q.half(), q.half()), (pos, q[..., ::2], q[..., ::2]), (None, q, q)):
        with pytest.raises(ValueError):
            last.last_rope(rope, *args)
    with pytest.raises(ValueError):
        last.last_rope(rope, pos, q, q, k=q)
    with pytest.raises(ValueError):
        last.last_rope(rope, pos, q, q, k=q[:3], k_out=q[:3])
    with pytest.raises(last.LastError):
        last.last_rope(last.Rope.sections([9]), pos, q, q)   # 18 elements of 16

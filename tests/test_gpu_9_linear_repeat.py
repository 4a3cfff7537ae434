"""GPU test of a checkpoint written in the epilogue of the large tiles: again the same bits, and every code one that a
float32 sum may give.

A code sits next to a border of its format wherever the sum does, and a group's scale where its largest value does, so two
right sums of another order differ in some codes by a whole step.  What is held is that each group is the checkpoint of values
within the bound of a float32 sum, 2 (K + 8) 2^-24 times the sum of the terms' magnitudes (twice the textbook bound, for the
inner steps of the matrix instructions)."""

import pytest

from efs_gpu import announce
from oracle import linear_oracle as L

pytestmark = pytest.mark.gpu


def exponent(amax, fmt):
    """A group's exponent from its largest value, float64: the smallest from -100 on that fits."""
    import torch
    e = torch.floor(torch.log2(amax.clamp(min=2.0 ** -100))) - 10
    for _ in range(5):
        v = amax * torch.exp2(-e)
        e = e + ((v.round() > 127) if fmt == L.INT8 else (v > 448.0)).double()
    return e.clamp(min=-100)


@pytest.mark.parametrize("fmt", [L.INT8, L.E4M3])
def test_wide_forward_with_its_checkpoint_again_and_again(fmt):
    import torch
    import paper_2009_09271_amd as e
    n, i, o = 4096, 2048, 8192
    announce("wide forward", n, i, o, fmt)
    g = torch.Generator(device="cuda")
    g.manual_seed(17)
    x = torch.randn(n, i, generator=g, device="cuda").bfloat16()
    w = (torch.randn(o, i, generator=g, device="cuda") * i ** -0.5).bfloat16()
    b = torch.randn(o, generator=g, device="cuda").bfloat16()
    other = torch.randn(n, i, generator=g, device="cuda").bfloat16()
    ws = e.linear_workspace(e.EF_OP_FORWARD, n, i, o, torch.bfloat16)
    y = torch.empty(n, o, dtype=torch.bfloat16, device="cuda")
    q, s = e.ckpt_buffers(n, o)
    first = None
    e.timing_enable(True)
    for k in range(8):
        if k % 2:  # other values through the same buffers in between
            e.ef_linear_forward(other, w, y, ws, bias=b, act=e.EF_ACT_GELU_TANH, codes=q, scales=s, fmt=fmt)
        y.fill_(float("nan")), q.fill_(99), s.fill_(99)
        e.ef_linear_forward(x, w, y, ws, bias=b, act=e.EF_ACT_GELU_TANH, codes=q, scales=s, fmt=fmt)
        if first is None:
            first = y.clone(), q.clone(), s.clone()
        assert all(torch.equal(a.view(torch.uint8), c.view(torch.uint8)) for a, c in zip(first, (y, q, s))), k
    ran = e.timing_collect()
    e.timing_enable(False)
    assert "k_linear_bf16<256> forward" in ran, ran
    z = torch.matmul(x.double(), w.double().t().contiguous()) + b.double()
    off = torch.matmul(x.double().abs(), w.double().abs().t().contiguous()) + b.double().abs()
    off *= 2 * (i + 8) * 2.0 ** -24
    wide = z.view(n, o // 32, 32).abs()
    lo, hi = (exponent((wide + k * off.view(n, o // 32, 32)).amax(2).clamp(min=0), fmt) for k in (-1, 1))
    at = s.double() - 127
    assert bool(((lo <= at) & (at <= hi)).all())
    assert float((lo != hi).double().mean()) < 0.05  # (few groups stand at a border)
    kept = torch.empty(n, o, device="cuda")
    e.ef_ckpt_unpack(q, s, fmt, kept)
    step = torch.exp2(at).repeat_interleave(32, 1)
    half = step / 2 if fmt == L.INT8 else torch.maximum(z.abs() * 2.0 ** -4, step * 2.0 ** -10)
    assert bool(((kept.double() - z).abs() <= half + 1.1 * off).all())

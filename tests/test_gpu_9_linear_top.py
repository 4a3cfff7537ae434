"""GPU tests of checkpoints at the top of the range: finite activations, up to the largest of their type, come back finite,
from the packing pass and from every kernel that writes a checkpoint, and a padded token adds nothing through them."""

import numpy as np
import pytest

from efs_gpu import announce, host
from oracle import linear_oracle as L

pytestmark = pytest.mark.gpu

FMTS = [L.INT8, L.E4M3]
MOST = {"f32": float(np.finfo(np.float32).max), "bf16": float.fromhex("0x1.FEp127")}


def E():
    import paper_2009_09271_amd
    return paper_2009_09271_amd


def tt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def near_the_top(seed, n, c, dtype):
    """Values of `dtype` from a 2^-9th of its largest up to that, as float64; each row and group with its own largest."""
    import torch
    g = np.random.default_rng(seed)
    x = (1 - g.random((n, c)) * 2.0 ** -g.integers(0, 9, (n, c))) * 2.0 ** -g.integers(0, 3, (n, c)) * 2.0 ** -g.integers(0, 3, (n, 1))
    x[::3, ::7] = 1.0
    x = x * MOST[dtype] * g.choice([-1, 1], (n, c))
    x = torch.from_numpy(x).to(tt(dtype))
    return torch.where(x.isinf(), MOST[dtype] * x.sign(), x).double().numpy()


def same_codes(q, want, fmt):
    zero = 0 if fmt == L.INT8 else 128  # (the two zeros are one value)
    return np.array_equal(np.where(host(q) == zero, 0, host(q)), np.where(want == zero, 0, want))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pack(dtype, fmt):
    import torch
    n, c = 61, 200
    announce("top", dtype, fmt)
    x = near_the_top(1, n, c, dtype)
    q, s = E().ckpt_buffers(n, c)
    E().ef_ckpt_pack(torch.from_numpy(x).to(tt(dtype)).cuda(), q, s, fmt)
    wq, wsc = L.ckpt_pack(x, fmt)
    assert (wsc == (249 if fmt == L.INT8 else 247)).any() and (wsc < (249 if fmt == L.INT8 else 247)).any()
    assert np.array_equal(host(s), wsc) and same_codes(q, wq, fmt)
    for out in (torch.float32, torch.bfloat16):
        y = torch.empty(n, c, dtype=out, device="cuda")
        E().ef_ckpt_unpack(q, s, fmt, y)
        assert bool(y.isfinite().all())
        assert np.array_equal(y.double().cpu().numpy(), L.ckpt_unpack(wq, wsc, fmt, c))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("kernel,dtype,n,i,o,pad", [("k_linear_few forward", "bf16", 9, 96, 200, 0), ("k_linear_few forward", "f32", 9, 96, 200, 0),
                                                    ("k_linear_bf16<128> forward", "bf16", 200, 200, 200, 0),
                                                    ("k_linear_join forward", "bf16", 64, 8192, 200, 0),
                                                    ("k_linear_any forward", "bf16", 97, 99, 200, 1), ("k_linear_any forward", "f32", 97, 99, 200, 1)])
def test_forward(kernel, dtype, n, i, o, pad, fmt):
    """Each token is one 1: z's row is a column of the weights, exactly."""
    import torch
    announce("top forward", kernel, dtype, fmt)
    e, t = E(), tt(dtype)
    zz = near_the_top(2, n, o, dtype)
    wide = torch.zeros(o, i + pad, dtype=t)
    wide[:, i - n:i] = torch.from_numpy(zz).to(t).t()
    x = torch.zeros(n, i + pad, dtype=t)
    x[torch.arange(n), i - n + torch.arange(n)] = 1
    y = torch.empty(n, o, dtype=t, device="cuda")
    q, s = e.ckpt_buffers(n, o)
    ws = e.linear_workspace(e.EF_OP_FORWARD, n, i, o, t)
    e.timing_enable(True)
    try:
        e.ef_linear_forward(x.cuda()[:, :i], wide.cuda()[:, :i], y, ws, codes=q, scales=s, fmt=fmt)
        ran = e.timing_collect()
    finally:
        e.timing_enable(False)
    assert kernel in ran, ran
    assert np.array_equal(y.double().cpu().numpy(), zz)
    wq, wsc = L.ckpt_pack(zz, fmt)
    assert np.array_equal(host(s), wsc) and same_codes(q, wq, fmt)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype,pad", [("f32", 0), ("bf16", 0), ("bf16", 1)])
def test_a_padded_token_adds_nothing(dtype, pad, fmt):
    """dy is zero at the tokens whose kept rows are at the top: their groups' decoded values times 0 are 0."""
    import torch
    e, t = E(), tt(dtype)
    n, i, o = 130, 96, 64
    announce("top padded", dtype, pad, fmt)
    x = near_the_top(3, n, i, dtype)
    g = np.random.default_rng(5)
    live = np.arange(n) % 2 == 0
    x[live] = g.integers(-3, 4, (int(live.sum()), i))
    dy = g.integers(-3, 4, (n, o)) * live[:, None].astype(np.float64)
    q, s = e.ckpt_buffers(n, i)
    e.ef_ckpt_pack(torch.from_numpy(x).to(t).cuda(), q, s, fmt)
    wide = torch.zeros(n, o + pad, dtype=t, device="cuda")
    wide[:, :o] = torch.from_numpy(dy).cuda()
    dw = torch.empty(o, i, device="cuda")
    e.ef_linear_wgrad(wide[:, :o], q, s, fmt, dw, e.linear_workspace(e.EF_OP_WGRAD, n, i, o, t))
    assert np.array_equal(dw.double().cpu().numpy(), dy[live].T @ x[live])
    # and back through an activation kept there: its derivative is finite
    d = torch.ones(n, i, dtype=t, device="cuda")
    for act in range(5):
        dz = torch.empty_like(d)
        e.ef_ckpt_act_backward(act, q, s, fmt, d, dz)
        kept = L.ckpt_unpack(host(q), host(s), fmt, i)[~live]
        at_zero = [1, 0, 0.5, 0.5, 0.5][act]
        want = np.where(kept == 0, at_zero, kept > 0 if act else 1.0)
        assert np.array_equal(dz.double().cpu().numpy()[~live], want), act

"""GPU tests of what a checkpoint hands to the weight gradient at the ends of its range: every code under every scale,
and groups that stand for NaN, in each kernel that decodes one."""

import numpy as np
import pytest

from efs_gpu import announce
from oracle import linear_oracle as L

pytestmark = pytest.mark.gpu

FMTS = [L.INT8, L.E4M3]
# (kernel, type of dy, tokens, columns of x, rows of dw, ld of dy over its columns); a rule on sizes, types and alignment
# chooses the kernel, and the timing records say which one ran
KERNELS = [("k_linear_bf16<128> wgrad", "bf16", 256, 512, 256, 0), ("k_linear_bf16<256> wgrad", "bf16", 1024, 4096, 4096, 0),
           ("k_linear_any wgrad", "bf16", 256, 512, 256, 1), ("k_linear_any wgrad", "f32", 256, 512, 256, 0)]


def E():
    import paper_2009_09271_amd
    return paper_2009_09271_amd


def run(kernel, dy, q, s, fmt, pad, add=None):
    """(dw, db) of one call, which has to launch `kernel`; add: what dw and db hold before."""
    import torch
    e = E()
    (n, o), i = dy.shape, q.shape[1]
    wide = torch.zeros(n, o + pad, dtype=dy.dtype, device="cuda")
    wide[:, :o] = dy
    dw, db = (torch.full(shape, float("nan") if add is None else add, device="cuda") for shape in ((o, i), (o,)))
    ws = e.linear_workspace(e.EF_OP_WGRAD, n, i, o, dy.dtype)
    e.timing_enable(True)
    try:
        e.ef_linear_wgrad(wide[:, :o], q, s, fmt, dw, ws, db=db, accumulate=add is not None)
        ran = e.timing_collect()
    finally:
        e.timing_enable(False)
    assert kernel in ran, ran
    return dw, db


def values(q, s, fmt):
    """What codes and scales stand for, float64 on the GPU."""
    import torch
    table = L.ckpt_unpack(np.arange(256, dtype=np.uint8)[None], np.full((1, 8), 127, np.uint8), fmt, 256)[0]
    v = torch.from_numpy(table).cuda()[q.long()]
    return v * torch.exp2(s.double() - 127).repeat_interleave(32, 1)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("kernel,dtype,n,i,o,pad", KERNELS)
def test_every_code_and_scale(kernel, dtype, n, i, o, pad, fmt):
    """dy has a single 1 in each token's row: dw's row t is token t's kept values, bit for bit."""
    import torch
    announce("codes", kernel, dtype, fmt)
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    # every code but NaN's: int8 has no -128, e4m3 no 127 and 255; and every scale under which all of them are finite
    codes = [k for k in range(256) if (k != 128 if fmt == L.INT8 else k & 127 != 127)]
    top = 248 if fmt == L.INT8 else 246
    q = torch.tensor(codes, dtype=torch.uint8, device="cuda")[torch.arange(n * i, device="cuda") % len(codes)].view(n, i)
    s = (27 + (torch.arange(n, device="cuda")[:, None] + 7 * torch.arange(i // 32, device="cuda")) % (top - 26)).to(torch.uint8)
    assert int(s.min()) == 27 and int(s.max()) == top
    dy = torch.zeros(n, o, dtype=t, device="cuda")
    dy[torch.arange(n), torch.arange(n)] = 1
    dw, db = run(kernel, dy, q, s, fmt, pad)
    want = values(q, s, fmt)
    assert torch.equal(want.float().double(), want) and bool(want.isfinite().all())
    assert torch.equal(dw[:n].double(), want) and not dw[n:].any()
    assert torch.equal(db, dy.float().sum(0))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("kernel,dtype,n,i,o,pad", KERNELS)
def test_an_overflow_reaches_its_columns_of_dw(kernel, dtype, n, i, o, pad, fmt):
    """Groups that held an infinity or a NaN make their columns of dw NaN, written or added, and no others; so does a
    token whose dy is zero."""
    import torch
    announce("overflow", kernel, dtype, fmt)
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randint(-3, 4, (n, i), generator=g, device="cuda").float()
    dy = torch.randint(-2, 3, (n, o), generator=g, device="cuda").to(t)
    at = {3: (5, float("inf")), 67: (40, float("-inf")), 190: (n - 1, float("nan")), i - 1: (131, float("inf"))}
    for col, (row, v) in at.items():
        x[row, col] = v
    dy[131] = 0
    e = E()
    q, s = e.ckpt_buffers(n, i)
    e.ef_ckpt_pack(x, q, s, fmt)
    assert int((s == 255).sum()) == len(at)
    for row, col in ((r, c) for c, (r, _) in at.items()):
        assert int(s[row, col // 32]) == 255 and not q[row, col // 32 * 32:col // 32 * 32 + 32].any()
    bad = torch.zeros(i, dtype=torch.bool, device="cuda")
    for col in at:
        bad[col // 32 * 32:col // 32 * 32 + 32] = True
    want = torch.matmul(dy.double().t().contiguous(), torch.where(bad, torch.zeros_like(x), x).double())
    for add in (None, 2.0):
        dw, db = run(kernel, dy, q, s, fmt, pad, add)
        assert bool(dw[:, bad].isnan().all()), (int(dw[:, bad].isnan().sum()), dw[:, bad].numel())
        assert torch.equal(dw[:, ~bad].double(), want[:, ~bad] + (add or 0)) and torch.equal(db.double(), dy.double().sum(0) + (add or 0))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("kernel,dtype,n,i,o,pad", [("k_linear_bf16<128> dgrad", "bf16", 200, 512, 256, 0), ("k_linear_bf16<256> dgrad", "bf16", 4096, 4096, 256, 0),
                                                    ("k_linear_join dgrad", "bf16", 64, 256, 8192, 0), ("k_linear_any dgrad", "bf16", 200, 512, 256, 1),
                                                    ("k_linear_any dgrad", "f32", 200, 512, 256, 0)])
def test_an_overflow_reaches_its_group_of_dx(kernel, dtype, n, i, o, pad, fmt):
    """A group of the kept input of an activation that held an infinity or a NaN makes its 32 values of dx NaN, also
    where dy is zero, and no others; without an activation nothing of it is read."""
    import torch
    announce("overflow dgrad", kernel, dtype, fmt)
    e, t = E(), {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    z = torch.randint(-3, 4, (n, i), generator=g, device="cuda").float()
    bad = torch.zeros(n, i, dtype=torch.bool, device="cuda")
    for row, col, v in ((3, 5, float("inf")), (n - 1, i - 1, float("nan")), (33, 64, float("-inf")), (33, 31, float("inf"))):
        z[row, col] = v
        bad[row, col // 32 * 32:col // 32 * 32 + 32] = True
    q, s = e.ckpt_buffers(n, i)
    e.ef_ckpt_pack(z, q, s, fmt)
    dy = torch.randint(-2, 3, (n, o), generator=g, device="cuda").to(t)
    dy[33] = 0
    w = torch.randint(-2, 3, (o, i), generator=g, device="cuda").to(t)
    wide = torch.zeros(n, o + pad, dtype=t, device="cuda")
    wide[:, :o] = dy
    p = torch.matmul(dy.double(), w.double())
    ws = e.linear_workspace(e.EF_OP_DGRAD, n, i, o, t)
    for act in range(5):
        dx = torch.empty(n, i, dtype=t, device="cuda")
        e.timing_enable(True)
        try:
            e.ef_linear_dgrad(wide[:, :o], w, dx, ws, act=act, codes=q, scales=s, fmt=fmt)
            ran = e.timing_collect()
        finally:
            e.timing_enable(False)
        assert kernel in ran, ran
        dz = torch.empty(n, i, dtype=t, device="cuda")
        e.ef_ckpt_act_backward(act, q, s, fmt, torch.ones_like(dz), dz)
        if act == e.EF_ACT_NONE:
            assert torch.equal(dx.double(), p.to(t).double())
            continue
        assert torch.equal(dx.isnan(), bad) and torch.equal(dz.isnan(), bad)
        if act == e.EF_ACT_RELU:
            assert torch.equal(dx[~bad].double(), (p * (z > 0)).to(t).double()[~bad])

"""Rows of a checkpoint stand by themselves: every call that reads one, on rows [a, b) of a larger one, whose codes and
scales start anywhere, gives the bits that it gives on a copy of those rows."""

import pytest

from efs_gpu import announce
from oracle import linear_oracle as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [L.INT8, L.E4M3])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,i,o", [(1, 96, 64), (70, 96, 64), (200, 992, 264), (1000, 4064, 4096), (333, 33, 31)])
def test_rows_of_a_checkpoint(n, i, o, dtype, fmt):
    import torch
    import paper_2009_09271_amd as e
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    x = torch.randn(n + 8, i, generator=g, device="cuda")
    dy = torch.randn(n, o, generator=g, device="cuda").to(t)
    w = torch.randn(o, i, generator=g, device="cuda").to(t)
    q, s = e.ckpt_buffers(n + 8, i)
    e.ef_ckpt_pack(x, q, s, fmt)
    wg, dg = (e.linear_workspace(op, n, i, o, t) for op in (e.EF_OP_WGRAD, e.EF_OP_DGRAD))
    for a in (1, 2, 3, 7):
        announce("rows from", a, n, i, o, dtype, fmt)
        got = []
        for codes, scales in ((q[a:a + n], s[a:a + n]), (q[a:a + n].clone(), s[a:a + n].clone())):
            dw, db = torch.empty(o, i, device="cuda"), torch.empty(o, device="cuda")
            e.ef_linear_wgrad(dy, codes, scales, fmt, dw, wg, db=db)
            dx, y, dz = (torch.empty(n, i, dtype=t, device="cuda") for _ in range(3))
            e.ef_linear_dgrad(dy, w, dx, dg, act=e.EF_ACT_SILU, codes=codes, scales=scales, fmt=fmt)
            e.ef_ckpt_unpack(codes, scales, fmt, y)
            e.ef_ckpt_act_backward(e.EF_ACT_GELU, codes, scales, fmt, y, dz)
            got.append((dw, db, dx, y, dz))
        assert all(torch.equal(p, r) and bool(p.isfinite().all()) for p, r in zip(*got)), a
        part_q, part_s = e.ckpt_buffers(n, i)
        e.ef_ckpt_pack(x[a:a + n], part_q, part_s, fmt)
        assert torch.equal(part_q, q[a:a + n]) and torch.equal(part_s, s[a:a + n])

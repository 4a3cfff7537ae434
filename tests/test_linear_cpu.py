"""The checkpointed linear layer without a GPU: the oracle's own pins, and what the library and its binding refuse
before anything is enqueued."""

import ctypes
import math

import numpy as np
import pytest

E = pytest.importorskip("paper_2009_09271_amd")
from oracle import linear_oracle as L  # noqa: E402

FMTS = [L.INT8, L.E4M3]


# ---- the oracle --------------------------------------------------------------------------------------------------------
def test_pack_of_hand_worked_groups():
    x = np.zeros((4, 33))
    x[0, :4] = [127.0, 0.5, 1.5, -2.5]      # scale 1: ties to even
    x[1, :3] = [127.5, 3.0, -128.0]         # 128 does not fit: scale 2, 127.5 / 2 = 63.75, 3 / 2 = 1.5 -> 2
    x[2, 0] = 2.0 ** -130                   # under the least exponent: 0
    x[3, :2] = [np.inf, 1.0]
    x[:, 32] = 1.0                          # the second group has one column
    codes, scales = L.ckpt_pack(x, L.INT8)
    assert codes.shape == (4, 64) and scales.shape == (4, 2)
    assert codes[0, :4].view(np.int8).tolist() == [127, 0, 2, -2] and scales[0, 0] == 127
    assert codes[1, :3].view(np.int8).tolist() == [64, 2, -64] and scales[1, 0] == 128
    assert not codes[2, :32].any() and scales[2, 0] == 27
    assert not codes[3, :32].any() and scales[3, 0] == 255
    assert (codes[:, 32] == 64).all() and not codes[:, 33:].any() and (scales[:, 1] == 121).all()
    y = L.ckpt_unpack(codes, scales, L.INT8, 33)
    assert np.isnan(y[3, :32]).all() and (y[:, 32] == 1.0).all() and y[1, 2] == -128.0


def test_pack_e4m3_against_torch():
    import torch
    g = np.random.default_rng(1)
    x = (g.standard_normal((64, 96)) * np.exp(2 * g.standard_normal((64, 96)))).astype(np.float32)
    x[0, :3] = [448.0, 1.0 / 1024, -3.0 / 1024]  # ties among the smallest numbers
    codes, scales = L.ckpt_pack(x, L.E4M3)
    for r in range(64):
        for k in range(3):
            v = torch.from_numpy(np.ldexp(x[r, 32 * k:32 * k + 32], 127 - int(scales[r, k])))
            assert float(v.abs().max()) <= 448.0 < 2 * float(v.abs().max()) + 1e-3
            assert np.array_equal(v.to(torch.float8_e4m3fn).view(torch.uint8).numpy(), codes[r, 32 * k:32 * k + 32])


@pytest.mark.parametrize("fmt", FMTS)
def test_unpack_is_within_half_a_step_and_exact_in_bf16(fmt):
    import torch
    g = np.random.default_rng(2)
    x = (g.standard_normal((50, 130)) * 10.0 ** g.integers(-30, 30, (50, 1))).astype(np.float32)
    codes, scales = L.ckpt_pack(x, fmt)
    y = L.ckpt_unpack(codes, scales, fmt, 130)
    step = np.repeat(np.ldexp(1.0, scales.astype(int) - 127), 32, axis=1)[:, :130]
    half = step / 2 if fmt == L.INT8 else np.maximum(np.abs(x) * 2.0 ** -4, step * 2.0 ** -10)
    assert (np.abs(y - x) <= half).all()
    assert np.array_equal(torch.from_numpy(y).to(torch.bfloat16).double().numpy(), y)
    assert np.array_equal(L.ckpt_unpack(*L.ckpt_pack(y, fmt), fmt, 130), y)  # a second rounding changes nothing


@pytest.mark.parametrize("kind", range(5))
def test_activations_against_torch_and_differences(kind):
    import torch
    z = np.linspace(-9, 9, 1001) + 1e-3
    f = [lambda t: t, torch.relu, torch.nn.functional.gelu,
         lambda t: torch.nn.functional.gelu(t, approximate="tanh"), torch.nn.functional.silu][kind]
    t = torch.from_numpy(z).requires_grad_()
    y = f(t)
    y.sum().backward()
    np.testing.assert_allclose(L.act(z, kind), y.detach().numpy(), rtol=1e-9, atol=1e-14)
    np.testing.assert_allclose(L.act_slope(z, kind), t.grad.numpy(), rtol=1e-9, atol=1e-14)
    h = 1e-5
    np.testing.assert_allclose(L.act_slope(z, kind), (L.act(z + h, kind) - L.act(z - h, kind)) / (2 * h), atol=1e-8)
    assert math.isnan(L.act(np.array([np.nan]), kind)[0])


# ---- refusals ------------------------------------------------------------------------------------------------------------
P = ctypes.c_void_p


def at(k):
    return P(0x10000000 * (k + 1))  # never dereferenced: validation fails first


def test_row_bytes_and_workspaces():
    assert [E.lib().ef_ckpt_row_bytes(c) for c in (1, 32, 33, 4096, 0, -1, (1 << 26) + 1)] == [32, 32, 64, 4096, 0, 0, 0]
    for op in (E.EF_OP_FORWARD, E.EF_OP_DGRAD, E.EF_OP_WGRAD):
        for bad in ((-1, 8, 8, 0), (8, 0, 8, 0), (8, 8, 0, 0), (8, 8, 8, 7)):
            assert E.lib().ef_linear_workspace_bytes(op, *bad) == 0
        assert E.lib().ef_linear_workspace_bytes(op, 8192, 768, 768, E.EF_BF16) < 1 << 30
    assert E.lib().ef_linear_workspace_bytes(E.EF_OP_TOPK, 8, 8, 8, 0) == 0


def test_pack_and_unpack_refuse():
    lib = E.lib()

    def pack(n=4, c=40, x=at(0), ldx=40, dt=E.EF_F32, fmt=0, q=at(1), s=at(2)):
        return lib.ef_ckpt_pack(n, c, x, ldx, dt, fmt, q, s, None)

    def unpack(n=4, c=40, q=at(1), s=at(2), fmt=0, y=at(0), ldy=40, dt=E.EF_F32):
        return lib.ef_ckpt_unpack(n, c, q, s, fmt, y, ldy, dt, None)

    for f, name in ((pack, "x"), (unpack, "y")):
        assert f(n=-1) == E.EF_ERANGE and f(n=1 << 31) == E.EF_ERANGE and f(c=0) == E.EF_ERANGE
        assert f(c=(1 << 26) + 1, **{"ld" + name: 1 << 27}) == E.EF_ERANGE
        assert f(**{"ld" + name: 39}) == E.EF_EINVAL and f(**{name: None}) == E.EF_EINVAL
        assert f(**{name: P(0x10000002)}) == E.EF_EINVAL  # not on a float32
        assert f(dt=7) == E.EF_EINVAL and f(fmt=2) == E.EF_EINVAL
        assert f(q=None) == E.EF_EINVAL and f(s=None) == E.EF_EINVAL and f(q=P(0x20000008)) == E.EF_EINVAL
        assert f(q=at(0)) == E.EF_EINVAL and f(s=at(0)) == E.EF_EINVAL  # overlaps
        assert f(n=0, **{name: None}, q=None, s=None) == E.EF_OK       # no rows: nothing to do
    assert pack(s=at(1)) == E.EF_EINVAL


def test_act_backward_refuses():
    def call(n=4, c=40, act=1, q=at(1), s=at(2), fmt=0, dy=at(0), lddy=40, dz=at(3), lddz=40, dt=E.EF_BF16):
        return E.lib().ef_ckpt_act_backward(n, c, act, q, s, fmt, dy, lddy, dz, lddz, dt, None)

    assert call(act=-1) == E.EF_EINVAL and call(act=5) == E.EF_EINVAL and call(fmt=-1) == E.EF_EINVAL
    assert call(lddy=39) == E.EF_EINVAL and call(lddz=39) == E.EF_EINVAL and call(dy=None) == E.EF_EINVAL
    assert call(dz=P(0x10000000 + 2)) == E.EF_EINVAL                    # shifted over dy
    assert call(dz=at(0), lddz=41) == E.EF_EINVAL                       # dy itself, but another ld
    assert call(dz=at(1)) == E.EF_EINVAL and call(n=0, dy=None, dz=None, q=None, s=None) == E.EF_OK


def test_products_refuse():
    lib = E.lib()

    def fwd(n=4, i=8, o=40, x=at(0), ldx=8, w=at(1), ldw=8, b=None, act=0, r=None, ldr=0, y=at(2), ldy=40, dt=0, q=None,
            s=None, fmt=0):
        return lib.ef_linear_forward(n, i, o, x, ldx, w, ldw, b, act, r, ldr, y, ldy, dt, q, s, fmt, at(9), 1 << 40, None)

    assert fwd(n=-1) == fwd(i=0) == fwd(o=0) == fwd(o=1 << 27, ldy=1 << 27) == E.EF_ERANGE
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(ldx=7), dict(ldw=7), dict(ldy=39), dict(dt=2), dict(act=5),
                dict(b=P(0x30000001)), dict(r=at(3), ldr=39), dict(q=at(4)), dict(s=at(4)), dict(q=at(4), s=at(5), fmt=9),
                dict(q=P(0x50000004), s=at(5)), dict(y=at(0)), dict(y=at(1)), dict(q=at(2), s=at(5)), dict(q=at(4), s=at(4)),
                dict(r=P(0x30000000 + 4), ldr=40), dict(r=at(2), ldr=41), dict(q=at(4), s=at(0)), dict(b=at(2))):
        assert fwd(**bad) == E.EF_EINVAL, bad
    assert fwd(n=0, x=None, y=None) == E.EF_OK

    def dgr(n=4, i=40, o=8, dy=at(0), lddy=8, w=at(1), ldw=40, act=0, q=None, s=None, fmt=0, r=None, ldr=0, dx=at(2),
            lddx=40, dt=1):
        return lib.ef_linear_dgrad(n, i, o, dy, lddy, w, ldw, act, q, s, fmt, r, ldr, dx, lddx, dt, at(9), 1 << 40, None)

    for bad in (dict(dy=None), dict(w=None), dict(dx=None), dict(lddy=7), dict(ldw=39), dict(lddx=39), dict(dt=-1), dict(act=9),
                dict(act=1), dict(act=1, q=at(3)), dict(act=1, q=at(3), s=at(4), fmt=2), dict(act=1, q=at(2), s=at(4)),
                dict(act=1, q=at(3), s=at(2)), dict(r=at(2), ldr=48), dict(r=at(3), ldr=1), dict(dx=at(0)), dict(dx=at(1))):
        assert dgr(**bad) == E.EF_EINVAL, bad
    assert dgr(n=0, dy=None, dx=None) == E.EF_OK

    def wgr(n=4, i=40, o=8, dy=at(0), lddy=8, dt=1, q=at(1), s=at(2), fmt=0, dw=at(3), db=None, gd=0, add=0):
        return lib.ef_linear_wgrad(n, i, o, dy, lddy, dt, q, s, fmt, dw, db, gd, add, at(9), 1 << 40, None)

    for bad in (dict(dy=None), dict(q=None), dict(s=None), dict(dw=None), dict(lddy=7), dict(dt=3), dict(gd=3), dict(fmt=4),
                dict(gd=1, add=1), dict(dw=P(0x40000002)), dict(db=P(0x50000001)), dict(db=at(3)), dict(dw=at(0)),
                dict(dw=at(1)), dict(dw=at(2)), dict(db=at(0)), dict(q=P(0x20000001))):
        assert wgr(**bad) == E.EF_EINVAL, bad


def test_products_refuse_a_workspace_over_their_matrices():
    lib, n = E.lib(), 64
    for op in (E.EF_OP_FORWARD, E.EF_OP_DGRAD):
        assert lib.ef_linear_workspace_bytes(op, n, 8192, 8192, E.EF_BF16) > 0
    assert lib.ef_linear_workspace_bytes(E.EF_OP_WGRAD, 8192, 64, 64, E.EF_BF16) > 0
    size = 1 << 40
    for over in range(7):  # (at(k): the k-th buffer of the call, the workspace laid over it from its start)
        forward = lib.ef_linear_forward(n, 8192, 8192, at(0), 8192, at(1), 8192, at(2), 0, at(3), 8192, at(4), 8192, E.EF_BF16,
                                        at(5), at(6), 0, at(over), size, None)
        dgrad = lib.ef_linear_dgrad(n, 8192, 8192, at(0), 8192, at(1), 8192, 1, at(2), at(3), 0, at(4), 8192, at(5), 8192,
                                    E.EF_BF16, at(min(over, 5)), size, None)
        wgrad = lib.ef_linear_wgrad(8192, 64, 64, at(0), 64, E.EF_BF16, at(1), at(2), 0, at(3), at(4), E.EF_F32, 0,
                                    at(min(over, 4)), size, None)
        assert (forward, dgrad, wgrad) == (E.EF_EINVAL,) * 3, over


def test_products_refuse_more_tiles_than_a_grid_has():
    """A grid has less than 2^32 threads: 2^24 tiles of 128 x 128 or 2^23 of 256 x 256 are too many."""
    lib, n = E.lib(), (1 << 31) - 1
    far = [P(1 << (48 + k)) for k in range(5)]
    for dt, i, o in ((E.EF_F32, 1, 1), (E.EF_BF16, 1, 1), (E.EF_BF16, 8, 264)):
        assert lib.ef_linear_forward(n, i, o, far[0], i, far[1], i, None, 0, None, 0, far[2], o, dt, None, None, 0, far[3], 1 << 60,
                                     None) == E.EF_ERANGE
        assert lib.ef_linear_dgrad(n, o, i, far[0], i, far[1], o, 0, None, None, 0, None, 0, far[2], o, dt, far[3], 1 << 60,
                                   None) == E.EF_ERANGE


def test_binding_refuses_what_does_not_fit():
    import torch
    x, w, y = torch.zeros(4, 8), torch.zeros(40, 8), torch.zeros(4, 40)
    q, s = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8)
    for call in (lambda: E.ef_ckpt_pack(y, q, s), lambda: E.ef_ckpt_unpack(q, s, 0, y),
                 lambda: E.ef_ckpt_act_backward(1, q, s, 0, y, y), lambda: E.ef_linear_forward(x, w, y, None),
                 lambda: E.ef_linear_dgrad(y, w, x, None), lambda: E.ef_linear_wgrad(x, q, s, 0, w, None)):
        with pytest.raises(E.EfError) as ex:
            call()
        assert ex.value.code == E.EF_EINVAL and "not on a GPU" in str(ex.value)
    with pytest.raises(E.EfError) as ex:
        E.ef_linear_forward(None, w, y, None)
    assert "x is None" in str(ex.value)
    with pytest.raises(TypeError):
        E.linear_workspace(E.EF_OP_FORWARD, 4, 8, 40, torch.float16, "cpu")

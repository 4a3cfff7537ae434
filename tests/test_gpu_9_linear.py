"""GPU tests of the checkpointed linear layer against its float64 oracle.

Checkpoints are compared bit for bit.  Products are compared in two ways: bit for bit on small integers, whose sums
are exact in float32 in any order, and on random values within the bound of a float32 sum of K terms,
2 (K + 8) 2^-24 times the sum of the terms' magnitudes (twice the textbook bound, for the inner steps of the matrix
instructions), plus half a step of the stored type (2^-24 or 2^-8 of the value) and, where an activation is
applied, 1e-6 (1 + |z|): a dozen float32 roundings of a function whose slope stays under 1.13."""

import numpy as np
import pytest

from efs_gpu import announce, bits, dev, host
from oracle import efsparse_oracle as O
from oracle import linear_oracle as L

pytestmark = pytest.mark.gpu

FMTS = [L.INT8, L.E4M3]
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def E():
    import paper_2009_09271_amd
    return paper_2009_09271_amd


def tt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def put(x, dtype, ld=None, shift=0):
    """x on the GPU as `dtype`, its rows ld apart and starting `shift` elements into an allocation; what surrounds it
    is 77, and `around` tells whether it still is."""
    import torch
    n, c = x.shape
    ld = ld or c
    flat = torch.full((shift + n * ld + 8,), 77.0, dtype=tt(dtype), device="cuda")
    t = flat[shift:shift + n * ld].view(n, ld)[:, :c] if n else flat[:0].view(0, c)
    t.copy_(torch.from_numpy(np.ascontiguousarray(x, dtype=np.float64)).to(tt(dtype)))
    t.flat, t.place = flat, (shift, ld)
    return t


def around(t):
    import torch
    shift, ld = t.place
    n, c = t.shape
    m = torch.ones_like(t.flat, dtype=torch.bool)
    m[shift:shift + n * ld].view(n, ld)[:, :c] = False
    return bool((t.flat[m] == 77.0).all())


def val(t):
    return t.detach().double().cpu().numpy()


def rnd(rng, n, c, dtype, scale=1.0):
    """Random values that `dtype` holds exactly, as float64."""
    import torch
    x = torch.from_numpy(rng.standard_normal((n, c)) * scale).to(tt(dtype))
    return x.double().numpy()


def ints(rng, n, c):
    return rng.integers(-3, 4, (n, c)).astype(np.float64)


def kept(x, fmt):
    """A checkpoint on the GPU and what it stands for."""
    import torch
    q, s = L.ckpt_pack(x, fmt)
    return torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda(), L.ckpt_unpack(q, s, fmt, x.shape[1])


def ws(op, n, i, o, dtype):
    """Filled with NaN: nothing may rest on what a workspace held."""
    w = E().linear_workspace(op, n, i, o, tt(dtype))
    w.fill_(255)
    return w


def near(got, want, tol, where):
    got = val(got)
    assert got.shape == want.shape, where
    bad = ~(np.abs(got - want) <= tol)
    bad &= ~(np.isnan(got) & np.isnan(want))
    assert not bad.any(), f"{where}: {bad.sum()} of {bad.size} off, first {np.argwhere(bad)[:3].tolist()}: " \
                          f"{got[bad][:3]} for {want[bad][:3]} (bound {np.broadcast_to(tol, bad.shape)[bad][:3]})"


# ---- checkpoints ---------------------------------------------------------------------------------------------------------
def hard_values(rng, n, c):
    """Rows of ordinary, tied, tiny, huge, zero and non-finite values, exact in bfloat16."""
    x = rnd(rng, n, c, "bf16") * 2.0 ** rng.integers(-20, 20, (n, 1))
    for r in range(n):
        k = r % 8
        if k == 1:
            x[r] = rng.integers(-255, 256, c) / 2.0       # ties and groups that reach 127.5
        elif k == 2:
            x[r] = 0.0
        elif k == 3:
            x[r] *= 2.0 ** -120                           # at and under the least exponent
        elif k == 4:
            x[r] = np.sign(x[r]) * 3.3895313892515355e38  # the largest bfloat16
        elif k == 5:
            x[r, rng.integers(0, c)] = [np.inf, -np.inf, np.nan][r % 3]
        elif k == 6:
            x[r] = np.where(rng.random(c) < 0.9, 0.0, -0.0)
    return x


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,c,ld,shift", [(1, 1, 1, 0), (1, 32, 32, 0), (3, 31, 31, 1), (5, 33, 40, 0), (17, 96, 97, 3),
                                          (9, 771, 771, 0), (2, 4096, 4096, 0), (260, 100, 104, 8), (33, 2080, 2080, 5)])
def test_pack_and_unpack_bit_for_bit(n, c, ld, shift, dtype, fmt):
    import torch
    announce("pack", n, c, ld, shift, dtype, fmt)
    rng = np.random.default_rng([n, c, fmt])
    x = hard_values(rng, n, c)
    if dtype == "f32":
        fine = np.isfinite(x)
        x[fine] = (x[fine] * (1 + rng.integers(0, 1 << 12, int(fine.sum())) * 2.0 ** -23)).astype(np.float32)
    q, s = E().ckpt_buffers(n, c)
    q.fill_(99), s.fill_(99)
    t = put(x, dtype, ld, shift)
    E().ef_ckpt_pack(t, q, s, fmt)
    wq, wsc = L.ckpt_pack(x, fmt)
    assert np.array_equal(host(s), wsc)
    neg0 = 0 if fmt == L.INT8 else 128  # (the two zeros are one value)
    assert np.array_equal(np.where(host(q) == neg0, 0, host(q)), np.where(wq == neg0, 0, wq))
    y = put(np.zeros((n, c)), dtype, ld, shift)
    E().ef_ckpt_unpack(q, s, fmt, y)
    want = torch.from_numpy(L.ckpt_unpack(wq, wsc, fmt, c)).to(tt(dtype)).double().numpy()
    assert np.array_equal(val(y), want, equal_nan=True) and around(y) and around(t)


def test_pack_past_32_bit_offsets():
    import torch
    n, c = 70000, 65536
    announce("pack of", n, "x", c)
    x = torch.zeros(n, c, dtype=torch.bfloat16, device="cuda")
    rows = [0, 1, 32768, 32769, 65535, 65536, n - 1]
    want = {}
    rng = np.random.default_rng(3)
    for r in rows:
        v = rnd(rng, 1, c, "bf16")
        x[r] = torch.from_numpy(v[0]).to(x)
        want[r] = L.ckpt_pack(v, L.INT8)
    q, s = E().ckpt_buffers(n, c)
    E().ef_ckpt_pack(x, q, s)
    x.zero_()
    E().ef_ckpt_unpack(q, s, L.INT8, x)
    for r in rows:
        assert np.array_equal(host(q[r]), want[r][0][0]) and np.array_equal(host(s[r]), want[r][1][0])
        assert np.array_equal(val(x[r]), L.ckpt_unpack(*want[r], L.INT8, c)[0])
    assert int(s[2].min()) == int(s[2].max()) == 27 and not q[n - 2].any()


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("n,c,ld,shift,dtype,fmt", [(1, 1, 1, 0, "f32", 0), (7, 33, 35, 1, "bf16", 1), (40, 257, 257, 0, "f32", 1),
                                                    (21, 2304, 2304, 0, "bf16", 0)])
def test_act_backward(n, c, ld, shift, dtype, fmt, act):
    announce("act", n, c, dtype, fmt, act)
    rng = np.random.default_rng([n, c, act])
    z = rnd(rng, n, c, "f32") * 2.0 ** rng.integers(-3, 9, (n, 1))
    if n > 2:
        z[1, 0] = np.nan
        z[2] = 2.0 ** 100 * np.sign(z[2])
    q, s, zk = kept(z, fmt)
    dy = rnd(rng, n, c, dtype, 1e-2)
    want = dy * L.act_slope(zk, act)
    tol = np.abs(dy) * 2e-6 + HALF[dtype] * np.abs(want) + 1e-40
    t, dz = put(dy, dtype, ld, shift), put(np.zeros((n, c)), dtype)
    E().ef_ckpt_act_backward(act, q, s, fmt, t, dz)
    near(dz, want, tol, "dz")
    E().ef_ckpt_act_backward(act, q, s, fmt, t, t)
    assert np.array_equal(val(t), val(dz), equal_nan=True) and around(t) and around(dz)


# ---- products ------------------------------------------------------------------------------------------------------------
SIZES = [(1, 1, 1), (1, 64, 48), (2, 33, 31), (5, 7, 130), (17, 96, 64), (16, 512, 256), (64, 64, 64), (127, 129, 131),
         (200, 40, 264), (256, 256, 256), (333, 771, 97), (300, 512, 640), (513, 264, 520)]


def layout_of(k):
    """(extra ld, shift) of a case's matrices: contiguous and aligned, padded rows, odd rows at odd addresses."""
    return [(0, 0), (8, 8), (1, 1), (0, 3)][k % 4]


def forward(x, w, b, r, dtype, act, keep, fmt, k=0):
    (n, i), o = x.shape, w.shape[0]
    pad, sh = layout_of(k)
    e = E()
    y = put(np.zeros((n, o)), dtype, o + pad, sh)
    q, s = e.ckpt_buffers(n, o) if keep else (None, None)
    if keep:
        q.fill_(99), s.fill_(99)
    e.ef_linear_forward(put(x, dtype, i + pad, sh), put(w, dtype, i + pad, sh), y, ws(e.EF_OP_FORWARD, n, i, o, dtype),
                        bias=None if b is None else put(b[None], dtype, o, sh)[0], act=act,
                        res=None if r is None else put(r, dtype, o + pad, sh), codes=q, scales=s, fmt=fmt)
    assert around(y)
    return y, q, s


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,i,o", SIZES)
def test_forward_of_integers_bit_for_bit(n, i, o, dtype):
    import torch
    for k in range(4):
        announce("forward ints", n, i, o, dtype, k)
        rng = np.random.default_rng([n, i, o, k])
        x, w, b, r = ints(rng, n, i), ints(rng, o, i), ints(rng, 1, o)[0], ints(rng, n, o)
        z = x @ w.T + b
        y, q, s = forward(x, w, b, r, dtype, L.RELU, True, k % 2, k)
        want = torch.from_numpy(np.maximum(z, 0) + r).to(tt(dtype)).double().numpy()
        assert np.array_equal(val(y), want)
        wq, wsc = L.ckpt_pack(z, k % 2)
        assert np.array_equal(host(s), wsc) and np.array_equal(host(q), wq)


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("n,i,o,dtype,fmt,k", [(1, 512, 300, "bf16", 0, 0), (3, 333, 65, "f32", 1, 2), (70, 768, 200, "bf16", 1, 0),
                                               (129, 257, 96, "bf16", 0, 2), (260, 512, 384, "f32", 0, 0)])
def test_forward(n, i, o, dtype, fmt, k, act):
    announce("forward", n, i, o, dtype, fmt, act)
    rng = np.random.default_rng([n, i, act])
    x, w = rnd(rng, n, i, dtype), rnd(rng, o, i, dtype, i ** -0.5)
    b, r = rnd(rng, 1, o, dtype)[0], rnd(rng, n, o, dtype)
    z, mag = L.forward(x, w, b)
    ez = 2 * (i + 8) * 2.0 ** -24 * mag
    y, q, s = forward(x, w, b, r, dtype, act, True, fmt, k)
    want = L.act(z, act) + r
    ea = 1e-6 * (1 + np.abs(z)) if act else 0
    near(y, want, 1.13 * ez + ea + HALF[dtype] * (np.abs(want) + 1e-6) + 2.0 ** -24 * np.abs(want), "y")
    y0, q0, s0 = forward(x, w, b, r, dtype, act, False, fmt, k)
    assert np.array_equal(val(y0), val(y))  # keeping the checkpoint changes nothing
    step = np.repeat(np.ldexp(1.0, host(s).astype(int) - 127), 32, axis=1)[:, :o]
    half = step / 2 if fmt == L.INT8 else np.maximum(np.abs(z) * 2.0 ** -4, step * 2.0 ** -10)
    got = L.ckpt_unpack(host(q), host(s), fmt, o)
    assert (np.abs(got - z) <= half + 1.1 * ez + 1e-30).all()
    assert not host(q)[:, o:].any()
    if dtype == "f32":  # without activation and residual y is z: the checkpoint is y's own
        y1, q1, s1 = forward(x, w, b, None, dtype, L.NONE, True, fmt, k)
        wq, wsc = L.ckpt_pack(val(y1), fmt)
        assert np.array_equal(host(q1), wq) and np.array_equal(host(s1), wsc)


def dgrad(dy, w, z, r, dtype, act, fmt, k=0):
    (n, o), i = dy.shape, w.shape[1]
    pad, sh = layout_of(k)
    e = E()
    q, s, zk = kept(z, fmt)
    dx = put(np.zeros((n, i)), dtype, i + pad, sh)
    e.ef_linear_dgrad(put(dy, dtype, o + pad, sh), put(w, dtype, i + pad, sh), dx, ws(e.EF_OP_DGRAD, n, i, o, dtype), act=act,
                      codes=q if act else None, scales=s if act else None, fmt=fmt,
                      res=None if r is None else put(r, dtype, i + pad, sh))
    assert around(dx)
    return dx, zk


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,i,o", SIZES)
def test_dgrad_of_integers_bit_for_bit(n, i, o, dtype):
    import torch
    for k in range(4):
        announce("dgrad ints", n, i, o, dtype, k)
        rng = np.random.default_rng([n, i, o, k])
        dy, w, z, r = ints(rng, n, o), ints(rng, o, i), ints(rng, n, i), ints(rng, n, i)
        dx, _ = dgrad(dy, w, z, r, dtype, L.RELU, k % 2, k)
        want = torch.from_numpy((dy @ w) * (z > 0) + r).to(tt(dtype)).double().numpy()
        assert np.array_equal(val(dx), want)


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("n,i,o,dtype,fmt,k", [(1, 300, 512, "bf16", 0, 0), (3, 65, 333, "f32", 1, 2), (70, 200, 768, "bf16", 1, 0),
                                               (129, 96, 257, "bf16", 0, 2), (260, 384, 512, "f32", 0, 0)])
def test_dgrad(n, i, o, dtype, fmt, k, act):
    announce("dgrad", n, i, o, dtype, fmt, act)
    rng = np.random.default_rng([n, i, act])
    dy, w = rnd(rng, n, o, dtype, 1e-2), rnd(rng, o, i, dtype, i ** -0.5)
    z, r = rnd(rng, n, i, "f32", 2.0), rnd(rng, n, i, dtype, 1e-2) if act % 2 else None
    dx, zk = dgrad(dy, w, z, r, dtype, act, fmt, k)
    p, mag = L.dgrad(dy, w)
    want = p * L.act_slope(zk, act) + (0 if r is None else r)
    near(dx, want, 1.13 * 2 * (o + 8) * 2.0 ** -24 * mag + np.abs(p) * 2e-6 + (HALF[dtype] + 2.0 ** -24) * np.abs(want) + 1e-30, "dx")


def wgrad(dy, x, dtype, fmt, gtype="f32", add=None, k=0):
    import torch
    (n, o), i = dy.shape, x.shape[1]
    pad, sh = layout_of(k)
    e = E()
    q, s, xk = kept(x, fmt)
    flat = torch.full((sh + o * i + o + 9,), 77.0, dtype=tt(gtype), device="cuda")
    dw, db = flat[sh:sh + o * i].view(o, i), flat[sh + o * i:sh + o * i + o]
    if add is not None:
        flat[sh:sh + o * i + o] = dev(add.astype(np.float32))
    e.ef_linear_wgrad(put(dy, dtype, o + pad, sh), q, s, fmt, dw, ws(e.EF_OP_WGRAD, n, i, o, dtype), db=db,
                      accumulate=add is not None)
    assert bool((flat[:sh] == 77.0).all()) and bool((flat[sh + o * i + o:] == 77.0).all())
    return dw, db, xk


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,i,o", SIZES + [(4096, 96, 72), (2050, 256, 128)])
def test_wgrad_of_integers_bit_for_bit(n, i, o, dtype):
    import torch
    for k in range(4):
        announce("wgrad ints", n, i, o, dtype, k)
        rng = np.random.default_rng([n, i, o, k])
        dy, x = ints(rng, n, o), ints(rng, n, i)
        old = rng.integers(-9, 10, o * i + o).astype(np.float64)
        dw, db, _ = wgrad(dy, x, dtype, k % 2, "f32", old if k % 2 else None, k)
        want, wb = dy.T @ x, dy.sum(0)
        if k % 2:
            want, wb = want + old[:o * i].reshape(o, i), wb + old[o * i:]
        assert np.array_equal(val(dw), want) and np.array_equal(val(db), wb)
        dw, db, _ = wgrad(dy, x, dtype, k % 2, "bf16", None, k)
        for got, full in ((dw, dy.T @ x), (db, dy.sum(0))):
            assert np.array_equal(val(got), torch.from_numpy(full).to(torch.bfloat16).double().numpy())


@pytest.mark.parametrize("dtype,fmt", [("f32", 0), ("bf16", 1), ("bf16", 0), ("f32", 1)])
@pytest.mark.parametrize("n,i,o,k", [(1, 40, 30, 0), (77, 130, 33, 2), (600, 256, 300, 0), (3001, 96, 200, 1)])
def test_wgrad(n, i, o, k, dtype, fmt):
    announce("wgrad", n, i, o, dtype, fmt)
    rng = np.random.default_rng([n, i, fmt])
    dy = rnd(rng, n, o, dtype, 1e-2) * 2.0 ** rng.integers(-12, 3, (n, 1))
    dy[n // 2] = 0
    x = rnd(rng, n, i, "f32") * 2.0 ** rng.integers(-9, 9, (1, i))
    dw, db, xk = wgrad(dy, x, dtype, fmt, "f32", None, k)
    want, mag = L.wgrad(dy, xk)
    near(dw, want, 2 * (n + 8) * 2.0 ** -24 * mag + 1e-37, "dw")
    near(db, dy.sum(0), 2 * (n + 8) * 2.0 ** -24 * np.abs(dy).sum(0), "db")


def test_wgrad_accumulated_is_the_accumulate_step():
    """dw, db added to the error-feedback memory: bitwise ef_accumulate of the written gradient."""
    import torch
    e = E()
    rng = np.random.default_rng(5)
    n, i, o = 700, 160, 97
    lay = e.Layout(o * i + o, [0, o * i, o * i + o], 0.01).bind("cuda")
    dy, x = rnd(rng, n, o, "bf16", 1e-2), rnd(rng, n, i, "f32")
    q, s, _ = kept(x, 0)
    t, w = put(dy, "bf16"), ws(e.EF_OP_WGRAD, n, i, o, "bf16")
    mem = dev((1e-2 * rng.standard_normal(lay.d)).astype(np.float32))
    g, acc = torch.empty_like(mem), torch.empty_like(mem)
    e.ef_linear_wgrad(t, q, s, 0, g[:o * i].view(o, i), w, db=g[o * i:])
    e.ef_accumulate(lay, g, mem, acc)
    e.ef_linear_wgrad(t, q, s, 0, mem[:o * i].view(o, i), w, db=mem[o * i:], accumulate=True)
    assert np.array_equal(bits(host(mem)), bits(host(acc)))


def test_no_tokens():
    import torch
    e = E()
    for dtype in ("f32", "bf16"):
        q, s = e.ckpt_buffers(0, 40)
        empty = lambda c: torch.empty(0, c, dtype=tt(dtype), device="cuda")  # noqa: E731
        w = torch.ones(24, 40, dtype=tt(dtype), device="cuda")
        e.ef_ckpt_pack(empty(40), q, s)
        e.ef_ckpt_unpack(q, s, 0, empty(40))
        e.ef_ckpt_act_backward(e.EF_ACT_SILU, q, s, 0, empty(40), empty(40))
        e.ef_linear_forward(empty(40), w, empty(24), None)
        e.ef_linear_dgrad(empty(24), w, empty(40), None)
        dw, db = torch.full((24, 40), 7.0, device="cuda"), torch.full((24,), 7.0, device="cuda")
        wk = ws(e.EF_OP_WGRAD, 0, 40, 24, dtype)
        e.ef_linear_wgrad(empty(24), q, s, 0, dw, wk, db=db, accumulate=True)
        assert bool((dw == 7.0).all()) and bool((db == 7.0).all())
        e.ef_linear_wgrad(empty(24), q, s, 0, dw, wk, db=db)
        assert not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_finite_stays_where_it_belongs(dtype):
    """An infinity in one token's activations reaches its own row of y, its own column group of dw, and nothing else."""
    rng = np.random.default_rng(6)
    n, i, o = 70, 96, 64
    x, w = rnd(rng, n, i, dtype), rnd(rng, o, i, dtype)
    x[33, 40] = np.inf
    y, q, s = forward(x, w, None, None, dtype, L.NONE, True, 0)
    got = val(y)
    assert not np.isfinite(got[33]).any() and np.isfinite(np.delete(got, 33, 0)).all()
    assert (host(s)[33] == 255).all() and (np.delete(host(s), 33, 0) < 255).all()
    dw, db, _ = wgrad(rnd(rng, n, o, dtype), x, dtype, 0)
    got = val(dw)
    assert np.isnan(got[:, 32:64]).all() and np.isfinite(got[:, :32]).all() and np.isfinite(got[:, 64:]).all()
    assert np.isfinite(val(db)).all()


def test_results_in_place_and_on_another_stream():
    import torch
    e = E()
    rng = np.random.default_rng(7)
    n, i, o = 190, 256, 256
    for dtype in ("f32", "bf16"):
        x, w, r = rnd(rng, n, i, dtype), rnd(rng, o, i, dtype, 0.1), rnd(rng, n, o, dtype)
        q, s, _ = kept(r, 0)
        y, _, _ = forward(x, w, None, r, dtype, L.SILU, False, 0)
        t = put(r, dtype)
        e.ef_linear_forward(put(x, dtype), put(w, dtype), t, ws(e.EF_OP_FORWARD, n, i, o, dtype), act=L.SILU, res=t)
        assert np.array_equal(val(t), val(y))
        a, b = put(r, dtype), put(np.zeros((n, i)), dtype)
        e.ef_linear_dgrad(put(x, dtype), put(w, dtype), b, ws(e.EF_OP_DGRAD, n, i, o, dtype), act=L.GELU, codes=q, scales=s, res=a)
        e.ef_linear_dgrad(put(x, dtype), put(w, dtype), a, ws(e.EF_OP_DGRAD, n, i, o, dtype), act=L.GELU, codes=q, scales=s, res=a)
        assert np.array_equal(val(a), val(b))
        side = torch.cuda.Stream()
        t2, xs, wt, wk = put(r, dtype), put(x, dtype), put(w, dtype), ws(e.EF_OP_FORWARD, n, i, o, dtype)
        side.wait_stream(torch.cuda.current_stream())
        e.ef_linear_forward(xs, wt, t2, wk, act=L.SILU, res=t2, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert np.array_equal(val(t2), val(y))


# ---- together ------------------------------------------------------------------------------------------------------------
class Mlp:
    """Two layers with a skip connection, out = x + W2 act(W1 x + b1) + b2, loss = sum(out * t): forward with checkpoints,
    backward into the flat gradient or the error-feedback memory, as a worker makes it."""

    def __init__(self, n, i, h, dtype, act, fmt, seed):
        import torch
        e = self.e = E()
        rng = np.random.default_rng(seed)
        self.n, self.i, self.h, self.dtype, self.act, self.fmt = n, i, h, dtype, act, fmt
        self.np = {"x": rnd(rng, n, i, dtype), "w1": rnd(rng, h, i, dtype, i ** -0.5), "b1": rnd(rng, 1, h, dtype, 0.1),
                   "w2": rnd(rng, i, h, dtype, h ** -0.5), "b2": rnd(rng, 1, i, dtype, 0.1), "t": rnd(rng, n, i, dtype, 1e-2)}
        self.p = {k: put(v, dtype) for k, v in self.np.items()}
        sizes = [h * i, h, i * h, i]
        self.offs = [0] + np.cumsum(sizes).tolist()
        t = tt(dtype)
        mk = lambda c: torch.empty(n, c, dtype=t, device="cuda")  # noqa: E731
        self.a, self.out, self.dz, self.dx = mk(h), mk(i), mk(h), mk(i)
        self.kx, self.kz, self.ka = (e.ckpt_buffers(n, c) for c in (i, h, h))
        self.ws = torch.empty(max(int(e.linear_workspace(op, n, a, b, t).numel()) for op in (7, 8, 9) for a, b in ((i, h), (h, i))),
                              dtype=torch.uint8, device="cuda")

    def seg(self, g, l, shape=None):
        v = g[self.offs[l]:self.offs[l + 1]]
        return v.view(shape) if shape else v

    def step(self, g, accumulate):
        e, p, f = self.e, self.p, self.fmt
        e.ef_ckpt_pack(p["x"], *self.kx, f)
        e.ef_linear_forward(p["x"], p["w1"], self.a, self.ws, bias=p["b1"][0], act=self.act, codes=self.kz[0], scales=self.kz[1], fmt=f)
        e.ef_ckpt_pack(self.a, *self.ka, f)
        e.ef_linear_forward(self.a, p["w2"], self.out, self.ws, bias=p["b2"][0], res=p["x"])
        dy = p["t"]
        e.ef_linear_wgrad(dy, *self.ka, f, self.seg(g, 2, (self.i, self.h)), self.ws, db=self.seg(g, 3), accumulate=accumulate)
        e.ef_linear_dgrad(dy, p["w2"], self.dz, self.ws, act=self.act, codes=self.kz[0], scales=self.kz[1], fmt=f)
        e.ef_linear_wgrad(self.dz, *self.kx, f, self.seg(g, 0, (self.h, self.i)), self.ws, db=self.seg(g, 1), accumulate=accumulate)
        e.ef_linear_dgrad(self.dz, p["w1"], self.dx, self.ws, res=dy)

    def exact(self, xk=None, ak=None, zk=None):
        """The flat gradient and dx by the formula in float64, from given checkpoints or the exact activations."""
        v = self.np
        z = v["x"] @ v["w1"].T + v["b1"]
        a = L.act(z, self.act)
        dz = (v["t"] @ v["w2"]) * L.act_slope(z if zk is None else zk, self.act)
        parts = [dz.T @ (v["x"] if xk is None else xk), dz.sum(0), v["t"].T @ (a if ak is None else ak), v["t"].sum(0)]
        return np.concatenate([q.ravel() for q in parts]), dz @ v["w1"] + v["t"]


@pytest.mark.parametrize("dtype,act,fmt,n,i,h", [("f32", L.GELU, 0, 150, 64, 200), ("bf16", L.SILU, 1, 257, 96, 130),
                                                 ("bf16", L.GELU_TANH, 0, 300, 256, 512)])
def test_two_layers_into_the_error_feedback_memory_and_a_message(dtype, act, fmt, n, i, h):
    import torch
    announce("two layers", dtype, act, fmt)
    m = Mlp(n, i, h, dtype, act, fmt, 11)
    d = m.offs[-1]
    g = torch.zeros(d, device="cuda")
    m.step(g, False)
    un = lambda k, c: L.ckpt_unpack(host(k[0]), host(k[1]), fmt, c)  # noqa: E731
    want, wdx = m.exact(un(m.kx, i), un(m.ka, h), un(m.kz, h))
    # dz is stored in the layers' type before the first layer's products: half a step of it in their terms
    half = HALF[dtype] if dtype == "bf16" else 2.0 ** -20
    rel = np.linalg.norm(host(g) - want) / np.linalg.norm(want)
    assert rel <= 2 * half + 1e-5, rel
    assert np.linalg.norm(val(m.dx) - wdx) / np.linalg.norm(wdx) <= 4 * half + 1e-5
    # and against the exact activations: off by the checkpoints' steps (int8: half a step is 1/128 of a group's largest
    # value at most, e4m3: 1/16 of each value), which is what the 8 bits cost
    full, _ = m.exact()
    assert np.linalg.norm(host(g) - full) / np.linalg.norm(full) <= (0.06 if fmt else 0.03)
    # the worker's step from the memory: wgrad into e, then select; against the fused step on the written gradient
    e = E()
    lay = e.Layout(d, m.offs, 0.05).bind("cuda")
    mem = dev((1e-3 * np.random.default_rng(12).standard_normal(d)).astype(np.float32))
    other = mem.clone()
    idx, v = torch.empty(lay.K, dtype=torch.int32, device="cuda"), torch.empty(lay.K, device="cuda")
    idx2, v2 = torch.empty_like(idx), torch.empty_like(v)
    wk = lay.workspace(e.EF_OP_TOPK)
    m.step(mem, True)
    e.compress_topk(lay, mem, idx, v, wk)
    e.ef_update(lay, mem, e.EF_MSG_SPARSE, idx, mem)
    e.ef_step_topk(lay, g, other, idx2, v2, wk)
    assert torch.equal(idx, idx2) and torch.equal(v, v2) and np.array_equal(bits(host(mem)), bits(host(other)))


def test_gradient_against_differences():
    """The flat gradient, float32 and int8, against central differences of the loss in float64 at some coordinates."""
    import torch
    m = Mlp(40, 24, 40, "f32", L.GELU, L.INT8, 21)
    g = torch.zeros(m.offs[-1], device="cuda")
    m.step(g, False)
    got = host(g)

    def loss():
        v = m.np
        return float(((v["x"] + L.act(v["x"] @ v["w1"].T + v["b1"], L.GELU) @ v["w2"].T + v["b2"]) * v["t"]).sum())

    rng = np.random.default_rng(22)
    scale = np.linalg.norm(got) / np.sqrt(got.size)
    for l, name in enumerate(("w1", "b1", "w2", "b2")):
        p = m.np[name]
        for k in rng.integers(0, p.size, 6):
            old, hstep = p.flat[k], 1e-4
            p.flat[k] = old + hstep
            up = loss()
            p.flat[k] = old - hstep
            down = loss()
            p.flat[k] = old
            # n = 40 terms, each kept value off by 1/128 of its group's largest at most
            assert abs(got[m.offs[l] + k] - (up - down) / (2 * hstep)) <= 0.25 * scale


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_and_replayed(dtype):
    """The whole pass in a graph, replayed between eager passes on other data: every replay is the eager result."""
    import torch
    m = Mlp(300, 128, 512, dtype, L.GELU, 0, 31)
    other = Mlp(64, 96, 96, dtype, L.SILU, 1, 32)
    d = m.offs[-1]
    g, og = torch.zeros(d, device="cuda"), torch.zeros(other.offs[-1], device="cuda")
    m.step(g, False)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    cg = torch.zeros(d, device="cuda")
    with torch.cuda.graph(graph):
        m.step(cg, False)
    for k in range(4):
        m.p["x"].copy_(m.p["x"] * -0.5)
        g.fill_(3.0), cg.fill_(5.0)
        m.step(g, False)
        dx = m.dx.clone()
        m.dx.zero_()
        other.step(og, True)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(bits(host(g)), bits(host(cg))) and torch.equal(dx, m.dx), k


def test_refusals_on_the_gpu():
    import torch
    e = E()
    x, w, y = (torch.zeros(*s, device="cuda") for s in ((4, 8), (40, 8), (4, 40)))
    q, s = e.ckpt_buffers(4, 40)
    h = torch.float16
    cases = [lambda: e.ef_ckpt_pack(y.half(), q, s), lambda: e.ef_ckpt_pack(y.t(), q, s), lambda: e.ef_ckpt_pack(y, q[:3], s),
             lambda: e.ef_ckpt_pack(y, q, s.to(torch.int8)), lambda: e.ef_ckpt_pack(y, s, q), lambda: e.ef_ckpt_pack(y[0], q, s),
             lambda: e.ef_ckpt_pack(y[:1].expand(4, 40), q, s), lambda: e.ef_ckpt_pack(y, q, s, 5),
             lambda: e.ef_ckpt_pack(y, e.ckpt_buffers(8, 40)[0][::2], s), lambda: e.ef_ckpt_unpack(q, s, 0, y.to(h)),
             lambda: e.ef_ckpt_act_backward(9, q, s, 0, y, y), lambda: e.ef_ckpt_act_backward(1, q, s, 0, y, y.bfloat16()),
             lambda: e.ef_linear_forward(x, w.bfloat16(), y, None), lambda: e.ef_linear_forward(x, w.t(), y, None),
             lambda: e.ef_linear_forward(x, w, y[:3], None), lambda: e.ef_linear_forward(x, w, y, None, bias=torch.zeros(39, device="cuda")),
             lambda: e.ef_linear_forward(x, w, y, None, codes=q), lambda: e.ef_linear_forward(x, w, y, None, scales=s),
             lambda: e.ef_linear_forward(x, w, y, None, res=y.cpu()), lambda: e.ef_linear_forward(x, w, y, torch.zeros(256)),
             lambda: e.ef_linear_dgrad(y, w, x, None, act=e.EF_ACT_RELU), lambda: e.ef_linear_dgrad(y, w, x.bfloat16(), None),
             lambda: e.ef_linear_wgrad(x, q, s, 0, torch.zeros(8, 65, device="cuda"), None),
             lambda: e.ef_linear_wgrad(x, q, s, 0, torch.zeros(40, 8, device="cuda").t(), None),
             lambda: e.ef_linear_wgrad(x, q, s, 0, torch.zeros(8, 40, device="cuda", dtype=torch.bfloat16), None, accumulate=True),
             lambda: e.ef_linear_wgrad(x, q, s, 0, torch.zeros(8, 40, device="cuda"), None, db=torch.zeros(8, device="cuda").bfloat16())]
    for k, call in enumerate(cases):
        with pytest.raises(e.EfError) as ex:
            call()
        assert ex.value.code in (e.EF_EINVAL, e.EF_EWORKSPACE), k
    torch.cuda.synchronize()


def test_refuses_a_short_workspace():
    import torch
    e = E()
    n, i, o = 8192, 256, 128
    dy = torch.zeros(n, o, dtype=torch.bfloat16, device="cuda")
    q, s = e.ckpt_buffers(n, i)
    dw = torch.full((o, i), 3.0, device="cuda")
    need = int(e.lib().ef_linear_workspace_bytes(e.EF_OP_WGRAD, n, i, o, e.EF_BF16))
    if need == 0:
        pytest.skip("needs no workspace")
    for w, code in ((torch.empty(need - 1, dtype=torch.uint8, device="cuda"), e.EF_EWORKSPACE), (None, e.EF_EINVAL),
                    (torch.empty(need + 256, dtype=torch.uint8, device="cuda")[1:], e.EF_EINVAL)):
        with pytest.raises(e.EfError) as ex:
            e.ef_linear_wgrad(dy, q, s, 0, dw, w)
        assert ex.value.code == code
    torch.cuda.synchronize()
    assert bool((dw == 3.0).all())


# ---- large products ------------------------------------------------------------------------------------------------------
def gpu_ints(seed, *shape):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randint(-3, 4, shape, generator=g, device="cuda", dtype=torch.int8)


def strided(x, dtype, ld):
    """x as `dtype` with rows ld apart."""
    import torch
    t = torch.zeros(x.shape[0] * ld, dtype=tt(dtype), device="cuda").view(x.shape[0], ld)[:, :x.shape[1]]
    t.copy_(x)
    return t


def pack_ints(x, fmt):
    """The checkpoint of small whole numbers, which both formats hold exactly."""
    q, s = E().ckpt_buffers(*x.shape)
    E().ef_ckpt_pack(x.float().contiguous(), q, s, fmt)
    return q, s


def mm64(a, b):
    import torch
    return torch.matmul(a.double().contiguous(), b.double().contiguous())


@pytest.mark.parametrize("dtype,n,a,b", [("bf16", 4090, 1032, 4088), ("bf16", 2301, 2056, 2048), ("bf16", 3000, 1001, 999),
                                         ("f32", 1500, 600, 1100), ("bf16", 640, 4096, 8)])
def test_large_products_of_integers(dtype, n, a, b):
    """All three products at sizes of many tiles, each with a ragged edge: bit for bit."""
    import torch
    announce("large ints", dtype, n, a, b)
    e = E()
    t = tt(dtype)
    x, w, r = gpu_ints(1, n, a), gpu_ints(2, b, a), gpu_ints(3, n, b)
    y = torch.empty(n, b, dtype=t, device="cuda")
    e.ef_linear_forward(x.to(t), w.to(t), y, ws(e.EF_OP_FORWARD, n, a, b, dtype), act=L.RELU, res=r.to(t))
    assert torch.equal(y, (mm64(x, w.t()).clamp(min=0) + r).to(t))
    # back: dy [n][a], weight [a][b], the kept input of an activation [n][b]
    dy, wt, z = x, gpu_ints(4, a, b), gpu_ints(5, n, b)
    for fmt in FMTS:
        q, s = pack_ints(z, fmt)
        dx = torch.empty(n, b, dtype=t, device="cuda")
        e.ef_linear_dgrad(dy.to(t), wt.to(t), dx, ws(e.EF_OP_DGRAD, n, b, a, dtype), act=L.RELU, codes=q, scales=s, fmt=fmt, res=r.to(t))
        assert torch.equal(dx, (mm64(dy, wt) * (z > 0) + r).to(t))
    # weights [b][n], their gradient summed over a tokens
    dy, k = gpu_ints(6, a, b), gpu_ints(7, a, n)
    want, wb = mm64(dy.t(), k).float(), dy.double().sum(0).float()
    for fmt in FMTS:
        q, s = pack_ints(k, fmt)
        wk = ws(e.EF_OP_WGRAD, a, n, b, dtype)
        dw, db = torch.full((b, n), 2.0, device="cuda"), torch.full((b,), 2.0, device="cuda")
        e.ef_linear_wgrad(dy.to(t), q, s, fmt, dw, wk, db=db, accumulate=True)
        assert torch.equal(dw, want + 2.0) and torch.equal(db, wb + 2.0)
        h, hb = torch.empty(b, n, dtype=torch.bfloat16, device="cuda"), torch.empty(b, dtype=torch.bfloat16, device="cuda")
        e.ef_linear_wgrad(dy.to(t), q, s, fmt, h, wk, db=hb)
        assert torch.equal(h, want.bfloat16()) and torch.equal(hb, wb.bfloat16())


@pytest.mark.parametrize("ld", [1 << 21, (1 << 21) + 8])
def test_rows_far_apart(ld):
    """Leading dimensions at and past the one up to which a tile's offsets are taken in 32 bits."""
    import torch
    e = E()
    n, i, o = 300, 64, 72
    announce("rows", ld, "apart")
    x, w, dy = gpu_ints(1, n, i), gpu_ints(2, o, i), gpu_ints(3, n, o)
    y, dx = torch.empty(n, o, dtype=torch.bfloat16, device="cuda"), torch.empty(n, i, dtype=torch.bfloat16, device="cuda")
    wide = strided(x, "bf16", ld)
    e.ef_linear_forward(wide, w.bfloat16(), y, ws(e.EF_OP_FORWARD, n, i, o, "bf16"))
    assert torch.equal(y, mm64(x, w.t()).bfloat16())
    q, s = e.ckpt_buffers(n, i)
    e.ef_ckpt_pack(wide, q, s)
    del wide
    wide = strided(w, "bf16", ld)
    e.ef_linear_dgrad(dy.bfloat16(), wide, dx, ws(e.EF_OP_DGRAD, n, i, o, "bf16"))
    assert torch.equal(dx, mm64(dy, w).bfloat16())
    del wide
    wide = strided(dy, "bf16", ld)
    dw = torch.empty(o, i, device="cuda")
    e.ef_linear_wgrad(wide, q, s, L.INT8, dw, ws(e.EF_OP_WGRAD, n, i, o, "bf16"))
    assert torch.equal(dw, mm64(dy.t(), x).float())


def test_products_past_32_bit_offsets():
    import torch
    e = E()
    n, k, m = 40000, 64, 65536
    announce("products of", n, "x", m)
    x, w = gpu_ints(1, n, k), gpu_ints(2, m, k)
    rows = torch.tensor([0, 255, 256, 32767, 32768, n - 1], device="cuda")
    y = torch.empty(n, m, dtype=torch.bfloat16, device="cuda")
    q, s = e.ckpt_buffers(n, m)
    e.ef_linear_forward(x.bfloat16(), w.bfloat16(), y, ws(e.EF_OP_FORWARD, n, k, m, "bf16"), codes=q, scales=s)
    want = mm64(x[rows], w.t())
    assert torch.equal(y[rows], want.bfloat16())
    z = torch.empty(len(rows), m, device="cuda")
    e.ef_ckpt_unpack(q[rows].contiguous(), s[rows].contiguous(), L.INT8, z)
    step = torch.exp2((s[rows].double() - 127).floor()).repeat_interleave(32, 1)
    assert bool(((z.double() - want).abs() <= step / 2).all())
    # back through the activation that these were kept of: dy [n][k], weight [k][m]
    wt = gpu_ints(3, k, m)
    e.ef_linear_dgrad(x.bfloat16(), wt.bfloat16(), y, ws(e.EF_OP_DGRAD, n, m, k, "bf16"), act=L.RELU, codes=q, scales=s)
    assert torch.equal(y[rows], (mm64(x[rows], wt) * (z > 0)).bfloat16())
    del y, q, s
    dy, c = gpu_ints(4, k, n), gpu_ints(5, k, m)
    q, s = pack_ints(c, L.E4M3)
    dw = torch.zeros(n, m, device="cuda")
    e.ef_linear_wgrad(dy.bfloat16(), q, s, L.E4M3, dw, ws(e.EF_OP_WGRAD, k, m, n, "bf16"), accumulate=True)
    assert torch.equal(dw[rows], mm64(dy[:, rows].t(), c).float())


def test_two_streams_at_once_and_twice_the_same():
    """Products that run at the same time in workspaces of their own, and again: bitwise the same."""
    import torch
    e = E()
    n, i, o = 2000, 512, 384
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    dy = torch.randn(n, o, generator=g, device="cuda").bfloat16()
    q, s = e.ckpt_buffers(n, i)
    e.ef_ckpt_pack(torch.randn(n, i, generator=g, device="cuda"), q, s)
    wsp = [ws(e.EF_OP_WGRAD, n, i, o, "bf16") for _ in range(2)]
    dw = [torch.empty(o, i, device="cuda") for _ in range(3)]
    e.ef_linear_wgrad(dy, q, s, 0, dw[2], wsp[0])
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for k in range(2):
            dw[k].fill_(float("nan"))
        torch.cuda.synchronize()
        for k in range(2):
            e.ef_linear_wgrad(dy, q, s, 0, dw[k], wsp[k], stream=side[k])
        torch.cuda.synchronize()
        assert torch.equal(dw[0], dw[2]) and torch.equal(dw[1], dw[2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,i,o", [(1, 4096, 1000), (3, 264, 16), (16, 1032, 40), (17, 8, 4100), (32, 520, 33), (33, 520, 33), (2, 36, 50)])
def test_few_tokens_of_integers_bit_for_bit(n, i, o, dtype):
    import torch
    for k in range(2):  # contiguous rows, padded rows
        announce("few ints", n, i, o, dtype, k)
        rng = np.random.default_rng([n, i, o, k])
        x, w, b, r = ints(rng, n, i), ints(rng, o, i), ints(rng, 1, o)[0], ints(rng, n, o)
        z = x @ w.T + b
        for keep in (False, True):
            y, q, s = forward(x, w, b, r, dtype, L.RELU, keep, k, k)
            assert np.array_equal(val(y), torch.from_numpy(np.maximum(z, 0) + r).to(tt(dtype)).double().numpy())
        wq, wsc = L.ckpt_pack(z, k)
        assert np.array_equal(host(s), wsc)
        neg0 = 0 if k == L.INT8 else 128
        assert np.array_equal(np.where(host(q) == neg0, 0, host(q)), np.where(wq == neg0, 0, wq))


def test_columns_of_one_buffer():
    """Inputs and outputs side by side in the rows of one buffer, as slices of its columns."""
    import torch
    e = E()
    n, i, o = 96, 64, 128
    x, w, r = gpu_ints(1, n, i), gpu_ints(2, o, i), gpu_ints(3, n, o)
    for dtype in ("f32", "bf16"):
        t = tt(dtype)
        buf = torch.zeros(n, i + 2 * o + 8, dtype=t, device="cuda")
        a, y, res = buf[:, :i], buf[:, i:i + o], buf[:, i + o:i + 2 * o]
        a.copy_(x), res.copy_(r)
        wk = ws(e.EF_OP_FORWARD, n, i, o, dtype)
        e.ef_linear_forward(a, w.to(t), y, wk, act=L.RELU, res=res)
        assert torch.equal(y, (mm64(x, w.t()).clamp(min=0) + r).to(t))
        assert torch.equal(a, x.to(t)) and torch.equal(res, r.to(t)) and not buf[:, i + 2 * o:].any()
        with pytest.raises(e.EfError):
            e.ef_linear_forward(a, w.to(t), buf[:, i - 1:i - 1 + o], wk)
        with pytest.raises(e.EfError):
            e.ef_linear_forward(a, w.to(t), y, wk, res=buf[:, i + 1:i + 1 + o])


def test_passes_over_more_rows_than_one_grid_dimension_has():
    """2^32 threads and more: 2^30 rows of one group each."""
    import torch
    e, n = E(), (1 << 30) + 100
    announce("passes over", n, "rows")
    x = torch.arange(n, device="cuda", dtype=torch.int32).remainder_(15).sub_(7).to(torch.bfloat16).unsqueeze(1)
    q, s = e.ckpt_buffers(n, 1)
    e.ef_ckpt_pack(x, q, s)
    y = torch.empty_like(x)
    e.ef_ckpt_unpack(q, s, L.INT8, y)
    assert torch.equal(x, y)
    e.ef_ckpt_act_backward(L.RELU, q, s, L.INT8, x, y)
    assert torch.equal(x.clamp_(min=0), y)

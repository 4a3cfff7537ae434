"""Checkpoints at the top of the range, without a GPU: hand-worked groups whose values would round to 2^128."""

import numpy as np
import pytest

from oracle import linear_oracle as L

MOST = {"f32": float(np.finfo(np.float32).max), "bf16": float.fromhex("0x1.FEp127")}


@pytest.mark.parametrize("kind", sorted(MOST))
def test_hand_worked_groups(kind):
    x = np.zeros((4, 32))
    x[0, :4] = [MOST[kind], -MOST[kind], 2.0 ** 127, 1.4 * 2.0 ** 122]
    x[1, :3] = [127.0 * 2.0 ** 121, -(127.0 * 2.0 ** 121), 2.0 ** 120]    # int8: fits under 2^121
    x[2, :3] = [127.5 * 2.0 ** 121, 126.0 * 2.0 ** 121, 2.0 ** 122]       # int8: rounds to 128 there, to 63.75 under 2^122
    x[3, :3] = [248.0 * 2.0 ** 120, 240.0 * 2.0 ** 120, -447.0 * 2.0 ** 119]
    q, s = L.ckpt_pack(x, L.INT8)
    assert s[:, 0].tolist() == [249, 248, 249, 248]
    assert q[0, :4].view(np.int8).tolist() == [63, -63, 32, 1]
    assert q[1, :3].view(np.int8).tolist() == [127, -127, 0]  # 2^120 is half a step: to the even code
    assert q[2, :3].view(np.int8).tolist() == [63, 63, 1]
    assert q[3, :3].view(np.int8).tolist() == [124, 120, -112]
    q, s = L.ckpt_pack(x, L.E4M3)
    assert s[:, 0].tolist() == [247, 247, 247, 247]
    assert q[0, :3].tolist() == [0x77, 0xF7, 0x70]            # 240, -240, 128
    assert q[3, :3].tolist() == [0x77, 0x77, 0xF6]            # 240, 240, -224 (223.5)


@pytest.mark.parametrize("fmt", [L.INT8, L.E4M3])
@pytest.mark.parametrize("kind", sorted(MOST))
def test_finite_values_come_back_finite(kind, fmt):
    g = np.random.default_rng(4)
    x = MOST[kind] * (1 - g.random((64, 96)) * 2.0 ** -g.integers(0, 8, (64, 96))) * g.choice([-1, 1], (64, 96))
    x = x.astype(np.float32).astype(np.float64)
    q, s = L.ckpt_pack(x, fmt)
    y = L.ckpt_unpack(q, s, fmt, 96)
    assert np.isfinite(y.astype(np.float32)).all()
    # less than a step: 2^e for int8; e4m3 has 16 of them between its two highest finite values
    step = np.repeat(np.ldexp(1.0 if fmt == L.INT8 else 16.0, s.astype(int) - 127), 32, axis=1)
    assert (np.abs(y - x) < np.maximum(step, np.abs(x) * 2.0 ** -4 if fmt else 0)).all()

"""Pins of the 8-bit oracle (oracle/quant_oracle.py) against torch's e4m3 type,
closed forms and brute force, CPU only."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as Q


def test_table_is_e4m3():
    codes = torch.arange(256, dtype=torch.int16).to(torch.uint8)
    v = codes.view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(Q.decode(codes.numpy()), v)
    assert Q.TABLE[-1] == 448.0 and np.all(np.diff(Q.TABLE) > 0)


def test_encode_matches_torch_and_brute_force():
    g = np.random.default_rng(0)
    mid = (Q.TABLE[1:] + Q.TABLE[:-1]) / 2
    v = np.concatenate([g.normal(size=4000) * np.exp2(g.integers(-12, 8, 4000)), Q.TABLE, mid,
                        np.nextafter(mid, 0), np.nextafter(mid, 1000)])
    v = np.clip(np.concatenate([v, -v]), -448, 448).astype(np.float32).astype(np.float64)
    want = torch.from_numpy(v.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(Q.encode(v), want)
    d = np.abs(Q.decode(Q.encode(v)) - v)
    assert np.all(d <= np.abs(np.abs(v)[:, None] - Q.TABLE[None]).min(1))
    np.testing.assert_array_equal(Q.encode([np.nan, np.inf, -np.inf]), [0x7F] * 3)


@pytest.mark.parametrize("top,byte", [
    (0.0, 0), (448.0, 127), (np.nextafter(448.0, 500), 128), (224.0, 126), (1.0, 119),
    (1.75, 119), (1.7500001, 120), (2.0 ** -149, 0), (448 * 2.0 ** -127, 0),
    (449 * 2.0 ** -127, 1), (float(np.finfo(np.float32).max), 247)])
def test_scale_is_the_smallest_that_holds_the_top(top, byte):
    assert int(Q.scale_byte(np.array(top))) == byte
    if top > 0:
        assert top <= 448 * 2.0 ** (byte - 127)
        assert byte == 0 or top > 448 * 2.0 ** (byte - 128)


def test_rows_and_matrices():
    g = np.random.default_rng(1)
    x = g.normal(size=(5, 300)) * np.exp(g.normal(size=(5, 1)) * 3)
    q, s = Q.quant_rows(x)
    assert q.shape == (5, 384) and s.shape == (5, 3) and not q[:, 300:].any()
    v = Q.row_values(q, s, 300)
    # half a step of three mantissa bits, or of the subnormals
    two = np.repeat(2.0 ** (s.astype(float) - 127), 128, 1)[:, :300]
    assert np.all(np.abs(v - x) <= np.maximum(np.abs(x) * 2.0 ** -4, two * 2.0 ** -10))
    # a power of two in front of everything moves the scales only
    q2, s2 = Q.quant_rows(x * 2.0 ** 5)
    np.testing.assert_array_equal(q, q2)
    np.testing.assert_array_equal(s + 5, s2)
    W = g.normal(size=(130, 200))
    qm, sm = Q.quant_matrix(W)
    assert qm.shape == (130, 256) and sm.shape == (2, 2)
    # the block of two rows has the scale of its own largest magnitude
    assert sm[1, 0] == Q.scale_byte(np.abs(W[128:, :128]).max())
    assert np.all(np.abs(Q.matrix_values(qm, sm, 200) - W) <= np.abs(W) * 2.0 ** -4 + 2.0 ** -15)


def test_neighbours_hold_what_lies_between():
    g = np.random.default_rng(2)
    x = g.normal(size=(20, 140))
    r = 10.0 ** g.uniform(-8, -1, x.shape)
    lo, hi = Q.neighbours(x - r, x + r)
    for _ in range(20):
        v = Q.round_trip(x + r * g.uniform(-1, 1, x.shape))
        assert np.all(v >= lo) and np.all(v <= hi)

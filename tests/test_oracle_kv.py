"""Pins of the KV oracle (oracle/kv.py): closed forms and hand-worked rows."""
import math

import numpy as np
import pytest

from oracle import kv as O


def test_frequencies_of_each_scaling():
    f = O.frequencies(8, base=16.0)
    assert np.allclose(f, [1, 0.5, 0.25, 0.125], rtol=1e-15)
    assert np.allclose(O.frequencies(8, base=16.0, scaling="linear", factor=4), f / 4, rtol=1e-15)
    # the slowest pair of the stretched base turns `factor` times slower, the fastest as before
    g = O.frequencies(8, base=16.0, scaling="ntk", factor=4)
    assert math.isclose(g[0], f[0]) and math.isclose(g[-1], f[-1] / 4)
    # 8 turns in 16 pi positions for f = 1: at `high` = 8 kept, at `low` = 1 (f = 1/8) divided, half way between blended
    n = 50  # turns = 50 f / 2 pi = 7.96, 3.98, 1.99, 0.99
    g = O.frequencies(8, base=16.0, scaling="turns", factor=4, low=1.0, high=4.0, original_len=n)
    u = (n * 0.25 / (2 * math.pi) - 1) / 3
    assert math.isclose(g[0], 1) and math.isclose(g[3], 0.125 / 4) and math.isclose(g[2], (1 - u) * 0.25 / 4 + u * 0.25)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_complex_product(interleaved):
    rng = np.random.default_rng(1)
    x = rng.normal(size=(3, 2, 10))
    cs = O.angles(O.frequencies(6), [0, 1, 7])
    y = O.rotate(x, cs, interleaved)
    assert (y[0] == x[0]).all() and (y[..., 6:] == x[..., 6:]).all()
    a, b = (x[..., 0:6:2], x[..., 1:6:2]) if interleaved else (x[..., :3], x[..., 3:6])
    z = (a + 1j * b) * (cs[:, None, :, 0] + 1j * cs[:, None, :, 1])
    c, d = (y[..., 0:6:2], y[..., 1:6:2]) if interleaved else (y[..., :3], y[..., 3:6])
    assert np.allclose(c, z.real, atol=1e-14) and np.allclose(d, z.imag, atol=1e-14)
    assert np.allclose(O.rotate(y, cs, interleaved, inverse=True), x, atol=1e-14)


def test_hand_worked_rows():
    c, s, m = O.chosen(np.array([[-1.0, 14.0, 6.4, 6.5, 7.5], [3.0, 3.0, 3.0, 3.0, 3.0], [0.0, 1.0, np.inf, 0.0, 0.0], [0, np.nan, 0, 0, 0]]))
    assert s[0] == 1 and m[0] == -1 and c[0].tolist() == [0, 15, 7, 8, 8]  # 7.4 -> 7, the ties 7.5 -> 8 and 8.5 -> 8
    assert s[1] == 0 and m[1] == 3 and c[1].tolist() == [0] * 5
    assert np.isnan(s[2:]).all() and np.isnan(m[2:]).all() and (c[2:] == 0).all()
    assert O.to_bf16(np.float32(1 + 2 ** -8)) == 1 and O.to_bf16(np.float32(1 + 3 * 2 ** -8)) == 1 + 2 ** -6  # ties to even


@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_page_holds_each_code_once(d):
    seen = {O.value_nibble(t, c, d) for t in range(32) for c in range(d)}
    assert seen == {(b, n) for b in range(16 * d) for n in (0, 1)}
    pages = np.random.default_rng(0).integers(0, 256, (2, 2 * 32 * (d + 8)), dtype=np.uint8)
    o = O.KvOracle(pages, 2, d, 32)
    rng = np.random.default_rng(1)
    rows = {(t, v): O.chosen(rng.normal(size=(1, d))) for t in (0, 5, 31) for v in (0, 1)}
    for (t, v), (c, s, m) in rows.items():
        o.write(1, t, 1, v, c[0], s[0], m[0])
    for (t, v), (c, s, m) in rows.items():
        assert (o.row(1, t, 1, v) == m[0] + s[0] * c[0]).all()


def test_attention_of_equal_keys_is_a_mean_and_of_none_is_zero():
    v = np.arange(6.0).reshape(3, 1, 2)
    out, _, _ = O.attend(np.ones((2, 2, 2)), np.ones((3, 1, 2)), v, 0.5, [0, 2], causal=True)
    assert out[0].tolist() == [[0, 1]] * 2 and np.allclose(out[1], [[2, 3]] * 2)
    out, _, _ = O.attend(np.ones((1, 1, 2)), np.ones((3, 1, 2)), v, 0.5, [2], window=2)
    assert np.allclose(out, [[[3, 4]]])
    out, _, _ = O.attend(np.ones((1, 1, 2)), np.ones((3, 1, 2)), v, 0.5, [-1])
    assert (out == 0).all()
    out, _, _ = O.attend(np.ones((1, 1, 2)), np.ones((3, 1, 2)), v, 0.5, [2], holes=[0, 1])
    assert (out == v[2]).all()

"""The oracle of the base layer's operators against torch's own types and against hand-made values."""
import numpy as np
import torch

from oracle import base as O


def test_codes_are_torchs():
    x = np.concatenate([np.random.default_rng(0).normal(size=20000) * np.float32(90), O._MIDDLE, -O._MIDDLE, O.e4m3_table(), [0.0, -0.0, 448.00003, 2.0 ** -10]])
    x = np.clip(x, -448.00003, 448.00003).astype(np.float32)
    t = torch.from_numpy(x).to(torch.float8_e4m3fn)
    assert (O.to_codes(x) == t.view(torch.uint8).numpy()).all()
    assert (O.values(O.to_codes(x)) == t.double().numpy()).all()


def test_rows_and_weights_by_hand():
    x = np.zeros((3, 136), np.float32)
    x[0, :3] = [448, -1, 2.0 ** -10]  # scale 1; a tie between 0 and the smallest code: even
    x[1, 130] = 7.0
    x[2, 5] = np.inf
    c, s = O.rows(x)
    assert s.shape == (2, 3) and s[0, 0] == 1 and s[1, 0] == 0 and s[1, 1] == np.float32(7) / np.float32(448) and np.isnan(s[0, 2]) and s[1, 2] == 0
    assert O.values(c)[0, 0] == 448 and O.values(c)[0, 1] == -1 and O.values(c)[0, 2] == 0 and O.values(c)[1, 130] == 448 and not c[2].any()
    assert abs(O.row_values(c, s)[1, 130] - 7) < 1e-6
    w = np.random.default_rng(1).normal(size=(136, 144)).astype(np.float32)
    c, s = O.weights(w)
    assert s.shape == (2, 2) and np.abs(O.weight_values(c, s) - w).max() <= 2.0 ** -4 * np.abs(w).max()
    assert s[1, 1] == np.abs(w[128:, 128:]).max() / np.float32(448)


def test_route_by_hand():
    x = np.array([[1, 3, 3, 0], [-np.inf] * 4, [5, -np.inf, np.nan, 5]], np.float32)
    e, w, o, r, p = O.route(x, 3)
    assert e.tolist() == [[1, 2, 0], [-1] * 3, [0, 3, -1]] and o.tolist() == [0, 2, 3, 4, 5]
    assert r.tolist() == [0, 2, 0, 0, 2, -1, -1, -1, -1] and p.tolist() == [[2, 3, 0], [-1] * 3, [1, 4, -1]]
    assert abs(w[0].sum() - 1) < 1e-12 and (w[1] == 0).all() and np.isnan(w[2]).all()
    _, v, _, _, _ = O.route(x[:1], 2, renormalise=False, scale=2.0)
    assert np.allclose(v[0], 2 * np.exp([3, 3]) / np.exp([1, 3, 3, 0]).sum())


def test_activations_and_norms_are_torchs():
    x = np.random.default_rng(2).normal(size=(5, 48)) * 4
    a, b = torch.from_numpy(x).chunk(2, 1)
    assert np.allclose(O.activated(x, "silu"), (torch.nn.functional.silu(a) * b).numpy())
    assert np.allclose(O.activated(x, "gelu"), (torch.nn.functional.gelu(a, approximate="tanh") * b).numpy())
    g, c = np.linspace(.5, 2, 48), np.linspace(-1, 1, 48)
    t = torch.from_numpy
    assert np.allclose(O.norm(x, g, c, 1e-5, True), torch.nn.functional.layer_norm(t(x), (48,), t(g), t(c), 1e-5).numpy())
    assert np.allclose(O.norm(x, g, offset=1.0, eps=1e-5), torch.nn.functional.rms_norm(t(x), (48,), t(1 + g), 1e-5).numpy())
    assert np.allclose(O.gathered(x, [[4, -1], [0, 5]], [[.5, np.nan], [2., 1.]]), [x[4] * .5, x[0] * 2])

"""Pins of the 8-bit rows' oracle: the code table, rounding against exact
neighbours, the norm's gradient against differences."""
import numpy as np
import pytest

from oracle import eight_bits as E


def test_codes_against_torch():
    torch = pytest.importorskip("torch")
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(t), np.isnan(E.E4M3))
    assert np.array_equal(t[~np.isnan(t)], E.E4M3[~np.isnan(E.E4M3)])
    g = np.random.default_rng(0)
    x = np.concatenate([g.normal(size=4000) * 10.0 ** g.uniform(-4, 2, 4000), E.E4M3[:127], (E.E4M3[:126] + E.E4M3[1:127]) / 2])
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    unit = np.full((1, E.scale_cols(len(x))), 127, np.uint8)
    assert np.array_equal(E.codes(x[None], unit)[0], want)


def test_the_scale_is_the_smallest_that_holds_the_group():
    g = np.random.default_rng(1)
    x = g.normal(size=(50, 300)) * 2.0 ** g.integers(-100, 100, (50, 1))
    s = E.scale_bytes(x).astype(int)
    assert s.shape == (50, 4) and (s[:, 3] == 127).all()
    for q in range(3):
        top = np.abs(x[:, 128 * q:128 * q + 128]).max(axis=1)
        assert (top <= 448 * 2.0 ** (s[:, q] - 127)).all() and (top > 448 * 2.0 ** (s[:, q] - 128)).all()
    edge = np.array([[448.0], [np.nextafter(448.0, 500)], [0.0], [np.inf], [2.0 ** -149], [3.4e38]])
    assert E.scale_bytes(edge)[:, 0].tolist() == [127, 128, 0, 0, 0, 247]


def test_quantised_rows_are_within_half_a_step():
    g = np.random.default_rng(2)
    x = g.normal(size=(20, 1031))
    q, s = E.quant(x)
    step = E.spread(s, 1031)
    assert (np.abs(E.values(q, s) - x) <= np.maximum(np.abs(x) * 2.0 ** -4, step * 2.0 ** -10)).all()
    x[3, 5], x[4, 200] = np.nan, -np.inf
    q, t = E.quant(x)
    assert q[3, 5] & 127 == 127 and q[4, 200] & 127 == 127 and np.array_equal(s[:, 2:], t[:, 2:])


def test_norm_gradient_against_differences():
    g = np.random.default_rng(3)
    h, gamma, dy, dh = g.normal(size=(3, 17)), g.normal(size=17), g.normal(size=(3, 17)), g.normal(size=(3, 17))
    _, rstd = E.rms_forward(h, gamma, 1e-3)
    dx, dgamma = E.rms_backward(dy, h, gamma, rstd, dh)

    def loss(hh, gg):
        return (E.rms_forward(hh, gg, 1e-3)[0] * dy).sum() + (hh * dh).sum()

    for at in [(0, 0), (1, 7), (2, 16)]:
        d = np.zeros_like(h)
        d[at] = 1e-6
        assert abs((loss(h + d, gamma) - loss(h - d, gamma)) / 2e-6 - dx[at]) < 1e-7
    for n in (0, 9):
        d = np.zeros(17)
        d[n] = 1e-6
        assert abs((loss(h, gamma + d) - loss(h, gamma - d)) / 2e-6 - dgamma[n]) < 1e-7


def test_products_are_of_the_values():
    g = np.random.default_rng(4)
    a, w, dy = g.normal(size=(5, 272)), g.normal(size=(7, 272)), g.normal(size=(5, 7))
    (qa, sa), (qw, sw) = E.quant(a), E.quant(w)
    want = np.zeros((5, 7))
    for m in range(5):
        for n in range(7):
            for k in range(272):
                want[m, n] += E.E4M3[qa[m, k]] * 2.0 ** (int(sa[m, k // 128]) - 127) * E.E4M3[qw[n, k]] * 2.0 ** (int(sw[n, k // 128]) - 127)
    assert np.allclose(E.product(qa, sa, qw, sw), want, rtol=1e-12, atol=1e-12)
    assert np.allclose(E.weight_grad(dy, qa, sa), dy.T @ E.values(qa, sa))
    assert np.abs(want - a @ w.T).max() < 2 * 2.0 ** -4 * (np.abs(a) @ np.abs(w).T).max()

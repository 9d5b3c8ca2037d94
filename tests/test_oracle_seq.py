"""The fp64 forms of oracle/seq.py against differences, complex arithmetic, torch's conversions and hand values."""
import numpy as np
import pytest
import torch

from oracle import seq as O


def _differences(f, x, d=1e-6):
    g = np.zeros_like(x)
    for at in np.ndindex(x.shape):
        keep = x[at]
        x[at] = keep + d
        up = f()
        x[at] = keep - d
        g[at] = (up - f()) / (2 * d)
        x[at] = keep
    return g


def test_norm_gradients_are_the_differences():
    rng = np.random.default_rng(1)
    x, res, dy, ds = (rng.standard_normal((3, 5)) for _ in range(4))
    w = rng.standard_normal(5)

    def loss():
        y, s, _, _ = O.rms_norm(x, w, res)
        return (y * dy).sum() + (s * ds).sum()

    _, s, rstd, _ = O.rms_norm(x, w, res)
    dx, dw, _, _ = O.rms_norm_bwd(dy, s, w, rstd, ds)
    for t, g in ((x, dx), (res, dx), (w, dw)):
        np.testing.assert_allclose(_differences(loss, t), g, rtol=1e-6, atol=1e-7)


@pytest.mark.parametrize("lengths", [None, [0, 4], [2, 1]])
@pytest.mark.parametrize("with_h0", [False, True])
def test_scan_gradients_are_the_differences(lengths, with_h0):
    rng = np.random.default_rng(2)
    x, r, i, dh = (rng.standard_normal((2, 4, 3)) for _ in range(4))
    lam, h0, dl = rng.standard_normal(3), rng.standard_normal((2, 3)) * with_h0, rng.standard_normal((2, 3))
    n = None if lengths is None else np.array(lengths)

    def loss():
        h, last, _, _ = O.gated_scan(x, r, i, lam, h0, n)
        return (h * dh).sum() + (last * dl).sum()

    grads, _ = O.gated_scan_bwd(x, r, i, lam, h0, n, dh, dl)
    for t, g in zip((x, r, i, lam, h0), grads):
        np.testing.assert_allclose(_differences(loss, t), g, rtol=2e-6, atol=2e-8)


def test_scan_of_one_token_by_hand():
    # softplus(0) = ln 2, sigmoid(0) = 1/2: a = 2^-4, m = sqrt(1 - 2^-8)
    h, last, _, _ = O.gated_scan(np.array([[[3.0]]]), np.zeros((1, 1, 1)), np.zeros((1, 1, 1)), np.zeros(1),
                                 np.array([[16.0]]))
    want = 1.0 + np.sqrt(1 - 2.0 ** -8) * 0.5 * 3.0
    assert abs(h[0, 0, 0] - want) < 1e-14 and abs(last[0, 0] - want) < 1e-14


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_is_a_complex_product(interleaved):
    rng = np.random.default_rng(3)
    x = rng.standard_normal((2, 3, 2, 10))
    f = np.array([0.7, 0.01, 3.0])
    pos = rng.integers(-50, 50, (2, 3))
    y, _ = O.rotary(x, f, pos, interleaved, 1.5)
    turn = 1.5 * np.exp(1j * pos[..., None] * f)[:, :, None]
    a, b = (x[..., 0:6:2], x[..., 1:6:2]) if interleaved else (x[..., :3], x[..., 3:6])
    z = (a + 1j * b) * turn
    ya, yb = (y[..., 0:6:2], y[..., 1:6:2]) if interleaved else (y[..., :3], y[..., 3:6])
    np.testing.assert_allclose(ya, z.real, atol=1e-13)
    np.testing.assert_allclose(yb, z.imag, atol=1e-13)
    assert (y[..., 6:] == x[..., 6:]).all()
    back, _ = O.rotary(y, f, pos, interleaved, 1 / 1.5, True)
    np.testing.assert_allclose(back, x, atol=1e-13)


def test_rotary_two_axes_is_the_layers_rotation():
    import oracle
    rng = np.random.default_rng(4)
    H, W = 3, 5
    x = rng.standard_normal((1, H * W, 2, 64))
    f = 10000.0 ** (-2 * np.arange(16) / 32)
    pos = np.stack(np.divmod(np.arange(H * W), W), -1)[None]
    y, _ = O.rotary(x, np.concatenate([f, f]), pos, True)
    np.testing.assert_allclose(y, oracle.apply_rope(x, H, W), atol=1e-12)


def test_e4m3_rounding_is_torchs():
    v = np.concatenate([np.linspace(-448, 448, 20001), np.linspace(-0.1, 0.1, 20001)]).astype(np.float32)
    want = torch.tensor(v).to(torch.float8_e4m3fn).double().numpy()
    assert (O.e4m3(v.astype(np.float64)) == want).all()


def test_quantize_scales_and_zero_groups():
    y = np.zeros((2, 40))
    y[0, 3], y[0, 39], y[1, 0] = -448.0, 7.0, 1.0
    q, s = O.quantize(y, 32)
    assert s.shape == (2, 2) and s[0, 0] == 1.0 and s[0, 1] == 7 / 448 and s[1, 1] == 1.0
    assert q[0, 3] == -448 and q[0, 39] == 448 and q[1, 0] == 448 and np.count_nonzero(q) == 3

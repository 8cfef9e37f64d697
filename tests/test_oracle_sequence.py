"""Pins of the sequence operators' oracle: its gradients against differences
of its own forward passes, its 8-bit values against torch's, its draws against
the definition's frequencies."""
import numpy as np
import pytest

from oracle import sequence as seq


def _differences(f, x, eps=1e-6):
    """d f / d x for a scalar f, by central differences in place."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        keep = x[i]
        x[i] = keep + eps
        hi = f()
        x[i] = keep - eps
        lo = f()
        x[i] = keep
        g[i] = (hi - lo) / (2 * eps)
    return g


def _tol(size):
    """size: the sum of the loss's terms' absolute values.  A difference of two losses that each carry a rounding error
    of up to 8 2^-53 size (a chain of a few products and sums), over 2 eps = 2e-6, is off by 8 2^-53 size / 1e-6 =
    8.9e-10 size; the curvature's share, eps^2 / 6 times the third derivative, is 1e-12 / 6 times a few hundred size."""
    return dict(rtol=1e-6, atol=1e-7 + 1e-9 * size)


@pytest.mark.parametrize("lengths", [None, [3, 0, 1]])
@pytest.mark.parametrize("act", [True, False])
def test_conv_gradients(lengths, act):
    r = np.random.default_rng(3)
    B, T, C, K = 3, 5, 2, 4
    x, w, bias, state = r.normal(size=(B, T, C)), r.normal(size=(C, K)), r.normal(size=C), r.normal(size=(B, K - 1, C))
    dy, ds = r.normal(size=(B, T, C)), r.normal(size=(B, K - 1, C))

    def loss():
        o = seq.conv(x, w, bias, lengths, state, act)
        return (o["y"] * dy).sum() + (o["state_out"] * ds).sum()

    o = seq.conv(x, w, bias, lengths, state, act, dy, ds)
    tol = _tol(np.abs(o["y"] * dy).sum() + np.abs(o["state_out"] * ds).sum())
    for name, v in (("dx", x), ("dw", w), ("dbias", bias), ("dstate", state)):
        np.testing.assert_allclose(o[name], _differences(loss, v), **tol)


@pytest.mark.parametrize("lengths", [None, [4, 0, 1]])
@pytest.mark.parametrize("gate,plus", [(True, True), (False, False), (False, True)])
def test_scan_gradients(lengths, gate, plus):
    r = np.random.default_rng(4)
    B, T, C, N, G = 3, 5, 4, 3, 2
    v = {"u": r.normal(size=(B, T, C)), "delta": r.normal(size=(B, T, C)), "A": -r.uniform(0.5, 2, size=(C, N)),
         "Bm": r.normal(size=(B, T, G, N)), "Cm": r.normal(size=(B, T, G, N)), "D": r.normal(size=C),
         "z": r.normal(size=(B, T, C)) if gate else None, "delta_bias": r.normal(size=C), "h0": r.normal(size=(B, C, N))}
    dy, dhT = r.normal(size=(B, T, C)), r.normal(size=(B, C, N))

    def loss():
        o = seq.scan(**v, lengths=lengths, plus=plus)
        return (o["y"] * dy).sum() + (o["hT"] * dhT).sum()

    o = seq.scan(**v, lengths=lengths, plus=plus, dy=dy, dhT=dhT)
    tol = _tol(np.abs(o["y"] * dy).sum() + np.abs(o["hT"] * dhT).sum())
    for name, of in (("du", "u"), ("ddelta", "delta"), ("dA", "A"), ("dB", "Bm"), ("dC", "Cm"), ("dD", "D"),
                     ("dz", "z"), ("ddelta_bias", "delta_bias"), ("dh0", "h0")):
        if v[of] is not None:
            np.testing.assert_allclose(o[name], _differences(loss, v[of]), **tol)


def test_absolute_bounds_the_values():
    r = np.random.default_rng(5)
    B, T, C, N, G = 2, 6, 4, 3, 2
    args = dict(u=r.normal(size=(B, T, C)), delta=r.normal(size=(B, T, C)), A=-r.uniform(0.5, 2, size=(C, N)),
                Bm=r.normal(size=(B, T, G, N)), Cm=r.normal(size=(B, T, G, N)), D=r.normal(size=C),
                z=r.normal(size=(B, T, C)), h0=r.normal(size=(B, C, N)), dy=r.normal(size=(B, T, C)))
    o, s = seq.scan(**args), seq.scan(**args, absolute=True)
    for k in o:
        assert (np.abs(o[k]) <= s[k] * (1 + 1e-12)).all(), k


def test_pack_is_the_nearest_e4m3():
    import torch
    r = np.random.default_rng(6)
    x = (r.normal(size=(2, 3, 200)) * np.exp(4 * r.normal(size=200))).astype(np.float32)
    x[0, 0, :128] = 0.0
    x[0, 1, 5], x[0, 1, 6], x[1, 2, 130] = np.inf, np.nan, -np.inf
    x[1, 0, :128] = 448.0 * 2.0 ** -3 * np.sign(x[1, 0, :128])       # the largest value of a scale exactly
    x[1, 1, :3] = [1e-45, -1e-40, 1e-38]
    q, scale = seq.pack(x)
    assert scale[0, 0, 0] == 1.0 and scale[1, 0, 0] == 2.0 ** -3
    assert q[0, 1, 5] & 0x7F == 0x7F and q[0, 1, 6] & 0x7F == 0x7F
    fine = np.isfinite(x)
    full = np.repeat(scale, 128, axis=2)[:, :, :200]
    want = torch.from_numpy((x / full).astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(q[fine], want[fine])
    v = seq.unpack(q, scale)
    # half a step of three mantissa bits, 2^-4 of the value, and half the smallest step below 2^-6 of the scale
    assert (np.abs(v - x)[fine] <= np.maximum(np.abs(x) * 2.0 ** -4, full * 2.0 ** -10)[fine]).all()


def test_sample_by_the_definition():
    z = np.array([0.0, 2.0, 2.0, -np.inf, 1.0, np.nan])
    assert seq.sample(z, 0.0, temperature=0.0)[0] == 1
    assert seq.sample(z, 0.0, top_k=1)[2] == [1]
    assert seq.sample(z, 0.9, top_k=2)[0] == 2
    assert seq.sample(z, 0.5, min_p=np.exp(-1.0) * 0.999)[2] == [1, 2, 4]
    assert seq.sample(z, 0.5, top_p=0.0)[2] == [1]
    assert seq.sample(np.array([np.nan, -np.inf]), 0.5)[0] == -1
    assert seq.sample(np.array([1.0, np.inf, 3.0, np.inf]), 0.7)[0] == 3
    p = np.exp(z[[0, 1, 2, 4]])
    p /= p.sum()
    u = (np.arange(20000) + 0.5) / 20000
    n = np.bincount([seq.sample(z, v)[0] for v in u], minlength=6)[[0, 1, 2, 4]]
    assert np.abs(n / 20000 - p).max() < 1e-4                        # a border moves a share by at most a grid step

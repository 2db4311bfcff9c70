"""The layers' gradients against differences of the layer itself, with a tolerance for each entry.

loss = sum(c act(x w^T + b + r)), r placing z on the values of its checkpoint.  A central difference of step h in one entry is off by
  h^2 / 6 of the third derivative: |act'''| <= 1, times what the entry moves z by, cubed, over the outputs it moves;
  the outputs' own errors over h, (K + 19) 2^-24 of an output's sum of magnitudes and 1e-6 |z| + 1e-7 of the activation, over those outputs;
  the distance of z from its checkpoint, the first of these errors, times |act''| <= 1 and what the entry moves z by.
The slope's own error, 4e-6 of dy, and the gradient's sums, (n + 16) 2^-24 of their magnitudes, are below a hundredth of that.
"""
import numpy as np
import pytest

from tests.test_dense import act64, pack64, slope64, to64, values64

SMOOTH = ["silu", "gelu", "gelu_tanh"]
M, N, K = 4, 12, 8
H = 2.0 ** -4


def _inputs(seed=9):
    """x (on its checkpoint's values), w, b, c in fp32's values, as 64-bit arrays, and the checkpoint of x."""
    rng = np.random.default_rng(seed)
    draw = lambda *shape: rng.standard_normal(shape).astype(np.float32).astype(np.float64)
    q, e = pack64(draw(M, K), "float32")
    return values64(q, e), 0.5 * draw(N, K), draw(N), draw(M, N), (q, e)


def _differences(t, loss):
    """Central differences of loss() in each entry of t, which is changed in place and put back."""
    out = np.zeros(t.shape)
    for i in np.ndindex(*t.shape):
        keep = t[i]
        up = np.float64(np.float32(keep + H))
        down = np.float64(np.float32(keep - H))
        t[i] = up
        high = loss()
        t[i] = down
        low = loss()
        t[i] = keep
        out[i] = (high - low) / (up - down)
    return out


def _tolerances(x, w, b, r, c, z):
    a, total = np.abs(c), np.abs(x) @ np.abs(w).T + np.abs(b) + np.abs(r) + H * 4       # (a step moves z by no more than 4 H)
    off_z = (K + 19) * 2.0 ** -24 * total
    off_y = a * (1.13 * off_z + 1e-6 * (np.abs(z) + 4 * H) + 1e-7)
    third = a * H * H / 6
    return {"dx": third @ np.abs(w) ** 3 + (off_y.sum(1) / H)[:, None] + (a * off_z) @ np.abs(w),
            "dw": third.T @ np.abs(x) ** 3 + (off_y.sum(0) / H)[:, None] + (a * off_z).T @ np.abs(x),
            "db": third.sum(0) + off_y.sum(0) / H + (a * off_z).sum(0),
            "dz": third + off_y / H + a * off_z}


def _gradients(x, w, c, slope):
    dz = c * slope
    return {"dx": dz @ w, "dw": dz.T @ x, "db": dz.sum(0), "dz": dz}


def _first_term(z, act):
    """The slope without the term that comes from the activation's second factor."""
    from scipy.special import expit, ndtr
    return {"silu": expit(z), "gelu": ndtr(z), "gelu_tanh": expit(2 * np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3))}[act]


@pytest.mark.parametrize("act", SMOOTH)
def test_derivatives_are_within_their_bounds(act):
    z, d = np.linspace(-20, 20, 400001), 1e-3
    assert np.abs(slope64(z + d, act) - slope64(z - d, act)).max() / (2 * d) <= 1
    assert np.abs(slope64(z + d, act) - 2 * slope64(z, act) + slope64(z - d, act)).max() / d ** 2 <= 1


@pytest.mark.parametrize("act", SMOOTH)
def test_tolerances_let_the_formula_through_and_nothing_else(act):
    """In 64 bits: the formula's gradients pass; those of a slope that lacks a term, is twice as large or zero fail in each of the four, in
    most of their entries."""
    x, w, b, c, _ = _inputs()
    z = values64(*pack64(x @ w.T + b, "float32"))
    r = z - (x @ w.T + b)
    loss = lambda: float((c * act64(x @ w.T + b + r, act)).sum())
    tolerance = _tolerances(x, w, b, r, c, z)
    right, wrong = _gradients(x, w, c, slope64(z, act)), _gradients(x, w, c, _first_term(z, act))
    for name, t in (("dx", x), ("dw", w), ("db", b), ("dz", r)):
        seen = _differences(t, loss)
        assert np.all(np.abs(seen - right[name]) <= tolerance[name]), name
        for bad in (wrong[name], 2 * right[name], 0 * right[name]):
            assert np.mean(np.abs(seen - bad) > tolerance[name]) > 0.75, name


@pytest.mark.gpu
@pytest.mark.parametrize("act", SMOOTH)
def test_gradients_against_differences_entry_by_entry(act):
    import torch
    from paper_2012_15667_amd import binding as B
    x, w, b, c, (q, e) = _inputs()
    up = lambda t: torch.from_numpy(t.astype(np.float32)).cuda()
    x8 = B.Checkpoint(torch.from_numpy(q).cuda(), torch.from_numpy(e).cuda())
    _, z8 = B.linear(up(x), up(w), up(b), act=act, checkpoint=True)
    z = to64(B.checkpoint_unpack(z8))
    r = (z - to64(B.linear(up(x), up(w), up(b)))).astype(np.float32).astype(np.float64)
    loss = lambda: float((c * to64(B.linear(up(x), up(w), up(b), act=act, residual=up(r), residual_first=True))).sum())
    g = B.linear_backward(up(c), up(w), x8, z8, act=act, want_dz=True)
    tolerance = _tolerances(x, w, b, r, c, z)
    for name, t, got in (("dx", x, g.dx), ("dw", w, g.dw), ("db", b, g.db), ("dz", r, g.dz)):
        off = np.abs(_differences(t, loss) - to64(got)) - tolerance[name]
        assert np.all(off <= 0), (name, off.max())

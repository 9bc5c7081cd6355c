"""Group norm of groups far from zero: the mean is as good as its 32 bits, not as its sum's roundings."""
import numpy as np
import pytest

import label_reference as ref
from test_gpu_norm import both, close, data, nb  # noqa: F401

pytestmark = pytest.mark.gpu
E, D, EPS = ref.E, ref.D, 1e-5

# held by a work-group; cut into chunks; with the chunks joined in a launch of their own
SIZES = [(6, 2, 5), (18, 3, 33), (40, 2, 70), (96, 2, 100), (546, 2, 37), (1000, 1, 64), (2250, 1, 64), (9001, 1, 40), (160003, 1, 70)]


@pytest.mark.parametrize("F,G,B", SIZES)
def test_groups_of_one_number(nb, F, G, B):
    """All differences are 0, whatever the number.  The mean of 32-bit sums is off by at most D roundings (of the number, c), the differences d to it are exact,
    their mean is d up to D roundings, which leaves c after the correction's rounding: (D E)^2 c is far below half a step of c.  The squares keep what
    the two sums' roundings leave of d^2, 3 D E d^2 at most."""
    rng = np.random.default_rng(F)
    c = np.resize(np.array([1000.1, -1000.3, 0.1, 3333.333, 1e-3, -7.7e3], np.float32), B)
    X = np.broadcast_to(c, (F, B)).copy()
    _, gamma, beta, dY = data(rng, F, B)
    y, mean, rstd, dx, dg, db = (t.cpu().numpy().astype(np.float64) for t in both(nb, X, gamma, beta, dY, G, 0, 0.0, (0, 3, 0, 1, 2), EPS))
    assert np.array_equal(mean, np.broadcast_to(c, (G, B)))
    assert np.array_equal(y, np.broadcast_to(beta[:, None], (F, B)))
    assert not dg.any()
    rel = 0.5 * 3 * D * E * (D * E * np.abs(c.astype(np.float64))) ** 2 / EPS + 4 * E
    close(rstd, np.full((G, B), EPS ** -0.5), EPS ** -0.5 * rel, "rstd")
    h = (gamma[:, None].astype(np.float64) * dY).reshape(G, F // G, B)
    s, size = h.mean(1, keepdims=True), np.abs(h).mean(1, keepdims=True)
    want = EPS ** -0.5 * (h - s)
    close(dx, want.reshape(F, B), (EPS ** -0.5 * ((D + 1) * E * size + 3 * E * (np.abs(h) + np.abs(s))) + (rel + 2 * E) * np.abs(want)).reshape(F, B), "dX")


@pytest.mark.parametrize("F,G,B", SIZES)
def test_a_mean_10_000_times_the_spread(nb, F, G, B):
    """Bounds: those of the same numbers less 10^4, whose sums lose no more than the differences' do, and the mean's own rounding: one where a work-group holds the group,
    two where chunks leave rounded means, and D roundings of D roundings."""
    rng = np.random.default_rng(F + 1)
    X, gamma, beta, dY = data(rng, F, B, offset=1e4)
    want = ref.Norm(X.astype(np.float64) - 1e4, gamma, beta, G, EPS, 0, np.ones((F, B)), dY)
    y, mean, rstd, dx, dg, db = both(nb, X, gamma, beta, dY, G, 0, 0.0, (0, 3, 0, 1, 2), EPS)
    off = ((2 if F // G > 1024 else 1) * E + 2 * (D * E) ** 2) * 10010
    close(mean, want.mean + 1e4, want.mean_tol + off, "mean")
    # (where chunks' means are rounded, the squares take the mean of their errors' squares and of their products with the differences)
    var_off = off ** 2 + 2 * off / np.sqrt(F // G) if F // G > 1024 else 0
    r = np.repeat(want.rstd, F // G, axis=0)
    rstd_off = 0.5 * want.rstd ** 3 * var_off
    close(rstd, want.rstd, want.rstd_tol + rstd_off, "rstd")
    xh = (want.Y - beta[:, None]) / gamma[:, None]
    moved = r * off + np.abs(xh) * 0.5 * r * r * var_off
    close(y, want.Y, want.Y_tol + np.abs(gamma[:, None]) * moved + 2 * E * np.abs(beta[:, None]), "Y")
    h = gamma[:, None].astype(np.float64) * dY

    def avg(t):
        return np.repeat(t.reshape(G, F // G, B).mean(1), F // G, axis=0)
    close(dx, want.dX, want.dX_tol + r * (moved * np.abs(avg(h * xh)) + np.abs(xh) * avg(np.abs(h) * moved)) + 0.5 * r * r * var_off * np.abs(want.dX), "dX")
    close(dg, want.dgamma, want.dgamma_tol + (np.abs(dY) * moved).sum(1), "dgamma")
    close(db, want.dbeta, want.dbeta_tol, "dbeta")


@pytest.mark.parametrize("F,G,B", [(40, 2, 70), (1000, 1, 64), (9001, 1, 40), (160003, 1, 70)])
def test_relu_takes_the_same_side_both_ways_far_from_zero(nb, F, G, B):
    """dbeta of ones counts the columns whose output is positive; many arguments lie within a rounding of 0."""
    rng = np.random.default_rng(F + 2)
    X, _, _, _ = data(rng, F, B, offset=1e4)
    X[:, ::3] = np.round(X[:, ::3])
    y, _, _, _, _, db = both(nb, X, None, None, np.ones((F, B), np.float32), G, 1, 0.0)
    assert np.array_equal(db.cpu().numpy(), (y > 0).sum(1).float().cpu().numpy())


def test_a_group_with_an_infinite_entry_has_an_infinite_mean(nb):
    rng = np.random.default_rng(3)
    for F, G, B in ((48, 2, 9), (4500, 2, 9)):
        X, gamma, beta, dY = data(rng, F, B)
        m = F // G
        X[m, 2], X[m + 1, 5], X[m + 2, 6] = np.inf, -np.inf, np.nan
        y, mean, rstd, *_ = (t.cpu().numpy() for t in both(nb, X, gamma, beta, dY, G, 0, 0.0))
        assert mean[1, 2] == np.inf and mean[1, 5] == -np.inf and np.isnan(mean[1, 6])
        assert np.isnan(rstd[1, [2, 5, 6]]).all() and np.isfinite(rstd[0]).all() and np.isfinite(y[:m]).all() and np.isnan(y[m:, [2, 5, 6]]).all()

"""Operands beyond the caches, whose results are written past them, and chunks of logits of several steps, against 64 bits."""
import numpy as np
import pytest

import label_reference as ref
from test_gpu_losses import nans, run_policy, workspace
from test_gpu_norm import LAYER, SEED, STEP, blank, both, close, data, gpu, matrix, nb, padding_untouched, state  # noqa: F401

pytestmark = pytest.mark.gpu

E = ref.E


def logits(rng, C, B):
    """In every second stretch of 32 classes the logits are higher by 6 in even columns and lower in odd ones, so that a running maximum moves between the steps of a
    thread, or does not; some classes are closed, some columns do not count."""
    Z = (2 * rng.standard_normal((C, B), dtype=np.float32))
    Z += 6 * ((np.arange(C) // 32 % 2)[:, None] * np.where(np.arange(B) % 2 == 0, 1, -1)).astype(np.float32)
    Z[rng.integers(0, C, 1000), rng.integers(0, B, 1000)] = -np.inf
    Z[:, B - 3] = -np.inf
    labels = rng.integers(0, C, B).astype(np.int32)
    labels[rng.random(B) < 0.1] = -1
    return Z, labels


def blocks(B, width=1500):
    return [slice(a, min(B, a + width)) for a in range(0, B, width)]


# in chunks, two steps each, and the last of 9; held by work-groups; neither batch a multiple of a tile
@pytest.mark.parametrize("C,B", [(9001, 8190), (1000, 17003)])
def test_losses(nb, C, B):
    import torch
    rng = np.random.default_rng(C)
    Z, labels = logits(rng, C, B)
    lp = np.concatenate([ref.Labels(Z[:, b], labels[b]).logp for b in blocks(B)])
    old, refs = ((lp + 0.3 * rng.standard_normal(B)).astype(np.float32) for _ in range(2))
    A, w = rng.standard_normal(B).astype(np.float32), rng.random(B).astype(np.float32)
    print("policy", flush=True)
    stats, logp, dz = run_policy(nb, Z, labels, old, refs, A, w, 0.2, 0.28, 0.04, (2, 5))
    total, tol = np.zeros(4), np.zeros(4)
    for b in blocks(B):
        want = ref.Policy(Z[:, b], labels[b], old[b], refs[b], A[b], w[b], 0.2, 0.28, 0.04)
        close(logp[b], want.L.logp, want.L.logp_tol, "logp")
        close(dz[:, b], want.dZ, want.dZ_tol, "dZ")
        total, tol = total + want.stats, tol + want.stats_tol
    close(stats, total, tol, "stats")
    stats2, logp2, dz2 = run_policy(nb, Z, labels, old, refs, A, w, 0.2, 0.28, 0.04, (1, 0), in_place=True)
    assert torch.equal(dz2, dz) and torch.equal(stats2, stats) and torch.equal(logp2, logp)
    del dz2
    print("preference", flush=True)
    pairs = 8
    starts = np.sort(rng.integers(0, B + 1, 2 * pairs + 1)).astype(np.int32)
    z, sums, margins, loss, ws = matrix(Z, 3), nans(2 * pairs), nans(pairs), nans(1), workspace(nb, C, B, 2 * pairs)
    nb.preference_loss(z, gpu(labels), gpu(starts), None, C, B, pairs, 0.01, 0.1, dz, sums, margins, loss, ws)
    off = np.concatenate([ref.Labels(Z[:, b], labels[b]).off for b in blocks(B)])
    s, s_off = (np.array([t[a:e].sum() for a, e in zip(starts[:-1], starts[1:])]) for t in (lp, off))
    close(sums, s, s_off + E * np.abs(s), "sums")
    beta, t = float(np.float32(0.01)), float(np.float32(0.1))
    x, x_off = beta * (s[0::2] - s[1::2]), beta * (s_off[0::2] + s_off[1::2])
    close(margins, x, x_off + E * np.abs(x), "margins")
    want = ((1 - t) * np.logaddexp(0, -x) + t * np.logaddexp(0, x)).mean()
    close(loss, np.array([want]), x_off.mean() + E * want, "loss")
    slope = (t * ref.sigmoid(x) - (1 - t) * ref.sigmoid(-x)) * beta / pairs
    c, c_off = np.zeros(B), np.zeros(B)
    for k in range(2 * pairs):
        c[starts[k]:starts[k + 1]] = (1, -1)[k % 2] * slope[k // 2]
        c_off[starts[k]:starts[k + 1]] = 0.25 * x_off[k // 2] * beta / pairs + 2 * E * np.abs(slope[k // 2])
    for b in blocks(B):
        L = ref.Labels(Z[:, b], labels[b])
        g, tol = L.gradient(np.where(L.counts, c[b], 0), np.where(L.counts, c_off[b], 0))
        close(dz[:, b], g, tol, "dZ")
    assert padding_untouched(z, dz)
    nb.preference_loss(z, gpu(labels), gpu(starts), None, C, B, pairs, 0.01, 0.1, z, None, None, None, ws)
    assert torch.equal(z, dz) and padding_untouched(z)
    nb.label_log_probs(matrix(Z), gpu(labels), C, B, gpu(starts), 2 * pairs, nans(B), sums2 := nans(2 * pairs), ws)
    assert torch.equal(sums2, sums)


def test_dropout(nb):
    import torch
    F, B = 4103, 4101
    X = np.random.default_rng(1).standard_normal((F, B), dtype=np.float32)
    x, y = matrix(X, 2), blank(F, B, 3)
    nb.dropout(x, F, B, 0.25, LAYER, state(), y)
    factor = ref.factors(F, B, 0.25, LAYER, SEED, STEP)
    want = np.where(factor > 0, X * np.float32(factor.max()), np.float32(0))
    assert np.array_equal(y.cpu().numpy(), want) and padding_untouched(x, y)
    nb.dropout(x, F, B, 0.25, LAYER, state(), x)
    assert torch.equal(x, y) and padding_untouched(x)


# in chunks; held, in tiles of which the last is not whole
@pytest.mark.parametrize("F,G,B", [(4100, 1, 4099), (512, 8, 33001)])
def test_norm(nb, F, G, B):
    rng = np.random.default_rng(F)
    X, gamma, beta, dY = data(rng, F, B, offset=2.0)
    y, mean, rstd, dx, dg, db = both(nb, X, gamma, beta, dY, G, 2, 0.1, (1, 3, 0, 2, 5))
    factor = ref.factors(F, B, 0.1, LAYER, SEED, STEP)
    want = [np.zeros(F) for _ in range(4)]
    for b in blocks(B, 4000):
        n = ref.Norm(X[:, b], gamma, beta, G, 1e-5, 2, factor[:, b], dY[:, b])
        for got, name in ((y, "Y"), (mean, "mean"), (rstd, "rstd"), (dx, "dX")):
            close(got[:, b], getattr(n, name), getattr(n, name + "_tol"), name)
        for k, name in enumerate(("dgamma", "dgamma_tol", "dbeta", "dbeta_tol")):
            want[k] += getattr(n, name)
    # (sums over the columns: some hundred terms one after the other, of the columns' tiles, in a thread, then the slabs)
    close(dg, want[0], want[1] * (1 + B / 1000), "dgamma")
    close(db, want[2], want[3] * (1 + B / 1000), "dbeta")

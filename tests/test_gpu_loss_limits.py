"""The losses of labels where one work-group holds all columns, and a class or a column beyond it, against 64 bits."""
import numpy as np
import pytest

import label_reference as ref
from test_gpu_losses import cuts, logits, nans, policy_inputs, run_policy, workspace
from test_gpu_norm import blank, close, gpu, matrix, nb, padding_untouched  # noqa: F401

pytestmark = pytest.mark.gpu


# (the layouts that these sizes stand for are counted in test_loss_plans.py)
@pytest.mark.parametrize("C,B,kind", [(128, 128, "plain"), (129, 128, "masked"), (128, 125, "masked"), (256, 64, "wide"), (250, 61, "masked"), (512, 32, "lowest"), (1024, 16, "plain"),
                                      (1025, 16, "masked"), (1021, 13, "masked"), (2048, 8, "far"), (2048, 5, "masked"), (2049, 8, "plain"), (33, 256, "masked"), (64, 250, "plain"),
                                      (2048, 4, "masked"), (2047, 3, "plain"), (2049, 3, "masked")])
def test_all_three_losses(nb, C, B, kind):
    rng = np.random.default_rng(C * 13 + B)
    Z, labels = logits(rng, C, B, kind)
    old, refs, A, w = policy_inputs(rng, Z, labels)
    want = ref.Policy(Z, labels, old, refs, A, w, 0.2, 0.28, 0.04)
    stats, lp, dz = run_policy(nb, Z, labels, old, refs, A, w, 0.2, 0.28, 0.04, (1, 2))
    close(lp, want.L.logp, want.L.logp_tol, "logp"), close(stats, want.stats, want.stats_tol, "stats"), close(dz, want.dZ, want.dZ_tol, "dZ")
    stats2, lp2, dz2 = run_policy(nb, Z, labels, old, refs, A, w, 0.2, 0.28, 0.04, (3, 0), in_place=True)
    assert bool((dz2 == dz).all()) and bool((stats2 == stats).all()) and bool((lp2 == lp).all())
    starts = cuts(rng, B, 6)
    want = ref.Preference(Z, labels, starts, None, 0.02, 0.1)
    z, dz, sums, margins, loss, scores, ws = matrix(Z, 5), blank(C, B, 3), nans(6), nans(3), nans(1), nans(6), workspace(nb, C, B, 6)
    nb.preference_loss(z, gpu(labels), gpu(starts), None, C, B, 3, 0.02, 0.1, dz, sums, margins, loss, ws)
    close(sums, want.sums, want.sums_tol, "sums"), close(margins, want.margins, want.margins_tol, "margins"), close(loss, np.array([want.loss]), want.loss_tol, "loss")
    close(dz, want.dZ, want.dZ_tol, "dZ")
    assert padding_untouched(z, dz)
    nb.preference_loss(z, gpu(labels), gpu(starts), None, C, B, 3, 0.02, 0.1, z, None, None, None, ws)
    assert bool((z == dz).all())
    nb.label_log_probs(matrix(Z), gpu(labels), C, B, gpu(starts), 6, None, scores, ws)
    assert bool((scores == sums).all())

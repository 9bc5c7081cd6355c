"""Policy and preference loss: an advantage, a KL factor or a smoothing of 0 takes nothing of a term, however large that is."""
import numpy as np
import pytest

import label_reference as ref
from test_gpu_losses import logits, nans, policy_inputs, run_policy, workspace
from test_gpu_norm import blank, gpu, matrix, nb  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C,B", [(10, 100), (300, 3001), (3000, 300)])
def test_factors_of_0(nb, C, B):
    import torch
    rng = np.random.default_rng(C)
    Z, labels = logits(rng, C, B)
    old, refs, A, w = policy_inputs(rng, Z, labels)
    lp = ref.Labels(Z, labels).logp
    A[::3] = 0
    old[::3] = lp[::3]
    near = run_policy(nb, Z, labels, old, None, A, w, 0.2, 0.3, 0.0)
    for far in (-800, -1e30, -np.inf, np.inf):
        old[::3] = far
        stats, _, dz = run_policy(nb, Z, labels, old, None, A, w, 0.2, 0.3, 0.0)
        assert torch.equal(stats, near[0]) and torch.equal(dz, near[2]) and bool(torch.isfinite(dz).all())
    # a reference that is known but not to hold the policy: whatever it says, only its own sum takes it
    for far in (-1, 700, 1e30, np.inf, -np.inf):
        refs[1::3] = lp[1::3] + far
        stats, _, dz = run_policy(nb, Z, labels, old, refs, A, w, 0.2, 0.3, 0.0)
        assert torch.equal(stats[[0, 1, 3]], near[0][[0, 1, 3]]) and torch.equal(dz, near[2])
        assert float(stats[2]) > 0
    # what is not multiplied by 0 is as large as it is
    stats, _, dz = run_policy(nb, Z, labels, old, refs, A, w, 0.2, 0.3, 0.1)
    assert np.isposinf(stats[[0, 2]].cpu().numpy()).all() and bool((stats[1] == near[0][1]).all())
    # a NaN is none of these
    Z[0, 0] = np.nan
    stats, _, dz = run_policy(nb, Z, labels, old, None, A, w, 0.2, 0.3, 0.0)
    assert bool(torch.isnan(dz[:, 0]).all()) and bool(torch.isnan(stats[:2]).all()) and bool(torch.isfinite(dz[:, 1:]).all())


@pytest.mark.parametrize("C,B", [(10, 100), (300, 3001), (3000, 300)])
def test_pairs_that_are_decided(nb, C, B):
    """A reference that gives a sequence no probability decides its pair: the loss of the side that it wins is 0."""
    rng = np.random.default_rng(C + 1)
    Z, labels = logits(rng, C, B)
    starts = np.array([0, B // 9, B // 5, B // 4, B // 2, B - 3, B], np.int32)
    sums = (ref.Labels(Z, labels).sums(starts)[0] + rng.standard_normal(6)).astype(np.float32)
    sums[2] = -np.inf
    for t, sign in ((0.0, 1), (1.0, -1)):
        if sign < 0:
            sums[2], sums[3] = sums[3], sums[2]
        dz, margins, loss = blank(C, B), nans(3), nans(1)
        nb.preference_loss(matrix(Z), gpu(labels), gpu(starts), gpu(sums), C, B, 3, 0.1, t, dz, None, margins, loss, workspace(nb, C, B, 6))
        x = margins.cpu().numpy().astype(np.float64)
        assert x[1] == sign * np.inf
        # (a margin of 32 bits is off by one rounding, and the logarithm's slope is below 1)
        want = np.log1p(np.exp(-sign * x)).mean()
        assert abs(float(loss) - want) <= ref.E * (np.abs(x[[0, 2]]).max() + 2 * want)
        assert bool(torch_finite(dz)) and not bool(dz[:, starts[2]:starts[4]].any()) and bool(dz[:, :starts[2]].any())
        # with any smoothing the other side counts
        nb.preference_loss(matrix(Z), gpu(labels), gpu(starts), gpu(sums), C, B, 3, 0.1, 0.5, dz, None, None, loss, workspace(nb, C, B, 6))
        assert np.isposinf(float(loss)) and bool(torch_finite(dz))


def torch_finite(t):
    import torch
    return torch.isfinite(t).all()

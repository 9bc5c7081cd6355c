"""Policy loss: an advantage or a KL factor of 0 takes nothing of a term, however large that is."""
import numpy as np
import pytest

import label_reference as ref
from test_gpu_losses import logits, policy_inputs, run_policy
from test_gpu_norm import nb  # noqa: F401

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

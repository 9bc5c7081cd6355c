"""Group norm and dropout in tiles of columns that the batch does not fill, against 64 bits, in place and not."""
import numpy as np
import pytest

import label_reference as ref
from test_gpu_norm import LAYER, SEED, STEP, blank, both, close, data, gpu, matrix, nb, padding_untouched, state  # noqa: F401

pytestmark = pytest.mark.gpu


# every number of columns that a tile's last lanes may have, in one tile and behind whole ones
@pytest.mark.parametrize("B", [1, 2, 3, 4, 5, 6, 7, 8, 9, 31, 33, 34, 35, 36, 99, 100, 101, 127, 129, 130, 131, 255, 257, 258, 259])
def test_tiles_that_are_not_whole(nb, B):
    import torch
    rng = np.random.default_rng(B)
    for F, G in ((10, 2), (64, 1), (1030, 5), (4100, 1)):
        X, gamma, beta, dY = data(rng, F, B)
        factor = ref.factors(F, B, 0.25, LAYER, SEED, STEP)
        want = ref.Norm(X, gamma, beta, G, 1e-5, 2, factor, dY)
        y, mean, rstd, dx, dg, db = both(nb, X, gamma, beta, dY, G, 2, 0.25, (3, 1, 2, 5, 1))
        for got, name in ((y, "Y"), (mean, "mean"), (rstd, "rstd"), (dx, "dX"), (dg, "dgamma"), (db, "dbeta")):
            close(got, getattr(want, name), getattr(want, name + "_tol"), (name, F))
        x = matrix(X, 1)
        ws = torch.full((max(4, nb.group_norm_workspace_bytes(F, G, B) // 4),), float("nan"), device="cuda")
        nb.group_norm_forward(x, gpu(gamma), gpu(beta), F, G, B, 1e-5, 2, 0.25, LAYER, state(), x, None, None, ws)
        assert torch.equal(x, y) and padding_untouched(x)
        x, z = matrix(X, 7), blank(F, B, 2)
        nb.dropout(x, F, B, 0.25, LAYER, state(), z)
        assert np.array_equal(z.cpu().numpy(), np.where(factor > 0, X * np.float32(factor.max() if factor.any() else 0), np.float32(0))) and padding_untouched(x, z)
        nb.dropout(x, F, B, 0.25, LAYER, state(), x)
        assert torch.equal(x, z) and padding_untouched(x)

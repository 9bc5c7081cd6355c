"""Lists of gradients that name an array more than once."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24   # half a step of fp32, relative


@pytest.fixture(scope="module")
def nb():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2407_17437_amd import binding
    return binding


def workspace(nb, n):
    import torch
    return torch.full((nb.gradient_norm_workspace_bytes(n) // 4,), float("nan"), device="cuda")


@pytest.mark.parametrize("lengths,order", [
    ([1000], [0, 0]), ([5000, 3], [0, 1, 0, 1, 0]), ([17] * 60, list(range(60)) * 3), ([2049] * 300, list(range(300)) + list(range(299, -1, -2))),
    ([400_000] * 3, [0, 1, 2, 2, 0]), ([5] * 400, [i // 2 for i in range(800)])], ids=lambda x: str(len(x)))
def test_a_gradient_twice_is_clipped_once(nb, lengths, order):
    """Tied layers: the list names a gradient several times, which counts as often in the norm; in place and to arrays of its own it becomes c * gradient."""
    import torch
    rng = np.random.default_rng(len(order))
    arrays = [torch.as_tensor(rng.standard_normal(n).astype(np.float32)).cuda() for n in lengths]
    want = np.sqrt(sum(float((arrays[i].double() ** 2).sum()) for i in order))
    max_norm = float(np.float32(want / 3))
    # c is rounded once, and so is every product
    expected = [max_norm / want * a.double() for a in arrays]
    for in_place in (True, False):
        grads = [a.clone() for a in arrays]
        out = grads if in_place else [torch.full_like(a, float("nan")) for a in arrays]
        norm = torch.zeros(1, device="cuda")
        nb.gradient_clip([grads[i] for i in order], [out[i] for i in order], max_norm, workspace(nb, len(order)), norm)
        assert abs(float(norm) - want) <= want * U * 1.001
        for got, e in zip(out, expected):
            assert ((got.double() - e).abs() <= e.abs() * 2 * U * 1.01).all()

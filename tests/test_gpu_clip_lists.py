"""Lists of gradients that name an array more than once, and longer lists than one launch, or the step of an MLP, holds at a time."""
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


@pytest.mark.parametrize("counts", [[60_000 + i for i in range(600)], [16_384 + i % 7 for i in range(800)]], ids=["past the cache", "in the cache"])
def test_lists_whose_partial_sums_are_added_up_on_their_own(nb, counts):
    """More than 2048 partial sums: more than two launches of the norm's first kernel, and one that adds up what they leave.  The workspace is as
    large as the call asks for, and what lies behind it stays."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(5)
    assert sum(-(-n // 8192) for n in counts) > 2048
    new = lambda scale: [scale * torch.randn(n, generator=g, device="cuda") for n in counts]
    grads, w, v = new(1.0), new(1.0), new(0.1)
    grads[3][77], grads[-1][-1] = 3e4, -2e4        # (first and last: no part of the sum may be left out)
    want = float(torch.stack([x.double().square().sum() for x in grads]).sum().sqrt())
    need = nb.gradient_norm_workspace_bytes(len(counts)) // 4
    room, norm = torch.full((need + 256,), float("nan"), device="cuda"), torch.zeros(1, device="cuda")
    ws, behind = room[:need], room[need:]
    behind.fill_(7)
    max_norm = float(np.float32(want / 5))
    c = float(np.float32(max_norm / want))          # the kernel's factor, whose last step the sum's order in 64 bits does not reach
    nb.gradient_norm(grads, ws, norm)
    assert abs(float(norm) - want) <= want * U * 1.001
    out = [torch.full_like(x, float("nan")) for x in grads]
    norm.zero_()
    nb.gradient_clip(grads, out, max_norm, ws, norm)
    assert abs(float(norm) - want) <= want * U * 1.001 and all(torch.equal(a, c * x) for a, x in zip(out, grads))
    w2, v2 = [t.clone() for t in w], [t.clone() for t in v]
    norm.zero_()
    nb.sgd_update_clipped(w, v, grads, 0.05, 0.9, max_norm, False, ws, norm)
    for a, b, x in zip(w2, v2, grads):
        nb.sgd_update_values(a, b, c * x, x.numel(), 0.05, 0.9)
    assert abs(float(norm) - want) <= want * U * 1.001 and all(torch.equal(a, b) for a, b in zip(w + v, w2 + v2))
    assert (behind == 7).all()


@pytest.mark.parametrize("nesterov", [False, True])
def test_clipped_step_of_many_layers(nb, nesterov):
    """35 layers, whose arrays are more than the step's own list holds: the step on all of them with one norm."""
    import torch
    from paper_2407_17437_amd import workloads as wl
    batch, lr, mu = 30, 0.05, 0.9
    sizes = (40,) + tuple(20 + 3 * (i % 5) for i in range(34)) + (10,)
    mlp = wl.make_mlp(sizes, pattern_seed=41, value_seed=42, sparsity=0.3, bias_std=0.3)
    flags = nb.NERVA_MLP_NESTEROV if nesterov else 0
    A, T = nb.MLP(mlp, batch, flags), nb.MLP(mlp, batch, flags | nb.NERVA_MLP_UNFUSED)
    n = len(A.layers)
    assert 2 * n > 64
    Xs, Ts = wl.make_batches(sizes[0], sizes[-1], batch, 1, seed=9)
    X, labels = nb.to_dense(Xs[0]), torch.as_tensor(Ts[0]).cuda()
    arrays = [x for L in A.layers for x in ((L.values, L.velocity), (L.bias, L.bias_velocity))]
    before = [(w.clone(), v.clone()) for w, v in arrays]
    T.train_step(X, labels, batch, lr, mu)          # its gradients are the same
    grads = [T.view(kind, l, batch).clone() for l in range(n) for kind in ("g", "db")]
    want = float(torch.stack([x.double().square().sum() for x in grads]).sum().sqrt())
    assert want > 0 and all(float(x.abs().max()) > 0 for x in grads[-8:])
    max_norm = float(np.float32(want / 4))
    c = float(np.float32(max_norm / want))
    A.train_step_clipped(X, labels, batch, lr, mu, max_norm)
    assert abs(float(A.norm) - want) <= want * U * 1.001
    for (w, v), (w2, v2), x in zip(arrays, before, grads):
        (nb.sgd_update_values_nesterov if nesterov else nb.sgd_update_values)(w2, v2, c * x, x.numel(), lr, mu)
        assert torch.equal(w, w2) and torch.equal(v, v2)
    A.close(); T.close()


@pytest.mark.parametrize("dense", [None, 0.5])
def test_captured_clipped_steps_of_an_mlp(nb, dense):
    """The whole clipped step in a graph, replayed on changing batches, with plain steps between: the bits of the same steps outside a graph."""
    import torch
    from paper_2407_17437_amd import workloads as wl
    batch, sizes = 64, (128, 96, 64, 10)
    mlp = wl.make_mlp(sizes, pattern_seed=3, value_seed=4, sparsity=0.4, bias_std=0.1)
    A, B = nb.MLP(mlp, batch, dense_from_density=dense), nb.MLP(mlp, batch, dense_from_density=dense)
    Xs, Ts = wl.make_batches(sizes[0], sizes[-1], batch, 5, seed=8)
    batches = [(nb.to_dense(x), torch.as_tensor(t).cuda()) for x, t in zip(Xs, Ts)]
    X, labels = batches[0][0].clone(), batches[0][1].clone()
    for M in (A, B):
        M.train_step(X, labels, batch, 0.05, 0.9)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        A.train_step_clipped(X, labels, batch, 0.05, 0.9, 0.3, ldx=X.stride(0))
    for t, (x, y) in enumerate(batches):
        X.copy_(x)
        labels.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        B.train_step_clipped(X, labels, batch, 0.05, 0.9, 0.3)
        assert torch.equal(A.norm, B.norm) and float(A.norm) > 0 and torch.equal(A.loss, B.loss)
        if t % 2:
            for M in (A, B):
                M.train_step(X, labels, batch, 0.05, 0.9)
        for a, b in zip(A.layers, B.layers):
            assert all(torch.equal(getattr(a, n), getattr(b, n)) for n in ("values", "velocity", "bias", "bias_velocity"))
    A.close(); B.close()

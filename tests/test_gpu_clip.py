"""The norm over many gradients, clipped gradients and the clipped momentum step, alone and inside a training step of an MLP."""
import numpy as np
import pytest

from paper_2407_17437_amd import workloads as wl

pytestmark = pytest.mark.gpu
U = 2.0 ** -24   # half a step of fp32, relative


@pytest.fixture(scope="module")
def nb():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2407_17437_amd import binding
    return binding


def arrays(rng, counts, scale, offset=0):
    """fp32 arrays on the device, each `offset` entries behind a 16-byte boundary."""
    import torch
    out = []
    for n in counts:
        full = torch.zeros(n + offset, device="cuda")
        full[offset:] = torch.as_tensor((scale * rng.standard_normal(n)).astype(np.float32)).cuda()
        out.append(full[offset:])
    return out


def norm_of(grads):
    return np.sqrt(sum(float((g.cpu().numpy().astype(np.float64) ** 2).sum()) for g in grads))


def workspace(nb, n):
    import torch
    return torch.full((nb.gradient_norm_workspace_bytes(n) // 4,), float("nan"), device="cuda")


def steps(w, v, g, lr, mu, c, nesterov):
    """The step in 64 bits and the bounds of its errors: c, c g, lr c g, the multiply-add and the sum are rounded once each."""
    w, v, g = (t.cpu().numpy().astype(np.float64) for t in (w, v, g))
    lr, mu = float(np.float32(lr)), float(np.float32(mu))
    step = lr * c * g
    nv = mu * v - step
    ev = (4 * np.abs(step) + np.abs(nv)) * U * 1.01
    move = mu * nv - step if nesterov else nv
    em = mu * ev + (4 * np.abs(step) + np.abs(move)) * U * 1.01 if nesterov else ev
    return w + move, nv, em + np.abs(w + move) * U * 1.01 + 1e-37, ev + 1e-37


LISTS = [[], [0], [1], [0, 3, 0, 2], [5, 4095, 4096, 4097, 1], [1023, 70000, 10], [3_000_001, 17], [7] * 63, [100 + i for i in range(64)], [33] * 65, [2049] * 200]


@pytest.mark.parametrize("counts", LISTS, ids=lambda c: f"{len(c)}x{sum(c)}")
@pytest.mark.parametrize("offset", [0, 1])
def test_norm_clip_and_step(nb, counts, offset):
    import torch
    rng = np.random.default_rng(len(counts) + offset)
    grads = arrays(rng, counts, 0.7, offset)
    want = norm_of(grads)
    ws, norm = workspace(nb, len(counts)), torch.full((1,), -1.0, device="cuda")
    nb.gradient_norm(grads, ws, norm)
    assert abs(float(norm) - want) <= want * U * 1.001
    for max_norm in (0.25, 1e6, float("inf")):
        m = float(np.float32(max_norm))
        c = min(1.0, m / want) if want > 0 else 1.0
        out = [torch.full((n,), float("nan"), device="cuda") for n in counts]
        norm.fill_(-1)
        nb.gradient_clip(grads, out, max_norm, ws, norm)
        assert abs(float(norm) - want) <= want * U * 1.001
        for a, g in zip(out, grads):
            g64 = g.cpu().numpy().astype(np.float64)
            assert np.all(np.abs(a.cpu().numpy() - c * g64) <= np.abs(c * g64) * 2 * U * 1.01)
            assert c < 1 or torch.equal(a, g)
        in_place = [g.clone() for g in grads]
        nb.gradient_clip(in_place, in_place, max_norm, ws, None)
        assert all(torch.equal(a, b) for a, b in zip(in_place, out))
        for nesterov in (False, True):
            values, velocities = arrays(rng, counts, 1.0, offset), arrays(rng, counts, 0.1)
            expected = [steps(w, v, g, 0.05, 0.9, c, nesterov) for w, v, g in zip(values, velocities, grads)]
            norm.fill_(-1)
            nb.sgd_update_clipped(values, velocities, grads, 0.05, 0.9, max_norm, nesterov, ws, norm)
            assert abs(float(norm) - want) <= want * U * 1.001
            for w, v, (rw, rv, ew, ev) in zip(values, velocities, expected):
                assert np.all(np.abs(w.cpu().numpy() - rw) <= ew) and np.all(np.abs(v.cpu().numpy() - rv) <= ev)


def test_step_without_clipping_is_the_plain_step(nb):
    """c = 1: the same bits as sgd_update_values on every array."""
    import torch
    rng = np.random.default_rng(2)
    counts = [5000, 1, 12345]
    grads = arrays(rng, counts, 1e-4)
    ws = workspace(nb, 3)
    for nesterov, plain in ((False, nb.sgd_update_values), (True, nb.sgd_update_values_nesterov)):
        w, v = arrays(rng, counts, 1.0), arrays(rng, counts, 0.1)
        w2, v2 = [t.clone() for t in w], [t.clone() for t in v]
        nb.sgd_update_clipped(w, v, grads, 0.05, 0.9, 1.0, nesterov, ws, None)
        for a, b, g in zip(w2, v2, grads):
            plain(a, b, g, g.numel(), 0.05, 0.9)
        assert all(torch.equal(a, b) for a, b in zip(w + v, w2 + v2))


@pytest.mark.parametrize("nesterov", [False, True])
def test_step_on_more_than_the_cache_holds(nb, nesterov):
    """Lists beyond 256 MiB of arrays, in several launches: without clipping the bits of the plain step, with it the step of scaled gradients."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    counts = [65537, 12, 150001] * 74 + [4097]
    assert 20 * sum(counts) > 256 << 20 and len(counts) > 192
    new = lambda scale: [scale * torch.randn(n, generator=g, device="cuda") for n in counts]
    grads, w, v = new(1.0), new(1.0), new(0.1)
    total = sum(float(x.double().square().sum()) for x in grads) ** 0.5
    ws, norm = workspace(nb, len(counts)), torch.zeros(1, device="cuda")
    plain = nb.sgd_update_values_nesterov if nesterov else nb.sgd_update_values
    for max_norm in (float("inf"), 2.5):
        w2, v2 = [t.clone() for t in w], [t.clone() for t in v]
        nb.sgd_update_clipped(w, v, grads, 0.05, 0.9, max_norm, nesterov, ws, norm)
        assert abs(float(norm) - total) <= total * U * 1.001
        # the kernel's factor is the fp32 nearest to max_norm / norm, whose last step the sum's order in 64 bits does not reach
        c = float(np.float32(min(1.0, max_norm / total)))
        for a, b, x in zip(w2, v2, grads):
            plain(a, b, c * x, x.numel(), 0.05, 0.9)
        assert all(torch.equal(a, b) for a, b in zip(w + v, w2 + v2))


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan"), 3.0e38])
def test_a_norm_that_is_not_finite_changes_nothing(nb, value):
    import torch
    rng = np.random.default_rng(6)
    counts = [3000, 50000, 3]
    grads = arrays(rng, counts, 1.0)
    grads[1][49999] = value
    grads[2][:2] = value          # (twice 3e38: each is finite, their norm lies beyond fp32)
    w, v = arrays(rng, counts, 1.0), arrays(rng, counts, 0.1)
    before = [t.clone() for t in w + v + grads]
    ws, norm = workspace(nb, 3), torch.zeros(1, device="cuda")
    nb.sgd_update_clipped(w, v, grads, 0.05, 0.9, 1.0, False, ws, norm)
    assert not torch.isfinite(norm).any()
    nb.gradient_clip(grads, grads, 1.0, ws, None)
    assert all(torch.equal(a.view(torch.int32), b.view(torch.int32)) for a, b in zip(w + v + grads, before))


def test_large_and_small_entries(nb):
    """Squares beyond and below fp32: 1e25 squared, 1e-30 squared; and small entries beside a large one."""
    import torch
    ws, norm = workspace(nb, 2), torch.zeros(1, device="cuda")
    for fill, n in ((1e25, 1000), (1e-30, 5000), (1e-40, 100)):
        g = torch.full((n,), fill, device="cuda")
        want = float(g[0]) * np.sqrt(n)
        nb.gradient_norm([g, g], ws, norm)
        assert abs(float(norm) - want * np.sqrt(2)) <= want * 2 * U + 1e-45
    g = torch.full((1 << 24,), 1e-4, device="cuda")
    big = torch.full((1,), 1.0, device="cuda")
    want = np.sqrt(1 + (1 << 24) * float(g[0]) ** 2)
    nb.gradient_norm([g, big], ws, norm)
    assert abs(float(norm) - want) <= want * U * 1.001


def test_an_array_twice_is_stepped_twice(nb):
    import torch
    rng = np.random.default_rng(9)
    (w,), (v,) = arrays(rng, [1000], 1.0), arrays(rng, [1000], 0.1)
    g = arrays(rng, [1000, 1000, 1000], 1e-3)
    w2, v2 = w.clone(), v.clone()
    nb.sgd_update_clipped([w, w, w], [v, v, v], g, 0.05, 0.9, 1e3, False, workspace(nb, 3), None)
    for x in g:
        nb.sgd_update_values(w2, v2, x, 1000, 0.05, 0.9)
    assert torch.equal(w, w2) and torch.equal(v, v2)


def test_captured_step_of_changing_gradients(nb):
    import torch
    rng = np.random.default_rng(12)
    counts = [70001, 300, 5]
    g, w, v = arrays(rng, counts, 1.0), arrays(rng, counts, 1.0), arrays(rng, counts, 0.1)
    ws, norm = workspace(nb, 3), torch.zeros(1, device="cuda")
    ew, ev, enorm = [t.clone() for t in w], [t.clone() for t in v], torch.zeros(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        nb.sgd_update_clipped(w, v, g, 0.05, 0.9, 2.0, True, ws, norm)
    for t in range(4):
        for x in g:
            x.mul_(0.02 if t == 2 else 1.5)
        graph.replay()
        torch.cuda.synchronize()
        nb.sgd_update_clipped(ew, ev, g, 0.05, 0.9, 2.0, True, ws, enorm)
        assert torch.equal(norm, enorm) and all(torch.equal(a, b) for a, b in zip(w + v, ew + ev))


@pytest.mark.parametrize("sizes,kw,flags", [
    ((300, 200, 100, 10), dict(sparsity=0.9, bias_std=0.1), 0),                 # fused head
    ((300, 200, 100, 10), dict(sparsity=0.9, bias_std=0.1), 2 | 4),             # Nesterov, separate head
    ((200, 128, 10), dict(sparsity=0.4, bias_std=0.1), 0),                      # the hidden layer on the dense route
    ((100, 50), dict(sparsity=0.8, bias_std=0.1), 0),                           # one layer
])
def test_clipped_training_steps_of_an_mlp(nb, sizes, kw, flags):
    """Against the same gradients (those of an unfused step on a twin), the norm over them and the step; several steps, so that the copies
    of the weights that a step reads are the updated ones."""
    import torch
    batch, lr, mu = 70, 0.05, 0.9
    mlp = wl.make_mlp(sizes, pattern_seed=31, value_seed=32, **kw)
    A, T = nb.MLP(mlp, batch, flags), nb.MLP(mlp, batch, flags | nb.NERVA_MLP_UNFUSED)
    n = len(A.layers)
    for t, max_norm in enumerate((0.05, 1e6, 0.2)):
        Xs, Ts = wl.make_batches(sizes[0], sizes[-1], batch, 1, seed=50 + t)
        X, labels = nb.to_dense(Xs[0]), torch.as_tensor(Ts[0]).cuda()
        start = [[x.clone() for x in (l.values, l.velocity, l.bias, l.bias_velocity)] for l in A.layers]
        for L, s in zip(T.layers, start):     # the twin's gradients at the same weights
            L.values.copy_(s[0]); L.bias.copy_(s[2])
            nb.sparse_linear_sync_values(L.handle)
        T.train_step(X, labels, batch, lr, mu)
        A.train_step_clipped(X, labels, batch, lr, mu, max_norm)
        g = [(T.view("g", l, batch).clone(), T.view("db", l, batch).clone()) for l in range(n)]
        for l in range(n):
            assert torch.equal(A.view("g", l, batch), g[l][0]) and torch.equal(A.view("db", l, batch), g[l][1])
        assert float(A.loss) == float(T.loss)
        want = norm_of([x for pair in g for x in pair])
        assert abs(float(A.norm) - want) <= want * U * 1.001
        c = min(1.0, float(np.float32(max_norm)) / want)
        assert (c < 1) == (max_norm < 1e3)
        for L, (w, v, b, bv), (gw, gb) in zip(A.layers, start, g):
            for now, vel, old, oldv, grad in ((L.values, L.velocity, w, v, gw), (L.bias, L.bias_velocity, b, bv, gb)):
                rw, rv, ew, ev = steps(old, oldv, grad, lr, mu, c, flags & 2)
                assert np.all(np.abs(now.cpu().numpy() - rw) <= ew) and np.all(np.abs(vel.cpu().numpy() - rv) <= ev)
    # a step with a batch that holds no number leaves the state
    X = X.clone()
    X[3, 5] = float("nan")
    before = [x.clone() for L in A.layers for x in (L.values, L.velocity, L.bias, L.bias_velocity)]
    A.train_step_clipped(X, labels, batch, lr, mu, 1.0)
    assert torch.isnan(A.norm).all()
    assert all(torch.equal(a, b) for a, b in zip(before, [x for L in A.layers for x in (L.values, L.velocity, L.bias, L.bias_velocity)]))
    A.close(); T.close()

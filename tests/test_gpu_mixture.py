"""A mixture of sparse layers from end to end: router, experts and output layer trained with clipped gradients, the calls
strung together as a program would, against the same in 64 bits with dense matrices; and captured in a graph."""
import numpy as np
import pytest

import mixture_reference as ref
from paper_2407_17437_amd import workloads as wl

pytestmark = pytest.mark.gpu

F, H, E, K, CLASSES, BATCH, CAPACITY = 40, 24, 6, 2, 10, 90, 30   # (30 places an expert, which is the mean of its choices: some are dropped, some places stay empty)
LR, MU, MAX_NORM, SCALE = 0.05, 0.9, 0.5, 1.25


@pytest.fixture(scope="module")
def nb():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2407_17437_amd import binding
    return binding


def layer(rows, cols, density, relu, seed):
    rng = np.random.default_rng(seed)
    mask = rng.random((rows, cols)) < density
    indptr = np.concatenate([[0], mask.sum(1).cumsum()]).astype(np.int32)
    indices = np.nonzero(mask)[1].astype(np.int32)
    values = (rng.standard_normal(indices.size) * np.sqrt(2 / max(1, density * cols))).astype(np.float32)
    return wl.SparseLayerData(rows, cols, indptr, indices, values, (0.1 * rng.standard_normal(rows)).astype(np.float32), relu)


class Mixture:
    """router (E, F) -> experts (H, F) -> output (CLASSES, H); buffers for one batch size."""

    def __init__(self, nb, flags):
        import torch
        self.nb, self.flags = nb, flags
        data = [layer(E, F, 0.5, False, 1)] + [layer(H, F, 0.3, True, 2 + e) for e in range(E)] + [layer(CLASSES, H, 0.6, False, 99)]
        self.layers = [nb.SparseLinear(d, max_batch=BATCH) for d in data]
        new = lambda rows: torch.zeros(rows, 96, device="cuda")[:, :BATCH]
        self.Z, self.dZ, self.Y, self.dY, self.O, self.dO, self.dX, self.dXr = new(E), new(E), new(H), new(H), new(CLASSES), new(CLASSES), new(F), new(F)
        self.w, self.dw = new(K), new(K)
        self.chosen, self.slots = (torch.zeros(K, 96, dtype=torch.int32, device="cuda")[:, :BATCH] for _ in range(2))
        self.counts = torch.zeros(E, dtype=torch.int32, device="cuda")
        self.bias = torch.linspace(-0.02, 0.02, E, device="cuda")
        self.Xe, self.dXe, self.Ye, self.dYe = (nb.expert_blocks(E, n, CAPACITY) for n in (F, F, H, H))
        self.placement = torch.empty(nb.expert_placement_bytes(E, BATCH, K) // 4, dtype=torch.int32, device="cuda")
        self.room = torch.empty(nb.expert_combine_workspace_bytes(H, BATCH, K) // 4, device="cuda")
        self.g = [torch.zeros(L.nnz, device="cuda") for L in self.layers]
        self.db = [torch.zeros(L.rows, device="cuda") for L in self.layers]
        self.loss, self.norm = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
        self.ws = torch.empty(nb.gradient_norm_workspace_bytes(2 * len(self.layers)) // 4, device="cuda")

    def step(self, X, labels):
        nb, router, experts, out = self.nb, self.layers[0], self.layers[1:-1], self.layers[-1]
        nb.sparse_linear_forward(router.handle, X, self.Z, BATCH)
        nb.expert_route(self.Z, self.bias, E, BATCH, K, 1, 1, self.flags, SCALE, self.chosen, self.w)
        nb.expert_place(self.chosen, E, BATCH, K, CAPACITY, self.slots, self.counts, self.placement)
        nb.expert_dispatch(X, self.placement, F, E, BATCH, K, CAPACITY, self.Xe)
        for e, L in enumerate(experts):
            nb.sparse_linear_forward(L.handle, self.Xe[e], self.Ye[e], CAPACITY)
        nb.expert_combine(self.Ye, self.placement, self.w, H, E, BATCH, K, CAPACITY, self.Y)
        nb.sparse_linear_forward(out.handle, self.Y, self.O, BATCH)
        nb.softmax_cross_entropy(self.O, labels, CLASSES, BATCH, self.dO, self.loss)
        nb.sparse_linear_backward(out.handle, self.Y, None, self.dO, self.dY, self.g[-1], self.db[-1], BATCH)
        nb.expert_combine_backward(self.Ye, self.dY, self.placement, self.w, H, E, BATCH, K, CAPACITY, self.dYe, self.dw, self.room)
        for e, L in enumerate(experts):
            nb.sparse_linear_backward(L.handle, self.Xe[e], self.Ye[e], self.dYe[e], self.dXe[e], self.g[1 + e], self.db[1 + e], CAPACITY)
        nb.expert_combine(self.dXe, self.placement, None, F, E, BATCH, K, CAPACITY, self.dX)
        nb.expert_route_backward(self.Z, self.chosen, self.dw, E, BATCH, K, self.flags, SCALE, self.dZ)
        nb.sparse_linear_backward(router.handle, X, None, self.dZ, self.dXr, self.g[0], self.db[0], BATCH)
        Ls = self.layers
        nb.sgd_update_clipped([L.values for L in Ls] + [L.bias for L in Ls], [L.velocity for L in Ls] + [L.bias_velocity for L in Ls], self.g + self.db,
                              LR, MU, MAX_NORM, True, self.ws, self.norm)

    def state(self):
        return [t for L in self.layers for t in (L.values, L.velocity, L.bias, L.bias_velocity)]


def batch(seed):
    import torch
    rng = np.random.default_rng(seed)
    X = rng.standard_normal((F, BATCH)).astype(np.float32)
    t = torch.zeros(F, 96, device="cuda")[:, :BATCH]
    t.copy_(torch.as_tensor(X))
    labels = rng.integers(0, CLASSES, BATCH).astype(np.int32)
    return X.astype(np.float64), labels, t, torch.as_tensor(labels).cuda()


def dense(L):
    W = np.zeros((L.rows, L.cols))
    indptr, indices, values = (x.cpu().numpy() for x in (L.indptr, L.indices, L.values))
    row = np.repeat(np.arange(L.rows), np.diff(indptr))
    W[row, indices] = values
    return W, L.bias.cpu().numpy().astype(np.float64)[:, None], (row, indices)


@pytest.mark.parametrize("sigmoid,renorm", [(0, 0), (0, 1), (1, 1)])
def test_training_step_of_a_mixture(nb, sigmoid, renorm):
    M = Mixture(nb, nb.NERVA_EXPERT_SIGMOID * sigmoid | nb.NERVA_EXPERT_RENORMALISE * renorm)
    X, labels, Xd, ld = batch(3)
    W = [dense(L) for L in M.layers]
    before = [t.cpu().numpy().astype(np.float64) for t in M.state()]
    M.step(Xd, ld)
    # forward
    Z = W[0][0] @ X + W[0][1]
    chosen, w, _ = ref.route(Z, M.bias.cpu().numpy(), K, 1, 1, sigmoid, renorm, 0, SCALE)
    slots, counts = ref.place(chosen, E, CAPACITY)
    assert counts.max() > CAPACITY and counts.min() < CAPACITY            # some are dropped, some places are empty
    assert np.array_equal(M.chosen.cpu().numpy(), chosen) and np.array_equal(M.slots.cpu().numpy(), slots) and np.array_equal(M.counts.cpu().numpy(), counts)
    Ye = [np.maximum(W[1 + e][0] @ X + W[1 + e][1], 0) for e in range(E)]   # of every column
    on = slots >= 0
    gate = np.zeros((E, BATCH))
    for j, c in zip(*np.nonzero(on)):
        gate[chosen[j, c], c] = w[j, c]
    Y = sum(gate[e] * Ye[e] for e in range(E))
    O = W[-1][0] @ Y + W[-1][1]
    p = np.exp(O - O.max(0))
    p /= p.sum(0)
    loss = -np.log(p[labels, np.arange(BATCH)]).mean()
    # backward
    dO = p.copy()
    dO[labels, np.arange(BATCH)] -= 1
    dO /= BATCH
    grads = {len(W) - 1: (dO @ Y.T, dO.sum(1))}
    dY = W[-1][0].T @ dO
    dX = np.zeros((F, BATCH))
    dw = np.zeros((K, BATCH))
    for e in range(E):
        taken = (gate[e] != 0)
        dpre = gate[e] * dY * (Ye[e] > 0) * taken
        grads[1 + e] = (dpre @ X.T, dpre.sum(1))
        dX += W[1 + e][0].T @ dpre
    for j, c in zip(*np.nonzero(on)):
        dw[j, c] = Ye[chosen[j, c]][:, c] @ dY[:, c]
    dZ, _ = ref.route_loss_gradient(Z, chosen, dw, sigmoid, renorm, SCALE)
    grads[0] = (dZ @ X.T, dZ.sum(1))
    # six products one behind the other of at most 90 terms and 16 roundings more each, and sums of terms that are
    # a few times larger than the largest result
    tol = 6 * (90 + 16) * ref.U * 4
    near = lambda got, want: np.abs(got.cpu().numpy() - want).max() <= tol * np.abs(want).max()
    assert abs(float(M.loss) - loss) <= tol * loss
    assert near(M.Y, Y) and near(M.dY, dY) and near(M.dX, dX) and near(M.dw, dw) and near(M.dZ, dZ)
    flat = []
    for l, (_, _, (row, col)) in enumerate(W):
        g, db = grads[l]
        assert near(M.g[l], g[row, col]) and near(M.db[l], db), l
        flat.append((g[row, col], db))
    norm = np.sqrt(sum((a ** 2).sum() + (b ** 2).sum() for a, b in flat))
    assert abs(float(M.norm) - norm) <= tol * norm
    c = min(1.0, MAX_NORM / norm)
    for l in range(len(W)):
        for i, g in ((0, flat[l][0]), (2, flat[l][1])):
            v = MU * before[4 * l + i + 1] - LR * c * g
            now, vel = M.state()[4 * l + i], M.state()[4 * l + i + 1]
            assert np.abs(vel.cpu().numpy() - v).max() <= tol * LR * np.abs(g).max() + 1e-12
            assert np.abs(now.cpu().numpy() - (before[4 * l + i] + MU * v - LR * c * g)).max() <= 2 * tol * LR * np.abs(g).max() + ref.U * np.abs(before[4 * l + i]).max() + 1e-12


def test_captured_step_of_a_mixture(nb):
    """The whole step in one graph, replayed on changing batches between eager steps of a twin; two graphs of it take turns."""
    import torch
    A, B = Mixture(nb, nb.NERVA_EXPERT_RENORMALISE), Mixture(nb, nb.NERVA_EXPERT_RENORMALISE)
    _, _, X, labels = batch(20)
    A.step(X, labels)
    B.step(X, labels)
    graphs = []
    for _ in range(2):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            A.step(X, labels)
        graphs.append(g)
    for t in range(6):
        _, _, Xt, lt = batch(21 + t)
        X.copy_(Xt)
        labels.copy_(lt)
        graphs[t % 2].replay()
        torch.cuda.synchronize()
        B.step(X, labels)
        torch.cuda.synchronize()
        for a, b in zip(A.state() + [A.loss, A.norm, A.Y, A.dX, A.dZ, A.slots], B.state() + [B.loss, B.norm, B.Y, B.dX, B.dZ, B.slots]):
            assert torch.equal(a, b), t

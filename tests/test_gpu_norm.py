"""Group norm with an activation and dropout, and dropout by itself, against plain forms in 64 bits (label_reference.py)."""
import numpy as np
import pytest

import label_reference as ref

pytestmark = pytest.mark.gpu

SEED, STEP, LAYER = 0x1234567890ABCDEF, 41, 5


@pytest.fixture(scope="module")
def nb():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2407_17437_amd import binding
    return binding


def matrix(array, pad=0, fill=float("nan")):
    """The array on the device with `pad` more columns a row, NaN in them."""
    import torch
    a = np.ascontiguousarray(array, dtype=np.float32)
    full = torch.full((a.shape[0], a.shape[1] + pad), fill, device="cuda")
    full[:, :a.shape[1]] = torch.as_tensor(a).cuda()
    return full[:, :a.shape[1]]


def blank(rows, columns, pad=0):
    return matrix(np.full((rows, columns), np.nan), pad)


def padding_untouched(*ts):
    import torch
    return all(bool(torch.isnan(t.as_strided((t.shape[0], t.stride(0)), t.stride())[:, t.shape[1]:]).all()) for t in ts if t.shape[0] > 1)


def state(seed=SEED, step=STEP):
    import torch
    return torch.tensor([seed, step], dtype=torch.int64, device="cuda")


def workspace(nb, F, G, B):
    import torch
    return torch.full((max(4, nb.group_norm_workspace_bytes(F, G, B) // 4),), float("nan"), device="cuda")


def close(got, want, tol, what):
    got = got.detach().cpu().numpy().astype(np.float64) if hasattr(got, "detach") else got
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.shape, np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3], np.broadcast_to(tol, want.shape)[bad][:3])


def data(rng, F, B, affine=True, offset=0.0):
    X = (rng.standard_normal((F, B)) * (0.5 + rng.random((F, 1))) + 0.5 * rng.standard_normal((F, 1)) + offset).astype(np.float32)
    gamma = (1 + 0.3 * rng.standard_normal(F)).astype(np.float32) if affine else None
    beta = (0.3 * rng.standard_normal(F)).astype(np.float32) if affine else None
    return X, gamma, beta, rng.standard_normal((F, B)).astype(np.float32)


def gpu(v):
    import torch
    return None if v is None else torch.as_tensor(v).cuda()


def both(nb, X, gamma, beta, dY, G, act, drop, pads=(0, 0, 0, 0, 0), eps=1e-5, stream=None):
    import torch
    F, B = X.shape
    x, dy = matrix(X, pads[0]), matrix(dY, pads[1])
    y, dx = blank(F, B, pads[2]), blank(F, B, pads[3])
    mean, rstd = blank(G, B, pads[4]), blank(G, B, pads[4])
    dg, db = torch.full((F,), float("nan"), device="cuda"), torch.full((F,), float("nan"), device="cuda")
    ga, be, st, ws = gpu(gamma), gpu(beta), state(), workspace(nb, F, G, B)
    nb.group_norm_forward(x, ga, be, F, G, B, eps, act, drop, LAYER, st if drop else None, y, mean, rstd, ws, stream)
    nb.group_norm_backward(x, ga, be, mean, rstd, dy, F, G, B, act, drop, LAYER, st if drop else None, dx, dg, db, ws, stream)
    torch.cuda.synchronize()
    assert padding_untouched(x, dy, y, dx, mean, rstd)
    return y, mean, rstd, dx, dg, db


# one row, one column; groups of one row, of odd lengths that start at odd rows; what one work-group holds and a row more, both ways; chunks that
# end inside a pair of rows; batches around the widths of a lane, a tile and a wave
SIZES = [(1, 1, 1), (5, 5, 3), (2, 1, 7), (6, 2, 5), (21, 3, 33), (35, 5, 130), (64, 1, 1), (1024, 16, 1), (1024, 32, 100), (513, 3, 31), (600, 1, 4), (1023, 1, 64),
         (1024, 1, 32), (1025, 1, 66), (2047, 1, 9), (2048, 1, 33), (2049, 1, 40), (2050, 2, 36), (4097, 1, 3), (8190, 2, 37), (9001, 1, 2), (64, 8, 2100)]


@pytest.mark.parametrize("F,G,B", SIZES)
def test_norm_against_64_bits(nb, F, G, B):
    rng = np.random.default_rng(F * 7 + B)
    k = SIZES.index((F, G, B))
    for act, drop, affine in ((k % 3, 0.0, True), ((k + 1) % 3, 0.25, k % 2 == 0), (2, 0.1, True)):
        X, gamma, beta, dY = data(rng, F, B, affine)
        pads = [(0, 0, 0, 0, 0), (3, 1, 0, 7, 2), (-B % 32,) * 5][k % 3]
        factor = ref.factors(F, B, drop, LAYER, SEED, STEP)
        want = ref.Norm(X, gamma, beta, G, 1e-5, act, factor, dY)
        y, mean, rstd, dx, dg, db = both(nb, X, gamma, beta, dY, G, act, drop, pads)
        close(y, want.Y, want.Y_tol, "Y")
        close(mean, want.mean, want.mean_tol, "mean")
        close(rstd, want.rstd, want.rstd_tol, "rstd")
        assert np.array_equal((y.cpu().numpy() == 0) | (factor > 0), np.ones((F, B), bool)), "a dropped entry that is not 0"
        if act == 1:
            # the gradient goes by the output's sign, which only arguments within their rounding of 0 may have wrong
            positive = y.cpu().numpy() > 0
            sure = (np.abs(want.u) > want.Y_tol / np.maximum(factor, 1)) & (factor > 0)
            assert np.array_equal(positive[sure], want.u[sure] > 0)
            want = ref.Norm(X, gamma, beta, G, 1e-5, act, factor, dY, positive)
        close(dx, want.dX, want.dX_tol, "dX")
        close(dg, want.dgamma, want.dgamma_tol, "dgamma")
        close(db, want.dbeta, want.dbeta_tol, "dbeta")


def test_groups_of_very_many_chunks(nb):
    """Chunks whose sums a launch of its own adds up."""
    rng = np.random.default_rng(12)
    F, G, B = 160003, 1, 40
    X, gamma, beta, dY = data(rng, F, B, offset=3.0)
    want = ref.Norm(X, gamma, beta, G, 1e-5, 2, ref.factors(F, B, 0.1, LAYER, SEED, STEP), dY)
    y, mean, rstd, dx, dg, db = both(nb, X, gamma, beta, dY, G, 2, 0.1, (0, 3, 0, 1, 2))
    for got, name in ((y, "Y"), (mean, "mean"), (rstd, "rstd"), (dx, "dX"), (dg, "dgamma"), (db, "dbeta")):
        close(got, getattr(want, name), getattr(want, name + "_tol"), name)
    F, G, B = 2 * 60000, 2, 9
    X, gamma, beta, dY = data(rng, F, B)
    want = ref.Norm(X, gamma, beta, G, 1e-5, 1, np.ones((F, B)))
    y, *_ = both(nb, X, gamma, beta, dY, G, 1, 0.0)
    close(y, want.Y, want.Y_tol, "Y")


# what a work-group holds at most, both ways, and a pair of rows more, in tiles that are not narrowed; tiles that few rows widen
@pytest.mark.parametrize("F,G,B", [(512, 1, 8200), (1024, 1, 8201), (1026, 1, 8200), (2048, 1, 8193), (2052, 2, 4100), (256, 128, 4099), (130, 65, 5000)])
def test_norm_of_many_columns(nb, F, G, B):
    rng = np.random.default_rng(F + B)
    X, gamma, beta, dY = data(rng, F, B)
    want = ref.Norm(X, gamma, beta, G, 1e-5, 2, ref.factors(F, B, 0.1, LAYER, SEED, STEP), dY)
    y, mean, rstd, dx, dg, db = both(nb, X, gamma, beta, dY, G, 2, 0.1, (0, 3, 0, 1, 2))
    for got, name in ((y, "Y"), (mean, "mean"), (rstd, "rstd"), (dx, "dX")):
        close(got, getattr(want, name), getattr(want, name + "_tol"), name)
    # (sums over the columns: some hundred terms one after the other, of the columns' tiles, in a thread, then the slabs)
    for got, name in ((dg, "dgamma"), (db, "dbeta")):
        close(got, getattr(want, name), getattr(want, name + "_tol") * (1 + B / 1000), name)


def test_relu_is_taken_from_the_same_number_both_ways(nb):
    """Entries whose argument is 0, and many close to it: dbeta counts the columns whose output is positive."""
    rng = np.random.default_rng(4)
    F, G, B = 96, 4, 500
    X, _, _, _ = data(rng, F, B)
    X[:, ::7] = np.round(X[:, ::7])
    X[:, 3] = 2.0                                # (all arguments 0)
    y, _, _, dx, dg, db = both(nb, X, None, None, np.ones((F, B), np.float32), G, 1, 0.0)
    assert np.array_equal(db.cpu().numpy(), (y > 0).sum(1).float().cpu().numpy())
    assert float(y[:, 3].abs().max()) == 0 and float(dx[:, 3].abs().max()) == 0


def test_numbers_far_from_zero(nb):
    """A mean 10^4 times the spread: sums of squares without the mean would leave nothing.  An entry 10^4 times the others first in its group."""
    rng = np.random.default_rng(5)
    for F, G, B in ((64, 2, 40), (6000, 1, 40)):
        X, gamma, beta, dY = data(rng, F, B, offset=1e4)
        want = ref.Norm(X, gamma, beta, G, 1e-5, 0, np.ones((F, B)), dY)
        y, mean, rstd, dx, dg, db = both(nb, X, gamma, beta, dY, G, 0, 0.0)
        close(y, want.Y, want.Y_tol, "Y"), close(rstd, want.rstd, want.rstd_tol, "rstd"), close(dx, want.dX, want.dX_tol, "dX")
        X, gamma, beta, dY = data(rng, F, B)
        X[0] = 1e4
        want = ref.Norm(X, gamma, beta, G, 1e-5, 2, np.ones((F, B)), dY)
        y, mean, rstd, dx, dg, db = both(nb, X, gamma, beta, dY, G, 2, 0.0)
        close(y, want.Y, want.Y_tol, "Y"), close(rstd, want.rstd, want.rstd_tol, "rstd"), close(dx, want.dX, want.dX_tol, "dX")


def test_constant_groups_and_numbers_that_are_none(nb):
    rng = np.random.default_rng(6)
    for F, G, B in ((48, 3, 70), (4500, 2, 9)):
        X, gamma, beta, dY = data(rng, F, B)
        m = F // G
        X[:m, 4] = 3.25
        X[m, 5], X[m + 1, 6], X[m + 2, 7] = np.nan, np.inf, -np.inf
        y, mean, rstd, dx, dg, db = (t.cpu().numpy() for t in both(nb, X, gamma, beta, dY, G, 2, 0.0))
        assert np.allclose(rstd[0, 4], 1e-5 ** -0.5, rtol=1e-6) and np.all(np.abs(y[:m, 4] - ref.act_of(beta[:m].astype(np.float64), 2)) < 1e-6)
        for c in (5, 6, 7):
            assert np.isnan(y[m:2 * m, c]).all() and np.isnan(dx[m:2 * m, c]).all()
        ok = np.ones((F, B), bool)
        ok[m:2 * m, 5:8] = False
        assert np.isfinite(y[ok]).all() and np.isfinite(dx[ok]).all()
        assert np.isfinite(dg[:m]).all() and np.isnan(dg[m:2 * m]).all()
        other = both(nb, np.where(ok, X, 1), gamma, beta, dY, G, 2, 0.0)
        assert np.array_equal(other[0].cpu().numpy()[ok], y[ok]) and np.array_equal(other[3].cpu().numpy()[ok], dx[ok])


@pytest.mark.parametrize("F,G,B", [(40, 5, 70), (3001, 1, 23)])
def test_in_place_and_without_what_is_optional(nb, F, G, B):
    import torch
    rng = np.random.default_rng(7)
    X, gamma, beta, dY = data(rng, F, B)
    y, mean, rstd, dx, dg, db = both(nb, X, gamma, beta, dY, G, 2, 0.25)
    x, dy, ws = matrix(X, 5), matrix(dY, 2), workspace(nb, F, G, B)
    nb.group_norm_forward(x, gpu(gamma), gpu(beta), F, G, B, 1e-5, 2, 0.25, LAYER, state(), x, None, None, ws)
    assert torch.equal(x, y) and padding_untouched(x)
    nb.group_norm_backward(matrix(X), gpu(gamma), gpu(beta), mean, rstd, dy, F, G, B, 2, 0.25, LAYER, state(), dy, None, None, ws)
    assert torch.equal(dy, dx) and padding_untouched(dy)
    one = torch.full((F,), float("nan"), device="cuda")
    nb.group_norm_backward(matrix(X), gpu(gamma), gpu(beta), mean, rstd, matrix(dY), F, G, B, 2, 0.25, LAYER, state(), blank(F, B), None, one, ws)
    assert torch.equal(one, db)
    nb.group_norm_backward(matrix(X), gpu(gamma), gpu(beta), mean, rstd, matrix(dY), F, G, B, 2, 0.25, LAYER, state(), blank(F, B), one, None, ws)
    assert torch.equal(one, dg)


def test_gradients_against_differences(nb):
    """The kernel's gradients along directions against differences of the reference's forward pass in 64 bits."""
    rng = np.random.default_rng(8)
    for F, G, B in ((60, 4, 30), (2200, 1, 30)):
        X, gamma, beta, dY = data(rng, F, B)
        factor = ref.factors(F, B, 0.2, LAYER, SEED, STEP)
        _, _, _, dx, dg, db = (t.cpu().numpy().astype(np.float64) for t in both(nb, X, gamma, beta, dY, G, 2, 0.2))
        tol = ref.Norm(X, gamma, beta, G, 1e-5, 2, factor, dY)

        def value(h, vx=0, vg=0, vb=0):
            return (ref.Norm(X + h * vx, gamma + h * vg, beta + h * vb, G, 1e-5, 2, factor).Y * dY).sum()
        for name, grad, bound in (("vx", dx, tol.dX_tol), ("vg", dg, tol.dgamma_tol), ("vb", db, tol.dbeta_tol)):
            v = rng.standard_normal(grad.shape)
            d = (value(1e-5, **{name: v}) - value(-1e-5, **{name: v})) / 2e-5
            # (differences: third derivatives below 10 here, over 1e-10, and the cancellation of 64-bit sums)
            assert abs(d - (grad * v).sum()) < (bound * np.abs(v)).sum() + 1e-6 * (1 + np.abs(grad * v).sum()), name


def test_same_bits_again_and_on_another_stream(nb):
    import torch
    rng = np.random.default_rng(9)
    for F, G, B in ((128, 4, 3000), (5000, 1, 200)):
        X, gamma, beta, dY = data(rng, F, B)
        first = both(nb, X, gamma, beta, dY, G, 2, 0.1)
        again = both(nb, X, gamma, beta, dY, G, 2, 0.1, pads=(1, 0, 3, 2, 0))
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            third = both(nb, X, gamma, beta, dY, G, 2, 0.1)
        for a, b, c in zip(first, again, third):
            assert torch.equal(a, b) and torch.equal(a, c)


# ---- dropout

@pytest.mark.parametrize("F,B,drop,pads", [(1, 1, 0.5, (0, 0)), (2, 3, 0.5, (1, 2)), (7, 5, 0.1, (0, 0)), (33, 64, 0.9, (0, 4)), (1024, 100, 0.5, (28, 28)), (101, 257, 0.25, (0, 0)),
                                           (3, 5000, 0.999, (5, 0)), (9, 77, 1e-9, (0, 1)), (9, 77, 0.0, (0, 1)), (64, 64, 0.9999999, (0, 0))])
def test_dropout(nb, F, B, drop, pads):
    import torch
    rng = np.random.default_rng(F + B)
    X = rng.standard_normal((F, B)).astype(np.float32)
    X.flat[0] = np.nan
    x, y = matrix(X, pads[0]), blank(F, B, pads[1])
    nb.dropout(x, F, B, drop, LAYER, state() if drop else None, y)
    factor = ref.factors(F, B, drop, LAYER, SEED, STEP)
    want = np.where(factor > 0, (X * np.float32(factor.max() if factor.any() else 0)).astype(np.float32), np.float32(0))
    assert np.array_equal(y.cpu().numpy(), want, equal_nan=True) and padding_untouched(x, y)
    nb.dropout(x, F, B, drop, LAYER, state() if drop else None, x)
    assert torch.equal(torch.nan_to_num(x), torch.nan_to_num(y)) and padding_untouched(x)


def test_masks_follow_seed_step_and_layer_but_not_the_batch(nb):
    import torch
    F, B = 64, 200
    x = torch.ones(F, B, device="cuda")

    def mask(F=F, B=B, layer=LAYER, **kw):
        y = blank(F, B)
        nb.dropout(x[:F, :B], F, B, 0.5, layer, state(**kw), y)
        return y > 0
    m = mask()
    assert torch.equal(m[:33, :77], mask(33, 77)) and torch.equal(m, mask(step=STEP + 2 ** 32))
    for kw in (dict(seed=SEED + 1), dict(seed=SEED - 2 ** 40), dict(step=STEP + 1), dict(layer=LAYER + 1), dict(layer=-1), dict(seed=-SEED)):
        other = mask(**kw)
        assert 0.4 < float((m == other).float().mean()) < 0.6, kw
    assert np.array_equal(mask(layer=-1).cpu().numpy(), ref.factors(F, B, 0.5, -1, SEED, STEP) > 0)
    assert np.array_equal(mask(seed=-5).cpu().numpy(), ref.factors(F, B, 0.5, LAYER, -5 % 2 ** 64, STEP) > 0)


def test_captured_steps_go_on_drawing(nb):
    """Norm, dropout and their backward passes in a graph that raises the step: every replay gives what the same calls give outside."""
    import torch
    rng = np.random.default_rng(10)
    F, G, B = 1500, 3, 70
    X, gamma, beta, dY = data(rng, F, B)
    x, dy, ga, be, st, ws = matrix(X), matrix(dY), gpu(gamma), gpu(beta), state(), workspace(nb, F, G, B)
    bufs = [blank(F, B), blank(G, B), blank(G, B), blank(F, B), torch.zeros(F, device="cuda"), torch.zeros(F, device="cuda"), blank(F, B)]

    def calls(st, y, mean, rstd, dx, dg, db, z):
        nb.group_norm_forward(x, ga, be, F, G, B, 1e-5, 2, 0.25, 0, st, y, mean, rstd, ws)
        nb.dropout(y, F, B, 0.5, 1, st, z)
        nb.group_norm_backward(x, ga, be, mean, rstd, dy, F, G, B, 2, 0.25, 0, st, dx, dg, db, ws)
    calls(st, *bufs)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls(st, *bufs)
        st[1] += 1
    for k in range(3):
        g.replay()
        torch.cuda.synchronize()
        got = [b.clone() for b in bufs]
        other = [torch.zeros_like(b) for b in bufs]
        calls(state(step=STEP + k), *other)
        for a, b in zip(got, other):
            assert torch.equal(a, b), k
        assert int(st[1]) == STEP + k + 1


def test_rows_far_apart(nb):
    """Rows 2^26 entries apart: offsets beyond 32 bits."""
    import torch
    F, G, B, ld = 70, 2, 33, 1 << 26
    rng = np.random.default_rng(11)
    X, gamma, beta, dY = data(rng, F, B)
    memory = torch.empty(F * ld, device="cuda")
    x = memory.as_strided((F, B), (ld, 1))
    other = memory.as_strided((F, B), (ld, 1), 4096)
    x.copy_(torch.as_tensor(X))
    y, mean, rstd, dx, dg, db = both(nb, X, gamma, beta, dY, G, 2, 0.1)
    m2, r2, ws = blank(G, B), blank(G, B), workspace(nb, F, G, B)
    nb.group_norm_forward(x, gpu(gamma), gpu(beta), F, G, B, 1e-5, 2, 0.1, LAYER, state(), other, m2, r2, ws)
    assert torch.equal(other, y)
    other.copy_(torch.as_tensor(dY))
    nb.group_norm_backward(x, gpu(gamma), gpu(beta), m2, r2, other, F, G, B, 2, 0.1, LAYER, state(), other, dg, db, ws)
    assert torch.equal(other, dx)
    nb.dropout(x, F, B, 0.5, LAYER, state(), other)
    z = blank(F, B)
    nb.dropout(matrix(X), F, B, 0.5, LAYER, state(), z)
    assert torch.equal(other, z)

"""Routing to experts, places, and the exchange of columns with the experts' blocks against plain forms (mixture_reference.py)."""
import numpy as np
import pytest

import mixture_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nb():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2407_17437_amd import binding
    return binding


def device_matrix(array, ld=None, dtype=None):
    """The array on the device with rows `ld` apart; NaN (or 7) in the padding."""
    import torch
    t = torch.as_tensor(np.ascontiguousarray(array))
    ld = ld or t.shape[1]
    full = torch.full((t.shape[0], ld), float("nan") if t.dtype == torch.float32 else 7, dtype=t.dtype, device="cuda")
    full[:, :t.shape[1]] = t.cuda()
    return full[:, :t.shape[1]]


def blocks(nb, array=None, shape=None, ld=None):
    import torch
    E, F, C = shape if array is None else array.shape
    t = nb.expert_blocks(E, F, C, ld=ld)
    if array is not None:
        t.copy_(torch.as_tensor(array))
    return t


def padding_untouched(t):
    import torch
    width = t.stride(-2)
    if width == t.shape[-1]:
        return True
    full = t.as_strided((*t.shape[:-1], width), t.stride())[..., t.shape[-1]:]
    return bool(torch.isnan(full).all()) if t.dtype == torch.float32 else bool((full == 7).all())


def logits(rng, E, B, kind):
    Z = rng.standard_normal((E, B)).astype(np.float32)
    if kind == "masked":
        Z[rng.random((E, B)) < 0.3] = -np.inf
        Z[:, rng.random(B) < 0.1] = -np.inf
        Z[:, B // 2] = -np.inf
    elif kind == "ties":
        Z = np.round(Z)
    elif kind == "wide":
        Z *= 30
    elif kind == "lowest":
        Z[rng.random((E, B)) < 0.5] = np.finfo(np.float32).min
        Z[:, 0] = np.finfo(np.float32).min
    return Z


ROUTES = [  # experts, batch, k, groups, top_groups
    (1, 1, 1, 1, 1), (2, 3, 2, 1, 1), (5, 64, 3, 1, 1), (8, 65, 2, 1, 1), (8, 130, 2, 4, 2), (60, 77, 4, 6, 3), (64, 1, 6, 8, 3), (64, 600, 8, 64, 9), (65, 33, 5, 5, 1),
    (128, 40, 1, 1, 1), (129, 31, 9, 1, 1), (256, 517, 8, 8, 4), (257, 20, 17, 1, 1), (513, 9, 4, 27, 5), (1024, 12, 32, 16, 7), (32, 50, 32, 1, 1), (7, 2100, 2, 7, 2),
    (64, 8200, 6, 8, 2),
]


@pytest.mark.parametrize("E,B,k,groups,top", ROUTES)
@pytest.mark.parametrize("sigmoid,renorm,bias,pair", [(0, 0, 0, 0), (0, 1, 1, 0), (1, 1, 1, 1), (1, 0, 0, 0), (0, 0, 1, 1), (1, 1, 0, 0), (0, 1, 0, 0)])
def test_route(nb, E, B, k, groups, top, sigmoid, renorm, bias, pair):
    import torch
    rng = np.random.default_rng(E * 1000 + B + 7 * sigmoid + 3 * renorm)
    for n, kind in enumerate(("plain", "masked", "ties", "wide", "lowest") if B < 1000 else ("masked",)):
        Z = logits(rng, E, B, kind)
        b = (0.3 * rng.standard_normal(E)).astype(np.float32) if bias else None
        scale = (1.0, 2.5)[n % 2]
        want, weights, bound = ref.route(Z, b, k, groups, top, sigmoid, renorm, pair, scale)
        flags = nb.NERVA_EXPERT_SIGMOID * sigmoid | nb.NERVA_EXPERT_RENORMALISE * renorm | nb.NERVA_EXPERT_GROUP_PAIR * pair
        ld = B + (0, 5, 32)[n % 3]
        Zd = device_matrix(Z, ld)
        chosen, w = device_matrix(np.zeros((k, B), np.int32), ld + 1), device_matrix(np.zeros((k, B), np.float32), ld + 1)
        nb.expert_route(Zd, None if b is None else torch.as_tensor(b).cuda(), E, B, k, groups, top, flags, scale, chosen, w)
        got, gw = chosen.cpu().numpy(), w.cpu().numpy().astype(np.float64)
        assert np.array_equal(got, want), (kind, np.argwhere(got != want)[:4])
        assert np.all(np.abs(gw - weights) <= bound), (kind, np.abs(gw - weights).max())
        assert padding_untouched(chosen) and padding_untouched(w)


@pytest.mark.parametrize("E,B,k,groups,top,sigmoid,renorm,bias,pair", [
    (16, 6200, 2, 1, 1, 0, 0, 0, 0), (1, 6150, 1, 1, 1, 1, 1, 1, 0), (130, 6500, 7, 1, 1, 0, 1, 1, 0), (256, 6144, 8, 8, 4, 1, 1, 1, 1), (7, 6145, 1, 7, 3, 0, 0, 0, 1),
    (1000, 6144, 4, 8, 5, 0, 0, 1, 1), (45, 6201, 8, 3, 2, 1, 0, 0, 1), (60, 6150, 5, 15, 9, 0, 1, 0, 0), (40, 6144, 3, 1, 1, 0, 1, 0, 0), (96, 6144, 9, 1, 1, 1, 1, 1, 0),
    (34, 6160, 4, 17, 6, 0, 0, 1, 1)])
def test_route_of_many_columns(nb, E, B, k, groups, top, sigmoid, renorm, bias, pair):
    import torch
    rng = np.random.default_rng(E + B + k)
    Z = logits(rng, E, B, "masked")
    Z[:, 3000:] = np.round(Z[:, 3000:] * (1 if not (bias or pair) else 4096)) / (1 if not (bias or pair) else 4096)
    Z[rng.integers(0, E, 5), rng.integers(0, B, 5)] = np.nan
    Z[rng.integers(0, E, 5), rng.integers(0, B, 5)] = np.inf
    Z[:, 17] = np.finfo(np.float32).min
    b = (0.3 * rng.standard_normal(E)).astype(np.float32) if bias else None
    if bias and E > 8:
        b[3], b[5], b[6] = -np.inf, np.nan, np.inf
    want, weights, bound = ref.route(Z, b, k, groups, top, sigmoid, renorm, pair, 1.5)
    flags = nb.NERVA_EXPERT_SIGMOID * sigmoid | nb.NERVA_EXPERT_RENORMALISE * renorm | nb.NERVA_EXPERT_GROUP_PAIR * pair
    chosen, w = device_matrix(np.zeros((k, B), np.int32), B + 3), device_matrix(np.zeros((k, B), np.float32), B + 3)
    nb.expert_route(device_matrix(Z, B + 1), None if b is None else torch.as_tensor(b).cuda(), E, B, k, groups, top, flags, 1.5, chosen, w)
    got, gw = chosen.cpu().numpy(), w.cpu().numpy().astype(np.float64)
    assert np.array_equal(got, want), np.argwhere(got != want)[:4]
    assert np.array_equal(np.isnan(gw), np.isnan(weights)) and np.all(np.isnan(weights) | (np.abs(gw - weights) <= bound))
    assert padding_untouched(chosen) and padding_untouched(w)


@pytest.mark.parametrize("E,B,k,groups,top,sigmoid,renorm,bias,pair", [
    (128, 2048, 5, 1, 1, 0, 1, 0, 0), (256, 4096, 8, 16, 5, 0, 1, 1, 1), (1000, 2049, 8, 8, 5, 0, 0, 1, 1), (129, 3001, 6, 3, 2, 1, 0, 0, 1), (200, 2500, 7, 1, 1, 1, 1, 1, 0),
    (128, 2047, 5, 1, 1, 1, 1, 1, 0), (127, 2048, 5, 1, 1, 0, 1, 0, 0), (15, 4608, 2, 5, 2, 1, 0, 0, 1), (15, 4609, 2, 5, 2, 1, 0, 0, 1), (64, 4097, 6, 8, 2, 1, 1, 0, 0), (256, 8192, 8, 8, 4, 1, 1, 1, 1),
    (300, 4133, 1, 1, 1, 0, 0, 0, 0), (16, 8193, 2, 1, 1, 0, 1, 0, 0), (1, 8200, 1, 1, 1, 1, 1, 1, 0), (130, 9000, 7, 1, 1, 0, 1, 1, 0), (256, 16384, 8, 8, 4, 1, 1, 1, 1),
    (45, 12001, 4, 3, 2, 1, 0, 0, 1), (40, 16385, 3, 1, 1, 0, 1, 0, 0), (40, 16385, 3, 1, 1, 0, 1, 1, 0), (77, 20001, 8, 7, 4, 0, 0, 1, 1)])
def test_route_of_many_columns_in_work_groups_of_every_size(nb, E, B, k, groups, top, sigmoid, renorm, bias, pair):
    test_route_of_many_columns(nb, E, B, k, groups, top, sigmoid, renorm, bias, pair)


@pytest.mark.parametrize("B", [3, 6200])
def test_route_by_scores_far_out(nb, B):
    """Sums of two scores whose logits lie where a sigmoid of 32 bits, or the exponential in it, has left its range."""
    import torch
    E = 16
    z = np.array([-720, -700, -690.5, -650, -100, -89, -20, -1, 0, 1, 17, 36, -708, np.finfo(np.float32).min, -np.inf, -30], np.float32)
    rng = np.random.default_rng(1)
    Z = np.stack([rng.permutation(z) for _ in range(B)], 1)
    for groups, top, k in ((8, 3, 6), (4, 2, 8)):
        want, weights, bound = ref.route(Z, None, k, groups, top, 1, 0, 1, 1.0)
        chosen, w = device_matrix(np.zeros((k, B), np.int32)), device_matrix(np.zeros((k, B), np.float32))
        nb.expert_route(device_matrix(Z), None, E, B, k, groups, top, nb.NERVA_EXPERT_SIGMOID | nb.NERVA_EXPERT_GROUP_PAIR, 1.0, chosen, w)
        # Scores are compared in 42 bits, and some sums here are nearly equal: 1/(1+e) + e/(1+e) = 1 and 1/(1+exp(-36)) = 1 - 2.3e-16.  A key is cut
        # by less than 2^-42 of it, so is the sum of two cut keys, and two such sums are compared: nearer than 2^-40, and not equal, either may win.
        with np.errstate(over="ignore"):
            z = Z.astype(np.float64)
            key = np.sort(np.where(z >= 0, 1 / (1 + np.exp(-z)), np.exp(z) / (1 + np.exp(z))).reshape(groups, E // groups, B), axis=1)
        score = np.sort(key[:, -1] + key[:, -2], axis=0)
        gap = np.diff(score, axis=0)
        clear = ~((gap > 0) & (gap < 2.0 ** -40 * score[1:])).any(0)
        assert clear.mean() > 0.5
        assert np.array_equal(chosen.cpu().numpy()[:, clear], want[:, clear])
        assert np.all(np.abs(w.cpu().numpy() - weights)[:, clear] <= bound[:, clear])


def test_route_of_logits_that_are_no_numbers(nb):
    """NaN is not chosen and shows in the column's weights; +inf likewise under a softmax and the best score under a sigmoid."""
    import torch
    rng = np.random.default_rng(5)
    Z = rng.standard_normal((10, 6)).astype(np.float32)
    Z[3, 1], Z[4, 2], Z[:, 3], Z[0, 4], Z[1, 4] = np.nan, np.inf, np.nan, np.inf, np.nan
    Z[:, 5] = -np.inf
    b = np.zeros(10, np.float32)
    b[2], b[7], b[8] = -np.inf, np.nan, np.inf
    for sigmoid in (0, 1):
        for bias in (None, b):
            for renorm in (0, 1):
                want, weights, bound = ref.route(Z, bias, 4, 1, 1, sigmoid, renorm, 0, 1.0)
                chosen, w = torch.zeros(4, 6, dtype=torch.int32, device="cuda"), torch.zeros(4, 6, device="cuda")
                nb.expert_route(torch.as_tensor(Z).cuda(), None if bias is None else torch.as_tensor(bias).cuda(), 10, 6, 4, 1, 1, sigmoid | 2 * renorm, 1.0, chosen, w)
                got = w.cpu().numpy().astype(np.float64)
                assert np.array_equal(chosen.cpu().numpy(), want), (sigmoid, renorm)
                assert np.array_equal(np.isnan(got), np.isnan(weights)) and np.all(np.isnan(weights) | (np.abs(got - weights) <= bound))
                assert np.isnan(got[:, 1]).all() and not np.isnan(got[:, 5]).any() and (chosen[:, 5] == -1).all()


@pytest.mark.parametrize("E,B,k,groups,top", ROUTES)
@pytest.mark.parametrize("sigmoid,renorm", [(0, 0), (0, 1), (1, 0), (1, 1)])
def test_route_backward(nb, E, B, k, groups, top, sigmoid, renorm):
    rng = np.random.default_rng(E + B)
    for n, kind in enumerate(("plain", "masked", "wide") if B < 1000 else ("masked",)):
        Z = logits(rng, E, B, kind)
        chosen, _, _ = ref.route(Z, None, k, groups, top, sigmoid, renorm, 0, 1.5)
        d = rng.standard_normal((k, B)).astype(np.float32)
        d[chosen < 0] = np.nan          # not read
        want, bound = ref.route_loss_gradient(Z, chosen, d, sigmoid, renorm, 1.5)
        ld = B + (0, 3)[n % 2]
        dZ = device_matrix(np.full((E, B), np.nan, np.float32), B + 2)
        nb.expert_route_backward(device_matrix(Z, ld), device_matrix(chosen, ld), device_matrix(d, ld), E, B, k, sigmoid | 2 * renorm, 1.5, dZ)
        got = dZ.cpu().numpy().astype(np.float64)
        assert np.all(np.abs(got - want) <= bound), (kind, np.abs(got - want).max())
        if renorm or sigmoid:
            off = np.ones((E, B), bool)
            for j in range(k):
                on = chosen[j] >= 0
                off[chosen[j, on], np.nonzero(on)[0]] = False
            assert (got[off] == 0).all()
        assert padding_untouched(dZ)


@pytest.mark.parametrize("sigmoid,renorm", [(0, 0), (0, 1), (1, 0), (1, 1)])
def test_route_gradient_against_differences(nb, sigmoid, renorm):
    """Central differences of the 64-bit form with the choices held fixed: their error is of the order of h^2 = 1e-8."""
    rng = np.random.default_rng(17)
    E, B, k, h = 9, 5, 3, 1e-4
    Z = rng.standard_normal((E, B)).astype(np.float32)
    chosen, _, _ = ref.route(Z, None, k, 1, 1, sigmoid, renorm, 0, 1.5)
    d = rng.standard_normal((k, B)).astype(np.float32)

    def loss(Z):
        s = 1 / (1 + np.exp(-Z)) if sigmoid else np.exp(Z) / np.exp(Z).sum(0)
        w = np.take_along_axis(s, chosen.astype(int), 0)
        return 1.5 * (d * (w / w.sum(0) if renorm else w)).sum()

    want = np.zeros((E, B))
    for e in range(E):
        for c in range(B):
            step = np.zeros((E, B))
            step[e, c] = h
            want[e, c] = (loss(Z + step) - loss(Z - step)) / (2 * h)
    dZ = device_matrix(np.zeros((E, B), np.float32))
    nb.expert_route_backward(device_matrix(Z), device_matrix(chosen), device_matrix(d), E, B, k, sigmoid | 2 * renorm, 1.5, dZ)
    assert np.abs(dZ.cpu().numpy() - want).max() <= 2e-6


def test_route_backward_of_one_expert_twice_and_of_none(nb):
    """Choices that no router makes: the same expert twice in a column adds up, an expert out of range is left out."""
    rng = np.random.default_rng(3)
    E, B, k = 12, 70, 5
    Z = rng.standard_normal((E, B)).astype(np.float32)
    chosen = rng.integers(0, E, (k, B)).astype(np.int32)
    chosen[1, ::3] = chosen[0, ::3]
    chosen[2, ::4], chosen[3, ::5], chosen[4, ::7] = E, -5, 2 ** 31 - 1
    d = rng.standard_normal((k, B)).astype(np.float32)
    for sigmoid, renorm in ((0, 0), (0, 1), (1, 0), (1, 1)):
        want, bound = ref.route_loss_gradient(Z, chosen, d, sigmoid, renorm, 1.0)
        dZ = device_matrix(np.zeros((E, B), np.float32))
        nb.expert_route_backward(device_matrix(Z), device_matrix(chosen), device_matrix(d), E, B, k, sigmoid | 2 * renorm, 1.0, dZ)
        assert np.all(np.abs(dZ.cpu().numpy() - want) <= bound)


PLACES = [  # experts, features, batch, k, capacity
    (1, 1, 1, 1, 1), (3, 5, 2, 2, 1), (8, 64, 100, 2, 30), (60, 33, 77, 4, 6), (64, 17, 4, 6, 4), (16, 40, 256, 2, 64), (16, 40, 257, 2, 20), (5, 16, 1023, 3, 700),
    (7, 7, 1025, 1, 100), (256, 20, 1500, 8, 60), (1024, 9, 300, 32, 12), (4, 130, 2300, 3, 2300), (33, 18, 64, 33 - 1, 70),
]


def choices(rng, E, B, k, kind):
    if kind == "routed":
        return np.argsort(rng.standard_normal((E, B)) + rng.standard_normal((E, 1)), axis=0)[:k].astype(np.int32)
    chosen = rng.integers(-1, E + 1, (k, B)).astype(np.int32)      # twice the same, and none (-1 and E)
    if kind == "one expert":
        chosen[:] = E - 1
    return chosen


@pytest.mark.parametrize("kind", ["routed", "any", "one expert"])
@pytest.mark.parametrize("E,F,B,k,C", PLACES)
def test_exchange(nb, E, F, B, k, C, kind):
    import torch
    if kind == "routed" and k > E:
        pytest.skip("no router picks more experts than there are")
    rng = np.random.default_rng(E + F + B)
    chosen = choices(rng, E, B, k, kind)
    slots, counts = ref.place(chosen, E, C)
    ld, lde = B + (3 if B % 2 else 0), C + (0 if C % 2 else 1)
    cd, sd, nd = device_matrix(chosen, ld), device_matrix(np.zeros_like(chosen), ld), torch.zeros(E, dtype=torch.int32, device="cuda")
    placement = torch.full((nb.expert_placement_bytes(E, B, k) // 4,), -77, dtype=torch.int32, device="cuda")
    nb.expert_place(cd, E, B, k, C, sd, nd, placement)
    assert np.array_equal(sd.cpu().numpy(), slots) and np.array_equal(nd.cpu().numpy(), counts) and padding_untouched(sd)
    again = torch.full_like(placement, 99)
    nb.expert_place(cd, E, B, k, C, None, None, again)

    X, Ye = rng.standard_normal((F, B)).astype(np.float32), rng.standard_normal((E, F, C)).astype(np.float32)
    w, dY = rng.standard_normal((k, B)).astype(np.float32), rng.standard_normal((F, B)).astype(np.float32)
    filled = np.minimum(counts, C)
    Ye[np.arange(C)[None, None, :] >= np.broadcast_to(filled[:, None, None], (E, F, 1))[:, :, :1]] = np.nan   # places that hold no column are not read
    w[slots < 0] = np.nan
    Xe = blocks(nb, shape=(E, F, C), ld=lde)
    nb.expert_dispatch(device_matrix(X, ld), placement, F, E, B, k, C, Xe)
    assert np.array_equal(Xe.cpu().numpy(), ref.dispatch(X, chosen, slots, E, C)) and padding_untouched(Xe)

    Yd, wd = blocks(nb, Ye, ld=lde), device_matrix(w, ld)
    for weights in (w, None):
        Y = device_matrix(np.full((F, B), np.nan, np.float32), B + 1)
        nb.expert_combine(Yd, placement, None if weights is None else wd, F, E, B, k, C, Y)
        assert np.array_equal(Y.cpu().numpy(), ref.combine(Ye, chosen, slots, weights)) and padding_untouched(Y)

    want, bound = ref.weight_gradient(Ye, dY, chosen, slots)
    room = torch.full((nb.expert_combine_workspace_bytes(F, B, k) // 4,), float("nan"), device="cuda")
    for weights, which in ((w, 3), (None, 3), (w, 1), (w, 2)):
        dYe = blocks(nb, shape=(E, F, C), ld=lde) if which & 1 else None
        dw = device_matrix(np.full((k, B), np.nan, np.float32), ld) if which & 2 else None
        nb.expert_combine_backward(Yd if which & 2 else None, device_matrix(dY, ld), placement, None if weights is None else wd, F, E, B, k, C, dYe, dw,
                                   room if which & 2 else None)
        if which & 1:
            assert np.array_equal(dYe.cpu().numpy(), ref.dispatch(dY, chosen, slots, E, C, weights)) and padding_untouched(dYe)
        if which & 2:
            got = dw.cpu().numpy().astype(np.float64)
            assert np.all(np.abs(got - want) <= bound), np.abs(got - want).max()
            assert (got[slots < 0] == 0).all() and padding_untouched(dw)


@pytest.mark.parametrize("E,F,B,k,C,variant", [
    (128, 600, 5000, 6, 260, "a row per wave"), (8, 700, 2048, 2, 600, "two rows, short tiles"), (8, 1600, 4096, 2, 1100, "four rows, short tiles"),
    (64, 1200, 6000, 4, 400, "four rows, long tiles"), (96, 1001, 8192, 8, 760, "work-groups of eight waves"), (128, 803, 8191, 10, 700, "weights not staged"),
    (300, 301, 2500, 3, 30, "short runs")])
def test_large_exchange_is_the_same_on_every_run(nb, E, F, B, k, C, variant):
    """Many tiles and work-groups, in every way that the sizes choose: against the plain forms, and the sums' order must not depend on which work-groups
    come first."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(4)
    chosen = (torch.rand(E, B, generator=g, device="cuda") + 0.1 * torch.rand(E, 1, generator=g, device="cuda")).topk(k, dim=0).indices.to(torch.int32)
    Ye, dY, X = torch.randn(E, F, C, generator=g, device="cuda"), torch.randn(F, B, generator=g, device="cuda"), torch.randn(F, B, generator=g, device="cuda")
    w = torch.rand(k, B, generator=g, device="cuda")
    placement = torch.empty(nb.expert_placement_bytes(E, B, k) // 4, dtype=torch.int32, device="cuda")
    room = torch.empty(nb.expert_combine_workspace_bytes(F, B, k) // 4, device="cuda")
    slots, counts = torch.empty_like(chosen), torch.empty(E, dtype=torch.int32, device="cuda")
    first = None
    for _ in range(3):
        Y, dYe, dw, Xe, dX = torch.empty(F, B, device="cuda"), torch.empty_like(Ye), torch.empty_like(w), torch.empty_like(Ye), torch.empty(F, B, device="cuda")
        nb.expert_place(chosen, E, B, k, C, slots, counts, placement)
        nb.expert_dispatch(X, placement, F, E, B, k, C, Xe)
        nb.expert_combine(Ye, placement, w, F, E, B, k, C, Y)
        nb.expert_combine_backward(Ye, dY, placement, w, F, E, B, k, C, dYe, dw, room)
        nb.expert_combine(Ye, placement, None, F, E, B, k, C, dX)
        if first is None:
            first = [Y, dYe, dw, Xe, dX]
            h = [t.cpu().numpy() for t in (chosen, Ye, dY, X, w)]
            want, n = ref.place(h[0], E, C)
            assert np.array_equal(slots.cpu().numpy(), want) and np.array_equal(counts.cpu().numpy(), n)
            assert np.array_equal(Y.cpu().numpy(), ref.combine(h[1], h[0], want, h[4]))
            assert np.array_equal(dX.cpu().numpy(), ref.combine(h[1], h[0], want))
            assert np.array_equal(Xe.cpu().numpy(), ref.dispatch(h[3], h[0], want, E, C))
            assert np.array_equal(dYe.cpu().numpy(), ref.dispatch(h[2], h[0], want, E, C, h[4]))
            gw, bound = ref.weight_gradient(h[1], h[2], h[0], want)
            assert np.all(np.abs(dw.cpu().numpy() - gw) <= bound)
        assert all(torch.equal(a, b) for a, b in zip(first, [Y, dYe, dw, Xe, dX]))


def test_blocks_beyond_32_bits(nb):
    """2.3 G entries: offsets that 32 bits do not hold, in entries; the same bits as the columns that went in."""
    import torch
    E, F, B, k, C = 8, 4096, 9, 2, 70000
    Xe = torch.empty(E, F, C, device="cuda")
    assert Xe.numel() > 2 ** 31
    chosen = torch.tensor([[7, 0, 7, 3, 7, 6, 7, 5, 7], [0, 7, 6, 7, 5, 7, 4, 7, 3]], dtype=torch.int32, device="cuda")
    slots, w = torch.empty_like(chosen), torch.rand(k, B, device="cuda")
    X, dY = torch.randn(F, B, device="cuda"), torch.randn(F, B, device="cuda")
    placement = torch.empty(nb.expert_placement_bytes(E, B, k) // 4, dtype=torch.int32, device="cuda")
    nb.expert_place(chosen, E, B, k, C, slots, None, placement)
    nb.expert_dispatch(X, placement, F, E, B, k, C, Xe)
    for j in range(k):
        for c in range(B):
            assert torch.equal(Xe[int(chosen[j, c]), :, int(slots[j, c])], X[:, c])
    assert int(torch.count_nonzero(Xe[7, -1])) == 9 and int(torch.count_nonzero(Xe[7])) == int(torch.count_nonzero(X))
    Y, dw = torch.empty(F, B, device="cuda"), torch.empty(k, B, device="cuda")
    nb.expert_combine(Xe, placement, None, F, E, B, k, C, Y)
    assert torch.equal(Y, X + X)
    room = torch.empty(nb.expert_combine_workspace_bytes(F, B, k) // 4, device="cuda")
    nb.expert_combine_backward(Xe, dY, placement, w, F, E, B, k, C, None, dw, room)
    want = (X.double() * dY.double()).sum(0)
    bound = (X.double() * dY.double()).abs().sum(0) * (18 + F // 4) * ref.U
    assert ((dw - want).abs() <= bound).all()


def test_placement_of_other_sizes_stays_inside_the_operands(nb):
    """A placement that was made for other sizes gives other values, and writes nothing outside the operands of the call."""
    import torch
    E, F, B, k, C = 16, 20, 300, 3, 80
    chosen = torch.randint(0, E, (k, B), device="cuda", dtype=torch.int32)
    placement = torch.empty(nb.expert_placement_bytes(E, B, k) // 4, dtype=torch.int32, device="cuda")
    nb.expert_place(chosen, E, B, k, C, None, None, placement)
    e, b, c = 5, 40, 7
    X, full = torch.randn(F, b, device="cuda"), torch.full((e * F * c + 4096,), 3.0, device="cuda")
    nb.expert_dispatch(X, placement, F, e, b, 2, c, full[2048:2048 + e * F * c].view(e, F, c))
    Y = torch.full((F * b + 4096,), 3.0, device="cuda")
    nb.expert_combine(torch.randn(e, F, c, device="cuda"), placement, torch.randn(2, b, device="cuda"), F, e, b, 2, c, Y[2048:2048 + F * b].view(F, b))
    for t, n in ((full, e * F * c), (Y, F * b)):
        assert (t[:2048] == 3).all() and (t[2048 + n:] == 3).all()


def test_calls_on_another_stream_and_through_ctypes(nb):
    """The compiled call layer and the one through ctypes make the same calls, on torch's current stream or a given one."""
    import torch
    from paper_2407_17437_amd.calls import Calls
    E, F, B, k, C = 12, 24, 90, 3, 20
    rng = np.random.default_rng(8)
    Z, X = device_matrix(rng.standard_normal((E, B)).astype(np.float32), 96), device_matrix(rng.standard_normal((F, B)).astype(np.float32), 96)
    placement = torch.empty(nb.expert_placement_bytes(E, B, k) // 4, dtype=torch.int32, device="cuda")
    room = torch.empty(nb.expert_combine_workspace_bytes(F, B, k) // 4, device="cuda")
    ws = torch.empty(nb.gradient_norm_workspace_bytes(1) // 4, device="cuda")
    side = torch.cuda.Stream()
    results = []
    for calls in (nb._fastcall, Calls(nb.lib, nb._stream)):
        for stream in (None, side):
            torch.cuda.synchronize()
            chosen, w = torch.zeros(k, 96, dtype=torch.int32, device="cuda")[:, :B], torch.zeros(k, 96, device="cuda")[:, :B]
            slots, counts, dZ = torch.zeros_like(chosen), torch.zeros(E, dtype=torch.int32, device="cuda"), torch.zeros(E, B, device="cuda")
            slots = torch.zeros(k, 96, dtype=torch.int32, device="cuda")[:, :B]
            Xe, Y, dYe, dw = nb.expert_blocks(E, F, C), torch.zeros(F, B, device="cuda"), nb.expert_blocks(E, F, C), torch.zeros(k, 96, device="cuda")[:, :B]
            norm, scaled = torch.zeros(1, device="cuda"), torch.zeros(F, B, device="cuda")
            torch.cuda.synchronize()
            rcs = [calls.route(Z, None, E, B, k, 3, 2, 2, 1.0, chosen, w, stream),
                   calls.place(chosen, E, B, k, C, slots, counts, placement, stream),
                   calls.dispatch(X, placement, F, E, B, k, C, Xe, stream),
                   calls.combine(Xe, placement, w, F, E, B, k, C, Y, stream),
                   calls.combine_backward(Xe, Y, placement, w, F, E, B, k, C, dYe, dw, room, stream),
                   calls.route_backward(Z, chosen, dw, E, B, k, 2, 1.0, dZ, stream),
                   calls.clip([Y], [scaled], 0.5, ws, norm, stream)]
            torch.cuda.synchronize()
            assert rcs == [0] * 7
            results.append([t.clone() for t in (chosen, w, slots, counts, Xe, Y, dYe, dw, dZ, norm, scaled)])
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], r))


def test_tensors_of_other_shapes_are_refused(nb):
    import torch
    from paper_2407_17437_amd.calls import Calls
    E, F, B, k, C = 4, 6, 20, 2, 12
    new = lambda *shape: torch.zeros(*shape, device="cuda")
    ints = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device="cuda")
    p, ws = ints(nb.expert_placement_bytes(E, B, k) // 4), new(nb.expert_combine_workspace_bytes(F, B, k) // 4 + 8192)
    for calls in (nb._fastcall, Calls(nb.lib, nb._stream)):
        for Z, b, chosen, w in ((new(E - 1, B), None, ints(k, B), new(k, B)), (new(E, B - 1), None, ints(k, B), new(k, B)), (new(B, E).t(), None, ints(k, B), new(k, B)),
                                (new(E, B), new(E - 1), ints(k, B), new(k, B)), (new(E, B), None, ints(k - 1, B), new(k, B)), (new(E, B), None, ints(k, B), new(k, B + 1)),
                                (new(E, B), None, ints(k, B).long(), new(k, B)), (new(E, B), None, ints(k, B), new(k, B).half())):
            with pytest.raises(AssertionError):
                calls.route(Z, b, E, B, k, 1, 1, 0, 1.0, chosen, w, None)
        for chosen, slots, counts in ((ints(k, B - 1), None, None), (ints(k, B), ints(k, B + 1), None), (ints(k, B), None, ints(E - 1)), (ints(k, B), None, ints(2 * E)[::2])):
            with pytest.raises(AssertionError):
                calls.place(chosen, E, B, k, C, slots, counts, p, None)
        for X, Xe in ((new(F - 1, B), new(E, F, C)), (new(F, B), new(E - 1, F, C)), (new(F, B), new(E, F + 1, C)), (new(F, B), new(E, F, C - 1)),
                      (new(F, B), new(E, F + 2, C)[:, :F]), (new(F, B), new(E, C, F).transpose(1, 2)), (new(F, B), new(E * F, C))):
            with pytest.raises(AssertionError):
                calls.dispatch(X, p, F, E, B, k, C, Xe, None)
            with pytest.raises(AssertionError):
                calls.combine(Xe, p, None, F, E, B, k, C, X, None)
        with pytest.raises(AssertionError):
            calls.combine_backward(new(E, F, C), new(F, B), p, new(k, B), F, E, B, k, C, new(E, F, C + 1)[:, :, :C], new(k, B), ws, None)
        with pytest.raises(AssertionError):
            calls.combine_backward(new(E, F, C), new(F, B), p, new(k, B), F, E, B, k, C, None, new(k, B + 1)[:, :B], ws, None)
        with pytest.raises(AssertionError):
            calls.clip([new(5)], [new(6)], 1.0, ws, None, None)
        with pytest.raises(AssertionError):
            calls.clip([new(5), new(5)], [new(5)], 1.0, ws, None, None)
        with pytest.raises(AssertionError):
            calls.norm([new(10)[::2]], ws, new(1), None)
        with pytest.raises(AssertionError):
            calls.norm([new(5)], ws, new(0), None)
        with pytest.raises(OverflowError if calls is nb._fastcall else Exception):
            calls.dispatch(new(F, B), p, F, E, B, k, 2 ** 31, new(E, F, C), None)

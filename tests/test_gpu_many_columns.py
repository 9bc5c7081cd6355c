"""Places of many columns in the experts' blocks, and the exchange where what it stages elsewhere has no room."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nb():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2407_17437_amd import binding
    return binding


def places(chosen, experts, capacity):
    """slots and counts: choices sorted by expert, stably, in the order of columns and then of choices."""
    k, batch = chosen.shape
    flat = chosen.T.reshape(-1).astype(np.int64)
    flat = np.where((flat >= 0) & (flat < experts), flat, experts)
    order = np.argsort(flat, kind="stable")
    counts = np.bincount(flat, minlength=experts + 1)
    first = np.cumsum(counts) - counts
    place = np.empty_like(flat)
    place[order] = np.arange(flat.size) - first[flat[order]]
    place[(place >= capacity) | (flat == experts)] = -1
    return place.reshape(batch, k).T.astype(np.int32), counts[:experts].astype(np.int32)


@pytest.mark.parametrize("E,B,k,C", [(64, 200_001, 1, 3000), (1000, 70_000, 3, 211), (3, 100_000, 2, 90_000), (256, 1 << 18, 2, 2048), (7, 4097, 1, 400), (65, 1400, 3, 50),
                                     (1, 300_000, 1, 250_000), (1024, 33_000, 32, 1000),
                                     (256, 8192, 3, 90), (255, 8192, 3, 90), (256, 7936, 1, 40)])
@pytest.mark.parametrize("kind", ["any", "one expert", "by turns"])
def test_places_of_many_columns(nb, E, B, k, C, kind):
    import torch
    rng = np.random.default_rng(E + B)
    if kind == "any":
        chosen = rng.integers(-1, E + 1, (k, B)).astype(np.int32)      # twice the same, and none (-1 and E)
    elif kind == "one expert":
        chosen = np.full((k, B), E - 1, np.int32)
    else:                                                              # experts that fill up one after the other, along the batch
        chosen = np.minimum(np.arange(B) * E // B, E - 1)[None].repeat(k, 0).astype(np.int32)
    slots, counts = places(chosen, E, C)
    sd, nd = torch.full((k, B), 7, dtype=torch.int32, device="cuda"), torch.zeros(E, dtype=torch.int32, device="cuda")
    room = nb.expert_placement_bytes(E, B, k) // 4
    placement = torch.full((room + 64,), -77, dtype=torch.int32, device="cuda")
    nb.expert_place(torch.as_tensor(chosen).cuda(), E, B, k, C, sd, nd, placement[:room])
    assert np.array_equal(nd.cpu().numpy(), counts) and np.array_equal(sd.cpu().numpy(), slots)
    assert (placement[room:] == -77).all()
    # the lists, through the calls that read them: every place holds its column, every column finds its places
    F = 2
    X = torch.as_tensor(rng.integers(-1000, 1000, (F, B)).astype(np.float32)).cuda()
    Xe, Y = torch.full((E, F, C), float("nan"), device="cuda"), torch.empty(F, B, device="cuda")
    nb.expert_dispatch(X, placement, F, E, B, k, C, Xe)
    nb.expert_combine(Xe, placement, None, F, E, B, k, C, Y)
    kept = torch.as_tensor(slots >= 0).cuda()
    j, c = torch.nonzero(kept, as_tuple=True)
    e, s = torch.as_tensor(chosen).cuda()[j, c].long(), sd[j, c].long()
    want = torch.zeros(E, F, C, device="cuda")
    want[e, :, s] = X[:, c].t()
    assert torch.equal(Xe, want)
    assert torch.equal(Y, X * kept.sum(0))                             # (small whole numbers: exact)


def test_time_of_places_grows_with_the_columns(nb):
    """Four times as many columns take about four times as long, and would take sixteen times as long if each run of columns went
    through all runs before it; between them is twice four."""
    import torch
    E, k, C = 256, 1, 1 << 22
    times = []
    for B in (1 << 20, 1 << 22):
        chosen = torch.randint(0, E, (k, B), device="cuda", dtype=torch.int32)
        placement = torch.empty(nb.expert_placement_bytes(E, B, k) // 4, dtype=torch.int32, device="cuda")
        one = []
        for _ in range(7):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            nb.expert_place(chosen, E, B, k, C, None, None, placement)
            b.record()
            b.synchronize()
            one.append(a.elapsed_time(b))
        times.append(sorted(one)[3])
    print("ms:", times, flush=True)
    assert times[1] < 8 * times[0], times


def test_blocks_of_weighted_columns_whose_weights_have_no_room_in_lds(nb):
    """Many choices, long tiles and 16 rows for a work-group: with the rows the weights would take more than 160 KiB, and are read where they lie."""
    import torch
    E, F, B, k, C = 256, 2048, 4096, 28, 300
    g = torch.Generator(device="cuda").manual_seed(6)
    chosen = (torch.rand(E, B, generator=g, device="cuda") + 0.2 * torch.rand(E, 1, generator=g, device="cuda")).topk(k, dim=0).indices.to(torch.int32)
    dY, w, Ye = torch.randn(F, B, generator=g, device="cuda"), torch.randn(k, B, generator=g, device="cuda"), torch.randn(E, F, C, generator=g, device="cuda")
    slots, _ = places(chosen.cpu().numpy(), E, C)
    placement = torch.empty(nb.expert_placement_bytes(E, B, k) // 4, dtype=torch.int32, device="cuda")
    nb.expert_place(chosen, E, B, k, C, None, None, placement)
    sd = torch.as_tensor(slots).cuda()
    j, c = torch.nonzero(sd >= 0, as_tuple=True)
    e, s = chosen[j, c].long(), sd[j, c].long()
    assert 0 < j.numel() < B * k
    want = torch.zeros(E, F, C, device="cuda")
    want[e, :, s] = (w[j, c] * dY[:, c]).t()            # (one product, rounded once: the same bits)
    room = torch.full((nb.expert_combine_workspace_bytes(F, B, k) // 4,), float("nan"), device="cuda")
    for with_dw in (False, True):
        dYe, dw = torch.full((E, F, C), float("nan"), device="cuda"), torch.full((k, B), float("nan"), device="cuda")
        nb.expert_combine_backward(Ye if with_dw else None, dY, placement, w, F, E, B, k, C, dYe, dw if with_dw else None, room if with_dw else None)
        assert torch.equal(dYe, want)
    sums, sizes = torch.zeros(k, B, dtype=torch.float64, device="cuda"), torch.zeros(k, B, dtype=torch.float64, device="cuda")
    for at in torch.arange(j.numel(), device="cuda").split(8192):
        y, d = Ye[e[at], :, s[at]].double(), dY[:, c[at]].t().double()
        sums[j[at], c[at]], sizes[j[at], c[at]] = (y * d).sum(1), (y * d).abs().sum(1)
    # 16 products in a sum of 32 bits, the sums of F / 16 of those in 64, rounded once
    assert ((dw - sums).abs() <= sizes * 18 * 2.0 ** -24).all() and (dw[sd < 0] == 0).all()

"""What the calls of mixtures and of clipped gradients refuse, before anything reaches the device (no GPU needed)."""
import ctypes

import numpy as np
import pytest

P = 1 << 20   # an address that is aligned and never read


@pytest.fixture(scope="module")
def nb():
    from paper_2407_17437_amd import binding
    return binding


def route(nb, **kw):
    a = dict(Z=P, ldz=8, bias=None, experts=8, batch=8, k=2, groups=1, top=1, flags=0, scale=1.0, chosen=P, weights=P, ldk=8)
    a.update(kw)
    return nb.lib.expert_route(a["Z"], a["ldz"], a["bias"], a["experts"], a["batch"], a["k"], a["groups"], a["top"], a["flags"], a["scale"], a["chosen"], a["weights"],
                               a["ldk"], None)


@pytest.mark.parametrize("kw,code,words", [
    (dict(Z=None), "ARGUMENT", "null"), (dict(chosen=None), "ARGUMENT", "null"), (dict(weights=None), "ARGUMENT", "null"),
    (dict(experts=0), "ARGUMENT", "experts = 0"), (dict(experts=1025), "ARGUMENT", "1025"), (dict(k=0), "ARGUMENT", "k = 0"), (dict(k=33, experts=64), "ARGUMENT", "k = 33"),
    (dict(k=9), "ARGUMENT", "9 choices among 8"), (dict(batch=0), "ARGUMENT", "batch"), (dict(batch=-3), "ARGUMENT", "batch"), (dict(ldz=7), "SHAPE", "ldz"),
    (dict(ldk=7), "SHAPE", "ldk"), (dict(ldz=1 << 30), "SHAPE", "ldz"), (dict(groups=3), "ARGUMENT", "3 groups"), (dict(groups=0), "ARGUMENT", "groups"),
    (dict(experts=128, groups=128, top=2), "ARGUMENT", "128 groups"), (dict(groups=4, top=5), "ARGUMENT", "top_groups"), (dict(groups=4, top=0), "ARGUMENT", "top_groups"),
    (dict(groups=8, top=1), "ARGUMENT", "2 choices among 1"), (dict(flags=8), "ARGUMENT", "flags"), (dict(flags=-1), "ARGUMENT", "flags"),
    (dict(scale=float("inf")), "ARGUMENT", "scale"), (dict(scale=float("nan")), "ARGUMENT", "scale"),
    (dict(batch=1 << 29, ldz=1 << 29, ldk=1 << 29), "SHAPE", "choices"),
])
def test_route_refuses(nb, kw, code, words):
    assert route(nb, **kw) == getattr(nb, "NERVA_ERR_" + code)
    assert words in nb.last_error()


def test_route_backward_refuses(nb):
    def call(Z=P, ldz=8, chosen=P, dw=P, ldk=8, experts=8, batch=8, k=2, flags=0, scale=1.0, dZ=P, lddz=8):
        return nb.lib.expert_route_backward(Z, ldz, chosen, dw, ldk, experts, batch, k, flags, scale, dZ, lddz, None)
    for kw in (dict(Z=None), dict(chosen=None), dict(dw=None), dict(dZ=None), dict(experts=0), dict(k=40), dict(flags=64), dict(scale=float("nan")), dict(batch=0)):
        assert call(**kw) == nb.NERVA_ERR_ARGUMENT, kw
    for kw in (dict(ldz=7), dict(ldk=7), dict(lddz=7), dict(lddz=1 << 30)):
        assert call(**kw) == nb.NERVA_ERR_SHAPE, kw


def test_place_and_exchange_refuse(nb):
    room = nb.expert_placement_bytes(8, 100, 2)
    assert room % 16 == 0 and room >= 100 * 2 * 8 + 8 * 4
    assert nb.lib.expert_placement_bytes(0, 100, 2) == 0 and nb.lib.expert_placement_bytes(8, 0, 2) == 0 and nb.lib.expert_placement_bytes(8, 100, 33) == 0
    with pytest.raises(nb.NervaError, match="k = 33"):
        nb.expert_placement_bytes(8, 100, 33)

    def place(chosen=P, ldk=100, experts=8, batch=100, k=2, capacity=9, placement=P, room=room):
        return nb.lib.expert_place(chosen, ldk, experts, batch, k, capacity, None, None, placement, room, None)

    def dispatch(X=P, ldx=100, placement=P, room=room, features=16, experts=8, batch=100, k=2, capacity=9, Xe=P, lde=9):
        return nb.lib.expert_dispatch(X, ldx, placement, room, features, experts, batch, k, capacity, Xe, lde, None)

    def combine(Ye=P, lde=9, placement=P, room=room, w=P, ldk=100, features=16, experts=8, batch=100, k=2, capacity=9, Y=P, ldy=100):
        return nb.lib.expert_combine(Ye, lde, placement, room, w, ldk, features, experts, batch, k, capacity, Y, ldy, None)

    need = nb.expert_combine_workspace_bytes(16, 100, 2)
    assert need >= 100 * 2 * 4 and nb.expert_combine_workspace_bytes(0, 100, 2) == 0

    def backward(Ye=P, lde=9, dY=P, lddy=100, placement=P, room=room, w=P, ldk=100, features=16, experts=8, batch=100, k=2, capacity=9, dYe=P, dw=P, ws=P, need=need):
        return nb.lib.expert_combine_backward(Ye, lde, dY, lddy, placement, room, w, ldk, features, experts, batch, k, capacity, dYe, dw, ws, need, None)

    for call in (place, dispatch, combine, backward):
        for kw in (dict(placement=None), dict(experts=0), dict(experts=1025), dict(batch=0), dict(k=0), dict(k=33), dict(capacity=0), dict(capacity=-1), dict(capacity=1 << 30)):
            assert call(**kw) == nb.NERVA_ERR_ARGUMENT, (call, kw)
        for kw in (dict(room=room - 16), dict(placement=P + 4)):
            assert call(**kw) == nb.NERVA_ERR_WORKSPACE, (call, kw)
        assert nb.last_error() != ""
    for call, names in ((place, ["chosen"]), (dispatch, ["X", "Xe"]), (combine, ["Ye", "Y"]), (backward, ["dY"])):
        for name in names:
            assert call(**{name: None}) == nb.NERVA_ERR_ARGUMENT
    for call, lds in ((place, ["ldk"]), (dispatch, ["ldx"]), (combine, ["ldk", "ldy"]), (backward, ["ldk", "lddy"])):
        for name in lds:
            for ld in (99, 1 << 30):
                assert call(**{name: ld}) == nb.NERVA_ERR_SHAPE, (call, name)
    for call in (dispatch, combine, backward):
        assert call(lde=8) == nb.NERVA_ERR_SHAPE and call(lde=1 << 30) == nb.NERVA_ERR_SHAPE
        assert call(features=0) == nb.NERVA_ERR_ARGUMENT and call(features=2 ** 31 - 1) == nb.NERVA_ERR_SHAPE
    assert backward(Ye=None) == nb.NERVA_ERR_ARGUMENT and backward(dYe=None, dw=None) == nb.NERVA_ERR_ARGUMENT and backward(ws=None) == nb.NERVA_ERR_ARGUMENT
    assert backward(need=need - 4) == nb.NERVA_ERR_WORKSPACE and backward(ws=P + 4) == nb.NERVA_ERR_WORKSPACE


def test_clipped_gradients_refuse(nb):
    def lists(ptrs, counts):
        return len(counts), (ctypes.c_void_p * len(counts))(*ptrs), (ctypes.c_int64 * len(counts))(*counts)
    room = nb.gradient_norm_workspace_bytes(2)
    assert nb.lib.gradient_norm_workspace_bytes(-1) == 0 and nb.gradient_norm_workspace_bytes(1000) > nb.gradient_norm_workspace_bytes(0) > 0
    n, g, c = lists([P, P], [5, 6])

    def norm(n=n, g=g, c=c, ws=P, room=room, out=P):
        return nb.lib.gradient_norm(n, g, c, ws, room, out, None)

    def clip(n=n, g=g, out=g, c=c, max_norm=1.0, ws=P, room=room):
        return nb.lib.gradient_clip(n, g, out, c, max_norm, ws, room, None, None)

    def update(n=n, w=g, v=g, g=g, c=c, max_norm=1.0, ws=P, room=room):
        return nb.lib.sgd_update_clipped(n, w, v, g, c, 0.1, 0.9, max_norm, 0, ws, room, None, None)

    null = lists([P, None], [5, 6])[1]
    for call in (norm, clip, update):
        for kw in (dict(n=-1), dict(g=None), dict(c=None), dict(g=null), dict(c=lists([P, P], [5, -6])[2]), dict(ws=None)):
            assert call(**kw) == nb.NERVA_ERR_ARGUMENT, (call, kw)
        assert call(room=room - 8) == nb.NERVA_ERR_WORKSPACE and call(ws=P + 4) == nb.NERVA_ERR_WORKSPACE
        assert call(c=lists([P, P], [5, (1 << 40) + 1])[2]) == nb.NERVA_ERR_SHAPE
    assert norm(out=None) == nb.NERVA_ERR_ARGUMENT
    assert clip(out=None) == nb.NERVA_ERR_ARGUMENT and clip(out=null) == nb.NERVA_ERR_ARGUMENT
    for kw in (dict(w=None), dict(v=None), dict(w=null), dict(v=null)):
        assert update(**kw) == nb.NERVA_ERR_ARGUMENT
    for call in (clip, update):
        for bad in (0.0, -1.0, float("nan"), float("-inf")):
            assert call(max_norm=bad) == nb.NERVA_ERR_ARGUMENT and "max_norm" in nb.last_error()
    assert nb.lib.mlp_train_step_clipped(None, P, 4, P, 4, 0.1, 0.9, 1.0, P, 0, None, None, None) == nb.NERVA_ERR_ARGUMENT
    assert nb.lib.mlp_clipped_workspace_bytes(None, 4) == 0


def test_tensors_that_do_not_fit_the_call(nb):
    """Both call layers look at types and devices (shapes: with tensors on the device, in the GPU tests)."""
    import torch
    from paper_2407_17437_amd.calls import Calls
    f, i = torch.zeros(4, 8), torch.zeros(4, 8, dtype=torch.int32)
    for calls in (nb._fastcall, Calls(nb.lib, lambda s: s)):
        with pytest.raises(AssertionError, match="GPU"):
            calls.route(f, None, 4, 8, 2, 1, 1, 0, 1.0, i, f, 0)
        with pytest.raises(AssertionError, match="Z.*float32"):
            calls.route(f.double(), None, 4, 8, 2, 1, 1, 0, 1.0, i, f, 0)
        with pytest.raises(TypeError):
            calls.route(None, None, 4, 8, 2, 1, 1, 0, 1.0, i, f, 0)
        with pytest.raises(AssertionError, match="GPU"):
            calls.route_backward(f, i, f, 4, 8, 2, 0, 1.0, f, 0)
        with pytest.raises(AssertionError, match="chosen"):
            calls.place(f, 4, 8, 2, 3, None, None, i, 0)
        with pytest.raises(AssertionError, match="GPU"):
            calls.dispatch(f, i, 4, 4, 8, 2, 3, f, 0)
        with pytest.raises(AssertionError, match="GPU"):
            calls.combine(f.view(2, 2, 8), i, f, 2, 2, 8, 2, 8, f, 0)
        with pytest.raises(AssertionError, match="GPU"):
            calls.combine_backward(f.view(2, 2, 8), f, i, f, 2, 2, 8, 2, 8, None, f, f, 0)
        with pytest.raises(AssertionError, match="grads"):
            calls.norm([f], f, f, 0)
        with pytest.raises(AssertionError, match="list"):
            calls.clip(f, [f], 1.0, f, f, 0)
        with pytest.raises(AssertionError, match="grads"):
            calls.update_clipped([f], [f], [f.double()], 0.1, 0.9, 1.0, 0, f, f, 0)
        assert calls.norm([], None, None, 0) == nb.NERVA_ERR_ARGUMENT     # (no workspace)

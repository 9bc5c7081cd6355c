"""Group norm, dropout and the losses of labels without a GPU: what the calls refuse, and that the tests' reference is right."""
import numpy as np
import pytest

import label_reference as ref

P = 1 << 20   # an address that is aligned and never read


@pytest.fixture(scope="module")
def nb():
    from paper_2407_17437_amd import binding
    return binding


# ---- the reference

def test_generator_gives_the_published_numbers():
    """Test vectors of the generator's publication: counters and keys of zeros, and of ones."""
    ones = 0xFFFFFFFF
    assert [int(w) for w in ref.philox([0, 0, 0, 0], [0, 0])] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert [int(w) for w in ref.philox([ones] * 4, [ones] * 2)] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def test_factors_are_drawn_at_their_rate():
    for drop in (0.1, 0.5, 0.9):
        f = ref.factors(256, 1000, drop, 3, 12345678901234, 7)
        kept = (f > 0).mean()
        assert abs(kept - (1 - drop)) < 5 * np.sqrt(drop * (1 - drop) / f.size)
        assert abs(f.mean() - 1) < 5 * np.sqrt(drop / (1 - drop) / f.size)
    a = ref.factors(8, 64, 0.5, 3, 1, 7)
    assert all((a != ref.factors(8, 64, 0.5, *other)).any() for other in ((4, 1, 7), (3, 2, 7), (3, 1, 8), (3, 1 + 2 ** 32, 7)))


@pytest.mark.parametrize("act", [0, 1, 2])
def test_gradients_of_the_norm_are_those_of_differences(act):
    rng = np.random.default_rng(act)
    X, ga, be, dY = rng.standard_normal((12, 5)), rng.standard_normal(12), rng.standard_normal(12), rng.standard_normal((12, 5))
    keep = ref.factors(12, 5, 0.3, 0, 9, 9)

    def value(X=X, ga=ga, be=be):
        return (ref.Norm(X, ga, be, 3, 1e-3, act, keep).Y * dY).sum()
    n = ref.Norm(X, ga, be, 3, 1e-3, act, keep, dY)
    for name, at, grad in (("X", X, n.dX), ("ga", ga, n.dgamma), ("be", be, n.dbeta)):
        for _ in range(4):
            v = rng.standard_normal(at.shape)
            d = (value(**{name: at + 1e-5 * v}) - value(**{name: at - 1e-5 * v})) / 2e-5
            assert abs(d - (grad * v).sum()) < 1e-6 * (1 + abs(d)), name


def test_gradients_of_the_losses_are_those_of_differences():
    rng = np.random.default_rng(3)
    Z, labels = rng.standard_normal((7, 20)), rng.integers(-1, 7, 20)
    old, adv, w = -2 + 0.3 * rng.standard_normal(20), rng.standard_normal(20), rng.random(20)
    refs = -2 + 0.3 * rng.standard_normal(20)
    starts, sums = np.array([1, 4, 9, 9, 18]), -8 + rng.standard_normal(4)

    def policy(Z):
        return ref.Policy(Z, labels, old, refs, adv, w, 0.2, 0.3, 0.1)

    def preference(Z):
        return ref.Preference(Z, labels, starts, sums, 0.3, 0.1)
    for of, value in ((policy, lambda t: t.stats[0]), (preference, lambda t: t.loss)):
        for _ in range(4):
            v = rng.standard_normal(Z.shape)
            d = (value(of(Z + 1e-6 * v)) - value(of(Z - 1e-6 * v))) / 2e-6
            assert abs(d - (of(Z).dZ * v).sum()) < 1e-7 * (1 + abs(d))


# ---- refusals

def norm(nb, **kw):
    a = dict(X=P, ldx=8, gamma=None, beta=None, features=12, groups=3, batch=8, eps=1e-5, act=0, drop=0.0, layer=0, state=None, Y=P + 4096, ldy=8, mean=P, rstd=P, lds=8, ws=P,
             room=1 << 30)
    a.update(kw)
    return nb.lib.group_norm_forward(*[a[k] for k in ("X", "ldx", "gamma", "beta", "features", "groups", "batch", "eps", "act", "drop", "layer", "state", "Y", "ldy", "mean",
                                                      "rstd", "lds", "ws", "room")], None)


def norm_back(nb, **kw):
    a = dict(X=P, ldx=8, gamma=None, beta=None, mean=P, rstd=P, lds=8, dY=P + 4096, lddy=8, features=12, groups=3, batch=8, act=0, drop=0.0, layer=0, state=None,
             dX=P + 8192, lddx=8, dgamma=P, dbeta=P, ws=P, room=1 << 30)
    a.update(kw)
    return nb.lib.group_norm_backward(*[a[k] for k in ("X", "ldx", "gamma", "beta", "mean", "rstd", "lds", "dY", "lddy", "features", "groups", "batch", "act", "drop", "layer",
                                                       "state", "dX", "lddx", "dgamma", "dbeta", "ws", "room")], None)


def drop(nb, **kw):
    a = dict(X=P, ldx=8, features=12, batch=8, drop=0.5, layer=0, state=P, Y=P + 4096, ldy=8)
    a.update(kw)
    return nb.lib.dropout(*[a[k] for k in ("X", "ldx", "features", "batch", "drop", "layer", "state", "Y", "ldy")], None)


def test_norm_and_dropout_refuse(nb):
    nan, inf = float("nan"), float("inf")
    for call in (norm, norm_back):
        for kw in (dict(X=None), dict(features=0), dict(features=-4), dict(groups=0), dict(groups=-1), dict(groups=5), dict(groups=24), dict(batch=0), dict(batch=-1), dict(act=3),
                   dict(act=-1), dict(drop=-0.1), dict(drop=1.0), dict(drop=nan), dict(drop=0.5), dict(drop=0.5, state=P + 4)):
            assert call(nb, **kw) == nb.NERVA_ERR_ARGUMENT, (call, kw)
            assert nb.last_error()
        for kw in (dict(ldx=7), dict(lds=7), dict(ldx=1 << 30), dict(lds=1 << 30), dict(features=1 << 30, groups=1)):
            assert call(nb, **kw) == nb.NERVA_ERR_SHAPE, (call, kw)
        for kw in (dict(features=1 << 20, groups=1, room=16), dict(features=1 << 20, groups=1, ws=P + 4)):
            assert call(nb, **kw) == nb.NERVA_ERR_WORKSPACE, (call, kw)
        assert call(nb, features=1 << 20, groups=1, ws=None) == nb.NERVA_ERR_ARGUMENT
    for kw in (dict(Y=None), dict(mean=None), dict(rstd=None), dict(eps=0.0), dict(eps=-1.0), dict(eps=nan), dict(eps=inf)):
        assert norm(nb, **kw) == nb.NERVA_ERR_ARGUMENT, kw
    for kw in (dict(ldy=7), dict(Y=P, ldy=9)):
        assert norm(nb, **kw) == nb.NERVA_ERR_SHAPE, kw
    for kw in (dict(dY=None), dict(dX=None), dict(mean=None), dict(rstd=None), dict(dX=P)):
        assert norm_back(nb, **kw) == nb.NERVA_ERR_ARGUMENT, kw
    for kw in (dict(lddy=7), dict(lddx=7), dict(dX=P + 4096, lddx=9)):
        assert norm_back(nb, **kw) == nb.NERVA_ERR_SHAPE, kw
    for kw in (dict(X=None), dict(Y=None), dict(features=0), dict(batch=0), dict(drop=1.0), dict(drop=-0.5), dict(drop=nan), dict(state=None), dict(state=P + 4)):
        assert drop(nb, **kw) == nb.NERVA_ERR_ARGUMENT, kw
    for kw in (dict(ldx=7), dict(ldy=7), dict(Y=P, ldy=16), dict(features=1 << 30)):
        assert drop(nb, **kw) == nb.NERVA_ERR_SHAPE, kw
    # more threads than a launch holds
    assert drop(nb, features=1 << 29, batch=1 << 20, ldx=1 << 20, ldy=1 << 20) == nb.NERVA_ERR_SHAPE and "columns" in nb.last_error()
    big = dict(features=1 << 29, groups=1 << 27, batch=1 << 20, ldx=1 << 20, lds=1 << 20, room=1 << 62)
    assert norm(nb, ldy=1 << 20, **big) == nb.NERVA_ERR_SHAPE and "columns" in nb.last_error()
    assert norm_back(nb, lddy=1 << 20, lddx=1 << 20, **big) == nb.NERVA_ERR_SHAPE and "columns" in nb.last_error()
    with pytest.raises(nb.NervaError, match="5 groups"):
        nb.group_norm_workspace_bytes(12, 5, 8)
    assert nb.group_norm_workspace_bytes(12, 3, 8) % 4 == 0 and nb.group_norm_workspace_bytes(1 << 20, 1, 100) > 0


def test_losses_refuse(nb):
    nan, inf = float("nan"), float("inf")
    room = nb.label_loss_workspace_bytes(10, 8, 6)
    assert nb.lib.label_loss_workspace_bytes(0, 8, 6) == 0 and nb.lib.label_loss_workspace_bytes(10, 0, 6) == 0 and nb.lib.label_loss_workspace_bytes(10, 8, -1) == 0
    with pytest.raises(nb.NervaError, match="classes"):
        nb.label_loss_workspace_bytes(0, 8, 6)

    def score(Z=P, ldz=8, labels=P, classes=10, batch=8, starts=P, n=6, logp=P, sums=P, ws=P, room=room):
        return nb.lib.label_log_probs(Z, ldz, labels, classes, batch, starts, n, logp, sums, ws, room, None)

    def policy(Z=P, ldz=8, labels=P, old=P, refs=None, adv=P, w=None, classes=10, batch=8, low=0.2, high=0.2, beta=0.0, dZ=P + 4096, lddz=8, logp=None, stats=P, ws=P, room=room):
        return nb.lib.policy_loss(Z, ldz, labels, old, refs, adv, w, classes, batch, low, high, beta, dZ, lddz, logp, stats, ws, room, None)

    def preference(Z=P, ldz=8, labels=P, starts=P, refs=None, classes=10, batch=8, pairs=3, beta=0.1, t=0.0, dZ=P + 4096, lddz=8, ws=P, room=room):
        return nb.lib.preference_loss(Z, ldz, labels, starts, refs, classes, batch, pairs, beta, t, dZ, lddz, None, None, None, ws, room, None)

    for call in (score, policy, preference):
        for kw in (dict(Z=None), dict(labels=None), dict(classes=0), dict(classes=-1), dict(batch=0), dict(batch=-8), dict(ws=None)):
            assert call(**kw) == nb.NERVA_ERR_ARGUMENT, (call, kw)
            assert nb.last_error()
        for kw in (dict(ldz=7), dict(ldz=1 << 30), dict(classes=1 << 30)):
            assert call(**kw) == nb.NERVA_ERR_SHAPE, (call, kw)
        for kw in (dict(room=16), dict(ws=P + 8)):
            assert call(**kw) == nb.NERVA_ERR_WORKSPACE, (call, kw)
    for kw in (dict(logp=None, sums=None), dict(starts=None), dict(n=0), dict(n=-1), dict(n=-1, sums=None)):
        assert score(**kw) == nb.NERVA_ERR_ARGUMENT, kw
    for kw in (dict(old=None), dict(adv=None), dict(dZ=None), dict(stats=None), dict(low=-0.1), dict(high=-0.1), dict(low=nan), dict(high=inf), dict(beta=nan), dict(beta=-1.0)):
        assert policy(**kw) == nb.NERVA_ERR_ARGUMENT, kw
    for kw in (dict(starts=None), dict(dZ=None), dict(pairs=0), dict(pairs=-1), dict(pairs=1 << 30), dict(beta=nan), dict(beta=inf), dict(t=-0.1), dict(t=1.1), dict(t=nan)):
        assert preference(**kw) == nb.NERVA_ERR_ARGUMENT, kw
    for call in (policy, preference):
        for kw in (dict(lddz=7), dict(dZ=P, lddz=9)):
            assert call(**kw) == nb.NERVA_ERR_SHAPE, (call, kw)


def test_tensors_that_do_not_fit_the_calls(nb):
    import torch
    from paper_2407_17437_amd.calls import Calls
    f, i, v, st = torch.zeros(4, 8), torch.zeros(8, dtype=torch.int32), torch.zeros(8), torch.zeros(2, dtype=torch.int64)
    for calls in (nb._fastcall, Calls(nb.lib, lambda s: s)):
        good = {"norm_forward": [f, v, v, 4, 2, 8, 1e-5, 0, 0.5, 0, st, f, f, f, v, 0], "norm_backward": [f, v, v, f, f, f, 4, 2, 8, 0, 0.5, 0, st, f, v, v, v, 0],
                "dropout": [f, 4, 8, 0.5, 0, st, f, 0], "log_probs": [f, i, 4, 8, i, 3, v, v, v, 0],
                "policy": [f, i, v, v, v, v, 4, 8, 0.2, 0.2, 0.1, f, v, v, v, 0], "preference": [f, i, i, v, 4, 8, 3, 0.1, 0.0, f, v, v, v, v, 0]}
        for name, args in good.items():
            call = getattr(calls, name)
            with pytest.raises(AssertionError, match="GPU"):
                call(*args)
            for k, a in enumerate(args):
                if isinstance(a, torch.Tensor) and k < len(args) - 2:
                    with pytest.raises(AssertionError):
                        call(*args[:k], a.double() if a.dtype != torch.int64 else a.int(), *args[k + 1:])
                elif isinstance(a, int) and k < len(args) - 1:
                    for n in (2 ** 31, 2 ** 32 + 1, -2 ** 31 - 1):
                        with pytest.raises(OverflowError):
                            call(*args[:k], n, *args[k + 1:])
            with pytest.raises(TypeError):
                call(None, *args[1:])

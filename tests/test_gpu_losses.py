"""Log-probabilities of labels, the clipped policy loss and the preference loss against plain forms in 64 bits (label_reference.py)."""
import numpy as np
import pytest

import label_reference as ref
from test_gpu_norm import blank, close, gpu, matrix, nb, padding_untouched  # noqa: F401

pytestmark = pytest.mark.gpu


def workspace(nb, classes, batch, sequences=0):
    import torch
    return torch.full((nb.label_loss_workspace_bytes(classes, batch, sequences) // 4 + 4,), float("nan"), device="cuda")


def nans(n):
    import torch
    return torch.full((n,), float("nan"), device="cuda")


def logits(rng, C, B, kind="plain"):
    Z = (2 * rng.standard_normal((C, B))).astype(np.float32)
    labels = rng.integers(0, C, B).astype(np.int32)
    if kind == "masked":
        Z[rng.random((C, B)) < 0.4] = -np.inf
        Z[:, rng.random(B) < 0.1] = -np.inf
        labels[rng.random(B) < 0.2] = -1
        labels[rng.random(B) < 0.05] = C
        labels[rng.random(B) < 0.05] = 2 ** 31 - 1
        labels[-1] = -2 ** 31
    elif kind == "lowest":
        # masks of the type's lowest value: a column of nothing else is uniform
        Z[rng.random((C, B)) < 0.5] = np.finfo(np.float32).min
        Z[:, 0] = np.finfo(np.float32).min
        keep = np.argmax(Z, axis=0)
        labels[1:] = keep[1:]
    elif kind == "wide":
        Z *= 30
        labels = np.argmax(Z, axis=0).astype(np.int32)
    elif kind == "far":
        Z += 10000
    return Z, labels


def cuts(rng, B, n):
    """Starts of n ragged sequences: some columns outside, an empty sequence among them."""
    s = np.sort(rng.integers(0, B + 1, n + 1))
    if n > 2:
        s[1] = s[2]
    return np.sort(s).astype(np.int32)


SIZES = [(1, 1), (2, 1), (10, 100), (2, 257), (3, 5), (63, 33), (1000, 1), (32768, 1), (257, 1000), (1025, 66), (2049, 31), (40000, 3), (17, 5000), (5003, 259)]
KINDS = ["plain", "masked", "lowest", "wide", "far"]


@pytest.mark.parametrize("C,B", SIZES)
@pytest.mark.parametrize("kind", KINDS)
def test_log_probs(nb, C, B, kind):
    rng = np.random.default_rng(C + B)
    Z, labels = logits(rng, C, B, kind)
    pad = [0, 3, -B % 32][SIZES.index((C, B)) % 3]
    n = min(5, B)
    starts = cuts(rng, B, n)
    z, lp, sums, ws = matrix(Z, pad), nans(B), nans(n), workspace(nb, C, B, n)
    nb.label_log_probs(z, gpu(labels), C, B, gpu(starts), n, lp, sums, ws)
    want = ref.Labels(Z, labels)
    close(lp, want.logp, want.logp_tol, "logp")
    s, off = want.sums(starts)
    close(sums, s, off + ref.E * np.abs(s) + 1e-37, "sums")
    again = nans(B)
    nb.label_log_probs(z, gpu(labels), C, B, None, 0, again, None, ws)
    assert bool((again == lp).all())
    nb.label_log_probs(z, gpu(labels), C, B, gpu(starts), n, None, sums, ws)
    close(sums, s, off + ref.E * np.abs(s) + 1e-37, "sums")


def policy_inputs(rng, Z, labels):
    C, B = Z.shape
    lp = ref.Labels(Z, labels).logp
    old = (lp + 0.3 * rng.standard_normal(B)).astype(np.float32)
    return old, (lp + 0.3 * rng.standard_normal(B)).astype(np.float32), rng.standard_normal(B).astype(np.float32), rng.random(B).astype(np.float32)


def run_policy(nb, Z, labels, old, refs, A, w, low, high, beta, pads=(0, 0), in_place=False, ws=None, out=None):
    import torch
    C, B = Z.shape
    z = matrix(Z, pads[0])
    dz = z if in_place else blank(C, B, pads[1])
    lp, stats = nans(B), nans(4)
    nb.policy_loss(z, gpu(labels), gpu(old), gpu(refs), gpu(A), gpu(w), C, B, low, high, beta, dz, lp, stats, workspace(nb, C, B) if ws is None else ws)
    torch.cuda.synchronize()
    assert padding_untouched(z, dz)
    return stats, lp, dz


@pytest.mark.parametrize("C,B", SIZES)
@pytest.mark.parametrize("kind", KINDS)
def test_policy(nb, C, B, kind):
    rng = np.random.default_rng(C * 3 + B)
    Z, labels = logits(rng, C, B, kind)
    old, refs, A, w = policy_inputs(rng, Z, labels)
    w[rng.random(B) < 0.1] = 0
    k = SIZES.index((C, B))
    for r, weights, low, high, beta in ((None, None, 0.2, 0.2, 0.0), (refs, w, 0.1, 0.3, 0.05), (refs, None, 1.5, 0.5, 1.0)):
        want = ref.Policy(Z, labels, old, r, A, weights, low, high, beta)
        stats, lp, dz = run_policy(nb, Z, labels, old, r, A, weights, low, high, beta, [(0, 0), (5, 2), (-B % 32,) * 2][k % 3])
        close(lp, want.L.logp, want.L.logp_tol, "logp")
        close(stats, want.stats, want.stats_tol, "stats")
        close(dz, want.dZ, want.dZ_tol, "dZ")
        stats2, lp2, dz2 = run_policy(nb, Z, labels, old, r, A, weights, low, high, beta, (1, 0), in_place=True)
        assert bool((dz2 == dz).all()) and bool((stats2 == stats).all()) and bool((lp2 == lp).all())


# one tile for all and one class more; what a work-group holds at most and a class more, in narrow tiles and in tiles that are not narrowed
@pytest.mark.parametrize("C,B,kind", [(16, 256, "masked"), (64, 256, "plain"), (65, 256, "plain"), (64, 257, "masked"), (2048, 130, "masked"), (2049, 130, "plain"), (1024, 8200, "plain"),
                                      (1025, 8193, "masked"), (4, 9001, "masked"), (300, 3001, "wide")])
def test_around_the_limits(nb, C, B, kind):
    rng = np.random.default_rng(C * 11 + B)
    Z, labels = logits(rng, C, B, kind)
    old, refs, A, w = policy_inputs(rng, Z, labels)
    want = ref.Policy(Z, labels, old, refs, A, w, 0.2, 0.28, 0.04)
    stats, lp, dz = run_policy(nb, Z, labels, old, refs, A, w, 0.2, 0.28, 0.04, (1, 2))
    close(lp, want.L.logp, want.L.logp_tol, "logp"), close(stats, want.stats, want.stats_tol, "stats"), close(dz, want.dZ, want.dZ_tol, "dZ")
    starts = cuts(rng, B, 14)
    want = ref.Preference(Z, labels, starts, None, 0.02, 0.1)
    dz, sums, margins, loss, scores, ws = blank(C, B, 3), nans(14), nans(7), nans(1), nans(14), workspace(nb, C, B, 14)
    nb.preference_loss(matrix(Z, 5), gpu(labels), gpu(starts), None, C, B, 7, 0.02, 0.1, dz, sums, margins, loss, ws)
    close(sums, want.sums, want.sums_tol, "sums"), close(margins, want.margins, want.margins_tol, "margins"), close(loss, np.array([want.loss]), want.loss_tol, "loss")
    close(dz, want.dZ, want.dZ_tol, "dZ")
    nb.label_log_probs(matrix(Z), gpu(labels), C, B, gpu(starts), 14, None, scores, ws)
    assert bool((scores == sums).all()) and padding_untouched(dz)


def test_policy_borders_are_decided_in_64_bits(nb):
    """Ratios that lie on their borders to within the last bits that an fp32 old log-probability can express: on both sides, and a clip of 0
    with the policy unmoved, where every column lies on its border."""
    rng = np.random.default_rng(12)
    for C, B in ((10, 600), (3000, 300)):
        Z, labels = logits(rng, C, B)
        lp = ref.Labels(Z, labels).logp
        A = np.where(rng.random(B) < 0.5, -1, 1).astype(np.float32)
        low, high = float(np.float32(0.2)), float(np.float32(0.3))
        border = np.where(A > 0, np.log1p(high), np.log1p(-low))
        old = (lp - border).astype(np.float32)
        old = np.where(rng.random(B) < 0.5, np.nextafter(old, np.float32(0)), np.where(rng.random(B) < 0.5, np.nextafter(old, np.float32(-99)), old))
        want = ref.Policy(Z, labels, old, None, A, None, 0.2, 0.3, 0.0)
        assert 0.2 < want.clipped.mean() < 0.8
        stats, _, dz = run_policy(nb, Z, labels, old, None, A, None, 0.2, 0.3, 0.0)
        close(dz, want.dZ, want.dZ_tol, "dZ")
        close(stats, want.stats, want.stats_tol, "stats")
        old = lp.astype(np.float32)
        want = ref.Policy(Z, labels, old, None, A, None, 0.0, 0.0, 0.0)
        stats, _, dz = run_policy(nb, Z, labels, old, None, A, None, 0.0, 0.0, 0.0)
        close(dz, want.dZ, want.dZ_tol, "dZ")
        close(stats, want.stats, want.stats_tol, "stats")


@pytest.mark.parametrize("C,B,pairs", [(1, 2, 1), (10, 100, 3), (2, 9, 4), (63, 33, 2), (1000, 2, 1), (257, 1000, 40), (1025, 66, 5), (2049, 31, 1), (17, 5000, 2), (5003, 259, 64)])
@pytest.mark.parametrize("kind", KINDS)
def test_preference(nb, C, B, pairs, kind):
    import torch
    rng = np.random.default_rng(C * 5 + B)
    Z, labels = logits(rng, C, B, kind)
    starts = cuts(rng, B, 2 * pairs)
    s, _ = ref.Labels(Z, labels).sums(starts)
    sums_of_ref = (s + 3 * rng.standard_normal(2 * pairs)).astype(np.float32)
    for refs, beta, t in ((None, 0.05, 0.0), (sums_of_ref, 0.3, 0.1), (sums_of_ref, -0.2, 1.0)):
        want = ref.Preference(Z, labels, starts, refs, beta, t)
        pads = [(0, 0), (5, 2), (-B % 32,) * 2][pairs % 3]
        z, dz, sums, margins, loss, ws = matrix(Z, pads[0]), blank(C, B, pads[1]), nans(2 * pairs), nans(pairs), nans(1), workspace(nb, C, B, 2 * pairs)
        nb.preference_loss(z, gpu(labels), gpu(starts), gpu(refs), C, B, pairs, beta, t, dz, sums, margins, loss, ws)
        assert padding_untouched(z, dz)
        close(sums, want.sums, want.sums_tol, "sums")
        close(margins, want.margins, want.margins_tol, "margins")
        close(loss, np.array([want.loss]), want.loss_tol, "loss")
        close(dz, want.dZ, want.dZ_tol, "dZ")
        nb.preference_loss(z, gpu(labels), gpu(starts), gpu(refs), C, B, pairs, beta, t, z, None, None, None, ws)
        assert torch.equal(z, dz)


def test_columns_of_nan_and_infinity(nb):
    rng = np.random.default_rng(13)
    for C, B in ((12, 40), (4001, 40)):
        Z, labels = logits(rng, C, B)
        old, refs, A, w = policy_inputs(rng, Z, labels)
        Z[1, 3], Z[2, 4], Z[0, 5], Z[3, 6] = np.nan, np.inf, np.nan, np.nan
        labels[5], labels[6] = -1, C + 4
        stats, lp, dz = (t.cpu().numpy() for t in run_policy(nb, Z, labels, old, refs, A, w, 0.2, 0.2, 0.1))
        for c in (3, 4):
            assert np.isnan(lp[c]) and np.isnan(dz[:, c]).all()
        for c in (5, 6):
            assert lp[c] == 0 and (dz[:, c] == 0).all()
        rest = np.setdiff1d(np.arange(B), (3, 4))
        assert np.isfinite(dz[:, rest]).all() and np.isfinite(lp[rest]).all() and np.isnan(stats[:3]).all()
        w[3] = w[4] = 0
        stats, lp, dz = (t.cpu().numpy() for t in run_policy(nb, Z, labels, old, refs, A, w, 0.2, 0.2, 0.1))
        assert np.isfinite(stats).all() and np.isfinite(dz).all() and (dz[:, 3:7] == 0).all() and np.isnan(lp[3])
        starts = np.array([0, 8, 20, 30, 40], np.int32)
        dz, loss, margins = blank(C, B), nans(1), nans(2)
        nb.preference_loss(matrix(Z), gpu(labels), gpu(starts), None, C, B, 2, 0.1, 0.0, dz, None, margins, loss, workspace(nb, C, B, 4))
        dz = dz.cpu().numpy()
        assert np.isnan(float(loss)) and bool(margins.isnan()[0]) and not bool(margins.isnan()[1])
        assert np.isfinite(dz[:, 20:]).all() and np.isnan(dz[:, :5]).all() and (dz[:, 5:7] == 0).all()


def test_starts_that_are_none(nb):
    """Whatever starts holds, nothing beyond the operands is touched; sequences that lie inside are as they would be."""
    import torch
    rng = np.random.default_rng(14)
    C, B = 30, 50
    Z, labels = logits(rng, C, B)
    want, ws = ref.Labels(Z, labels), workspace(nb, C, B, 4)
    for starts in ([-5, 10, 20, 90, 2 ** 31 - 1], [40, 30, 20, 10, 0], [-2 ** 31, -1, 10, 20, 30]):
        sums, dz = nans(4), blank(C, B, 6)
        st = gpu(np.array(starts, np.int32))
        nb.label_log_probs(matrix(Z), gpu(labels), C, B, st, 4, None, sums, ws)
        nb.preference_loss(matrix(Z), gpu(labels), st, None, C, B, 2, 0.1, 0.0, dz, None, None, None, ws)
        torch.cuda.synchronize()
        assert padding_untouched(dz)
        for k in range(4):
            a, b = starts[k], starts[k + 1]
            if 0 <= a <= b <= B:
                assert abs(float(sums[k]) - want.logp[a:b].sum()) < 1e-4


def test_gradients_against_differences(nb):
    rng = np.random.default_rng(15)
    for C, B in ((12, 60), (1500, 60)):
        Z, labels = logits(rng, C, B)
        old, refs, A, w = policy_inputs(rng, Z, labels)
        v = rng.standard_normal(Z.shape)
        _, _, dz = run_policy(nb, Z, labels, old, refs, A, w, 0.2, 0.3, 0.1)

        def policy(h):
            return ref.Policy(Z + h * v, labels, old, refs, A, w, 0.2, 0.3, 0.1)
        d = (policy(1e-6).stats[0] - policy(-1e-6).stats[0]) / 2e-6
        # (64-bit sums of some 10, over 2e-6, and the reference's own curvature)
        assert abs(d - (dz.cpu().numpy() * v).sum()) < (policy(0).dZ_tol * np.abs(v)).sum() + 1e-7
        starts = np.array([0, 10, 25, 30, 60], np.int32)
        sums, _ = ref.Labels(Z, labels).sums(starts)
        sums = (sums + rng.standard_normal(4)).astype(np.float32)
        dz = blank(C, B)
        nb.preference_loss(matrix(Z), gpu(labels), gpu(starts), gpu(sums), C, B, 2, 0.1, 0.05, dz, None, None, None, workspace(nb, C, B, 4))

        def preference(h):
            return ref.Preference(Z + h * v, labels, starts, sums, 0.1, 0.05)
        d = (preference(1e-5).loss - preference(-1e-5).loss) / 2e-5
        assert abs(d - (dz.cpu().numpy() * v).sum()) < (preference(0).dZ_tol * np.abs(v)).sum() + 1e-7


def test_captured_losses(nb):
    """All three in one graph, replayed with new logits between eager calls."""
    import torch
    rng = np.random.default_rng(16)
    for C, B in ((10, 100), (3000, 300)):
        Z, labels = logits(rng, C, B, "masked")
        old, refs, A, w = (gpu(t) for t in policy_inputs(rng, Z, labels))
        starts = gpu(np.array([0, B // 5, B // 2, B // 2, B], np.int32))
        z, lab = matrix(Z, 4), gpu(labels)

        def outputs():
            return [nans(B), nans(4), blank(C, B), nans(B), nans(4), blank(C, B), nans(4), nans(2), nans(1)]

        def calls(ws, lp, sums, dz, lp2, stats, dz2, sums2, margins, loss):
            nb.label_log_probs(z, lab, C, B, starts, 4, lp, sums, ws)
            nb.policy_loss(z, lab, old, refs, A, w, C, B, 0.2, 0.3, 0.1, dz, lp2, stats, ws)
            nb.preference_loss(z, lab, starts, None, C, B, 2, 0.1, 0.05, dz2, sums2, margins, loss, ws)
        out, ws = outputs(), workspace(nb, C, B, 4)
        calls(ws, *out)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            calls(ws, *out)
        for _ in range(3):
            z += 0.1 * torch.randn(C, B, device="cuda")
            g.replay()
            torch.cuda.synchronize()
            other = outputs()
            calls(workspace(nb, C, B, 4), *other)
            for a, b in zip(out, other):
                assert torch.equal(a, b)


def test_two_streams_at_once(nb):
    """Calls that overlap, each with a workspace of its own, on streams given as an argument and as the current one."""
    import torch
    rng = np.random.default_rng(19)
    C, B = 3000, 500
    Z, labels = logits(rng, C, B, "masked")
    inputs = [gpu(t) for t in policy_inputs(rng, Z, labels)]
    z, lab, starts = matrix(Z, 4), gpu(labels), gpu(np.array([0, 100, 250, 400, 500], np.int32))
    x, ga, st = matrix(rng.standard_normal((1200, B))), gpu(np.ones(1200, np.float32)), gpu(np.array([3, 4], np.int64))

    def policy(ws, out, stream=None):
        nb.policy_loss(z, lab, *inputs, C, B, 0.2, 0.3, 0.1, out[0], out[1], out[2], ws, stream)

    def preference(ws, out, stream=None):
        nb.preference_loss(z, lab, starts, None, C, B, 2, 0.1, 0.05, out[0], out[1], out[2], None, ws, stream)

    def norm(ws, out, stream=None):
        nb.group_norm_forward(x, ga, None, 1200, 1, B, 1e-5, 2, 0.3, 0, st, out[0], out[1], out[2], ws, stream)
        nb.group_norm_backward(x, ga, None, out[1], out[2], x, 1200, 1, B, 2, 0.3, 0, st, out[3], out[4], None, ws, stream)
    sets = [(policy, lambda: [blank(C, B), nans(B), nans(4)], lambda: workspace(nb, C, B)), (preference, lambda: [blank(C, B), nans(4), nans(2)], lambda: workspace(nb, C, B, 4)),
            (norm, lambda: [blank(1200, B), blank(1, B), blank(1, B), blank(1200, B), nans(1200)],
             lambda: torch.zeros(max(4, nb.group_norm_workspace_bytes(1200, 1, B) // 4), device="cuda"))]
    alone = []
    for call, outputs, ws in sets:
        out = outputs()
        call(ws(), out)
        alone.append(out)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    runs = [[(s[1](), s[2]()) for s in sets] for _ in range(4)]
    torch.cuda.synchronize()
    for run in runs:
        for k, (call, _, _) in enumerate(sets):
            if k % 2:
                with torch.cuda.stream(streams[k]):
                    call(run[k][1], run[k][0])
            else:
                call(run[k][1], run[k][0], streams[k])
    torch.cuda.synchronize()
    for run in runs:
        for k in range(3):
            assert all(torch.equal(a, b) for a, b in zip(run[k][0], alone[k]) if not bool(b.isnan().any()))
            assert all(torch.equal(torch.nan_to_num(a), torch.nan_to_num(b)) for a, b in zip(run[k][0], alone[k]))


def test_rows_far_apart(nb):
    """Rows 2^26 entries apart: offsets beyond 32 bits."""
    import torch
    C, B, ld = 70, 33, 1 << 26
    rng = np.random.default_rng(17)
    Z, labels = logits(rng, C, B)
    labels[:] = C - 1
    old, refs, A, w = policy_inputs(rng, Z, labels)
    stats, lp, dz = run_policy(nb, Z, labels, old, refs, A, w, 0.2, 0.2, 0.1)
    z = torch.empty(C * ld, device="cuda").as_strided((C, B), (ld, 1))
    z.copy_(torch.as_tensor(Z))
    lp2, stats2, ws = nans(B), nans(4), workspace(nb, C, B)
    nb.policy_loss(z, gpu(labels), gpu(old), gpu(refs), gpu(A), gpu(w), C, B, 0.2, 0.2, 0.1, z, lp2, stats2, ws)
    assert torch.equal(z, dz) and torch.equal(lp, lp2) and torch.equal(stats, stats2)


def test_what_the_call_layers_refuse(nb):
    """Shapes, with tensors on the device, by both layers; and that both make the same calls."""
    import torch
    from paper_2407_17437_amd.calls import Calls
    f, i, v, st = torch.randn(4, 8, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda"), torch.ones(8, device="cuda"), torch.ones(2, dtype=torch.int64, device="cuda")
    ws = torch.zeros(4096, device="cuda")
    starts = torch.tensor([0, 2, 4, 6, 8], dtype=torch.int32, device="cuda")
    results = []
    for calls in (nb._fastcall, Calls(nb.lib, nb._stream)):
        outs = [torch.zeros(4, 8, device="cuda") for _ in range(8)] + [torch.zeros(8, device="cuda") for _ in range(8)]
        good = {"norm_forward": [f, v, v, 4, 2, 8, 1e-5, 2, 0.5, 0, st, outs[0], outs[1], outs[2], ws, None],
                "norm_backward": [f, v, v, outs[1], outs[2], f, 4, 2, 8, 2, 0.5, 0, st, outs[3], outs[8], outs[9], ws, None],
                "dropout": [f, 4, 8, 0.5, 0, st, outs[4], None], "log_probs": [f, i, 4, 8, starts, 4, outs[10], outs[11], ws, None],
                "policy": [f, i, v, v, v, v, 4, 8, 0.2, 0.2, 0.1, outs[5], outs[12], outs[13], ws, None],
                "preference": [f, i, starts, v, 4, 8, 2, 0.1, 0.0, outs[6], outs[14], outs[15], v.clone(), ws, None]}
        for name, args in good.items():
            call = getattr(calls, name)
            assert call(*args) == 0, (name, nb.last_error())
            for k, a in enumerate(args):
                if not isinstance(a, torch.Tensor) or a is ws or (name, k) == ("preference", 12):
                    continue
                for bad in ([a[:1], a[:, :7], a.t()] if a.dim() == 2 else [a[:1], torch.zeros(16, dtype=a.dtype, device="cuda")[::2], a.cpu()]):
                    with pytest.raises(AssertionError):
                        call(*args[:k], bad, *args[k + 1:])
        torch.cuda.synchronize()
        results.append(outs)
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_one_training_step_of_them_together(nb):
    """Sparse layer, norm with activation and dropout, sparse layer, policy loss (then preference loss) and everything backwards, against 64 bits."""
    import torch
    from paper_2407_17437_amd import workloads as wl
    rng = np.random.default_rng(18)
    B, G, drop = 60, 4, 0.2
    mlp = wl.make_mlp((48, 64, 12), sparsity=0.7, pattern_seed=3, value_seed=4, bias_std=0.1)
    layers = [nb.SparseLinear(l, B) for l in mlp.layers]
    X = rng.standard_normal((48, B)).astype(np.float32)
    gamma, beta = (1 + 0.2 * rng.standard_normal(64)).astype(np.float32), (0.2 * rng.standard_normal(64)).astype(np.float32)
    labels = rng.integers(-1, 12, B).astype(np.int32)
    st = gpu(np.array([77, 5], np.int64))

    def dense(l):
        W = np.zeros((l.rows, l.cols))
        W[np.repeat(np.arange(l.rows), np.diff(l.indptr)), l.indices] = l.values
        return W
    W1, W2 = dense(mlp.layers[0]), dense(mlp.layers[1])
    layers[0].relu = False
    lin = nb.sparse_linear_create(layers[0].rows, layers[0].cols, layers[0].nnz, layers[0].indptr, layers[0].indices, layers[0].values, layers[0].bias, nb.NERVA_ACT_NONE, B)
    x, h, a, z = matrix(X, 4), blank(64, B, 4), blank(64, B, 4), blank(12, B, 4)
    mean, rstd, ws, lws = blank(G, B), blank(G, B), torch.empty(max(4, nb.group_norm_workspace_bytes(64, G, B) // 4), device="cuda"), workspace(nb, 12, B, 4)
    nb.sparse_linear_forward(lin, x, h, B)
    nb.group_norm_forward(h, gpu(gamma), gpu(beta), 64, G, B, 1e-5, nb.NERVA_ACT_SILU, drop, 0, st, a, mean, rstd, ws)
    nb.sparse_linear_forward(layers[1].handle, a, z, B)
    # the plain chain
    b1, b2 = mlp.layers[0].bias.astype(np.float64), mlp.layers[1].bias.astype(np.float64)
    factor = ref.factors(64, B, drop, 0, 77, 5)
    H = W1 @ X + b1[:, None]
    n = ref.Norm(H, gamma, beta, G, 1e-5, 2, factor)
    Zr = W2 @ n.Y + b2[:, None]
    assert np.abs(z.cpu().numpy() - Zr).max() < 2e-5 * max(1, np.abs(Zr).max())
    old, refs, A, w = policy_inputs(rng, Zr, labels)
    old[np.abs(np.exp(ref.Labels(Zr, labels).logp - old) - 1.2) < 1e-3] += 0.01     # (borders are another test's)
    old[np.abs(np.exp(ref.Labels(Zr, labels).logp - old) - 0.8) < 1e-3] += 0.01
    starts = np.array([0, 12, 30, 45, 60], np.int32)
    for kind in ("policy", "preference"):
        dz, da, dh, dx = blank(12, B), blank(64, B), blank(64, B), blank(48, B)
        dv2, db2, dv1, db1, dg, dbe = nans(layers[1].nnz), nans(12), nans(layers[0].nnz), nans(64), nans(64), nans(64)
        if kind == "policy":
            nb.policy_loss(z, gpu(labels), gpu(old), gpu(refs), gpu(A), gpu(w), 12, B, 0.2, 0.2, 0.1, dz, None, nans(4), lws)
            dZ = ref.Policy(Zr, labels, old, refs, A, w, 0.2, 0.2, 0.1).dZ
        else:
            nb.preference_loss(z, gpu(labels), gpu(starts), None, 12, B, 2, 0.1, 0.05, dz, None, None, None, lws)
            dZ = ref.Preference(Zr, labels, starts, None, 0.1, 0.05).dZ
        nb.sparse_linear_backward(layers[1].handle, a, None, dz, da, dv2, db2, B)
        nb.group_norm_backward(h, gpu(gamma), gpu(beta), mean, rstd, da, 64, G, B, nb.NERVA_ACT_SILU, drop, 0, st, dh, dg, dbe, ws)
        nb.sparse_linear_backward(lin, x, None, dh, dx, dv1, db1, B)
        back = ref.Norm(H, gamma, beta, G, 1e-5, 2, factor, W2.T @ dZ)

        def entries(l, D):
            return D[np.repeat(np.arange(l.rows), np.diff(l.indptr)), l.indices]
        for name, got, want in (("dZ", dz, dZ), ("dW2", dv2, entries(mlp.layers[1], dZ @ n.Y.T)), ("db2", db2, dZ.sum(1)), ("dgamma", dg, back.dgamma), ("dbeta", dbe, back.dbeta),
                                ("dW1", dv1, entries(mlp.layers[0], back.dX @ X.T)), ("db1", db1, back.dX.sum(1)), ("dX", dx, W1.T @ back.dX)):
            # (each stage's own bound is tested by itself; through five of them some hundred roundings of the largest entry)
            got = got.cpu().numpy()
            assert np.abs(got - want).max() < 300 * ref.E * max(np.abs(want).max(), 1e-3), (kind, name, np.abs(got - want).max(), np.abs(want).max())
    nb.sparse_linear_destroy(lin)
    for l in layers:
        l.close()

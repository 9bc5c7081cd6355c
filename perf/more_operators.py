"""What stands between sparse layers and behind the last one when they are trained: group norm with an activation, dropout, and the
losses of policies and preferences; the work of these operators as measurable cases.

`run` with `own` true makes the calls of `paper_2407_17437_amd.binding`; with `own` false it computes the same in
elementary torch operations.  As everywhere in the library an operand holds one example (or token) per column.

norm        groups of features normalised in every column, scaled and shifted, an activation, dropout; with the gradients of all inputs.
dropout     by itself, of activations and of their gradient, with a mask that both passes draw anew from counters.
score       log-probabilities of labels under columns of logits, and their sums over sequences of columns.
policy      clipped policy loss with a KL term, and the gradient of the logits.
preference  loss of paired sequences by the ratio of their log-probabilities to those of a reference, and the gradient of the logits.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
LAYER = 3                      # number of the call among those that drop in one training step
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.04
BETA, SMOOTHING = 0.1, 0.05


def listed():
    return [
        # Serving one example: a hidden layer of the paper's network, normalised.  Every launch counts.
        {"name": "norm one", "kind": "norm", "features": 1024, "groups": 16, "batch": 1, "act": "relu", "drop": 0.0, "affine": True, "train": False, "padded": True},
        # A training step of that layer at the paper's batch.
        {"name": "norm batch", "kind": "norm", "features": 1024, "groups": 32, "batch": 100, "act": "silu", "drop": 0.1, "affine": True, "train": True, "padded": True},
        # One group, longer than what a work-group can hold, and a short last mini-batch without padding.
        {"name": "norm tall", "kind": "norm", "features": 8190, "groups": 1, "batch": 777, "act": "none", "drop": 0.0, "affine": True, "train": True, "padded": False},
        # Wide layers and a large batch, everything in one pass.
        {"name": "norm large", "kind": "norm", "features": 8192, "groups": 32, "batch": 8192, "act": "silu", "drop": 0.1, "affine": True, "train": True, "padded": True},
        # The paper's hidden layer at its batch: both passes fit the caches.
        {"name": "dropout batch", "kind": "dropout", "features": 1024, "batch": 100, "drop": 0.5, "padded": True},
        # Odd sizes, no padding, far beyond the caches.
        {"name": "dropout large", "kind": "dropout", "features": 8191, "batch": 9001, "drop": 0.1, "padded": False},
        # The log-probability of one answer among many classes.
        {"name": "score one", "kind": "score", "classes": 32768, "batch": 1, "sequences": 1, "closed": 0.0, "masked": 0.0, "padded": True},
        # A reference's log-probabilities of sequences of tokens.
        {"name": "score sequences", "kind": "score", "classes": 8192, "batch": 4000, "sequences": 32, "closed": 0.0, "masked": 0.2, "padded": True},
        # Ten classes as actions, the paper's output layer and batch.
        {"name": "policy batch", "kind": "policy", "classes": 10, "batch": 100, "kl": False, "weighted": False, "closed": 0.0, "masked": 0.0, "padded": True},
        # Tokens of many answers: prompts do not count, every answer has its weight, and a reference holds the policy.
        {"name": "policy large", "kind": "policy", "classes": 16384, "batch": 8192, "kl": True, "weighted": True, "closed": 0.0, "masked": 0.2, "padded": True},
        # A few ragged pairs, closed classes (and columns with no open one), no padding.
        {"name": "preference ragged", "kind": "preference", "classes": 1001, "batch": 777, "pairs": 12, "closed": 0.1, "masked": 0.3, "padded": False},
        # Many pairs over many classes.
        {"name": "preference large", "kind": "preference", "classes": 8192, "batch": 8192, "pairs": 32, "closed": 0.0, "masked": 0.3, "padded": True},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {"bytes": max(work(c)["bytes"] for c in listed()), "flops": max(work(c)["flops"] for c in listed())}
    while True:
        kind = rng.choice(["norm"] * 3 + ["dropout", "score"] + ["policy"] * 2 + ["preference"] * 2)
        case = {"kind": kind}
        if kind == "norm":
            groups = rng.choice([1, 1, 2, 5, 8, 16, 32, 60])
            case.update(features=groups * _log_int(rng, 8, 8192 // groups), groups=groups, batch=_log_int(rng, 1, 16384), act=rng.choice(["none", "silu", "silu"]),
                        drop=rng.choice([0.0, 0.0, 0.1, 0.5]), affine=rng.random() < 0.8, train=rng.random() < 0.7)
        elif kind == "dropout":
            case.update(features=_log_int(rng, 1, 8192), batch=_log_int(rng, 1, 16384), drop=round(rng.uniform(0.01, 0.9), 3))
        else:
            batch = _log_int(rng, 1 if kind != "preference" else 2, 16384)
            case.update(classes=_log_int(rng, 2, 32768), batch=batch)
            if kind == "score":
                case["sequences"] = _log_int(rng, 1, max(1, min(128, batch)))
            elif kind == "policy":
                case.update(kl=rng.random() < 0.6, weighted=rng.random() < 0.5)
            else:
                case["pairs"] = _log_int(rng, 1, max(1, min(64, batch // 2)))
            case.update(closed=rng.choice([0.0, 0.0, 0.1, 0.5]), masked=rng.choice([0.0, 0.2, 0.6]))
        case["padded"] = rng.random() < 0.6
        w = work(case)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return case


# ---- inputs ------------------------------------------------------------------------------------

def _ld(case, columns):
    """Rows on 128-byte lines, or without padding."""
    return (columns + 31) // 32 * 32 if case["padded"] else columns


def _matrix(case, rows, columns, gen=None):
    t = torch.zeros(rows, _ld(case, columns), device="cuda")[:, :columns]
    if gen is not None:
        t.copy_(torch.randn(rows, columns, generator=gen, device="cuda"))
    return t


def _cuts(case, sequences, gen):
    """First columns of ragged sequences, and the end of the last: some columns lie outside, and a sequence may be empty."""
    batch = case["batch"]
    if sequences == 1:
        return torch.tensor([0, batch], dtype=torch.int32, device="cuda")
    cuts = torch.randint(0, batch + 1, (sequences + 1,), generator=gen, device="cuda")
    return cuts.sort().values.to(torch.int32)


def _logits(s, gen):
    """Logits, labels drawn from them (-1: does not count) and the labels' log-probabilities."""
    classes, batch = s["classes"], s["batch"]
    s["Z"] = Z = _matrix(s, classes, batch, gen)
    Z *= 2
    if s["closed"] > 0:
        closed = torch.rand(classes, batch, generator=gen, device="cuda") < s["closed"]
        closed |= torch.rand(1, batch, generator=gen, device="cuda") < 0.02
        Z.masked_fill_(closed, -math.inf)
        del closed
    noise = torch.empty(classes, batch, device="cuda").exponential_(generator=gen)
    labels = (Z - noise.log_()).argmax(0)
    del noise
    at = Z.gather(0, labels[None])[0]
    logp = torch.where(torch.isneginf(at), torch.zeros_like(at), at - torch.logsumexp(Z, 0))
    out = torch.rand(batch, generator=gen, device="cuda") < s["masked"]
    s["labels"] = labels.masked_fill(out, -1).to(torch.int32)
    return logp.masked_fill(out, 0)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case)
    kind, batch = case["kind"], case["batch"]

    def vector(n, scale=1.0, shift=0.0):
        return shift + scale * torch.randn(n, generator=gen, device="cuda")

    if kind in ("norm", "dropout"):
        features = case["features"]
        s["X"] = _matrix(case, features, batch, gen)
        s["Y"] = _matrix(case, features, batch)
        # seed and step of the training run, on the device, as a captured step takes them
        s["state"] = torch.randint(0, 2 ** 62, (2,), generator=gen, device="cuda")
        s["state"][1] %= 100000
        if kind == "dropout" or case["train"]:
            s["dY"], s["dX"] = _matrix(case, features, batch, gen), _matrix(case, features, batch)
        if kind == "norm":
            # features differ in scale and centre, as the outputs of layers with biases do
            s["X"] *= (0.5 + torch.rand(features, 1, generator=gen, device="cuda"))
            s["X"] += 0.5 * vector(features)[:, None]
            s["gamma"], s["beta"] = (vector(features, 0.2, 1.0), vector(features, 0.2)) if case["affine"] else (None, None)
            s["mean"], s["rstd"] = _matrix(case, case["groups"], batch), _matrix(case, case["groups"], batch)
            if case["train"]:
                s["dgamma"], s["dbeta"] = torch.zeros(features, device="cuda"), torch.zeros(features, device="cuda")
            if own:
                from paper_2407_17437_amd import binding as nb
                s["act_code"] = {"none": nb.NERVA_ACT_NONE, "relu": nb.NERVA_ACT_RELU, "silu": nb.NERVA_ACT_SILU}[case["act"]]
                s["workspace"] = torch.empty(max(4, nb.group_norm_workspace_bytes(features, case["groups"], batch) // 4), device="cuda")
        return s
    classes = case["classes"]
    logp = _logits(s, gen)
    s["logp"] = torch.zeros(batch, device="cuda")
    sequences = {"score": case.get("sequences"), "policy": 0, "preference": 2 * case.get("pairs", 0)}[kind]
    if kind == "score":
        s["starts"] = _cuts(case, sequences, gen)
        s["sums"] = torch.zeros(sequences, device="cuda")
    elif kind == "policy":
        # the policy has moved since it answered, and away from the reference
        s["old"] = logp + vector(batch, 0.2)
        s["ref"] = logp + vector(batch, 0.3) if case["kl"] else None
        s["advantages"] = vector(batch)
        s["weights"] = (0.5 + torch.rand(batch, generator=gen, device="cuda")) / batch if case["weighted"] else None
        s["dZ"], s["stats"] = _matrix(case, classes, batch), torch.zeros(4, device="cuda")
    else:
        s["starts"] = _cuts(case, sequences, gen)
        total = torch.cat([torch.zeros(1, device="cuda", dtype=torch.float64), logp.double().cumsum(0)])
        s["ref_sums"] = (total[s["starts"][1:].long()] - total[s["starts"][:-1].long()]).float() + vector(sequences, 5.0)
        s["dZ"], s["sums"] = _matrix(case, classes, batch), torch.zeros(sequences, device="cuda")
        s["margins"], s["loss"] = torch.zeros(case["pairs"], device="cuda"), torch.zeros(1, device="cuda")
    if own:
        from paper_2407_17437_amd import binding as nb
        s["workspace"] = torch.empty(max(4, nb.label_loss_workspace_bytes(classes, batch, sequences) // 4), device="cuda")
    return s


# ---- the plain forms ---------------------------------------------------------------------------

def _plain_kept(s):
    """What every entry is multiplied by: 0 where it is dropped.  Philox4x32 of 10 rounds (Salmon, Moraes, Dror, Shaw 2011); a product of two 32-bit
    numbers wraps in 64 signed bits without losing one."""
    features, batch = s["X"].shape
    cut = min(65535, int(math.floor(s["drop"] * 65536 + 0.5)))
    device, low = s["X"].device, 0xFFFFFFFF
    k0, k1 = s["state"][0] & low, (s["state"][0] >> 32) & low
    c0 = torch.arange((batch + 3) // 4, device=device)[None, :]
    c1 = torch.arange((features + 1) // 2, device=device)[:, None]
    c2, c3 = torch.full((1, 1), LAYER, device=device), (s["state"][1] & low).view(1, 1)
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([t.expand(c0.shape) for t in (c0, c1, c2, c3)], dim=-1).flatten(1)
    kept = torch.stack([words & 0xFFFF, words >> 16], dim=1).flatten(0, 1)[:features, :batch] >= cut
    return kept.float() * (65536.0 / (65536 - cut))


def _plain_norm(s):
    X, groups, act = s["X"], s["groups"], s["act"]
    features, batch = X.shape
    x = X.view(groups, features // groups, batch) if X.is_contiguous() else X.reshape(groups, features // groups, batch)
    gamma = 1.0 if s["gamma"] is None else s["gamma"].view(groups, -1, 1)
    beta = 0.0 if s["beta"] is None else s["beta"].view(groups, -1, 1)
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    xh = d * rstd
    u = gamma * xh + beta
    if act == "silu":
        sig = 1 / (1 + torch.exp(-u))
        y = u * sig
    else:
        y = torch.clamp(u, min=0) if act == "relu" else u
    kept = _plain_kept(s).view_as(x) if s["drop"] > 0 else None
    if kept is not None:
        y = y * kept
    out = [y.reshape(features, batch), mean[:, 0], rstd[:, 0]]
    if s["train"]:
        e = s["dY"].reshape(x.shape)
        if kept is not None:
            e = e * kept
        if act == "silu":
            e = e * (sig * (1 + u * (1 - sig)))
        elif act == "relu":
            e = e * (u > 0)
        h = e * gamma
        dX = rstd * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
        out += [dX.reshape(features, batch), (e * xh).sum(2).flatten(), e.sum(2).flatten()]
    return out


def _plain_columns(s):
    """Which columns count, their labels, the largest logit and the logarithm of the sum of exponentials beyond it.  The sums of exponentials
    and what is subtracted from them are held in 64 bits: log-probabilities are added up over sequences and compared with borders."""
    Z = s["Z"]
    label = s["labels"].long()
    inside = (label >= 0) & (label < Z.shape[0])
    label = label.clamp(0, Z.shape[0] - 1)
    at = Z.gather(0, label[None])[0]
    counts = inside & ~torch.isneginf(at)
    top = Z.amax(0)
    top = torch.where(torch.isneginf(top), torch.zeros_like(top), top)
    if s["kind"] == "policy":
        log_sum = torch.exp(Z.double() - top).sum(0).log()
    else:
        log_sum = torch.exp(Z - top).sum(0, dtype=torch.float64).log()
    logp = torch.where(counts, at.double() - top - log_sum, 0.0)
    return counts, label, top, log_sum, logp


def _plain_gradient(s, c, label, top, log_sum):
    """c (onehot - p), c of every column; 0 in columns that do not count"""
    p = torch.exp((s["Z"] - top) - log_sum.float())
    dZ = torch.where(c == 0, 0.0, -c * p)
    return dZ.scatter_add_(0, label[None], c[None])


def _plain_sums(s, logp):
    n = s["starts"].numel() - 1
    column = torch.arange(logp.numel(), device=logp.device)
    of = (column[:, None] >= s["starts"][None, :]).sum(1) - 1
    held = (of >= 0) & (of < n)
    sums = torch.zeros(n + 1, dtype=torch.float64, device=logp.device)
    sums.index_add_(0, torch.where(held, of, n), logp)
    return sums[:n], of, held


def _plain_score(s):
    logp = _plain_columns(s)[-1]
    return [logp.float(), _plain_sums(s, logp)[0].float()]


def _plain_policy(s):
    counts, label, top, log_sum, logp = _plain_columns(s)
    A = s["advantages"].double()
    w = torch.full_like(A, 1 / A.numel()) if s["weights"] is None else s["weights"].double()
    used = counts & (w != 0)
    r = torch.exp(logp - s["old"].double())
    clipped = torch.where(A > 0, r > 1 + CLIP_HIGH, (A < 0) & (r < 1 - CLIP_LOW))
    loss = -torch.minimum(r * A, r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * A)
    slope = torch.where(clipped, 0.0, -r * A)
    kl = torch.zeros_like(loss)
    if s["ref"] is not None:
        q = torch.exp(s["ref"].double() - logp)
        kl = q - (s["ref"].double() - logp) - 1
        slope = slope + KL * (1 - q)
    w = torch.where(used, w, 0.0)
    total = torch.stack([(w * (loss + KL * kl)).sum(), (w * loss).sum(), (w * kl).sum(), (w * clipped).sum()])
    return [total.float(), logp.float(), _plain_gradient(s, (w * slope).float(), label, top, log_sum)]


def _plain_preference(s):
    counts, label, top, log_sum, logp = _plain_columns(s)
    sums, of, held = _plain_sums(s, logp)
    pairs = sums.numel() // 2
    beyond = (sums - s["ref_sums"].double()).view(pairs, 2)
    margin = BETA * (beyond[:, 0] - beyond[:, 1])
    tail = torch.log1p(torch.exp(-margin.abs()))
    loss = (1 - SMOOTHING) * (tail + torch.clamp(-margin, min=0)) + SMOOTHING * (tail + torch.clamp(margin, min=0))
    slope = (1 / (1 + torch.exp(-margin)) - (1 - SMOOTHING)) * BETA / pairs
    both = torch.stack([slope, -slope], 1).flatten()
    c = torch.where(held & counts, both[of.clamp(0, 2 * pairs - 1)], 0.0)
    return [loss.mean().float().view(1), sums.float(), margin.float(), _plain_gradient(s, c.float(), label, top, log_sum)]


# ---- one pass ----------------------------------------------------------------------------------

def run(state):
    s, kind = state, state["kind"]
    if not own:
        if kind == "dropout":
            # the mask is never stored: each pass draws it
            return [s["X"] * _plain_kept(s), s["dY"] * _plain_kept(s)]
        return {"norm": _plain_norm, "score": _plain_score, "policy": _plain_policy, "preference": _plain_preference}[kind](s)
    from paper_2407_17437_amd import binding as nb
    batch = s["batch"]
    if kind == "norm":
        features, groups, act, drop = s["features"], s["groups"], s["act_code"], s["drop"]
        nb.group_norm_forward(s["X"], s["gamma"], s["beta"], features, groups, batch, EPS, act, drop, LAYER, s["state"], s["Y"], s["mean"], s["rstd"], s["workspace"])
        if not s["train"]:
            return [s["Y"], s["mean"], s["rstd"]]
        nb.group_norm_backward(s["X"], s["gamma"], s["beta"], s["mean"], s["rstd"], s["dY"], features, groups, batch, act, drop, LAYER, s["state"],
                               s["dX"], s["dgamma"], s["dbeta"], s["workspace"])
        return [s["Y"], s["mean"], s["rstd"], s["dX"], s["dgamma"], s["dbeta"]]
    if kind == "dropout":
        nb.dropout(s["X"], s["features"], batch, s["drop"], LAYER, s["state"], s["Y"])
        nb.dropout(s["dY"], s["features"], batch, s["drop"], LAYER, s["state"], s["dX"])
        return [s["Y"], s["dX"]]
    classes = s["classes"]
    if kind == "score":
        nb.label_log_probs(s["Z"], s["labels"], classes, batch, s["starts"], s["sequences"], s["logp"], s["sums"], s["workspace"])
        return [s["logp"], s["sums"]]
    if kind == "policy":
        nb.policy_loss(s["Z"], s["labels"], s["old"], s["ref"], s["advantages"], s["weights"], classes, batch, CLIP_LOW, CLIP_HIGH, KL,
                       s["dZ"], s["logp"], s["stats"], s["workspace"])
        return [s["stats"], s["logp"], s["dZ"]]
    nb.preference_loss(s["Z"], s["labels"], s["starts"], s["ref_sums"], classes, batch, s["pairs"], BETA, SMOOTHING,
                       s["dZ"], s["sums"], s["margins"], s["loss"], s["workspace"])
    return [s["loss"], s["sums"], s["margins"], s["dZ"]]


# ---- the definitions in 64 bits ----------------------------------------------------------------

def _exact_factor(s):
    """0 or 1/(1-p) of every entry: the generator in limbs of 16 bits, its words looked up entry by entry"""
    features, batch = s["X"].shape
    device = s["X"].device
    seed, step = int(s["state"][0]), int(s["state"][1]) % 2 ** 32
    key = [seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32]

    def product(constant, t):
        part = constant * (t % 65536)
        rest = constant * (t // 65536) + part // 65536
        return rest // 65536, rest % 65536 * 65536 + part % 65536

    quads, pairs = (batch + 3) // 4, (features + 1) // 2
    every = torch.arange(quads * pairs, device=device)
    x = [every % quads, every // quads, torch.full_like(every, LAYER), torch.full_like(every, step)]
    for r in range(10):
        (h0, l0), (h2, l2) = product(0xD2511F53, x[0]), product(0xCD9E8D57, x[2])
        x = [h2 ^ x[1] ^ ((key[0] + r * 0x9E3779B9) % 2 ** 32), l2, h0 ^ x[3] ^ ((key[1] + r * 0xBB67AE85) % 2 ** 32), l0]
    cut = min(65535, math.floor(s["drop"] * 65536 + 0.5))
    factor = torch.zeros(features, batch, dtype=torch.float64, device=device)
    for word in range(min(4, batch)):
        for half in range(min(2, features)):
            number = x[word].view(pairs, quads) // 65536 ** half % 65536
            part = factor[half::2, word::4]
            part.copy_((number >= cut)[:part.shape[0], :part.shape[1]])
    return factor * (65536 / (65536 - cut))


def _exact_norm(s):
    features, batch = s["X"].shape
    train = s["train"]
    x = s["X"].double().t().contiguous().requires_grad_(train)
    gamma = (torch.ones(features, device=x.device) if s["gamma"] is None else s["gamma"]).double().requires_grad_(train)
    beta = (torch.zeros(features, device=x.device) if s["beta"] is None else s["beta"]).double().requires_grad_(train)
    var, mean = torch.var_mean(x.view(batch, s["groups"], -1), dim=2, correction=0, keepdim=True)
    y = torch.addcmul(beta, ((x.view(batch, s["groups"], -1) - mean) / (var + EPS).sqrt()).view(batch, features), gamma)
    y = torch.nn.functional.silu(y) if s["act"] == "silu" else torch.relu(y) if s["act"] == "relu" else y
    if s["drop"] > 0:
        y = y * _exact_factor(s).t()
    out = [t.detach().t().contiguous() for t in (y, mean[:, :, 0], (var[:, :, 0] + EPS).rsqrt())]
    if train:
        y.backward(s["dY"].double().t())
        out += [x.grad.t().contiguous(), gamma.grad, beta.grad]
    return out


def _exact_logp(s, Z):
    """log-probabilities by columns of those that count, and which do"""
    label = s["labels"].long()
    counts = (label >= 0) & (label < Z.shape[0])
    column = torch.nonzero(counts).flatten()
    column = column[~torch.isneginf(s["Z"][label[column], column])]
    # (only the columns that count: an empty one has no logarithm)
    logs = torch.log_softmax(Z[:, column], 0)
    return column, logs.gather(0, label[column][None])[0]


def _spread(s, column, values):
    return torch.zeros(s["Z"].shape[1], dtype=torch.float64, device=values.device).index_copy(0, column, values)


def _exact_sums(s, logp):
    starts = s["starts"].tolist()
    return torch.stack([logp[a:b].sum() for a, b in zip(starts[:-1], starts[1:])])


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    with torch.enable_grad():
        if kind == "norm":
            return _exact_norm(s)
        if kind == "dropout":
            factor = _exact_factor(s)
            return [s["X"].double() * factor, s["dY"].double() * factor]
        Z = s["Z"].double().requires_grad_(kind != "score")
        column, values = _exact_logp(s, Z)
        logp = _spread(s, column, values)
        if kind == "score":
            return [logp, _exact_sums(s, logp)]
        if kind == "policy":
            A = s["advantages"].double()[column]
            w = torch.full_like(A, 1 / case["batch"]) if s["weights"] is None else s["weights"].double()[column]
            r = torch.exp(values - s["old"].double()[column])
            bounded = torch.clamp(r, 1 - CLIP_LOW, 1 + CLIP_HIGH)
            gain = torch.minimum(r * A, bounded * A)
            kl = torch.zeros_like(gain)
            if s["ref"] is not None:
                apart = s["ref"].double()[column] - values
                kl = torch.expm1(apart) - apart
            shares = [(w * (KL * kl - gain)).sum(), -(w * gain).sum(), (w * kl).sum(), (w * (r * A > bounded * A)).sum()]
            shares[0].backward()
            return [torch.stack([t.detach() for t in shares]), logp.detach(), Z.grad]
        sums = _exact_sums(s, logp)
        beyond = sums - s["ref_sums"].double()
        margin = BETA * (beyond[0::2] - beyond[1::2])
        log_sigmoid = torch.nn.functional.logsigmoid
        loss = -((1 - SMOOTHING) * log_sigmoid(margin) + SMOOTHING * log_sigmoid(-margin)).mean()
        loss.backward()
        return [loss.detach().view(1), sums.detach(), margin.detach(), Z.grad]


def work(case):
    """Inputs read once and outputs written once, fp32 and int32; an exponential or a draw of the generator counts as one operation."""
    kind, batch = case["kind"], case["batch"]
    if kind == "norm":
        n = case["features"] * batch
        byt = 8 * n + 8 * case["groups"] * batch + (8 * case["features"] if case["affine"] else 0)
        flops = 9 * n + (3 * n if case["act"] == "silu" else 0)
        if case["train"]:
            byt += 8 * n + 8 * case["features"]
            flops += 14 * n + (5 * n if case["act"] == "silu" else 0)
        return {"bytes": byt, "flops": flops}
    if kind == "dropout":
        n = case["features"] * batch
        return {"bytes": 16 * n, "flops": 4 * n}
    n = case["classes"] * batch
    if kind == "score":
        return {"bytes": 4 * n + 8 * batch + 8 * case["sequences"], "flops": 3 * n}
    if kind == "policy":
        return {"bytes": 8 * n + batch * (16 + 4 * case["kl"] + 4 * case["weighted"]) + 16, "flops": 6 * n}
    return {"bytes": 8 * n + 4 * batch + 28 * case["pairs"], "flops": 6 * n}

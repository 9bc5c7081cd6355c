"""Mixtures of sparse layers and the clipped momentum step: the work of these operators as measurable cases.

`run` with `own` true makes the calls of `paper_2407_17437_amd.binding`; with `own` false it computes the same in
elementary torch operations.  As everywhere in the library an operand holds one example per column.

route     logits (experts, batch) -> the k experts of every column and their weights, and the gradient of the logits.
exchange  the columns of X go to one block (features, capacity) per expert, the operand that a sparse layer takes, and
          the experts' results come back weighted; with the gradients of both ways.
update    one momentum step on the arrays of many layers with their gradients clipped to a norm that is taken over all of them.
clip      such gradients themselves, clipped, for a program with an optimiser of its own.
"""
from __future__ import annotations

import math

import torch

own = False

LR, MOMENTUM, MAX_NORM = 0.015625, 0.875, 1.0
PAPER = "3072-1024-512-10"
WIDE = "3072-8192-8192-10"


def listed():
    return [
        # Serving one example: every launch counts.  Sigmoid scores with a bias for balance, best three of eight groups.
        {"name": "route one", "kind": "route", "experts": 64, "batch": 1, "k": 6, "sigmoid": True, "renorm": True, "bias": True, "groups": 8, "top_groups": 3,
         "pair": True, "masked": 0.0, "train": False, "padded": True},
        # A small mixture at an ordinary mini-batch, plain softmax weights, with the gradient of the logits.
        {"name": "route batch", "kind": "route", "experts": 16, "batch": 1024, "k": 2, "sigmoid": False, "renorm": False, "bias": False, "groups": 1, "top_groups": 1,
         "pair": False, "masked": 0.0, "train": True, "padded": True},
        # The short last mini-batch of an epoch, stored without padding; some experts are closed to some columns, and some columns have none.
        {"name": "route ragged", "kind": "route", "experts": 60, "batch": 777, "k": 4, "sigmoid": False, "renorm": True, "bias": False, "groups": 1, "top_groups": 1,
         "pair": False, "masked": 0.1, "train": True, "padded": False},
        # Many experts and a large batch.
        {"name": "route large", "kind": "route", "experts": 256, "batch": 16384, "k": 8, "sigmoid": True, "renorm": True, "bias": True, "groups": 8, "top_groups": 4,
         "pair": True, "masked": 0.0, "train": True, "padded": True},
        # Serving a few examples through a mixture of 1024-wide layers.
        {"name": "exchange few", "kind": "exchange", "experts": 64, "features": 1024, "batch": 4, "k": 6, "capacity": 4, "train": False, "padded": True},
        # A training step of a mixture of the paper's hidden layers.
        {"name": "exchange batch", "kind": "exchange", "experts": 8, "features": 1024, "batch": 1024, "k": 2, "capacity": 320, "train": True, "padded": True},
        # Odd sizes without padding, and blocks that are too small for the most popular experts.
        {"name": "exchange ragged", "kind": "exchange", "experts": 60, "features": 1501, "batch": 777, "k": 4, "capacity": 52, "train": True, "padded": False},
        # Wide layers and a large batch: the largest of all cases.
        {"name": "exchange large", "kind": "exchange", "experts": 64, "features": 4096, "batch": 8192, "k": 4, "capacity": 640, "train": True, "padded": True},
        # The arrays of the paper's network at 99 % sparsity: all of them fit the caches, so launches count.
        {"name": "update paper", "kind": "update", "sizes": PAPER, "density": 0.01, "copies": 1, "norm": 3.0, "nesterov": True, "padded": True},
        # The wide network at 5 %, its arrays right behind each other.
        {"name": "update wide", "kind": "update", "sizes": WIDE, "density": 0.05, "copies": 1, "norm": 0.5, "nesterov": False, "padded": False},
        # 64 experts of two layers each: 256 arrays, 134 M entries.
        {"name": "update mixture", "kind": "update", "sizes": "4096-4096-4096", "density": 0.0625, "copies": 64, "norm": 8.0, "nesterov": False, "padded": True},
        # The gradients of 16 such experts, clipped and kept beside the raw ones.
        {"name": "clip mixture", "kind": "clip", "sizes": "4096-4096-4096", "density": 0.0625, "copies": 16, "norm": 8.0, "padded": True},
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(_log_uniform(rng, lo, hi)))))


def draw(rng):
    most = work(listed()[7])
    while True:
        kind = rng.choice(["route"] * 4 + ["exchange"] * 4 + ["update"] * 3 + ["clip"])
        if kind == "route":
            groups = rng.choice([1, 1, 2, 4, 7, 8])
            experts = groups * _log_int(rng, max(1, 4 // groups), 256 // groups)
            top_groups = rng.randint(1, groups)
            k = min(rng.choice([1, 2, 2, 3, 4, 6, 8]), experts // groups * top_groups)
            case = {"kind": kind, "experts": experts, "batch": _log_int(rng, 1, 16384), "k": k, "sigmoid": rng.random() < 0.5, "renorm": rng.random() < 0.6,
                    "bias": rng.random() < 0.5, "groups": groups, "top_groups": top_groups, "pair": groups > 1 and rng.random() < 0.5,
                    "masked": rng.choice([0.0, 0.0, 0.1, 0.4]), "train": rng.random() < 0.6, "padded": rng.random() < 0.6}
        elif kind == "exchange":
            experts, batch = _log_int(rng, 4, 256), _log_int(rng, 1, 8192)
            k = min(rng.choice([1, 2, 2, 3, 4, 6, 8]), experts)
            case = {"kind": kind, "experts": experts, "features": _log_int(rng, 64, 4096), "batch": batch, "k": k,
                    "capacity": max(1, min(batch, int(math.ceil(batch * k / experts * rng.uniform(0.8, 2.0))))), "train": rng.random() < 0.7,
                    "padded": rng.random() < 0.6}
        else:
            sizes = "-".join(str(_log_int(rng, 10, 4096)) for _ in range(rng.choice([2, 3, 3, 4])))
            case = {"kind": kind, "sizes": sizes, "density": round(_log_uniform(rng, 0.001, 0.5), 5), "copies": _log_int(rng, 1, 64),
                    "norm": round(_log_uniform(rng, 0.2, 20.0), 3), "padded": rng.random() < 0.6}
            if kind == "update":
                case["nesterov"] = rng.random() < 0.5
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


def _blocks(case, gen=None):
    """(experts, features, capacity): one operand of a sparse layer per expert."""
    t = torch.zeros(case["experts"], case["features"], _ld(case, case["capacity"]), device="cuda")[:, :, :case["capacity"]]
    if gen is not None:
        t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
    return t


def _counts(case):
    """Lengths of the arrays: entries and biases of every layer, expert after expert."""
    sizes = [int(s) for s in case["sizes"].split("-")]
    one = []
    for cols, rows in zip(sizes[:-1], sizes[1:]):
        one += [max(1, int(rows * cols * case["density"])), rows]
    return one * case["copies"]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case)
    kind = case["kind"]
    if kind == "route":
        experts, batch, k = case["experts"], case["batch"], case["k"]
        # experts differ in popularity, as they do before a bias has balanced them
        s["Z"] = _matrix(case, experts, batch, gen)
        s["Z"] += 0.5 * torch.randn(experts, 1, generator=gen, device="cuda")
        if case["masked"] > 0:
            closed = torch.rand(experts, batch, generator=gen, device="cuda") < case["masked"]
            closed |= torch.rand(1, batch, generator=gen, device="cuda") < 0.02
            s["Z"].masked_fill_(closed, -math.inf)
        s["b"] = 0.1 * torch.randn(experts, generator=gen, device="cuda") if case["bias"] else None
        s["chosen"] = torch.zeros(k, _ld(case, batch), dtype=torch.int32, device="cuda")[:, :batch]
        s["weights"] = _matrix(case, k, batch)
        if case["train"]:
            s["dweights"] = _matrix(case, k, batch, gen)
            s["dZ"] = _matrix(case, experts, batch)
    elif kind == "exchange":
        experts, batch, k, features = case["experts"], case["batch"], case["k"], case["features"]
        z = torch.randn(experts, batch, generator=gen, device="cuda") + 0.5 * torch.randn(experts, 1, generator=gen, device="cuda")
        top = z.topk(k, dim=0)
        s["chosen"] = torch.zeros(k, _ld(case, batch), dtype=torch.int32, device="cuda")[:, :batch]
        s["chosen"].copy_(top.indices)
        s["weights"] = _matrix(case, k, batch)
        s["weights"].copy_(torch.softmax(top.values, dim=0))
        s["X"], s["Xe"] = _matrix(case, features, batch, gen), _blocks(case)
        s["Ye"], s["Y"] = _blocks(case, gen), _matrix(case, features, batch)
        s["slots"] = torch.zeros(k, _ld(case, batch), dtype=torch.int32, device="cuda")[:, :batch]
        s["counts"] = torch.zeros(experts, dtype=torch.int32, device="cuda")
        if case["train"]:
            s["dY"], s["dX"] = _matrix(case, features, batch, gen), _matrix(case, features, batch)
            s["dXe"], s["dYe"] = _blocks(case, gen), _blocks(case)
            s["dweights"] = _matrix(case, k, batch)
        if own:
            from paper_2407_17437_amd import binding as nb
            s["placement"] = torch.empty(nb.expert_placement_bytes(experts, batch, k) // 4, dtype=torch.int32, device="cuda")
            s["workspace"] = torch.empty(max(4, nb.expert_combine_workspace_bytes(features, batch, k)) // 4, device="cuda")
    else:
        counts = _counts(case)
        sigma = case["norm"] * MAX_NORM / math.sqrt(sum(counts))
        # one allocation for all arrays of a sort, every array on a 128-byte line of its own or right behind the one before
        step = 32 if case["padded"] else 1
        starts, room = [], 0
        for n in counts:
            starts.append(room)
            room += (n + step - 1) // step * step

        def arrays(scale):
            flat = scale * torch.randn(room, generator=gen, device="cuda")
            return flat, [flat[at:at + n] for at, n in zip(starts, counts)]

        _, s["grads"] = arrays(sigma)
        if kind == "update":
            s["all_values"], s["values"] = arrays(0.1)
            s["all_velocities"], s["velocities"] = arrays(LR * sigma)
        else:
            s["all_clipped"], s["clipped"] = arrays(0.0)
        s["norm_out"] = torch.zeros(1, device="cuda")
        if own:
            from paper_2407_17437_amd import binding as nb
            s["workspace"] = torch.empty(nb.gradient_norm_workspace_bytes(len(counts)) // 4, device="cuda")
    return s


# ---- the plain forms ---------------------------------------------------------------------------

def _log_score(z, sigmoid):
    """Logarithm of a sigmoid score; of a softmax score up to the column's sum."""
    return torch.clamp(z, max=0) - torch.log1p(torch.exp(-z.abs())) if sigmoid else z


def _plain_route(s):
    Z, k, groups = s["Z"], s["k"], s["groups"]
    experts, batch = Z.shape
    # two scores that lie closer than 32 bits tell apart are ordered in 64
    z = Z.double()
    closed = torch.isneginf(z)
    top = z.amax(0)
    top = torch.where(torch.isneginf(top), torch.zeros_like(top), top)
    e = torch.exp(z - top)
    score = 1 / (1 + torch.exp(-z)) if s["sigmoid"] else e / e.sum(0).clamp(min=1)
    key = z if s["b"] is None and not s["pair"] else score if s["b"] is None else score + s["b"].double()[:, None]
    key = key.masked_fill(closed, -math.inf)
    if groups > 1:
        of_group = key.view(groups, experts // groups, batch).sort(dim=1, descending=True).values
        best = of_group[:, 0]
        if s["pair"] and experts // groups > 1:
            second = of_group[:, 1]
            best = torch.where(torch.isneginf(second), best, best + second)
        order = best.sort(dim=0, descending=True, stable=True).indices[:s["top_groups"]]
        kept = torch.zeros(groups, batch, dtype=torch.bool, device=Z.device).scatter_(0, order, True)
        key = key.masked_fill(~kept.repeat_interleave(experts // groups, 0), -math.inf)
    key, chosen = key.sort(dim=0, descending=True, stable=True)
    key, chosen = key[:k], chosen[:k]
    none = torch.isneginf(key)
    zc = Z.gather(0, chosen)
    if s["renorm"]:
        log_score = _log_score(zc, s["sigmoid"]).masked_fill(none, -math.inf)
        high = log_score.amax(0)
        high = torch.where(torch.isneginf(high), torch.zeros_like(high), high)
        w = torch.exp(log_score - high)
        w = w / w.sum(0).clamp(min=1)
    else:
        w = score.gather(0, chosen).float()
    w = (2.5 * w).masked_fill(none, 0)
    chosen = chosen.to(torch.int32).masked_fill(none, -1)
    if not s["train"]:
        return [chosen, w]
    # gradient of the logits
    dw = s["dweights"].masked_fill(none, 0)
    at = chosen.long().clamp(min=0)
    if s["renorm"]:
        g = w * (dw - (w / 2.5 * dw).sum(0))
        if s["sigmoid"]:
            g = g / (1 + torch.exp(zc))
    elif s["sigmoid"]:
        g = dw * w / (1 + torch.exp(zc))
    else:
        g = dw * w
    g = g.masked_fill(none, 0)
    dZ = torch.zeros(experts, batch, device=Z.device).scatter_add_(0, at, g)
    if not s["renorm"] and not s["sigmoid"]:
        dZ = dZ - score.float() * g.sum(0)
    return [chosen, w, dZ]


def _plain_exchange(s):
    experts, features, capacity, k, batch = s["experts"], s["features"], s["capacity"], s["k"], s["batch"]
    X, Ye, w = s["X"], s["Ye"], s["weights"]
    device = X.device
    # places: the choices sorted by expert, stably, in the order of columns and then of choices
    by_column = s["chosen"].t().reshape(-1).long()
    order = by_column.sort(stable=True).indices
    counts = torch.bincount(by_column, minlength=experts)
    first = counts.cumsum(0) - counts
    place = torch.empty_like(by_column)
    place[order] = torch.arange(batch * k, device=device) - first[by_column[order]]
    place = place.masked_fill(place >= capacity, -1)
    slots = place.view(batch, k).t()
    kept = place >= 0
    block_column = torch.where(kept, by_column * capacity + place, experts * capacity)
    # column of X in every slot (one behind the last: none) and its weight
    source = torch.full((experts * capacity + 1,), batch, device=device)
    source[block_column] = torch.arange(batch * k, device=device) // k
    source = source[:-1]
    weight = torch.zeros(experts * capacity + 1, device=device)
    weight[block_column] = w.t().reshape(-1)
    weight = weight[:-1]
    none = torch.zeros(features, 1, device=device)

    def blocks(columns):
        return torch.cat([columns, none], 1)[:, source].view(features, experts, capacity).permute(1, 0, 2)

    def back(of_blocks, weights):
        flat = torch.cat([of_blocks.permute(1, 0, 2).reshape(features, experts * capacity), none], 1)
        at = block_column.view(batch, k)
        out = torch.zeros(features, batch, device=device)
        for j in range(k):
            part = flat[:, at[:, j]]
            out += part if weights is None else part * weights[j]
        return out

    out = [slots.to(torch.int32), counts.to(torch.int32), blocks(X).contiguous(), back(Ye, w)]
    if s["train"]:
        dY = s["dY"]
        out.append((blocks(dY) * weight.view(experts, 1, capacity)).contiguous())
        flat = torch.cat([Ye.permute(1, 0, 2).reshape(features, experts * capacity), none], 1)
        at = block_column.view(batch, k)
        out.append(torch.stack([(flat[:, at[:, j]] * dY).sum(0) for j in range(k)]))
        out.append(back(s["dXe"], None))
    return out


def _plain_norm(grads):
    total = torch.zeros((), dtype=torch.float64, device=grads[0].device)
    for g in grads:
        total += g.double().square().sum()
    return total.sqrt()


def _plain_clip(s):
    norm = _plain_norm(s["grads"])
    clip = torch.clamp(MAX_NORM / norm, max=1.0).float()
    for out, g in zip(s["clipped"], s["grads"]):
        out.copy_(clip * g)
    return [norm.float().view(1), s["all_clipped"]]


def _plain_update(s):
    norm = _plain_norm(s["grads"])
    clip = torch.clamp(MAX_NORM / norm, max=1.0).float()
    for w, v, g in zip(s["values"], s["velocities"], s["grads"]):
        step = LR * (clip * g)
        v.copy_(MOMENTUM * v - step)
        w.copy_(w + (MOMENTUM * v - step if s["nesterov"] else v))
    return [norm.float().view(1), s["all_values"], s["all_velocities"]]


# ---- one pass ----------------------------------------------------------------------------------

def run(state):
    s, kind = state, state["kind"]
    if not own:
        if kind == "route":
            return _plain_route(s)
        if kind == "exchange":
            return _plain_exchange(s)
        return _plain_clip(s) if kind == "clip" else _plain_update(s)
    from paper_2407_17437_amd import binding as nb
    if kind == "route":
        flags = (nb.NERVA_EXPERT_SIGMOID * s["sigmoid"]) | (nb.NERVA_EXPERT_RENORMALISE * s["renorm"]) | (nb.NERVA_EXPERT_GROUP_PAIR * s["pair"])
        nb.expert_route(s["Z"], s["b"], s["experts"], s["batch"], s["k"], s["groups"], s["top_groups"], flags, 2.5, s["chosen"], s["weights"])
        if not s["train"]:
            return [s["chosen"], s["weights"]]
        nb.expert_route_backward(s["Z"], s["chosen"], s["dweights"], s["experts"], s["batch"], s["k"], flags, 2.5, s["dZ"])
        return [s["chosen"], s["weights"], s["dZ"]]
    if kind == "exchange":
        experts, features, batch, k, capacity, placement = s["experts"], s["features"], s["batch"], s["k"], s["capacity"], s["placement"]
        nb.expert_place(s["chosen"], experts, batch, k, capacity, s["slots"], s["counts"], placement)
        nb.expert_dispatch(s["X"], placement, features, experts, batch, k, capacity, s["Xe"])
        nb.expert_combine(s["Ye"], placement, s["weights"], features, experts, batch, k, capacity, s["Y"])
        out = [s["slots"], s["counts"], s["Xe"], s["Y"]]
        if s["train"]:
            nb.expert_combine_backward(s["Ye"], s["dY"], placement, s["weights"], features, experts, batch, k, capacity, s["dYe"], s["dweights"], s["workspace"])
            nb.expert_combine(s["dXe"], placement, None, features, experts, batch, k, capacity, s["dX"])
            out += [s["dYe"], s["dweights"], s["dX"]]
        return out
    if kind == "clip":
        nb.gradient_clip(s["grads"], s["clipped"], MAX_NORM, s["workspace"], s["norm_out"])
        return [s["norm_out"], s["all_clipped"]]
    nb.sgd_update_clipped(s["values"], s["velocities"], s["grads"], LR, MOMENTUM, MAX_NORM, s["nesterov"], s["workspace"], s["norm_out"])
    return [s["norm_out"], s["all_values"], s["all_velocities"]]


# ---- the definitions in 64 bits ----------------------------------------------------------------

def _exact_route(s):
    Z, k, groups = s["Z"].double(), s["k"], s["groups"]
    experts, batch = Z.shape
    size = experts // groups
    neg = torch.tensor(-math.inf, dtype=torch.float64, device=Z.device)
    columns = torch.arange(batch, device=Z.device)
    if s["sigmoid"]:
        log_score = -torch.logaddexp(torch.zeros_like(Z), -Z)
    else:
        log_score = Z - torch.logsumexp(Z, 0)
        log_score = torch.where(torch.isneginf(Z), neg, log_score)
    p = torch.exp(log_score)
    order_by = Z.clone()
    if s["b"] is not None or s["pair"]:
        order_by = p + (0 if s["b"] is None else s["b"].double()[:, None])
        order_by = torch.where(torch.isneginf(Z), neg, order_by)

    def lowest_best(t):
        """index of the first of the largest values of each column"""
        high = t.amax(0)
        return torch.where(t == high, torch.arange(t.shape[0], device=t.device)[:, None], t.shape[0]).amin(0), high

    if groups > 1:
        rows = []
        for g in range(groups):
            part = order_by[g * size:(g + 1) * size].clone()
            at, high = lowest_best(part)
            total = high
            if s["pair"]:
                part[at, columns] = neg
                second = part.amax(0)
                total = torch.where(torch.isneginf(second), high, high + second)
            rows.append(total)
        by_group = torch.stack(rows)
        open_groups = torch.zeros(groups, batch, dtype=torch.bool, device=Z.device)
        taken = by_group.clone()
        for _ in range(s["top_groups"]):
            left = torch.where(open_groups, neg, taken)
            # (a group without an open expert has nothing to choose from, taken or not)
            at, _ = lowest_best(left)
            open_groups[at, columns] = True
        order_by = torch.where(open_groups[torch.arange(experts, device=Z.device) // size], order_by, neg)
    chosen, logs = [], []
    left = order_by.clone()
    for _ in range(k):
        at, high = lowest_best(left)
        none = torch.isneginf(high)
        chosen.append(torch.where(none, -1, at))
        logs.append(torch.where(none, neg, log_score[at, columns]))
        left[at, columns] = neg
    chosen, logs = torch.stack(chosen), torch.stack(logs)
    none = chosen < 0
    base = torch.logsumexp(logs, 0) if s["renorm"] else torch.zeros(batch, dtype=torch.float64, device=Z.device)
    zero = torch.zeros_like(base)
    u = torch.where(none, zero, torch.exp(logs - base))
    if not s["train"]:
        return [chosen.to(torch.int32), 2.5 * u]
    # d log_score, column by column of the Jacobian, then through the score
    dw = torch.where(none, zero, 2.5 * s["dweights"].double())
    d_log = u * dw
    if s["renorm"]:
        d_log = d_log - u * d_log.sum(0)
    onto = torch.zeros(experts + 1, batch, dtype=torch.float64, device=Z.device)
    onto.scatter_add_(0, torch.where(none, experts, chosen.long()), d_log)
    onto = onto[:experts]
    if s["sigmoid"]:
        dZ = onto * torch.exp(-torch.logaddexp(torch.zeros_like(Z), Z))
    else:
        dZ = onto - p * onto.sum(0)
        if s["renorm"]:
            dZ = onto
    return [chosen.to(torch.int32), 2.5 * u, dZ]


def _exact_exchange(s):
    experts, features, capacity, k, batch = s["experts"], s["features"], s["capacity"], s["k"], s["batch"]
    device = s["X"].device
    chosen = s["chosen"].long()
    # number of earlier choices of the same expert, by counting over columns (a column chooses an expert once)
    took = torch.zeros(experts, batch, dtype=torch.int64, device=device)
    took.scatter_(0, chosen, 1)
    before = took.cumsum(1) - took
    slots = before.gather(0, chosen)
    slots = torch.where(slots < capacity, slots, -1)
    counts = took.sum(1)
    e, c = torch.nonzero(took & (before < capacity), as_tuple=True)
    at = before[e, c]
    j = (chosen[:, c] == e).int().argmax(0)
    w = s["weights"].double()[j, c]

    def scatter(columns):
        out = torch.zeros(features, experts, capacity, dtype=torch.float64, device=device)
        out[:, e, at] = columns
        return out.permute(1, 0, 2)

    def gather(of_blocks):
        return of_blocks.permute(1, 0, 2)[:, e, at].double()

    def add_up(parts):
        return torch.zeros(features, batch, dtype=torch.float64, device=device).index_add_(1, c, parts)

    out = [slots.to(torch.int32), counts.to(torch.int32), scatter(s["X"].double()[:, c]), add_up(gather(s["Ye"]) * w)]
    if s["train"]:
        dY = s["dY"].double()[:, c]
        out.append(scatter(dY * w))
        dw = torch.zeros(k, batch, dtype=torch.float64, device=device)
        dw[j, c] = (gather(s["Ye"]) * dY).sum(0)
        out.append(dw)
        out.append(add_up(gather(s["dXe"])))
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "route":
        return _exact_route(s)
    if case["kind"] == "exchange":
        return _exact_exchange(s)
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g.double()) for g in s["grads"]]))
    ratio = 1.0 if norm <= MAX_NORM else MAX_NORM / norm
    if case["kind"] == "clip":
        clipped = s["all_clipped"].double()
        for g in s["grads"]:
            at = slice(g.storage_offset(), g.storage_offset() + g.numel())
            clipped[at] = g.double() * ratio
        return [norm.view(1), clipped]
    values, velocities = s["all_values"].double(), s["all_velocities"].double()
    for w, g in zip(s["values"], s["grads"]):
        at = slice(w.storage_offset(), w.storage_offset() + w.numel())
        step = g.double() * (LR * ratio)
        velocities[at] = velocities[at] * MOMENTUM - step
        values[at] += velocities[at] * MOMENTUM - step if case["nesterov"] else velocities[at]
    return [norm.view(1), values, velocities]


def work(case):
    """Inputs read once and outputs written once, fp32 and int32."""
    kind = case["kind"]
    if kind == "route":
        experts, batch, k = case["experts"], case["batch"], case["k"]
        byt = 4 * experts * batch + 8 * k * batch + (4 * experts if case["bias"] else 0)
        flops = 8 * experts * batch
        if case["train"]:
            byt += 4 * k * batch + 4 * experts * batch
            flops += 4 * experts * batch
        return {"bytes": byt, "flops": flops}
    if kind == "exchange":
        experts, batch, k, features, capacity = case["experts"], case["batch"], case["k"], case["features"], case["capacity"]
        room = experts * capacity
        kept = min(batch * k, room)
        byt = 12 * batch * k + 4 * experts                       # choices, weights and places
        byt += 4 * features * (batch + room)                     # X to the blocks
        byt += 4 * features * (kept + batch)                     # the blocks' results to Y
        flops = 2 * kept * features
        if case["train"]:
            byt += 4 * features * (batch + room)                 # dY to the gradients of the blocks (their results are read above)
            byt += 4 * batch * k                                 # gradients of the weights
            byt += 4 * features * (kept + batch)                 # dX
            flops += 4 * kept * features
        return {"bytes": byt, "flops": flops}
    n = sum(_counts(case))
    if kind == "clip":
        return {"bytes": 8 * n + 4, "flops": 3 * n}
    return {"bytes": 20 * n + 4, "flops": 7 * n}

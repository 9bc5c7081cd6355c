"""Plain 64-bit forms of routing, places and the exchange with the experts' blocks, written from their definitions with loops over
columns; and error bounds of the fp32 forms, counted in roundings (u = 2^-24, half a step of fp32 relative to the value).

exp, log1p and their like are taken to be within 2 steps (4 u) of the exact value."""
import numpy as np

U = 2.0 ** -24
TINY = 1e-37   # results below the smallest normal number may be flushed


def log_sigmoid(z):
    with np.errstate(over="ignore"):
        return np.minimum(z, 0) - np.log1p(np.exp(-np.abs(z)))


def route(Z, bias, k, groups, top_groups, sigmoid, renorm, pair, scale):
    """chosen, weights, and the bound of the weights' errors."""
    Z = np.asarray(Z, np.float64)
    E, B = Z.shape
    size = E // groups
    chosen = np.full((k, B), -1, np.int32)
    weights = np.zeros((k, B))
    bound = np.zeros((k, B))
    for c in range(B):
        z = Z[:, c].copy()
        bad = np.isnan(z) | (np.isposinf(z) & (not sigmoid))
        z[bad] = -np.inf
        open_ = z > -np.inf
        top = z[open_].max() if open_.any() else 0.0
        with np.errstate(over="ignore", invalid="ignore"):
            total = np.exp(z[open_] - top).sum()
            score = np.where(open_, np.where(z >= 0, 1 / (1 + np.exp(-z)), np.exp(z) / (1 + np.exp(z))) if sigmoid else np.exp(z - top) / max(total, 1), 0)
        key = z.copy()
        if bias is not None or (pair and groups > 1):
            key = np.where(open_, score + (0 if bias is None else np.asarray(bias, np.float64)), -np.inf)
        key[np.isnan(key)] = -np.inf
        if groups > 1:
            value = []
            for g in range(groups):
                q = np.sort(key[g * size:(g + 1) * size])[::-1]
                value.append(q[0] + q[1] if pair and size > 1 and q[1] > -np.inf else q[0])
            taken = sorted(range(groups), key=lambda g: (-value[g], g))[:top_groups]
            for g in range(groups):
                if g not in taken:
                    key[g * size:(g + 1) * size] = -np.inf
        order = [e for e in sorted(range(E), key=lambda e: (-key[e], e)) if key[e] > -np.inf][:k]
        n = len(order)
        chosen[:n, c] = order
        zc = z[order]
        if renorm and n:
            with np.errstate(invalid="ignore"):
                L = log_sigmoid(zc) if sigmoid else zc
                w = np.exp(L - L.max())
            weights[:n, c] = scale * w / w.sum()
            # the exponent is off by the roundings of both logarithms and of their difference
            far = np.abs(L).max() if sigmoid else 0.0
            err = (2 * far + 2 * (L.max() - L).clip(max=110) + 48) * U
        elif n:
            weights[:n, c] = scale * score[order]
            err = 16 * U if sigmoid else (2 * np.clip(top - z[open_].min(), 0, 110) + 48) * U
        if n:
            bound[:n, c] = np.abs(weights[:n, c]) * err + TINY * max(1.0, abs(scale))
        if bad.any():
            weights[:, c] = np.nan
    return chosen, weights, bound


def route_loss_gradient(Z, chosen, d, sigmoid, renorm, scale):
    """Gradient of sum(d * weights) with respect to Z, the choices held fixed, and the bound of its errors."""
    Z = np.asarray(Z, np.float64)
    E, B = Z.shape
    dZ, bound = np.zeros((E, B)), np.zeros((E, B))
    for c in range(B):
        js = [j for j in range(chosen.shape[0]) if 0 <= chosen[j, c] < E]
        open_ = Z[:, c] > -np.inf
        if not js and (renorm or sigmoid or not open_.any()):
            continue
        e = np.array([chosen[j, c] for j in js], int)
        dj = np.array([d[j, c] for j in js], np.float64)
        z = Z[e, c]
        with np.errstate(over="ignore"):
            s, not_s = 1 / (1 + np.exp(-z)), 1 / (1 + np.exp(z))   # (1 - s itself would cancel)
        if renorm:
            L = log_sigmoid(z) if sigmoid else z
            u = np.exp(L - L.max())
            u /= u.sum()
            g = scale * u * (dj - (u * dj).sum())
            far = np.abs(L).max() if sigmoid else 0.0
            size = scale * u * 2 * np.abs(dj).max() * (2 * far + 2 * (L.max() - L.min()) + 80 + 4 * len(js)) * U
            if sigmoid:
                g, size = g * not_s, size * not_s
            np.add.at(dZ[:, c], e, g)
            np.add.at(bound[:, c], e, size)
        elif sigmoid:
            np.add.at(dZ[:, c], e, scale * dj * s * not_s)
            np.add.at(bound[:, c], e, np.abs(scale * dj * s * not_s) * 32 * U)
        else:
            top = Z[open_, c].max()
            p = np.where(open_, np.exp(Z[:, c] - top), 0)
            p /= p.sum()
            g = scale * p[e] * dj
            np.add.at(dZ[:, c], e, g)
            np.add.at(bound[:, c], e, np.abs(g))
            dZ[:, c] -= p * g.sum()
            bound[:, c] += p * np.abs(g).sum()
            bound[:, c] *= (4 * (top - Z[open_, c].min()) + 96 + 4 * len(js)) * U
        bound[:, c] += TINY * max(1.0, abs(scale))
    return dZ, bound


def place(chosen, experts, capacity):
    k, B = chosen.shape
    slots, counts = np.full((k, B), -1, np.int32), np.zeros(experts, np.int32)
    for c in range(B):
        for j in range(k):
            e = chosen[j, c]
            if 0 <= e < experts:
                if counts[e] < capacity:
                    slots[j, c] = counts[e]
                counts[e] += 1
    return slots, counts


def dispatch(X, chosen, slots, experts, capacity, weights=None):
    """fp32 in, fp32 out: a copy, or one rounded product per entry."""
    X = np.asarray(X, np.float32)
    out = np.zeros((experts, X.shape[0], capacity), np.float32)
    for j, c in zip(*np.nonzero(slots >= 0)):
        out[chosen[j, c], :, slots[j, c]] = X[:, c] if weights is None else np.float32(weights[j, c]) * X[:, c]
    return out


def combine(Ye, chosen, slots, weights=None):
    """In fp32, the products rounded and added up in the order of the experts (of places, where a column has one expert twice)."""
    Ye = np.asarray(Ye, np.float32)
    k, B = chosen.shape
    out = np.zeros((Ye.shape[1], B), np.float32)
    for c in range(B):
        for j in sorted((j for j in range(k) if slots[j, c] >= 0), key=lambda j: (chosen[j, c], slots[j, c])):
            y = Ye[chosen[j, c], :, slots[j, c]]
            out[:, c] += y if weights is None else np.float32(weights[j, c]) * y
    return out


def weight_gradient(Ye, dY, chosen, slots):
    """dweights in 64 bits and the bound of their errors: products of 16 rows in one sum, then the sums of the rows' groups."""
    k, B = chosen.shape
    F = dY.shape[0]
    out, bound = np.zeros((k, B)), np.zeros((k, B))
    for j, c in zip(*np.nonzero(slots >= 0)):
        y, d = np.asarray(Ye[chosen[j, c], :, slots[j, c]], np.float64), np.asarray(dY[:, c], np.float64)
        out[j, c] = y @ d
        bound[j, c] = (np.abs(y) @ np.abs(d)) * (18 + (F + 15) // 16) * U
    return out, bound

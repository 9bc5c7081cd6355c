"""Group norm, dropout and the losses of labels in 64 bits on the CPU: plain forms that share no code with the library, and the bounds that its 32-bit
results are held to.

Bounds count roundings of half a step, E = 2^-24 relative, through the formulas.  D is what a sum may lose, in roundings of the mean of its terms'
sizes: 16 terms one after the other in a thread, then 10 levels of pairs and up to 16 waves, rounded up to 48."""
import numpy as np

E = 2.0 ** -24
D = 48


# ---- dropout

def philox(counter, key, rounds=10):
    """Philox4x32 on arrays of 32-bit words (as 64-bit numbers)."""
    low = np.uint64(0xFFFFFFFF)
    c = [np.asarray(x, dtype=np.uint64) & low for x in counter]
    k = [int(x) for x in key]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def factors(features, batch, drop, layer, seed, step):
    """0 or 1 / (1 - drop) for every entry"""
    cut = min(65535, int(drop * 65536 + 0.5))
    if cut == 0:
        return np.ones((features, batch))
    i, c = np.arange(features)[:, None], np.arange(batch)[None, :]
    words = philox([np.broadcast_to(c // 4, (features, batch)), np.broadcast_to(i // 2, (features, batch)), np.full((features, batch), layer % 2 ** 32),
                    np.full((features, batch), step % 2 ** 32)], [seed % 2 ** 32, (seed >> 32) % 2 ** 32])
    word = np.choose(np.broadcast_to(c % 4, (features, batch)), words)
    bits = np.where(i % 2 == 1, word >> np.uint64(16), word & np.uint64(0xFFFF))
    return np.where(bits >= cut, 65536 / (65536 - cut), 0.0)


# ---- group norm

def sigmoid(u):
    return np.where(u > 0, 1 / (1 + np.exp(-np.abs(u))), np.exp(-np.abs(u)) / (1 + np.exp(-np.abs(u))))


def act_of(u, act):
    return [u, np.maximum(u, 0), u * sigmoid(u)][act]


def slope_of(u, act):
    s = sigmoid(u)
    return [np.ones_like(u), (u > 0) * 1.0, s * (1 + u * (1 - s))][act]


class Norm:
    """Forward and backward, and what the 32-bit results may be off by: .Y, .mean, .rstd, .dX, .dgamma, .dbeta and the same with _tol."""

    def __init__(self, X, gamma, beta, groups, eps, act, factor, dY=None, positive=None):
        """positive: where a ReLU lets the gradient through, for arguments that 32 bits may put on either side of 0"""
        F, B = X.shape
        m = F // groups
        gamma = np.ones(F) if gamma is None else gamma
        beta = np.zeros(F) if beta is None else beta
        x, ga, be = (t.astype(np.float64).reshape(groups, m, -1) for t in (X, gamma, beta))
        keep = factor.reshape(groups, m, B)
        mean = x.mean(1, keepdims=True)
        var = ((x - mean) ** 2).mean(1, keepdims=True)
        rstd = 1 / np.sqrt(var + eps)
        xh = (x - mean) * rstd
        u = ga * xh + be
        # the mean is off by D roundings of the mean size; the squares about it by as many and by the square of that
        off = D * E * np.abs(x).mean(1, keepdims=True)
        var_off = (D + 4) * E * var + off ** 2
        rel = 0.5 * var_off / (var + eps) + 4 * E
        xh_off = rstd * (off + 2 * E * np.abs(x - mean)) + np.abs(xh) * rel
        u_off = np.abs(ga) * xh_off + 2 * E * (np.abs(ga * xh) + np.abs(be))
        # Slopes of the activations stay below 1.1, of their slopes below 0.51.  An exponential is off by (2 |u| + 2) E, a sigmoid s = 1 / (1 + e) by
        # that times e / (1 + e) and 3 E for the sum and the reciprocal: below 1.2 E for u >= 0 (where (2 u + 2) e / (1 + e) has its largest value), 2 |u| E
        # more for u < 0.  The slope s (1 + u (1 - s)) = s + u s (1 - s) has s' u as its second term, which loses as much again.
        exp_off = (12 + 4 * np.maximum(-u, 0) * (act == 2)) * E
        y = keep * act_of(u, act)
        self.u = u.reshape(F, B)
        self.Y, self.Y_tol = y.reshape(F, B), (keep * 1.1 * u_off + exp_off * np.abs(y) + 1e-37).reshape(F, B)
        self.mean, self.mean_tol = mean[:, 0], (off + E * np.abs(mean))[:, 0] + 1e-37
        self.rstd, self.rstd_tol = rstd[:, 0], (rstd * rel)[:, 0] + 1e-37
        if dY is None:
            return
        e0 = keep * dY.astype(np.float64).reshape(groups, m, B)
        e = e0 * (slope_of(u, act) if positive is None else positive.reshape(groups, m, B))
        h = ga * e
        e_off = np.abs(e0) * ((0.51 if act == 2 else 0) * u_off + exp_off)
        h_off = np.abs(ga) * e_off + E * np.abs(h)

        def avg(t):
            return t.mean(1, keepdims=True)
        hx = h * xh
        s, sx = avg(h), avg(hx)
        s_off = avg(h_off) + D * E * avg(np.abs(h))
        hx_off = h_off * np.abs(xh) + np.abs(h) * xh_off + 2 * E * np.abs(hx)
        sx_off = avg(hx_off) + D * E * avg(np.abs(hx))
        inner = h - s - xh * sx
        inner_off = h_off + s_off + np.abs(xh) * sx_off + xh_off * np.abs(sx) + 3 * E * (np.abs(h) + np.abs(s) + np.abs(xh * sx))
        self.dX, self.dX_tol = (rstd * inner).reshape(F, B), (rstd * (inner_off + (rel + 2 * E) * np.abs(inner)) + 1e-37).reshape(F, B)
        ex = e * xh
        self.dgamma, self.dbeta = ex.sum(2).ravel(), e.sum(2).ravel()
        self.dgamma_tol = ((e_off * np.abs(xh) + np.abs(e) * xh_off + 2 * E * np.abs(ex)).sum(2) + D * E * np.abs(ex).sum(2)).ravel() + 1e-37
        self.dbeta_tol = (e_off.sum(2) + D * E * np.abs(e).sum(2)).ravel() + 1e-37


# ---- losses of labels

class Labels:
    """l of every column with what it may be off by: an exponential by 2 |z - top| + 2 roundings, of which the mean over p is at most
    2 log(classes) + 2, and their sum by D."""

    def __init__(self, Z, labels):
        Z = Z.astype(np.float64)
        classes, batch = Z.shape
        self.Z, self.labels = Z, labels
        inside = (labels >= 0) & (labels < classes)
        at = np.where(inside, Z[np.where(inside, labels, 0), np.arange(batch)], -np.inf)
        self.counts = inside & (at != -np.inf)
        with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
            top = Z.max(0)
            top = np.where(np.isneginf(top), 0, top)
            # (beside a largest logit of -3e38 the logarithm would be lost)
            log_sum = np.log(np.exp(Z - top).sum(0))
            self.logp = np.where(self.counts, (at - top) - log_sum, 0.0)
            self.p = np.exp((Z - top) - log_sum)
            self.size = np.where(self.p > 0, np.abs(Z - top), 0)
        self.off = np.where(self.counts, (2 * np.log(classes) + 4 + D) * E, 0.0)
        self.logp_tol = self.off + E * np.abs(self.logp) + 1e-37

    def gradient(self, c, c_off):
        """c (onehot - p) and its bound, for slopes that may be off by c_off"""
        classes = self.Z.shape[0]
        one = (np.arange(classes)[:, None] == self.labels[None, :]) * 1.0
        used = c != 0
        with np.errstate(invalid="ignore"):
            g = np.where(used, c * (one - self.p), 0.0)
            tol = np.where(used, c_off * (one + self.p) + np.abs(c) * (self.p * ((2 * self.size + 6) * E + self.off) + 2 * E * (one + self.p)), 0.0)
        return g, tol + 1e-37

    def sums(self, starts):
        s = np.array([self.logp[a:b].sum() for a, b in zip(starts[:-1], starts[1:])])
        off = np.array([self.off[a:b].sum() for a, b in zip(starts[:-1], starts[1:])])
        return s, off


class Policy:
    def __init__(self, Z, labels, old, ref, A, weights, low, high, beta):
        L = Labels(Z, labels)
        old, A = old.astype(np.float64), A.astype(np.float64)
        low, high, beta = (float(np.float32(t)) for t in (low, high, beta))
        w = np.full(len(labels), 1 / len(labels)) if weights is None else weights.astype(np.float64)
        w = np.where(L.counts, w, 0)
        r = np.exp(L.logp - old)
        self.clipped = ((A > 0) & (r > 1 + high)) | ((A < 0) & (r < 1 - low))
        first = -np.minimum(r * A, np.clip(r, 1 - low, 1 + high) * A)
        kl, slope, steep = np.zeros_like(r), np.where(self.clipped, 0, -r * A), np.abs(r * A)
        if ref is not None:
            g = ref.astype(np.float64) - L.logp
            kl = np.exp(g) - g - 1
            slope, steep = slope + beta * (1 - np.exp(g)), steep + beta * np.exp(g)
        used = w != 0

        def total(t):
            return np.where(used, w * t, 0.0).sum()
        self.stats = np.array([total(first + beta * kl), total(first), total(kl), total(self.clipped * 1.0)])
        sized = [total(L.off * steep), total(L.off * np.abs(r * A)), total(L.off * np.abs(1 - np.exp(L.logp * 0 if ref is None else g))), 0.0]
        self.stats_tol = np.abs(sized) * 1.01 + E * np.abs(self.stats) + 1e-12 + 2 * E * np.abs(sized)
        c = np.where(used, w * slope, 0.0)
        self.dZ, self.dZ_tol = L.gradient(c, np.where(used, np.abs(w) * steep * L.off * 1.01 + E * np.abs(c), 0.0))
        self.L = L


class Preference:
    def __init__(self, Z, labels, starts, ref, beta, smoothing):
        L = Labels(Z, labels)
        s, off = L.sums(starts)
        ref = np.zeros(len(s)) if ref is None else ref.astype(np.float64)
        beta, t = float(np.float32(beta)), float(np.float32(smoothing))
        pairs = len(s) // 2
        beyond = s - ref
        x = beta * (beyond[0::2] - beyond[1::2])
        x_off = abs(beta) * (off[0::2] + off[1::2])
        tail = np.log1p(np.exp(-np.abs(x)))
        self.loss = ((1 - t) * (tail + np.maximum(-x, 0)) + t * (tail + np.maximum(x, 0))).mean()
        self.loss_tol = x_off.mean() + E * abs(self.loss) + 1e-37
        self.sums, self.sums_tol = s, off + E * np.abs(s) + 1e-37
        self.margins, self.margins_tol = x, x_off + E * np.abs(x) + 1e-37
        slope = (t * sigmoid(x) - (1 - t) * sigmoid(-x)) * beta / pairs
        slope_off = 0.25 * x_off * abs(beta) / pairs + 2 * E * np.abs(slope)
        c, c_off = np.zeros(len(labels)), np.zeros(len(labels))
        for k in range(2 * pairs):
            at = slice(starts[k], starts[k + 1])
            c[at], c_off[at] = (1, -1)[k % 2] * slope[k // 2], slope_off[k // 2]
        c = np.where(L.counts, c, 0.0)
        self.dZ, self.dZ_tol = L.gradient(c, np.where(L.counts, c_off, 0.0))
        self.L = L

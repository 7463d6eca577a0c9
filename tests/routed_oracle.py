"""Float64 reference, with bounds, of what stands between the layers of a block with routed experts, written from the definitions in
include/runlora.h with numpy alone.

Bounds.  h: half a unit in the last place of the type, relative (bf16 2^-8, f16 2^-11, f32 2^-24): the rounding of an output.  u = 2^-24: one fp32
operation.  FLOOR: half the smallest step of the type, where a result is below its normal range."""
import numpy as np

HALF_ULP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
FLOOR = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -150}
U = 2.0 ** -24


def norm_forward(h, gain, eps, dtype):
    """y, its bound, and 1 / sqrt(mean h^2 + eps) [n, 1] for h [n, d] as stored.  A sum of squares adds at most 64 of a thread's and, by a tree, 16
    threads' of 64 lanes (10 steps; wider rows add up to 16 waves' in a row): under 96 roundings of a sum of positive terms, so 96 u; its root halves that; the
    root's own two units, eps, 1/d and the two products are six more: (48 + 6) u < 64 u."""
    rstd = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    y = h * rstd * gain
    return y, HALF_ULP[dtype] * np.abs(y) * (1 + 64 * U) + 64 * U * np.abs(y) + FLOOR[dtype], rstd


def norm_backward(dy, h, gain, eps, dh, dtype):
    """(dx, dgain) and their bounds.  mean(N xhat) is a sum of d terms in the same order, each off by rstd's 64 u and three products: at most
    (96 + 64 + 4) u of the terms' magnitudes; then the difference, rstd once more and dh: 256 u covers each of them.  dgain: a workgroup's rows in
    turn, ceil(n / 1024), or ceil(n / 256) of wide rows, which is under 96 more for n < 2^15; up to 1024 workgroups' sums, 32 in a row and 5 steps; 16 rows
    side by side, 64 u for rstd and three operations: under ceil(n / 1024) + 256 roundings."""
    rstd = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    xhat, N = h * rstd, dy * gain
    mean = (N * xhat).mean(1, keepdims=True)
    dx = rstd * (N - xhat * mean)
    b = 256 * U * rstd * (np.abs(N) + np.abs(xhat) * np.abs(N * xhat).mean(1, keepdims=True))
    if dh is not None:
        dx = dx + dh
        b = b + 2 * U * np.abs(dx)
    dgain = (dy * xhat).sum(0)
    bg = (-(-len(dy) // 1024) + 256) * U * np.abs(dy * xhat).sum(0)
    h_ = HALF_ULP[dtype]
    return (dx, dgain), (b * (1 + h_) + h_ * np.abs(dx) + FLOOR[dtype], bg * (1 + h_) + h_ * np.abs(dgain) + FLOOR[dtype])


class Routing:
    """expert, weight, place, source, ends of logits [n, E] (float64), and what the backward needs."""

    def __init__(self, l, top, score="softmax", renormalise=True, groups=1, groups_kept=None, group_top=1, scale=1.0, bias=None):
        n, E = l.shape
        self.l, self.top, self.score, self.renormalise, self.scale = l, top, score, renormalise, scale
        kept = groups if groups_kept is None else groups_kept
        with np.errstate(all="ignore"):
            m = l.max(1, keepdims=True)
            m = np.where(np.isneginf(m), 0.0, m)
            if score == "softmax":
                p = np.exp(l - m)
                s = p / np.where(p.sum(1, keepdims=True) == 0, 1.0, p.sum(1, keepdims=True))
            else:
                s = 1.0 / (1.0 + np.exp(-l))
        c = s + bias if bias is not None else s
        out = np.isneginf(l) | (np.isneginf(bias) if bias is not None else False)
        key = np.where(out, -np.inf, c if bias is not None else l)
        c = np.where(out, -np.inf, c)
        if groups > 1 and kept < groups:
            best = -np.sort(-c.reshape(n, groups, -1), axis=2)[:, :, :group_top]
            # one of each group by its logit where nothing is added (scores that round to the same number keep their order)
            if group_top == 1 and bias is None:
                best = np.where(out, -np.inf, l).reshape(n, groups, -1).max(2, keepdims=True)
            rank = np.where(np.isneginf(best), 0.0, best).sum(2)
            rank = np.where(np.isneginf(best[:, :, 0]), -np.inf, rank)
            order = np.argsort(-rank, axis=1, kind="stable")
            allowed = np.zeros((n, groups), dtype=bool)
            np.put_along_axis(allowed, order[:, :kept], True, axis=1)
            key = np.where(np.repeat(allowed, E // groups, axis=1), key, -np.inf)
        expert = np.argsort(-key, axis=1, kind="stable")[:, :top]
        self.chosen = ~np.isneginf(np.take_along_axis(key, expert, 1))
        lj = np.take_along_axis(l, expert, 1)
        with np.errstate(all="ignore"):
            if renormalise:
                a = lj if score == "softmax" else -np.logaddexp(0.0, -lj)  # log s, however small s is
                a = np.where(self.chosen, a, -np.inf)
                top_a = a.max(1, keepdims=True)
                q = np.where(self.chosen, np.exp(a - np.where(np.isneginf(top_a), 0.0, top_a)), 0.0)
                self.q = np.where(self.chosen, q / np.where(q.sum(1, keepdims=True) == 0, 1.0, q.sum(1, keepdims=True)), 0.0)
            else:
                self.q = np.where(self.chosen, np.take_along_axis(s, expert, 1), 0.0)
            self.left = np.where(self.chosen, 1.0 / (1.0 + np.exp(lj)), 0.0)  # 1 - sigmoid
        self.s = s
        self.weight = scale * self.q
        self.expert = np.where(self.chosen, expert, -1)
        flat = np.where(self.chosen, expert, E).ravel()
        order = np.argsort(flat, kind="stable")
        placed = int((flat < E).sum())
        self.place = np.full(n * top, -1, dtype=np.int64)
        self.place[order[:placed]] = np.arange(placed)
        self.place = self.place.reshape(n, top)
        self.source = np.where(np.arange(n * top) < placed, order, -1)
        self.ends = np.bincount(flat, minlength=E + 1)[:E].cumsum()

    def spread(self):
        """Largest difference of a row's finite logits: exp of a difference d that is off by u |d| is off by as much, relatively."""
        f = np.where(np.isfinite(self.l), self.l, np.nan)
        with np.errstate(all="ignore"):
            import warnings
            with warnings.catch_warnings():
                warnings.simplefilter("ignore")
                return float(np.nan_to_num(np.nanmax(np.nanmax(f, 1) - np.nanmin(f, 1)), nan=0.0))

    def weight_bound(self):
        """A weight is a quotient of exponentials: two units each, the argument's u |d| each, a sum of up to 1024 in 16 + 6 steps, three more operations."""
        return (64 + 4 * min(self.spread() + np.abs(np.where(np.isfinite(self.l), self.l, 0.0)).max(), 200.0)) * U * np.abs(self.weight) + 2.0 ** -126

    def backward(self, dw, dtype):
        """dlogits and its bound: every factor as a weight's, the difference of D and the mean by its parts' magnitudes."""
        D = np.where(self.chosen, self.scale * dw, 0.0)
        n, E = self.l.shape
        out, b = np.zeros((n, E)), np.zeros((n, E))
        rel = (128 + 8 * min(self.spread() + np.abs(np.where(np.isfinite(self.l), self.l, 0.0)).max(), 200.0)) * U
        mean, amean = (D * self.q).sum(1, keepdims=True), np.abs(D * self.q).sum(1, keepdims=True)
        at = np.where(self.chosen, self.expert, 0)
        if self.renormalise:
            left = self.left if self.score == "sigmoid" else 1.0
            v, bv = self.q * left * (D - mean), rel * self.q * left * (np.abs(D) + amean)
        elif self.score == "sigmoid":
            v = self.q * self.left * D
            bv = rel * np.abs(v)
        else:
            v, bv = self.q * D, rel * self.q * np.abs(D)
        rows = np.arange(n)[:, None]
        np.add.at(out, (np.broadcast_to(rows, at.shape), at), np.where(self.chosen, v, 0.0))
        np.add.at(b, (np.broadcast_to(rows, at.shape), at), np.where(self.chosen, bv, 0.0))
        if not self.renormalise and self.score == "softmax":
            out -= self.s * mean
            b += rel * self.s * amean
        return out, b * (1 + HALF_ULP[dtype]) + HALF_ULP[dtype] * np.abs(out) + FLOOR[dtype] + 2.0 ** -126


def gather(x, place):
    """rows [n top, d]; zeros where no copy stands."""
    n, top = place.shape
    rows = np.zeros((n * top, x.shape[1]))
    for t in range(n):
        for p in place[t]:
            if p >= 0:
                rows[p] = x[t]
    return rows


def join(rows, place, weight, add, dtype):
    """add + sum over j of weight rows[place], and its bound: a product and a sum a term."""
    n, top = place.shape
    y = np.zeros((n, rows.shape[1])) if add is None else add.copy()
    b = np.abs(y)
    for t in range(n):
        for j in range(top):
            if place[t, j] >= 0:
                v = weight[t, j] * rows[place[t, j]]
                y[t] += v
                b[t] += np.abs(v)
    h = HALF_ULP[dtype]
    return y, (top + 2) * U * b * (1 + h) + h * np.abs(y) + FLOOR[dtype]


def spread(dy, rows, place, weight, dtype):
    """drows and dweight of the combine, and their bounds: a product's rounding (and the output's); a dot product of d columns, each thread's share in
    turn (a 64th of them at most), then ten steps."""
    n, top = place.shape
    drows, dweight, bw = np.zeros_like(rows), np.zeros((n, top)), np.zeros((n, top))
    for t in range(n):
        for j in range(top):
            p = place[t, j]
            if p >= 0:
                drows[p] = weight[t, j] * dy[t]
                dweight[t, j] = dy[t] @ rows[p]
                bw[t, j] = np.abs(dy[t]) @ np.abs(rows[p])
    h = HALF_ULP[dtype]
    return (drows, dweight), (h * np.abs(drows) + 2 * U * np.abs(drows) + FLOOR[dtype], (rows.shape[1] / 64 + 16) * U * bw + 2.0 ** -149)

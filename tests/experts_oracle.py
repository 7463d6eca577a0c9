"""Float64 reference of the layers over 8-bit weights and stacks of expert weights, written from their definitions (include/runlora.h) with
numpy alone, and the inputs that their tests draw."""
import numpy as np


def nearest_e4m3(v):
    """Nearest e4m3 value, ties to even, of float64 values of magnitude <= 448."""
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.round(v / step) * step


def block_exponent(top):
    """Smallest integer e >= -127 with top <= 448 * 2^e (0 for top = 0)."""
    if top == 0.0:
        return 0
    e = -127
    while top > 448.0 * 2.0 ** e:
        e += 1
    return e


def round_blocks(x, rows, cols):
    """x with every block of rows x cols rounded to e4m3 * 2^e; also the exponents."""
    out = np.empty_like(x)
    n, k = x.shape
    exps = np.zeros((-(-n // rows), -(-k // cols)), dtype=np.int64)
    for a in range(0, n, rows):
        for b in range(0, k, cols):
            p = x[a:a + rows, b:b + cols]
            if not np.isfinite(p).all():
                out[a:a + rows, b:b + cols] = np.nan
                continue
            e = block_exponent(np.abs(p).max())
            exps[a // rows, b // cols] = e
            out[a:a + rows, b:b + cols] = nearest_e4m3(p * 2.0 ** -e) * 2.0 ** e
    return out, exps


def e4m3_value(byte):
    byte = byte.astype(np.int64)
    e, m = (byte >> 3) & 15, byte & 7
    v = np.where(e > 0, np.ldexp(1.0 + m / 8.0, e - 7), np.ldexp(m / 8.0, -6))
    v = np.where((byte & 127) == 127, np.nan, v)
    return np.where(byte & 128, -v, v)


def weight_value(data, scales):
    """[i, o] values of e4m3 bytes and scale bytes."""
    i, o = data.shape
    s = np.ldexp(1.0, scales.astype(np.int64) - 127)
    s = np.where(scales == 255, np.nan, s)
    return e4m3_value(data) * s[np.arange(i) // 128][:, np.arange(o) // 128]


# Per-element bounds beside the values.  h: half a unit in the last place of the storage type, relative (2^-8 bf16, 2^-11 f16).
#   - the rounding of an output: h |want|;
#   - a rank-r factor rounded to the storage type in front of the product it enters (T, Z): h |factor| per term, independent from term to
#     term: at most the sum of the terms' magnitudes times h, and for many terms six standard deviations, 6 h / sqrt(3) times the root of
#     the sum of their squares;
#   - fp32 sums over the contraction: 2^-20 of the sum of the terms' magnitudes; where the operands are e4m3 the matrix instruction adds
#     128 terms to less than fp32 accuracy (found on operands spread over all of e4m3's range: 2^-13.3 of that sum): 2^-12.
HALF_ULP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _rounded_factor(F, G, h):
    """Bound for F G when F's elements are off by up to h relative, independently."""
    return np.minimum(h * (np.abs(F) @ np.abs(G)), 6 * h / np.sqrt(3.0) * np.sqrt((F * F) @ (G * G)))


def _sums(quantised):
    return 2.0 ** -12 if quantised else 2.0 ** -20


def forward(X, ends, W, A, B, bias, s, quantised, dtype="bf16"):
    """(Y, T), and their bounds, for X [n, i], W [E, i, o], A [E, i, r] or None, ...; rows behind the last expert's give zeros."""
    n, o, h = X.shape[0], W.shape[2], HALF_ULP[dtype]
    Y, bY = np.zeros((n, o)), np.zeros((n, o))
    T, bT = (np.zeros((n, 0 if A is None else A.shape[2])) for _ in range(2))
    Xq = round_blocks(X, 1, 128)[0] if quantised else X
    lo = 0
    for e, hi in enumerate(ends):
        Y[lo:hi] = Xq[lo:hi] @ W[e]
        bY[lo:hi] = _sums(quantised) * (np.abs(Xq[lo:hi]) @ np.abs(W[e]))
        if A is not None:
            T[lo:hi] = s * (X[lo:hi] @ A[e])
            bT[lo:hi] = h * np.abs(T[lo:hi]) + 2.0 ** -20 * s * (np.abs(X[lo:hi]) @ np.abs(A[e]))
            Y[lo:hi] += T[lo:hi] @ B[e]
            bY[lo:hi] += _rounded_factor(T[lo:hi], B[e], h) + 2.0 ** -20 * s * (np.abs(X[lo:hi]) @ np.abs(A[e])) @ np.abs(B[e])
        if bias is not None:
            Y[lo:hi] += bias[e]
        bY[lo:hi] += h * np.abs(Y[lo:hi])
        lo = max(lo, hi)
    return (Y, T), (bY, bT)


def backward(dY, X, ends, W, A, B, s, quantised, dtype="bf16"):
    """(dX, dA, dB), and their bounds."""
    h = HALF_ULP[dtype]
    dX, bX = np.zeros((dY.shape[0], W.shape[1])), np.zeros((dY.shape[0], W.shape[1]))
    dA = dB = bA = bB = None
    if A is not None:
        dA, dB, bA, bB = np.zeros(A.shape), np.zeros(B.shape), np.zeros(A.shape), np.zeros(B.shape)
    dYq = round_blocks(dY, 1, 128)[0] if quantised else dY
    lo = 0
    for e, hi in enumerate(ends):
        x, g = X[lo:hi], dY[lo:hi]
        dX[lo:hi] = dYq[lo:hi] @ W[e].T
        bX[lo:hi] = _sums(quantised) * (np.abs(dYq[lo:hi]) @ np.abs(W[e]).T)
        if A is not None:
            Z, T = s * (g @ B[e].T), s * (x @ A[e])
            aZ, aT = 2.0 ** -20 * s * (np.abs(g) @ np.abs(B[e]).T), 2.0 ** -20 * s * (np.abs(x) @ np.abs(A[e]))
            dX[lo:hi] += Z @ A[e].T
            bX[lo:hi] += _rounded_factor(Z, A[e].T, h) + aZ @ np.abs(A[e]).T
            dA[e] = x.T @ Z
            bA[e] = h * np.abs(dA[e]) + _rounded_factor(Z.T, x, h).T + np.abs(x).T @ (aZ + 2.0 ** -20 * np.abs(Z))
            dB[e] = T.T @ g
            bB[e] = h * np.abs(dB[e]) + _rounded_factor(T.T, g, h) + (aT + 2.0 ** -20 * np.abs(T)).T @ np.abs(g)
        bX[lo:hi] += h * np.abs(dX[lo:hi])
        lo = max(lo, hi)
    return (dX, dA, dB), (bX, bA, bB)


def counts(kind, n, experts, rng):
    """Rows per expert."""
    c = np.zeros(experts, dtype=np.int64)
    if kind == "one":          # all rows to the last but one expert
        c[max(0, experts - 2)] = n
    elif kind == "even":
        c[:] = n // experts
        c[: n - int(c.sum())] += 1
    elif kind == "rest":       # uneven, and a third of the rows behind the last expert's
        p = rng.dirichlet(np.ones(experts))
        c[:] = rng.multinomial(n - n // 3, p)
    elif kind == "none":       # no rows for any expert
        pass
    else:                      # uneven, some experts empty
        p = rng.dirichlet(np.full(experts, 0.5))
        p[::3] = 0.0
        p = p / p.sum() if p.sum() > 0 else np.full(experts, 1.0 / experts)
        c[:] = rng.multinomial(n, p)
    return c

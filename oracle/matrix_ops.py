"""Oracle of the 8-bit products and of the matrix update, in 64 bits (NumPy).  Written from the definitions; shares no code with the library.

The 8-bit format: codes of e4m3 (bias 7, no infinities, 0x7f NaN) and one power of two for every 128 of the contraction."""
import numpy as np

DEFAULT_COEFF = (3.4445, -4.7750, 2.0315)


def e4m3_value(code):
    """Value of each code 0 .. 255."""
    code = np.asarray(code, dtype=np.int64)
    sign, e, m = code >> 7, (code >> 3) & 15, code & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((code & 0x7f) == 0x7f, np.nan, v)
    return np.where(sign == 1, -v, v)


def e4m3_code(y):
    """Nearest code, ties to the even one; |y| <= 448 or NaN."""
    y = np.asarray(y, dtype=np.float64)
    a = np.abs(y)
    grid = e4m3_value(np.arange(127))                     # 0 .. 448, ascending
    hi = np.clip(np.searchsorted(grid, np.nan_to_num(a)), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - grid[lo], grid[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(a == grid[hi], hi, code)
    code = code | np.where(np.signbit(y), 128, 0)
    return np.where(np.isnan(y), 0x7f, code).astype(np.uint8)


def scale_exponent(amax):
    """The smallest e >= -127 with amax <= 448 * 2^e; 0 for amax == 0."""
    amax = np.asarray(amax, dtype=np.float64)
    e = np.full(amax.shape, -127, dtype=np.int64)
    for k in range(-127, 122):
        e = np.where(amax > 448.0 * 2.0 ** k, k + 1, e)
    return np.where(amax == 0, 0, e)


def quantize(x, tile=False):
    """(codes [R, whole blocks], scale bytes [R, blocks]) of x [R, C] along its columns; what is not finite becomes NaN and does not count."""
    x = np.asarray(x, dtype=np.float64)
    R, C = x.shape
    kb, rb = -(-C // 128), -(-R // 128)
    pad = np.zeros((rb * 128, kb * 128))
    pad[:R, :C] = x
    size = np.where(np.isfinite(pad), np.abs(pad), 0.0)
    amax = size.reshape(rb * 128, kb, 128).max(2)
    if tile:
        amax = np.repeat(amax.reshape(rb, 128, kb).max(1), 128, axis=0)
    e = scale_exponent(amax)
    y = np.where(np.isfinite(pad), pad, np.nan) / 2.0 ** np.repeat(e, 128, axis=1)
    return e4m3_code(y)[:R], (e + 127).astype(np.uint8)[:R]


def dequantize(q, s, n):
    """Values [R, n] that codes and scale bytes stand for."""
    blocks = np.arange(n) // 128
    return e4m3_value(q[:, :n]) * 2.0 ** (s.astype(np.float64)[:, blocks] - 127.0)


def gemm_fp8(a, as_, b, bs, K, bias=None, old=None, beta=0.0):
    """(C, sum of the products' sizes): the second bounds what roundings can do to the first."""
    x, y = dequantize(a, as_, K), dequantize(b, bs, K)
    c = x @ y.T
    size = np.abs(x) @ np.abs(y).T
    if bias is not None:
        c, size = c + bias, size + np.abs(bias)
    if old is not None and beta != 0.0:
        c, size = c + beta * old, size + np.abs(beta * old)
    return c, size


def _keep(x, bits):
    """x rounded to `bits` significant bits (None: as it is)."""
    if bits is None:
        return x
    f, e = np.frexp(x)
    return np.ldexp(np.round(np.ldexp(f, bits)), e - bits)


def _sum32(pairs):
    """Sum of the products of the pairs in 32 bits, 16 of a contraction at a time."""
    c = 0.0
    for p, q in pairs:
        for k in range(0, p.shape[1], 16):
            c = (c + p[:, k:k + 16] @ q[k:k + 16]).astype(np.float32).astype(np.float64)
    return c


def orthogonalize(x, steps=5, coeff=None, eps=1e-7, numbers=None, runs=None):
    """O(x).  numbers: None for 64-bit arithmetic throughout; 1 or 2 for products of operands rounded to that many numbers of 11 bits each (two: hi hi + hi lo +
    lo hi), summed in 32 bits, where X is always kept as two such numbers and everything between the products is 32 bits: how the roundings of products
    in fewer bits are derived.  runs: with numbers, the steps are taken in runs of these lengths, each on A alone (S_i from A_i, A_(i+1) = S_i A_i S_i, the product Q
    of the run's S_i applied to X at its end), every one of these matrices rounded off its diagonal."""
    f32 = (lambda p: p) if numbers is None else (lambda p: np.asarray(p, dtype=np.float32).astype(np.float64))

    def parts(p):
        hi = _keep(p, 11)
        return hi, _keep(p - hi, 11)

    def times(p, q):
        if numbers is None:
            return p @ q
        (ph, pl), (qh, ql) = parts(p), parts(q)
        return _sum32([(ph, qh)] + ([(ph, ql), (pl, qh)] if numbers == 2 else []))

    x = np.asarray(x, dtype=np.float64)
    coeff = [DEFAULT_COEFF] * steps if coeff is None else coeff
    norm = np.sqrt(np.sum(x * x))
    X = f32(x / (norm + eps)) if norm != 0 else np.zeros_like(x)
    tall = X.shape[0] > X.shape[1]
    X = X.T if tall else X
    if numbers is not None and runs is not None:
        def kept(p):
            d = np.diag(np.diag(p))
            return f32(d) + sum(parts(p - d)[:numbers])

        def both(p, q):
            """Product of two kept matrices: the parts off the diagonal by times(), the rest in 32 bits."""
            dp, dq = np.diag(p), np.diag(q)
            e, f = p - np.diag(dp), q - np.diag(dq)
            return f32(f32(times(e, f) + f32(dp[:, None] * f)) + f32(e * dq[None, :])) + np.diag(f32(dp * dq))

        k = 0
        for n in runs:
            X = f32(sum(parts(X)))
            A, Q = kept(times(X, X.T)), None
            for j in range(n):
                a, b, c = coeff[k + j]
                S = kept(f32(f32(a * np.eye(len(A)) + b * A) + f32(c * both(A, A))))
                if j + 1 < n:
                    A = kept(both(kept(both(S, A)), S))
                Q = S if Q is None else kept(both(S, Q))
            d = np.diag(Q)
            X = f32(f32(d[:, None] * X) + times(Q - np.diag(d), X))
            k += n
        return X.T if tall else X
    for a, b, c in coeff:
        if numbers is None:
            A = X @ X.T
            X = a * X + (b * A + c * (A @ A)) @ X
        else:
            X = f32(sum(parts(X)))
            A = f32(sum(parts(times(X, X.T))[:numbers]))
            S = f32(f32(b * A) + f32(c * times(A, A)))
            d = np.diag(S).copy()
            X = f32(f32(f32(a + d)[:, None] * X) + times(S - np.diag(d), X))
    return X.T if tall else X


def muon_step(w, m, G, lr, momentum, nesterov=True, weight_decay=0.0, rms=0.2, denom=0.0, **ortho):
    """(w, m, O) of one matrix after the update."""
    g = G / denom if denom > 0 else G
    m = momentum * m + g
    u = g + momentum * m if nesterov else m
    rows, cols = w.shape
    s = rms * np.sqrt(max(rows, cols)) if rms > 0 else np.sqrt(max(1.0, rows / cols))
    O = orthogonalize(u, **ortho)
    return (1.0 - lr * weight_decay) * w - lr * s * O, m, O

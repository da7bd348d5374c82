"""The definitions of a mixture of experts in plain NumPy: sorting, rows to experts and back, blocks of 8-bit floating point numbers.

Matrices of floats are float64; 8-bit numbers are uint8 bytes with the number of their exponent's bits (4: e4m3, 5: e5m2).
"""
import numpy as np

BLOCK = 128
MOST = {4: 448.0, 5: 57344.0}


def sort(experts, E):
    """(offsets [E + 1], slots [T, k]): a stable sort of the pairs by expert; pairs without one come last, as -2 - place."""
    flat = np.asarray(experts, np.int64).reshape(-1)
    key = np.where((flat >= 0) & (flat < E), flat, E)
    place = np.empty(len(flat), np.int64)
    place[np.argsort(key, kind="stable")] = np.arange(len(flat))
    offsets = np.concatenate([[0], np.cumsum(np.bincount(key, minlength=E + 1)[:E])])
    return offsets, np.where(key < E, place, -2 - place).reshape(np.shape(experts))


def rows_to(x, slots, out):
    out = out.copy()
    for t in range(slots.shape[0]):
        for s in slots[t]:
            if 0 <= s < len(out):
                out[s] = x[t]
    return out


def rows_from(y, slots, weights=None, residual=None):
    out = np.zeros((slots.shape[0], y.shape[1])) if residual is None else residual.astype(np.float64)
    for t in range(slots.shape[0]):
        for j, s in enumerate(slots[t]):
            if 0 <= s < len(y):
                out[t] += y[s] if weights is None else weights[t, j] * y[s]
    return out


def rows_from_grad(grad, y, slots, weights, grad_y):
    grad_y, grad_w = grad_y.astype(np.float64), np.zeros(slots.shape)
    for t in range(slots.shape[0]):
        for j, s in enumerate(slots[t]):
            if 0 <= s < len(grad_y):
                grad_y[s] = grad[t] if weights is None else weights[t, j] * grad[t]
                grad_w[t, j] = 0.0 if y is None else grad[t] @ y[s]
            elif 0 <= -2 - s < len(grad_y):
                grad_y[-2 - s] = 0.0
    return grad_y, grad_w


def f8_table(exponent):
    """The numbers that the 256 bytes stand for."""
    mantissa, bias = 7 - exponent, 2 ** (exponent - 1) - 1
    out = np.empty(256)
    for b in range(256):
        e, m = b >> mantissa & (2 ** exponent - 1), b & (2 ** mantissa - 1)
        v = m * 2.0 ** (1 - bias - mantissa) if e == 0 else (1 + m / 2 ** mantissa) * 2.0 ** (e - bias)
        if exponent == 4 and b & 127 == 127:
            v = np.nan
        if exponent == 5 and e == 31:
            v = np.nan if m else np.inf
        out[b] = -v if b & 128 else v
    return out


def f8_round(v, exponent):
    """Bytes of the nearest numbers, ties to the even mantissa; beyond the largest, the largest.  v: float32 quotients as float64."""
    table = f8_table(exponent)
    up = table[:128]
    last = int(np.flatnonzero(np.isfinite(up))[-1])
    up = up[:last + 1]
    a = np.abs(np.nan_to_num(v, nan=0.0, posinf=MOST[exponent], neginf=-MOST[exponent])).clip(max=MOST[exponent])
    hi = np.searchsorted(up, a).clip(max=last)
    lo = (hi - 1).clip(min=0)
    mid = (up[lo] + up[hi]) / 2
    code = np.where((a > mid) | ((a == mid) & (hi % 2 == 0)), hi, lo)
    code = np.where(a == up[hi], hi, code)
    code = np.where(np.isnan(v), 127, code | np.where(np.signbit(v), 128, 0))
    return code.astype(np.uint8)


def _scales(top, exponent):
    with np.errstate(all="ignore"):
        return (top.astype(np.float32) / np.float32(MOST[exponent])).astype(np.float32)


def _quotients(x, scale):
    with np.errstate(all="ignore"):
        q = x.astype(np.float32) / scale.astype(np.float32)
    return np.where(scale == 0, 0.0, q).astype(np.float64)


def quantize_blocks(x, exponent):
    """(bytes [M, K], scales float32 [blocks, M]); x: values of a 32-bit or shorter type as float64."""
    M, K = x.shape
    nb = -(-K // BLOCK)
    wide = np.zeros((M, nb * BLOCK))
    wide[:, :K] = x
    scale = _scales(np.abs(wide.reshape(M, nb, BLOCK)).max(2), exponent)
    return f8_round(_quotients(x, np.repeat(scale, BLOCK, 1)[:, :K]), exponent), scale.T


def quantize_tiles(w, exponent):
    """(bytes [N, K], scales float32 [row blocks, blocks])."""
    N, K = w.shape
    rb, nb = -(-N // BLOCK), -(-K // BLOCK)
    wide = np.zeros((rb * BLOCK, nb * BLOCK))
    wide[:N, :K] = w
    scale = _scales(np.abs(wide.reshape(rb, BLOCK, nb, BLOCK)).max((1, 3)), exponent)
    spread = np.repeat(np.repeat(scale, BLOCK, 0), BLOCK, 1)[:N, :K]
    return f8_round(_quotients(w, spread), exponent), scale

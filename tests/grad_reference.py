"""Plain float64 references of the gradient operators (CPU, numpy), each written
from its definition in ``include/lionmuon_grad.h``."""
import numpy as np

BLOCK = 128


def e4m3(v):
    """Nearest e4m3 value, ties to even: three fraction bits from 2^-6 on, steps
    of 2^-9 below; |v| <= 448."""
    a = np.abs(v)
    _, k = np.frexp(np.maximum(a, 2.0 ** -6))       # a = m 2^k, 0.5 <= m < 1
    step = np.ldexp(1.0, k - 1 - 3)
    return np.where(np.isnan(v), np.nan, np.round(v / step) * step)


def block_exponents(x):
    """e of each block of 128 columns: least e >= -100 with max|x| <= 448 2^e."""
    rows, cols = x.shape
    out = np.empty((rows, -(-cols // BLOCK)), dtype=np.int64)
    for b in range(out.shape[1]):
        part = np.abs(x[:, b * BLOCK:(b + 1) * BLOCK])
        top = np.where(np.isfinite(part), part, 0.0).max(axis=1)
        e = np.full(rows, -100)
        for _ in range(400):
            e = np.where(top > 448.0 * np.ldexp(1.0, e), e + 1, e)
        out[:, b] = e
    return out


def checkpoint(x):
    """(values, exponents) of the checkpoint of x; NaN for NaN and infinities."""
    x = np.asarray(x, dtype=np.float64)
    e = block_exponents(x)
    s = np.ldexp(1.0, np.repeat(e, BLOCK, axis=1)[:, :x.shape[1]])
    return e4m3(np.where(np.isfinite(x), x, np.nan) / s) * s, e


def sigmoid(x):
    return np.where(x >= 0, 1.0 / (1.0 + np.exp(-np.abs(x))),
                    np.exp(-np.abs(x)) / (1.0 + np.exp(-np.abs(x))))


GELU_C, GELU_A = np.sqrt(2.0 / np.pi), 0.044715


def activation(a, kind):
    if kind == "swiglu":
        g, u = np.split(a, 2, axis=1)
        return g * sigmoid(g) * u
    # 0.5 (1 + tanh z) = sigmoid(2 z), which keeps its digits for negative z
    return a * sigmoid(2.0 * GELU_C * (a + GELU_A * a ** 3))


def activation_grad(dh, a, kind):
    if kind == "swiglu":
        g, u = np.split(a, 2, axis=1)
        s = sigmoid(g)
        return np.concatenate([dh * u * (s + g * s * (1 - s)), dh * g * s], axis=1)
    z = 2.0 * GELU_C * (a + GELU_A * a ** 3)
    p = sigmoid(z)
    return dh * (p + a * p * sigmoid(-z) * 2.0 * GELU_C * (1 + 3 * GELU_A * a * a))


def rmsnorm(s, w, eps):
    rstd = 1.0 / np.sqrt((s * s).mean(axis=1) + eps)
    return s * rstd[:, None] * w, rstd


def rmsnorm_grad(dy, s, w, rstd, dres=None):
    xhat = s * rstd[:, None]
    t = dy * w
    dx = rstd[:, None] * (t - xhat * (t * xhat).mean(axis=1, keepdims=True))
    return dx if dres is None else dx + dres, (dy * xhat).sum(axis=0)


def grouped(x, w, at):
    """(Y, sum of |products|) of Y = X W_e^T; rows of no expert are 0."""
    y = np.zeros((x.shape[0], w.shape[1]))
    mag = np.zeros_like(y)
    for e in range(w.shape[0]):
        r = slice(at[e], at[e + 1])
        y[r] = x[r] @ w[e].T
        mag[r] = np.abs(x[r]) @ np.abs(w[e]).T
    return y, mag


def grouped_weight(dy, x, at):
    n = len(at) - 1
    dw = np.zeros((n, dy.shape[1], x.shape[1]))
    mag = np.zeros_like(dw)
    for e in range(n):
        r = slice(at[e], at[e + 1])
        dw[e] = dy[r].T @ x[r]
        mag[e] = np.abs(dy[r]).T @ np.abs(x[r])
    return dw, mag

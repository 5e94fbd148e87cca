"""The tail of the forward f_theta (Alg. 1) around the paper's step: the norms
around a block, linear layers with 4-bit weights, and the rules a server puts
on logits, as the plain definitions in float64.  TEST INFRASTRUCTURE ONLY, like
the rest of ``oracle/``.

* ``residual_norm``  u = rms(y) w_post, h' = h + a g u, n = rms(h') w_pre, with
  rms(x) = x / sqrt(mean(x^2) + eps) over the last axis.
* ``mx4_weights``    OCP Microscaling MXFP4 (v1.0, Sec. 5.1 and 5.3.3): E2M1
  elements (1 sign, 2 exponent, 1 mantissa bit, bias 1), one E8M0 scale
  2^(e - 127) per 32.
* ``history``        what the committed prefix of a request holds.
* ``rule_logits``    repetition penalty (divide positive logits of seen tokens
  by r, multiply the others), presence and frequency penalties, biases, and
  a mask; each operation rounded to float32, as the operator is defined.
* ``predict``        x_hat and p of rows that may have nothing left.
"""
import numpy as np

from . import update


def rms(x, eps):
    return x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)


def residual_norm(y, h, gate, w_post, w_pre, eps, a):
    """float64 rows (gate already per row, or None); returns (h', n)."""
    if y is not None:
        u = y if w_post is None else rms(y, eps) * w_post
        h = h + a * (u if gate is None else gate * u)
    n = rms(h, eps)
    return h, n if w_pre is None else n * w_pre


def e2m1(code):
    """The value of a 4-bit code, by the format's definition."""
    s, e, m = code >> 3, (code >> 1) & 3, code & 1
    v = m * 0.5 if e == 0 else (1 + m * 0.5) * 2.0 ** (e - 1)
    return -v if s else v


def mx4_weights(codes, scales):
    """uint8 [N, K/2] (element 2i in the low half of byte i) and uint8
    [N, K/32] -> float64 [N, K]."""
    table = np.array([e2m1(c) for c in range(16)])
    N, half = codes.shape
    w = np.empty((N, 2 * half))
    w[:, 0::2] = table[codes & 15]
    w[:, 1::2] = table[codes >> 4]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return w * np.repeat(s, 32, axis=1)


def history(tokens, prompt_len, o, V):
    """(seen bool [V], count int [V]) of one request's tokens [T]."""
    seen, count = np.zeros(V, dtype=bool), np.zeros(V, dtype=np.int64)
    for pos in range(o):
        v = tokens[pos]
        if 0 <= v < V:
            seen[v] = True
            count[v] += pos >= prompt_len
    return seen, count


def rule_logits(z, seen, count, bias, biased, params, allowed):
    """One row under its rules, every operation rounded to float32.
    z float [V]; bias float [V] (sums, float32); biased bool [V]; params
    (repetition, presence, frequency); allowed bool [V] or None."""
    f = np.float32
    r, p, q = (f(x) for x in params)
    z = np.asarray(z, dtype=f)
    with np.errstate(all="ignore"):
        z1 = np.where(seen, np.where(z > 0, z / r, z * r), z)
        add = (bias.astype(f) - np.where(count > 0, p, f(0))) - q * count.astype(f)
        out = np.where(seen | biased, z1 + add, z)
    if allowed is not None:
        out = np.where(allowed, out, f(-np.inf))
    return out.astype(np.float64)


def predict(z):
    """(x_hat, p) per row; (-1, 0) where a row is -inf throughout.  Finite
    values below -2^26 count as -2^26."""
    z = np.asarray(z, dtype=np.float64)
    z = np.where(np.isneginf(z), z, np.maximum(z, -2.0 ** 26))
    xhat = np.full(len(z), -1, dtype=np.int64)
    p = np.zeros(len(z))
    some = z.max(axis=1) > -np.inf
    if some.any():
        xhat[some], p[some] = update.vocab_reduce(z[some])
    return xhat, p

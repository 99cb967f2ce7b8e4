"""Plain 64-bit forms of the token layers, with bounds on what float32
arithmetic and one rounding to the io dtype may change.

Each function returns (value, size) pairs: `size` is the same sum over absolute
values, which the rounding errors of its terms scale with.
"""
import numpy as np

U32 = 2.0 ** -24
UNIT = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8}


def np64(t):
    return None if t is None else t.detach().cpu().double().numpy()


def counts(lengths, B, T):
    return [T] * B if lengths is None else [min(max(int(n), 0), T) for n in lengths]


def sigmoid(v):
    e = np.exp(-np.abs(v))
    return np.where(v >= 0, 1.0, e) / (1.0 + e)


def activate(v, act):
    return v * sigmoid(v) if act == "silu" else np.maximum(v, 0.0) if act == "relu" else v


def shortconv(x, w, bias, state, lengths, act):
    """x (B, T, C), w (C, K), state (B, K-1, C) or None."""
    B, T, C = x.shape
    K = w.shape[1]
    y, size = np.zeros(x.shape), np.zeros(x.shape)
    new = np.zeros((B, K - 1, C))
    for i, n in enumerate(counts(lengths, B, T)):
        old = np.zeros((K - 1, C)) if state is None else state[i]
        seen = np.concatenate((old, x[i, :n]))
        new[i] = seen[n:]
        for t in range(n):
            terms = w.T * seen[t:t + K]
            b = np.zeros(C) if bias is None else bias
            y[i, t] = activate(terms.sum(0) + b, act)
            size[i, t] = np.abs(terms).sum(0) + np.abs(b)
    return y, size, new


def scan(x, dt, b, c, A, D, dt_bias, softplus, state, lengths):
    """x (B, T, H, P), dt (B, T, H), b and c (B, T, G, N), state (B, H, P, N) or None."""
    B, T, H, P = x.shape
    G, N = b.shape[2:]
    y, size = np.zeros(x.shape), np.zeros(x.shape)
    S = np.zeros((B, H, P, N)) if state is None else state.copy()
    M = np.abs(S)
    for i, n in enumerate(counts(lengths, B, T)):
        for t in range(n):
            d = dt[i, t] + (0 if dt_bias is None else dt_bias)
            d = np.logaddexp(0.0, d) if softplus else d
            a = np.exp(d * A)[:, None, None]
            bt, ct = np.repeat(b[i, t], H // G, 0), np.repeat(c[i, t], H // G, 0)
            u = (d[:, None] * x[i, t])[:, :, None] * bt[:, None, :]
            S[i], M[i] = a * S[i] + u, a * M[i] + np.abs(u)
            skip = 0 if D is None else D[:, None] * x[i, t]
            y[i, t] = np.einsum("hpn,hn->hp", S[i], ct) + skip
            size[i, t] = np.einsum("hpn,hn->hp", M[i], np.abs(ct)) + np.abs(skip)
    return y, size, S, M


def norm(x, z, r, w, scale, groups, eps, gate, residual):
    """Rows (R, D) -> (y, new residual), either None where the form has none."""
    a = x
    z = None if z is None else z * sigmoid(z)
    s = 1.0 if scale is None else scale
    new = None
    if gate == "before":
        a = a * z
    if residual == "before":
        a = new = r + s * a
    v = a.reshape(a.shape[0], groups, -1)
    y = (v / np.sqrt((v * v).mean(-1, keepdims=True) + eps)).reshape(a.shape)
    y = y * (1.0 if w is None else w)
    if gate == "after":
        y = y * z
    if residual == "after":
        return None, r + s * y
    return y, new


def within(got, ref, bound, what):
    """Every element of the tensor `got` within `bound` of `ref` (NaN and
    infinities in neither)."""
    got = np64(got)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    if not got.size:
        return
    assert np.isfinite(got).all(), f"{what}: not finite"
    err = np.abs(got - ref)
    worst = float((err / np.maximum(bound, 1e-300)).max())
    print(f"{what}: worst element at {worst:.3f} of its bound", flush=True)
    assert worst <= 1.0, f"{what}: an element is off by {worst:.2f} times its bound"


def relative(got, ref):
    """2-norm of the difference over 2-norm of the reference."""
    n = float(np.linalg.norm(ref))
    d = float(np.linalg.norm(np64(got) - ref))
    return d / n if n else d

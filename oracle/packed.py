"""Attention over packed samples with grouped heads, rotary positions with several axes and counter-based dropout, in 64 bits.

Written from the definitions, without the library's code.  `attention_bounds` also returns, element by element, the sums of magnitudes that a kernel's
roundings are measured against."""
import numpy as np


def _softmax_parts(q, k, scale, causal):
    z = scale * (q @ k.T)
    if causal:
        n = len(q)
        z = np.where(np.arange(n)[None, :] <= np.arange(n)[:, None], z, -np.inf)
    m = z.max(axis=1, keepdims=True)
    w = np.exp(z - m)
    total = w.sum(axis=1, keepdims=True)
    return z, (m + np.log(total))[:, 0], w / total      # (from z - m: at scores of 1e16 a sum of two is lost in lse)


def attention_fwd(qkv, starts, heads, kv_heads, d, causal, scale=None):
    """qkv [tokens, (heads + 2 kv_heads) d].  O [tokens, heads d] (zero in rows of no sample), lse [heads, tokens], and sum_t P |V| of O's shape."""
    qkv = np.asarray(qkv, dtype=np.float64)
    scale = 1 / np.sqrt(d) if scale is None else scale
    x = qkv.reshape(len(qkv), heads + 2 * kv_heads, d)
    O, mag, lse = np.zeros((len(qkv), heads, d)), np.zeros((len(qkv), heads, d)), np.zeros((heads, len(qkv)))
    for lo, hi in zip(starts, starts[1:]):
        if lo == hi:
            continue
        for a in range(heads):
            g = a * kv_heads // heads
            q, k, v = x[lo:hi, a], x[lo:hi, heads + g], x[lo:hi, heads + kv_heads + g]
            _, lse[a, lo:hi], P = _softmax_parts(q, k, scale, causal)
            O[lo:hi, a], mag[lo:hi, a] = P @ v, P @ np.abs(v)
    return O.reshape(len(qkv), -1), lse, mag.reshape(len(qkv), -1)


def attention_bwd(qkv, O, dO, lse, starts, heads, kv_heads, d, causal, scale=None):
    """dqkv as a function of qkv, O, dO and lse; the sums of the magnitudes of what is rounded to the operands' type before it is summed (P |dO| for
    dV, |dS| |K|, |dS| |Q| for dQ, dK); and of what dS is a difference of, P (|dO| |V| + |dO| |O|) against |K| or |Q|."""
    qkv, O, dO, lse = (np.asarray(t, dtype=np.float64) for t in (qkv, O, dO, lse))
    scale = 1 / np.sqrt(d) if scale is None else scale
    n = len(qkv)
    x, o, do = qkv.reshape(n, heads + 2 * kv_heads, d), O.reshape(n, heads, d), dO.reshape(n, heads, d)
    grad, weighted, parts = (np.zeros_like(x) for _ in range(3))
    for lo, hi in zip(starts, starts[1:]):
        if lo == hi:
            continue
        for a in range(heads):
            g = a * kv_heads // heads
            ik, iv = heads + g, heads + kv_heads + g
            q, k, v = x[lo:hi, a], x[lo:hi, ik], x[lo:hi, iv]
            z, _, _ = _softmax_parts(q, k, scale, causal)
            P = np.exp(z - lse[a, lo:hi, None])
            D = (do[lo:hi, a] * o[lo:hi, a]).sum(axis=1, keepdims=True)
            dS = P * (do[lo:hi, a] @ v.T - D)
            of = P * (np.abs(do[lo:hi, a]) @ np.abs(v.T) + (np.abs(do[lo:hi, a]) * np.abs(o[lo:hi, a])).sum(axis=1, keepdims=True))
            grad[lo:hi, a] = scale * (dS @ k)
            grad[lo:hi, ik] += scale * (dS.T @ q)
            grad[lo:hi, iv] += P.T @ do[lo:hi, a]
            weighted[lo:hi, a] = scale * (np.abs(dS) @ np.abs(k))
            weighted[lo:hi, ik] += scale * (np.abs(dS.T) @ np.abs(q))
            weighted[lo:hi, iv] += P.T @ np.abs(do[lo:hi, a])
            parts[lo:hi, a] = scale * (of @ np.abs(k))
            parts[lo:hi, ik] += scale * (of.T @ np.abs(q))
            parts[lo:hi, iv] += P.T @ np.abs(do[lo:hi, a])
    return tuple(t.reshape(n, -1) for t in (grad, weighted, parts))


def rotary(x, positions, axis_dims, heads, d, base=10000.0, inverse=False):
    """x [rows, heads d] turned; pairs of neighbouring columns as complex numbers."""
    x = np.asarray(x, dtype=np.float64).reshape(len(positions), heads, d)
    out, at = x.copy(), 0
    for k, w in enumerate(axis_dims):
        angle = np.asarray(positions, dtype=np.float64)[:, k:k + 1] * float(base) ** (-np.arange(0, w, 2) / max(w, 1))
        turn = np.exp((-1j if inverse else 1j) * angle)[:, None, :]
        z = (x[..., at:at + w:2] + 1j * x[..., at + 1:at + w:2]) * turn
        out[..., at:at + w:2], out[..., at + 1:at + w:2] = z.real, z.imag
        at += w
    return out.reshape(len(positions), heads * d)


def philox(counter, seed):
    """The four 32-bit results of Philox4x32-10 (Salmon et al., 2011) for each 64-bit counter, [n, 4] uint32."""
    low = np.uint64(0xFFFFFFFF)
    counter = np.asarray(counter, dtype=np.uint64)
    c = [counter & low, counter >> np.uint64(32), np.zeros_like(counter), np.zeros_like(counter)]
    k0, k1 = seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    return np.stack(c, axis=1).astype(np.uint32)


def dropout_factors(n, p, seed, first=0):
    """What each of n elements is multiplied by: 0, or one over the share that stays."""
    drop = int(np.floor(p * 65536 + 0.5))
    words = philox(np.arange(first // 8, (first + n + 7) // 8, dtype=np.uint64), seed)
    words = np.stack([words & 0xFFFF, words >> 16], axis=2).reshape(-1)[:n]
    return np.where(words >= drop, 65536.0 / (65536 - drop), 0.0)

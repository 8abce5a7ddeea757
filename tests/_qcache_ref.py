"""The 8-bit cache and the logit rules in 64 bits, on the CPU, token by token:
what the GPU tests of the operators compare with. Shares no code with the
library."""
import numpy as np
import torch

TOP = {0: 127.0, 1: 448.0}  # by format: int8, e4m3
MIN_EXP = -60


def round_to_grid(y, fmt):
    """float64 y, |y| <= TOP, to the nearest value of the format (ties to even)."""
    if fmt == 0:
        return np.round(y)
    _, x = np.frexp(y)
    step = np.ldexp(1.0, np.maximum(x - 1, -6) - 3)
    return np.round(y / step) * step


def exponent(absmax, fmt):
    """Least e >= MIN_EXP with absmax <= TOP 2^e (None: not finite)."""
    if not np.isfinite(absmax):
        return None
    e = MIN_EXP
    while absmax > TOP[fmt] * 2.0 ** e:
        e += 1
    return e


def decode(q, fmt):
    """Bytes (uint8 array) as float64."""
    if fmt == 0:
        return q.view(np.int8).astype(np.float64)
    u = q.astype(np.int64)
    m, x = u & 7, (u >> 3) & 15
    v = np.where(x == 0, np.ldexp(m / 8.0, -6), np.ldexp(1.0 + m / 8.0, x - 7))
    return np.where(u & 128, -v, v)


class RefCache:
    """One head's K or V: values in units of each block's scale, and scales."""

    def __init__(self, slots, hd, block, fmt):
        self.q, self.e = np.zeros((slots, hd)), [MIN_EXP] * (slots // block)
        self.block, self.fmt = block, fmt

    def write(self, slot0, pos0, rows):
        """rows at positions pos0 .. of a sequence that starts at slot0 (one call)."""
        B = self.block
        t = max(pos0, 0)
        end = pos0 + len(rows)
        while t < end:
            stop = min(end, (t // B + 1) * B)
            new = rows[t - pos0:stop - pos0]
            b, held = (slot0 + t) // B, t % B
            top = np.abs(new).max() if np.isfinite(new).all() else np.inf
            e = exponent(top, self.fmt)
            old = self.e[b] if held else MIN_EXP
            if e is None or (held and old is None):
                self.e[b] = None
            else:
                e = max(e, old)
                a = slot0 + t - held
                self.q[a:a + held] = round_to_grid(np.ldexp(self.q[a:a + held], old - e), self.fmt)
                self.q[slot0 + t:slot0 + stop] = round_to_grid(np.ldexp(new, -e), self.fmt)
                self.e[b] = e
            t = stop

    def values(self, a, n):
        s = np.array([np.nan if self.e[i // self.block] is None else 2.0 ** self.e[i // self.block]
                      for i in range(a, a + n)])
        return self.q[a:a + n] * s[:, None]


def attention(q, k, v, scale, first, causal):
    """q [n, G, hd] at positions first .. first + n - 1 of one sequence over k, v
    [len, hd] (float64). Returns out, lse, the sums of p |v| and, for every row,
    the largest sum_d |q_d k_jd| over the tokens it sees."""
    n, G, hd = q.shape
    out, lse = np.zeros((n, G, hd)), np.full((n, G), -np.inf)
    pv, qk = np.zeros((n, G, hd)), np.zeros((n, G))
    for i in range(n):
        pos = first + i
        m = 0 if pos < 0 else pos + 1 if causal else len(k)
        if m == 0:
            continue
        with np.errstate(invalid="ignore"):
            z = (q[i] @ k[:m].T) * scale
            top = z.max(1, keepdims=True)
            p = np.exp(z - top)
            l = p.sum(1, keepdims=True)
            out[i] = (p / l) @ v[:m]
            lse[i] = (top + np.log(l))[:, 0]
            pv[i] = (p / l) @ np.abs(v[:m])
            qk[i] = (np.abs(q[i]) @ np.abs(k[:m]).T).max(1)
    return out, lse, pv, qk


def adjust(z, history, prompt, rep, pres, freq, bias, allow):
    """One row of logits (float64): history a list of ids, bias a list of (id,
    value), allow a bool array or None. Also the largest magnitude met."""
    z = z.astype(np.float64).copy()
    V, big = len(z), np.abs(np.where(np.isfinite(z), z, 0.0))
    hist = [h for h in history]
    for v in {h for h in hist if 0 <= h < V}:
        z[v] = z[v] / rep if z[v] > 0 else z[v] * rep
        big[v] = max(big[v], abs(z[v]) if np.isfinite(z[v]) else 0.0)
    for v in {h for h in hist[prompt:] if 0 <= h < V}:
        c = sum(h == v for h in hist[prompt:])
        z[v] -= freq * c + pres
        big[v] = max(big[v], abs(freq) * c + abs(pres), abs(z[v]) if np.isfinite(z[v]) else 0.0)
    for v, x in bias:
        if 0 <= v < V:
            z[v] += x
            big[v] += abs(x)
    if allow is not None:
        z[~allow] = -np.inf
    return z, big


def half_step(dtype):
    return torch.finfo(dtype).eps / 2

"""Independent reference of include/qqq_layer.h in 64 bits (numpy): residual norm and gated activation to int8 codes, the 8-bit paged
cache, attention over it.  Test infrastructure only; written from the definitions, in plain loops where that is clearer.
"""
import numpy as np


def add_rmsnorm(x, gain, residual, eps):
    """-> (sum in the residual's type or None, y in 64 bits)."""
    h, total = x.astype(np.float64), None
    if residual is not None:
        total = (h + residual.astype(np.float64)).astype(residual.dtype)
        h = total.astype(np.float64)
    root = np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    return total, np.divide(h, root, out=np.zeros_like(h), where=root > 0) * gain.astype(np.float64)


def gated_act(gate, up, act):
    g = gate.astype(np.float64)
    if act == "silu":
        a = g * np.exp(-np.logaddexp(0, -g))
    else:
        a = g * np.exp(-np.logaddexp(0, -2 * np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3)))
    return a * up.astype(np.float64)


def finite(x):
    """What the cache takes of an fp16 value."""
    return np.nan_to_num(x, nan=0.0, posinf=65504.0, neginf=-65504.0)


def quantise_page(x):
    """[heads, tokens, dim] fp16 -> (codes uint8, scale fp32): the framework's quantiser, one block a head."""
    amax = np.abs(x).max((1, 2)).astype(np.float32)
    s = amax / np.float32(127)
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(s[:, None, None] > 0, np.rint(x.astype(np.float32) / s[:, None, None]), 0)
    return (q + 128).astype(np.uint8), s


class Cache:
    """A cache in the same layout, on the host."""

    def __init__(self, pages, heads, dim, page, slots):
        self.P = page
        self.k_codes = np.full((pages, heads, page, dim), 128, np.uint8)
        self.v_codes = np.full((pages, heads, dim, page), 128, np.uint8)
        self.k_scale, self.v_scale = np.zeros((pages, heads), np.float32), np.zeros((pages, heads), np.float32)
        self.k_tail, self.v_tail = np.zeros((slots, heads, page, dim), np.float16), np.zeros((slots, heads, dim, page), np.float16)

    def append(self, table, kv_len, cu, slots, k, v):
        """One token after the other."""
        for b in range(len(kv_len)):
            n = cu[b + 1] - cu[b]
            for i in range(n):
                pos, slot = kv_len[b] - n + i, slots[b]
                if pos < 0:
                    continue
                self.k_tail[slot, :, pos % self.P] = finite(k[cu[b] + i])
                self.v_tail[slot, :, :, pos % self.P] = finite(v[cu[b] + i])
                if pos % self.P == self.P - 1:
                    page = table[b, pos // self.P]
                    self.k_codes[page], self.k_scale[page] = quantise_page(self.k_tail[slot])
                    self.v_codes[page], self.v_scale[page] = quantise_page(self.v_tail[slot])

    def tokens(self, table_row, length, slot):
        """All of a sequence's keys and values [length, heads, dim] in 64 bits."""
        heads, dim = self.k_codes.shape[1], self.k_codes.shape[3]
        k, v = np.zeros((length, heads, dim)), np.zeros((length, heads, dim))
        for pos in range(length):
            t = pos % self.P
            if pos < length // self.P * self.P:
                page = table_row[pos // self.P]
                k[pos] = (self.k_codes[page, :, t].astype(np.float64) - 128) * self.k_scale[page].astype(np.float64)[:, None]
                v[pos] = (self.v_codes[page, :, :, t].astype(np.float64) - 128) * self.v_scale[page].astype(np.float64)[:, None]
            else:
                k[pos], v[pos] = self.k_tail[slot, :, t], self.v_tail[slot, :, :, t]
        return k, v


def attention(q, k, v, scale, causal=True, window=0):
    """Queries [n, q_heads, dim] at the end of keys [length, heads, dim] -> (out, lse, what a bound of the error goes by: sum p |v|
    and the largest scale * sum |q| |k| of a row)."""
    n, hq, dim = q.shape
    length, heads = k.shape[0], k.shape[1]
    out, lse, mag, big = np.zeros((n, hq, dim)), np.full((n, hq), -np.inf), np.zeros((n, hq, dim)), np.zeros((n, hq))
    q = q.astype(np.float64)
    for i in range(n):
        pos = length - n + i
        hi = min(length, pos + 1) if causal else length
        lo = max(0, pos - window + 1) if window else 0
        if hi <= lo:
            continue
        for h in range(hq):
            kv = h // (hq // heads)
            s = k[lo:hi, kv] @ q[i, h] * scale
            p = np.exp(s - s.max())
            lse[i, h] = s.max() + np.log(p.sum())
            p /= p.sum()
            out[i, h], mag[i, h] = p @ v[lo:hi, kv], p @ np.abs(v[lo:hi, kv])
            big[i, h] = (np.abs(k[lo:hi, kv]) @ np.abs(q[i, h])).max() * scale
    return out, lse, mag, big

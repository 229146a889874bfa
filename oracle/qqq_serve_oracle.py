"""Independent reference of include/qqq_serve.h (numpy, 64 bits): a step's tables one sequence and one page at a time, the int8 product, log
probabilities.  Test infrastructure only.
"""
import numpy as np


class Sessions:
    """What a program keeps of its sessions, on the host."""

    def __init__(self, sessions, columns, pages, page_tokens):
        self.P = page_tokens
        self.pages = np.zeros((sessions, columns), np.int32)
        self.held = np.zeros(sessions, np.int32)
        self.free = np.arange(pages - 1, -1, -1, dtype=np.int32)
        self.count = pages

    def plan(self, ids, new, max_new, max_len, table, sequence, positions, tokens=None):
        """Fills table, sequence and positions where it should -> (kv_len, cu, lacking)."""
        tokens = len(sequence) if tokens is None else tokens
        kv_len, cu, lacking, count = [], [0], 0, min(max(self.count, 0), len(self.free))
        for b, s in enumerate(range(len(new)) if ids is None else ids):
            exists = 0 <= s < len(self.held)
            h = min(max(int(self.held[s]), 0), max_len) if exists else 0
            n = min(min(max(int(new[b]), 0), max_new), max_len - h, tokens - cu[-1]) if exists else 0
            for j in range(h // self.P, (h + n) // self.P):
                if count > 0:
                    count -= 1
                    self.pages[s, j] = self.free[count]
                else:
                    lacking += 1
                    self.pages[s, j] = -1
            closed = (h + n) // self.P
            if closed:
                table[b, :closed] = self.pages[s, :closed]
            for i in range(n):
                sequence[cu[-1] + i], positions[cu[-1] + i] = b, h + i
            if exists:
                self.held[s] = h + n
            kv_len.append(h + n)
            cu.append(cu[-1] + n)
        self.count = count
        return np.array(kv_len, np.int32), np.array(cu, np.int32), lacking

    def release(self, ids):
        count = min(max(self.count, 0), len(self.free))
        for s in ids:
            if not 0 <= s < len(self.held):
                continue
            for page in self.pages[s, :min(max(int(self.held[s]), 0) // self.P, self.pages.shape[1])]:
                if page >= 0 and count < len(self.free):
                    self.free[count] = page
                    count += 1
            self.held[s] = 0
        self.count = count


def logprobs(x, tokens, top):
    """x [M,V] -> (logprob, entropy, lse, top_tokens, top_logprobs) in 64 bits, row by row."""
    M, V = x.shape
    logprob, entropy, lse = np.zeros(M), np.zeros(M), np.zeros(M)
    top_tokens, top_logprobs = np.full((M, top), -1, np.int32), np.full((M, top), -np.inf)
    for m in range(M):
        r = x[m].astype(np.float64)
        broken, nothing = bool(np.isnan(r).any() or (r == np.inf).any()), bool((r == -np.inf).all())
        if broken:
            lse[m] = entropy[m] = np.nan
        elif nothing:
            lse[m], entropy[m] = -np.inf, 0.0
        else:
            largest = r.max()                    # (taken off first: 64 bits do not hold 3e38 and log V)
            seen = r[r > -np.inf] - largest
            log_z = np.log(np.exp(seen).sum())
            lse[m] = largest + log_z
            entropy[m] = -np.sum(np.exp(seen - log_z) * (seen - log_z))
        relative = np.full(V, -np.inf) if nothing else np.full(V, np.nan) if broken else (r - largest) - log_z
        t = -1 if tokens is None else int(tokens[m])
        logprob[m] = 0.0 if t < 0 else relative[t] if t < V else np.nan
        order = np.lexsort((np.arange(V), -np.where(np.isnan(r), 0.0, r), ~np.isnan(r)))[:top]
        top_tokens[m, :len(order)], top_logprobs[m, :len(order)] = order, relative[order]
    return logprob, entropy, lse, top_tokens, top_logprobs

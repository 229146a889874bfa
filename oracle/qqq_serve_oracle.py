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
                if 0 <= page < len(self.free) and count < len(self.free):
                    self.free[count] = page
                    count += 1
            self.held[s] = 0
        self.count = count

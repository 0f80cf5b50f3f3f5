"""CPU oracle for the page step -- TEST INFRASTRUCTURE ONLY.

Only ``tests/`` may import this module; the GPU product path never does, and the
two share no code. One Python loop over requests and one over tokens, with lists
of pages and a list as the stack, from the definition.

Parity status: pinned by ``tests/test_pages_pins.py`` (hand-worked steps, no page
held twice or lost over random steps, a step taken back restores the pool, planted
mistakes).
"""
from __future__ import annotations

import numpy as np


class Pool:
    def __init__(self, pages, page, requests, width):
        self.P, self.W, self.R = page, width, requests
        self.tables = [[] for _ in range(requests)]
        self.length = [0] * requests
        self.free = list(range(pages))   # the last one is on top
        self.pages = pages

    def _need(self, tokens):
        return (tokens + self.P - 1) // self.P

    def step(self, new, T, keep=None, ld=0):
        """Row starts, tokens taken and, of each row, position, slot, dense row and visible tokens."""
        start, starts, taken = 0, [], []
        rows = [(0, -1, -1, 0)] * T
        given, asked, stack = [], 0, len(self.free)
        for r in range(self.R):
            n = max(int(new[r]), 0)
            k = self.length[r] if keep is None else min(max(int(keep[r]), 0), self.length[r])
            starts.append(min(start, T))
            more = max(0, self._need(k + n) - len(self.tables[r]))
            fits = start + n <= T and self._need(k + n) <= self.W
            asked += more if fits else 0
            served = fits and (more == 0 or asked <= stack)
            self.length[r] = k + n if served else k
            if served:
                for _ in range(more):
                    self.tables[r].append(self.free.pop())
            have = self._need(self.length[r])
            given += self.tables[r][have:]
            del self.tables[r][have:]
            taken.append(n if served else 0)
            for i in range(taken[-1]):
                p = k + i
                rows[start + i] = (p, self.tables[r][p // self.P] * self.P + p % self.P, r * ld + p if p < ld else -1,
                                   p + 1)
            start += n
        self.free += reversed(given)
        starts.append(min(start, T))
        cols = np.array(rows, dtype=np.int64).reshape(T, 4)
        return {"q_start": np.array(starts, np.int32), "taken": np.array(taken, np.int32),
                "positions": cols[:, 0].astype(np.int32), "slots": cols[:, 1].copy(), "dense": cols[:, 2].copy(),
                "row_len": cols[:, 3].astype(np.int32)}

    def table(self):
        t = np.full((self.R, self.W), -1, np.int32)
        for r, pages in enumerate(self.tables):
            t[r, :len(pages)] = pages
        return t

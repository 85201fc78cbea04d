"""Pages for growing sequences, and drafted tokens against the target's probabilities: one sequence after another, in
Python integers and fractions, from the definitions."""
from __future__ import annotations

from fractions import Fraction
import math


ENDS = -2  # in a page table: where the pages of an empty sequence end that was parked


class Pool:
    """A page table, lengths, and the pages that nobody holds."""

    def __init__(self, table, lens, held, free, page, max_len):
        self.table = [list(map(int, row)) for row in table]
        self.lens, self.held, self.free = list(map(int, lens)), list(map(int, held)), list(map(int, free))
        self.page, self.max_len = page, max_len

    def grow(self, new):
        """Lengths, pages and the slots of the new tokens, sequence after sequence."""
        slots, asked, room = [], 0, len(self.free)
        for s, n in enumerate(new):
            len0 = self.lens[s]
            need = 0
            if 0 <= len0 and len0 + n <= self.max_len:
                need = max(-(-(len0 + n) // self.page) - self.held[s], 0)
                granted = need == 0 or asked + need <= room
                asked += need
            else:
                granted = False
            if not granted:
                if len0 == 0 < self.held[s] < len(self.table[s]):
                    self.table[s][self.held[s]] = ENDS
                self.lens[s] = len0 if len0 < 0 else ~len0
                slots += [-1] * n
                continue
            for _ in range(need):
                self.table[s][self.held[s]] = self.free.pop()
                self.held[s] += 1
            self.lens[s] = len0 + n
            slots += [self.table[s][j // self.page] * self.page + j % self.page for j in range(len0, len0 + n)]
        return slots

    def compact(self, budgets):
        """Lengths; and of every sequence, whether its rows are stored: not where it is parked, but for an empty one with pages."""
        taken = []
        for s, n in enumerate(budgets):
            row = self.table[s][:max(-(-n // self.page), 1)]
            taken.append(self.lens[s] >= 0 or (self.lens[s] == -1 and row[0] >= 0 and ENDS not in row))
            if taken[s]:
                self.lens[s] = n
        return taken

    def release(self, lens=None):
        back = []
        for s, now in enumerate(self.lens):
            full = ~now if now < 0 else now
            keep = full
            if lens is not None and lens[s] >= 0:
                keep = self.lens[s] = min(int(lens[s]), full)
            kept = min(self.held[s], -(-keep // self.page))
            for e in range(kept, self.held[s]):
                back.append(self.table[s][e])
                self.table[s][e] = -1
            self.held[s] = kept
        self.free += back[::-1]


def weight(x):
    """A probability as an exact number; what is none counts as 0."""
    x = float(x)
    return Fraction(x) if math.isfinite(x) and x > 0 else Fraction(0)


def next_token(weights, pick):
    """The least j whose sum of weights is over pick times all; -1 where nothing weighs."""
    total = sum(weights)
    if total == 0:
        return -1
    at, last = Fraction(0), -1
    for j, w in enumerate(weights):
        if w:
            last = j
        at += w
        if at > Fraction(float(pick)) * total:
            return j
    return last


def verify(target, draft, tokens, accept, pick):
    """One sequence: target [n][vocab], draft the same or None, tokens and accept [n], pick.  Accepted tokens and the next."""
    n, vocab = len(target), len(target[0])
    for t in range(n - 1):
        x, u = int(tokens[t]), float(accept[t])
        good = 0 <= x < vocab and not math.isnan(u)
        if good:
            p, q = weight(target[t][x]), Fraction(1) if draft is None else weight(draft[t][x])
            good = Fraction(u) * q < p
        if not good:
            if draft is None:
                w = [Fraction(0) if j == x else weight(target[t][j]) for j in range(vocab)]
            else:
                w = [max(weight(target[t][j]) - weight(draft[t][j]), Fraction(0)) for j in range(vocab)]
            if sum(w) == 0:
                w = [weight(v) for v in target[t]]
            return [int(v) for v in tokens[:t]] + [next_token(w, pick)]
    return [int(v) for v in tokens[:n - 1]] + [next_token([weight(v) for v in target[n - 1]], pick)]

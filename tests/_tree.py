"""Plain 64-bit references of the operators of a tree's pass, and the passes that their tests make."""
import math
from dataclasses import dataclass, field

import numpy as np

from tests._operators import bf16, bf16_value

PAGE = 64


@dataclass
class Pass:
    """A pass's rows as the host knows them; `behind` rows belong to no sequence."""
    lens: list
    counts: list
    parents: list                 # of every sequence; None: a chain
    behind: int = 0
    stride: int = 0               # of the table; 0: as wide as needed
    first: list = field(init=False)

    def __post_init__(self):
        self.first = [sum(self.counts[:b]) for b in range(len(self.counts) + 1)]
        self.n = self.first[-1]
        self.rows = self.n + self.behind
        self.stride = self.stride or max(1, max(-(-(l + c) // PAGE) for l, c in zip(self.lens, self.counts)))

    def parent(self, b, j):
        return j - 1 if self.parents is None else self.parents[b][j]

    def line(self, b, j):
        """Row j and its ancestors, the eldest first."""
        got = []
        while j >= 0:
            got.insert(0, j)
            j = self.parent(b, j)
        return got

    def flat_parents(self):
        return np.array(sum((list(p) for p in self.parents), []) + [-7] * self.behind, np.int32)


def random_tree(rng, n, wide=3, roots=False):
    return [-1] + [int(rng.integers(-1 if roots else max(0, j - wide), j)) for j in range(1, n)]


def table_of(p, rng, extra=1):
    """A shuffled pool's table [B][stride] and its number of pages; entries of pages without slots lead nowhere."""
    need = [-(-(l + c) // PAGE) for l, c in zip(p.lens, p.counts)]
    pool = sum(need) + extra
    order, at = rng.permutation(pool), 0
    table = np.full((len(need), p.stride), -1, np.int32)
    for b, k in enumerate(need):
        table[b, :k] = order[at:at + k]
        at += k
    return table, pool


def rotate(x, angle):
    """Adjacent pairs of x [..., D] by angle [..., D/2]."""
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * np.exp(1j * angle)
    return np.stack([z.real, z.imag], -1).reshape(x.shape)


def axes(D, section, interleaved):
    return [d % 3 if interleaved else 0 if d < section[0] else 1 if d < section[0] + section[1] else 2 for d in range(D // 2)]


def attention(q, k, v, scale):
    """One row over the slots it sees: out, lse, sum p |v|, largest sum |q||k| scale."""
    with np.errstate(invalid="ignore", over="ignore"):
        z = k @ q * scale
        m = z.max()
        e = np.exp(z - m)
        p = e / e.sum()
        fine = np.isfinite(v)
        out = p @ np.where(fine, v, 0) + np.where(fine, 0, v).sum(0)     # a value that is not finite counts whole
        return out, m + math.log(e.sum()), p @ np.where(fine, np.abs(v), 0), float((np.abs(k) @ np.abs(q)).max() * scale)


def attention_bounds(out, lse, absum, big, D, slots, v_big):
    """How far out and lse may be off.  A score is a sum of D products, each exact in 32 bits, times the scale in log2
    units: off by (D + 4) 2^-24 of the sum of their magnitudes, `big` at most, and once more in the exponent's
    argument, taken from the maximum: e in all, twice in a quotient of sums.  A hardware exponential is within 2^-22,
    probabilities as two bf16 numbers within 2^-16, sums of `slots` terms within slots 2^-24 of their magnitudes.  What
    leaves the range of 32 bits at its lower end is under 2^-126 of the largest value a slot.  Then out is rounded to
    bf16 (half a step, 2^-8)."""
    e = 2 * (D + 4) * 2.0 ** -24 * big
    rel = 2 * e + 2.0 ** -22 + 2.0 ** -16 + 2 * (slots + 64) * 2.0 ** -24
    fine = np.isfinite(out)
    tol = np.where(fine, 2.0 ** -8 * np.abs(np.where(fine, out, 0)) + 1.01 * rel * absum + slots * 2.0 ** -126 * max(1.0, v_big), 0)
    return tol, e + 2.0 ** -22 + (slots + 64) * 2.0 ** -24 + 2.0 ** -22 * (1 + abs(lse)) if np.isfinite(lse) else 0.0


def commit(p, tokens, greedy, stop=-1, budget=None):
    """Rows of the committed steps of every sequence."""
    got = []
    for b in range(len(p.lens)):
        at, taken = p.first[b], []
        most = p.counts[b] if budget is None else min(p.counts[b], budget[b])
        j = 0
        while j is not None and len(taken) < most:
            taken.append(j)
            if stop != -1 and greedy[at + j] == stop:
                break
            j = next((i for i in range(j + 1, p.counts[b]) if p.parent(b, i) == j and tokens[at + i] == greedy[at + j]), None)
        got.append(taken)
    return got


__all__ = ["PAGE", "Pass", "random_tree", "table_of", "rotate", "axes", "attention", "attention_bounds", "commit", "bf16",
           "bf16_value"]

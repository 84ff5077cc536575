"""A check of attention rows that sees a lost, doubled or misplaced page of a long
prefix, and the shapes that it is put to.

The error of a row, in the 2-norm over its d values, comes from roundings that are
independent of each other: of each P to bfloat16, relative and at most 2^-8 (so a
variance of 2^-16 / 3 at most), which moves the row by p_j (v_j - out), as the kernels
normalise by the sum of the rounded P; and of the result, the same.  What fp32 adds
(2^-24 in sums of d products and of the keys) is a thousandth of that.  The bound is
twice the standard deviation of the norm, four times its mean square: over d >= 64 values, or d
sums over keys, the mean square does not come near it by chance, and where one key
carries a row each rounding is within sqrt(3) standard deviations anyway.  Of n keys of
like weight a page of 16 is sqrt(16 / n) of the row's norm, 2^-8 / sqrt(3) * sqrt(2) *
2 is the bound: at n = 65536 they are 1.6 % and 0.6 %."""
import torch

from tests.kv4_cases import BY_PLAN, RAGGED_256

# (n_q, n_kv, d, prefix tokens, suffix tokens): those of the plan rule's kernels, and long prefixes over one to
# eight KV heads
PREFILLS = [s for shapes in BY_PLAN.values() for s in shapes] + RAGGED_256 + [
    (32, 8, 128, 65536, 512), (64, 8, 128, 32768, 512), (32, 8, 128, 65536, 1), (32, 8, 128, 32763, 2), (4, 1, 128, 65536, 1),
    (8, 1, 128, 131072, 4), (4, 2, 64, 131072, 1), (8, 2, 64, 100_001, 33), (12, 6, 64, 40_000, 300)]

# (n_q, n_kv, d, lengths, room above the longest)
DECODES = [
    (64, 8, 128, [32768, 31111, 30000, 32001, 28672, 32767, 29999, 32700], 0),
    (32, 8, 128, [22288, 11664, 12704, 11440, 4992, 6512, 28560, 8144, 17, 129, 0, 4096, 1000, 2049, -1, 16384, 777, 3333,
                  64, 511, 9000, 15, 16, 1, 20000, 5120, -1, 333, 8191, 12345, 2500, 640], 50),
    (32, 8, 128, [32763], 5), (4, 1, 128, [100_000], 900), (8, 2, 64, [65536], 0), (40, 1, 128, [20003, 9001], 100),
    (8, 8, 64, [5000 + 37 * i for i in range(60)], 10), (4, 2, 64, [3000 + 11 * i for i in range(140)], 0),
    (16, 2, 128, [40_000, 3, 25_000, -1, 39_999], 7000), (2, 1, 128, [8000 + i for i in range(100)], 500),
]


def rows(q, k, v, seen):
    """(out, variance of the row's norm) of one KV head in float64: q [rows][d], k and v [keys][d], on any device; row
    i sees the first seen[i] keys."""
    s = q @ k.T / q.shape[1] ** 0.5
    s = s.masked_fill(torch.arange(k.shape[0], device=k.device)[None] >= seen[:, None], -torch.inf)
    p = torch.softmax(s, 1)
    del s
    out = p @ v
    p *= p
    # sum_e sum_j p_j^2 (v_je - out_e)^2
    square = (p @ (v * v)).sum(1) - 2 * (out * (p @ v)).sum(1) + (out * out).sum(1) * p.sum(1)
    return out, (square.clamp(min=0) + (out * out).sum(1)) * 2.0 ** -16 / 3


def off(got, out, variance):
    """By how many times the bound each row of `got` is off (NaN: it is not finite)."""
    return (got.double() - out).norm(dim=1) / (2 * variance.sqrt() + 1e-30)

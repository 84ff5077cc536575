"""The check of tests/attention_norm.py, put to results with planted mistakes, on the CPU:
for every shape of the GPU tests it takes what the kernels may round to, and refuses a page
of 16 keys that is left out, counted twice or read with another's values."""
import pytest
import torch

from tests import attention_norm as norm


def as_computed(q, k, v, seen, weight):
    """Rows with P and the result rounded to bfloat16; `weight` counts each key (0: left out)."""
    s = q @ k.T / q.shape[1] ** 0.5
    s = s.masked_fill(torch.arange(k.shape[0])[None] >= seen[:, None], -torch.inf)
    p = torch.exp(s - s.amax(1, keepdim=True)).bfloat16().double() * weight
    return (p @ v / p.sum(1, keepdim=True)).bfloat16()


def shapes():
    for nq, nkv, d, tp, ts in norm.PREFILLS:
        yield d, tp, ts
    for nq, nkv, d, lengths, _ in norm.DECODES:
        for n in sorted({max(lengths), sorted(lengths)[len(lengths) // 2]}):
            yield d, n, 1


@pytest.mark.parametrize("d,tp,ts", sorted(set(shapes())))
def test_a_page_is_seen(d, tp, ts):
    g = torch.Generator().manual_seed(tp * 7 + ts)
    normal = lambda *s: torch.randn(*s, generator=g).bfloat16().double()  # noqa: E731
    at = torch.tensor(sorted({0, ts // 2, ts - 1}))
    seen = tp + 1 + at
    n = int(seen[-1])
    q, k, v = normal(len(at), d), normal(n, d), normal(n, d)
    want = norm.rows(q, k, v, seen)
    one = torch.ones(n, dtype=torch.double)
    assert (norm.off(as_computed(q, k, v, seen, one), *want) < 1).all()
    pages = sorted({0, tp // 16 // 2, max(0, tp // 16 - 1)}) if tp >= 16 else []
    for page in pages:
        here = slice(page * 16, page * 16 + 16)
        for times in (0.0, 2.0):
            weight = one.clone()
            weight[here] = times
            assert (norm.off(as_computed(q, k, v, seen, weight), *want) > 1).all(), (page, times)
        other = v.clone()
        other[here] = normal(16, d)
        assert (norm.off(as_computed(q, k, other, seen, one), *want) > 1).all(), page

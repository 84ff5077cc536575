"""Scores of any size that fp32 holds: from some 2^24 on, two scores that differ at all
are whole powers of two apart, so a row is the mean of the values whose keys reach its
largest score.  Keys are signs times a power of two, so that every dot product is exact
and rows may tie; every fourth row keeps ordinary scores beside them."""
import numpy as np
import pytest

from tests import kv4_ref as ref
from tests.attention_cases import BY_PLAN as BY_PLAN16
from tests.gpu_util import require_gpu
from tests.kv4_cases import BY_PLAN as BY_PLAN4

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()
    import torch
    torch.cuda.synchronize()
    yield
    torch.cuda.synchronize()


def dev(a):
    import torch
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16).copy()).cuda().view(torch.bfloat16)
    return torch.from_numpy(a.copy()).cuda()


def host16(t):
    import torch
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


def signs(rng, *shape):
    return rng.integers(0, 2, shape) * 2.0 - 1.0


def inputs(rng, nq, nkv, d, keys, seen):
    """q [rows][nq][d], k and v [keys][nkv][d], and the rows of q that are of ordinary size, as float64; row i sees
    the first seen[i] keys.  All but those rows and v are signs."""
    k, v = signs(rng, keys, nkv, d), rng.standard_normal((keys, nkv, d))
    per = nq // nkv
    q = signs(rng, len(seen), nq, d)
    plain = np.zeros((len(seen), nq, 1), bool)
    for i, n in enumerate(seen):
        for h in range(nq):
            kind = (i * nq + h) % 4
            if kind == 0:                     # one key stands out
                q[i, h] = k[rng.integers(n), h // per]
            elif kind == 1:                   # its own key is the least
                q[i, h] = -k[n - 1, h // per]
            elif kind == 2:
                q[i, h], plain[i, h] = rng.standard_normal(d), True
    return q, k, v, plain


# Keys and all but the ordinary rows times 2^a, those times 2^-a: scores of up to sqrt(d) * 2^(2a).  What they
# have for softmax does not depend on a, from 9 on: scores that differ do by 2^(2a) * 2 / sqrt(d) at least.
EXPONENTS = [9, 12, 14, 16, 17, 20, 40, 59]


def scaled(q, k, plain, a):
    return ref.f64_to_bf16(q * np.where(plain, 2.0 ** -a, 2.0 ** a)), ref.f64_to_bf16(k * 2.0 ** a)


def expected(q, k, v, plain, seen):
    """Of the values v as they are stored."""
    qa, ka = scaled(q, k, plain, 9)
    return ref.attention(ref.bf16_to_f64(qa), ref.bf16_to_f64(ka), v, seen)


# of each tile and head size: the keys in one piece, and split over workgroups
SHAPES4, SHAPES16 = ([(min(plans[key], key=lambda s: s[1] * s[3]), key) for key in plans] for plans in (BY_PLAN4, BY_PLAN16))


def some_rows(ts, grp):
    return sorted({0, 1 % ts, 15 // grp % ts, 31 // grp % ts, 32 // grp % ts, 256 // grp % ts, ts // 2, ts - 1})


class Pool4:
    """Keys of signs and values, encoded once: another a is another scale byte of the keys."""

    def __init__(self, pages, nkv, d):
        self.ref = ref.Pool4(1, pages, nkv, 16, d)

    def put(self, table, k, v):
        """Returns the values that are stored."""
        self.ref.put(0, 0, table, 0, ref.f64_to_bf16(k))
        self.ref.put(0, 1, table, 0, ref.f64_to_bf16(v))
        assert np.array_equal(self.ref.get(0, 0, table, len(k)), k)          # a sign is a code
        return self.ref.get(0, 1, table, len(k))

    def scaled(self, a):
        raw = self.ref.raw.copy()
        scales = raw[0, 0, :, self.ref.code_bytes:]
        scales[scales != 255] += a
        return raw


@pytest.mark.parametrize("shape,key", SHAPES4)
def test_prefill_in_4_bits(shape, key):
    import torch
    import paper_2605_22850_amd as oc
    nq, nkv, d, tp, ts = shape
    need = -(-tp // 16)
    lay = oc.Layout(1, nq, nkv, d, 16, 16, need + 1)
    rng = np.random.default_rng(tp + ts)
    table = rng.permutation(need + 1)[:need].astype(np.int32)
    seen, rows = tp + 1 + np.arange(ts), some_rows(ts, nq // nkv)
    ws = torch.empty(oc.oc_kv4_attention_workspace_bytes(lay, tp, ts), dtype=torch.uint8, device="cuda")
    q, k, v, plain = inputs(rng, nq, nkv, d, tp + ts, seen)
    pool, v_new = Pool4(need + 1, nkv, d), ref.f64_to_bf16(v[tp:])
    stored = pool.put(table, k[:tp], v[:tp])
    want = expected(q[rows], k, np.concatenate((stored, ref.bf16_to_f64(v_new))), plain[rows], seen[rows])
    for a in EXPONENTS:
        qa, ka = scaled(q, k, plain, a)
        out = torch.empty((ts, nq, d), dtype=torch.bfloat16, device="cuda")
        oc.oc_kv4_suffix_prefill_layer(dev(qa), dev(ka[tp:]), dev(v_new), ts, dev(pool.scaled(a)), lay, dev(table), tp, 0,
                                       out, ws)
        ref.assert_rows_close(host16(out)[rows], *want, what=f"{key} 2^{2 * a}")


@pytest.mark.parametrize("nq,nkv,d,lengths", [(4, 2, 64, [250]), (32, 8, 128, [-1, 31, 0, 700, 1]), (40, 1, 128, [77, 300]),
                                              (8, 1, 64, [9000, 3, 0, -1, 2500]), (4, 1, 128, [2048] * 3)])
def test_decode_in_4_bits(nq, nkv, d, lengths):
    import torch
    import paper_2605_22850_amd as oc
    rng = np.random.default_rng(sum(lengths))
    most, B = max(lengths) + 800, len(lengths)
    needs = [max(n, 0) // 16 + 1 for n in lengths]
    P = max(sum(needs), most // 16 + 1)
    lay = oc.Layout(1, nq, nkv, d, 16, 16, P)
    tables, perm = np.zeros((B, most // 16 + 1), np.int32), rng.permutation(P).astype(np.int32)
    for i, n in enumerate(needs):
        tables[i, :n] = perm[sum(needs[:i]):sum(needs[:i + 1])]
    ws = torch.empty(oc.oc_kv4_decode_workspace_bytes(lay, B, most), dtype=torch.uint8, device="cuda")
    pool, v_new = Pool4(P, nkv, d), np.zeros((B, nkv, d), np.uint16)
    q, k, plain, want = np.ones((B, nq, d)), np.ones((B, nkv, d)), np.zeros((B, nq, 1), bool), {}
    for i, n in enumerate(lengths):
        if n < 0:
            continue
        qi, ki, vi, plain[i:i + 1] = inputs(rng, nq, nkv, d, n + 1, [n + 1])
        stored = pool.put(tables[i], ki[:n], vi[:n])
        q[i], k[i], v_new[i] = qi[0], ki[n], ref.f64_to_bf16(vi[n])
        want[i] = expected(qi, ki, np.concatenate((stored, ref.bf16_to_f64(v_new[i:i + 1]))), plain[i:i + 1], [n + 1])
    for a in EXPONENTS:
        qa, ka = scaled(q, k, plain, a)
        out = torch.empty((B, nq, d), dtype=torch.bfloat16, device="cuda")
        oc.oc_kv4_decode_layer(dev(qa), dev(ka), dev(v_new), B, dev(pool.scaled(a)), lay, dev(tables),
                               dev(np.array(lengths, np.int32)), most, 0, out, ws)
        got = host16(out)
        for i, w in want.items():
            ref.assert_rows_close(got[i:i + 1], *w, what=f"request {i} of {lengths[i]} tokens, 2^{2 * a}")


@pytest.mark.parametrize("shape,key", SHAPES16)
def test_prefill(shape, key):
    import torch
    import paper_2605_22850_amd as oc
    nq, nkv, d, tp, ts = shape
    need = -(-tp // 16)
    P = need + 1
    lay = oc.Layout(1, nq, nkv, d, 16, 16, P)
    rng = np.random.default_rng(tp + ts)
    table = rng.permutation(P)[:need].astype(np.int32)
    seen, rows = tp + 1 + np.arange(ts), some_rows(ts, nq // nkv)
    ws = torch.empty(oc.oc_attention_workspace_bytes(lay, tp, ts), dtype=torch.uint8, device="cuda")
    q, k, v, plain = inputs(rng, nq, nkv, d, tp + ts, seen)
    v = ref.f64_to_bf16(v)
    want = expected(q[rows], k, ref.bf16_to_f64(v), plain[rows], seen[rows])
    t = np.arange(tp)
    for a in EXPONENTS:
        qa, ka = scaled(q, k, plain, a)
        raw = np.full((2, P, nkv, 16, d), 0x7FC0, np.uint16)
        for kv, x in ((0, ka), (1, v)):
            raw[kv, table[t // 16], :, t % 16] = x[:tp]
        out = torch.empty((ts, nq, d), dtype=torch.bfloat16, device="cuda")
        oc.oc_suffix_prefill_layer(dev(qa), dev(ka[tp:]), dev(v[tp:]), ts, dev(raw), lay, dev(table), tp, 0, out, ws)
        ref.assert_rows_close(host16(out)[rows], *want, what=f"{key} 2^{2 * a}")

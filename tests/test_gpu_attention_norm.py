"""Attention over a 4-bit prefix, every row of it, against float64 within the 2-norm that
its roundings give (tests/attention_norm.py): a page lost from a prefix of 100,000 tokens
shows.  The prefix is stored and read back by the library, both exact to the bit."""
import pytest
import torch

from tests import attention_norm as norm
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()
    torch.cuda.synchronize()
    yield
    torch.cuda.synchronize()


class Prefixes:
    """Prefixes of several requests in one pool whose other bytes say NaN, and their values in float64."""

    def __init__(self, nq, nkv, d, lengths, room, seed):
        import paper_2605_22850_amd as oc
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        needs = [(max(n, 0) + room) // 16 + 1 for n in lengths]
        P = sum(needs) + 3
        self.lay = oc.Layout(2, nq, nkv, d, 16, 1, P)
        self.pool = torch.full((oc.oc_kv4_pool_bytes(self.lay),), 0xFF, dtype=torch.uint8, device="cuda")
        perm = torch.randperm(P, device="cuda", generator=self.g).to(torch.int32)
        self.tables = torch.full((len(needs), max(needs)), 1 << 30, dtype=torch.int32, device="cuda")
        self.values, at = [], 0
        for i, (n, need) in enumerate(zip(lengths, needs)):
            self.tables[i, :need] = perm[at:at + need]
            at += need
            back = torch.empty((max(n, 0), 2, nkv, d), dtype=torch.bfloat16, device="cuda")
            if n > 0:
                oc.oc_kv4_layer_ingest(self.normal(n, 2, nkv, d), n, self.tables[i], n, self.pool, self.lay, 1)
                oc.oc_kv4_layer_gather(self.tables[i], n, self.pool, self.lay, 1, back, n)
            self.values.append(back)

    def normal(self, *shape):
        return torch.randn(*shape, dtype=torch.bfloat16, device="cuda", generator=self.g)

    def worst(self, i, q, k_new, v_new, got, seen):
        """Of request i's rows q [T][nq][d], by how many times the bound the worst is off."""
        grp, most = q.shape[1] // k_new.shape[1], 0.0
        for h in range(k_new.shape[1]):
            k, v = (torch.cat((self.values[i][:, kv, h], new[:, h])).double() for kv, new in ((0, k_new), (1, v_new)))
            for x in range(h * grp, h * grp + grp):
                for t in range(0, q.shape[0], 1024):
                    here = slice(t, t + 1024)
                    off = norm.off(got[here, x], *norm.rows(q[here, x].double(), k, v, seen[here]))
                    assert bool(torch.isfinite(off).all())
                    most = max(most, float(off.max()))
        return most


@pytest.mark.parametrize("nq,nkv,d,tp,ts", norm.PREFILLS)
def test_prefill(nq, nkv, d, tp, ts):
    import paper_2605_22850_amd as oc
    c = Prefixes(nq, nkv, d, [tp], 0, tp + ts)
    q, k, v = c.normal(ts, nq, d), c.normal(ts, nkv, d), c.normal(ts, nkv, d)
    ws = torch.full((oc.oc_kv4_attention_workspace_bytes(c.lay, tp, ts),), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    oc.oc_kv4_suffix_prefill_layer(q, k, v, ts, c.pool, c.lay, c.tables[0], tp, 1, out, ws)
    assert c.worst(0, q, k, v, out, tp + 1 + torch.arange(ts, device="cuda")) < 1


@pytest.mark.parametrize("nq,nkv,d,lengths,room", norm.DECODES)
def test_decode(nq, nkv, d, lengths, room):
    import paper_2605_22850_amd as oc
    c, B, most = Prefixes(nq, nkv, d, lengths, room, sum(lengths)), len(lengths), max(lengths) + room
    q, k, v = c.normal(B, nq, d), c.normal(B, nkv, d), c.normal(B, nkv, d)
    ws = torch.full((oc.oc_kv4_decode_workspace_bytes(c.lay, B, most),), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    oc.oc_kv4_decode_layer(q, k, v, B, c.pool, c.lay, c.tables, torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                           most, 1, out, ws)
    for i, n in enumerate(lengths):
        if n >= 0:
            one = slice(i, i + 1)
            assert c.worst(i, q[one], k[one], v[one], out[one], torch.tensor([n + 1], device="cuda")) < 1, (i, n)

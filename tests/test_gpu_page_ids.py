"""Tables that name pages outside the pool, as a fork or take without enough pages
leaves them on the device: whatever call they reach, nothing outside the pool is
touched, and the rest of the call does its work."""
import numpy as np
import pytest

from tests import kv4_ref as ref
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu

GUARD = 1 << 16           # bytes before and behind the pool
OUTSIDE = [-1, -(1 << 31), (1 << 31) - 1]


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


def normal(rng, *shape):
    return ref.f64_to_bf16(rng.standard_normal(shape))


class Guarded:
    """A pool's bytes between two guards."""

    def __init__(self, raw):
        rng = np.random.default_rng(1)
        self.before, self.behind = (rng.integers(0, 256, GUARD, dtype=np.uint8) for _ in range(2))
        self.all = dev(np.concatenate((self.before, raw.reshape(-1), self.behind)))
        self.pool = self.all[GUARD:GUARD + raw.size]

    def check(self, raw):
        got = self.all.cpu().numpy()
        assert np.array_equal(got[:GUARD], self.before) and np.array_equal(got[-GUARD:], self.behind)
        assert np.array_equal(got[GUARD:-GUARD].reshape(raw.shape), raw)


def table_with_holes(rng, P, need):
    """A table some of whose entries name no page, and which those are."""
    table = rng.permutation(P)[:need].astype(np.int32)
    bad = rng.permutation(need)[:max(1, need // 3)]
    bad = np.unique(np.append(bad, need - 1))
    table[bad] = [(OUTSIDE + [P])[i % 4] for i in range(len(bad))]
    return table, bad


@pytest.mark.parametrize("nkv,d,ps,G,chunks,ts", [(2, 64, 16, 16, 9, 3), (8, 128, 16, 64, 3, 40), (3, 96, 24, 24, 7, 25),
                                                  (1, 32, 8, 12, 6, 9)])
def test_stores_in_4_bits(nkv, d, ps, G, chunks, ts):
    import torch
    import paper_2605_22850_amd as oc
    rng = np.random.default_rng(nkv + d + ts)
    tp = chunks * G
    need = -(-(tp + ts) // ps)
    P = need + 3
    table, bad = table_with_holes(rng, P, need)
    lay = oc.Layout(3, nkv, nkv, d, ps, G, P)
    want = ref.Pool4(3, P, nkv, ps, d, fill=0x5A)
    pool = Guarded(want.raw)
    k, v = normal(rng, tp + ts, nkv, d), normal(rng, tp + ts, nkv, d)
    there = ~np.isin(np.arange(tp + ts) // ps, bad)
    for layer in (0, 2):
        for t in np.flatnonzero(there):
            want.put(layer, 0, table, t, k[t:t + 1])
            want.put(layer, 1, table, t, v[t:t + 1])
        payload = np.stack((k[:tp].reshape(chunks, G, nkv, d), v[:tp].reshape(chunks, G, nkv, d)), 1)
        oc.oc_kv4_layer_ingest(dev(payload), chunks, dev(table), tp, pool.pool, lay, layer)
        oc.oc_kv4_suffix_append(dev(k[tp:]), dev(v[tp:]), ts, dev(table), tp, pool.pool, lay, layer)
    pool.check(want.raw)
    # read back: the parts of pages that are not there stay as they were
    for layer in (0, 2):
        out = torch.full((chunks, 2, G, nkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
        oc.oc_kv4_layer_gather(dev(table), tp, pool.pool, lay, layer, out, chunks)
        got = out.float().cpu().numpy().astype(np.float64)
        inside = np.where(np.isin(np.arange(len(table)), bad), 0, table)
        for kv in (0, 1):
            values = want.get(layer, kv, inside, tp)
            values[~there[:tp]] = 7.0
            assert np.array_equal(got[:, kv].reshape(tp, nkv, d), values)


@pytest.mark.parametrize("tile,nq,nkv,d,tp,ts", [
    (16, 32, 8, 128, 67, 43), (16, 8, 2, 64, 4661, 170), (32, 32, 8, 128, 458, 143), (32, 32, 4, 64, 420, 211),
    (256, 32, 8, 128, 122, 626), (256, 32, 4, 64, 3655, 547)])
def test_prefill_in_4_bits(tile, nq, nkv, d, tp, ts):
    """Page 0 is read in their place: the same rows as with a table that says so."""
    import torch
    import paper_2605_22850_amd as oc
    from tests.test_kv4_host import plan
    assert plan(nq, nkv, d, tp, ts)[0] == tile
    rng = np.random.default_rng(tp + ts)
    need = -(-tp // 16)
    P = need + 2
    table, bad = table_with_holes(rng, P, need)
    lay = oc.Layout(2, nq, nkv, d, 16, 16, P)
    want = ref.Pool4(2, P, nkv, 16, d, fill=0)
    for kv in (0, 1):
        want.put(1, kv, np.arange(P), 0, normal(rng, P * 16, nkv, d))
    pool = Guarded(want.raw)
    q, k, v = (dev(normal(rng, ts, n, d)) for n in (nq, nkv, nkv))
    ws = torch.empty(oc.oc_kv4_attention_workspace_bytes(lay, tp, ts), dtype=torch.uint8, device="cuda")
    outs = []
    for t in (table, np.where(np.isin(np.arange(need), bad), 0, table).astype(np.int32)):
        outs.append(torch.full((ts, nq, d), 3.0, dtype=torch.bfloat16, device="cuda"))
        oc.oc_kv4_suffix_prefill_layer(q, k, v, ts, pool.pool, lay, dev(t), tp, 1, outs[-1], ws)
    assert torch.equal(*outs) and bool(torch.isfinite(outs[0].float()).all())
    pool.check(want.raw)


def test_append_to_a_child_that_got_no_page():
    """Fork, append and attention queued one after the other: the host never sees that no page was left."""
    import torch
    import paper_2605_22850_amd as oc
    rng = np.random.default_rng(3)
    nq, nkv, d, P, tp = 4, 2, 64, 6, 40
    lay = oc.Layout(2, nq, nkv, d, 16, 16, P)
    want = ref.Pool4(2, P, nkv, 16, d, fill=0x33)
    table = np.array([4, 0, 2], np.int32)
    for layer in (0, 1):
        for kv in (0, 1):
            want.put(layer, kv, table, 0, normal(rng, tp, nkv, d))
    pool = Guarded(want.raw)
    counts = torch.tensor([1, 1, 1, 1, 1, 0], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kids = torch.full((2, 3), 1, dtype=torch.int32, device="cuda")
    k, v, q = (dev(normal(rng, 5, n, d)) for n in (nkv, nkv, nq))
    out = torch.zeros((5, nq, d), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(oc.oc_kv4_attention_workspace_bytes(lay, tp, 5), dtype=torch.uint8, device="cuda")
    oc.oc_kv_pages_fork(pool.pool, lay, 4, dev(table), tp, 2, kids, counts, status)
    for layer in (0, 1):
        oc.oc_kv4_suffix_prefill_layer(q, k, v, 5, pool.pool, lay, kids[1], tp, layer, out, ws)
        oc.oc_kv4_suffix_append(k, v, 5, kids[1], tp, pool.pool, lay, layer)
    assert int(status) == -7 and kids.tolist() == [[1, 1, -1]] * 2 and counts.tolist() == [1, 1, 1, 1, 1, 0]
    pool.check(want.raw)


# ---- bfloat16 pools ----------------------------------------------------------

def pool16(layers, P, nkv, ps, d):
    return np.full((layers, 2, P, nkv, ps, d), 0x3F80, np.uint16)


def put16(raw, layer, kv, table, first, rows):
    t = first + np.arange(rows.shape[0])
    raw[layer, kv, np.asarray(table)[t // raw.shape[4]], :, t % raw.shape[4]] = rows


@pytest.mark.parametrize("nkv,d,ps,G,chunks,ts", [(2, 64, 16, 16, 9, 3), (8, 128, 16, 64, 3, 40), (3, 96, 24, 24, 7, 25),
                                                  (1, 8, 8, 12, 6, 9)])
@pytest.mark.parametrize("objects", [False, True])
def test_stores(nkv, d, ps, G, chunks, ts, objects):
    """Layer payloads and whole chunk objects in, a suffix appended, and both read back."""
    import torch
    import paper_2605_22850_amd as oc
    rng = np.random.default_rng(nkv + d + ts)
    tp, L = chunks * G, 3
    need = -(-(tp + ts) // ps)
    P = need + 3
    table, bad = table_with_holes(rng, P, need)
    lay = oc.Layout(L, nkv, nkv, d, ps, G, P)
    want = pool16(L, P, nkv, ps, d)
    pool = Guarded(want.view(np.uint8))
    rows = normal(rng, L, 2, tp + ts, nkv, d)
    there = ~np.isin(np.arange(tp + ts) // ps, bad)
    # chunk objects [chunk][layer][K|V][token][head][dim]
    chunk_objects = rows[:, :, :tp].reshape(L, 2, chunks, G, nkv, d).transpose(2, 0, 1, 3, 4, 5)
    if objects:
        oc.oc_kv_chunks_ingest(dev(chunk_objects), chunks, 0, dev(table), tp, pool.pool, lay)
    for layer in range(L):
        for kv in (0, 1):
            for t in np.flatnonzero(there):
                put16(want, layer, kv, table, t, rows[layer, kv, t:t + 1])
        if not objects:
            oc.oc_kv_layer_ingest(dev(chunk_objects[:, layer]), chunks, dev(table), tp, pool.pool, lay, layer)
        oc.oc_kv_suffix_append(dev(rows[layer, 0, tp:]), dev(rows[layer, 1, tp:]), ts, dev(table), tp, pool.pool, lay, layer)
    pool.check(want.view(np.uint8))
    back = np.where(there[:tp, None, None], rows[:, :, :tp], 0x40E0).reshape(L, 2, chunks, G, nkv, d).transpose(2, 0, 1, 3, 4, 5)
    out = torch.full(back.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    if objects:
        oc.oc_kv_chunks_gather(dev(table), tp, pool.pool, lay, 0, chunks, out)
    else:
        for layer in range(L):
            one = torch.full((chunks, 2, G, nkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
            oc.oc_kv_layer_gather(dev(table), tp, pool.pool, lay, layer, one, chunks)
            out[:, layer] = one
    assert np.array_equal(out.view(torch.int16).cpu().numpy().view(np.uint16), back)


@pytest.mark.parametrize("tile,nq,nkv,d,tp,ts", [
    (32, 8, 2, 128, 264, 3), (32, 8, 8, 64, 8200, 1), (64, 32, 8, 128, 104, 400), (64, 32, 4, 64, 8200, 200),
    (256, 32, 8, 128, 72, 2200), (256, 20, 5, 128, 8005, 300), (256, 16, 16, 64, 8005, 700)])
def test_prefill(tile, nq, nkv, d, tp, ts):
    """The last page is read in their place: the same rows as with a table that says so."""
    import torch
    import paper_2605_22850_amd as oc
    from tests.test_dispatch import attention_plan as plan
    assert plan(nq, nkv, d, tp, ts)[0] == tile
    rng = np.random.default_rng(tp + ts)
    need = -(-tp // 16)
    P = need + 2
    table, bad = table_with_holes(rng, P, need)
    lay = oc.Layout(2, nq, nkv, d, 16, 16, P)
    raw = normal(rng, 2, 2, P, nkv, 16, d)
    pool = Guarded(raw.view(np.uint8))
    q, k, v = (dev(normal(rng, ts, n, d)) for n in (nq, nkv, nkv))
    ws = torch.empty(oc.oc_attention_workspace_bytes(lay, tp, ts), dtype=torch.uint8, device="cuda")
    outs = []
    for t in (table, np.where(np.isin(np.arange(need), bad), P - 1, table).astype(np.int32)):
        outs.append(torch.full((ts, nq, d), 3.0, dtype=torch.bfloat16, device="cuda"))
        oc.oc_suffix_prefill_layer(q, k, v, ts, pool.pool, lay, dev(t), tp, 1, outs[-1], ws)
    assert torch.equal(*outs) and bool(torch.isfinite(outs[0].float()).all())
    pool.check(raw.view(np.uint8))


@pytest.mark.parametrize("per_request", [False, True])
def test_pipeline(per_request):
    """A run whose requests' tables have holes: layers ingested beside an attention, suffixes appended."""
    import torch
    import paper_2605_22850_amd as oc
    from tests.gpu_util import RequestSet, from_dev
    rng = np.random.default_rng(9)
    rs = RequestSet(4, 8, 2, 64, [2048, 512, 1024], [40, 7, 100], 400, seed=5, suffix_room=True)
    rs.upload(fill=0, with_payload=True)
    want = rs.expected_pool(fill=0, appended=True)
    guarded = Guarded(np.zeros_like(want).view(np.uint8))
    rs.d_pool = guarded.pool
    inside = []
    for r, req in enumerate(rs.reqs):
        table = rs.tables[r].copy()
        bad = np.unique(np.append(rng.permutation(len(table))[:len(table) // 5], len(table) - 1))
        want[:, :, table[bad]] = 0
        table[bad] = [(OUTSIDE + [rs.P])[i % 4] for i in range(len(bad))]
        req.pages = dev(table)
        inside.append(dev(np.where(np.isin(np.arange(len(table)), bad), rs.P - 1, table).astype(np.int32)))

    def run(mode, **kw):
        ctx = rs.context(mode, attention_per_request=per_request, **kw)
        try:
            oc.oc_pipeline_run(ctx, rs.reqs, rs.L)
        finally:
            oc.oc_context_destroy(ctx)
        return [from_dev(r.out) for r in rs.reqs]
    outs = run(oc.OC_MODE_DEVICE_STAGED, append_suffix=True)
    torch.cuda.synchronize()
    guarded.check(want.view(np.uint8))
    for req, pages in zip(rs.reqs, inside):
        req.pages = pages
    for a, b in zip(outs, run(oc.OC_MODE_HBM_RESIDENT)):
        assert np.array_equal(a, b)

"""Pages forked, copied, taken, freed and moved together on the GPU, both kinds
of pool, against plain Python: bytes, counts and tables are equal."""
import numpy as np
import pytest

from tests import kv4_ref as ref
from tests.gpu_util import require_gpu

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
    return torch.from_numpy(np.ascontiguousarray(a).copy()).cuda()


class Pages:
    def __init__(self, bits, layers, nkv, d, ps, P, seed=0):
        import torch
        import paper_2605_22850_amd as oc
        self.rng = np.random.default_rng(seed + P * 13 + layers)
        self.bits, self.ps, self.P = bits, ps, P
        self.lay = oc.Layout(layers, nkv, nkv, d, ps, 16, P)
        n = oc.oc_kv4_pool_bytes(self.lay) if bits == 4 else self.lay.pool_elems * 2
        self.pool = self.rng.integers(0, 256, n, dtype=np.uint8).reshape(2 * layers, P, -1)
        self.counts = np.zeros(P, np.int32)
        self.d_pool = dev(self.pool)
        self.status = torch.full((1,), 99, dtype=torch.int32, device="cuda")

    def hold(self, share):
        self.counts[:] = self.rng.integers(1, 4, self.P) * (self.rng.random(self.P) < share)
        self.upload()

    def upload(self):
        self.d_counts = dev(self.counts)

    def check(self):
        assert np.array_equal(self.d_counts.cpu().numpy(), self.counts)
        assert np.array_equal(self.d_pool.cpu().numpy(), self.pool)


KINDS = [(16, 3, 2, 64, 16), (4, 2, 2, 64, 16), (16, 1, 1, 8, 8), (4, 2, 3, 96, 24), (16, 2, 9, 128, 32), (4, 1, 20, 128, 32)]


@pytest.mark.parametrize("bits,layers,nkv,d,ps", KINDS)
def test_copy(bits, layers, nkv, d, ps):
    import paper_2605_22850_amd as oc
    for n in (1, 5, 11):
        t = Pages(bits, layers, nkv, d, ps, 23)
        t.upload()
        perm = t.rng.permutation(23).astype(np.int32)
        src, dst = t.rng.choice(perm[:11], n).astype(np.int32), perm[12:12 + n]
        t.pool[:, dst] = t.pool[:, src]
        # pairs with an id outside the pool are left out
        src, dst = np.append(src, [23, 1, -1]).astype(np.int32), np.append(dst, [perm[11], -1, perm[11]]).astype(np.int32)
        oc.oc_kv_pages_copy(t.d_pool, t.lay, bits, dev(src), dev(dst), n + 3)
        t.check()


@pytest.mark.parametrize("P,share", [(1, 0.0), (1, 1.0), (63, 0.5), (64, 0.9), (1025, 0.3), (16384, 0.999), (16385, 0.5),
                                     (40000, 0.9)])
def test_take(P, share):
    import torch
    import paper_2605_22850_amd as oc
    t = Pages(4, 1, 1, 32, 8, P)
    t.hold(share)
    if P > 100:
        t.counts[5] = -2                      # released once too often: free
        t.upload()
    free = int((t.counts <= 0).sum())
    for n in sorted({0, 1, free // 3, max(0, free - 1 - free // 3), free, P}):
        out = torch.full((n + 2,), 77, dtype=torch.int32, device="cuda")
        before = t.counts.copy()
        status, pages = ref.take(t.counts, n)
        oc.oc_kv_pages_take(t.d_counts, t.lay, n, out, t.status)
        assert int(t.status) == status and out.tolist() == pages + [77, 77]
        assert status == 0 or np.array_equal(before, t.counts)
        t.check()


@pytest.mark.parametrize("bits,layers,nkv,d,ps", KINDS)
@pytest.mark.parametrize("pages,part,n", [(0, 0, 2), (0, 1, 3), (1, 0, 2), (4, 3, 1), (7, 5, 6), (3, 1, 0)])
def test_fork(bits, layers, nkv, d, ps, pages, part, n):
    import torch
    import paper_2605_22850_amd as oc
    t = Pages(bits, layers, nkv, d, ps, 40)
    t.hold(0.3)
    need = pages + (part > 0)
    table = t.rng.permutation(40)[:need].astype(np.int32)
    t.counts[table] = 1
    t.upload()
    kids = torch.full((n, need + 3), 77, dtype=torch.int32, device="cuda")
    tokens = pages * ps + part
    status, want = ref.fork(t.pool, t.counts, table.tolist(), tokens, ps, n)
    assert status == 0
    oc.oc_kv_pages_fork(t.d_pool, t.lay, bits, dev(table) if need else None, tokens, n, kids, t.d_counts, t.status)
    assert int(t.status) == 0 and kids.tolist() == [w + [77] * 3 for w in want]
    t.check()


def test_fork_of_many_pages_and_children():
    import torch
    import paper_2605_22850_amd as oc
    t = Pages(4, 1, 1, 32, 8, 20000)
    table = t.rng.permutation(20000)[:9001].astype(np.int32)
    t.counts[table] = 1
    t.upload()
    kids = torch.full((33, 9001), 77, dtype=torch.int32, device="cuda")
    _, want = ref.fork(t.pool, t.counts, table.tolist(), 9000 * 8 + 1, 8, 33)
    oc.oc_kv_pages_fork(t.d_pool, t.lay, 4, dev(table), 9000 * 8 + 1, 33, kids, t.d_counts, t.status)
    assert np.array_equal(kids.cpu().numpy(), np.array(want))
    t.check()


def test_fork_without_enough_pages():
    import torch
    import paper_2605_22850_amd as oc
    t = Pages(16, 2, 2, 64, 16, 12)
    t.counts[:] = 1
    t.counts[[3, 8]] = 0
    t.upload()
    table = dev(np.array([0, 1, 2], np.int32))
    kids = torch.full((3, 3), 77, dtype=torch.int32, device="cuda")
    oc.oc_kv_pages_fork(t.d_pool, t.lay, 16, table, 40, 3, kids, t.d_counts, t.status)
    assert int(t.status) == -7 and kids.tolist() == [[77, 77, -1]] * 3
    t.check()
    # two fit, and whole pages need none
    oc.oc_kv_pages_fork(t.d_pool, t.lay, 16, table, 40, 2, kids, t.d_counts, t.status)
    assert int(t.status) == 0 and kids[:2].tolist() == [[0, 1, 3], [0, 1, 8]]
    oc.oc_kv_pages_fork(t.d_pool, t.lay, 16, table, 48, 3, kids, t.d_counts, t.status)
    assert int(t.status) == 0 and kids.tolist() == [[0, 1, 2]] * 3
    assert t.d_counts.tolist() == [6, 6, 4, 1, 1, 1, 1, 1, 1, 1, 1, 1]


def test_release():
    import paper_2605_22850_amd as oc
    t = Pages(4, 1, 1, 32, 8, 500)
    t.hold(1.0)
    table = t.rng.permutation(500)[:301].astype(np.int32)
    oc.oc_kv_pages_release(dev(table), 300 * 8 - 5, t.lay, t.d_counts)      # 300 of the 301 entries
    t.counts[table[:300]] -= 1
    oc.oc_kv_pages_release(dev(np.array([7, -1, 500, 7], np.int32)), 32, t.lay, t.d_counts)
    t.counts[7] -= 2
    oc.oc_kv_pages_release(None, 0, t.lay, t.d_counts)
    t.check()


@pytest.mark.parametrize("bits,layers,nkv,d,ps,P,share", [
    *[(b, n, k, d, ps, 37, 0.5) for b, n, k, d, ps in KINDS],
    (4, 1, 1, 32, 8, 1, 0.0), (4, 1, 1, 32, 8, 1, 1.0), (4, 1, 1, 32, 8, 2, 0.5), (16, 1, 1, 8, 8, 300, 0.0),
    (16, 1, 1, 8, 8, 300, 1.0), (16, 1, 1, 8, 8, 16385, 0.2), (4, 1, 1, 32, 8, 33000, 0.8), (16, 2, 2, 64, 16, 200, 0.05)])
def test_compact(bits, layers, nkv, d, ps, P, share):
    import torch
    import paper_2605_22850_amd as oc
    t = Pages(bits, layers, nkv, d, ps, P)
    t.hold(share)
    tables = t.rng.integers(0, P, (3, 50)).astype(np.int32)
    tables[1, 40:] = -1                      # left alone: outside the pool
    tables[2, 0] = P
    wide = torch.full((3, 55), 0, dtype=torch.int32, device="cuda")
    wide[:, :50] = dev(tables)
    live = torch.full((1,), 99, dtype=torch.int32, device="cuda")
    ws = torch.full((oc.oc_kv_pages_workspace_bytes(t.lay),), 0xFF, dtype=torch.uint8, device="cuda")
    held = t.counts > 0
    n = ref.compact(t.pool, t.counts, tables)
    oc.oc_kv_pages_compact(t.d_pool, t.lay, bits, t.d_counts, wide[:, :50], live, ws)
    assert int(live) == n == held.sum() and np.array_equal(wide[:, :50].cpu().numpy(), tables)
    assert bool((wide[:, 50:] == 0).all())
    t.check()
    # nothing is left to move
    oc.oc_kv_pages_compact(t.d_pool, t.lay, bits, t.d_counts, wide[:0], live, ws)
    assert int(live) == n
    t.check()


def test_operations_replayed_from_a_graph():
    """Fork, release and compact in one captured graph, replayed while the program changes the counts."""
    import torch
    import paper_2605_22850_amd as oc
    t = Pages(4, 2, 2, 64, 16, 300)
    t.upload()
    kids = torch.zeros((2, 5), dtype=torch.int32, device="cuda")
    live = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(oc.oc_kv_pages_workspace_bytes(t.lay), dtype=torch.uint8, device="cuda")
    table = torch.zeros((1, 5), dtype=torch.int32, device="cuda")

    def step():
        oc.oc_kv_pages_fork(t.d_pool, t.lay, 4, table[0], 70, 2, kids, t.d_counts, t.status)
        oc.oc_kv_pages_release(table[0], 70, t.lay, t.d_counts)
        oc.oc_kv_pages_compact(t.d_pool, t.lay, 4, t.d_counts, kids, live, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        t.counts[:] = t.rng.integers(1, 3, 300) * (t.rng.random(300) < 0.4)
        h_table = t.rng.permutation(300)[:5].astype(np.int32)
        t.counts[h_table] += 1
        t.d_counts.copy_(dev(t.counts))
        table.copy_(dev(h_table[None]))
        graph.replay()
        torch.cuda.synchronize()
        status, want = ref.fork(t.pool, t.counts, h_table.tolist(), 70, 16, 2)
        for p in h_table:
            t.counts[p] -= 1
        want = np.array(want)
        n = ref.compact(t.pool, t.counts, want)
        assert int(t.status) == status == 0 and int(live) == n and np.array_equal(kids.cpu().numpy(), want)
        t.check()

"""The prefix held in 4 bits on the GPU, against the float64 reference: stored
bytes are equal to the bit, attention rows within the bound that their roundings
give."""
import numpy as np
import pytest

from tests import kv4_ref as ref
from tests.kv4_cases import BY_PLAN, RAGGED_256
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
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16).copy()).cuda().view(torch.bfloat16)
    return torch.from_numpy(a.copy()).cuda()


def host16(t):
    import torch
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


def normal(rng, *shape, scale=1.0):
    return ref.f64_to_bf16(rng.standard_normal(shape) * scale)


def layout(layers, nq, nkv, d, ps, G, pages):
    import paper_2605_22850_amd as oc
    return oc.Layout(layers, nq, nkv, d, ps, G, pages)


def payload_of(rows_k, rows_v, G):
    """Layer payload [chunk][K|V][G][nkv][d] of rows [T][nkv][d]."""
    n = rows_k.shape[0] // G
    return np.stack((rows_k.reshape(n, G, *rows_k.shape[1:]), rows_v.reshape(n, G, *rows_v.shape[1:])), 1)


# ---- store and read back ----------------------------------------------------

STORES = [
    # (nkv, d, page, chunk, chunks, appended tokens)
    (2, 64, 16, 16, 5, 3), (1, 128, 16, 16, 1, 1), (8, 128, 16, 64, 3, 40), (3, 96, 24, 24, 4, 24), (2, 32, 8, 12, 5, 9),
    (1, 32, 8, 1, 3, 1), (5, 128, 16, 7, 9, 17), (1, 256, 32, 40, 2, 33), (2, 64, 16, 16, 0, 5), (3, 160, 8, 16, 2, 0),
]


def special_rows(rng, T, nkv, d):
    """Random rows among which whole blocks are unusual."""
    x = normal(rng, T, nkv, d)
    b = x.reshape(-1, 32)
    kinds = [lambda r: r.__setitem__(slice(None), 0), lambda r: r.__setitem__(slice(None), 0x8000),
             lambda r: r.__setitem__(3, 0x7F80), lambda r: r.__setitem__(31, 0xFF80), lambda r: r.__setitem__(0, 0x7FC1),
             lambda r: r.__setitem__(7, 0x7F7F), lambda r: r.__setitem__(slice(None), np.arange(32) * 3 + 1),
             lambda r: r.__setitem__(slice(None), rng.integers(0, 1 << 16, 32) & 0x80FF),
             lambda r: r.__setitem__(slice(None), rng.integers(0, 1 << 16, 32))]
    for i in range(0, b.shape[0], 2):
        kinds[(i // 2) % len(kinds)](b[i])
    return x


@pytest.mark.parametrize("nkv,d,ps,G,chunks,ts", STORES)
def test_store_is_exact(nkv, d, ps, G, chunks, ts):
    import torch
    import paper_2605_22850_amd as oc
    rng = np.random.default_rng(nkv * 1000 + d + ts)
    tp = chunks * G
    need = -(-(tp + ts) // ps)
    P = need + 3
    table = rng.permutation(P)[:need].astype(np.int32)
    want = ref.Pool4(3, P, nkv, ps, d, fill=0xA7)
    lay = layout(3, nkv, nkv, d, ps, G, P)
    pool = dev(want.raw)
    k, v = special_rows(rng, tp + ts, nkv, d), special_rows(rng, tp + ts, nkv, d)
    for kv, rows in ((0, k), (1, v)):
        want.put(1, kv, table, 0, rows)
    d_table = dev(table) if need else None
    if chunks:
        oc.oc_kv4_layer_ingest(dev(payload_of(k[:tp], v[:tp], G)), chunks, d_table, tp, pool, lay, 1)
    oc.oc_kv4_suffix_append(dev(k[tp:]), dev(v[tp:]), ts, d_table, tp, pool, lay, 1)
    got = pool.cpu().numpy()
    # every byte: codes, scales, slots behind the last token, the other layers and pages
    assert np.array_equal(got, want.raw)
    # and back, as values (a NaN is a NaN)
    n = (tp + ts) // G
    if n:
        out = torch.full((n * 2 * G * nkv * d + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
        oc.oc_kv4_layer_gather(d_table, n * G, pool, lay, 1, out, n)
        assert bool((out[-64:] == 7.0).all())
        back = ref.bf16_to_f64(host16(out[:-64])).reshape(n, 2, G, nkv, d)
        values = [want.get(1, kv, table, n * G).reshape(n, G, nkv, d) for kv in (0, 1)]
        for kv in (0, 1):
            assert np.array_equal(back[:, kv], values[kv], equal_nan=True)


def test_every_bfloat16_as_a_block_maximum():
    """Each bit pattern leads one block; the rest of the block are smaller magnitudes of both signs."""
    import paper_2605_22850_amd as oc
    rng = np.random.default_rng(5)
    T, d = 2048, 32 * 32
    top = np.arange(1 << 16, dtype=np.uint16)
    x = np.minimum(rng.integers(0, 1 << 15, (1 << 16, 32)), (top & 0x7FFF)[:, None])
    near = np.maximum((top & 0x7FFF).astype(np.int64)[:, None] - rng.integers(0, 520, (1 << 16, 32)), 0)
    x = np.where(rng.random(x.shape) < 0.7, near, x).astype(np.uint16)
    x |= (rng.integers(0, 2, x.shape) << 15).astype(np.uint16)
    x[np.arange(1 << 16), rng.integers(0, 32, 1 << 16)] = top
    rows = x.reshape(T, 1, d)
    P = T // 16
    table = rng.permutation(P).astype(np.int32)
    want = ref.Pool4(1, P, 1, 16, d)
    want.put(0, 0, table, 0, rows)
    want.put(0, 1, table, 0, rows[::-1])
    pool = dev(np.full_like(want.raw, 0xFF))
    oc.oc_kv4_suffix_append(dev(rows), dev(rows[::-1]), T, dev(table), 0, pool, layout(1, 1, 1, d, 16, 16, P), 0)
    assert np.array_equal(pool.cpu().numpy(), want.raw)


# ---- attention --------------------------------------------------------------

class Case:
    """A request over a pool whose every unwritten byte says NaN."""

    def __init__(self, nq, nkv, d, tp, ts, seed=0, extra_pages=3, layers=2, layer=1, scale=1.0):
        import torch
        rng = np.random.default_rng(seed * 7919 + nq * 31 + tp * 7 + ts)
        self.nq, self.nkv, self.d, self.tp, self.ts, self.layer = nq, nkv, d, tp, ts, layer
        need = -(-tp // 16)
        P = need + extra_pages
        self.lay = layout(layers, nq, nkv, d, 16, 16, P)
        self.table = rng.permutation(P)[:need].astype(np.int32)
        self.pool = ref.Pool4(layers, P, nkv, 16, d)
        self.k0, self.v0 = normal(rng, tp, nkv, d), normal(rng, tp, nkv, d)
        self.pool.put(layer, 0, self.table, 0, self.k0)
        self.pool.put(layer, 1, self.table, 0, self.v0)
        self.q, self.k, self.v = normal(rng, ts, nq, d, scale=scale), normal(rng, ts, nkv, d), normal(rng, ts, nkv, d)
        self.d_pool, self.d_table = dev(self.pool.raw), dev(self.table) if need else None
        self.d_q, self.d_k, self.d_v = dev(self.q), dev(self.k), dev(self.v)
        self.torch = torch

    def run(self, stream=None, workspace=None, out=None):
        import paper_2605_22850_amd as oc
        torch = self.torch
        out = torch.full(self.q.shape, float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
        if workspace is None:
            n = oc.oc_kv4_attention_workspace_bytes(self.lay, self.tp, self.ts)
            workspace = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        oc.oc_kv4_suffix_prefill_layer(self.d_q, self.d_k, self.d_v, self.ts, self.d_pool, self.lay, self.d_table,
                                       self.tp, self.layer, out, workspace, stream)
        return out

    def expected(self, rows=None):
        rows = np.arange(self.ts) if rows is None else np.asarray(rows)
        k = np.concatenate((self.pool.get(self.layer, 0, self.table, self.tp), ref.bf16_to_f64(self.k)))
        v = np.concatenate((self.pool.get(self.layer, 1, self.table, self.tp), ref.bf16_to_f64(self.v)))
        return ref.attention(ref.bf16_to_f64(self.q[rows]), k, v, self.tp + rows + 1)

    def check(self, out, rows=None, what=""):
        got = host16(out)
        ref.assert_rows_close(got if rows is None else got[rows], *self.expected(rows), what=what)


SHAPES = [
    # (nq, nkv, d, prefix, suffix): one row and more than a tile, prefixes around pages, units and
    # rounds of the wavefronts, no prefix at all, group sizes that are no power of two
    *[(4, 2, 64, tp, 1) for tp in (0, 1, 15, 16, 17, 31, 32, 33, 255, 256, 257)],
    *[(8, 2, 128, tp, 5) for tp in (0, 1, 16, 40, 511, 513)],
    (4, 1, 128, 300, 4), (4, 1, 128, 300, 5), (16, 1, 64, 47, 1), (17, 1, 64, 47, 1), (33, 1, 128, 100, 3),
    (6, 2, 128, 130, 33), (5, 5, 64, 70, 31), (5, 5, 64, 70, 32), (5, 5, 64, 70, 33), (12, 4, 64, 100, 100),
    (2, 2, 128, 0, 200), (3, 1, 64, 9, 129), (64, 1, 128, 264, 9), (40, 8, 128, 205, 21),
]


@pytest.mark.parametrize("nq,nkv,d,tp,ts", SHAPES)
def test_attention(nq, nkv, d, tp, ts):
    c = Case(nq, nkv, d, tp, ts)
    c.check(c.run())


@pytest.mark.parametrize("nq,nkv,d,tp,ts", [s for shapes in BY_PLAN.values() for s in shapes] + RAGGED_256)
def test_every_kernel(nq, nkv, d, tp, ts):
    """Row tiles of each size, keys whole and split over workgroups."""
    c = Case(nq, nkv, d, tp, ts)
    out = c.run()
    grp = nq // nkv
    rows = sorted({0, 1 % ts, 15 // grp % ts, 16 // grp % ts, 256 // grp % ts, ts // 3, ts // 2, ts - 1})
    c.check(out, rows)
    assert bool(c.torch.isfinite(out.float()).all())
    # the same call again, into another workspace: the same bits
    assert c.torch.equal(c.run(), out)


def test_large_scores():
    """Scores of some hundreds: single keys carry rows, and maxima rise late."""
    for seed in range(3):
        c = Case(8, 2, 128, 700, 40, seed=seed, scale=40.0)
        # scores of some 2^11 in fp32: their error of 2^-24 * 128 products is 2^-6 at most, through exp another
        # 2^-6 of sum p|v| on top of the bound
        got = ref.bf16_to_f64(host16(c.run()))
        out, mag = c.expected()
        assert (np.abs(got - out) <= (2 * 2.0 ** -6 + 3 * 2.0 ** -8) * mag + 1e-30).all()


@pytest.mark.parametrize("nq,nkv,d,tp,ts", [(8, 2, 128, 40, 50), (4, 2, 64, 0, 70), (8, 2, 128, 37, 300),
                                            (32, 4, 64, 21, 400), (32, 8, 128, 100, 1200)])
def test_values_of_later_tokens_reach_no_earlier_row(nq, nkv, d, tp, ts):
    c = Case(nq, nkv, d, tp, ts)
    bad = ts // 2
    rows = np.array(sorted({0, bad // 2, bad - 2, bad - 1}))
    want = c.expected(rows)
    c.v[bad, :, ::3], c.v[bad, :, 1::3] = 0x7F80, 0x7FC0
    c.k[bad + 1] = 0x7FC0
    c.d_k, c.d_v = dev(c.k), dev(c.v)
    got = host16(c.run())
    assert np.isfinite(ref.bf16_to_f64(got[:bad])).all()
    ref.assert_rows_close(got[rows], *want)
    seen = ref.bf16_to_f64(got[bad])
    assert not np.isfinite(seen[:, ::3]).any() and np.isnan(seen[:, 1::3]).all()
    assert np.isfinite(seen[:, 2::3]).all() and np.isnan(ref.bf16_to_f64(got[bad + 1:])).all()


def test_nan_blocks_of_the_prefix():
    """A cached block that is NaN: K's reaches every row of its head, V's the block's dimensions."""
    c = Case(4, 2, 128, 90, 6)
    c.v0[5, 0, 33] = 0x7F80
    c.pool.put(c.layer, 1, c.table, 0, c.v0)
    c.d_pool = dev(c.pool.raw)
    got = ref.bf16_to_f64(host16(c.run()))
    want, _ = c.expected()
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(got[:, :2, 32:64]).all()
    c.k0[7, 1, 0] = 0xFFC0
    c.pool.put(c.layer, 0, c.table, 0, c.k0)
    c.d_pool = dev(c.pool.raw)
    got = ref.bf16_to_f64(host16(c.run()))
    assert np.isnan(got[:, 2:]).all() and np.isfinite(got[:, :2, :32]).all()


def test_pages_past_four_gigabytes():
    """Page ids whose byte offsets pass 32 bits, K and V apart by more than that."""
    import torch
    import paper_2605_22850_amd as oc
    c = Case(8, 8, 128, 100, 3, layers=1, layer=0)
    P = 600_000
    lay = layout(1, 8, 8, 128, 16, 16, P)
    table = np.array([P - 1, 3, P - 77, 493_448, 493_447, 0, 599_000], np.int32)
    pool = torch.empty(oc.oc_kv4_pool_bytes(lay), dtype=torch.uint8, device="cuda")
    small = c.pool.raw
    view = pool.view(2, P, c.pool.page_bytes)
    for i, p in enumerate(table):
        view[:, p] = dev(small[0, :, c.table[i]])
    c.d_pool, c.lay, c.d_table = pool, lay, dev(table)
    c.check(c.run())
    back = torch.empty(6 * 2 * 16 * 8 * 128, dtype=torch.bfloat16, device="cuda")
    oc.oc_kv4_layer_gather(c.d_table, 96, pool, lay, 0, back, 6)
    got = ref.bf16_to_f64(host16(back)).reshape(6, 2, 16, 8, 128)
    assert np.array_equal(got[:, 1].reshape(96, 8, 128), c.pool.get(0, 1, c.table, 96))


def test_two_streams_and_a_side_stream():
    """Two calls at once, each with its workspace, on streams of their own; a third waits for neither."""
    import torch
    cs = [Case(32, 8, 128, 6000 + 500 * i, 3, seed=i) for i in range(3)]
    want = [c.run() for c in cs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    outs = []
    for c, s in zip(cs, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs.append(c.run())
    torch.cuda.synchronize()
    for a, b in zip(want, outs):
        assert torch.equal(a, b)


def test_prefill_captured_and_replayed():
    import torch
    import paper_2605_22850_amd as oc
    c = Case(32, 8, 128, 5000, 7)
    want = c.run()
    ws = torch.empty(oc.oc_kv4_attention_workspace_bytes(c.lay, c.tp, c.ts), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(workspace=ws, out=out)
    for i in range(4):
        out.zero_()
        ws.fill_(255 - i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        c.run()                                  # eager work of the program's own in between
        torch.cuda.synchronize()


# ---- one token for each request ----------------------------------------------

class Batch:
    def __init__(self, nq, nkv, d, lengths, seed=0, room=40, entries_more=2):
        rng = np.random.default_rng(seed + len(lengths) * 101 + sum(lengths))
        self.nq, self.nkv, self.d, self.lengths = nq, nkv, d, list(lengths)
        self.most = max(0, max(lengths)) + room
        B = len(lengths)
        entries = self.most // 16 + 1
        needs = [(max(n, 0) + room) // 16 + 1 for n in lengths]
        P = sum(needs) + 2
        perm = rng.permutation(P).astype(np.int32)
        # entries that no request uses name pages outside the pool
        self.tables = np.full((B, entries + entries_more), 1 << 30, np.int32)
        at = 0
        for i, n in enumerate(needs):
            self.tables[i, :n] = perm[at:at + n]
            at += n
        self.lay = layout(2, nq, nkv, d, 16, 16, P)
        self.pool = ref.Pool4(2, P, nkv, 16, d)
        for i, n in enumerate(self.lengths):
            if n > 0:
                for kv in (0, 1):
                    self.pool.put(1, kv, self.tables[i], 0, normal(rng, n, nkv, d))
        self.q, self.k, self.v = normal(rng, B, nq, d), normal(rng, B, nkv, d), normal(rng, B, nkv, d)
        self.d_pool, self.d_tables = dev(self.pool.raw), dev(self.tables)
        self.d_lengths = dev(np.array(self.lengths, np.int32))
        self.d_q, self.d_k, self.d_v = dev(self.q), dev(self.k), dev(self.v)

    def workspace(self, most=None):
        import torch
        import paper_2605_22850_amd as oc
        n = oc.oc_kv4_decode_workspace_bytes(self.lay, len(self.lengths), self.most if most is None else most)
        return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")

    def run(self, out=None, workspace=None, most=None, stream=None):
        import torch
        import paper_2605_22850_amd as oc
        most = self.most if most is None else most
        out = torch.full(self.q.shape, 3.0, dtype=torch.bfloat16, device="cuda") if out is None else out
        workspace = self.workspace(most) if workspace is None else workspace
        oc.oc_kv4_decode_layer(self.d_q, self.d_k, self.d_v, len(self.lengths), self.d_pool, self.lay, self.d_tables,
                               self.d_lengths, most, 1, out, workspace, stream)
        return out

    def check(self, out):
        """Rows, rows of empty places, and every byte of the pool after the append."""
        got = host16(out)
        for i, n in enumerate(self.lengths):
            if n < 0:
                assert (got[i] == 0x4040).all(), f"request {i} is an empty place"
                continue
            k, v = (np.concatenate((self.pool.get(1, kv, self.tables[i], n), ref.bf16_to_f64(x[i:i + 1])))
                    for kv, x in ((0, self.k), (1, self.v)))
            ref.assert_rows_close(got[i:i + 1], *ref.attention(ref.bf16_to_f64(self.q[i:i + 1]), k, v, [n + 1]),
                                  what=f"request {i} of {n} tokens")
        self.append()
        assert np.array_equal(self.d_pool.cpu().numpy(), self.pool.raw)

    def append(self):
        for i, n in enumerate(self.lengths):
            if n >= 0:
                self.pool.put(1, 0, self.tables[i], n, self.k[i:i + 1])
                self.pool.put(1, 1, self.tables[i], n, self.v[i:i + 1])


BATCHES = [
    (4, 2, 64, [0]), (4, 2, 64, [15]), (4, 2, 64, [16]), (32, 8, 128, [-1, 31, 0, 32, 33, 1, 511, 700]),
    (5, 1, 128, [100, -1, 0, 2000, 17]), (8, 8, 64, [250, 3]), (17, 1, 64, [90, 1, 5]), (40, 1, 128, [77, 300]),
    (64, 8, 128, [1500, 40]), (32, 4, 64, [5000, 12, -5]), (32, 8, 128, [-1, -2]),
]


@pytest.mark.parametrize("nq,nkv,d,lengths", BATCHES)
def test_decode(nq, nkv, d, lengths):
    b = Batch(nq, nkv, d, lengths)
    b.check(b.run())


# (n_q, n_kv, d, lengths) that make a list of ranges: a lane to a request and two, equal and
# very unequal lengths, whole ranges only, no tokens at all, empty places first and last
def _lists():
    rng = np.random.default_rng(21)
    some = lambda n, most: (np.exp(rng.uniform(0, np.log(most), n)).astype(int) - 1).tolist()  # noqa: E731
    return [
        (8, 1, 64, [9000, 3, 0, -1, 1, 2500, 2500]), (4, 1, 128, [2048] * 3), (16, 8, 64, [1024] * 4), (2, 2, 64, [0, 0, 0]),
        (2, 2, 64, [-1, -1]), (4, 4, 64, [-1, 1000, -1, -1]), (34, 1, 64, [1000, 30, 2000]), (8, 8, 64, [40] + some(20, 7000)),
        (4, 1, 64, some(64, 3000)), (4, 1, 64, some(65, 3000)), (2, 1, 64, [-1] + some(126, 2000) + [-1]),
        (6, 3, 64, [1900] * 80), (4, 1, 64, [0] * 64 + [6000]), (4, 1, 64, [6000] + [-1] * 127),
    ]


@pytest.mark.parametrize("nq,nkv,d,lengths", _lists())
def test_decode_by_list(nq, nkv, d, lengths):
    b = Batch(nq, nkv, d, lengths, room=800)
    b.check(b.run())


def test_decode_long_and_short_together():
    b = Batch(8, 1, 128, [20000, 3, 9000, 0, 500, -1, 31])
    first = b.run()
    b.check(first)
    import torch
    assert torch.equal(b.run(), first)          # the token is stored again where it stood


def test_decode_two_calls_at_once():
    """Two batches of one pool on two streams, each with its workspace and tables."""
    import torch
    bs = [Batch(32, 8, 128, [3000, 40, -1, 700], seed=s) for s in range(2)]
    want = [b.run() for b in bs]
    torch.cuda.synchronize()
    outs = []
    for b in bs:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs.append(b.run())
    torch.cuda.synchronize()
    for b, a, o in zip(bs, want, outs):
        assert torch.equal(a, o)
        b.check(o)


def test_decode_many_requests():
    """More requests than a workgroup has threads, of a few tokens each."""
    rng = np.random.default_rng(8)
    b = Batch(4, 2, 64, rng.integers(-1, 40, 600).tolist(), room=3)
    got = host16(b.run())
    for i in rng.permutation(600)[:60]:
        n = b.lengths[i]
        if n < 0:
            assert (got[i] == 0x4040).all()
            continue
        k, v = (np.concatenate((b.pool.get(1, kv, b.tables[i], n), ref.bf16_to_f64(x[i:i + 1])))
                for kv, x in ((0, b.k), (1, b.v)))
        ref.assert_rows_close(got[i:i + 1], *ref.attention(ref.bf16_to_f64(b.q[i:i + 1]), k, v, [n + 1]))
    b.append()
    assert np.array_equal(b.d_pool.cpu().numpy(), b.pool.raw)


def test_decode_special_tokens():
    """The new token's own row may be infinite, NaN or zero: its row alone shows it, its blocks say NaN."""
    b = Batch(4, 2, 64, [20, 40, 60, 0])
    b.v[1, 0, :32], b.v[2, 1, 40], b.k[3] = 0x7F80, 0x7FC0, 0
    b.d_k, b.d_v = dev(b.k), dev(b.v)
    got = ref.bf16_to_f64(host16(b.run()))
    assert np.isposinf(got[1, :2, :32]).all() and np.isfinite(got[1, 2:]).all() and np.isfinite(got[1, :2, 32:]).all()
    assert np.isnan(got[2, 2:, 40]).all() and np.isnan(got[2]).sum() == 2
    assert np.isfinite(got[[0, 3]]).all()
    b.append()
    assert np.array_equal(b.d_pool.cpu().numpy(), b.pool.raw)


def test_decode_lengths_above_max_tokens():
    """They are held to it: the pages behind are neither read nor written."""
    b = Batch(4, 2, 64, [100, 30])
    b.lengths = [64, 30]
    b.check(b.run(most=64))


def test_decode_page_ids_outside_the_pool():
    """As a fork or take without pages leaves them: a token without a page is not appended, and where a prefix
    names none page 0 is read; the other rows are as ever, and nothing else is written."""
    b = Batch(4, 2, 64, [40, 96, 33, 16])
    b.d_tables[1, 6], b.d_tables[3, 1], b.d_tables[2, 0] = -1, b.lay.num_pages, -5
    got = host16(b.run())
    for i in (0, 1, 3):
        n = b.lengths[i]
        k, v = (np.concatenate((b.pool.get(1, kv, b.tables[i], n), ref.bf16_to_f64(x[i:i + 1])))
                for kv, x in ((0, b.k), (1, b.v)))
        ref.assert_rows_close(got[i:i + 1], *ref.attention(ref.bf16_to_f64(b.q[i:i + 1]), k, v, [n + 1]))
    b.lengths = [40, -1, 33, -1]
    b.append()
    assert np.array_equal(b.d_pool.cpu().numpy(), b.pool.raw)


def test_decode_captured_while_requests_grow():
    """One captured call, replayed as the lengths grow on the device, with a place that empties."""
    import torch
    b = Batch(8, 2, 128, [14, 600, -1, 31], room=12)
    ws, out = b.workspace(), torch.zeros(b.q.shape, dtype=torch.bfloat16, device="cuda")
    saved = b.d_pool.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.run(out=out, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    b.d_pool.copy_(saved)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run(out=out, workspace=ws)
    rng = np.random.default_rng(3)
    for step in range(6):
        b.q, b.k, b.v = (normal(rng, *x.shape) for x in (b.q, b.k, b.v))
        for t, x in ((b.d_q, b.q), (b.d_k, b.k), (b.d_v, b.v)):
            t.copy_(dev(x))
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        b.check(out)
        b.lengths = [n + 1 if n >= 0 else n for n in b.lengths]
        if step == 3:
            b.lengths[3] = -1
        b.d_lengths.copy_(dev(np.array(b.lengths, np.int32)))


# ---- as they are used together --------------------------------------------------

def test_a_request_from_payload_to_forks_and_back():
    """A prefix arrives layer by layer, a prompt's tokens are computed and appended, the request forks, each
    continuation decodes tokens of its own, one ends, the pool is compacted, decoding goes on, and the
    first request's layers are written back."""
    import torch
    import paper_2605_22850_amd as oc
    rng = np.random.default_rng(11)
    L, nq, nkv, d, G, P = 2, 8, 2, 64, 16, 64
    tp, ts, n_kids, steps = 48, 21, 3, 5
    lay = layout(L, nq, nkv, d, 16, G, P)
    want = ref.Pool4(L, P, nkv, 16, d, fill=0)
    pool = dev(want.raw)
    counts, status = torch.zeros(P, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    h_counts = np.zeros(P, np.int64)
    # pages that an ended request leaves free in front
    junk = torch.empty(7, dtype=torch.int32, device="cuda")
    oc.oc_kv_pages_take(counts, lay, 7, junk, status)
    need = -(-(tp + ts) // 16)
    entries = need + 2
    tables = torch.full((1 + n_kids, entries), -1, dtype=torch.int32, device="cuda")
    h_tables = np.full((1 + n_kids, entries), -1, np.int64)
    ref.take(h_counts, 7)
    oc.oc_kv_pages_take(counts, lay, entries, tables[0], status)
    h_tables[0] = ref.take(h_counts, entries)[1]
    oc.oc_kv_pages_release(junk, 7 * 16, lay, counts)
    h_counts[:7] -= 1
    ws = torch.empty(max(oc.oc_kv4_attention_workspace_bytes(lay, tp, ts), oc.oc_kv4_decode_workspace_bytes(lay, 4, 160)),
                     dtype=torch.uint8, device="cuda")
    for l in range(L):
        k, v = normal(rng, tp, nkv, d), normal(rng, tp, nkv, d)
        oc.oc_kv4_layer_ingest(dev(payload_of(k, v, G)), tp // G, tables[0], tp, pool, lay, l)
        for kv, x in ((0, k), (1, v)):
            want.put(l, kv, h_tables[0], 0, x)
        q, k, v = normal(rng, ts, nq, d), normal(rng, ts, nkv, d), normal(rng, ts, nkv, d)
        out = torch.empty(ts, nq, d, dtype=torch.bfloat16, device="cuda")
        oc.oc_kv4_suffix_prefill_layer(dev(q), dev(k), dev(v), ts, pool, lay, tables[0], tp, l, out, ws)
        kk, vv = (np.concatenate((want.get(l, kv, h_tables[0], tp), ref.bf16_to_f64(x))) for kv, x in ((0, k), (1, v)))
        ref.assert_rows_close(host16(out), *ref.attention(ref.bf16_to_f64(q), kk, vv, tp + 1 + np.arange(ts)))
        oc.oc_kv4_suffix_append(dev(k), dev(v), ts, tables[0], tp, pool, lay, l)
        for kv, x in ((0, k), (1, v)):
            want.put(l, kv, h_tables[0], tp, x)
    n = tp + ts
    flat = want.raw.reshape(2 * L, P, -1)
    oc.oc_kv_pages_fork(pool, lay, 4, tables[0], n, n_kids, tables[1:], counts, status)
    st, kids = ref.fork(flat, h_counts, h_tables[0].tolist(), n, 16, n_kids)
    assert st == 0
    for i, t in enumerate(kids):
        h_tables[1 + i, :need] = t
    more = torch.empty(n_kids * 2, dtype=torch.int32, device="cuda")
    oc.oc_kv_pages_take(counts, lay, n_kids * 2, more, status)
    tables[1:, need:] = more.view(n_kids, 2)
    h_tables[1:, need:] = np.array(ref.take(h_counts, n_kids * 2)[1]).reshape(n_kids, 2)
    lengths = torch.full((1 + n_kids,), n, dtype=torch.int32, device="cuda")
    h_len = [n] * (1 + n_kids)
    live = torch.zeros(1, dtype=torch.int32, device="cuda")
    pws = torch.empty(oc.oc_kv_pages_workspace_bytes(lay), dtype=torch.uint8, device="cuda")
    for step in range(steps * 2):
        if step == steps:
            # child 2 ends; everything that is held moves to the front
            oc.oc_kv_pages_release(tables[2], entries * 16, lay, counts)
            for p in h_tables[2]:
                h_counts[p] -= 1
            lengths[2], h_len[2] = -1, -1
            oc.oc_kv_pages_compact(pool, lay, 4, counts, tables, live, pws)
            n_live = ref.compact(flat, h_counts, h_tables)
            assert int(live) == n_live and n_live < h_tables.size
            assert int(tables[[0, 1, 3]].max()) < n_live
        B = 1 + n_kids
        for l in range(L):
            q, k, v = normal(rng, B, nq, d), normal(rng, B, nkv, d), normal(rng, B, nkv, d)
            out = torch.empty(B, nq, d, dtype=torch.bfloat16, device="cuda")
            oc.oc_kv4_decode_layer(dev(q), dev(k), dev(v), B, pool, lay, tables, lengths, entries * 16 - 1, l, out, ws)
            got = host16(out)
            for i in range(B):
                if h_len[i] < 0:
                    continue
                kk, vv = (np.concatenate((want.get(l, kv, h_tables[i], h_len[i]), ref.bf16_to_f64(x[i:i + 1])))
                          for kv, x in ((0, k), (1, v)))
                ref.assert_rows_close(got[i:i + 1], *ref.attention(ref.bf16_to_f64(q[i:i + 1]), kk, vv, [h_len[i] + 1]))
                for kv, x in ((0, k), (1, v)):
                    want.put(l, kv, h_tables[i], h_len[i], x[i:i + 1])
        lengths += (lengths >= 0).int()
        h_len = [x + 1 if x >= 0 else x for x in h_len]
    assert np.array_equal(pool.cpu().numpy(), want.raw)
    assert np.array_equal(counts.cpu().numpy(), h_counts) and np.array_equal(tables.cpu().numpy(), h_tables)
    whole = h_len[0] // G
    for l in range(L):
        back = torch.empty(whole * 2 * G * nkv * d, dtype=torch.bfloat16, device="cuda")
        oc.oc_kv4_layer_gather(tables[0], whole * G, pool, lay, l, back, whole)
        got = ref.bf16_to_f64(host16(back)).reshape(whole, 2, G, nkv, d)
        for kv in (0, 1):
            assert np.array_equal(got[:, kv].reshape(-1, nkv, d), want.get(l, kv, h_tables[0], whole * G))

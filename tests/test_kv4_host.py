"""The 4-bit cache and the page operations without a GPU: the reference's own
checks, sizes, refusals (every call here fails validation or has nothing to do)
and the binding's marshalling."""
import ctypes
from ctypes import CFUNCTYPE, POINTER, c_int, c_int32, c_int64, c_size_t, c_void_p

import numpy as np
import pytest

import paper_2605_22850_amd as oc
from paper_2605_22850_amd import _lib as L
from tests import kv4_ref as ref
from tests.kv4_cases import BY_PLAN, RAGGED_256

FAKE = 1 << 20            # aligned non-null "device" address; never dereferenced
BIG = 1 << 40


def _layout(**kw):
    base = dict(num_layers=2, num_q_heads=4, num_kv_heads=2, head_dim=64, page_size=16, chunk_tokens=16, num_pages=64)
    base.update(kw)
    return L.c_layout(*base.values())


# ---- the reference ----------------------------------------------------------

def test_reference_encodes_every_bfloat16():
    u = np.arange(1 << 16, dtype=np.uint16)
    x = ref.bf16_to_f64(u)
    for top in (0x3F80, 0x3FE0, 0x3FE1, 0x0080, 0x7F7F, 0x42C8):
        m = ref.bf16_to_f64(np.uint16(top))
        own = u[np.isfinite(x) & (np.abs(x) <= m)]
        own = own[:own.size // 31 * 31].reshape(-1, 31)
        block = np.concatenate([np.full((own.shape[0], 1), top, np.uint16), own], 1)
        code, scale = ref.encode(block)
        step = 2.0 ** (scale.astype(np.int64) - 127)
        v, w = ref.bf16_to_f64(block), ref.decode(code, scale)
        # half a step of the code's binade; a magnitude of 6 to 7 scales is off by one scale at most
        mag = np.abs(v) / step
        half = np.where(mag < 2, 0.25, np.where(mag < 4, 0.5, 1.0)) * step
        if top != 0x7F7F:
            assert (np.abs(v - w) <= half).all() and (np.signbit(v) == (code >= 8)).all()
            assert (m <= 7 * step).all() and ((m > 3.5 * step) | (scale[:, :1] == 2)).all()


def test_reference_scale_bytes():
    def byte(top):
        return int(ref.encode(np.array([top] + [0] * 31, np.uint16))[1][0])
    assert byte(0) == 2 and byte(0x8000) == 2 and byte(1) == 2          # zero and subnormals
    assert byte(0x3F80) == 125                                          # 1 = 4 / 4
    assert byte(0x3FE0) == 125 and byte(0x3FE1) == 126                  # 1.75 = 7 / 4, and the next
    assert byte(0x7F7F) == 252 and byte(0x7F80) == 255 and byte(0xFFC0) == 255
    code, scale = ref.encode(np.array([0x7FC0] + [0x3F80] * 31, np.uint16))
    assert (code == 0).all() and np.isnan(ref.decode(code, scale)).all()


# ---- sizes ------------------------------------------------------------------

@pytest.mark.parametrize("nkv,d,ps", [(2, 64, 16), (8, 128, 16), (1, 32, 8), (3, 96, 24), (1, 128, 8)])
def test_pool_bytes(nkv, d, ps):
    lay = oc.Layout(3, nkv, nkv, d, ps, 16, 7)
    assert oc.oc_kv4_pool_bytes(lay) == ref.Pool4(3, 7, nkv, ps, d).raw.size


def test_sizes_of_unsupported_layouts():
    for kw in (dict(head_dim=48), dict(page_size=12), dict(num_q_heads=3), dict(num_pages=0)):
        assert oc.lib().oc_kv4_pool_bytes(ctypes.byref(_layout(**kw))) == 0
    with pytest.raises(oc.OcError, match="multiple of 32"):
        oc.oc_kv4_pool_bytes(oc.Layout(1, 1, 1, 40, 16, 16, 4))
    for kw in (dict(head_dim=96), dict(page_size=32)):
        lay = _layout(**kw)
        assert oc.lib().oc_kv4_attention_workspace_bytes(ctypes.byref(lay), 64, 8) == 0
        assert oc.lib().oc_kv4_decode_workspace_bytes(ctypes.byref(lay), 2, 64) == 0
    lay = ctypes.byref(_layout())
    for tp, ts in ((-1, 8), (64, 0), (1 << 30, 1), (1 << 62, 1), (0, 1 << 62)):
        assert oc.lib().oc_kv4_attention_workspace_bytes(lay, tp, ts) == 0
    for b, most in ((0, 64), (1, -1), (65536, 64), (1, 1 << 30), (1 << 62, 1 << 62)):
        assert oc.lib().oc_kv4_decode_workspace_bytes(lay, b, most) == 0
    assert oc.lib().oc_kv4_attention_workspace_bytes(lay, 0, 1) >= 256
    assert oc.lib().oc_kv4_decode_workspace_bytes(lay, 1, 0) >= 256
    # a pool whose size has no 64-bit number
    assert oc.lib().oc_kv4_pool_bytes(ctypes.byref(_layout(num_layers=1 << 30, num_pages=1 << 60))) == 0
    for f in ("oc_kv4_pool_bytes", "oc_kv_pages_workspace_bytes"):
        assert getattr(oc.lib(), f)(None) == 0
    assert oc.oc_kv_pages_workspace_bytes(oc.Layout(1, 1, 1, 32, 8, 8, 9)) >= (9 + 2 * 4) * 4


# ---- plans ------------------------------------------------------------------

def plan(nq, nkv, d, tp, ts, batch=0):
    """Tile rows, row tiles, key units, splits, units per split."""
    lay, out = L.c_layout(1, nq, nkv, d, 16, 16, 1 << 40), (c_int64 * 5)()
    assert oc.lib().oc_internal_kv4_plan(ctypes.byref(lay), c_int64(batch), c_int64(tp), c_int64(ts), out) == 0
    return list(out)


@pytest.mark.parametrize("want", BY_PLAN)
def test_every_kernel_has_its_shapes(want):
    for shape in BY_PLAN[want]:
        tile, _, _, splits, _ = plan(*shape)
        assert (tile, shape[2], "none" if splits == 1 else "few" if splits <= 8 else "many") == want, shape


def test_ragged_prefixes_reach_the_large_tiles():
    assert {plan(*s)[0] for s in RAGGED_256} == {256}


def test_plans_cover_rows_and_keys():
    rng = np.random.default_rng(2)
    for _ in range(2000):
        nkv = int(rng.integers(1, 17))
        nq, d = nkv * int(rng.integers(1, 20)), int(rng.choice([64, 128]))
        tp, ts = int(np.exp(rng.uniform(0, 11.5))) - 1, int(np.exp(rng.uniform(0, 9)))
        tile, m_tiles, units, splits, per = plan(nq, nkv, d, tp, ts)
        rows = ts * nq // nkv
        assert (m_tiles - 1) * tile < rows <= m_tiles * tile
        assert (splits - 1) * per < units <= splits * per
        pages = (-(-tp // 16), -(-ts // 16))
        assert units == (-(-sum(pages) // 4) if tile == 256 else -(-pages[0] // 2) + -(-ts // 32))
        need = oc.oc_kv4_attention_workspace_bytes(oc.Layout(1, nq, nkv, d, 16, 16, 8), tp, ts)
        assert need >= (splits * nkv * rows * (d + 2) * 4 if splits > 1 else 256)
        batch = int(rng.integers(1, 300))
        tile, m_tiles, units, splits, per = plan(nq, nkv, d, tp, 1, batch)
        assert m_tiles * tile >= nq // nkv and units == -(-(-(-tp // 16)) // 2) and per % 8 == 0
        assert splits * per >= units and (splits == 1 or (splits - 1) * per < units)
        need = oc.oc_kv4_decode_workspace_bytes(oc.Layout(1, nq, nkv, d, 16, 16, 8), batch, tp)
        assert need >= (decode_ranges(nq, nkv, d, batch, tp)[1] * nq * (d + 2) * 4 if splits > 1 else 256)


def decode_ranges(nq, nkv, d, batch, most):
    """Ranges wanted (0: no list), ranges at most."""
    lay, out = L.c_layout(1, nq, nkv, d, 16, 16, 1 << 40), (c_int64 * 2)()
    assert oc.lib().oc_internal_kv4_ranges(ctypes.byref(lay), c_int64(batch), c_int64(most), out) == 0
    return tuple(out)


def test_the_ranges_of_a_decode_have_their_workgroups():
    """Whatever the lengths: as many ranges as were planned for at most, every unit in one, and counts that the
    list's fields hold."""
    rng = np.random.default_rng(4)
    lists = 0
    for _ in range(3000):
        nkv = int(rng.integers(1, 17))
        nq, d, batch = nkv * int(rng.integers(1, 20)), int(rng.choice([64, 128])), int(np.exp(rng.uniform(0, 6)))
        most = int(np.exp(rng.uniform(0, 11)))
        wanted, at_most = decode_ranges(nq, nkv, d, batch, most)
        _, m_tiles, _, splits, per = plan(nq, nkv, d, most, 1, batch)
        kind = rng.integers(4)
        lengths = (np.full(batch, most) if kind == 0 else np.exp(rng.uniform(0, np.log(most + 1), batch)).astype(int) - 1
                   if kind == 1 else np.where(rng.random(batch) < 0.1, most, 0) if kind == 2 else rng.integers(-1, most + 1, batch))
        units = -(-(-(-np.maximum(lengths, 0) // 16)) // 2)
        if wanted:
            lists += 1
            # the kernels' own arithmetic, in 32 bits
            per = max(per, (int(np.float32(units.sum()) * (np.float32(1) / np.float32(wanted))) + 8) // 8 * 8)
            assert units.sum() < 1 << 24 and per * wanted >= units.sum() and batch <= 128
            assert (units // per).sum() <= wanted < 1024 and wanted * nkv * m_tiles <= max(256, nkv * m_tiles)
        else:
            assert at_most == batch * splits
        assert np.where(lengths < 0, 0, np.maximum(1, -(-units // per))).sum() <= at_most
    assert lists > 300


def test_which_decodes_make_a_list():
    for args, want in (((32, 8, 128, 1, 30000), 0), ((32, 8, 128, 2, 768), 0), ((32, 8, 128, 2, 769), 32),
                       ((32, 8, 128, 32, 5120), 32), ((32, 8, 128, 33, 5120), 0), ((32, 8, 128, 33, 5121), 32),
                       ((32, 8, 128, 128, 30000), 32), ((32, 8, 128, 129, 30000), 0), ((64, 1, 128, 2, 4000), 128),
                       ((512, 512, 64, 4, 30000), 1), ((8, 1, 128, 128, 1 << 23), 0)):
        assert decode_ranges(*args)[0] == want, args


# ---- refusals ---------------------------------------------------------------

def _table(entries=16, tokens=256, pages=FAKE):
    return L.c_block_table(pages, entries, tokens)


def _ingest(lay, chunks=16, S=None, entries=16, tokens=256, layer=0, data=FAKE, base=FAKE):
    S = 2 * lay.chunk_tokens * lay.num_kv_heads * lay.head_dim * 2 if S is None else S
    st, bt, kp = L.c_staging(data, chunks, S), _table(entries, tokens), L.c_kv_pool(base, lay)
    return oc.lib().oc_kv4_layer_ingest(ctypes.byref(st), ctypes.byref(bt), ctypes.byref(kp), layer, None)


def _gather(lay, chunks=16, entries=16, tokens=256, layer=0, data=FAKE, base=FAKE):
    S = 2 * lay.chunk_tokens * lay.num_kv_heads * lay.head_dim * 2
    bt, kp = _table(entries, tokens), L.c_kv_pool(base, lay)
    return oc.lib().oc_kv4_layer_gather(ctypes.byref(bt), ctypes.byref(kp), layer, data, chunks, S, None)


def _append(lay, n=8, entries=17, tokens=256, layer=0, k=FAKE, v=FAKE, base=FAKE):
    bt, kp = _table(entries, tokens), L.c_kv_pool(base, lay)
    return oc.lib().oc_kv4_suffix_append(k, v, n, ctypes.byref(bt), ctypes.byref(kp), layer, None)


def test_store_refusals():
    lay = _layout()
    for f in (_ingest, _gather):
        assert f(lay, layer=2) == L.OC_ERANGE and f(lay, layer=-1) == L.OC_ERANGE
        assert f(lay, chunks=15) == L.OC_ESHAPE and f(lay, entries=15) == L.OC_ERANGE
        assert f(lay, data=FAKE + 8) == L.OC_EALIGN and f(lay, base=FAKE + 8) == L.OC_EALIGN
        assert f(lay, data=None) == L.OC_EINVAL and f(lay, base=None) == L.OC_EINVAL
        assert f(_layout(head_dim=48)) == L.OC_ESHAPE and b"multiple of 32" in oc.lib().oc_last_error()
        assert f(_layout(page_size=12)) == L.OC_ESHAPE
        assert f(_layout(num_pages=8)) == L.OC_ERANGE
        assert f(lay, chunks=0, entries=0, tokens=0) == L.OC_OK
        big = _layout(num_pages=BIG)
        assert f(big, chunks=1 << 27, entries=BIG, tokens=1 << 31) == L.OC_ERANGE
    assert _ingest(lay, S=1000) == L.OC_ESHAPE
    assert _append(lay, entries=16) == L.OC_ERANGE and _append(lay, n=-1) == L.OC_EINVAL
    assert _append(lay, layer=2) == L.OC_ERANGE and _append(lay, k=None) == L.OC_EINVAL
    assert _append(lay, v=FAKE + 4) == L.OC_EALIGN and _append(lay, n=0) == L.OC_OK
    assert _append(_layout(num_pages=16)) == L.OC_ERANGE
    assert _append(_layout(num_pages=BIG), n=1 << 40, entries=BIG) == L.OC_ERANGE
    assert _append(_layout(num_pages=BIG), n=1 << 62, entries=BIG) == L.OC_ERANGE
    assert oc.lib().oc_kv4_layer_ingest(None, None, None, 0, None) == L.OC_EINVAL
    assert oc.lib().oc_kv4_layer_gather(None, None, 0, None, 0, 0, None) == L.OC_EINVAL
    assert oc.lib().oc_kv4_suffix_append(None, None, 1, None, None, 0, None) == L.OC_EINVAL


def _prefill(lay, q=FAKE, k=FAKE, v=FAKE, ts=8, entries=16, tokens=256, layer=0, out=FAKE, base=FAKE, ws=FAKE, n=1 << 30):
    bt, kp = _table(entries, tokens), L.c_kv_pool(base, lay)
    return oc.lib().oc_kv4_suffix_prefill_layer(q, k, v, ts, ctypes.byref(kp), ctypes.byref(bt), layer, out, ws, n, None)


def test_prefill_refusals():
    lay = _layout()
    assert _prefill(lay, ts=0) == L.OC_EINVAL and _prefill(lay, layer=2) == L.OC_ERANGE
    assert _prefill(lay, entries=15) == L.OC_ERANGE and _prefill(_layout(head_dim=96)) == L.OC_ESHAPE
    assert _prefill(_layout(page_size=32)) == L.OC_ESHAPE
    for name in ("q", "k", "v", "out"):
        assert _prefill(lay, **{name: None}) == L.OC_EINVAL and _prefill(lay, **{name: FAKE + 8}) == L.OC_EALIGN
    assert _prefill(lay, base=None) == L.OC_EINVAL and _prefill(lay, base=FAKE + 8) == L.OC_EALIGN
    assert _prefill(lay, ws=None) == L.OC_EINVAL and _prefill(lay, ws=FAKE + 16) == L.OC_EALIGN
    assert _prefill(lay, n=8) == L.OC_EINVAL and b"too small" in oc.lib().oc_last_error()
    assert _prefill(lay, ts=1 << 30) == L.OC_ERANGE and _prefill(lay, ts=1 << 62) == L.OC_ERANGE


def _decode(lay, batch=3, tables=3, entries=17, stride=20, pages=FAKE, lengths=FAKE, most=256, layer=0, q=FAKE, k=FAKE,
            v=FAKE, out=FAKE, base=FAKE, ws=FAKE, n=1 << 30):
    t, kp = L.c_page_tables(pages, tables, entries, stride), L.c_kv_pool(base, lay)
    return oc.lib().oc_kv4_decode_layer(q, k, v, batch, ctypes.byref(kp), ctypes.byref(t), lengths, most, layer, out, ws,
                                        n, None)


def test_decode_refusals():
    lay = _layout()
    assert _decode(lay, batch=0) == L.OC_OK and _decode(lay, batch=-1) == L.OC_EINVAL
    assert _decode(lay, batch=1 << 17, tables=1 << 17) == L.OC_ERANGE
    assert _decode(lay, tables=2) == L.OC_ERANGE and _decode(lay, entries=16) == L.OC_ERANGE
    assert _decode(lay, stride=16) == L.OC_EINVAL and _decode(lay, most=-1) == L.OC_EINVAL
    assert _decode(lay, most=64 * 16, entries=65, stride=65) == L.OC_ERANGE           # a 65th page
    assert _decode(lay, layer=2) == L.OC_ERANGE and _decode(_layout(head_dim=96)) == L.OC_ESHAPE
    for name in ("q", "k", "v", "out"):
        assert _decode(lay, **{name: None}) == L.OC_EINVAL and _decode(lay, **{name: FAKE + 8}) == L.OC_EALIGN
    for name in ("pages", "lengths", "base", "ws"):
        assert _decode(lay, **{name: None}) == L.OC_EINVAL
    assert _decode(lay, ws=FAKE + 16) == L.OC_EALIGN and _decode(lay, n=8) == L.OC_EINVAL
    kp = L.c_kv_pool(FAKE, lay)
    assert oc.lib().oc_kv4_decode_layer(FAKE, FAKE, FAKE, 1, ctypes.byref(kp), None, FAKE, 8, 0, FAKE, FAKE, 1 << 30,
                                        None) == L.OC_EINVAL


def test_pages_refusals():
    lib, lay = oc.lib(), _layout()
    kp, bt, tabs = L.c_kv_pool(FAKE, lay), _table(), L.c_page_tables(FAKE, 2, 16, 16)
    P, T = ctypes.byref(kp), ctypes.byref(tabs)

    def take(n=4, counts=FAKE, out=FAKE, status=FAKE, layout=lay):
        return lib.oc_kv_pages_take(ctypes.byref(layout), counts, n, out, status, None)
    assert take(n=-1) == L.OC_EINVAL and take(n=65) == L.OC_ERANGE and take(counts=None) == L.OC_EINVAL
    assert take(out=None) == L.OC_EINVAL and take(status=None) == L.OC_EINVAL
    assert take(layout=_layout(num_pages=1 << 31)) == L.OC_ERANGE

    def copy(bits=16, n=4, src=FAKE, dst=FAKE, pool=P):
        return lib.oc_kv_pages_copy(pool, bits, src, dst, n, None)
    assert copy(bits=8) == L.OC_EINVAL and copy(n=-1) == L.OC_EINVAL and copy(n=65) == L.OC_ERANGE
    assert copy(n=0) == L.OC_OK and copy(src=None) == L.OC_EINVAL and copy(dst=None) == L.OC_EINVAL
    assert copy(pool=None) == L.OC_EINVAL
    assert copy(pool=ctypes.byref(L.c_kv_pool(FAKE + 8, lay))) == L.OC_EALIGN
    assert copy(bits=4, pool=ctypes.byref(L.c_kv_pool(FAKE, _layout(head_dim=40)))) == L.OC_ESHAPE

    def fork(tables=T, n=2, table=bt, counts=FAKE, status=FAKE, bits=4):
        return lib.oc_kv_pages_fork(P, bits, ctypes.byref(table), tables, n, counts, status, None)
    assert fork(n=-1) == L.OC_EINVAL and fork(n=3) == L.OC_ERANGE and fork(bits=0) == L.OC_EINVAL
    assert fork(table=_table(17, 257)) == L.OC_ERANGE                       # children of 16 entries
    assert fork(tables=None) == L.OC_EINVAL and fork(counts=None) == L.OC_EINVAL and fork(status=None) == L.OC_EINVAL
    assert fork(tables=ctypes.byref(L.c_page_tables(FAKE, 2, 16, 8))) == L.OC_EINVAL
    assert fork(table=_table(15, 256)) == L.OC_ERANGE

    def release(table=bt, counts=FAKE):
        return lib.oc_kv_pages_release(ctypes.byref(table), ctypes.byref(lay), counts, None)
    assert release(table=_table(15, 256)) == L.OC_ERANGE and release(counts=None) == L.OC_EINVAL
    assert release(table=_table(0, 0, None)) == L.OC_OK
    assert lib.oc_kv_pages_release(ctypes.byref(bt), None, FAKE, None) == L.OC_EINVAL

    def compact(tables=T, counts=FAKE, live=FAKE, ws=FAKE, n=1 << 20, bits=16, pool=P):
        return lib.oc_kv_pages_compact(pool, bits, counts, tables, live, ws, n, None)
    assert compact(tables=None) == L.OC_EINVAL and compact(counts=None) == L.OC_EINVAL
    assert compact(live=None) == L.OC_EINVAL and compact(ws=None) == L.OC_EINVAL and compact(n=64) == L.OC_EINVAL
    assert compact(ws=FAKE + 4) == L.OC_EALIGN and compact(bits=3) == L.OC_EINVAL
    assert compact(tables=ctypes.byref(L.c_page_tables(FAKE, 2, 16, 15))) == L.OC_EINVAL
    assert compact(tables=ctypes.byref(L.c_page_tables(None, 2, 16, 16))) == L.OC_EINVAL
    assert compact(pool=ctypes.byref(L.c_kv_pool(None, lay))) == L.OC_EINVAL


def test_a_fork_refuses_the_parents_table_among_the_childrens():
    lib, lay = oc.lib(), _layout()
    kp, word = L.c_kv_pool(FAKE, lay), 4

    def fork(parent, n, tokens, stride):
        tabs = L.c_page_tables(FAKE, n, 16, stride)
        return lib.oc_kv_pages_fork(ctypes.byref(kp), 16, ctypes.byref(_table(16, tokens, FAKE + word * parent)),
                                    ctypes.byref(tabs), n, FAKE, FAKE, None)
    for n, stride in ((1, 16), (1, 0), (4, 16), (4, 40)):
        for c in range(n):
            for near in (-9, 0, 9):                     # ten entries each
                assert fork(c * stride + near, n, 150, stride) == L.OC_EINVAL, (n, stride, c, near)
                assert b"parent" in lib.oc_last_error()


# ---- marshalling ------------------------------------------------------------

KP, BT, ST, PT, LAY = (POINTER(t) for t in (L.c_kv_pool, L.c_block_table, L.c_staging, L.c_page_tables, L.c_layout))
SIGS = {
    "oc_kv4_layer_ingest": (ST, BT, KP, c_int32, c_void_p),
    "oc_kv4_suffix_append": (c_void_p, c_void_p, c_int64, BT, KP, c_int32, c_void_p),
    "oc_kv4_layer_gather": (BT, KP, c_int32, c_void_p, c_int64, c_int64, c_void_p),
    "oc_kv4_suffix_prefill_layer": (c_void_p, c_void_p, c_void_p, c_int64, KP, BT, c_int32, c_void_p, c_void_p, c_size_t,
                                    c_void_p),
    "oc_kv4_decode_layer": (c_void_p, c_void_p, c_void_p, c_int64, KP, PT, c_void_p, c_int64, c_int32, c_void_p, c_void_p,
                            c_size_t, c_void_p),
    "oc_kv_pages_take": (LAY, c_void_p, c_int64, c_void_p, c_void_p, c_void_p),
    "oc_kv_pages_copy": (KP, c_int32, c_void_p, c_void_p, c_int64, c_void_p),
    "oc_kv_pages_fork": (KP, c_int32, BT, PT, c_int64, c_void_p, c_void_p, c_void_p),
    "oc_kv_pages_release": (BT, LAY, c_void_p, c_void_p),
    "oc_kv_pages_compact": (KP, c_int32, c_void_p, PT, c_void_p, c_void_p, c_size_t, c_void_p),
}


class Tensor:
    def __init__(self, ptr, shape=(1,), stride=None, size=2):
        self.ptr, self.shape, self.steps, self.size = ptr, shape, stride or (1,) * len(shape), size

    def data_ptr(self):
        return self.ptr

    def numel(self):
        return int(np.prod(self.shape))

    def element_size(self):
        return self.size

    def stride(self):
        return self.steps


def plain(v):
    if isinstance(v, ctypes._Pointer):
        return plain(v.contents)
    if isinstance(v, ctypes.Structure):
        return {f[0]: plain(getattr(v, f[0])) for f in v._fields_}
    return v


@pytest.fixture
def calls():
    m = L._native()
    seen, keep = [], []
    for name in L._FAST_KV4:
        keep.append(CFUNCTYPE(c_int, *SIGS[name])(lambda *a, name=name: seen.append((name, [plain(x) for x in a])) or 0))
    m.bind_kv4(*(ctypes.cast(cb, c_void_p).value for cb in keep))
    try:
        yield seen
    finally:
        m.bind_kv4(*(ctypes.cast(getattr(oc.lib(), f), c_void_p).value for f in L._FAST_KV4))


def test_every_argument_arrives(calls):
    lay = oc.Layout(3, 8, 2, 64, 16, 32, 1 << 33)
    lay_c = {"num_layers": 3, "num_q_heads": 8, "num_kv_heads": 2, "head_dim": 64, "page_size": 16, "chunk_tokens": 32,
             "num_pages": 1 << 33}
    kp, bt = {"base": 0x7000, "layout": lay_c}, {"pages": 0x300, "num_entries": 9, "num_tokens": 130}
    pt = {"pages": 0x400, "num_tables": 5, "num_entries": 9, "stride": 12}
    t, pages, pool, tabs = Tensor, Tensor(0x300, (9,)), Tensor(0x7000), Tensor(0x400, (5, 9), (12, 1))
    S = 2 * 32 * 2 * 64 * 2
    oc.oc_kv4_layer_ingest(t(0x10), 4, pages, 130, pool, lay, 2, stream=7)
    oc.oc_kv4_suffix_append(t(0x11), t(0x12), 21, pages, 130, pool, lay, 1, stream=7)
    oc.oc_kv4_layer_gather(pages, 130, pool, lay, 1, t(0x13), 4, stream=7)
    oc.oc_kv4_suffix_prefill_layer(t(0x14), t(0x15), t(0x16), 21, pool, lay, pages, 130, 2, t(0x17),
                                   t(0x18, (100,), size=4), stream=7)
    oc.oc_kv4_decode_layer(t(0x14), t(0x15), t(0x16), 5, pool, lay, tabs, t(0x19), 130, 2, t(0x17), t(0x18, (100,)),
                           stream=7)
    oc.oc_kv_pages_take(t(0x20), lay, 6, t(0x21), t(0x22), stream=7)
    oc.oc_kv_pages_copy(pool, lay, 4, t(0x23), t(0x24), 6, stream=7)
    oc.oc_kv_pages_fork(pool, lay, 16, pages, 130, 5, tabs, t(0x20), t(0x22), stream=7)
    oc.oc_kv_pages_release(pages, 130, lay, t(0x20), stream=7)
    oc.oc_kv_pages_compact(pool, lay, 4, t(0x20), tabs, t(0x25), t(0x18, (100,), size=1), stream=7)
    assert calls == [
        ("oc_kv4_layer_ingest", [{"data": 0x10, "num_chunks": 4, "per_layer_chunk_bytes": S}, bt, kp, 2, 7]),
        ("oc_kv4_suffix_append", [0x11, 0x12, 21, bt, kp, 1, 7]),
        ("oc_kv4_layer_gather", [bt, kp, 1, 0x13, 4, S, 7]),
        ("oc_kv4_suffix_prefill_layer", [0x14, 0x15, 0x16, 21, kp, bt, 2, 0x17, 0x18, 400, 7]),
        ("oc_kv4_decode_layer", [0x14, 0x15, 0x16, 5, kp, pt, 0x19, 130, 2, 0x17, 0x18, 200, 7]),
        ("oc_kv_pages_take", [lay_c, 0x20, 6, 0x21, 0x22, 7]),
        ("oc_kv_pages_copy", [kp, 4, 0x23, 0x24, 6, 7]),
        ("oc_kv_pages_fork", [kp, 16, bt, pt, 5, 0x20, 0x22, 7]),
        ("oc_kv_pages_release", [bt, lay_c, 0x20, 7]),
        ("oc_kv_pages_compact", [kp, 4, 0x20, pt, 0x25, 0x18, 100, 7]),
    ]


def test_tables_must_be_rows(calls):
    lay, pool, t = oc.Layout(3, 8, 2, 64, 16, 32, 64), Tensor(0x7000), Tensor
    for tabs in (Tensor(0x400, (5,), (1,)), Tensor(0x400, (5, 9), (1, 5)), Tensor(0x400, (5, 9, 1), (9, 1, 1))):
        with pytest.raises(ValueError):
            oc.oc_kv_pages_compact(pool, lay, 4, t(0x20), tabs, t(0x25), t(0x18), stream=7)
    with pytest.raises(AttributeError):
        oc.oc_kv_pages_compact(pool, lay, 4, t(0x20), None, t(0x25), t(0x18), stream=7)
    for bad in (1.5, "4", None):
        with pytest.raises(TypeError):
            oc.oc_kv_pages_take(t(0x20), lay, bad, t(0x21), t(0x22), stream=7)
    assert calls == []

"""Limits of the 4-bit attention at their edges, without a GPU."""
import ctypes

import paper_2605_22850_amd as oc
from paper_2605_22850_amd import _lib as L


def test_query_heads_of_a_decode():
    """Row tiles of 32 query heads are a grid's second dimension, of at most 65535."""
    for nq, ok in ((65535 * 32, True), (65535 * 32 + 1, False), (1 << 22, False)):
        lay = oc.Layout(1, nq, 1, 64, 16, 16, 8).c()
        assert (oc.lib().oc_kv4_decode_workspace_bytes(ctypes.byref(lay), 1, 64) > 0) == ok
        if not ok:
            assert b"65535 * 32 query heads" in oc.lib().oc_last_error()


def test_pools_whose_offsets_have_no_64_bit_number():
    """They are refused by every call, like the sizes of such pools: an offset that wrapped would be a place in memory."""
    far = 1 << 20                    # aligned, non-null, never dereferenced
    lib, ref = oc.lib(), ctypes.byref
    S = 2 * 16 * 64 * 2
    lay = L.c_layout(1 << 20, 1, 1, 64, 16, 16, 1 << 40)           # 2^61 pages of 544 bytes
    kp, bt, st = L.c_kv_pool(far, lay), L.c_block_table(far, 4, 32), L.c_staging(far, 2, S)
    tabs = L.c_page_tables(far, 1, 4, 4)
    assert lib.oc_kv4_pool_bytes(ref(lay)) == 0 and b"2^63" in lib.oc_last_error()
    for call in (lambda: lib.oc_kv4_layer_ingest(ref(st), ref(bt), ref(kp), 1 << 19, None),
                 lambda: lib.oc_kv4_suffix_append(far, far, 3, ref(bt), ref(kp), 1 << 19, None),
                 lambda: lib.oc_kv4_layer_gather(ref(bt), ref(kp), 1 << 19, far, 2, S, None),
                 lambda: lib.oc_kv4_suffix_prefill_layer(far, far, far, 3, ref(kp), ref(bt), 1 << 19, far, far, 1 << 30, None),
                 lambda: lib.oc_kv4_decode_layer(far, far, far, 1, ref(kp), ref(tabs), far, 32, 1 << 19, far, far, 1 << 30, None)):
        assert call() == L.OC_ERANGE and b"2^63" in lib.oc_last_error()
    for shape in ((1 << 29, 1, 1, 1 << 20, 16, 16, (1 << 31) - 1), (1, 1 << 30, 1 << 30, 1 << 20, 1 << 20, 16, 64),
                  (1, 1 << 30, 1 << 30, 1 << 30, 8, 16, 64)):
        kp = L.c_kv_pool(far, L.c_layout(*shape))
        for call in (lambda: lib.oc_kv_pages_copy(ref(kp), 16, far, far, 2, None),
                     lambda: lib.oc_kv_pages_fork(ref(kp), 16, ref(bt), ref(tabs), 1, far, far, None),
                     lambda: lib.oc_kv_pages_compact(ref(kp), 16, far, ref(tabs), far, far, 1 << 62, None)):
            assert call() == L.OC_ERANGE and b"2^63" in lib.oc_last_error(), shape

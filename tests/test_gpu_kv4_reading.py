"""Reading a 4-bit pool that holds what no store writes, and two decode calls that append
to one pool at a time."""
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
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16).copy()).cuda().view(torch.bfloat16)
    return torch.from_numpy(a.copy()).cuda()


def host16(t):
    import torch
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


def normal(rng, *shape):
    return ref.f64_to_bf16(rng.standard_normal(shape))


def test_every_code_with_every_scale_byte():
    """Subnormals are kept (b = 0 and 1), what passes bfloat16's range is infinite (b = 254), a zero has its sign,
    and b = 255 is NaN throughout."""
    import torch
    import paper_2605_22850_amd as oc
    T, d = 256, 64                                    # token t has scale byte t in its first block, 255 - t in its second
    pool = ref.Pool4(1, T // 16, 1, 16, d, fill=0)
    codes, scales = pool.views()
    every = np.arange(32) % 16
    packed = np.tile(every[0::2] | every[1::2] << 4, 2).astype(np.uint8)
    for t in range(T):
        codes[0, :, t // 16, 0, t % 16] = packed
        scales[0, :, t // 16, 0, t % 16] = (t, 255 - t)
    out = torch.zeros((T // 16, 2, 16, 1, d), dtype=torch.bfloat16, device="cuda")
    lay = oc.Layout(1, 1, 1, d, 16, 16, T // 16)
    oc.oc_kv4_layer_gather(dev(np.arange(T // 16, dtype=np.int32)), T, dev(pool.raw), lay, 0, out, T // 16)
    got = host16(out)[:, :, :, 0].transpose(1, 0, 2, 3).reshape(2, T, d)
    value = np.where(every >= 8, -1.0, 1.0) * ref.VALUES[every & 7]
    for t in range(T):
        for block, b in ((0, t), (1, 255 - t)):
            here = got[:, t, block * 32:block * 32 + 32]
            if b == 255:
                assert np.isnan(ref.bf16_to_f64(here)).all()
                continue
            x = value * 2.0 ** (b - 127)
            # exact in float64 and, below 2^128, in bfloat16: eight bits above 2^-133
            with np.errstate(over="ignore"):
                want = (x.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
            assert np.array_equal(here, np.broadcast_to(want, here.shape)), b


def test_two_decodes_append_to_one_pool_at_once():
    """Two batches of disjoint tables in one pool, on two streams, each with its workspace: rows, and every byte of
    the pool afterwards."""
    import torch
    import paper_2605_22850_amd as oc
    rng = np.random.default_rng(6)
    nq, nkv, d, most = 32, 8, 128, 3100
    batches = [[3000, 40, -1, 700], [15, 2500, 16, 0, 1111]]
    needs = [[max(n, 0) // 16 + 1 for n in b] for b in batches]
    P = sum(map(sum, needs)) + 2
    lay = oc.Layout(2, nq, nkv, d, 16, 16, P)
    pool, perm, at = ref.Pool4(2, P, nkv, 16, d), rng.permutation(P).astype(np.int32), 0
    calls = []
    for lengths, need in zip(batches, needs):
        B = len(lengths)
        tables = np.full((B, most // 16 + 1), 1 << 30, np.int32)
        for i, n in enumerate(need):
            tables[i, :n] = perm[at:at + n]
            at += n
            if lengths[i] > 0:
                for kv in (0, 1):
                    pool.put(1, kv, tables[i], 0, normal(rng, lengths[i], nkv, d))
        calls.append((lengths, tables, normal(rng, B, nq, d), normal(rng, B, nkv, d), normal(rng, B, nkv, d)))
    d_pool = dev(pool.raw)
    args, outs = [], []
    for lengths, tables, q, k, v in calls:
        ws = torch.full((oc.oc_kv4_decode_workspace_bytes(lay, len(lengths), most),), 0xFF, dtype=torch.uint8, device="cuda")
        outs.append(torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda"))
        args.append((dev(q), dev(k), dev(v), len(lengths), d_pool, lay, dev(tables), dev(np.array(lengths, np.int32)), most, 1,
                     outs[-1], ws))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in args]
    for a, s in zip(args, streams):
        oc.oc_kv4_decode_layer(*a, stream=s)
    torch.cuda.synchronize()
    for (lengths, tables, q, k, v), out in zip(calls, outs):
        got = host16(out)
        for i, n in enumerate(lengths):
            if n < 0:
                continue
            keys, values = (np.concatenate((pool.get(1, kv, tables[i], n), ref.bf16_to_f64(x[i:i + 1]))) for kv, x in ((0, k), (1, v)))
            ref.assert_rows_close(got[i:i + 1], *ref.attention(ref.bf16_to_f64(q[i:i + 1]), keys, values, [n + 1]),
                                  what=f"{n} tokens")
    for lengths, tables, q, k, v in calls:
        for i, n in enumerate(lengths):
            if n >= 0:
                pool.put(1, 0, tables[i], n, k[i:i + 1])
                pool.put(1, 1, tables[i], n, v[i:i + 1])
    assert np.array_equal(d_pool.cpu().numpy(), pool.raw)

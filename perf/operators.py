"""Performance cases of the 4-bit paged cache and of the page operations.

Each case is one call, or a short run of calls, that a serving program makes:
attention of a prompt's new tokens over a prefix held in 4 bits, one new token
for each request of a batch, a layer's prefix stored, extended and read back,
and pages forked or moved together.  `listed()` names the representative ones,
`draw()` gives more of the same ranges.

The 4-bit page holds, for each KV head and slot, head_dim codes (sign,
two exponent bits, one mantissa bit: 0 0.5 1 1.5 2 3 4 6), two to a byte, the
even dimension in the low half, and behind all the heads' codes one scale byte
b for every 32 codes, which stands for 2^(b - 127).  255 says that the 32 are
NaN.  A page's bytes are rounded up to a multiple of 16.
"""
import math

import torch

DEV = "cuda"
PAGE = 16
own = False


def _oc():
    """The framework, loaded only where its kernels are asked for."""
    import paper_2605_22850_amd
    return paper_2605_22850_amd


def listed():
    return [
        # The smallest layer: 256 cached tokens, 32 new ones, launch latency.
        {"name": "attn4_tiny", "kind": "attention", "nq": 4, "nkv": 2, "d": 64, "prefix": 256, "suffix": 32},
        # A prompt found whole in the cache: its last token alone streams the
        # prefix, which ends inside a page.
        {"name": "attn4_full_hit", "kind": "attention", "nq": 32, "nkv": 8, "d": 128, "prefix": 32763, "suffix": 1},
        # An ordinary hit: 4K cached, a short question behind it.
        {"name": "attn4_8b_4k", "kind": "attention", "nq": 32, "nkv": 8, "d": 128, "prefix": 4096, "suffix": 128},
        # The long context, bound by the matrix cores.
        {"name": "attn4_8b_64k", "kind": "attention", "nq": 32, "nkv": 8, "d": 128, "prefix": 65536, "suffix": 512},
        # One token of one short request: launch latency.
        {"name": "decode4_tiny", "kind": "decode", "nq": 4, "nkv": 2, "d": 64, "lengths": "250"},
        # One token each of 32 requests of very different lengths, two of
        # them empty slots of a padded batch, one without a cache yet.
        {"name": "decode4_8b_batch", "kind": "decode", "nq": 32, "nkv": 8, "d": 128,
         "lengths": "22288 11664 12704 11440 4992 6512 28560 8144 17 129 0 4096 1000 2049 -1 16384 777 3333 64 511 "
                    "9000 15 16 1 20000 5120 -1 333 8191 12345 2500 640"},
        # Eight query heads to a KV head, eight long requests.
        {"name": "decode4_70b", "kind": "decode", "nq": 64, "nkv": 8, "d": 128,
         "lengths": "32768 31111 30000 32001 28672 32767 29999 32700"},
        # The smallest layer stored, extended and read back.
        {"name": "store4_tiny", "kind": "store", "nkv": 2, "d": 64, "page": 16, "chunk": 16, "prefix": 256,
         "suffix": 16},
        # A long layer's payload (256 MiB) stored in 4 bits, 512 tokens
        # appended, and all of it read back for write-back.
        {"name": "store4_8b_64k", "kind": "store", "nkv": 8, "d": 128, "page": 16, "chunk": 16, "prefix": 65536,
         "suffix": 512},
        # 16 continuations of one prompt: full pages shared, the partial last
        # page copied for each, all 32 layers.
        {"name": "fork_8b_16", "kind": "fork", "bits": 16, "layers": 32, "nkv": 8, "d": 128, "pages": 512,
         "tokens": 4090, "children": 16},
        # A small pool in 4 bits after requests have ended: few pages move.
        {"name": "compact4_small", "kind": "compact", "bits": 4, "layers": 4, "nkv": 8, "d": 128, "pages": 256,
         "live": 100, "moves": 20, "tables": 4},
        # A pool of 1 GiB in bfloat16, more than half live, 160 pages move.
        {"name": "compact_8b", "kind": "compact", "bits": 16, "layers": 32, "nkv": 8, "d": 128, "pages": 512,
         "live": 300, "moves": 160, "tables": 8},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention"] * 4 + ["decode"] * 3 + ["store"] * 2 + ["fork", "compact"])
    if kind == "attention":
        while True:
            nq, nkv, d = rng.choice([(4, 2, 64), (8, 8, 64), (32, 8, 128), (32, 8, 128), (64, 8, 128), (4, 1, 128),
                                     (32, 4, 64), (6, 2, 128)])
            case = {"kind": kind, "nq": nq, "nkv": nkv, "d": d, "prefix": _log_uniform(rng, 1, 65536),
                    "suffix": _log_uniform(rng, 1, 3584)}
            if work(case)["flops"] <= 4 * 32 * 128 * 512 * 65536:
                return case
    if kind == "decode":
        nq, nkv, d = rng.choice([(4, 2, 64), (32, 8, 128), (32, 8, 128), (64, 8, 128), (32, 4, 64), (5, 1, 128)])
        n = _log_uniform(rng, 1, 64)
        lengths = [_log_uniform(rng, 1, 32768) - 1 for _ in range(n)]
        if n > 2:
            lengths[rng.randrange(1, n)] = -1
        while sum(lengths) > 300000:
            lengths[lengths.index(max(lengths))] //= 2
        return {"kind": kind, "nq": nq, "nkv": nkv, "d": d, "lengths": " ".join(str(x) for x in lengths)}
    if kind == "store":
        nkv, d = rng.choice([(2, 64), (8, 128), (8, 128), (1, 128), (3, 96), (2, 32)])
        page, chunk = rng.choice([(16, 16), (16, 64), (16, 16), (32, 256), (24, 24), (8, 12)])
        return {"kind": kind, "nkv": nkv, "d": d, "page": page, "chunk": chunk,
                "prefix": chunk * max(1, _log_uniform(rng, 64, 65000) // chunk),
                "suffix": chunk * rng.randint(1, max(1, 512 // chunk))}
    bits = rng.choice([16, 4])
    nkv, d = rng.choice([(2, 64), (8, 128), (8, 128), (1, 128)])
    layers = rng.randint(2, 32)
    if kind == "fork":
        pages = rng.randint(160, 512)
        return {"kind": kind, "bits": bits, "layers": layers, "nkv": nkv, "d": d, "pages": pages,
                "tokens": _log_uniform(rng, 16, 16 * (pages // 2)) - rng.randint(0, 15), "children": rng.randint(1, 24)}
    pages = _log_uniform(rng, 64, 512)
    live = rng.randint(pages // 4, (3 * pages) // 4)
    moves = rng.randint(0, min(live, pages - live))
    return {"kind": kind, "bits": bits, "layers": layers, "nkv": nkv, "d": d, "pages": pages, "live": live,
            "moves": min(moves, 160), "tables": rng.randint(1, 12)}


# ---------------------------------------------------------------------------
# the 4-bit page
# ---------------------------------------------------------------------------

def _page4(nkv, page, d):
    """(bytes of the codes, of the scales, of one page of K or V)."""
    codes, scales = nkv * page * d // 2, nkv * page * d // 32
    return codes, scales, (codes + scales + 15) // 16 * 16


def _quantise(x):
    """bfloat16 [..., d] -> codes uint8 [..., d/2] and scale bytes uint8 [..., d/32].

    The scale is the least power of two of which seven cover the block's
    largest magnitude (a magnitude of 6 to 7 scales becomes 6: off by one
    scale, as the rounding between 4 and 6 is), between 2^-125 and 2^125.
    Codes are rounded to nearest, ties to the even code."""
    b = x.float().unflatten(-1, (-1, 32))
    mag = b.abs()
    top = mag.amax(-1, keepdim=True)
    top = torch.where(torch.isnan(mag).any(-1, keepdim=True), torch.full_like(top, math.inf), top)
    bad = torch.isinf(top)
    # exponent of top / 7 rounded up, from the bits of the bfloat16 maximum
    bits = torch.where(bad, torch.zeros_like(top), top).to(torch.bfloat16).view(torch.int16).int()
    scale = (((bits + 31) >> 7) - 2).clamp(2, 252)
    y = torch.ldexp(torch.where(bad, torch.zeros_like(mag), mag), 127 - scale)
    v = torch.where(y < 2, torch.round(y * 2) / 2, torch.where(y < 4, torch.round(y), torch.round(y / 2) * 2))
    v = v.clamp(max=6)
    code = torch.where(v < 2, v * 2, torch.where(v < 4, v + 2, v / 2 + 4)).to(torch.uint8)
    code = code | (torch.signbit(b).to(torch.uint8) << 3)
    code = torch.where(bad, torch.zeros_like(code), code).flatten(-2)
    scale = torch.where(bad, torch.full_like(scale, 255), scale).squeeze(-1).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


_VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _dequantise(codes, scales):
    """The float32 values of codes [..., d/2] with scales [..., d/32]."""
    table = torch.tensor(_VALUES + [-v for v in _VALUES], device=codes.device)
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    v = table[code.long()].unflatten(-1, (-1, 32))
    s = scales.int().unsqueeze(-1)
    return torch.where(s == 255, torch.full_like(v, math.nan), torch.ldexp(v, s - 127)).flatten(-2)


class _Pool4:
    """Views of K's (0) or V's (1) pages of a one-layer pool: codes and scales by page, head, slot."""

    def __init__(self, pool, nkv, page, d, kv):
        c, s, _ = _page4(nkv, page, d)
        self.codes = pool[kv, :, :c].unflatten(1, (nkv, page, d // 2))
        self.scales = pool[kv, :, c:c + s].unflatten(1, (nkv, page, d // 32))

    def write(self, pages, slots, x):
        """x [T][nkv][d] to the slots of the pages."""
        codes, scales = _quantise(x)
        self.codes[pages, :, slots] = codes
        self.scales[pages, :, slots] = scales

    def read(self, pages, slots):
        return _dequantise(self.codes[pages, :, slots], self.scales[pages, :, slots])


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, dtype=torch.bfloat16, device=DEV, generator=g)


def _where(table, first, n, page):
    """Pages and slots of the logical positions first .. first + n - 1."""
    t = torch.arange(first, first + n, device=DEV)
    return table[t // page].long(), t % page


def _random_pool4(g, regions, pages, nkv, page, d):
    """Every slot holds something: random values, quantised, in blocks of bounded memory."""
    c, s, total = _page4(nkv, page, d)
    pool = torch.zeros(regions, pages, total, dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 25) // (nkv * page * d))
    for r in range(regions):
        for p in range(0, pages, step):
            n = min(step, pages - p)
            codes, scales = _quantise(_normal(g, n, nkv, page, d))
            pool[r, p:p + n, :c] = codes.flatten(1)
            pool[r, p:p + n, c:c + s] = scales.flatten(1)
    return pool


def _layout(st, layers, nq, nkv, d, page, chunk, pages):
    if own:
        st["layout"] = _oc().Layout(layers, nq, nkv, d, page, chunk, pages)


def prepare(case, seed):
    g = _gen(seed)
    st = dict(case)
    kind, nkv, d = case["kind"], case["nkv"], case["d"]
    if kind == "attention":
        nq, tp, ts = case["nq"], case["prefix"], case["suffix"]
        need = -(-tp // PAGE)
        st["pool"] = _random_pool4(g, 2, need + max(4, need // 4), nkv, PAGE, d)
        pages = st["pool"].shape[1]
        st["table"] = torch.randperm(pages, device=DEV, generator=g).to(torch.int32)[:need].clone()
        st["q"], st["k"], st["v"] = _normal(g, ts, nq, d), _normal(g, ts, nkv, d), _normal(g, ts, nkv, d)
        st["out"] = torch.empty_like(st["q"])
        _layout(st, 1, nq, nkv, d, PAGE, 16, pages)
        if own:
            n = _oc().oc_kv4_attention_workspace_bytes(st["layout"], tp, ts)
            st["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    elif kind == "decode":
        nq = case["nq"]
        lengths = [int(x) for x in case["lengths"].split()]
        b, most = len(lengths), max(lengths)
        needs = [max(0, x) // PAGE + 1 for x in lengths]
        st["pool"] = _random_pool4(g, 2, sum(needs) + 3, nkv, PAGE, d)
        pages = st["pool"].shape[1]
        perm = torch.randperm(pages, device=DEV, generator=g).to(torch.int32)
        st["tables"] = torch.zeros(b, most // PAGE + 1, dtype=torch.int32, device=DEV)
        at = 0
        for i, n in enumerate(needs):
            st["tables"][i, :n] = perm[at:at + n]
            at += n
        st["host_lengths"], st["most"] = lengths, most
        st["num_tokens"] = torch.tensor(lengths, dtype=torch.int32, device=DEV)
        st["q"], st["k"], st["v"] = _normal(g, b, nq, d), _normal(g, b, nkv, d), _normal(g, b, nkv, d)
        st["out"] = torch.zeros_like(st["q"])
        _layout(st, 1, nq, nkv, d, PAGE, 16, pages)
        if own:
            n = _oc().oc_kv4_decode_workspace_bytes(st["layout"], b, most)
            st["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    elif kind == "store":
        page, chunk, tp, ts = case["page"], case["chunk"], case["prefix"], case["suffix"]
        need = -(-(tp + ts) // page)
        pages = need + max(4, need // 8)
        st["pool"] = torch.zeros(2, pages, _page4(nkv, page, d)[2], dtype=torch.uint8, device=DEV)
        st["table"] = torch.randperm(pages, device=DEV, generator=g).to(torch.int32)[:need].clone()
        st["payload"] = _normal(g, tp // chunk, 2, chunk, nkv, d)
        st["k"], st["v"] = _normal(g, ts, nkv, d), _normal(g, ts, nkv, d)
        st["back"] = torch.empty((tp + ts) // chunk, 2, chunk, nkv, d, dtype=torch.bfloat16, device=DEV)
        _layout(st, 1, nkv, nkv, d, page, chunk, pages)
    else:
        layers, pages = case["layers"], case["pages"]
        page_bytes = _page4(nkv, PAGE, d)[2] if case["bits"] == 4 else nkv * PAGE * d * 2
        # bytes that are moved as they are
        st["pool"] = torch.randint(-2**31, 2**31, (layers * 2, pages, page_bytes // 4), dtype=torch.int32, device=DEV,
                                   generator=g).view(torch.uint8)
        perm = torch.randperm(pages, device=DEV, generator=g).to(torch.int32)
        counts = torch.zeros(pages, dtype=torch.int32, device=DEV)
        if kind == "fork":
            need, n = -(-case["tokens"] // PAGE), case["children"]
            st["table"] = perm[:need].clone()
            # some other requests' pages are taken too
            taken = max(0, min(pages - need - n, pages // 4))
            counts[perm[:need + taken].long()] = 1
            st["children"] = torch.zeros(n, need, dtype=torch.int32, device=DEV)
            st["n_children"], st["status"] = n, torch.zeros(1, dtype=torch.int32, device=DEV)
        else:
            live, moves, n = case["live"], case["moves"], case["tables"]
            low = torch.randperm(live, device=DEV, generator=g)
            high = torch.randperm(pages - live, device=DEV, generator=g) + live
            used = torch.cat((low[moves:], high[:moves]))
            counts[used] = torch.randint(1, 4, (live,), dtype=torch.int32, device=DEV, generator=g)
            pick = torch.randint(0, live, (n, -(-live // n) + 3), device=DEV, generator=g)
            st["tables_before"] = used[pick].to(torch.int32)
            st["tables"] = st["tables_before"].clone()
            st["num_live"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        st["counts_before"], st["counts"] = counts, counts.clone()
        _layout(st, layers, nkv, nkv, d, PAGE, 16, pages)
        if own and kind == "compact":
            n = _oc().oc_kv_pages_workspace_bytes(st["layout"])
            st["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

# Pools that a pass writes are returned as their bytes: a page operation moves
# bytes, and a stored token's codes and scales are defined to the bit.

def run(st):
    return (_own if own else _plain)[st["kind"]](st)


def _plain_attention(st):
    nq, nkv, d, tp, ts = (st[x] for x in ("nq", "nkv", "d", "prefix", "suffix"))
    grp = nq // nkv
    pages, slots = _where(st["table"], 0, tp, PAGE)
    k, v = (torch.cat((_Pool4(st["pool"], nkv, PAGE, d, i).read(pages, slots), new.float())).transpose(0, 1)
            for i, new in enumerate((st["k"], st["v"])))
    k, v = k.contiguous(), v.contiguous()
    # one row for each new token and query head of a KV head's group
    q = st["q"].float().view(ts, nkv, grp, d).transpose(0, 1).reshape(nkv, ts * grp, d)
    s = torch.matmul(q, k.transpose(1, 2)).mul_(1.0 / math.sqrt(d))
    own_part = s.view(nkv, ts, grp, tp + ts)[..., tp:]
    at = torch.arange(ts, device=DEV)
    own_part.masked_fill_((at[None, :] > at[:, None])[None, :, None, :], -math.inf)
    s.sub_(s.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(s, v) / s.sum(-1, keepdim=True)
    return o.view(nkv, ts, grp, d).transpose(0, 1).reshape(ts, nq, d).to(torch.bfloat16)


def _plain_decode(st):
    nq, nkv, d = st["nq"], st["nkv"], st["d"]
    grp = nq // nkv
    rk, rv = (_Pool4(st["pool"], nkv, PAGE, d, r) for r in (0, 1))
    out = st["out"]
    # request by request: padded to the longest, they would read several times as much
    for b, n in enumerate(st["host_lengths"]):
        if n < 0:
            continue
        pages, slots = _where(st["tables"][b], 0, n, PAGE)
        k = torch.cat((rk.read(pages, slots), st["k"][b:b + 1].float())).transpose(0, 1)
        v = torch.cat((rv.read(pages, slots), st["v"][b:b + 1].float())).transpose(0, 1)
        q = st["q"][b].float().view(nkv, grp, d)
        s = torch.matmul(q, k.transpose(1, 2)) * (1.0 / math.sqrt(d))
        p = (s - s.amax(-1, keepdim=True)).exp()
        out[b] = (torch.matmul(p, v) / p.sum(-1, keepdim=True)).view(nq, d).to(out.dtype)
        pages, slots = _where(st["tables"][b], n, 1, PAGE)
        rk.write(pages, slots, st["k"][b:b + 1])
        rv.write(pages, slots, st["v"][b:b + 1])
    return out, st["pool"]


def _plain_store(st):
    nkv, d, page, chunk, tp, ts = (st[x] for x in ("nkv", "d", "page", "chunk", "prefix", "suffix"))
    for r, new in ((0, st["k"]), (1, st["v"])):
        pool = _Pool4(st["pool"], nkv, page, d, r)
        pages, slots = _where(st["table"], 0, tp, page)
        pool.write(pages, slots, st["payload"][:, r].reshape(tp, nkv, d))
        pages, slots = _where(st["table"], tp, ts, page)
        pool.write(pages, slots, new)
        pages, slots = _where(st["table"], 0, tp + ts, page)
        st["back"][:, r] = pool.read(pages, slots).to(torch.bfloat16).view(-1, chunk, nkv, d)
    return st["back"]


def _plain_fork(st):
    st["counts"].copy_(st["counts_before"])
    counts, table, n, children = st["counts"], st["table"].long(), st["n_children"], st["children"]
    full = st["tokens"] // PAGE
    children[:, :full] = st["table"][:full]
    counts[table[:full]] += n
    st["status"].zero_()
    if st["tokens"] % PAGE:
        fresh = torch.nonzero(counts <= 0).squeeze(1)[:n]
        children[:, full] = fresh.to(torch.int32)
        counts[fresh] = 1
        st["pool"][:, fresh] = st["pool"][:, table[full]].unsqueeze(1)
    return children, counts, st["status"], st["pool"]


def _plain_compact(st):
    st["counts"].copy_(st["counts_before"])
    st["tables"].copy_(st["tables_before"])
    counts, tables = st["counts"], st["tables"]
    live = counts > 0
    st["num_live"].copy_(live.sum())
    at = torch.arange(counts.shape[0], device=DEV)
    low = at < st["num_live"]
    src, dst = torch.nonzero(live & ~low).squeeze(1), torch.nonzero(~live & low).squeeze(1)
    to = at.to(torch.int32)
    to[src] = dst.to(torch.int32)
    st["pool"][:, dst] = st["pool"][:, src]
    counts[dst] = counts[src]
    counts[src] = 0
    tables.copy_(to[tables.long()])
    return tables, counts, st["num_live"], st["pool"]


def _own_attention(st):
    _oc().oc_kv4_suffix_prefill_layer(st["q"], st["k"], st["v"], st["suffix"], st["pool"], st["layout"], st["table"],
                                      st["prefix"], 0, st["out"], st["workspace"])
    return st["out"]


def _own_decode(st):
    _oc().oc_kv4_decode_layer(st["q"], st["k"], st["v"], len(st["host_lengths"]), st["pool"], st["layout"],
                              st["tables"], st["num_tokens"], st["most"], 0, st["out"], st["workspace"])
    return st["out"], st["pool"]


def _own_store(st):
    oc, lay, tp, ts = _oc(), st["layout"], st["prefix"], st["suffix"]
    oc.oc_kv4_layer_ingest(st["payload"], tp // st["chunk"], st["table"], tp, st["pool"], lay, 0)
    oc.oc_kv4_suffix_append(st["k"], st["v"], ts, st["table"], tp, st["pool"], lay, 0)
    oc.oc_kv4_layer_gather(st["table"], tp + ts, st["pool"], lay, 0, st["back"], (tp + ts) // st["chunk"])
    return st["back"]


def _own_fork(st):
    st["counts"].copy_(st["counts_before"])
    _oc().oc_kv_pages_fork(st["pool"], st["layout"], st["bits"], st["table"], st["tokens"], st["n_children"],
                           st["children"], st["counts"], st["status"])
    return st["children"], st["counts"], st["status"], st["pool"]


def _own_compact(st):
    st["counts"].copy_(st["counts_before"])
    st["tables"].copy_(st["tables_before"])
    _oc().oc_kv_pages_compact(st["pool"], st["layout"], st["bits"], st["counts"], st["tables"], st["num_live"],
                              st["workspace"])
    return st["tables"], st["counts"], st["num_live"], st["pool"]


_plain = {"attention": _plain_attention, "decode": _plain_decode, "store": _plain_store, "fork": _plain_fork,
          "compact": _plain_compact}
_own = {"attention": _own_attention, "decode": _own_decode, "store": _own_store, "fork": _own_fork,
        "compact": _own_compact}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    kind, nkv, d = case["kind"], case["nkv"], case["d"]
    token4 = 2 * nkv * (d // 2 + d // 32)                 # K and V of one token in 4 bits, one layer
    token16 = 2 * nkv * d * 2
    if kind == "attention":
        nq, tp, ts = case["nq"], case["prefix"], case["suffix"]
        pairs = ts * tp + ts * (ts + 1) // 2
        return {"bytes": tp * token4 + ts * (token16 + 2 * nq * d * 2) + -(-tp // PAGE) * 4,
                "flops": 4 * nq * d * pairs}
    if kind == "decode":
        nq, lengths = case["nq"], [int(x) for x in case["lengths"].split() if int(x) >= 0]
        n = len(lengths)
        return {"bytes": sum(lengths) * token4 + n * (token16 + token4 + 2 * nq * d * 2),
                "flops": 4 * nq * d * (sum(lengths) + n)}
    if kind == "store":
        n = case["prefix"] + case["suffix"]
        return {"bytes": n * (2 * token16 + 2 * token4), "flops": 3 * n * 2 * nkv * d}
    page = case["layers"] * 2 * (_page4(nkv, PAGE, d)[2] if case["bits"] == 4 else nkv * PAGE * d * 2)
    if kind == "fork":
        need, n = -(-case["tokens"] // PAGE), case["children"]
        copies = n + 1 if case["tokens"] % PAGE else 0
        return {"bytes": copies * page + (n + 1) * need * 4 + 3 * case["pages"] * 4, "flops": 0}
    entries = case["tables"] * (-(-case["live"] // case["tables"]) + 3)
    return {"bytes": 2 * case["moves"] * page + 4 * entries * 4 + 4 * case["pages"] * 4, "flops": 0}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_values(raw, nkv, page, d, ids, slots, head):
    """float64 [T][d]: the values at these slots of one head, from a region's bytes [P][page bytes]."""
    flat = raw.reshape(-1).long()
    row = ids * raw.shape[1] + (head * page + slots) * (d // 2)
    at = torch.arange(d, device=raw.device)
    byte = flat[row[:, None] + at // 2]
    code = torch.where(at % 2 == 0, byte % 16, byte // 16)
    exponent, half = (code // 2) % 4, (code % 2).double()
    # exponent 0 is the subnormal step 0, 0.5; the others are (1 + m/2) 2^(e-1)
    mag = torch.where(exponent == 0, half / 2, (1 + half / 2) * 2.0 ** (exponent - 1).double())
    first = ids * raw.shape[1] + nkv * page * d // 2 + (head * page + slots) * (d // 32)
    b = flat[first[:, None] + at // 32]
    v = mag * torch.pow(2.0, (b - 127).double()) * torch.where(code >= 8, -1.0, 1.0).double()
    return torch.where(b == 255, torch.full_like(v, math.nan), v)


def _exact_bytes(x):
    """Codes [..., d/2] and scale bytes [..., d/32] of finite or non-finite float64 x, by search over the values."""
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    size = blocks.abs()
    finite = torch.isfinite(blocks).all(-1)
    top = torch.where(finite, size.nan_to_num(0, 0, 0).amax(-1), torch.zeros_like(finite, dtype=torch.float64))
    e = torch.full_like(top, -125)
    _, up = torch.frexp(top / 7)                            # top / 7 < 2^up, and >= 2^(up - 1)
    up = up.double()
    fits = top <= 7 * torch.pow(2.0, up - 1)
    e = torch.where(top > 0, torch.where(fits, up - 1, up), e).clamp(-125, 125)
    y = torch.where(finite[..., None], size, torch.zeros_like(size)) / torch.pow(2.0, e)[..., None]
    code = torch.zeros_like(y, dtype=torch.uint8)
    # halfway points; an even code keeps its upper halfway point
    for i, (mid, upper_even) in enumerate(((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False),
                                           (3.5, True), (5.0, False))):
        code = torch.where((y >= mid) if upper_even else (y > mid), torch.full_like(code, i + 1), code)
    code = code + torch.signbit(blocks).to(torch.uint8) * 8
    code = torch.where(finite[..., None], code, torch.zeros_like(code)).reshape(*x.shape[:-1], -1, 2)
    scale = torch.where(finite, e + 127, torch.full_like(e, 255)).to(torch.uint8)
    return code[..., 0] + 16 * code[..., 1], scale


def _exact_softmax_rows(q, k, v, seen):
    s = q @ k.T / math.sqrt(q.shape[1])
    s = torch.where(torch.arange(k.shape[0], device=q.device)[None] < seen[:, None], s, -math.inf)
    return torch.softmax(s, 1) @ v


def exact(case, seed):
    st = prepare(case, seed)
    kind, nkv, d = case["kind"], case["nkv"], case["d"]
    pos = lambda n, first=0: torch.arange(first, first + n, device=DEV)
    if kind == "attention":
        nq, tp, ts = case["nq"], case["prefix"], case["suffix"]
        per = nq // nkv
        t = pos(tp)
        ids, slots = st["table"].long()[t // PAGE], t % PAGE
        out = torch.empty(ts, nq, d, dtype=torch.float64, device=DEV)
        for h in range(nq):
            if h % per == 0:
                k, v = (torch.cat((_exact_values(st["pool"][r], nkv, PAGE, d, ids, slots, h // per),
                                   (st["k"], st["v"])[r][:, h // per].double())) for r in (0, 1))
            for i in range(0, ts, 256):
                rows = pos(min(256, ts - i), i)
                out[rows, h] = _exact_softmax_rows(st["q"][rows, h].double(), k, v, rows + tp + 1)
        return out
    if kind == "decode":
        nq, per = case["nq"], case["nq"] // nkv
        out = st["out"].double()
        pool = st["pool"].clone()
        c = nkv * PAGE * d // 2
        for b, n in enumerate(st["host_lengths"]):
            if n < 0:
                continue
            t = pos(n)
            ids, slots = st["tables"][b].long()[t // PAGE], t % PAGE
            for g in range(nkv):
                k, v = (torch.cat((_exact_values(st["pool"][r], nkv, PAGE, d, ids, slots, g),
                                   (st["k"], st["v"])[r][b, g][None].double())) for r in (0, 1))
                out[b, g * per:(g + 1) * per] = _exact_softmax_rows(st["q"][b, g * per:(g + 1) * per].double(), k, v,
                                                                    torch.full((per,), n + 1, device=DEV))
                page, slot = int(st["tables"][b, n // PAGE]), n % PAGE
                for r in (0, 1):
                    codes, scales = _exact_bytes((st["k"], st["v"])[r][b, g].double())
                    i = (g * PAGE + slot) * (d // 2)
                    pool[r, page, i:i + d // 2] = codes
                    i = c + (g * PAGE + slot) * (d // 32)
                    pool[r, page, i:i + d // 32] = scales
        return out, pool
    if kind == "store":
        tokens = case["prefix"] + case["suffix"]
        back = torch.empty(2, tokens, nkv, d, dtype=torch.float64, device=DEV)
        for r in (0, 1):
            x = torch.cat((st["payload"][:, r].reshape(-1, nkv, d), (st["k"], st["v"])[r]))
            for i in range(0, tokens, 8192):
                codes, scales = _exact_bytes(x[i:i + 8192].double())
                n = codes.shape[0]
                raw = torch.cat((codes.reshape(n, -1), scales.reshape(n, -1)), 1)       # pages of one slot
                for h in range(nkv):
                    back[r, i:i + n, h] = _exact_values(raw, nkv, 1, d, pos(n), 0 * pos(n), h)
        return back.view(2, -1, case["chunk"], nkv, d).transpose(0, 1).contiguous()
    counts = st["counts_before"].tolist()
    pool = st["pool"].clone()
    if kind == "fork":
        table, full, part = st["table"].tolist(), case["tokens"] // PAGE, case["tokens"] % PAGE
        kids = []
        for _ in range(case["children"]):
            kid = table[:full]
            for p in kid:
                counts[p] += 1
            if part:
                p = next(i for i, n in enumerate(counts) if n == 0)
                counts[p] = 1
                pool[:, p] = pool[:, table[full]]
                kid.append(p)
            kids.append(kid)
        return (torch.tensor(kids, dtype=torch.int32, device=DEV), torch.tensor(counts, dtype=torch.int32, device=DEV),
                torch.zeros(1, dtype=torch.int32, device=DEV), pool)
    live = sum(n > 0 for n in counts)
    moved, hole = {}, 0
    for p in range(live, len(counts)):
        if counts[p] > 0:
            while counts[hole] > 0:
                hole += 1
            pool[:, hole] = pool[:, p]
            counts[hole], counts[p] = counts[p], 0
            moved[p] = hole
    tables = [[moved.get(p, p) for p in row] for row in st["tables_before"].tolist()]
    return (torch.tensor(tables, dtype=torch.int32, device=DEV), torch.tensor(counts, dtype=torch.int32, device=DEV),
            torch.tensor([live], dtype=torch.int32, device=DEV), pool)

"""Plain reference of the 4-bit paged cache and of the page operations, in
numpy and float64, from the definitions in include/objectcache.h."""
import numpy as np

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def bf16_to_f64(u):
    return (np.asarray(u, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def f64_to_bf16(x):
    """Nearest bfloat16, ties to even, of finite values within its range."""
    b = np.asarray(x, np.float32).view(np.uint32)
    return ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)


def encode(u):
    """bfloat16 bits [..., d] -> (codes uint8 [..., d], scale bytes uint8 [..., d/32])."""
    x = bf16_to_f64(u).reshape(*np.shape(u)[:-1], -1, 32)
    finite = np.isfinite(x).all(-1)
    a = np.where(finite[..., None], np.abs(x), 0.0)
    top = a.max(-1)
    # the least exponent of -125..125 with top <= 7 * 2^e (the last one where none is)
    exps = np.arange(-125, 126)
    e = exps[np.minimum((top[..., None] > 7 * 2.0 ** exps).sum(-1), len(exps) - 1)]
    y = a / 2.0 ** e[..., None]
    near = np.abs(y[..., None] - VALUES)
    least = near.min(-1, keepdims=True)
    code = np.where(near == least, np.arange(8), 99)
    # of two equally near codes, the even one
    code = np.where((near == least).sum(-1) > 1, np.where(code % 2 == 0, code, 99).min(-1), code.min(-1))
    sign = (np.asarray(u, np.uint16) >> 15).reshape(x.shape).astype(np.int64)
    code = np.where(finite[..., None], code + 8 * sign, 0)
    return code.reshape(np.shape(u)).astype(np.uint8), np.where(finite, e + 127, 255).astype(np.uint8)


def decode(code, scale):
    """float64 values of codes [..., d] with scale bytes [..., d/32]."""
    v = np.where(code >= 8, -1.0, 1.0) * VALUES[code & 7]
    s = np.repeat(scale.astype(np.int64), 32, -1)
    return np.where(s == 255, np.nan, v * 2.0 ** (s - 127))


class Pool4:
    """A 4-bit pool [L][2][P][page bytes] in host memory."""

    def __init__(self, layers, pages, nkv, ps, d, fill=0xFF):
        self.nkv, self.ps, self.d = nkv, ps, d
        self.code_bytes = nkv * ps * d // 2
        self.page_bytes = -(-(self.code_bytes + nkv * ps * d // 32) // 16) * 16
        self.raw = np.full((layers, 2, pages, self.page_bytes), fill, np.uint8)

    def views(self):
        c = self.raw[..., :self.code_bytes].reshape(*self.raw.shape[:3], self.nkv, self.ps, self.d // 2)
        s = self.raw[..., self.code_bytes:self.code_bytes + self.nkv * self.ps * self.d // 32]
        return c, s.reshape(*self.raw.shape[:3], self.nkv, self.ps, self.d // 32)

    def put(self, layer, kv, table, first, rows):
        """rows: bfloat16 bits [T][nkv][d] at the logical positions from `first` on."""
        if not rows.size:
            return
        code, scale = encode(rows)
        t = first + np.arange(rows.shape[0])
        page, slot = np.asarray(table)[t // self.ps], t % self.ps
        raw = self.raw[layer, kv]
        for h in range(self.nkv):
            for i in range(self.d // 2):
                raw[page, (h * self.ps + slot) * (self.d // 2) + i] = code[:, h, 2 * i] | code[:, h, 2 * i + 1] << 4
            for i in range(self.d // 32):
                raw[page, self.code_bytes + (h * self.ps + slot) * (self.d // 32) + i] = scale[:, h, i]

    def get(self, layer, kv, table, tokens):
        """float64 [tokens][nkv][d]."""
        c, s = self.views()
        t = np.arange(tokens)
        page, slot = np.asarray(table)[t // self.ps], t % self.ps
        packed = c[layer, kv][page, :, slot]
        code = np.stack((packed & 15, packed >> 4), -1).reshape(tokens, self.nkv, self.d)
        return decode(code, s[layer, kv][page, :, slot])


def attention(q, k, v, seen):
    """(out, sum of p |v|) in float64: q [T][nq][d], k and v [S][nkv][d]; row i sees the first seen[i] keys."""
    T, nq, d = q.shape
    per = nq // k.shape[1]
    out, mag = np.empty(q.shape), np.empty(q.shape)
    for h in range(nq):
        for i in range(T):
            kk, vv = k[:seen[i], h // per], v[:seen[i], h // per]
            s = kk @ q[i, h] / np.sqrt(d)
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h], mag[i, h] = p @ vv, p @ np.abs(vv)
    return out, mag


def assert_rows_close(got_u16, out, mag, what=""):
    """got: bfloat16 bits.  Each P is rounded to bfloat16 (half a step, 2^-8 of it), in the sum and in
    the normaliser, and so is the result: 3 * 2^-8 of sum p|v| at most.  In fp32, for rows of normal values:
    the |q k| / sqrt(d) of a score sum to less than 2^4, so its d <= 2^7 products are off by 2^-24 * 2^7 * 2^4
    = 2^-13 at most, and with it each P, in the sum and in the normaliser: 2^-12 of sum p|v|."""
    got = bf16_to_f64(got_u16)
    err, tol = np.abs(got - out), (3 * 2.0 ** -8 + 2.0 ** -12) * mag + 1e-30
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(err / tol):.2f} of the tolerance"


# ---- pages --------------------------------------------------------------------

def take(counts, n):
    """(status, pages): the n lowest free pages, counted."""
    free = [i for i, c in enumerate(counts) if c <= 0][:n]
    if len(free) < n:
        return -7, [-1] * n
    for p in free:
        counts[p] = 1
    return 0, free


def fork(pool, counts, table, tokens, ps, n):
    """(status, child tables); pool [regions][P][bytes] and counts are changed in place."""
    full = tokens // ps
    status, fresh = take(counts, n) if tokens % ps and n else (0, [])
    if status:
        return status, [[None] * full + [-1]] * n
    for p in table[:full]:
        counts[p] += n
    for p in fresh:
        pool[:, p] = pool[:, table[full]]
    return 0, [list(table[:full]) + fresh[i:i + 1] for i in range(n)]


def compact(pool, counts, tables):
    live = sum(c > 0 for c in counts)
    src = [p for p in range(live, len(counts)) if counts[p] > 0]
    dst = [p for p in range(live) if counts[p] <= 0]
    to = dict(zip(src, dst))
    for s, d in to.items():
        pool[:, d] = pool[:, s]
        counts[d], counts[s] = counts[s], 0
    tables[:] = np.vectorize(lambda p: to.get(p, p))(tables) if tables.size else tables
    return live

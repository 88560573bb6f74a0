"""The rotary embedding and the 8-bit cache from their definitions, in float64 (test infrastructure; nothing of the library in it)."""
import numpy as np
import torch

# the values of the 256 e4m3 codes: four exponent bits (bias 7), three of fraction, all ones is NaN
_c = np.arange(128)
_e, _f = _c >> 3, _c & 7
_pos = np.where(_e == 0, _f / 8.0 * 2.0 ** -6, (1 + _f / 8.0) * 2.0 ** (_e - 7.0))
_pos[127] = np.nan
VALUES = np.concatenate([_pos, -_pos])


def scale_value(byte):
    byte = np.asarray(byte).astype(np.int64)
    return np.where(byte == 255, np.nan, 2.0 ** (byte - 127.0))


def values(codes, scale_bytes):
    return VALUES[codes] * scale_value(scale_bytes)[..., None]


def quantise(x):
    """(codes, scale bytes) of the rows of x (float64, last dimension)."""
    mag = np.where(np.isfinite(x), np.abs(x), 0.0)
    top = mag.max(-1)
    e = np.full(top.shape, -126, dtype=np.int64)
    for k in range(-126, 128):                         # the smallest power that leaves the largest at 448 or less
        e = np.where((top > 448.0 * 2.0 ** k), k + 1, e)
    e = np.where(top == 0, 0, e)
    y = np.where(np.isfinite(x), x, 0.0) / (2.0 ** e.astype(np.float64))[..., None]
    grid = VALUES[:127]
    hi = np.clip(np.searchsorted(grid, np.abs(y)), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = np.abs(y) - grid[lo], grid[hi] - np.abs(y)
    code = np.where(dl < dh, lo, np.where(dl > dh, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(np.signbit(x), code + 128, code)
    return np.where(np.isfinite(x), code, 127).astype(np.uint8), (e + 127).astype(np.uint8)


def depths(parent):
    out = []
    for i in range(len(parent)):
        n, cur = -1, i
        while cur >= 0:
            n, cur = n + 1, int(parent[cur])
        out.append(n)
    return np.asarray(out)


def rotate(x, pos, freqs, interleaved, amplitude=1.0):
    """x [n, H, D] at positions pos [n]; returns (rotated, |a| + |b| of each column's pair: what errors scale with)."""
    R = 2 * len(freqs)
    x = x.astype(np.float64)
    angle = pos.astype(np.longdouble)[:, None] * freqs.astype(np.longdouble)
    turn = 2 * np.arctan2(np.longdouble(0), np.longdouble(-1))
    angle = (angle - np.rint(angle / turn) * turn).astype(np.float64)
    c, s = np.cos(angle)[:, None] * amplitude, np.sin(angle)[:, None] * amplitude
    ia, ib = (np.arange(0, R, 2), np.arange(1, R, 2)) if interleaved else (np.arange(R // 2), np.arange(R // 2, R))
    out, size = x.copy(), np.zeros_like(x)
    a, b = x[..., ia], x[..., ib]
    out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
    size[..., ia] = size[..., ib] = (np.abs(a) + np.abs(b)) * amplitude
    return out, size


def attention(q, K, V, seen, scale):
    """q [r, D], K and V [n, D], seen [r, n]: (out, lse, sum of p |v|), float64."""
    s = q @ K.T * scale
    s = np.where(seen, s, -np.inf)
    m = s.max(-1, keepdims=True)
    p = np.exp(s - m)
    z = p.sum(-1, keepdims=True)
    return p @ V / z, (m + np.log(z))[:, 0], p @ np.abs(V) / z


class Cache:
    """An 8-bit cache on the GPU with its page table, codes and scales drawn at random; `shape` orders of the dimensions in memory."""

    def __init__(self, B, lens, T, Hkv, D, ps, seed=0, paged=True, order="phsd", pad=0, decoys=3, fill=None):
        rng = np.random.default_rng(seed)
        total = np.asarray(lens, dtype=np.int64) + T
        if paged:
            n = -(-total // ps)
            ids = rng.permutation(int(n.sum()) + decoys).astype(np.int32)
            self.table = np.zeros((B, max(1, int(n.max()))), dtype=np.int32)
            at = 0
            for b in range(B):
                self.table[b, :n[b]] = ids[at:at + n[b]]
                at += int(n[b])
            pages = len(ids)
        else:
            self.table, pages, ps = None, B, int(total.max())
        self.ps, self.Hkv, self.D, self.lens, self.T = ps, Hkv, D, np.asarray(lens, dtype=np.int32), T
        self.shape = (pages, Hkv, ps, D)
        dims = dict(p=pages, h=Hkv, s=ps, d=D)

        def put(host, letters, extra):
            # memory in the order `letters`, seen as [page, head, slot(, column)]
            sizes = [dims[c] for c in letters]
            if extra:
                sizes[-1] += extra
            mem = torch.zeros(sizes, dtype=torch.uint8, device="cuda")
            if extra:
                mem = mem[..., :sizes[-1] - extra]
            seen = mem.permute([letters.index(c) for c in "phsd" if c in letters])
            seen.copy_(torch.from_numpy(host))
            return seen

        def draw():
            x = rng.standard_normal(self.shape) * np.exp(0.5 * rng.standard_normal(self.shape[:3]))[..., None]
            return quantise(x.astype(np.float32).astype(np.float64))

        if fill is None:
            (self.kc0, self.ks0), (self.vc0, self.vs0) = draw(), draw()
        else:
            self.kc0 = np.full(self.shape, fill, dtype=np.uint8)
            self.ks0 = np.full(self.shape[:3], 127, dtype=np.uint8)
            self.vc0, self.vs0 = self.kc0.copy(), self.ks0.copy()
        self._put, self._order, self._pad = put, order, pad
        self.up()

    def up(self):
        """The host's codes and scales to the GPU."""
        so = self._order.replace("d", "")
        self.kc, self.vc = (self._put(x, self._order, self._pad).view(torch.float8_e4m3fn) for x in (self.kc0, self.vc0))
        self.ks, self.vs = (self._put(x, so, 0).view(torch.float8_e8m0fnu) for x in (self.ks0, self.vs0))
        self.dev_table = None if self.table is None else torch.from_numpy(self.table).cuda()
        self.dev_lens = torch.from_numpy(self.lens).cuda()

    @property
    def args(self):
        return self.kc, self.vc, self.ks, self.vs, self.dev_table

    def place(self, b, pos):
        return (b, pos) if self.table is None else (int(self.table[b, pos // self.ps]), pos % self.ps)

    def host(self):
        """(K codes, K scales, V codes, V scales) as they are on the GPU now."""
        return [x.view(torch.uint8).cpu().numpy() for x in (self.kc, self.ks, self.vc, self.vs)]

    def logical(self, b, n, which=None):
        """K and V values of positions 0 .. n-1 of request b: [n, Hkv, D]."""
        kc, ks, vc, vs = which or (self.kc0, self.ks0, self.vc0, self.vs0)
        at = [self.place(b, i) for i in range(n)]
        pg, sl = np.asarray([a[0] for a in at], dtype=np.int64), np.asarray([a[1] for a in at], dtype=np.int64)
        return values(kc[pg, :, sl], ks[pg, :, sl]), values(vc[pg, :, sl], vs[pg, :, sl])


def seen_matrix(T, L, parent, start=0):
    s = np.zeros((T, L + T), dtype=bool)
    s[:, start:L] = True
    for i in range(T):
        cur = i
        while cur >= 0:
            s[i, L + cur] = True
            cur = int(parent[cur])
    return s


def expect_fwd(cache, q, parents, scale=None, starts=None, q_off=0):
    """(out, lse, size) of tree attention over the cache; q [B, Tq, Hq, D] float64, parents [B, T]."""
    B, Tq, Hq, D = q.shape
    G, T = Hq // cache.Hkv, cache.T
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    out, size, lse = np.zeros((B, Tq, Hq, D)), np.zeros((B, Tq, Hq, D)), np.zeros((B, Hq, Tq))
    for b in range(B):
        L = int(cache.lens[b])
        K, V = cache.logical(b, L + T)
        seen = seen_matrix(T, L, parents[b], 0 if starts is None else int(starts[b]))[q_off:q_off + Tq]
        for h in range(Hq):
            out[b, :, h], lse[b, h], size[b, :, h] = attention(q[b, :, h], K[:, h // G], V[:, h // G], seen, scale)
    return out, lse, size


def bound_fwd(out, size, bf16):
    """How far an output may be off.  bf16: the probabilities are rounded (2^-8 of each, so 2^-8 of sum p |v|), so is the output
    (2^-8 of it), and partial results are held to 2^-16 of their row's largest value, of which a few add up.  Scores are sums of D
    products in fp32, off by at most D 2^-24 sum |q k| scale, here below 1e-4, and so are the probabilities relative to themselves."""
    if bf16:
        return (2.0 ** -8 + 1e-4) * size + 2.0 ** -8 * np.abs(out) + 2.0 ** -14 * size.max(-1, keepdims=True)
    return 1e-4 * size

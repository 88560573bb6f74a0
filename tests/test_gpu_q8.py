"""GPU tests of the rotary embedding and the 8-bit cache against their definitions in float64."""
import numpy as np
import pytest
import torch

from tests import q8_reference as ref
from paper_2508_08192_amd import treeattn as ta
from paper_2508_08192_amd import workloads as W

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _say(*a):
    print(*a, flush=True)


def _rows(rng, shape, dtype, spread=0.0):
    x = rng.standard_normal(shape)
    if spread:
        x = x * np.exp(spread * rng.standard_normal(shape[:-1]))[..., None]
    t = torch.from_numpy(x.astype(np.float32)).to(DT[dtype]).cuda()
    return t, t.double().cpu().numpy()


def _freqs(R, base=10000.0):
    f = np.asarray(ta.tree_attn_rope_freqs(R, base)[0], dtype=np.float32)
    return torch.from_numpy(f).cuda(), f


def _trees(kind, B, T, rng):
    """(what the call gets, parents [B, T] or None)"""
    if kind == "line":
        return None, np.stack([W.chain_tree(T)] * B)
    if kind == "static":
        p = W.bfs_tree(T, [3, 2], 30)
        return torch.from_numpy(p).cuda(), np.stack([p] * B)
    p = np.stack([W.shuffle_tree(W.random_tree(T, 12, rng), rng)[0] for _ in range(B)])
    return torch.from_numpy(p).cuda(), p


def _assert_turned(got, x, pos, f, interleaved, dtype, amplitude=1.0, what=""):
    want, size = ref.rotate(x.reshape(-1, *x.shape[2:]), pos.reshape(-1), f, interleaved, amplitude)
    got = got.double().cpu().numpy().reshape(want.shape)
    # products and sums in fp32 and a sine and cosine good to two units of it: 2^-21 of the pair (positions past 2^30 cost the 64-bit
    # angle as much again), and one rounding to the row's type
    tol = 2.0 ** -20 * size + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want)
    R = 2 * len(f)
    assert np.array_equal(got[..., R:], want[..., R:]), what
    assert (np.abs(got - want) <= tol).all(), (what, np.abs(got - want).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,T,Hq,Hkv,D,R,tree", [
    (1, 1, 8, 1, 128, 128, "line"), (3, 8, 5, 1, 128, 64, "random"), (2, 64, 4, 2, 64, 64, "random"), (2, 45, 7, 1, 80, 32, "static"),
    (2, 17, 3, 3, 96, 96, "random"), (1, 700, 12, 3, 128, 128, "line"), (2, 9, 2, 2, 37, 18, "random"), (3, 5, 2, 1, 250, 250, "random"),
    (2, 33, 2, 1, 256, 256, "line"), (5, 2, 1, 1, 16, 16, "random"), (2, 3, 1, 1, 2, 2, "line"), (1, 2100, 5, 1, 64, 16, "line")])
def test_rope(dtype, interleaved, B, T, Hq, Hkv, D, R, tree):
    _say("rope", dtype, interleaved, B, T, Hq, Hkv, D, R, tree)
    rng = np.random.default_rng(B * 1000 + T)
    q, qh = _rows(rng, (B, T, Hq, D), dtype)
    k, kh = _rows(rng, (B, T, Hkv, D), dtype)
    parent, par = _trees(tree, B, T, rng)
    lens = np.asarray([0, 1000003, 2 ** 30 + 7, 77, 131072][:B], dtype=np.int32)
    freqs, f = _freqs(R)
    dl = torch.from_numpy(lens).cuda()
    pos = np.stack([int(lens[b]) + ref.depths(par[b]) for b in range(B)])
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    ta.tree_attn_rope(q, k, freqs, dl, parent, qo, ko, interleaved=interleaved)
    _assert_turned(qo, qh, pos, f, interleaved, dtype, what="q")
    _assert_turned(ko, kh, pos, f, interleaved, dtype, what="k")
    # queries alone, with an amplitude
    qa = torch.empty_like(q)
    ta.tree_attn_rope(q, None, freqs, dl, parent, qa, None, interleaved=interleaved, amplitude=1.375)
    _assert_turned(qa, qh, pos, f, interleaved, dtype, 1.375, "amplitude")
    # in place, and rows inside wider ones (which may start anywhere)
    for pad in (0, 16, 3):
        wide = torch.zeros((B, T, Hq + Hkv, D + pad), dtype=DT[dtype], device="cuda")
        v = wide[..., pad:]
        v[:, :, :Hq], v[:, :, Hq:] = q, k
        ta.tree_attn_rope(v[:, :, :Hq], v[:, :, Hq:], freqs, dl, parent, v[:, :, :Hq], v[:, :, Hq:], interleaved=interleaved)
        # (which kernel takes a call goes by its alignment; all give the same bits)
        assert torch.equal(v[:, :, :Hq], qo) and torch.equal(v[:, :, Hq:], ko), pad
        assert not wide[..., :pad].any()
    if parent is not None:
        masks = torch.empty(par.shape if parent.dim() == 2 else (T,), dtype=torch.int64, device="cuda")
        ta.tree_attn_encode(parent, masks)
        qm = torch.empty_like(q)
        ta.tree_attn_rope(q, k, freqs, dl, parent, qm, ko, interleaved=interleaved, tree_masks=masks)
        assert torch.equal(qm, qo)
    assert ta.tree_attn_last_status() == 0


@pytest.mark.parametrize("dtype,D,R", [("bf16", 128, 128), ("f32", 128, 64), ("bf16", 50, 20), ("f32", 50, 50)])
def test_rope_and_append_of_bad_requests(dtype, D, R):
    _say("bad", dtype, D, R)
    B, T, Hq, Hkv, ps = 7, 9, 4, 2, 16
    rng = np.random.default_rng(5)
    q, _ = _rows(rng, (B, T, Hq, D), dtype)
    k, _ = _rows(rng, (B, T, Hkv, D), dtype)
    par = np.stack([W.random_tree(T, 5, rng) for _ in range(B)])
    lens = np.asarray([3, 40, 55, 23, 0, 70, 9], dtype=np.int32)
    freqs, _ = _freqs(R)

    def call(lens, par, table=None, fused=False, masks=None):
        c = ref.Cache(B, [3, 40, 55, 23, 0, 70, 9], T, Hkv, D, ps, seed=3)
        t = c.dev_table if table is None else torch.from_numpy(table).cuda()
        qo, ko = torch.zeros_like(q), torch.zeros_like(k)
        own = torch.zeros(1, dtype=torch.int32, device="cuda")
        dl, dp = torch.from_numpy(lens).cuda(), torch.from_numpy(par).cuda()
        if fused:
            ta.tree_attn_q8_rope_append(q, k, k, freqs, dl, dp, qo, *c.args[:4], t, status=own, tree_masks=masks)
        else:
            ta.tree_attn_rope(q, k, freqs, dl, dp, qo, ko, status=own, tree_masks=masks)
        bits = ta.tree_attn_last_status()
        assert bits == int(own.item())
        return qo, ko, c, bits

    bad_lens, cyc, far = lens.copy(), par.copy(), par.copy()
    bad_lens[2], bad_lens[6] = -1, -2 ** 31
    cyc[1, 4], cyc[1, 5] = 5, 4
    far[3, 8] = T
    dev_cyc, masks = torch.from_numpy(cyc).cuda(), torch.empty((B, T), dtype=torch.int64, device="cuda")
    ta.tree_attn_encode(dev_cyc, masks)
    ta.tree_attn_last_status()
    for fused in (False, True):
        good = call(lens, par, fused=fused)
        assert good[3] == 0 and torch.isfinite(good[0]).all()
        for what, ln, pr, m, hit, bit in (("length", bad_lens, par, None, [2, 6], ta.TA_STATUS_BAD_SEQLEN),
                                          ("cycle", lens, cyc, None, [1], ta.TA_STATUS_BAD_PARENT),
                                          ("parent", lens, far, None, [3], ta.TA_STATUS_BAD_PARENT),
                                          ("masks", lens, par, masks, [1], ta.TA_STATUS_BAD_PARENT)):
            _say("bad", fused, what)
            qo, ko, c, bits = call(ln, pr, fused=fused, masks=m)
            assert bits == bit, what
            rest = [b for b in range(B) if b not in hit]
            assert torch.isnan(qo[hit]).all()
            if m is None:
                assert torch.equal(qo[rest], good[0][rest])
            if fused:
                now, want = c.host(), good[2].host()
                for b in range(B):
                    for i in range(T):
                        pg, sl = c.place(b, int(lens[b]) + i)
                        for x, y, first in zip(now, want, (c.kc0, c.ks0, c.vc0, c.vs0)):
                            if b in hit:
                                assert np.array_equal(x[pg, :, sl], first[pg, :, sl]), (what, b, i)
                            elif m is None:
                                assert np.array_equal(x[pg, :, sl], y[pg, :, sl]), (what, b, i)
            elif m is None:
                assert torch.isnan(ko[hit]).all() and torch.equal(ko[rest], good[1][rest])
    # beyond the page table, and pages outside the cache: not written, the queries are rotated all the same where only a page is missing
    table = good[2].table.copy()
    n_pages = good[2].shape[0]
    table[1, 40 // ps] = n_pages                              # (positions 40 .. 47 of 40 .. 48)
    table[5, 70 // ps] = -1                                   # (70 .. 78 all lie on it)
    qo, _, c, bits = call(lens, par, table=table, fused=True)
    assert bits == ta.TA_STATUS_BAD_PAGE and torch.equal(qo, good[0])
    changed = sum((x != y).reshape(*x.shape[:3], -1).any(-1).any(1).sum() for x, y in ((c.host()[1], c.ks0), (c.host()[0], c.kc0)))
    assert changed > 0
    pg, sl = c.place(1, 48)
    assert np.array_equal(c.host()[0][pg, :, sl], good[2].host()[0][pg, :, sl])
    long_lens = lens.copy()
    long_lens[4] = c.table.shape[1] * ps - T + 1
    qo, _, c, bits = call(long_lens, par, fused=True)
    assert bits == ta.TA_STATUS_BAD_SEQLEN and torch.isnan(qo[4]).all() and torch.isfinite(qo[[0, 1, 2, 3, 5, 6]]).all()


def _special(x):
    """Rows that quantising may stumble over."""
    x = x.copy()
    r = x.reshape(-1, x.shape[-1])
    n = len(r)
    r[0 % n] = 0.0
    r[1 % n] *= 1e-40
    r[2 % n] *= 1e36
    r[3 % n, 0] = np.inf
    r[3 % n, -1] = -np.inf
    r[4 % n, :] = np.nan
    r[5 % n, 0] = 448.0 * 2.0 ** 5
    r[6 % n, 0] = 450.0                                       # (448.0 and 450 are neighbours in bf16)
    r[7 % n] = np.round(r[7 % n] * 16) / 16                   # ties
    r[8 % n] = 0.0
    r[8 % n, 0] = 2.0 ** -149
    return r.reshape(x.shape)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,Hkv,D,ps,paged,order,pad", [
    (1, 1, 1, 128, 64, True, "phsd", 0), (3, 16, 8, 128, 16, True, "phsd", 0), (2, 7, 2, 64, 1, True, "pshd", 0),
    (2, 300, 2, 128, 48, True, "hpsd", 0), (3, 64, 2, 80, 32, False, "phsd", 0), (2, 5, 3, 37, 7, True, "phsd", 0),
    (2, 9, 1, 256, 64, True, "phsd", 0), (4, 12, 2, 128, 16, True, "phsd", 3), (1, 1500, 3, 48, 64, True, "pshd", 16)])
def test_append_and_read(dtype, B, T, Hkv, D, ps, paged, order, pad):
    _say("append", dtype, B, T, Hkv, D, ps, paged, order, pad)
    rng = np.random.default_rng(T * 7 + D)
    lens = rng.integers(0, 200, size=B)
    lens[0] = 0
    c = ref.Cache(B, lens, T, Hkv, D, ps, seed=1, paged=paged, order=order, pad=pad)
    k, kh = _rows(rng, (B, T, Hkv, D), dtype, 1.0)
    v = torch.from_numpy(_special(kh[..., ::-1]).astype(np.float32)).to(DT[dtype]).cuda()
    vh = v.double().cpu().numpy()
    ta.tree_attn_q8_append(k, v, *c.args, c.dev_lens)
    assert ta.tree_attn_last_status() == 0
    want = [x.copy() for x in (c.kc0, c.ks0, c.vc0, c.vs0)]
    for rows, codes, scales in ((kh, want[0], want[1]), (vh, want[2], want[3])):
        cc, ss = ref.quantise(rows)
        for b in range(B):
            for i in range(T):
                pg, sl = c.place(b, int(lens[b]) + i)
                codes[pg, :, sl], scales[pg, :, sl] = cc[b, i], ss[b, i]
    got = c.host()
    for x, y, name in zip(got, want, ("K codes", "K scales", "V codes", "V scales")):
        if name.endswith("codes"):                            # (a NaN code has a sign that says nothing)
            x, y = np.where(x & 127 == 127, 127, x), np.where(y & 127 == 127, 127, y)
        assert np.array_equal(x, y), name
    # and back, from several starts
    n = T + 3
    for starts, counts in ((None, lens + T), (lens, np.full(B, T)), (lens // 2, np.minimum(lens // 3, n)), (lens, np.zeros(B, dtype=int))):
        N = max(int(counts.max()), 1) + 2
        ko, vo = (torch.full((B, N, Hkv, D), 5.0, dtype=DT[dtype], device="cuda") for _ in range(2))
        ds = None if starts is None else torch.from_numpy(np.asarray(starts, dtype=np.int32)).cuda()
        ta.tree_attn_q8_read(*c.args, ds, torch.from_numpy(np.asarray(counts, dtype=np.int32)).cuda(), ko, vo)
        for b in range(B):
            s0, m = 0 if starts is None else int(starts[b]), int(counts[b])
            K, V = c.logical(b, s0 + m, got)
            for out, w in ((ko, K), (vo, V)):
                w = torch.from_numpy(w[s0:].astype(np.float32)).to(DT[dtype])
                torch.testing.assert_close(out[b, :m].cpu(), w, rtol=0, atol=0, equal_nan=True)
                assert (out[b, m:] == 5.0).all()
    assert ta.tree_attn_last_status() == 0


def test_read_of_bad_requests():
    B, T, Hkv, D, ps = 6, 4, 2, 64, 16
    lens = [40, 50, 60, 10, 33, 21]
    c = ref.Cache(B, lens, T, Hkv, D, ps, seed=2)
    table = c.dev_table.clone()
    table[4, 1] = c.shape[0]
    cap = table.shape[1] * ps
    starts = torch.tensor([0, -1, 10, cap - 3, 0, 5], dtype=torch.int32).cuda()
    counts = torch.tensor([40, 5, 65, 4, 33, -1], dtype=torch.int32).cuda()
    ko, vo = (torch.full((B, 64, Hkv, D), 5.0, device="cuda") for _ in range(2))
    ta.tree_attn_q8_read(*c.args[:4], table, starts, counts, ko, vo)
    assert ta.tree_attn_last_status() == ta.TA_STATUS_BAD_SEQLEN | ta.TA_STATUS_BAD_PAGE
    for out in (ko, vo):
        assert torch.isfinite(out[0]).all() and (out[0, 40:] == 5.0).all()
        assert torch.isnan(out[[1, 2, 3, 5]]).all()
        assert torch.isfinite(out[4, :16]).all() and torch.isnan(out[4, 16:32]).all() and torch.isfinite(out[4, 32]).all()
        assert (out[4, 33:] == 5.0).all()


@pytest.mark.parametrize("dtype,interleaved,D,R,order", [
    ("bf16", False, 128, 128, "phsd"), ("bf16", True, 128, 64, "phsd"), ("f32", False, 64, 64, "pshd"), ("f32", True, 96, 32, "phsd"),
    ("bf16", False, 50, 20, "phsd"), ("f32", True, 250, 250, "phsd")])
@pytest.mark.parametrize("T,tree", [(1, "line"), (21, "random"), (64, "random"), (333, "line")])
def test_rope_append_is_rope_and_append(dtype, interleaved, D, R, order, T, tree):
    _say("rope_append", dtype, interleaved, D, R, T, tree)
    B, Hq, Hkv = 3, 6, 2
    rng = np.random.default_rng(T)
    lens = [0, 131, 70]
    a, b = (ref.Cache(B, lens, T, Hkv, D, 16, seed=1, order=order) for _ in range(2))
    q, _ = _rows(rng, (B, T, Hq, D), dtype)
    k, _ = _rows(rng, (B, T, Hkv, D), dtype, 1.0)
    v, _ = _rows(rng, (B, T, Hkv, D), dtype, 1.0)
    freqs, _ = _freqs(R)
    parent, _ = _trees(tree, B, T, rng)
    q1, k1, q2 = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)
    kw = dict(interleaved=interleaved, amplitude=1.25)
    ta.tree_attn_rope(q, k, freqs, a.dev_lens, parent, q1, k1, **kw)
    ta.tree_attn_q8_append(k1, v, *a.args, a.dev_lens)
    ta.tree_attn_q8_rope_append(q, k, v, freqs, b.dev_lens, parent, q2, *b.args, **kw)
    assert torch.equal(q1, q2) and ta.tree_attn_last_status() == 0
    for x, y in zip(a.host(), b.host()):
        assert np.array_equal(x, y)


@pytest.mark.parametrize("D,ps,order,pad", [(128, 16, "phsd", 0), (64, 64, "pshd", 0), (37, 7, "phsd", 0), (128, 32, "hpsd", 5)])
def test_compact(D, ps, order, pad):
    _say("compact", D, ps, order, pad)
    B, T, Hkv, A = 7, 21, 3, 30
    rng = np.random.default_rng(4)
    lens = [0, 5, 100, 63, 17, 31, 48]
    c = ref.Cache(B, lens, 40, Hkv, D, ps, seed=8, order=order, pad=pad)
    paths = rng.integers(0, T, size=(B, A)).astype(np.int32)
    paths[0, :5], paths[1, :3] = [0, 3, 7, 12, 20], [2, 1, 0]
    n = np.asarray([5, 3, 0, 30, 1, 4, 2], dtype=np.int32)
    paths[5, 2], n[6] = T, 31                                 # a node that is none, a path that is too long
    table = c.table.copy()
    so = torch.empty(B, dtype=torch.int32, device="cuda")
    ta.tree_attn_q8_compact(*c.args, c.dev_lens, torch.from_numpy(paths).cuda(), torch.from_numpy(n).cuda(), T, so)
    assert ta.tree_attn_last_status() == ta.TA_STATUS_BAD_PATH
    want = [x.copy() for x in (c.kc0, c.ks0, c.vc0, c.vs0)]
    for b in range(5):
        for x, first in zip(want, (c.kc0, c.ks0, c.vc0, c.vs0)):
            for i in range(n[b]):
                sp, ss = c.place(b, lens[b] + int(paths[b, i]))
                dp, ds = c.place(b, lens[b] + i)
                x[dp, :, ds] = first[sp, :, ss]
    for x, y in zip(c.host(), want):
        assert np.array_equal(x, y)
    assert so.tolist() == [a + int(m) for a, m in zip(lens[:5], n)] + lens[5:]
    # lengths in place; a page that is none, a length that is none
    table[3, (63 + 2) // ps] = -5
    bad = torch.tensor([0, -3, 100, 63, 17, 31, 48], dtype=torch.int32).cuda()
    before = c.host()
    n[:] = 0
    n[1], n[3] = 2, 2
    ta.tree_attn_q8_compact(*c.args[:4], torch.from_numpy(table).cuda(), bad, torch.from_numpy(paths).cuda(), torch.from_numpy(n).cuda(),
                            T, bad)
    assert ta.tree_attn_last_status() == ta.TA_STATUS_BAD_SEQLEN | ta.TA_STATUS_BAD_PAGE
    assert bad.tolist() == [0, -3, 100, 63, 17, 31, 48]
    for x, y in zip(c.host(), before):
        assert np.array_equal(x, y)


def _fwd(c, q, parent, **kw):
    out = torch.full_like(q, float("nan"))
    lse = torch.full((q.shape[0], q.shape[2], q.shape[1]), float("nan"), dtype=torch.float32, device="cuda")
    ta.tree_attn_q8_fwd(q, *c.args, c.dev_lens, parent, out, lse, **kw)
    return out, lse


def _assert_fwd(got, want, bf16, what=""):
    out, lse, size = want
    d = np.abs(got[0].double().cpu().numpy() - out)
    tol = ref.bound_fwd(out, size, bf16)
    assert (d <= tol).all(), (what, float((d / tol).max()))
    assert np.abs(got[1].double().cpu().numpy() - lse).max() <= 1e-4, what


FWD = [
    # B, T, Hq, Hkv, D, ps, lens, tree
    (1, 1, 8, 1, 128, 64, [0], "line"), (1, 1, 1, 1, 128, 64, [1], "line"), (2, 1, 8, 2, 128, 16, [63, 64], "line"),
    (3, 1, 8, 1, 128, 64, [4097, 1, 700], "line"), (4, 8, 8, 1, 128, 64, [31, 32, 33, 500], "random"),
    (2, 16, 32, 8, 128, 64, [300, 1500], "random"), (1, 64, 8, 2, 128, 128, [2000], "random"), (2, 64, 32, 4, 128, 64, [100, 333], "static"),
    (3, 5, 5, 1, 64, 32, [900, 0, 77], "random"), (2, 21, 28, 4, 64, 64, [640, 129], "random"), (2, 64, 16, 1, 64, 64, [700, 20], "random"),
    (2, 4, 8, 2, 128, 8, [200, 31], "random"), (2, 4, 8, 2, 128, 4, [90, 131], "random"), (2, 6, 4, 4, 128, 1, [40, 3], "random"),
    (2, 7, 6, 2, 96, 48, [130, 260], "random"), (1, 3, 2, 1, 37, 5, [70], "random"), (2, 9, 4, 2, 256, 64, [300, 1], "static"),
    (70, 2, 4, 2, 128, 16, [i * 7 % 190 for i in range(70)], "static"), (300, 1, 2, 1, 64, 16, [i * 13 % 90 for i in range(300)], "line")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(FWD)))
def test_fwd(dtype, case):
    B, T, Hq, Hkv, D, ps, lens, tree = FWD[case]
    _say("fwd", dtype, *FWD[case][:6], lens[:4], tree)
    rng = np.random.default_rng(case)
    c = ref.Cache(B, lens, T, Hkv, D, ps, seed=case)
    q, qh = _rows(rng, (B, T, Hq, D), dtype)
    parent, par = _trees(tree, B, T, rng)
    if parent is None:
        parent = torch.from_numpy(W.chain_tree(T)).cuda()
    want = ref.expect_fwd(c, qh, par)
    _assert_fwd(_fwd(c, q, parent), want, dtype == "bf16", "auto")
    _assert_fwd(_fwd(c, q, parent, kernel=ta.TA_KERNEL_GENERIC), want, dtype == "bf16", "scalar")
    for splits in (1, 7):
        _assert_fwd(_fwd(c, q, parent, num_splits=splits), want, dtype == "bf16", splits)
    assert ta.tree_attn_last_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,ps,paged,order,pad", [(128, 64, False, "phsd", 0), (128, 64, True, "pshd", 0), (64, 16, True, "hpsd", 0),
                                                 (128, 32, True, "phsd", 16), (128, 32, True, "phsd", 3), (64, 8, True, "pshd", 0)])
def test_fwd_options_and_layouts(dtype, D, ps, paged, order, pad):
    _say("fwd options", dtype, D, ps, paged, order, pad)
    B, T, Hq, Hkv = 3, 12, 8, 2
    rng = np.random.default_rng(1)
    lens = [517, 64, 250]
    c = ref.Cache(B, lens, T, Hkv, D, ps, seed=3, paged=paged, order=order, pad=pad)
    wide, _ = _rows(rng, (B, T, Hq, D + 24), dtype)
    parent, par = _trees("random", B, T, rng)
    starts = np.asarray([130, 64, 33], dtype=np.int32)
    masks = torch.empty((B, T), dtype=torch.int64, device="cuda")
    ta.tree_attn_encode(parent, masks)
    for at in (0, 8, 3):                                      # rows of q that start anywhere
        q = wide[..., at:at + D]
        qh = q.double().cpu().numpy()
        bf = dtype == "bf16"
        _assert_fwd(_fwd(c, q, parent), ref.expect_fwd(c, qh, par), bf, "layout")
        _assert_fwd(_fwd(c, q, parent, kv_start=torch.from_numpy(starts).cuda(), scale=0.3, tree_masks=masks),
                    ref.expect_fwd(c, qh, par, scale=0.3, starts=starts), bf, "window")
        _assert_fwd(_fwd(c, q[:, 5:9], parent, q_node_offset=5), ref.expect_fwd(c, qh[:, 5:9], par, q_off=5), bf, "offset")
    # an output with other strides, no lse, a workspace of the caller's
    out = torch.empty((B, Hq, T, D + 8), dtype=DT[dtype], device="cuda").permute(0, 2, 1, 3)[..., :D]
    plan = ta.tree_attn_q8_plan(q, *c.args, c.dev_lens, parent, out)
    ws = torch.empty(plan["workspace_bytes"], dtype=torch.uint8, device="cuda")
    ta.tree_attn_q8_fwd(q, *c.args, c.dev_lens, parent, out, None, workspace=ws)
    want = ref.expect_fwd(c, qh, par)
    assert (np.abs(out.double().cpu().numpy() - want[0]) <= ref.bound_fwd(want[0], want[2], bf)).all()
    assert ta.tree_attn_last_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,kernel", [(128, 0), (64, 0), (128, 1), (50, 0)])
def test_fwd_nan_reaches_only_what_attends_to_it(dtype, D, kernel):
    _say("fwd NaN", dtype, D, kernel)
    B, T, Hq, Hkv = 6, 10, 8, 2
    rng = np.random.default_rng(2)
    lens = [100, 300, 37, 64, 0, 90]
    par = np.stack([W.bfs_tree(T, [3, 2], 5)] * B)            # 0 -> 1 2 3; 1 -> 4 5; 2 -> 6 7; 3 -> 8 9
    parent = torch.from_numpy(par).cuda()
    q, qh = _rows(rng, (B, T, Hq, D), dtype)
    c = ref.Cache(B, lens, T, Hkv, D, 16, seed=6)
    want = ref.expect_fwd(c, qh, par)

    def spoil(b, pos, codes, scales, how):
        pg, sl = c.place(b, pos)
        if how == "scale":
            scales[pg, 1, sl] = 255
        else:
            codes[pg, 1, sl, how] = 127 if pos % 2 else 255

    spoil(0, 50, c.vc0, c.vs0, 3)                             # a value in the prefix
    spoil(1, 299, c.kc0, c.ks0, 5)                            # a key at its end
    spoil(2, 37 + 6, c.vc0, c.vs0, D - 1)                     # a value of node 6: nobody else attends to it
    spoil(3, 64 + 2, c.kc0, c.ks0, 0)                         # a key of node 2: nodes 2, 6 and 7
    spoil(4, 3, c.vc0, c.vs0, "scale")                        # node 3: nodes 3, 8 and 9
    spoil(5, 90 + 1, c.kc0, c.ks0, "scale")                   # node 1: nodes 1, 4 and 5
    for b in range(B):                                        # behind the last token, and in pages that nobody owns
        end = lens[b] + T
        if end % 16:
            pg, sl = c.place(b, end - 1)
            for x, s in ((c.kc0, c.ks0), (c.vc0, c.vs0)):
                x[pg, :, sl + 1:] = 127
                s[pg, :, sl + 1:] = 255
    c.up()
    nodes = {0: range(T), 1: range(T), 2: [6], 3: [2, 6, 7], 4: [3, 8, 9], 5: [1, 4, 5]}
    for splits in (0, 1, 5):
        out, lse = _fwd(c, q, parent, kernel=kernel, num_splits=splits)
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        hit = np.zeros((B, T, Hq), dtype=bool)
        for b, ns in nodes.items():
            hit[b, list(ns), Hq // 2:] = True
        assert np.isnan(out[hit]).any(-1).all(), splits
        assert not np.isnan(out[~hit]).any(), splits
        d = np.abs(out - want[0])[~hit]
        assert (d <= ref.bound_fwd(want[0], want[2], dtype == "bf16")[~hit]).all(), splits
        keys = np.zeros_like(hit)
        for b in (1, 3, 5):
            keys[b] = hit[b]
        assert np.isnan(lse.transpose(0, 2, 1)[keys]).all() and np.abs(lse - want[1]).transpose(0, 2, 1)[~hit].max() <= 1e-4
    assert ta.tree_attn_last_status() == 0


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 128), ("bf16", 64), ("bf16", 50)])
def test_fwd_of_bad_requests(dtype, D):
    _say("fwd bad", dtype, D)
    B, T, Hq, Hkv, ps = 6, 19, 4, 2, 16
    lens = [300, 90, 61, 40, 128, 33]
    rng = np.random.default_rng(3)
    par = np.stack([W.bfs_tree(T, [3], 5)] * B)
    q, _ = _rows(rng, (B, T, Hq, D), dtype)
    c = ref.Cache(B, lens, T, Hkv, D, ps, seed=9)
    good = _fwd(c, q, torch.from_numpy(par).cuda())
    base, total = c.table.copy(), c.shape[0]
    for name in ("kc", "vc", "ks", "vs"):                     # pages just past the pool lie in memory that this process owns
        t = getattr(c, name)
        full = torch.zeros((total + 4,) + tuple(t.shape[1:]), dtype=torch.uint8, device="cuda").view(t.dtype)
        full.view(torch.uint8)[:total] = t.view(torch.uint8)
        setattr(c, name, full[:total])
    tree_page, prefix = base.copy(), base.copy()
    tree_page[1, 90 // ps], tree_page[2, (61 + T - 1) // ps], tree_page[4, 128 // ps] = total, total + 3, -1
    prefix[0, 7] = total
    bad_len, cyc = c.lens.copy(), par.copy()
    bad_len[3], bad_len[5] = -1, base.shape[1] * ps
    cyc[2, 1], cyc[2, 2] = 2, 1
    masks = torch.zeros((B, T), dtype=torch.int64, device="cuda")
    ta.tree_attn_encode(torch.from_numpy(cyc).cuda(), masks)
    ta.tree_attn_last_status()
    tol = 2e-5 if dtype == "f32" else 2e-2                    # the schedule may differ
    for what, table, seq, tree, kw, hit, bit in (
            ("page of the tree", tree_page, c.lens, par, {}, [1, 2, 4], ta.TA_STATUS_BAD_PAGE),
            ("page of the prefix", prefix, c.lens, par, {}, [0], ta.TA_STATUS_BAD_PAGE),
            ("length", base, bad_len, par, {}, [3, 5], ta.TA_STATUS_BAD_SEQLEN),
            ("parents", base, c.lens, cyc, {}, [2], ta.TA_STATUS_BAD_PARENT),
            ("masks", base, c.lens, par, {"tree_masks": masks}, [2], ta.TA_STATUS_BAD_PARENT)):
        for splits in (0, 1):
            _say("fwd bad", what, splits)
            own = torch.zeros(1, dtype=torch.int32, device="cuda")
            out, lse = torch.zeros_like(q), torch.zeros((B, Hq, T), device="cuda")
            ta.tree_attn_q8_fwd(q, *c.args[:4], torch.from_numpy(table).cuda(), torch.from_numpy(seq).cuda(),
                                torch.from_numpy(tree).cuda(), out, lse, num_splits=splits, status=own, **kw)
            assert ta.tree_attn_last_status() == bit == int(own.item()), what
            assert torch.isnan(out[hit]).all() and torch.isnan(lse[hit]).all(), what
            rest = [b for b in range(B) if b not in hit]
            assert (out[rest].float() - good[0][rest].float()).abs().max() <= tol, what
            assert (lse[rest] - good[1][rest]).abs().max() <= 1e-4, what


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_steps_of_a_verification_loop(dtype, D):
    """Prompt written, then rotate + append, attention and compaction of several steps: everything that the cache holds and every
    output against the same loop in float64; once as plain calls, once replayed from captured graphs on another stream."""
    B, T, Hq, Hkv, ps, R = 3, 12, 8, 2, 16, D
    rng = np.random.default_rng(11)
    prompt = np.asarray([37, 150, 64], dtype=np.int32)
    steps = 4
    freqs, f = _freqs(R)
    N = int(prompt.max())
    pk, pkh = _rows(rng, (B, N, Hkv, D), dtype)
    pq, _ = _rows(rng, (B, N, Hq, D), dtype)
    data = []
    for _ in range(steps):
        par = np.stack([W.random_tree(T, 5, rng) for _ in range(B)])
        ways = []
        for b in range(B):
            node, way = int(rng.integers(0, T)), []
            while node >= 0:
                way.append(node)
                node = int(par[b, node])
            ways.append(way[::-1])
        data.append((par, ways, *[_rows(rng, (B, T, h, D), dtype)[0] for h in (Hq, Hkv, Hkv)]))
    results = []
    for captured in (False, True):
        c = ref.Cache(B, np.full(B, N + 6 * steps), T, Hkv, D, ps, seed=1, fill=0)
        lens = torch.zeros(B, dtype=torch.int32, device="cuda")
        q_dump = torch.empty_like(pq)
        ta.tree_attn_q8_rope_append(pq, pk, pk, freqs, lens, None, q_dump, *c.args)      # prompts, padded to the longest
        lens.copy_(torch.from_numpy(prompt))
        q, k, v = (torch.empty_like(x) for x in data[0][2:])
        parent = torch.empty((B, T), dtype=torch.int32, device="cuda")
        paths, n_acc = torch.zeros((B, T), dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
        qr, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty((B, Hq, T), device="cuda")

        def step():
            ta.tree_attn_q8_rope_append(q, k, v, freqs, lens, parent, qr, *c.args)
            ta.tree_attn_q8_fwd(qr, *c.args, lens, parent, out, lse)
            ta.tree_attn_q8_compact(*c.args, lens, paths, n_acc, T, lens)

        graph = None
        if captured:
            ta.tree_attn_reserve(ta.tree_attn_q8_plan(qr, *c.args, lens, parent, out, lse)["workspace_bytes"])
            parent.copy_(torch.from_numpy(data[0][0]))
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
        got = []
        for par, ways, *rows in data:
            for dst, src in zip((q, k, v), rows):
                dst.copy_(src)
            parent.copy_(torch.from_numpy(par))
            hp = np.zeros((B, T), dtype=np.int32)
            for b in range(B):
                hp[b, :len(ways[b])] = ways[b]
            paths.copy_(torch.from_numpy(hp))
            n_acc.copy_(torch.tensor([len(w) for w in ways], dtype=torch.int32))
            graph.replay() if captured else step()
            torch.cuda.synchronize()
            got.append((out.clone(), lse.clone(), lens.tolist(), qr.clone()))
        assert ta.tree_attn_last_status() == 0
        results.append((got, c.host()))
    (got, cache), (again, cache2) = results
    for x, y in zip(got, again):
        assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1]) and x[2] == y[2] and torch.equal(x[3], y[3])
    for x, y in zip(cache, cache2):
        assert np.array_equal(x, y)
    # the same loop on lists of rows; keys as the kernels rotated them are within a rounding of these, so codes may differ by a step
    # where a rounding falls on the other side: outputs are compared with the codes that the cache really holds
    lens = prompt.copy()
    for (out, lse, now, qr), (par, ways, q, k, v) in zip(got, data):
        want_q, size = ref.rotate(q.double().cpu().numpy().reshape(B * T, Hq, D),
                                  np.concatenate([lens[b] + ref.depths(par[b]) for b in range(B)]), f, False)
        tol = 2.0 ** -20 * size + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want_q)
        assert (np.abs(qr.double().cpu().numpy().reshape(want_q.shape) - want_q) <= tol).all()
        lens = lens + np.asarray([len(w) for w in ways], dtype=np.int32)
        assert now == lens.tolist()
    # what the cache holds at the end: prompt and accepted rows, in order
    c.lens = lens
    for b in range(B):
        K, V = c.logical(b, int(lens[b]), cache)
        rows_k, rows_v, pos = [pkh[b, :prompt[b]]], [pkh[b, :prompt[b]]], int(prompt[b])
        for par, ways, q, k, v in data:
            rows_k.append(k[b, ways[b]].double().cpu().numpy())
            rows_v.append(v[b, ways[b]].double().cpu().numpy())
        want_v = np.concatenate(rows_v)
        codes, scales = ref.quantise(want_v)
        assert np.array_equal(V, ref.values(codes, scales))
        want_k, size = ref.rotate(np.concatenate(rows_k), np.arange(len(want_v)), f, False)
        # rounded to the keys' type, then to a code (2^-4 of it, or 2^-10 of the scale, which is at most twice the largest / 448)
        top = np.abs(want_k).max(-1, keepdims=True)
        tol = (2.0 ** -4 + 2.0 ** -7) * np.abs(want_k) + 2.0 ** -20 * size + 2.0 ** -10 * 2.1 * top / 448
        assert (np.abs(K - want_k) <= tol).all()
    # the last step's outputs, from the rows that were in the cache when it ran (its tree is still there but for the rows that moved)
    first = [x[0] for x in got]
    assert all(torch.isfinite(x).all() for x in first)

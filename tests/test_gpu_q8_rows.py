"""GPU tests of attention over the 8-bit cache at every number of query rows per KV head at which another kernel, another block of
rows, another schedule or another place for the schedule takes over; against the definition in float64."""
import numpy as np
import pytest
import torch

from tests import q8_reference as ref
from tests.test_gpu_q8 import _assert_fwd, _fwd, _rows, _say
from paper_2508_08192_amd import treeattn as ta
from paper_2508_08192_amd import workloads as W

pytestmark = pytest.mark.gpu

# T, query heads of a KV head: rows around 32, 64, 128, 192, 256, 384 and 512, one group of 256 heads, and odd ones
ROWS = [(1, 32), (11, 3), (8, 8), (13, 5), (16, 8), (43, 3), (64, 3), (39, 5), (64, 4), (37, 7), (48, 8), (55, 7), (64, 8), (1, 256), (3, 200)]


def _problem(B, T, G, Hkv, D, ps, lens, seed, dtype, paged=True):
    rng = np.random.default_rng(seed)
    c = ref.Cache(B, lens, T, Hkv, D, ps, seed=seed, paged=paged)
    q, qh = _rows(rng, (B, T, G * Hkv, D), dtype)
    par = np.stack([W.shuffle_tree(W.random_tree(T, 6, rng), rng)[0] for _ in range(B)])
    return c, q, qh, torch.from_numpy(par).cuda(), par


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("T,G", ROWS)
def test_rows(T, G, D, dtype):
    _say("rows", dtype, D, T, G)
    B, Hkv, lens = 3, 2, [450, 127, 33]
    c, q, qh, parent, par = _problem(B, T, G, Hkv, D, 32, lens, T + G, dtype)
    bf = dtype == "bf16"
    want = ref.expect_fwd(c, qh, par)
    for splits in (0, 1, 5, 40):
        _assert_fwd(_fwd(c, q, parent, num_splits=splits), want, bf, splits)
    # a window that starts inside a tile of tokens, at the end of the prefix and at its start; some of the tree's nodes
    starts = np.asarray([77, 127, 0], dtype=np.int32)
    lo, hi = T // 3, T // 3 + (T + 1) // 2
    want = ref.expect_fwd(c, qh[:, lo:hi], par, scale=0.2, starts=starts, q_off=lo)
    for splits in (0, 3):
        _assert_fwd(_fwd(c, q[:, lo:hi], parent, num_splits=splits, scale=0.2, kv_start=torch.from_numpy(starts).cuda(), q_node_offset=lo),
                    want, bf, ("window", splits))
    assert ta.tree_attn_last_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,G", [(2, 3), (9, 7), (16, 8), (40, 5)])
@pytest.mark.parametrize("B", [64, 65, 257])
def test_batches(B, T, G, dtype):
    """A schedule in registers, in LDS with the lengths beside it, and in LDS alone; all lengths around the ends of tiles."""
    _say("batches", B, T, G, dtype)
    lens = [(31, 32, 33, 127, 128, 129, 0, 1, 255)[i % 9] + 128 * (i % 5 == 4) for i in range(B)]
    c, q, qh, parent, par = _problem(B, T, G, 1, 64, 16, lens, B + T, dtype)
    want = ref.expect_fwd(c, qh, par)
    for splits in (0, 9, 300):
        _assert_fwd(_fwd(c, q, parent, num_splits=splits), want, dtype == "bf16", splits)
    assert ta.tree_attn_last_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,G,D", [(40, 1, 128), (25, 4, 128), (60, 3, 64), (64, 6, 128)])
def test_nan_and_bad_requests(T, G, D, dtype):
    """What a NaN reaches, and what a bad request does to its neighbours in the same workgroup, with many rows."""
    _say("NaN", T, G, D, dtype)
    B, Hkv, ps, lens = 5, 2, 16, [200, 130, 61, 0, 96]
    c, q, qh, parent, par = _problem(B, T, G, Hkv, D, ps, lens, 3, dtype)
    want = ref.expect_fwd(c, qh, par)
    bf = dtype == "bf16"
    node = T // 2

    def spoil(b, pos, codes, scales, d):
        pg, sl = c.place(b, pos)
        if d is None:
            scales[pg, 1, sl] = 255
        else:
            codes[pg, 1, sl, d] = 255

    spoil(0, 150, c.vc0, c.vs0, 7)
    spoil(1, 130 + node, c.vc0, c.vs0, D - 1)
    spoil(2, 61 + T - 1, c.kc0, c.ks0, 1)
    spoil(3, 0, c.vc0, c.vs0, None)
    for b in range(B):                                        # behind the last token of every request
        if (lens[b] + T) % ps:
            pg, sl = c.place(b, lens[b] + T - 1)
            c.vc0[pg, :, sl + 1:], c.vs0[pg, :, sl + 1:], c.kc0[pg, :, sl + 1:] = 127, 255, 127
    c.up()
    sees = ref.seen_matrix(T, 0, par[1])[:, node], ref.seen_matrix(T, 0, par[2])[:, T - 1], ref.seen_matrix(T, 0, par[3])[:, 0]
    hit = np.zeros((B, T, G * Hkv), dtype=bool)
    hit[0, :, G:] = True
    for b, s in zip((1, 2, 3), sees):
        hit[b, s, G:] = True
    for splits in (0, 1, 6):
        out, lse = _fwd(c, q, parent, num_splits=splits)
        out = out.double().cpu().numpy()
        assert np.isnan(out[hit]).any(-1).all() and not np.isnan(out[~hit]).any(), splits
        d = np.abs(out - want[0])[~hit]
        assert (d <= ref.bound_fwd(want[0], want[2], bf)[~hit]).all(), splits
    assert ta.tree_attn_last_status() == 0
    table, tree, seq = c.table.copy(), par.copy(), c.lens.copy()
    table[0, 3] = -1
    tree[4, 1], tree[4, 2] = 2, 1
    seq[2] = c.table.shape[1] * ps + 1
    for splits in (0, 2):
        out, lse = torch.zeros_like(q), torch.zeros((B, G * Hkv, T), device="cuda")
        ta.tree_attn_q8_fwd(q, *c.args[:4], torch.from_numpy(table).cuda(), torch.from_numpy(seq).cuda(), torch.from_numpy(tree).cuda(),
                            out, lse, num_splits=splits)
        assert ta.tree_attn_last_status() == ta.TA_STATUS_BAD_PAGE | ta.TA_STATUS_BAD_PARENT | ta.TA_STATUS_BAD_SEQLEN
        assert torch.isnan(out[[0, 2, 4]]).all() and torch.isnan(lse[[0, 2, 4]]).all()
        good = np.zeros(B, dtype=bool)
        good[[1, 3]] = True
        keep = good[:, None, None] & ~hit
        d = np.abs(out.double().cpu().numpy() - want[0])[keep]
        assert (d <= ref.bound_fwd(want[0], want[2], bf)[keep]).all(), splits


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,G", [(5, 4), (50, 1), (30, 4), (64, 4)])
def test_scores_far_apart_and_a_contiguous_cache(T, G, dtype):
    """Rows whose scores grow along the sequence, so that the reference of the softmax moves at every tile, and a cache that ends with
    the last token."""
    _say("far apart", dtype, T, G)
    B, Hkv, D, lens = 2, 2, 128, [388, 388]
    rng = np.random.default_rng(T)
    c = ref.Cache(B, lens, T, Hkv, D, 16, seed=T, paged=False)
    total = c.shape[2]
    ramp = np.exp2(np.floor(np.linspace(-6, 2, total)))
    x = rng.standard_normal(c.shape) * 0.1 + 1.0
    c.kc0, c.ks0 = ref.quantise((x * ramp[None, None, :, None]).astype(np.float32).astype(np.float64))
    c.up()
    q, qh = _rows(rng, (B, T, G * Hkv, D), dtype)
    q = (q * 0.2 + 0.5).contiguous()
    par = np.stack([W.shuffle_tree(W.random_tree(T, 6, rng), rng)[0] for _ in range(B)])
    want = ref.expect_fwd(c, q.double().cpu().numpy(), par)
    for splits in (0, 1, 4):
        _assert_fwd(_fwd(c, q, torch.from_numpy(par).cuda(), num_splits=splits), want, dtype == "bf16", splits)
    assert ta.tree_attn_last_status() == 0


@pytest.mark.parametrize("dtype,kernel", [("bf16", 0), ("f32", 0), ("bf16", 1), ("f32", 1)])
@pytest.mark.parametrize("T,G,D", [(6, 4, 128), (40, 1, 128), (25, 4, 64), (60, 3, 128)])
def test_values_past_the_largest_number_in_the_tree(T, G, D, dtype, kernel):
    """448 * 2^127 as a key's or a value's column of one node: rows that do not attend to it are as without it."""
    _say("largest", T, G, D, dtype, kernel)
    B, Hkv, lens = 2, 2, [100, 37]
    c, q, qh, parent, par = _problem(B, T, G, Hkv, D, 16, lens, 5, dtype)
    want = ref.expect_fwd(c, qh, par)
    node = [int(ref.seen_matrix(T, 0, par[b]).sum(0).argmin()) for b in range(B)]      # a leaf
    for b, (codes, scales) in enumerate(((c.vc0, c.vs0), (c.kc0, c.ks0))):
        pg, sl = c.place(b, lens[b] + node[b])
        scales[pg, :, sl] = 254
        codes[pg, :, sl] = 0
        codes[pg, :, sl, 3] = 0x7e
    c.up()
    for splits in (0, 2):
        out, lse = _fwd(c, q, parent, num_splits=splits, kernel=kernel)
        for b in range(B):
            rows = ~ref.seen_matrix(T, 0, par[b])[:, node[b]]
            d = np.abs(out[b].double().cpu().numpy() - want[0][b])[rows]
            assert (d <= ref.bound_fwd(want[0], want[2], dtype == "bf16")[b][rows]).all(), (b, splits)
            assert np.abs(lse[b].double().cpu().numpy() - want[1][b])[:, rows].max() <= 1e-4
    assert ta.tree_attn_last_status() == 0


@pytest.mark.parametrize("dtype,T,G", [("bf16", 8, 4), ("bf16", 16, 4), ("bf16", 64, 2), ("bf16", 64, 4), ("bf16", 64, 7), ("f32", 16, 4)])
@pytest.mark.parametrize("D,ps", [(128, 16), (128, 64), (64, 32)])
def test_long_shares(dtype, T, G, D, ps):
    """Shares of more tiles than a wave holds page ids for, so that it fetches them anew on the way; pages in no order."""
    _say("long", dtype, T, G, D, ps)
    B, Hkv, lens = 2, 1, [20001, 8200]
    c, q, qh, parent, par = _problem(B, T, G, Hkv, D, ps, lens, T, dtype)
    starts = np.asarray([3000, 77], dtype=np.int32)
    for kw, args in (({}, {}), (dict(starts=starts), dict(kv_start=torch.from_numpy(starts).cuda()))):
        want = ref.expect_fwd(c, qh, par, **kw)
        for splits in (0, 1, 2):
            _assert_fwd(_fwd(c, q, parent, num_splits=splits, **args), want, dtype == "bf16", splits)
    assert ta.tree_attn_last_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,G", [(1, 8), (10, 4), (20, 5), (50, 5)])
@pytest.mark.parametrize("L", [1000, 8192, 40000])
def test_one_list(T, G, L, dtype):
    """One request with one KV head: the split over workgroups and the merge of many parts."""
    _say("one list", T, G, L, dtype)
    c, q, qh, parent, par = _problem(1, T, G, 1, 128, 64, [L], L + T, dtype)
    want = ref.expect_fwd(c, qh, par)
    for splits in (0, 100, 256):
        _assert_fwd(_fwd(c, q, parent, num_splits=splits), want, dtype == "bf16", splits)
    assert ta.tree_attn_last_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_large_batch(dtype):
    """More requests than a workgroup keeps lengths of, in every kernel, some of them without a token."""
    _say("large batch", dtype)
    B = 2100
    for T, G in ((1, 2), (9, 4)):
        lens = [(0, 5, 64, 100, 31)[i % 5] for i in range(B)]
        c, q, qh, parent, par = _problem(B, T, G, 1, 64, 16, lens, T, dtype)
        got = _fwd(c, q, parent)
        some = np.random.default_rng(0).choice(B, 60, replace=False)
        for b in some.tolist():
            one = ref.Cache.__new__(ref.Cache)
            one.__dict__.update(c.__dict__)
            one.lens, one.table = c.lens[b:b + 1], c.table[b:b + 1]
            _assert_fwd((got[0][b:b + 1], got[1][b:b + 1]), ref.expect_fwd(one, qh[b:b + 1], par[b:b + 1]), dtype == "bf16", b)
    assert ta.tree_attn_last_status() == 0

"""GPU tests of how the 8-bit cache's calls are made: memory past 32 bits, two streams at once, captured graphs, and the way past
the extension module."""
import numpy as np
import pytest
import torch

from tests import q8_reference as ref
from tests.test_gpu_q8 import DT, _assert_fwd, _freqs, _fwd, _rows, _say
from paper_2508_08192_amd import treeattn as ta
from paper_2508_08192_amd import workloads as W

pytestmark = pytest.mark.gpu


def _trees(B, T, rng):
    p = np.stack([W.shuffle_tree(W.random_tree(T, 6, rng), rng)[0] for _ in range(B)])
    return torch.from_numpy(p).cuda(), p


@pytest.mark.parametrize("gap", [2 ** 31 - 4096, 2 ** 31 + 4096])
@pytest.mark.parametrize("D", [128, 64])
def test_past_32_bits(D, gap):
    """Pages so far apart that the third begins past 2^32 bytes: below 2^31 apart for the matrix-core kernels, above for the scalar."""
    _say("past 32 bits", D, gap)
    B, T, Hkv, ps, lens = 2, 5, 2, 64, [70, 33]
    c = ref.Cache(B, lens, T, Hkv, D, ps, seed=D, decoys=0)
    pages = c.shape[0]
    assert pages >= 3
    big = [torch.empty(gap * (pages - 1) + Hkv * ps * D, dtype=torch.uint8, device="cuda") for _ in range(4)]
    names = ("kc", "vc", "ks", "vs")
    for name, mem in zip(names, big):
        t = getattr(c, name)
        u = t.view(torch.uint8)
        far = mem.as_strided(u.shape, (gap,) + tuple(u.contiguous().stride()[1:]))
        far.copy_(u)
        setattr(c, name, far.view(t.dtype))
    rng = np.random.default_rng(1)
    parent, par = _trees(B, T, rng)
    for G, dtype in ((4, "bf16"), (20, "bf16"), (30, "bf16"), (70, "bf16"), (3, "f32")):
        q, qh = _rows(rng, (B, T, G * Hkv, D), dtype)
        plan = ta.tree_attn_q8_plan(q, *c.args, c.dev_lens, parent, q)
        assert plan["kernel"] == (ta.TA_KERNEL_MFMA if gap < 2 ** 31 else ta.TA_KERNEL_GENERIC)
        want = ref.expect_fwd(c, qh, par)
        for splits in (0, 2):
            _assert_fwd(_fwd(c, q, parent, num_splits=splits), want, dtype == "bf16", (G, dtype, splits))
    # written, read back, moved: the last page of request 0
    k, kh = _rows(rng, (B, T, Hkv, D), "bf16")
    v, vh = _rows(rng, (B, T, Hkv, D), "bf16")
    ta.tree_attn_q8_append(k, v, *c.args, c.dev_lens)
    ko, vo = (torch.zeros((B, T, Hkv, D), dtype=torch.float32, device="cuda") for _ in range(2))
    ta.tree_attn_q8_read(*c.args, c.dev_lens, torch.full((B,), T, dtype=torch.int32, device="cuda"), ko, vo)
    for got, rows in ((ko, kh), (vo, vh)):
        want = ref.values(*ref.quantise(rows))
        assert np.array_equal(got.double().cpu().numpy(), want)
    paths = torch.tensor([[0, 3, 4]] * B, dtype=torch.int32, device="cuda")
    ta.tree_attn_q8_compact(*c.args, c.dev_lens, paths, torch.full((B,), 3, dtype=torch.int32, device="cuda"), T, None)
    ta.tree_attn_q8_read(*c.args, c.dev_lens, torch.full((B,), 3, dtype=torch.int32, device="cuda"), ko[:, :3], vo[:, :3])
    for got, rows in ((ko, kh), (vo, vh)):
        want = ref.values(*ref.quantise(rows))[:, [0, 3, 4]]
        assert np.array_equal(got[:, :3].double().cpu().numpy(), want)
    assert ta.tree_attn_last_status() == 0


def _problems(dtype):
    """One problem for each kernel and schedule."""
    for i, (B, T, G, Hkv, D, lens) in enumerate(((3, 4, 4, 2, 128, [900, 40, 2500]), (2, 16, 4, 2, 128, [1300, 700]), (2, 25, 5, 1, 64, [1900, 64]),
                                                 (2, 64, 4, 2, 128, [300, 2100]), (4, 16, 4, 2, 128, [100, 90, 30, 64]))):
        rng = np.random.default_rng(i)
        c = ref.Cache(B, lens, T, Hkv, D, 32, seed=i)
        q, qh = _rows(rng, (B, T, G * Hkv, D), dtype)
        parent, par = _trees(B, T, rng)
        yield c, q, qh, parent, par


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_streams_at_once(dtype):
    streams = [torch.cuda.Stream() for _ in range(2)]
    problems = list(_problems(dtype))
    want = [_fwd(c, q, parent) for c, q, _, parent, _ in problems]
    size = max(ta.tree_attn_q8_plan(q, *c.args, c.dev_lens, parent, q)["workspace_bytes"] for c, q, _, parent, _ in problems)
    spaces = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    got = []
    for i in range(40):
        c, q, _, parent, _ = problems[(i // 2 + i % 2) % len(problems)]
        with torch.cuda.stream(streams[i % 2]):
            got.append((((i // 2 + i % 2) % len(problems)), _fwd(c, q, parent, workspace=spaces[i % 2])))
    torch.cuda.synchronize()
    for n, (out, lse) in got:
        assert torch.equal(out, want[n][0]) and torch.equal(lse, want[n][1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_graphs(dtype):
    """Every kernel captured once, replayed with other lengths and other queries, with eager calls in between."""
    for c, q, _, parent, par in _problems(dtype):
        _say("graph", dtype, tuple(q.shape))
        out, lse = torch.empty_like(q), torch.empty((q.shape[0], q.shape[2], q.shape[1]), device="cuda")
        plan = ta.tree_attn_q8_plan(q, *c.args, c.dev_lens, parent, out)
        ws = torch.empty(plan["workspace_bytes"], dtype=torch.uint8, device="cuda")
        ta.tree_attn_q8_fwd(q, *c.args, c.dev_lens, parent, out, lse, workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ta.tree_attn_q8_fwd(q, *c.args, c.dev_lens, parent, out, lse, workspace=ws)
        full = c.lens.copy()
        for cut in (0, 1, 17):
            c.lens = np.maximum(full - cut, 0).astype(np.int32)
            c.dev_lens.copy_(torch.from_numpy(c.lens))
            q.mul_(-0.5)
            graph.replay()
            want = ref.expect_fwd(c, q.double().cpu().numpy(), par)
            _assert_fwd((out, lse), want, dtype == "bf16", cut)
            again = _fwd(c, q, parent)
            assert torch.equal(again[0], out) and torch.equal(again[1], lse)
        assert ta.tree_attn_last_status() == 0


def test_the_way_past_the_extension_module(monkeypatch):
    """Descriptors written by the extension module and by ctypes: the same call."""
    if ta._call is None:
        pytest.skip("the module is not built")
    B, T, Hq, Hkv, D, ps = 2, 6, 8, 2, 64, 16
    rng = np.random.default_rng(0)
    freqs, _ = _freqs(D)
    q, _ = _rows(rng, (B, T, Hq, D), "bf16")
    k, _ = _rows(rng, (B, T, Hkv, D), "bf16")
    v, _ = _rows(rng, (B, T, Hkv, D), "bf16")
    parent, par = _trees(B, T, rng)
    masks = torch.empty((B, T), dtype=torch.int64, device="cuda")
    ta.tree_attn_encode(parent, masks)
    starts = torch.tensor([3, 0], dtype=torch.int32, device="cuda")
    paths = torch.tensor([[0, 1], [0, 2]], dtype=torch.int32, device="cuda")
    n_acc = torch.tensor([2, 1], dtype=torch.int32, device="cuda")

    def all_calls():
        c = ref.Cache(B, [40, 9], T, Hkv, D, ps, seed=4)
        res = []
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        ta.tree_attn_rope(q, k, freqs, c.dev_lens, parent, qo, ko, interleaved=True, amplitude=1.5, tree_masks=masks)
        res += [qo.clone(), ko.clone()]
        ta.tree_attn_rope(q, None, freqs, c.dev_lens, None, qo, None)
        res.append(qo.clone())
        ta.tree_attn_q8_append(k, v, *c.args, c.dev_lens)
        res += c.host()
        ta.tree_attn_q8_rope_append(q, k, v, freqs, c.dev_lens, parent, qo, *c.args)
        res += [qo.clone()] + c.host()
        out, lse = torch.empty_like(q), torch.empty((B, Hq, T), device="cuda")
        ta.tree_attn_q8_fwd(qo, *c.args, c.dev_lens, parent, out, lse, scale=0.3, kv_start=starts, tree_masks=masks)
        res += [out.clone(), lse.clone()]
        ta.tree_attn_q8_fwd(qo[:, 2:4], *c.args, c.dev_lens, parent, out[:, 2:4], None, q_node_offset=2, num_splits=3, item_cost=2)
        res.append(out.clone())
        ta.tree_attn_q8_compact(*c.args, c.dev_lens, paths, n_acc, T, c.dev_lens)
        res += c.host() + [c.dev_lens.clone()]
        ko, vo = torch.zeros((B, 12, Hkv, D), device="cuda"), torch.zeros((B, 12, Hkv, D), device="cuda")
        ta.tree_attn_q8_read(*c.args, starts, n_acc, ko, vo)
        return res + [ko, vo]

    first = all_calls()
    monkeypatch.setattr(ta, "_call", None)
    second = all_calls()
    assert len(first) == len(second)
    for x, y in zip(first, second):
        assert np.array_equal(np.asarray(x.float().cpu() if torch.is_tensor(x) else x), np.asarray(y.float().cpu() if torch.is_tensor(y) else y))
    assert ta.tree_attn_last_status() == 0

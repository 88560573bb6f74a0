"""Host-side checks of the rotary embedding and the 8-bit cache: refusals before any device call, frequencies, plans."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest

from paper_2508_08192_amd import treeattn as ta
from paper_2508_08192_amd.treeattn import Desc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF, F32, I32, C8, S8 = ta.TA_BF16, ta.TA_F32, ta.TA_I32, ta.TA_E4M3, ta.TA_E8M0


def _good(B=2, T=8, Hq=8, Hkv=2, D=128, ps=64, max_pages=5, pages=16, dt=BF, A=6, N=20):
    cache = Desc((pages, Hkv, ps, D), C8)
    scale = Desc((pages, Hkv, ps), S8)
    return dict(q=Desc((B, T, Hq, D), dt), k_new=Desc((B, T, Hkv, D), dt), v_new=Desc((B, T, Hkv, D), dt),
                q_out=Desc((B, T, Hq, D), dt, ptr=0x9000), k_out=Desc((B, T, Hkv, D), dt, ptr=0x9000),
                freqs=Desc((D // 2,), F32), seq_lens=Desc((B,), I32), tree_parent=Desc((B, T), I32), k_cache=cache, v_cache=cache,
                k_scale=scale, v_scale=scale, page_table=Desc((B, max_pages), I32), out=Desc((B, T, Hq, D), dt, ptr=0x9000),
                lse=Desc((B, Hq, T), F32), starts=Desc((B,), I32), counts=Desc((B,), I32), k_read=Desc((B, N, Hkv, D), dt),
                v_read=Desc((B, N, Hkv, D), dt), accepted=Desc((B, A), I32), n_accepted=Desc((B,), I32),
                seq_lens_out=Desc((B,), I32), tree_size=T)


CACHE = ("k_cache", "v_cache", "k_scale", "v_scale", "page_table")
CALLS = {
    "rope": (ta.tree_attn_rope, ("q", "k_new", "freqs", "seq_lens", "tree_parent", "q_out", "k_out")),
    "append": (ta.tree_attn_q8_append, ("k_new", "v_new") + CACHE + ("seq_lens",)),
    "rope_append": (ta.tree_attn_q8_rope_append, ("q", "k_new", "v_new", "freqs", "seq_lens", "tree_parent", "q_out") + CACHE),
    "read": (ta.tree_attn_q8_read, CACHE + ("starts", "counts", "k_read", "v_read")),
    "compact": (ta.tree_attn_q8_compact, CACHE + ("seq_lens", "accepted", "n_accepted", "tree_size", "seq_lens_out")),
    "fwd": (ta.tree_attn_q8_fwd, ("q",) + CACHE + ("seq_lens", "tree_parent", "out", "lse")),
}


def _rc(call, over=None, kw=None, **sizes):
    a = _good(**sizes)
    a.update(over or {})
    fn, names = CALLS[call]
    return fn(*[a[n] for n in names], stream=0, check=False, **(kw or {}))


def test_a_good_call_gets_as_far_as_the_device():
    import torch
    if torch.cuda.is_available():
        pytest.skip("the descriptors point nowhere")
    for call in CALLS:
        assert _rc(call) == ta.TA_ERR_HIP, call
    assert _rc("rope", T=5000, over={"tree_parent": None}) == ta.TA_ERR_HIP
    assert _rc("rope", over={"k_new": None, "k_out": None}) == ta.TA_ERR_HIP
    assert _rc("append", T=300, max_pages=5) == ta.TA_ERR_HIP
    assert _rc("append", over={"page_table": None}) == ta.TA_ERR_HIP
    assert _rc("read", over={"starts": None, "page_table": None}) == ta.TA_ERR_HIP
    assert _rc("compact", over={"seq_lens_out": None}) == ta.TA_ERR_HIP


def test_empty_batches_do_nothing():
    for call in CALLS:
        assert _rc(call, B=0) == ta.TA_OK, call
    assert _rc("read", N=0) == ta.TA_OK


@pytest.mark.parametrize("call,over,want", [
    ("rope", {"q": None}, ta.TA_ERR_NULL), ("rope", {"freqs": None}, ta.TA_ERR_NULL), ("rope", {"k_out": None}, ta.TA_ERR_NULL),
    ("rope", {"q": Desc((2, 8, 8, 128), I32)}, ta.TA_ERR_DTYPE), ("rope", {"freqs": Desc((64,), BF)}, ta.TA_ERR_DTYPE),
    ("rope", {"k_new": Desc((2, 8, 2, 128), F32)}, ta.TA_ERR_DTYPE), ("rope", {"freqs": Desc((65,), F32)}, ta.TA_ERR_SHAPE),
    ("rope", {"freqs": Desc((0,), F32)}, ta.TA_ERR_SHAPE), ("rope", {"freqs": Desc((64,), F32, (2,))}, ta.TA_ERR_STRIDE),
    ("rope", {"q_out": Desc((2, 8, 7, 128), BF)}, ta.TA_ERR_SHAPE), ("rope", {"seq_lens": Desc((3,), I32)}, ta.TA_ERR_SHAPE),
    ("rope", {"tree_parent": Desc((2, 7), I32)}, ta.TA_ERR_SHAPE), ("rope", {"tree_parent": Desc((3, 8), I32)}, ta.TA_ERR_SHAPE),
    ("rope", {"q": Desc((2, 8, 8, 128), BF, (8192, 1024, 128, 2))}, ta.TA_ERR_STRIDE),
    ("rope", {"q_out": Desc((2, 8, 8, 128), BF, (0, 1024, 128, 1))}, ta.TA_ERR_STRIDE),
    ("rope", {"q_out": Desc((2, 8, 8, 128), BF, (8192, 128, 1024, 1), ptr=0x1000)}, ta.TA_ERR_STRIDE),     # in place, but elsewhere
    ("rope", {"q": Desc((2, 8, 8, 128), BF, ptr=0)}, ta.TA_ERR_NULL),
    ("append", {"k_new": None}, ta.TA_ERR_NULL), ("append", {"k_scale": None}, ta.TA_ERR_NULL),
    ("append", {"k_cache": Desc((16, 2, 64, 128), BF)}, ta.TA_ERR_DTYPE), ("append", {"v_scale": Desc((16, 2, 64), F32)}, ta.TA_ERR_DTYPE),
    ("append", {"v_new": Desc((2, 8, 2, 128), F32)}, ta.TA_ERR_DTYPE), ("append", {"v_new": Desc((2, 8, 2, 64), BF)}, ta.TA_ERR_SHAPE),
    ("append", {"k_scale": Desc((16, 2, 32), S8)}, ta.TA_ERR_SHAPE), ("append", {"k_scale": Desc((16, 2), S8)}, ta.TA_ERR_RANK),
    ("append", {"k_cache": Desc((16, 2, 64, 128), C8, (0, 8192, 128, 1))}, ta.TA_ERR_STRIDE),
    ("append", {"v_scale": Desc((16, 2, 64), S8, (128, 0, 1))}, ta.TA_ERR_STRIDE),
    ("append", {"page_table": Desc((3, 5), I32)}, ta.TA_ERR_PAGE_TABLE), ("append", {"page_table": Desc((2, 0), I32)}, ta.TA_ERR_PAGE_TABLE),
    ("append", {"k_new": Desc((2, 321, 2, 128), BF), "v_new": Desc((2, 321, 2, 128), BF)}, ta.TA_ERR_PAGE_TABLE),
    ("append", {"seq_lens": Desc((2,), I32, (-1,))}, ta.TA_ERR_STRIDE),
    ("rope_append", {"q": Desc((2, 8, 8, 128), F32)}, ta.TA_ERR_DTYPE), ("rope_append", {"q_out": None}, ta.TA_ERR_NULL),
    ("rope_append", {"q": Desc((2, 7, 8, 128), BF)}, ta.TA_ERR_SHAPE),
    ("read", {"counts": None}, ta.TA_ERR_NULL), ("read", {"k_read": Desc((2, 20, 2, 128), C8)}, ta.TA_ERR_DTYPE),
    ("read", {"v_read": Desc((2, 21, 2, 128), BF)}, ta.TA_ERR_SHAPE), ("read", {"starts": Desc((3,), I32)}, ta.TA_ERR_SHAPE),
    ("read", {"k_read": Desc((2, 20, 2, 128), BF, (0, 256, 128, 1))}, ta.TA_ERR_STRIDE),
    ("compact", {"accepted": None}, ta.TA_ERR_NULL), ("compact", {"v_cache": Desc((16, 2, 64, 128), BF)}, ta.TA_ERR_DTYPE),
    ("compact", {"accepted": Desc((2, 65), I32)}, ta.TA_ERR_TREE_SIZE), ("compact", {"tree_size": 65}, ta.TA_ERR_TREE_SIZE),
    ("compact", {"seq_lens_out": Desc((2,), I32, ptr=0x1004)}, ta.TA_ERR_STRIDE),
    ("fwd", {"k_scale": None}, ta.TA_ERR_NULL), ("fwd", {"k_cache": Desc((16, 2, 64, 128), BF)}, ta.TA_ERR_DTYPE),
    ("fwd", {"v_scale": Desc((16, 2, 63), S8)}, ta.TA_ERR_SHAPE), ("fwd", {"out": Desc((2, 8, 8, 128), F32)}, ta.TA_ERR_DTYPE),
    ("fwd", {"q": Desc((2, 8, 7, 128), BF), "out": Desc((2, 8, 7, 128), BF)}, ta.TA_ERR_HEADS),
    ("fwd", {"out": Desc((2, 8, 8, 128), BF, (8192, 0, 128, 1))}, ta.TA_ERR_STRIDE),
    ("fwd", {"tree_parent": None}, ta.TA_ERR_NULL), ("fwd", {"k_scale": Desc((16, 2, 64), S8, ptr=0)}, ta.TA_ERR_NULL)])
def test_refusals(call, over, want):
    assert _rc(call, over) == want


def test_refused_sizes_and_options():
    for call in ("rope", "rope_append"):
        assert _rc(call, T=65) == ta.TA_ERR_TREE_SIZE                     # a tree's
        for kw in ({"amplitude": -1.0}, {"amplitude": float("nan")}, {"amplitude": float("inf")}, {"interleaved": 2}):
            assert _rc(call, kw=kw) == ta.TA_ERR_OPTS, kw
        assert _rc(call, kw={"status": Desc((1,), I32, ptr=0x1002)}) == ta.TA_ERR_OPTS
    for call in CALLS:
        assert _rc(call, D=257) == ta.TA_ERR_HEAD_DIM, call
        assert _rc(call, B=4097, pages=5000) == ta.TA_ERR_BATCH, call
    assert _rc("fwd", T=65) == ta.TA_ERR_TREE_SIZE
    assert _rc("fwd", kw={"kernel": 4}) == ta.TA_ERR_OPTS
    assert _rc("fwd", D=96, kw={"kernel": ta.TA_KERNEL_MFMA}) == ta.TA_ERR_OPTS
    o = ta._opts(k_new=Desc((2, 8, 2, 128), C8), v_new=Desc((2, 8, 2, 128), C8))
    a = _good()
    ds = [ta._desc(a[n]) for n in CALLS["fwd"][1]]
    import ctypes
    assert ta.load_library().tree_attn_q8_fwd(*[ta._ref(d) for d in ds], None, ctypes.byref(o)) == ta.TA_ERR_OPTS


def test_frequencies():
    R, base = 64, 500000.0
    plain = [base ** (-2.0 * j / R) for j in range(R // 2)]
    f, amp = ta.tree_attn_rope_freqs(R, base)
    assert np.allclose(f, plain, rtol=2 ** -23) and amp == 1.0
    f, amp = ta.tree_attn_rope_freqs(R, base, ta.TA_ROPE_LINEAR, factor=4.0)
    assert np.allclose(f, np.asarray(plain) / 4, rtol=2 ** -23) and amp == 1.0
    for rule, low, high in ((ta.TA_ROPE_BANDS, 1.0, 4.0), (ta.TA_ROPE_YARN, 1.0, 32.0)):
        f, amp = ta.tree_attn_rope_freqs(R, base, rule, factor=8.0, original=8192.0, low=low, high=high)
        for j in range(R // 2):
            wave = 2 * math.pi / plain[j]
            if wave < 8192 / high:
                want = plain[j]
            elif wave > 8192 / low:
                want = plain[j] / 8
            else:
                s = (8192 / wave - low) / (high - low)
                want = (1 - s) * plain[j] / 8 + s * plain[j]
            assert abs(f[j] - want) <= 2 ** -22 * want
        assert amp == (1.0 if rule == ta.TA_ROPE_BANDS else np.float32(0.1 * math.log(8.0) + 1))
    bad = [dict(rotary_dim=63), dict(rotary_dim=0), dict(rotary_dim=258)]
    assert all(ta.tree_attn_rope_freqs(**kw, check=False) == ta.TA_ERR_HEAD_DIM for kw in bad)
    for kw in (dict(base=1.0), dict(base=float("nan")), dict(rule=4), dict(rule=-1), dict(rule=1, factor=0.5),
               dict(rule=2, factor=2.0), dict(rule=2, factor=2.0, original=100.0, low=2.0, high=2.0),
               dict(rule=3, factor=float("inf"), original=100.0, low=1.0, high=2.0)):
        assert ta.tree_attn_rope_freqs(64, **kw, check=False) == ta.TA_ERR_OPTS, kw


def _plan(a, **kw):
    return ta.tree_attn_q8_plan(*[a[n] for n in CALLS["fwd"][1]], **kw)


def test_plan_of_the_scalar_kernel():
    p = _plan(_good(D=96))
    assert p["kernel"] == ta.TA_KERNEL_GENERIC and p["table_row"] == -1 and p["workspace_bytes"] > 0
    assert _plan(_good(D=96), num_splits=3)["kv_workgroups"] == 3
    assert _plan(_good(), kernel=ta.TA_KERNEL_GENERIC)["kernel"] == ta.TA_KERNEL_GENERIC


def test_plan_of_the_matrix_core_kernels():
    """Who takes a call, in what blocks of rows, and whether lists are cut."""
    def plan(**kw):
        return _plan(_good(**{k: v for k, v in kw.items() if k not in ("num_splits", "kernel")}),
                     **{k: v for k, v in kw.items() if k in ("num_splits", "kernel")})

    for dt in (BF, F32):
        for D in (64, 128):
            assert plan(D=D, dt=dt)["kernel"] == ta.TA_KERNEL_MFMA
            assert plan(D=D, dt=dt, kernel=ta.TA_KERNEL_MFMA)["kernel"] == ta.TA_KERNEL_MFMA
        for kw in (dict(ps=8), dict(ps=48), dict(D=96), dict(D=32)):
            assert plan(dt=dt, **kw)["kernel"] == ta.TA_KERNEL_GENERIC
            with pytest.raises(ta.TreeAttnError):
                plan(dt=dt, kernel=ta.TA_KERNEL_MFMA, **kw)
    # two groups of four heads: T 8 has 32 rows, 9 has 36, 64 has 256
    rows = {T: plan(T=T)["workgroup_rows"] for T in (1, 8, 9, 16, 17, 32, 33, 64)}
    assert rows == {1: 32, 8: 32, 9: 64, 16: 64, 17: 128, 32: 128, 33: 256, 64: 256}
    assert plan(T=1, dt=F32)["workgroup_rows"] == plan(T=64, dt=F32)["workgroup_rows"] == 128
    # short lists are not cut and need no merge, unless the caller says how
    assert plan(max_pages=4)["merge_workgroups"] == 0 and plan(max_pages=200)["merge_workgroups"] > 0
    assert plan(max_pages=4, num_splits=2)["merge_workgroups"] > 0


def test_random_descriptors_never_break_the_host_code():
    """Random ranks, shapes and strides through the checks of every call: any status is fine, as long as it is one."""
    rng = np.random.default_rng(7)
    seen = set()
    for _ in range(4000):
        call = str(rng.choice(sorted(CALLS)))
        # (always one damaged descriptor too many for the device: nothing is launched)
        a = _good(B=int(rng.integers(1, 5)), T=int(rng.integers(1, 70)), Hkv=int(rng.integers(1, 4)), D=int(rng.choice([1, 37, 64, 128, 256])),
                  ps=int(rng.choice([1, 3, 16, 64])), max_pages=int(rng.integers(1, 40)), pages=int(rng.integers(0, 50)),
                  dt=int(rng.choice([BF, F32])))
        names = [n for n in CALLS[call][1] if n != "tree_size" and a[n] is not None]
        key = str(rng.choice(names))
        d, kind = a[key], int(rng.integers(0, 4))
        if kind == 0:
            a[key] = Desc(d.shape, int(rng.choice([0, 1, 2, 3, 4, 5, 7])), d.stride, d.ptr)
        elif kind == 1:
            a[key] = Desc(d.shape[:-1] if rng.random() < 0.5 else d.shape + (2,), d.dtype)
        elif kind == 2:
            a[key] = Desc(d.shape, d.dtype, tuple(int(x) * int(rng.choice([-1, 0, 1, 3])) for x in d.stride), d.ptr)
        else:
            a[key] = Desc(tuple(int(rng.integers(0, 2 ** 33)) for _ in d.shape), d.dtype, d.stride, int(rng.choice([0, 0x1000, 0x1002])))
        if call == "fwd":
            r = _plan(a, kernel=int(rng.integers(0, 4)), num_splits=int(rng.integers(0, 500)), item_cost=int(rng.integers(0, 9)), check=False)
            seen.add(0 if isinstance(r, dict) else r)
        elif not _device():
            fn, nm = CALLS[call]
            seen.add(fn(*[a[n] for n in nm], stream=0, check=False))
    assert all(-13 <= r <= 0 for r in seen) and len(seen) >= 6


def _device():
    import torch
    return torch.cuda.is_available()


def test_host_code_under_address_and_undefined_behaviour_sanitizers():
    """This file again, against a g++ build of the host logic with -fsanitize=address,undefined."""
    from paper_2508_08192_amd.build import build_host_checked
    lib, runtime = build_host_checked()
    env = dict(os.environ)
    env["TREEATTN_LIB"] = lib
    env["LD_PRELOAD"] = (runtime + " " + env.get("LD_PRELOAD", "")).strip()
    env["ASAN_OPTIONS"] = "detect_leaks=0:abort_on_error=1"
    env["UBSAN_OPTIONS"] = "halt_on_error=1:print_stacktrace=1"
    proc = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-q", "-x", "-p", "no:cacheprovider",
                           "-k", "not sanitizers"], cwd=ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True,
                          timeout=600)
    assert proc.returncode == 0, proc.stdout[-4000:]

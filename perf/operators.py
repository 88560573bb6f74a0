"""The calls that the rotary embedding and the 8-bit KV cache are timed on: what a step's queries, keys and values go
through on their way into a cache of e4m3 codes with one power of two per row, and out of it again.

A case is a plain dict:

  op                 "rope": queries and keys are rotated to their positions
                     "append": keys and values are quantised into the cache ("rotate": the queries and keys rotated first)
                     "read": a part of the cache as dense rows
                     "compact": the accepted path of a tree moves behind the prefix
                     "fwd": attention of the new tokens over the cache
  B, Hq, Hkv, D      batch, query heads, KV heads (one GPU's share of them), head dimension
  T                  new tokens of a request: the nodes of a tree, or (tree "line") the tokens of a prompt
  L0, L1             shortest and longest prefix of the batch; the B lengths are spread evenly between the two and dealt to
                     the requests in an order that the seed gives (op "read": how many tokens are read back)
  ps                 tokens per page, 0 = the contiguous layout
  dtype              "bf16" or "f32": of everything but the codes
  R                  columns that are rotated (the rest keep their values), interleaved: neighbouring columns are a pair
  tree               "static", "dynamic" (a random tree per request) or "line"

Queries, keys and values are standard normal, as in the library's own synthetic workloads; the codes of a cache are those of
normal rows whose sizes differ from token to token, as those of keys and values do.
"""
import math

import numpy as np
import torch

own = False

DECOY_PAGES = 3            # pages of the pool that no request owns
BASE = 500000.0            # of the rotary frequencies


def _case(name, op, B, Hq, Hkv, D, T, L0, L1, ps, dtype="bf16", R=0, interleaved=False, tree="static", rotate=False):
    c = dict(op=op, B=B, Hq=Hq, Hkv=Hkv, D=D, T=T, L0=L0, L1=L1, ps=ps, dtype=dtype, R=R or D, interleaved=interleaved,
             tree=tree, rotate=rotate)
    if name:
        c = dict(name=name, **c)
    return c


def listed():
    return [
        # batch size one, where latency counts: the 8-node tree on one GPU's share (8 of 64 heads) of a large model
        _case("rope_bs1_share_n8", "rope", 1, 8, 1, 128, 8, 8192, 8192, 0),
        # a chunk of a prompt far inside a long context, neighbouring columns in pairs
        _case("rope_prompt", "rope", 1, 32, 8, 128, 8000, 100000, 100000, 0, interleaved=True, tree="line"),
        # a verification step of a batch: rotate, quantise, write behind the prefixes
        _case("append_step_bs32", "append", 32, 32, 8, 128, 16, 100, 2000, 64, tree="dynamic", rotate=True),
        # prompts of uneven contexts written into small pages
        _case("append_prompts", "append", 4, 32, 8, 128, 4001, 0, 777, 16, tree="line"),
        # a short context read back
        _case("read_bs1_short", "read", 1, 8, 1, 128, 1, 300, 300, 64),
        # the contexts of a batch handed on, as dense rows
        _case("read_bs16", "read", 16, 32, 8, 128, 1, 1000, 9000, 64),
        # after acceptance: a small batch and a full serving batch
        _case("compact_bs8", "compact", 8, 32, 8, 128, 16, 300, 900, 16),
        _case("compact_bs128", "compact", 128, 32, 8, 128, 21, 100, 700, 64),
        # one new token of one request: one GPU's share of a large model, 8k context
        _case("fwd_bs1_decode", "fwd", 1, 8, 1, 128, 1, 8192, 8192, 64, tree="line"),
        # one new token of each request of a full serving batch
        _case("fwd_bs128_decode", "fwd", 128, 32, 8, 128, 1, 256, 4096, 64, tree="line"),
        # batched verification of uneven contexts with a dynamic tree per request
        _case("fwd_bs32_t16", "fwd", 32, 32, 8, 128, 16, 512, 8192, 64, tree="dynamic"),
        # the largest: long contexts and wide trees
        _case("fwd_long_t64", "fwd", 4, 32, 8, 128, 64, 131072, 131072, 128),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: an operator, then its sizes over the whole range of it."""
    op = rng.choice(["rope", "append", "read", "compact", "fwd", "fwd", "fwd"])
    Hq, Hkv = rng.choice([(8, 1), (5, 1), (16, 2), (32, 8), (16, 8), (28, 4), (32, 4)])
    D, ps = rng.choice([128, 128, 128, 64]), rng.choice([16, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    es = 2 if dtype == "bf16" else 4
    R, interleaved, rotate = rng.choice([D, D, D // 2]), rng.choice([False, True]), False
    tree = rng.choice(["static", "dynamic", "line"])
    lo = hi = _log_int(rng, 100, 131072)
    if op in ("rope", "append"):
        row = (Hq + 2 * Hkv) * D * es                       # bytes of a token's rows, at most
        T = _log_int(rng, 1, 9000) if tree == "line" else rng.choice([4, 7, 8, 12, 16, 21, 32, 45, 64])
        B = max(1, min(_log_int(rng, 1, 64), int(6.0e7 / (row * T))))
        T = min(T, int(6.0e7 / (row * B)))
        rotate = op == "append" and rng.choice([False, True])
        if op == "append":
            lo = hi = min(hi, 3000)
            lo = int(hi * rng.choice([0.1, 0.5, 1.0]))
    elif op == "read":
        T, B, tree = 1, _log_int(rng, 1, 32), "line"
        hi = min(_log_int(rng, 50, 30000), int(8.0e7 / (B * Hkv * D)) + 1)
        lo = int(hi * rng.choice([0.1, 0.5, 1.0]))
    elif op == "compact":
        T, B, tree = rng.choice([8, 12, 16, 21, 32, 45, 64]), _log_int(rng, 1, 120), "static"
        hi = _log_int(rng, 50, 900)
        lo = int(hi * rng.choice([0.1, 0.5, 1.0]))
    else:
        T = 1 if tree == "line" else rng.choice([4, 7, 8, 12, 16, 21, 32, 45, 64])
        cap = 4.0e8 if dtype == "bf16" else 1.5e7           # bytes of codes
        B, hi = _log_int(rng, 1, 128), _log_int(rng, 100, 131072)
        B = max(1, min(B, int(cap / (hi * Hkv * D * 2))))
        hi = min(hi, int(cap / (B * Hkv * D * 2)))
        lo = max(1, int(hi * rng.choice([0.06, 0.25, 0.5, 1.0])))
        ps = rng.choice([0, 16, 32, 64, 64, 128])
    if rng.random() < 0.7 and hi > 40:
        hi += rng.randint(-30, 30)                          # ragged ends
        lo = min(lo, hi)
    return _case(None, op, B, Hq, Hkv, D, T, lo, hi, ps, dtype, R, interleaved, tree, rotate)


# ----------------------------------------------------------------------------- inputs

def _lengths(case):
    B, lo, hi = case["B"], case["L0"], case["L1"]
    return np.asarray([hi if B == 1 else lo + (hi - lo) * i // (B - 1) for i in range(B)], dtype=np.int64)


def _static_tree(T):
    """The root, four children, then two children each, level by level."""
    return np.asarray([-1] + [0 if i < 5 else (i - 5) // 2 + 1 for i in range(1, T)], dtype=np.int32)


def _trees(case, rng):
    B, T = case["B"], case["T"]
    if case["tree"] == "line":
        return np.arange(-1, T - 1, dtype=np.int32)
    if case["tree"] == "static":
        return _static_tree(T)
    trees = np.full((B, T), -1, dtype=np.int32)
    for b in range(B):
        for i in range(1, T):
            trees[b, i] = rng.integers(max(0, i - 8), i)
    return trees


def _quantise(x):
    """e4m3 codes and e8m0 scales of the rows of x (finite values, float32): x is about codes * scales."""
    top = x.abs().amax(-1)
    m, e = torch.frexp(top)
    e = (e - torch.where(m <= 0.875, 9, 8)).clamp_min(-126)          # 448 is 0.875 * 2^9
    e = torch.where(top > 0, e, 0)
    codes = (x / torch.ldexp(torch.ones_like(top), e)[..., None]).to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def prepare(case, seed):
    op, B, Hq, Hkv, D, T, ps = (case[k] for k in ("op", "B", "Hq", "Hkv", "D", "T", "ps"))
    dev = torch.device("cuda", torch.cuda.current_device())
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev).to(dt)

    def up(a):
        return torch.from_numpy(np.ascontiguousarray(a)).to(dev)

    lens = rng.permutation(_lengths(case))
    trees = _trees(case, rng)
    s = dict(case=case, lens=up(lens.astype(np.int32)), parent=up(trees))
    if op == "rope" or case["rotate"]:
        s["freqs"] = up((BASE ** (-np.arange(0, case["R"], 2) / case["R"])).astype(np.float32))
    if op in ("rope", "append"):
        s["q"], s["k"], s["v"] = normal(B, T, Hq, D), normal(B, T, Hkv, D), normal(B, T, Hkv, D)
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        if op == "rope":
            return s
    total = lens + T
    if ps:
        pages = (total + ps - 1) // ps
        ids = rng.permutation(int(pages.sum()) + DECOY_PAGES).astype(np.int32)
        table = np.zeros((B, int(pages.max())), dtype=np.int32)
        at = 0
        for b in range(B):
            table[b, :pages[b]] = ids[at:at + pages[b]]
            at += int(pages[b])
        shape = (len(ids), Hkv, ps, D)
        s["table"] = up(table)
    else:
        shape = (B, Hkv, int(total.max()), D)
        s["table"] = None
    for x in ("k", "v"):
        if op == "append":                                  # a fresh pool
            s[x + "c"] = torch.zeros(shape, dtype=torch.float8_e4m3fn, device=dev)
            s[x + "s"] = torch.full(shape[:3], 127, dtype=torch.uint8, device=dev).view(torch.float8_e8m0fnu)
        else:
            rows = torch.randn(shape, generator=gen, device=dev)
            rows *= torch.exp(0.3 * torch.randn(shape[:3], generator=gen, device=dev))[..., None]
            s[x + "c"], s[x + "s"] = _quantise(rows)
            del rows
    if op == "read":
        n = int(lens.max())
        s["k_out"], s["v_out"] = (torch.zeros((B, n, Hkv, D), dtype=dt, device=dev) for _ in range(2))
    if op == "compact":
        # the way from the root to a node; its nodes but the root lie behind the rows that it moves to, so that a second pass over the
        # same rows moves the same ones
        paths, n_acc = np.zeros((B, 8), dtype=np.int32), np.zeros(B, dtype=np.int32)
        ways = []
        for node in range(T):
            way = []
            while node >= 0:
                way.append(node)
                node = int(trees[node])
            if all(x >= len(way) for x in way[:-1]):
                ways.append(way[::-1])
        for b in range(B):
            way = ways[int(rng.integers(0, len(ways)))]
            paths[b, :len(way)], n_acc[b] = way, len(way)
        s["paths"], s["n_acc"], s["lens_out"] = up(paths), up(n_acc), torch.empty_like(s["lens"])
    if op == "fwd":
        s["q"] = normal(B, T, Hq, D)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((B, Hq, T), dtype=torch.float32, device=dev)
    return s


# ----------------------------------------------------------------------------- the plain form

def _ancestors(parent, T):
    """[.., T, T]: does column j lie on the way from the root to row i, i included?"""
    step = torch.eye(T, device=parent.device) + (parent[..., None] == torch.arange(T, device=parent.device))
    return torch.linalg.matrix_power(step, T) > 0


def _positions(s):
    T = s["case"]["T"]
    if s["case"]["tree"] == "line":
        depth = torch.arange(T, device=s["lens"].device)
    else:
        depth = _ancestors(s["parent"], T).sum(-1) - 1
    return s["lens"].long()[:, None] + depth                # [B, T]


def _rotate(x, pos, freqs, interleaved):
    R = 2 * freqs.shape[0]
    angle = pos.double()[..., None] * freqs.double()        # far positions need 64 bits
    c, sn = angle.cos().float()[:, :, None, :], angle.sin().float()[:, :, None, :]
    head, rest = x[..., :R].float(), x[..., R:]
    a, b = (head[..., 0::2], head[..., 1::2]) if interleaved else (head[..., :R // 2], head[..., R // 2:])
    u, w = a * c - b * sn, b * c + a * sn
    head = torch.stack((u, w), -1).flatten(-2) if interleaved else torch.cat((u, w), -1)
    return torch.cat((head.to(x.dtype), rest), -1)


def _rows(s, pos):
    """Page and slot of logical positions [B, n]."""
    if s["table"] is None:
        return torch.arange(pos.shape[0], device=pos.device)[:, None].expand_as(pos), pos
    ps = s["case"]["ps"]
    return s["table"].long().gather(1, pos // ps), pos % ps


def _gathered(codes, scales, page, slot):
    """Rows [B, n, Hkv, D] of the cache, float32."""
    scale = scales.view(torch.uint8)[page, :, slot].view(torch.float8_e8m0fnu).float()
    return codes.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).float() * scale[..., None]


def _plain(s):
    case = s["case"]
    op, B, Hq, Hkv, D, T = (case[k] for k in ("op", "B", "Hq", "Hkv", "D", "T"))
    dev = s["lens"].device
    if op == "rope":
        pos = _positions(s)
        return [_rotate(s["q"], pos, s["freqs"], case["interleaved"]), _rotate(s["k"], pos, s["freqs"], case["interleaved"])]
    if op == "append":
        out, k = [], s["k"]
        if case["rotate"]:
            pos = _positions(s)
            out.append(_rotate(s["q"], pos, s["freqs"], case["interleaved"]))
            k = _rotate(k, pos, s["freqs"], case["interleaved"])
        page, slot = _rows(s, s["lens"].long()[:, None] + torch.arange(T, device=dev))
        for rows, codes, scales in ((k, s["kc"], s["ks"]), (s["v"], s["vc"], s["vs"])):
            for x, held in zip(_quantise(rows.float()), (codes, scales)):
                held.view(torch.uint8)[page, :, slot] = x.view(torch.uint8)
        return out + [s["kc"], s["ks"], s["vc"], s["vs"]]
    if op == "read":
        n = s["k_out"].shape[1]
        at = torch.arange(n, device=dev).expand(B, n)
        page, slot = _rows(s, at.minimum(s["lens"].long()[:, None] - 1).clamp_min(0))
        there = (at < s["lens"][:, None])[..., None, None]
        for out, codes, scales in ((s["k_out"], s["kc"], s["ks"]), (s["v_out"], s["vc"], s["vs"])):
            out.copy_(torch.where(there, _gathered(codes, scales, page, slot), out.float()))
        return [s["k_out"], s["v_out"]]
    if op == "compact":
        A = s["paths"].shape[1]
        at = torch.arange(A, device=dev).expand(B, A)
        live = at < s["n_acc"][:, None]
        lens = s["lens"].long()[:, None]
        sp, ss = _rows(s, lens + torch.where(live, s["paths"].long(), 0))
        dp, ds = _rows(s, lens + torch.where(live, at, 0))              # (an entry past the path's end: the root onto itself)
        for x in (s["kc"], s["vc"], s["ks"], s["vs"]):
            x = x.view(torch.uint8)
            x[dp, :, ds] = x[sp, :, ss]
        s["lens_out"].copy_(s["lens"] + s["n_acc"])
        return [s["kc"], s["ks"], s["vc"], s["vs"], s["lens_out"]]
    lens = s["lens"].long()
    n = int(case["L1"]) + T
    at = torch.arange(n, device=dev).expand(B, n)
    page, slot = _rows(s, at.minimum(lens[:, None] + T - 1))
    G = Hq // Hkv
    q = s["q"].float().view(B, T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, D)
    k = _gathered(s["kc"], s["ks"], page, slot).permute(0, 2, 3, 1).contiguous()
    score = torch.matmul(q, k).view(B, Hkv, T, G, n) * (1.0 / math.sqrt(D))
    del k
    node = at - lens[:, None]                               # of the tree; negative in the prefix
    seen = _ancestors(s["parent"], T).expand(B, T, T).gather(2, node.clamp(0, T - 1)[:, None].expand(B, T, n))
    seen = (seen & (node < T)[:, None]) | (node < 0)[:, None]
    score.masked_fill_(~seen[:, None, :, None], -math.inf)
    m = score.amax(-1, keepdim=True)
    p = torch.exp_(score.sub_(m))
    total = p.sum(-1, keepdim=True)
    v = _gathered(s["vc"], s["vs"], page, slot).permute(0, 2, 1, 3).contiguous()
    out = torch.matmul(p.view(B, Hkv, T * G, n), v).view(B, Hkv, T, G, D) / total
    lse = (m + total.log()).view(B, Hkv, T, G)
    return [out.permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D).to(s["q"].dtype), lse.permute(0, 1, 3, 2).reshape(B, Hq, T)]


# ----------------------------------------------------------------------------- one pass

def run(s):
    if not own:
        return _plain(s)
    from paper_2508_08192_amd import treeattn as ta
    case = s["case"]
    op = case["op"]
    if op == "rope" or case["rotate"]:
        parent = None if case["tree"] == "line" else s["parent"]
    if op == "rope":
        ta.tree_attn_rope(s["q"], s["k"], s["freqs"], s["lens"], parent, s["q_out"], s["k_out"],
                          interleaved=case["interleaved"])
        return [s["q_out"], s["k_out"]]
    cache = (s["kc"], s["vc"], s["ks"], s["vs"], s["table"])
    if op == "append":
        if case["rotate"]:
            ta.tree_attn_q8_rope_append(s["q"], s["k"], s["v"], s["freqs"], s["lens"], parent, s["q_out"], *cache,
                                        interleaved=case["interleaved"])
            return [s["q_out"], s["kc"], s["ks"], s["vc"], s["vs"]]
        ta.tree_attn_q8_append(s["k"], s["v"], *cache, s["lens"])
        return [s["kc"], s["ks"], s["vc"], s["vs"]]
    if op == "read":
        ta.tree_attn_q8_read(*cache, None, s["lens"], s["k_out"], s["v_out"])
        return [s["k_out"], s["v_out"]]
    if op == "compact":
        ta.tree_attn_q8_compact(*cache, s["lens"], s["paths"], s["n_acc"], case["T"], s["lens_out"])
        return [s["kc"], s["ks"], s["vc"], s["vs"], s["lens_out"]]
    ta.tree_attn_q8_fwd(s["q"], *cache, s["lens"], s["parent"], s["out"], s["lse"])
    return [s["out"], s["lse"]]


def work(case):
    """Bytes and operations that one pass cannot do without."""
    op, B, Hq, Hkv, D, T, ps = (case[k] for k in ("op", "B", "Hq", "Hkv", "D", "T", "ps"))
    es = 2 if case["dtype"] == "bf16" else 4
    lens = _lengths(case)
    row = Hkv * (D + 1) * 2                                 # a token's codes and scales
    dense = Hkv * D * es
    meta = 4 * B + (4 * B * T if case["tree"] == "dynamic" else 4 * T)
    if op == "rope":
        return {"bytes": int(2 * B * T * (Hq + Hkv) * D * es + 2 * case["R"] + meta), "flops": int(3 * B * T * (Hq + Hkv) * case["R"])}
    if op == "append":
        size, flops = B * T * (2 * dense + row), 2 * B * T * 2 * Hkv * D
        if case["rotate"]:
            size, flops = size + 2 * B * T * Hq * D * es, flops + 3 * B * T * (Hq + Hkv) * case["R"]
        return {"bytes": int(size + meta + 4 * B * (T // (ps or T) + 1)), "flops": int(flops)}
    if op == "read":
        n = int(lens.sum())
        return {"bytes": int(n * (row + 2 * dense) + 4 * (n // (ps or n) + B)), "flops": int(n * Hkv * D * 2)}
    if op == "compact":
        return {"bytes": int(B * (2 * 3 * row + 4 * (8 + 4))), "flops": 0}          # three rows or so of a path move
    n = int(lens.sum()) + B * T
    size = n * row + 2 * B * T * Hq * D * es + 4 * B * T * Hq + meta + (4 * n // ps if ps else 0)
    return {"bytes": int(size), "flops": int(4 * D * Hq * (T * int(lens.sum()) + B * T * min(T, 5)))}


# ----------------------------------------------------------------------------- from the definitions, in 64 bits

def _parents_up(parent, node):
    way = []
    while node >= 0:
        way.append(node)
        node = int(parent[node])
    return way


def exact(case, seed):
    """What run() returns, from each operator's definition in float64; codes as the values that e4m3 has to round."""
    s = prepare(case, seed)
    op, B, Hq, Hkv, D, T, ps = (case[k] for k in ("op", "B", "Hq", "Hkv", "D", "T", "ps"))
    lens = s["lens"].tolist()
    dev = s["lens"].device
    table = None if op == "rope" or s["table"] is None else s["table"].long()
    trees = s["parent"].cpu().numpy()

    def ways(b):
        tree = trees if trees.ndim == 1 else trees[b]
        return [_parents_up(tree, i) for i in range(T)]

    def place(b, pos):
        if table is None:
            return torch.full_like(pos, b), pos
        return table[b][torch.div(pos, ps, rounding_mode="floor")], torch.remainder(pos, ps)

    def turned(x):
        """x [B, T, H, D] at its positions, one complex number per pair."""
        f = s["freqs"].double()
        R = 2 * len(f)
        y = x.double().clone()
        for b in range(B):
            if case["tree"] == "line":
                at = lens[b] + torch.arange(T, device=dev, dtype=torch.float64)
            else:
                at = lens[b] + torch.tensor([len(w) - 1.0 for w in ways(b)], device=dev, dtype=torch.float64)
            turn = torch.polar(torch.ones_like(at[:, None] * f), at[:, None] * f)[:, None]
            lo, hi = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
            z = torch.complex(y[b, :, :, lo], y[b, :, :, hi]) * turn
            y[b, :, :, lo], y[b, :, :, hi] = z.real, z.imag
        return y

    def values(c, sc, b, pos):
        page, slot = place(b, pos)
        power = sc.view(torch.uint8)[page, :, slot].double() - 127.0
        return c.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).double() * torch.exp2(power)[..., None]

    if op == "rope":
        return [turned(s["q"]), turned(s["k"])]
    if op == "append":
        out, k = [], s["k"].double()
        if case["rotate"]:
            out.append(turned(s["q"]))
            k = turned(s["k"]).to(s["k"].dtype).double()    # rounded to the type of the keys before it is quantised
        for rows, c, sc in ((k, s["kc"], s["ks"]), (s["v"].double(), s["vc"], s["vs"])):
            c, sc = c.double(), sc.double()
            for b in range(B):
                page, slot = place(b, lens[b] + torch.arange(T, device=dev))
                top = rows[b].abs().amax(-1)
                scale = torch.exp2(torch.ceil(torch.log2(top / 448.0)).clamp_min(-126.0))
                scale = torch.where(top > 0, scale, torch.ones_like(scale))
                c[page, :, slot], sc[page, :, slot] = rows[b] / scale[..., None], scale
            out += [c, sc]
        return out
    if op == "read":
        out = []
        for c, sc, dense in ((s["kc"], s["ks"], s["k_out"]), (s["vc"], s["vs"], s["v_out"])):
            dense = dense.double()
            for b in range(B):
                dense[b, :lens[b]] = values(c, sc, b, torch.arange(lens[b], device=dev))
            out.append(dense)
        return out
    if op == "compact":
        kc, ks, vc, vs = s["kc"].double(), s["ks"].double(), s["vc"].double(), s["vs"].double()
        paths, n_acc = s["paths"].tolist(), s["n_acc"].tolist()
        for x in (kc, ks, vc, vs):
            for b in range(B):
                n = n_acc[b]
                sp, ss = place(b, lens[b] + torch.tensor(paths[b][:n], device=dev))
                dp, ds = place(b, lens[b] + torch.arange(n, device=dev))
                x[dp, :, ds] = x[sp, :, ss].clone()
        return [kc, ks, vc, vs, torch.tensor([a + n for a, n in zip(lens, n_acc)], device=dev, dtype=torch.int32)]
    out = torch.empty((B, T, Hq, D), dtype=torch.float64, device=dev)
    lse = torch.empty((B, Hq, T), dtype=torch.float64, device=dev)
    G = Hq // Hkv
    for b in range(B):
        n = lens[b] + T
        pos = torch.arange(n, device=dev)
        K, V = values(s["kc"], s["ks"], b, pos), values(s["vc"], s["vs"], b, pos)
        seen = torch.zeros((T, n), dtype=torch.bool, device=dev)
        seen[:, :lens[b]] = True
        for i, way in enumerate(ways(b)):
            seen[i, [lens[b] + j for j in way]] = True
        for g in range(Hkv):
            q = s["q"][b, :, g * G:(g + 1) * G].double().reshape(T * G, D)
            score = (q @ K[:, g].t().contiguous()).view(T, G, n) / math.sqrt(D)
            score = torch.where(seen[:, None], score, torch.full_like(score, -math.inf))
            z = torch.logsumexp(score, -1)
            out[b, :, g * G:(g + 1) * G] = (torch.exp(score - z[..., None]).view(T * G, n) @ V[:, g].contiguous()).view(T, G, D)
            lse[b, g * G:(g + 1) * G] = z.t()
    return [out, lse]

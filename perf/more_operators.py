"""What is measured of the operators round a K/V cache in 8 bits, and their plain forms.

The set: the norm of each query and key head with its position rotation (positions of one to three axes: time, height,
width), which makes the rows that a step attends with and appends; the copy of K/V rows into a cache in 8 bits with a
power of two as the scale of each block of tokens and head; and the attention of a step's query nodes over such a cache.

Shapes: 4 KV heads x 128 with 28 query heads, and 2 KV heads x 64 with 14, 28 layers; sequence lengths are those of this
repository's workloads (8 to 256 frames of 196 or 169 tokens plus text), whole or at the share that pruning keeps.
Caches are [layers, 2, heads, rows, head_dim]; scales are [layers, 2, heads, blocks], bytes x that stand for 2 ** (x - 127).

`own = False`: elementary torch operations, in 32 bits (angles in 64), rounded once at the end.
`own = True`: the calls that a user makes.
"""
import functools
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn, "i8": torch.int8}
# the largest value of a code as m * 2 ** x with m in [0.5, 1)
TOP = {"e4m3": (0.875, 9), "i8": (0.9921875, 7)}
LEAST, MOST = -48, 48           # exponents of a scale


@functools.lru_cache(None)
def _sv():
    from paper_2511_08003_b200 import binding
    return binding


# ------------------------------------------------------------------------------------------ the cases
def _text(v):
    return ",".join(str(int(x)) for x in v)


def _ints(s):
    return [int(x) for x in s.split(",")]


# cached rows of the 16 videos of the ragged serving batch (8, 16, 32 or 64 frames of 196 tokens, 64 text
# tokens), at the share of the rows that stage two keeps, about 0.39
_RAGGED = [(int(8 * 2 ** e) * 196 * 39) // 100 + 64 for e in (0, 3, 1, 2, 2, 0, 3, 1, 1, 0, 2, 3, 0, 1, 3, 2)]
_LONG = 256 * 196 + 256
_TREES = [5, 24, 17, 33, 8, 41, 20, 13, 29, 6, 37, 12, 25, 9, 16, 31]


def _rope(name, dtype, H, G, D, tokens, sections, mixed, norm):
    return {"name": name, "op": "rope", "dtype": dtype, "kv_heads": H, "group": G, "head_dim": D, "tokens": tokens,
            "sections": _text(sections), "mixed": mixed, "norm": norm}


def _store(name, source, code, block, layers, H, D, rows, lens, spare, part):
    return {"name": name, "op": "store", "source": source, "code": code, "block": block, "layers": layers, "kv_heads": H,
            "head_dim": D, "rows": _text(rows), "lens": _text(lens), "spare": spare, "part": part}


def _attn(name, code, block, H, G, D, lens, nodes, tree):
    return {"name": name, "op": "attention", "code": code, "block": block, "kv_heads": H, "group": G, "head_dim": D,
            "lens": _text(lens), "nodes": _text(nodes), "tree": tree}


def listed():
    return [
        # one decoded token per sequence of the ragged serving batch: a call whose time is latency
        _rope("rope tokens", "bf16", 4, 7, 128, 16, [16, 24, 24], False, True),
        # the whole prompt of the 8-frame video in fp32, plain rotation (one axis), no norm
        _rope("rope prompt f32", "f32", 2, 7, 64, 8 * 196 + 32, [32], False, False),
        # the whole prompt of the 256-frame video, axes taking the pairs in turn
        _rope("rope prompt long", "bf16", 4, 7, 128, _LONG, [22, 21, 21], True, True),
        # the accepted path (1 to 6 nodes) of every tree of the ragged batch into all 28 layers, behind rows that are
        # in the first block already
        _store("store accepted", "bf16", "e4m3", 64, 28, 4, 128, [2, 4, 1, 6, 3, 1, 5, 2, 2, 1, 3, 6, 4, 1, 2, 5],
               [300, 901, 450, 640, 700, 310, 880, 420, 460, 330, 650, 910, 350, 470, 905, 620], 294, True),
        # the kept rows of the ragged batch out of the cache that the prompt left, all 28 layers
        _store("store pruned", "bf16", "e4m3", 64, 28, 4, 128, _RAGGED, [0] * 16, 20000, True),
        # the rows that stay when the ragged batch is over its budget, from one cache in 8 bits to another
        _store("store evicted", "i8", "i8", 32, 28, 4, 128, [n // 2 for n in _RAGGED], [0] * 16, sum(_RAGGED) // 2, True),
        # one decoded token over the cache of the 8-frame video: latency
        _attn("attn token tiny", "i8", 32, 2, 7, 64, [8 * 196 + 32], [1], False),
        # one decoded token per sequence of the ragged serving batch, after pruning
        _attn("attn token ragged", "e4m3", 64, 4, 7, 128, _RAGGED, [1] * 16, False),
        # one decoded token over the unpruned cache of the 256-frame video
        _attn("attn token long", "e4m3", 64, 4, 7, 128, [_LONG], [1], False),
        # a tree of 64 drafted tokens over the same cache
        _attn("attn tree long", "e4m3", 64, 4, 7, 128, [_LONG], [64], True),
        # trees of 5 to 41 drafted tokens over the ragged batch
        _attn("attn tree ragged", "i8", 32, 4, 7, 128, _RAGGED, _TREES, True),
        # a chunk of 509 question tokens (causal) over the cache of a 64-frame video
        _attn("attn chunk", "e4m3", 128, 4, 7, 128, [64 * 169 + 128], [509], False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "store", "attention", "attention"])
    while True:
        H, G = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8])
        if op == "rope":
            D, axes = rng.choice([64, 80, 96, 128, 128, 256]), rng.choice([1, 2, 3, 3])
            pairs = rng.choice([D // 2, D // 2, D // 32 * 8])
            first = pairs // 4 if axes > 1 else pairs
            second = (pairs - first) // (axes - 1) if axes > 1 else 0
            sections = [first, second, pairs - first - second][:axes]
            sections[-1] = pairs - sum(sections[:-1])
            mixed = rng.random() < 0.4
            if mixed:
                sections = [len(range(a, pairs, axes)) for a in range(axes)]
            c = _rope("", rng.choice(["bf16", "bf16", "f32"]), H, G, D, _log(rng, 1, _LONG), sections, mixed, rng.random() < 0.7)
            if work(c)["bytes"] > 8.3e8:
                continue
        elif op == "store":
            B, layers, D = rng.choice([1, 2, 5, 16]), rng.choice([1, 4, 24, 28]), rng.choice([64, 80, 96, 128, 128, 256])
            rows = [_log(rng, 1, 12000) if rng.random() < 0.9 else 0 for _ in range(B)]
            code, fresh = rng.choice(["e4m3", "i8"]), rng.random() < 0.5
            c = _store("", rng.choice(["bf16", "bf16", "f32", "e4m3", "i8"]), code, rng.choice([1, 16, 32, 64, 128, 256]), layers, H,
                       D, rows, [0 if fresh else _log(rng, 1, 4000) for _ in range(B)], rng.choice([0, 37, 1000]), rng.random() < 0.7)
            if sum(rows) == 0 or work(c)["bytes"] > 3.2e9 or layers * 2 * H * D * (sum(rows) * 2 + sum(_ints(c["lens"]))) > 4e9:
                continue
        else:
            D, B = rng.choice([64, 128, 128, 80, 96, 256]), rng.choice([1, 1, 2, 3, 7, 16])
            lens = [_log(rng, 1, _LONG) if rng.random() < 0.95 else 0 for _ in range(B)]
            one = rng.random() < 0.4
            nodes = [1 if one else _log(rng, 1, 512) for _ in range(B)]
            if max(lens) == 0:
                continue
            c = _attn("", rng.choice(["e4m3", "e4m3", "i8"]), rng.choice([1, 16, 32, 64, 128, 256]), H, G, D, lens, nodes,
                      max(nodes) <= 128 and rng.random() < 0.6)
            w = work(c)
            padded = B * max(nodes) * G * H * (max(lens) + max(nodes))
            if padded * D > 28 * 64 * _LONG * 128 or w["flops"] > 4.6e10 or w["bytes"] > 6e7 or \
                    B * max(lens) * H * D > 4 * 128 * 2 * _LONG:
                continue
        del c["name"]
        return c


def _width(kind):
    return torch.empty((), dtype=DTYPES[kind]).element_size()


def work(case):
    H, D = case["kv_heads"], case["head_dim"]
    if case["op"] == "rope":
        n, heads = case["tokens"], H * (case["group"] + 1)
        rotated = 2 * sum(_ints(case["sections"]))
        return {"bytes": 2 * n * heads * D * _width(case["dtype"]) + 4 * n * len(_ints(case["sections"])),
                "flops": n * heads * (3 * rotated + (4 * D if case["norm"] else 0))}
    if case["op"] == "store":
        planes, n = case["layers"] * 2 * H, sum(_ints(case["rows"]))
        blocks = sum((a % case["block"] + b + case["block"] - 1) // case["block"] for a, b in zip(_ints(case["lens"]), _ints(case["rows"])) if b)
        return {"bytes": n * planes * D * (_width(case["source"]) + 1) + planes * blocks + 4 * n, "flops": 0}
    lens, nodes, G = _ints(case["lens"]), _ints(case["nodes"]), case["group"]
    N, pairs = sum(nodes), sum(a * b for a, b in zip(lens, nodes))
    # of the drafted tokens a node sees at least itself; a causal chain half of them
    own_pairs = N if case["tree"] else sum(n * (n + 1) // 2 for n in nodes)
    return {"bytes": 2 * H * (sum(lens) * D + sum(-(-n // case["block"]) for n in lens)) + 4 * N * H * D + N * H * G * (4 * D + 4),
            "flops": 4 * (pairs + own_pairs) * H * G * D}


# ------------------------------------------------------------------------------------------ the inputs
def _table(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _starts(v):
    return np.concatenate([[0], np.cumsum(v)]).astype(np.int64)


def _up(n, block):
    return -(-n // block) * block


def _tree_bits(nodes, rng):
    """Random trees: a node's parent is one of the 8 nodes before it.  Bit j of row i: node i sees node j,
    that is itself and its ancestors."""
    words = (max(nodes) + 31) // 32
    rows = []
    for n in nodes:
        seen = np.zeros((n, words * 32), np.uint8)
        for i in range(n):
            p = int(rng.integers(max(-1, i - 8), i)) if i else -1
            if p >= 0:
                seen[i] = seen[p]
            seen[i, i] = 1
        rows.append(np.packbits(seen, axis=1, bitorder="little").view("<u4"))
    return np.concatenate(rows).view(np.int32)


def _values(shape, g, dtype):
    """K/V rows [layers, 2, heads, rows, D]: some channels of a head far larger than the others, some rows far smaller
    (the first tokens' values are, in earnest)."""
    x = torch.randn(shape, generator=g, device=DEV, dtype=dtype)
    x *= torch.exp(0.7 * torch.randn((*shape[:3], 1, shape[4]), generator=g, device=DEV)).to(dtype)
    x *= torch.where(torch.rand(shape[3], generator=g, device=DEV) < 0.03, 0.02, 1.0).to(dtype)[:, None]
    return x


def _held(shape, code, block, g):
    """A cache in 8 bits with its scales, as rows of `_values` leave it: [layers, 2, heads, blocks * block, D]."""
    L, two, H, T, D = shape
    x = _values(shape, g, torch.float32).view(L, two, H, T // block, block, D)
    e = _exponent(x.abs().amax((4, 5)), code)
    return _code(x * _two(-e)[..., None, None], code).view(shape), (e + 127).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    rng = np.random.default_rng(int(seed))
    H, D = case["kv_heads"], case["head_dim"]
    if case["op"] == "rope":
        n, dt, HQ = case["tokens"], DTYPES[case["dtype"]], H * case["group"]
        sections = _ints(case["sections"])
        # the fused projection's output: queries, keys and values of a token side by side
        qkv = torch.randn((n, HQ + 2 * H, D), generator=g, device=DEV, dtype=dt)
        qkv *= torch.exp(0.5 * torch.randn((HQ + 2 * H, D), generator=g, device=DEV)).to(dt)
        # positions of a video's tokens: frame, row and column on a grid of 14 x 14, behind some text
        at = np.arange(n) + int(rng.integers(0, 40000 if n < 1000 else 100))
        positions = np.stack([at if len(sections) == 1 else at // 196 + 17, at % 196 // 14 + 17, at % 14 + 17][:len(sections)])
        axis = np.arange(sum(sections)) % len(sections) if case["mixed"] else np.repeat(np.arange(len(sections)), sections)
        weight = (1 + 0.3 * torch.randn((2, D), generator=g, device=DEV)).to(dt)
        return {"case": case, "q": qkv[:, :HQ], "k": qkv[:, HQ:HQ + H], "positions": _table(positions),
                "pair_axis": [int(a) for a in axis], "axis": torch.from_numpy(axis).to(DEV), "weight": weight, "base": 1e6, "eps": 1e-6}
    block, code = case["block"], case["code"]
    if case["op"] == "store":
        rows, lens, L = _ints(case["rows"]), _ints(case["lens"]), case["layers"]
        begin = _starts([_up(a + b, block) + block for a, b in zip(lens, rows)])
        n = sum(rows)
        # a list in ascending order out of the source's rows (what pruning keeps, or the accepted nodes)
        pos = np.sort(rng.permutation(n + case["spare"])[:n]) if case["part"] else np.arange(n)
        source, scales = n + case["spare"], None
        if case["source"] in TOP:
            src, scales = _held((L, 2, H, _up(source, block), D), case["source"], block, g)
        else:
            src = _values((L, 2, H, source, D), g, DTYPES[case["source"]])
        # rows in front of the new ones: smaller by half, so that some blocks need a larger scale afterwards
        dst = torch.zeros((L, 2, H, int(begin[-1]), D), dtype=DTYPES[code], device=DEV)
        held = torch.full((L, 2, H, int(begin[-1]) // block), 127, dtype=torch.uint8, device=DEV)
        in_front = np.concatenate([np.arange(b + a // block * block, b + a) for a, b, r in zip(lens, begin, rows) if r]) \
            if any(rows) else np.zeros(0)
        if len(in_front):
            old, e = _held((L, 2, H, int(begin[-1]), D), code, block, g)
            dst, held = old, e - 1
        return {"case": case, "src": src, "src_scales": scales, "dst": dst, "scales": held, "src_pos": _table(pos),
                "offsets": _table(_starts(rows)), "dst_begin": _table(begin[:-1] + np.asarray(lens)), "total": n,
                "in_front": torch.from_numpy(in_front.astype(np.int64)).to(DEV)}
    lens, nodes, G = _ints(case["lens"]), _ints(case["nodes"]), case["group"]
    B, N = len(lens), sum(nodes)
    # every sequence's region begins at a block, with some blocks behind the last one
    off = _starts([_up(n, block) for n in lens])
    kv, scales = _held((1, 2, H, _up(int(off[-1]) + 24, block), D), code, block, g)
    q = torch.randn((N, H * G, D), generator=g, device=DEV, dtype=torch.float32) * 0.6
    # every head has a direction that some rows answer to: such rows take much of the weight, as the first tokens of a
    # prompt do
    heavy = [int(b + i) for b, n in zip(off[:-1], lens) for i in list(range(min(n, 2))) + [int(x) for x in rng.integers(0, max(n, 1), 6)] if n]
    axis = torch.randn((H, 1, D), generator=g, device=DEV)
    axis = axis / axis.norm(dim=-1, keepdim=True)
    rows = torch.tensor(heavy, device=DEV)
    keys, unit = kv[0, 0].view(torch.uint8), _two(scales[0, 0][:, rows // block].int() - 127)[..., None]
    keys[:, rows] = _code((0.3 * keys[:, rows].view(kv.dtype).float() * unit + 5 * axis) / unit, code).view(torch.uint8)
    q = (q + axis.repeat_interleave(G, 0).transpose(0, 1) * 6).to(torch.bfloat16)
    return {"case": case, "kv": kv, "scales": scales, "q": q, "seq_begin": _table(off[:-1]), "seq_len": _table(lens),
            "node_offsets": _table(_starts(nodes)), "longest": max(lens), "most": max(nodes),
            "draft": torch.randn((2, N, H, D), generator=g, device=DEV, dtype=torch.bfloat16),
            "tree": torch.from_numpy(_tree_bits(nodes, rng)).to(DEV) if case["tree"] else None}


# ------------------------------------------------------------------------------------------ the plain forms
def _two(e):
    """2 ** e, exactly."""
    return ((e.int().clamp(-126, 127) + 127) << 23).view(torch.float32)


def _exponent(top, code):
    """The least e with top <= largest code * 2 ** e, in [LEAST, MOST]; LEAST for 0."""
    m, x = torch.frexp(top)
    most, at = TOP[code]
    return torch.where(top == 0, LEAST, x - at + (m > most).int()).clamp(LEAST, MOST)


def _code(x, code):
    """Nearest code, ties to even."""
    if code == "i8":
        return torch.round(x).clamp_(-128, 127).to(torch.int8)
    return x.clamp(-448, 448).to(torch.float8_e4m3fn)


def _plain_rope(st):
    c = st["case"]
    half = st["axis"].shape[0]
    freq = torch.pow(torch.tensor(st["base"], dtype=torch.float64, device=DEV),
                     -torch.arange(half, dtype=torch.float64, device=DEV) / half)
    angle = st["positions"].double()[st["axis"]].T * freq                     # [tokens, pairs]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(x, weight):
        x = x.float()
        if c["norm"]:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + st["eps"]) * weight.float()
        a, b = x[..., :half], x[..., half:2 * half]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * half:]], -1).to(st["q"].dtype)

    return {"q": turned(st["q"], st["weight"][0]), "k": turned(st["k"], st["weight"][1])}


def _plain_store(st):
    c = st["case"]
    block, code = c["block"], c["code"]
    j = torch.arange(st["total"], device=DEV)
    b = torch.searchsorted(st["offsets"], j, right=True) - 1
    to = st["dst_begin"][b] + j - st["offsets"][b]
    pos = st["src_pos"].long()
    if st["src_scales"] is None:
        x = st["src"][:, :, :, pos].float()
    else:
        x = st["src"].view(torch.uint8)[:, :, :, pos].view(st["src"].dtype).float()
        x = x * _two(st["src_scales"][:, :, :, pos // block].int() - 127)[..., None]
    blocks = st["scales"].shape[-1]
    at = (to // block).long()
    lead = x.shape[:3]
    top = torch.zeros((*lead, blocks), device=DEV).index_reduce_(3, at, x.abs().amax(-1), "amax")
    e = _exponent(top, code)
    touched = torch.zeros(blocks, dtype=torch.bool, device=DEV).index_fill_(0, at, True)
    front = st["in_front"]
    partly = torch.zeros(blocks, dtype=torch.bool, device=DEV).index_fill_(0, front // block, True)
    old = st["scales"].int() - 127
    e = torch.where(partly, torch.maximum(e, old), e)
    d = st["dst"].view(torch.uint8)
    again = d[:, :, :, front].view(st["dst"].dtype).float() * _two((old - e)[:, :, :, front // block])[..., None]
    d[:, :, :, front] = _code(again, code).view(torch.uint8)
    d[:, :, :, to.long()] = _code(x * _two(-e[:, :, :, at])[..., None], code).view(torch.uint8)
    st["scales"].copy_(torch.where(touched, e + 127, st["scales"]))
    return {"codes": st["dst"], "scales": st["scales"]}


def _pad(begin, count, most):
    """[B, most] rows begin + 0..most-1 (clamped to the first row where there is none) and which of them are there."""
    i = torch.arange(most, device=DEV)
    there = i < count[:, None]
    return torch.where(there, begin[:, None] + i, 0).long(), there


def _plain_attention(st):
    c = st["case"]
    H, G, off = c["kv_heads"], c["group"], st["node_offsets"]
    at, there = _pad(off[:-1], off[1:] - off[:-1], st["most"])
    n = at.shape[1]
    q = st["q"][at].float().view(*at.shape, H, G, -1).permute(2, 0, 1, 3, 4).reshape(H, at.shape[0], n * G, -1)
    t = torch.arange(st["q"].shape[0], device=DEV)
    b = torch.searchsorted(off, t, right=True) - 1
    rows, cached = _pad(st["seq_begin"], st["seq_len"], st["longest"])
    held = st["kv"][0].view(torch.uint8)[:, :, rows].view(st["kv"].dtype).float()
    k, v = held * _two(st["scales"][0][:, :, rows // c["block"]].int() - 127)[..., None]
    dk, dv = st["draft"][:, at].permute(0, 3, 1, 2, 4).float()
    if st["tree"] is None:
        sees = torch.ones((n, n), dtype=torch.bool, device=DEV).tril() & there[:, None, :]
    else:
        j = torch.arange(n, device=DEV)
        sees = ((st["tree"][at][:, :, j // 32] >> (j % 32)) & 1).bool() & there[:, None, :]
    s = torch.cat([(q @ k.transpose(-1, -2)).masked_fill_(~cached[:, None, :], -math.inf),
                   (q @ dk.transpose(-1, -2)).masked_fill_(~sees.repeat_interleave(G, 1), -math.inf)], -1)
    s *= c["head_dim"] ** -0.5
    top = s.amax(-1, keepdim=True).clamp_min(-3e38)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    o = p @ torch.cat([v.masked_fill_(~cached[:, :, None], 0), dv], -2) / torch.where(total == 0, 1.0, total)
    lse = torch.log(total) + top
    back = lambda x: x.view(H, -1, n, G, x.shape[-1])[:, b, t - off[b]].transpose(0, 1).reshape(b.shape[0], H * G, -1)  # noqa: E731
    return {"out": back(o).to(st["q"].dtype), "lse": back(lse)[..., 0]}


def run(state):
    op = state["case"]["op"]
    if own:
        sv = _sv()
        if op == "rope":
            norm = state["case"]["norm"]
            return sv.sharpv_qk_norm_rope(state["q"], state["k"], state["positions"], state["pair_axis"], state["base"],
                                          norm=norm, q_weight=state["weight"][0] if norm else None,
                                          k_weight=state["weight"][1] if norm else None, eps=state["eps"])
        if op == "store":
            sv.sharpv_kv_append_q8(state["src"], state["dst"], state["scales"], state["case"]["block"], state["src_pos"],
                                   state["offsets"], state["dst_begin"], src_scales=state["src_scales"])
            return {"codes": state["dst"], "scales": state["scales"]}
        return sv.sharpv_tree_attention_q8(state["q"], state["kv"], state["scales"], state["case"]["block"], 0,
                                           state["seq_begin"], state["seq_len"], state["node_offsets"], state["draft"][0],
                                           state["draft"][1], tree_mask=state["tree"])
    return {"rope": _plain_rope, "store": _plain_store, "attention": _plain_attention}[op](state)


# ------------------------------------------------------------------------------------------ in 64 bits
def _power(x):
    """2 ** x for whole x, by the bits of a 64-bit number."""
    return torch.bitwise_left_shift(x.long() + 1023, 52).view(torch.float64)


def _stood_for(codes, scales, block):
    """The values of a plane [rows, D] of codes with its scales."""
    rows = torch.arange(codes.shape[0], device=DEV)
    return codes.double() * _power(scales[rows // block].long() - 127)[:, None]


def _nearest(x, code):
    """Codes' values nearest to x, ties to even, by the spacing of the codes round x."""
    if code == "i8":
        lower = torch.floor(x)
        up = (x - lower > 0.5) | ((x - lower == 0.5) & (lower % 2 == 1))
        return (lower + up).clamp(-128, 127)
    # e4m3: eight steps between neighbouring powers of two, down to 2 ** -6
    step = _power((torch.frexp(x.abs()).exponent - 1).clamp(-6, 8) - 3)
    lower = torch.floor(x / step)
    rest = x / step - lower
    return ((lower + ((rest > 0.5) | ((rest == 0.5) & (lower % 2 == 1)))) * step).clamp(-448, 448)


def _exact_store(case, st):
    """One plane and sequence at a time."""
    block, code = case["block"], case["code"]
    most = 448.0 if code == "e4m3" else 127.0
    rows, off, begin = _ints(case["rows"]), _starts(_ints(case["rows"])), st["dst_begin"].tolist()
    codes, scales = st["dst"].double(), st["scales"].clone()
    L, _, H = codes.shape[:3]
    for plane in np.ndindex(L, 2, H):
        src = st["src"][plane]
        src = src.double() if st["src_scales"] is None else _stood_for(src, st["src_scales"][plane], block)
        for b, n in enumerate(rows):
            if not n:
                continue
            x = src[st["src_pos"][off[b]:off[b + 1]].long()]
            d0, first = begin[b], begin[b] // block
            last = (d0 + n - 1) // block
            padded = torch.zeros(((last - first + 1) * block, x.shape[1]), dtype=torch.float64, device=DEV)
            padded[d0 - first * block:d0 - first * block + n] = x
            top = padded.abs().view(last - first + 1, -1).amax(1)
            e = torch.where(top == 0, -48.0, torch.ceil(torch.log2(top.clamp_min(1e-30) / most)))
            # the logarithm is off by a rounding at a power of two: one step either way is put right
            e = e + (top > most * _power(e)).double() - ((top <= most * _power(e - 1)) & (top > 0)).double()
            e = e.clamp(-48, 48)
            lead = d0 - first * block
            if lead:
                was = scales[plane][first].double() - 127
                e[0] = torch.maximum(e[0], was)
                old = codes[plane][first * block:d0] * _power(was - e[0])
                codes[plane][first * block:d0] = _nearest(old, code)
            of = torch.arange(lead, lead + n, device=DEV) // block
            codes[plane][d0:d0 + n] = _nearest(x * _power(-e[of])[:, None], code)
            scales[plane][first:last + 1] = (e + 127).to(torch.uint8)
    return {"codes": codes, "scales": scales}


def exact(case, seed):
    """The definitions, one head (or plane) and sequence at a time."""
    st = prepare(case, seed)
    H, D, G = case["kv_heads"], case["head_dim"], case.get("group")
    if case["op"] == "store":
        return _exact_store(case, st)
    if case["op"] == "rope":
        half = len(st["pair_axis"])
        got = {"q": torch.empty(st["q"].shape, dtype=torch.float64, device=DEV),
               "k": torch.empty(st["k"].shape, dtype=torch.float64, device=DEV)}
        for name, weight in (("q", st["weight"][0]), ("k", st["weight"][1])):
            for h in range(st[name].shape[1]):
                x = st[name][:, h].double()
                if case["norm"]:
                    x = x / torch.sqrt((x * x).sum(1, keepdim=True) / D + st["eps"]) * weight.double()
                # a pair as a complex number
                z = torch.complex(x[:, :half], x[:, half:2 * half])
                turn = torch.stack([st["positions"][a].double() * st["base"] ** (-i / half) for i, a in enumerate(st["pair_axis"])], 1)
                z = z * torch.polar(torch.ones_like(turn), turn)
                got[name][:, h] = torch.cat([z.real, z.imag, x[:, 2 * half:]], 1)
        return got
    lens, nodes = _ints(case["lens"]), _ints(case["nodes"])
    at, begin = _starts(nodes), st["seq_begin"].tolist()
    q = st["q"].double()
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    for h in range(H):
        ks, vs = (_stood_for(st["kv"][0, i, h], st["scales"][0, i, h], case["block"]) for i in range(2))
        for b, n in enumerate(lens):
            r, t = slice(begin[b], begin[b] + n), slice(int(at[b]), int(at[b + 1]))
            if case["tree"]:
                bits = np.unpackbits(st["tree"][t].cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :nodes[b]]
            else:
                bits = np.tri(nodes[b])
            sees = torch.cat([torch.ones((nodes[b], n)), torch.from_numpy(bits.astype(np.float32))], 1).bool().to(DEV)
            k = torch.cat([ks[r], st["draft"][0, t, h].double()])
            v = torch.cat([vs[r], st["draft"][1, t, h].double()])
            for x in range(h * G, (h + 1) * G):
                s = torch.where(sees, q[t, x] @ k.T / math.sqrt(D), -math.inf)
                lse[t, x] = torch.logsumexp(s, 1)
                out[t, x] = torch.softmax(s, 1) @ v
    return {"out": out, "lse": lse}

"""What is measured of the operators that decode over a pruned K/V cache, and their plain forms.

The set: attention of drafted tokens (a tree, a chain, one token) over the cached rows, the attention
weight that every cached row collects from those tokens, the choice of the rows that stay when the cache is
over its budget, and the copy of accepted tokens' rows (or of whole packed sequences) into a cache whose
sequences have room to grow.

Shapes: 4 KV heads x 128 with 28 query heads, and 2 KV heads x 64 with 14, 28 layers; sequence lengths are
those of this repository's workloads (8 to 256 frames of 196 or 169 tokens plus text), whole or at the share
that pruning keeps.  Caches are [layers, 2, heads, rows, head_dim].

`own = False`: elementary torch operations on padded batches, in 32 bits, rounded once at the end.
`own = True`: the calls that a user makes.
"""
import functools
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


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


def _attn(name, dtype, H, G, D, lens, nodes, tree):
    return {"name": name, "op": "attention", "dtype": dtype, "kv_heads": H, "group": G, "head_dim": D,
            "lens": _text(lens), "nodes": _text(nodes), "tree": tree}


def _mass(name, dtype, H, G, D, lens, nodes, decay):
    return {"name": name, "op": "mass", "dtype": dtype, "kv_heads": H, "group": G, "head_dim": D,
            "lens": _text(lens), "nodes": _text(nodes), "decay": decay}


def _evict(name, lens, share, sink, recent):
    return {"name": name, "op": "evict", "lens": _text(lens), "share": share, "sink": sink, "recent": recent}


def _append(name, dtype, layers, H, D, source, rows, lens, unpack):
    return {"name": name, "op": "append", "dtype": dtype, "layers": layers, "kv_heads": H, "head_dim": D,
            "source": source, "rows": _text(rows), "lens": _text(lens), "unpack": unpack}


def listed():
    return [
        # one decoded token over the small fp32 cache (8 frames x 196 tokens + 32 text tokens): a call whose
        # time is latency
        _attn("attn token tiny f32", "f32", 2, 7, 64, [8 * 196 + 32], [1], False),
        # one decoded token per sequence of the ragged serving batch, after pruning
        _attn("attn token ragged", "bf16", 4, 7, 128, _RAGGED, [1] * 16, False),
        # one decoded token over the unpruned cache of the 256-frame video: every K and V row is read once
        _attn("attn token long", "bf16", 4, 7, 128, [_LONG], [1], False),
        # a tree of 64 drafted tokens over the same cache: 448 query rows on every K and V row
        _attn("attn tree long", "bf16", 4, 7, 128, [_LONG], [64], True),
        # trees of 5 to 41 drafted tokens over the ragged batch
        _attn("attn tree ragged", "bf16", 4, 7, 128, _RAGGED,
              [5, 24, 17, 33, 8, 41, 20, 13, 29, 6, 37, 12, 25, 9, 16, 31], True),
        # a chunk of 509 question tokens (causal) over the cache of a 64-frame video
        _attn("attn chunk", "bf16", 4, 7, 128, [64 * 169 + 128], [509], False),
        # the weight that one decoded token leaves on every row of the 256-frame cache
        _mass("mass token long", "bf16", 4, 7, 128, [_LONG], [1], 1.0),
        # the same for the accepted nodes of the ragged batch's trees (about a third of the nodes count)
        _mass("mass tree ragged", "bf16", 4, 7, 128, _RAGGED,
              [5, 24, 17, 33, 8, 41, 20, 13, 29, 6, 37, 12, 25, 9, 16, 31], 0.95),
        # the rows that stay of the ragged batch, half of each sequence
        _evict("evict ragged", _RAGGED, 0.5, 4, 64),
        # the rows that stay of the 256-frame cache, a quarter
        _evict("evict long", [_LONG], 0.25, 4, 256),
        # the accepted path (1 to 6 nodes) of every tree of the ragged batch into all 28 layers
        _append("append accepted", "bf16", 28, 4, 128, 326, [2, 4, 1, 6, 3, 1, 5, 2, 2, 1, 3, 6, 4, 1, 2, 5],
                [300, 901, 450, 640, 700, 310, 880, 420, 460, 330, 650, 910, 350, 470, 905, 620], False),
        # the pruned ragged batch, packed back to back, into regions with room for the answers
        _append("append unpack", "bf16", 28, 4, 128, sum(_RAGGED), _RAGGED, [0] * 16, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "mass", "mass", "evict", "append"])
    while True:
        if op in ("attention", "mass"):
            f32 = rng.random() < 0.25
            H, G = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8])
            D = rng.choice([64, 128, 128, 80, 96, 256])
            B = rng.choice([1, 1, 2, 3, 7, 16])
            lens = [_log(rng, 1, 12000 if f32 else _LONG) if rng.random() < 0.95 else 0 for _ in range(B)]
            most = 40 if f32 else 512
            one = rng.random() < 0.4
            nodes = [1 if one else _log(rng, 1, most) for _ in range(B)]
            if max(lens) == 0:
                continue
            c = (_attn("", "f32" if f32 else "bf16", H, G, D, lens, nodes, max(nodes) <= 128 and rng.random() < 0.6)
                 if op == "attention" else
                 _mass("", "f32" if f32 else "bf16", H, G, D, lens, nodes, rng.choice([1.0, 0.9, 0.0])))
            w = work(c)
            padded = B * max(nodes) * G * H * (max(lens) + max(nodes))
            if padded * D > 28 * 64 * _LONG * 128 or w["flops"] > 4.6e10 or w["bytes"] > 1.2e8 or \
                    B * max(lens) * H * D > 4 * 128 * 2 * _LONG:
                continue
        elif op == "evict":
            B = rng.choice([1, 2, 5, 16, 40])
            lens = [_log(rng, 1, _LONG) if rng.random() < 0.95 else 0 for _ in range(B)]
            c = _evict("", lens, round(rng.uniform(0.05, 1.0), 3), rng.choice([0, 1, 4, 16]), rng.choice([0, 1, 32, 256]))
            if B * max(lens) > 8 * _LONG or max(lens) == 0:
                continue
        else:
            B = rng.choice([1, 2, 5, 16])
            layers, H, D = rng.choice([1, 4, 24, 28]), rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 128])
            rows = [_log(rng, 1, 12000) if rng.random() < 0.9 else 0 for _ in range(B)]
            unpack = rng.random() < 0.5
            lens = [0 if unpack else _log(rng, 1, 4000) for _ in range(B)]
            c = _append("", rng.choice(["bf16", "f32"]), layers, H, D, sum(rows) + rng.choice([1, 37, 1000]), rows, lens, unpack)
            if sum(rows) == 0 or work(c)["bytes"] > 4e9 or 4 * layers * 2 * H * D * (sum(rows) * 2 + sum(lens)) > 8e9:
                continue
        del c["name"]
        return c


def work(case):
    if case["op"] == "evict":
        L = sum(_ints(case["lens"]))
        k = sum(_budgets(case))
        return {"bytes": 4 * L + 8 * k, "flops": 0}
    es = 2 if case["dtype"] == "bf16" else 4
    H, D = case["kv_heads"], case["head_dim"]
    if case["op"] == "append":
        return {"bytes": 2 * sum(_ints(case["rows"])) * case["layers"] * 2 * H * D * es, "flops": 0}
    lens, nodes, G = _ints(case["lens"]), _ints(case["nodes"]), case["group"]
    N, pairs = sum(nodes), sum(a * b for a, b in zip(lens, nodes))
    if case["op"] == "mass":
        return {"bytes": sum(lens) * H * D * es + N * H * G * (D * es + 4) + 4 * sum(lens) * (2 if case["decay"] else 1),
                "flops": 2 * pairs * H * G * D}
    # of the drafted tokens a node sees at least itself; a causal chain half of them
    own_pairs = N if case["tree"] else sum(n * (n + 1) // 2 for n in nodes)
    return {"bytes": 2 * (sum(lens) + N) * H * D * es + N * H * G * (2 * D * es + 4),
            "flops": 4 * (pairs + own_pairs) * H * G * D}


# ------------------------------------------------------------------------------------------ the inputs
def _table(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _starts(v):
    return np.concatenate([[0], np.cumsum(v)]).astype(np.int64)


def _budgets(case):
    return [min(n, int(round(n * case["share"]))) for n in _ints(case["lens"])]


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


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    rng = np.random.default_rng(int(seed))
    lens = _ints(case["lens"])
    B = len(lens)
    if case["op"] == "evict":
        off = _starts(lens)
        budget = _budgets(case)
        # accumulated weights: long-tailed, a few rows far above the rest, many of exactly the same (small) weight
        mass = torch.randn(int(off[-1]) + 1, generator=g, device=DEV).mul_(2.0).exp_()[:int(off[-1])]
        mass = torch.where(mass < 0.2, torch.round(mass * 32) / 32, mass)
        return {"case": case, "mass": mass, "seq_begin": _table(off[:-1]), "seq_len": _table(lens),
                "budget": _table(budget), "total": sum(budget), "longest": max(lens)}
    dt = DTYPES[case["dtype"]]
    H, D = case["kv_heads"], case["head_dim"]
    if case["op"] == "append":
        rows = _ints(case["rows"])
        room = [a + b + 16 for a, b in zip(lens, rows)]
        begin = _starts(room)
        src = torch.randn((case["layers"], 2, H, case["source"], D), generator=g, device=DEV, dtype=dt)
        dst = torch.zeros((case["layers"], 2, H, int(begin[-1]), D), device=DEV, dtype=dt)
        n = sum(rows)
        pos = np.arange(n) if case["unpack"] else np.sort(rng.permutation(case["source"])[:n])
        return {"case": case, "src": src, "dst": dst, "src_pos": _table(pos), "offsets": _table(_starts(rows)),
                "dst_begin": _table(begin[:-1] + np.asarray(lens)), "total": n}
    nodes, G = _ints(case["nodes"]), case["group"]
    N, off = sum(nodes), _starts(lens)
    # a cache with some rows behind the last sequence
    rows = int(off[-1]) + 24
    kv = torch.randn((1, 2, H, rows, D), generator=g, device=DEV, dtype=dt)
    q = torch.randn((N, H * G, D), generator=g, device=DEV, dtype=torch.float32) * 1.5
    # every head has a direction that the first rows of a sequence and a few rows in it answer to: such rows take
    # much of the weight, as the first tokens of a prompt do
    axis = torch.randn((H, 1, D), generator=g, device=DEV)
    axis = axis / axis.norm(dim=-1, keepdim=True)
    heavy = [int(b + i) for b, n in zip(off[:-1], lens) for i in list(range(min(n, 2))) + [int(x) for x in rng.integers(0, n, 6)] if n]
    kv[0, 0, :, heavy] += (axis * 4).to(dt)
    q = (q + axis.repeat_interleave(G, 0).transpose(0, 1) * 6).to(dt)
    state = {"case": case, "kv": kv, "q": q, "seq_begin": _table(off[:-1]), "seq_len": _table(lens),
             "node_offsets": _table(_starts(nodes)), "longest": max(lens), "most": max(nodes)}
    if case["op"] == "attention":
        state["draft"] = torch.randn((2, N, H, D), generator=g, device=DEV, dtype=dt)
        state["tree"] = torch.from_numpy(_tree_bits(nodes, rng)).to(DEV) if case["tree"] else None
    else:
        # the attention pass's log-sum-exp (a softmax over the cached rows and the drafted tokens) comes with the
        # queries; here that of the cached rows, raised by what drafted tokens add
        lse = torch.empty((N, H * G), device=DEV)
        at = _starts(nodes)
        for b in range(B):
            if not lens[b]:
                lse[at[b]:at[b + 1]] = 0.5
                continue
            for h in range(H):
                k = kv[0, 0, h, int(off[b]):int(off[b]) + lens[b]].float()
                s = q[at[b]:at[b + 1], h * G:(h + 1) * G].float().reshape(-1, D) @ k.T
                lse[at[b]:at[b + 1], h * G:(h + 1) * G] = torch.logsumexp(s * D ** -0.5, -1).view(-1, G)
        state["lse"] = lse + 0.1 * torch.rand(lse.shape, generator=g, device=DEV)
        counts = rng.random(N) < (1.0 if max(nodes) == 1 else 0.34)
        counts[at[:-1]] = True
        state["weight"] = torch.from_numpy(counts.astype(np.float32)).to(DEV)
        state["history"] = torch.rand(rows, generator=g, device=DEV) * 3
        state["out"] = torch.zeros(rows, device=DEV)
    return state


# ------------------------------------------------------------------------------------------ the plain forms
def _pad(begin, count, most):
    """[B, most] rows begin + 0..most-1 (clamped to the first row where there is none) and which of them are there."""
    i = torch.arange(most, device=DEV)
    there = i < count[:, None]
    return torch.where(there, begin[:, None] + i, 0).long(), there


def _queries(st):
    """q as [H, B, most * G, D] in 32 bits, and for the way back the padded place of every node."""
    H, G, off = st["case"]["kv_heads"], st["case"]["group"], st["node_offsets"]
    at, there = _pad(off[:-1], off[1:] - off[:-1], st["most"])
    q = st["q"][at].float().view(*at.shape, H, G, -1).permute(2, 0, 1, 3, 4)
    t = torch.arange(st["q"].shape[0], device=DEV)
    b = torch.searchsorted(off, t, right=True) - 1
    return q.reshape(H, at.shape[0], -1, q.shape[-1]), at, there, b, t - off[b]


def _attention(st):
    c, kv = st["case"], st["kv"][0]
    H, G, D = c["kv_heads"], c["group"], c["head_dim"]
    q, at, there, b, i = _queries(st)
    rows, cached = _pad(st["seq_begin"], st["seq_len"], st["longest"])
    k, v = kv[:, :, rows].float()
    dk, dv = st["draft"][:, at].permute(0, 3, 1, 2, 4).float()
    n = at.shape[1]
    if st["tree"] is None:
        sees = torch.ones((n, n), dtype=torch.bool, device=DEV).tril() & there[:, None, :]
    else:
        j = torch.arange(n, device=DEV)
        sees = ((st["tree"][at][:, :, j // 32] >> (j % 32)) & 1).bool() & there[:, None, :]
    s = torch.cat([(q @ k.transpose(-1, -2)).masked_fill_(~cached[:, None, :], -math.inf),
                   (q @ dk.transpose(-1, -2)).masked_fill_(~sees.repeat_interleave(G, 1), -math.inf)], -1)
    s *= D ** -0.5
    top = s.amax(-1, keepdim=True).clamp_min(-3e38)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    o = p @ torch.cat([v.masked_fill_(~cached[:, :, None], 0), dv], -2) / torch.where(total == 0, 1.0, total)
    lse = torch.log(total) + top
    back = lambda x: x.view(H, -1, n, G, x.shape[-1])[:, b, i].transpose(0, 1).reshape(b.shape[0], H * G, -1)  # noqa: E731
    return {"out": back(o).to(st["q"].dtype), "lse": back(lse)[..., 0]}


def _plain_mass(st):
    c = st["case"]
    q, at, there, _, _ = _queries(st)
    rows, cached = _pad(st["seq_begin"], st["seq_len"], st["longest"])
    s = q @ st["kv"][0, 0][:, rows].float().transpose(-1, -2) * c["head_dim"] ** -0.5
    # a value for each node and head as [heads, sequences, nodes * group, 1], like the scores
    grouped = lambda x: x.view(*at.shape, c["kv_heads"], -1).permute(2, 0, 1, 3).reshape(c["kv_heads"], at.shape[0], -1, 1)  # noqa: E731
    lse = grouped(st["lse"][at])
    w = torch.where(there, st["weight"][at], 0.0).repeat_interleave(c["group"], 1)[..., None]
    mass = (torch.exp(s - lse) * w).sum((0, 2))
    # the sequences are packed: row p of the cache is row p - begin of its sequence
    p = torch.arange(st["out"].shape[0] - 24, device=DEV)
    b = torch.searchsorted(st["seq_begin"] + st["seq_len"], p, right=True)
    st["out"][:p.shape[0]] = c["decay"] * st["history"][:p.shape[0]] + mass[b, p - st["seq_begin"][b]]
    return st["out"]


def _plain_evict(st):
    c, n = st["case"], st["seq_len"][:, None]
    rows, there = _pad(st["seq_begin"], st["seq_len"], st["longest"])
    i = torch.arange(st["longest"], device=DEV)
    kind = torch.where((i < c["sink"]) | (i >= n - c["recent"]), 0, 1).masked_fill_(~there, 2)
    order = torch.sort(st["mass"][rows], dim=1, descending=True, stable=True).indices
    order = order.gather(1, torch.sort(kind.gather(1, order), dim=1, stable=True).indices)
    kept = torch.zeros_like(there).scatter_(1, order, i < st["budget"][:, None])
    place = kept.flatten().cumsum(0) - 1
    place = torch.where(kept.flatten(), place, st["total"])
    pos = torch.empty(st["total"] + 1, dtype=torch.int32, device=DEV).scatter_(0, place, rows.flatten().int())[:-1]
    return {"kept_pos": pos, "kept_seq_offsets": torch.nn.functional.pad(kept.sum(1).cumsum(0).int(), (1, 0)),
            "mass": st["mass"][pos.long()]}


def _plain_append(st):
    j = torch.arange(st["total"], device=DEV)
    b = torch.searchsorted(st["offsets"], j, right=True) - 1
    st["dst"][:, :, :, st["dst_begin"][b] + j - st["offsets"][b]] = st["src"][:, :, :, st["src_pos"]]
    return st["dst"]


def run(state):
    op = state["case"]["op"]
    if own:
        sv = _sv()
        if op == "attention":
            return sv.sharpv_tree_attention(state["q"], state["kv"], 0, state["seq_begin"], state["seq_len"],
                                            state["node_offsets"], state["draft"][0], state["draft"][1],
                                            tree_mask=state["tree"])
        if op == "mass":
            return sv.sharpv_attention_mass(state["q"], state["lse"], state["kv"], 0, state["seq_begin"],
                                            state["seq_len"], state["node_offsets"], mass=state["history"],
                                            node_weight=state["weight"], decay=state["case"]["decay"],
                                            out=state["out"])
        if op == "evict":
            return sv.sharpv_evict_select(state["mass"], state["seq_begin"], state["seq_len"], state["budget"],
                                          state["case"]["sink"], state["case"]["recent"], state["total"])
        return sv.sharpv_kv_append(state["src"], state["dst"], state["src_pos"], state["offsets"],
                                   state["dst_begin"], state["total"])
    return {"attention": _attention, "mass": _plain_mass, "evict": _plain_evict, "append": _plain_append}[op](state)


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    """The definitions, one sequence and one KV head at a time."""
    if case["op"] == "append":
        return None
    st = prepare(case, seed)
    lens = _ints(case["lens"])
    off = _starts(lens)
    if case["op"] == "evict":
        mass, kept = st["mass"].cpu().numpy().astype(np.float64), []
        budget = _budgets(case)
        for b, n in enumerate(lens):
            i = np.arange(n)
            second = (i >= case["sink"]) & (i < n - case["recent"])
            kept.append(np.sort(np.lexsort((i, -mass[off[b]:off[b + 1]], second))[:budget[b]]) + off[b])
        kept = np.concatenate(kept)
        return {"kept_pos": kept.astype(np.int32), "kept_seq_offsets": _starts(budget).astype(np.int32), "mass": mass[kept]}
    H, G, D = case["kv_heads"], case["group"], case["head_dim"]
    nodes = _ints(case["nodes"])
    at = _starts(nodes)
    q, kv = st["q"].double(), st["kv"][0]
    if case["op"] == "mass":
        out = torch.zeros(kv.shape[2], dtype=torch.float64, device=DEV)
        for b, n in enumerate(lens):
            r, t = slice(int(off[b]), int(off[b]) + n), slice(int(at[b]), int(at[b + 1]))
            got = case["decay"] * st["history"][r].double()
            for h in range(H):
                for x in range(G):
                    s = q[t, h * G + x] @ kv[0, h, r].double().T / math.sqrt(D)
                    got += st["weight"][t].double() @ torch.exp(s - st["lse"][t, h * G + x].double()[:, None])
            out[r] = got
        return out
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(lens):
        r, t = slice(int(off[b]), int(off[b]) + n), slice(int(at[b]), int(at[b + 1]))
        if case["tree"]:
            bits = np.unpackbits(st["tree"][t].cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :nodes[b]]
        else:
            bits = np.tri(nodes[b])
        sees = torch.cat([torch.ones((nodes[b], n)), torch.from_numpy(bits.astype(np.float32))], 1).bool().to(DEV)
        for h in range(H):
            k = torch.cat([kv[0, h, r], st["draft"][0, t, h]]).double()
            v = torch.cat([kv[1, h, r], st["draft"][1, t, h]]).double()
            for x in range(h * G, (h + 1) * G):
                s = torch.where(sees, q[t, x] @ k.T / math.sqrt(D), -math.inf)
                lse[t, x] = torch.logsumexp(s, 1)
                out[t, x] = torch.softmax(s, 1) @ v
    return {"out": out, "lse": lse}

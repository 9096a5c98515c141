"""Decoding over the pruned cache on the GPU: attention of drafted tokens, the weight the rows collect, eviction, append."""
import numpy as np
import pytest
import torch

import decode_reference as ref
from helpers import Guarded
from paper_2511_08003_b200 import binding as sv

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NAN = float("nan")


def _i32(v):
    return torch.tensor(np.asarray(v, dtype=np.int64).astype(np.int32), device="cuda")


def _f64(t):
    return t.detach().double().cpu().numpy()


def _needs_capture():
    if sv.lib().sharpv_version() >= 200 and sv.lib_path() != sv._build.LIB_PATH:
        pytest.skip("with the range-checking library every call is followed by a synchronise, which a capture refuses")


class Case:
    """A cache with every row outside the sequences NaN, gaps between the sequences, nodes behind the last sequence."""

    def __init__(self, dtype, H, G, D, lens, nodes, seed=0, layers=2, layer=1, gap=3, spare=2, spread=1.0, words=None,
                 tree="random", token_major=False, fused=False, draft=True):
        g = np.random.default_rng(seed)
        self.dtype, self.H, self.G, self.D, self.layer = DT[dtype], H, G, D, layer
        self.bf16 = dtype == "bf16"
        self.length = np.asarray(lens)
        self.begin = np.concatenate([[0], np.cumsum(self.length + gap)])[:-1].astype(int) + gap
        self.offsets = np.concatenate([[0], np.cumsum(nodes)]).astype(int)
        T, N = int(self.begin[-1] + self.length[-1]) + gap, int(self.offsets[-1]) + spare
        host = torch.full((layers, 2, H, T, D), NAN)
        for b, n in zip(self.begin, self.length):
            host[layer, :, :, b:b + n] = torch.from_numpy(g.standard_normal((2, H, n, D), dtype=np.float32))
        host = host.to(self.dtype)
        if token_major:                     # [layers, T, 2, H, D] in memory
            self.kv = host.permute(0, 3, 1, 2, 4).contiguous().cuda().permute(0, 2, 3, 1, 4)
        else:
            self.kv = host.cuda()
        qkv = torch.from_numpy(g.standard_normal((N, H * G + 2 * H, D), dtype=np.float32))
        qkv[:, :H * G] *= spread
        qkv[self.offsets[-1]:] = NAN
        if fused:                           # q, k and v of a node side by side, as a fused projection leaves them
            qkv = qkv.to(self.dtype).cuda()
            self.q, self.dk, self.dv = qkv[:, :H * G], qkv[:, H * G:H * G + H], qkv[:, H * G + H:]
        else:
            self.q, self.dk, self.dv = (x.to(self.dtype).cuda().contiguous()
                                        for x in (qkv[:, :H * G], qkv[:, H * G:H * G + H], qkv[:, H * G + H:]))
        if not draft:
            self.dk = self.dv = None
        self.tree = None
        if tree == "random":
            most = max(max(nodes), 1)
            words = words or (most + 31) // 32
            bits = np.zeros((N, words * 32), np.uint8)
            for b, n in enumerate(nodes):
                for i in range(n):
                    p = int(g.integers(max(-1, i - 6), i)) if i else -1
                    row = bits[self.offsets[b] + i]
                    if p >= 0:
                        row[:] = bits[self.offsets[b] + p]
                    if i < words * 32:
                        row[i] = 1
            bits[self.offsets[-1]:] = 1
            self.tree = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view("<i4").copy()).cuda()
        self.tables = (_i32(self.begin), _i32(self.length), _i32(self.offsets))

    def reference(self, scale):
        kv = _f64(self.kv[self.layer])
        return ref.attention(_f64(self.q), kv[0], kv[1], self.begin, self.length, self.offsets,
                             None if self.dk is None else _f64(self.dk), None if self.dv is None else _f64(self.dv),
                             None if self.tree is None else self.tree.cpu().numpy(), scale, self.bf16)

    def check(self, scale=None, what=""):
        scale_used = self.D ** -0.5 if scale is None else scale
        mem = Guarded()
        N = self.q.shape[0]
        out = {"out": mem.empty(self.q.shape, self.dtype), "lse": mem.empty((N, self.H * self.G), torch.float32)}
        out["out"].fill_(7.0)
        out["lse"].fill_(7.0)
        ws = mem.empty(sv.sharpv_tree_attention_workspace_bytes(len(self.length), N, self.H * self.G, self.H, self.D,
                                                               sv.BF16 if self.bf16 else sv.F32), torch.uint8)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = sv.sharpv_tree_attention(self.q, self.kv, self.layer, *self.tables, self.dk, self.dv, self.tree,
                                       scale=scale, out=out, workspace=ws, status_word=status)
        mem.check(what)
        assert status.item() == 0
        o, lse, o_tol, lse_tol = self.reference(scale_used)
        n = self.offsets[-1]
        assert bool((got["out"][n:] == 7).all()) and bool((got["lse"][n:] == 7).all()), "rows of no sequence were written"
        go, gl = _f64(got["out"])[:n], _f64(got["lse"])[:n]
        empty = np.isneginf(lse[:n])
        assert np.array_equal(np.isneginf(gl), empty)
        assert np.all(go[empty] == 0)
        assert np.all(np.isfinite(go)), what
        worst = np.max(np.abs(go - o[:n]) - o_tol[:n], initial=-1.0)
        assert worst <= 0, f"{what}: out is {worst:.3e} past its bound"
        fine = ~empty
        worst = np.max(np.abs(gl[fine] - lse[:n][fine]) - lse_tol[:n][fine], initial=-1.0)
        assert worst <= 0, f"{what}: lse is {worst:.3e} past its bound"
        return got


SHAPES = [
    # kv heads, group, head_dim, lens, nodes
    (2, 7, 64, [100], [1]),
    (1, 1, 16, [0, 1, 2], [1, 1, 1]),
    (2, 3, 80, [33, 0, 257], [5, 2, 1]),
    (1, 8, 128, [128, 31, 64, 65], [1, 0, 4, 2]),
    (4, 7, 128, [700, 1], [9, 33]),
    (3, 2, 256, [65, 190], [3, 20]),
    (2, 1, 128, [129, 0, 511], [70, 40, 1]),
    (1, 5, 96, [1030], [64]),
    (2, 16, 64, [300, 20], [12, 1]),
    (1, 7, 136, [77], [6]),
    (1, 4, 128, [1500, 3], [130, 64]),
    (1, 2, 64, [640], [300]),
    (1, 100, 128, [200, 9], [2, 1]),             # a node fills most of a row tile
    (1, 130, 64, [70, 300], [2, 3]),             # more heads in a group than a row tile holds
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tree", ["random", None])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "h%dx%d_d%d_%s" % (s[0], s[1], s[2], "-".join(map(str, s[4]))))
def test_tree_attention(shape, tree, dtype):
    H, G, D, lens, nodes = shape
    Case(dtype, H, G, D, lens, nodes, seed=sum(lens) + D, tree=tree).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["token_major", "fused", "no_draft", "no_draft_empty", "peaked", "long", "few_words", "many", "long_chain"])
def test_tree_attention_layouts_and_ranges(kind, dtype):
    if kind == "token_major":
        Case(dtype, 2, 4, 64, [90, 210], [3, 7], token_major=True).check()
    elif kind == "fused":
        Case(dtype, 2, 7, 128, [75, 300], [9, 1], fused=True).check()
    elif kind == "no_draft":
        Case(dtype, 2, 4, 128, [75, 300], [9, 30], draft=False, tree=None).check()
    elif kind == "no_draft_empty":          # rows without any key
        got = Case(dtype, 2, 4, 128, [0, 40, 0], [2, 30, 1], draft=False, tree=None).check()
        assert bool((got["out"][:2] == 0).all()) and bool(torch.isneginf(got["lse"][:2]).all())
    elif kind == "peaked":                  # scores of some hundreds: the running maximum moves often and far
        Case(dtype, 2, 7, 128, [900, 40], [5, 2], spread=40.0).check()
        Case(dtype, 1, 7, 128, [900, 40], [50, 20], spread=40.0).check()
    elif kind == "long":
        Case(dtype, 1, 7, 128, [20011], [1]).check()
        Case(dtype, 1, 4, 64, [9973, 12], [33, 1]).check()
    elif kind == "few_words":               # nodes past the mask's words see only what the words hold
        Case(dtype, 1, 2, 64, [50], [70], words=1).check()
    elif kind == "many":                    # more sequences than threads of a block, most of them tiny
        g = np.random.default_rng(5)
        Case(dtype, 1, 2, 64, list(g.integers(0, 40, 700)), list(g.integers(0, 3, 700)), gap=1).check()
    else:
        Case(dtype, 2, 4, 128, [333], [700], tree=None).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,G,D,lens,nodes", [
    (1, 2, 256, [12007], [1]),                      # parts of one segment for every warp of a joining CTA many times over
    (2, 1, 200, [6001, 0, 5003], [2, 3, 1]),
    (1, 4, 128, [4000] + [3] * 30, [1] * 31),       # one sequence in many parts among whole ones
    (1, 4, 128, [9000] + [70] * 39, [1] * 40),      # the same with more sequences than lanes
    (1, 4, 128, [9000, 300, 0, 5], [40, 3, 0, 1]),
])
def test_tree_attention_segments_in_many_parts(H, G, D, lens, nodes, dtype):
    Case(dtype, H, G, D, lens, nodes, seed=D + len(lens)).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nodes", [[6, 3], [90, 40]])
@pytest.mark.parametrize("value", [NAN, float("inf"), float("-inf")])
def test_tree_attention_ignores_what_is_not_seen(value, nodes, dtype):
    """Drafted rows that a node does not see may hold anything: its result is the same, bit for bit."""
    c = Case(dtype, 2, 4, 128, [100, 37], nodes, seed=4)
    # the last node of each sequence is seen by itself alone
    clean = c.check()
    tree = c.tree.cpu().numpy()
    last = [c.offsets[1] - 1, c.offsets[2] - 1]
    c.dk[last], c.dv[last] = value, value
    got = sv.sharpv_tree_attention(c.q, c.kv, c.layer, *c.tables, c.dk, c.dv, c.tree)
    keep = np.setdiff1d(np.arange(c.offsets[-1]), last)
    for b in range(2):
        i = last[b] - c.offsets[b]
        seen = (tree[c.offsets[b]:c.offsets[b + 1], i // 32] >> (i % 32)) & 1
        assert seen.sum() == 1
    assert torch.equal(got["out"][keep], clean["out"][keep]) and torch.equal(got["lse"][keep], clean["lse"][keep])
    assert not bool(torch.isfinite(got["out"][last]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nodes", [2, 50])
def test_tree_attention_shows_what_is_seen(nodes, dtype):
    """NaN in a value that every node sees reaches every result; an infinite value gives an infinity of its sign."""
    c = Case(dtype, 1, 4, 128, [200], [nodes], tree=None, spare=0)
    c.kv[c.layer, 1, 0, c.begin[0] + 150, 5] = NAN
    c.dv[0, 0, 9] = float("-inf")
    got = sv.sharpv_tree_attention(c.q, c.kv, c.layer, *c.tables, c.dk, c.dv, None)["out"].float()
    assert bool(torch.isnan(got[:, :, 5]).all()) and bool(torch.isneginf(got[:, :, 9]).all())
    rest = [i for i in range(128) if i not in (5, 9)]
    assert bool(torch.isfinite(got[:, :, rest]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tree_attention_empty_mask_rows(dtype):
    c = Case(dtype, 2, 4, 64, [0, 60], [40, 4])
    c.tree[3] = 0
    c.tree[37] = 0
    got = c.check()
    assert bool(torch.isneginf(got["lse"][3]).all()) and bool((got["out"][37] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tree_attention_tables_outside_the_cache(dtype):
    """Tables that reach outside are cut to the cache and reported; sequences that fit keep their results."""
    c = Case(dtype, 2, 4, 64, [50, 60], [3, 4], gap=0)
    good = c.check()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    T = c.kv.shape[3]
    tables = (_i32([c.begin[0], T - 10]), _i32([50, 1 << 30]), c.tables[2])
    got = sv.sharpv_tree_attention(c.q, c.kv, c.layer, *tables, c.dk, c.dv, c.tree, status_word=status)
    assert status.item() == sv.Status.ERR_BOUNDS
    assert torch.equal(got["out"][:3], good["out"][:3])
    status.zero_()
    sv.sharpv_tree_attention(c.q, c.kv, c.layer, _i32([-5, 1 << 30]), _i32([50, -3]), _i32([0, 3, 900]), c.dk, c.dv,
                             c.tree, status_word=status)
    assert status.item() == sv.Status.ERR_BOUNDS


@pytest.mark.parametrize("nodes", [[1, 1], [20, 33], [200, 30]])
def test_tree_attention_same_bits_again_captured_and_on_a_stream(nodes):
    _needs_capture()
    c = Case("bf16", 2, 7, 128, [3000, 411], nodes, spare=0)
    args = (c.q, c.kv, c.layer, *c.tables, c.dk, c.dv, c.tree)
    first = sv.sharpv_tree_attention(*args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = sv.sharpv_tree_attention(*args)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first["out"], again["out"]) and torch.equal(first["lse"], again["lse"])
    ws = torch.full((sv.sharpv_tree_attention_workspace_bytes(2, sum(nodes), 14, 2, 128),), 0xFF, dtype=torch.uint8, device="cuda")
    out = {k: torch.zeros_like(v) for k, v in first.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sv.sharpv_tree_attention(*args, out=out, workspace=ws)
    for _ in range(2):
        out["out"].zero_()
        graph.replay()
        assert torch.equal(first["out"], out["out"])
    # the captured call follows the tables' contents: a shorter second sequence
    c.length[1] = 100
    c.tables[1].copy_(_i32(c.length))
    graph.replay()
    got = out["out"].clone()
    assert torch.equal(got, sv.sharpv_tree_attention(*args)["out"])
    o, _, tol, _ = c.reference(c.D ** -0.5)
    assert np.all(np.abs(_f64(got) - o) <= tol)


# ------------------------------------------------------------------------------------------ collected weight
def _mass_case(dtype, H, G, D, lens, nodes, decay, weights, seed=0, spread=1.0):
    c = Case(dtype, H, G, D, lens, nodes, seed=seed, spread=spread)
    got = sv.sharpv_tree_attention(c.q, c.kv, c.layer, *c.tables, c.dk, c.dv, c.tree)
    g = np.random.default_rng(seed + 1)
    N, T = c.q.shape[0], c.kv.shape[3]
    w = None
    if weights:
        w = g.random(N).astype(np.float32) * (g.random(N) < 0.5)
        dead = np.nonzero(w == 0)[0]
        c.q[torch.from_numpy(dead).cuda()] = NAN            # a node of weight 0 is not looked at
        got["lse"][torch.from_numpy(dead).cuda()] = NAN
    hist = torch.from_numpy(g.random(T).astype(np.float32)).cuda()
    mem = Guarded()
    out = mem.empty(T, torch.float32)
    out.fill_(-3.0)
    ws = mem.empty(sv.sharpv_attention_mass_workspace_bytes(T, H, sv.BF16 if c.bf16 else sv.F32), torch.uint8)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    res = sv.sharpv_attention_mass(c.q, got["lse"], c.kv, c.layer, *c.tables, mass=hist,
                                   node_weight=None if w is None else torch.from_numpy(w).cuda(), decay=decay, out=out,
                                   workspace=ws, status_word=status)
    mem.check("mass")
    assert status.item() == 0
    want, tol = ref.attention_mass(_f64(c.q), _f64(got["lse"]), _f64(c.kv[c.layer, 0]), c.begin, c.length, c.offsets,
                                   D ** -0.5, w, np.float32(decay).astype(np.float64), _f64(hist), T)
    r = _f64(res)
    outside = np.isnan(want)
    assert np.all(r[outside] == -3.0), "rows of no sequence were written"
    worst = np.max(np.abs(r - want)[~outside] - tol[~outside], initial=-1.0)
    assert worst <= 0, f"mass is {worst:.3e} past its bound"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "h%dx%d_d%d_%s" % (s[0], s[1], s[2], "-".join(map(str, s[4]))))
def test_attention_mass(shape, weights, dtype):
    H, G, D, lens, nodes = shape
    _mass_case(dtype, H, G, D, lens, nodes, 0.75, weights, seed=D + len(lens))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_mass_long_and_many(dtype):
    _mass_case(dtype, 1, 7, 128, [20011, 5], [1, 3], 1.0, False)
    _mass_case(dtype, 1, 2, 64, [90, 700], [650, 2], 0.0, True)
    _mass_case(dtype, 1, 7, 128, [400], [20], 1.0, False, spread=20.0)


def test_attention_mass_sums_to_the_number_of_rows():
    """Over the cached tokens alone every row's weights add up to 1, so a sequence collects nodes * heads (n u per sum)."""
    c = Case("bf16", 2, 7, 128, [1000, 77], [5, 40], draft=False, tree=None, spare=0)
    got = sv.sharpv_tree_attention(c.q, c.kv, c.layer, *c.tables)
    mass = sv.sharpv_attention_mass(c.q, got["lse"], c.kv, c.layer, *c.tables)
    for b in range(2):
        total = float(mass[c.begin[b]:c.begin[b] + c.length[b]].double().sum())
        rows = 14 * (c.offsets[b + 1] - c.offsets[b])
        assert abs(total / rows - 1) <= 2e-4         # (1000 + rows + 128) u and the scores' error, about 1e-4
    out = mass.clone()
    twice = sv.sharpv_attention_mass(c.q, got["lse"], c.kv, c.layer, *c.tables, mass=out, out=out)     # in place
    used = torch.cat([torch.arange(b, b + n) for b, n in zip(c.begin, c.length)]).cuda()
    # the weights are the same bits; query rows that do not fit at a time add to the old value one lot after the other,
    # here two: (m + s0) + s1 against 2 (s0 + s1), all positive, three roundings of u each against one
    assert bool(((twice[used] - 2 * mass[used]).abs() <= 4 * ref.U * twice[used]).all())


def test_attention_mass_history_is_not_read_when_it_decays_to_nothing():
    c = Case("f32", 1, 2, 64, [30], [2], spare=0)
    lse = sv.sharpv_tree_attention(c.q, c.kv, c.layer, *c.tables, c.dk, c.dv, c.tree)["lse"]
    nan = torch.full((c.kv.shape[3],), NAN, device="cuda")
    a = sv.sharpv_attention_mass(c.q, lse, c.kv, c.layer, *c.tables, mass=nan, decay=0.0)
    b = sv.sharpv_attention_mass(c.q, lse, c.kv, c.layer, *c.tables)
    assert torch.equal(a, b)
    empty = torch.full_like(lse, float("-inf"))
    assert bool((sv.sharpv_attention_mass(c.q, empty, c.kv, c.layer, *c.tables) == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nodes", [[3, 1], [40, 30]])
def test_attention_mass_rows_that_saw_nothing(nodes, dtype):
    """A row whose log-sum-exp is -inf adds nothing, whatever its query holds."""
    c = Case(dtype, 2, 4, 128, [100, 333], nodes, spare=0)
    lse = sv.sharpv_tree_attention(c.q, c.kv, c.layer, *c.tables, c.dk, c.dv, c.tree)["lse"]
    dead = torch.tensor([0, int(c.offsets[1])], device="cuda")
    w = torch.ones(c.q.shape[0], device="cuda")
    w[dead] = 0
    want = sv.sharpv_attention_mass(c.q, lse, c.kv, c.layer, *c.tables, node_weight=w)
    lse[dead] = float("-inf")
    c.q[dead] = NAN
    got = sv.sharpv_attention_mass(c.q, lse, c.kv, c.layer, *c.tables)
    # the same rows weighed, in another order where rows of weight 0 are left out: 2 (rows + 2) u of the sum
    rows = 8 * (max(nodes) + 1)
    assert bool(((got - want).abs() <= 2 * (rows + 2) * ref.U * want).all())
    alive = torch.isfinite(want)
    assert bool(alive.all()) and float(want.sum()) > 0


# ------------------------------------------------------------------------------------------ far rows, other streams
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nodes", [1, 40])
def test_rows_more_than_32_bits_away(nodes, dtype):
    """A cache whose rows lie 32 KB apart, used at its far end, more than 4 GB behind its start."""
    D, rows = 128, 170000
    es = 4 if dtype == "f32" else 2
    step = 32768 // es
    big = torch.empty(rows * step, dtype=DT[dtype], device="cuda")
    kv = big.as_strided((1, 2, 2, rows, D), (0, 2 * D, D, step, 1))
    g = torch.Generator(device="cuda").manual_seed(1)
    begin, n = rows - 400, 390
    near = torch.randn((1, 2, 2, n, D), device="cuda", generator=g).to(DT[dtype])
    sv.sharpv_kv_append(near, kv, torch.arange(n, dtype=torch.int32, device="cuda"), _i32([0, n]), _i32([begin]))
    assert torch.equal(kv[:, :, :, begin:begin + n], near)
    q = torch.randn((nodes, 6, D), device="cuda", generator=g).to(DT[dtype])
    far = sv.sharpv_tree_attention(q, kv, 0, _i32([begin]), _i32([n]), _i32([0, nodes]))
    here = sv.sharpv_tree_attention(q, near, 0, _i32([0]), _i32([n]), _i32([0, nodes]))
    assert torch.equal(far["out"], here["out"]) and torch.equal(far["lse"], here["lse"])
    m_far = sv.sharpv_attention_mass(q, far["lse"], kv, 0, _i32([begin]), _i32([n]), _i32([0, nodes]))
    m_here = sv.sharpv_attention_mass(q, far["lse"], near, 0, _i32([0]), _i32([n]), _i32([0, nodes]))
    assert torch.equal(m_far[begin:begin + n], m_here) and float(m_far[:begin].abs().sum()) == 0


def test_calls_on_a_stream_that_is_not_the_current_one():
    c = Case("bf16", 2, 7, 128, [900, 41], [9, 2], spare=0)
    f = Case("f32", 2, 7, 64, [900, 41], [9, 2], spare=0)
    side = torch.cuda.Stream()
    for x in (c, f):
        here = sv.sharpv_tree_attention(x.q, x.kv, x.layer, *x.tables, x.dk, x.dv, x.tree)
        m_here = sv.sharpv_attention_mass(x.q, here["lse"], x.kv, x.layer, *x.tables)
        k_here = sv.sharpv_evict_select(m_here, x.tables[0], x.tables[1], _i32([300, 20]), 2, 4, 320)
        torch.cuda.synchronize()
        for _ in range(20):                     # what the wrappers allocate is in use until the stream is done with it
            there = sv.sharpv_tree_attention(x.q, x.kv, x.layer, *x.tables, x.dk, x.dv, x.tree, stream=side)
            m = sv.sharpv_attention_mass(x.q, there["lse"], x.kv, x.layer, *x.tables, stream=side)
            k = sv.sharpv_evict_select(m, x.tables[0], x.tables[1], _i32([300, 20]), 2, 4, 320, stream=side)
            junk = [torch.full((1 << 20,), NAN, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        del junk
        assert torch.equal(here["out"], there["out"]) and torch.equal(m_here, m) and torch.equal(k_here["kept_pos"], k["kept_pos"])


def test_two_captured_graphs_share_a_workspace_one_after_the_other():
    _needs_capture()
    a = Case("bf16", 2, 7, 128, [2000, 33], [1, 1], spare=0)
    b = Case("bf16", 2, 7, 128, [1500, 700], [30, 41], spare=0, seed=3)
    want = [sv.sharpv_tree_attention(x.q, x.kv, x.layer, *x.tables, x.dk, x.dv, x.tree) for x in (a, b)]
    need = max(sv.sharpv_tree_attention_workspace_bytes(2, x.q.shape[0], 14, 2, 128) for x in (a, b))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    outs, graphs = [], []
    for x, w in zip((a, b), want):
        out = {k: torch.zeros_like(v) for k, v in w.items()}
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sv.sharpv_tree_attention(x.q, x.kv, x.layer, *x.tables, x.dk, x.dv, x.tree, out=out, workspace=ws)
        outs.append(out)
        graphs.append(graph)
    for order in ((0, 1, 0), (1, 1, 0)):
        for i in order:
            outs[i]["out"].zero_()
            graphs[i].replay()
        for i in (0, 1):
            assert torch.equal(outs[i]["out"], want[i]["out"]) or i not in order
            assert torch.equal(outs[i]["lse"], want[i]["lse"])


# ------------------------------------------------------------------------------------------ eviction
@pytest.mark.parametrize("lens,budget,sink,recent", [
    ([100], [40], 4, 16),
    ([0, 1, 1, 7, 513], [3, 0, 5, 7, 512], 0, 0),
    ([40, 50], [5, 10], 4, 16),                  # the protected rows alone are more than the budget
    ([300, 300], [300, -2], 1000, 0),
    ([20000, 3, 9999], [5000, 2, 9998], 4, 256),
    ([257] * 33, list(range(0, 264, 8)), 2, 9),
])
@pytest.mark.parametrize("kind", ["random", "ties", "special"])
def test_evict_select(kind, lens, budget, sink, recent):
    g = np.random.default_rng(len(lens) + budget[0])
    lens = np.asarray(lens)
    begin = np.concatenate([[0], np.cumsum(lens + 5)])[:-1] + 2
    T = int(begin[-1] + lens[-1]) + 4
    mass = np.exp(3 * g.standard_normal(T)).astype(np.float32)
    if kind == "ties":
        mass = g.integers(0, 3, T).astype(np.float32)
    if kind == "special":
        mass = g.choice(np.array([0.0, -0.0, 1.0, -1.0, np.nan, -np.nan, np.inf, -np.inf, 1e-45, 3e38], np.float32), T)
    kept, offsets = ref.evict(mass, begin, lens, budget, sink, recent)
    mem = Guarded()
    n = len(kept)
    out = {"kept_pos": mem.empty(n, torch.int32), "kept_seq_offsets": mem.empty(len(lens) + 1, torch.int32),
           "mass": mem.empty(n, torch.float32)}
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    m = torch.from_numpy(mass).cuda()
    got = sv.sharpv_evict_select(m, _i32(begin), _i32(lens), _i32(budget), sink, recent, n, out=out, status_word=status)
    mem.check("evict")
    assert status.item() == 0
    assert np.array_equal(got["kept_seq_offsets"].cpu().numpy(), offsets)
    assert np.array_equal(got["kept_pos"].cpu().numpy(), kept)
    assert np.array_equal(got["mass"].cpu().numpy().view(np.int32), mass[kept].view(np.int32))
    if n > 1:                                    # too little room: the rest is right, nothing behind it, and it is said
        out = {"kept_pos": mem.empty(n - 1, torch.int32), "kept_seq_offsets": mem.empty(len(lens) + 1, torch.int32)}
        got = sv.sharpv_evict_select(m, _i32(begin), _i32(lens), _i32(budget), sink, recent, n - 1, out=out, status_word=status)
        mem.check("evict, short")
        assert status.item() == sv.Status.ERR_CAPACITY
        assert np.array_equal(got["kept_pos"].cpu().numpy(), kept[:-1])


def test_evict_select_longer_than_shared_memory_holds():
    g = np.random.default_rng(2)
    n = 300001
    mass = np.exp(2 * g.standard_normal(n)).astype(np.float32).round(2)
    kept, offsets = ref.evict(mass, [0], [n], [77777], 4, 1000)
    got = sv.sharpv_evict_select(torch.from_numpy(mass).cuda(), _i32([0]), _i32([n]), _i32([77777]), 4, 1000, 77777)
    assert np.array_equal(got["kept_pos"].cpu().numpy(), kept) and got["kept_seq_offsets"].tolist() == [0, 77777]


def test_evict_select_tables_outside_the_mass():
    mass = torch.rand(50, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = sv.sharpv_evict_select(mass, _i32([40, -7, 99]), _i32([30, 5, 5]), _i32([20, 5, 5]), 0, 0, status_word=status)
    assert status.item() == sv.Status.ERR_BOUNDS
    assert got["kept_seq_offsets"].tolist() == [0, 10, 10, 10]
    assert got["kept_pos"][:10].tolist() == list(range(40, 50))


# ------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 80), ("f32", 64), ("u8", 48)])
def test_kv_append(dtype, D):
    g = torch.Generator(device="cuda").manual_seed(3)
    src = torch.randint(0, 255, (3, 2, 2, 90, D), dtype=torch.uint8, device="cuda", generator=g)
    if dtype != "u8":
        src = torch.randn((3, 2, 2, 90, D), device="cuda", generator=g).to(DT[dtype])
    mem = Guarded()
    dst = mem.empty((3, 2, 2, 200, D), src.dtype)
    dst.zero_()
    rows, begin = [5, 0, 30, 1], [3, 50, 100, 199]
    offsets = np.concatenate([[0], np.cumsum(rows)])
    pos = torch.randperm(90, generator=torch.Generator().manual_seed(1))[:36]
    want = dst.clone()
    for b in range(4):
        want[1:, :, :, begin[b]:begin[b] + rows[b]] = src[1:][:, :, :, pos[offsets[b]:offsets[b + 1]].cuda()]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    sv.sharpv_kv_append(src, dst, pos.int().cuda(), _i32(offsets), _i32(begin), layer_begin=1, status_word=status)
    mem.check("append")
    assert status.item() == 0 and torch.equal(dst, want)
    # rows outside either cache are skipped and reported; more rows than `capacity` are not copied
    dst.zero_()
    bad = pos.int().cuda()
    bad[0], bad[1] = 90, -1
    sv.sharpv_kv_append(src, dst, bad, _i32(offsets), _i32([3, 50, 190, 199]), layer_begin=1, status_word=status)
    assert status.item() == sv.Status.ERR_BOUNDS
    mem.check("append outside")
    assert bool((dst[1:, :, :, 3:5] == 0).all()) and torch.equal(dst[1:, :, :, 5:8], want[1:, :, :, 5:8])
    assert torch.equal(dst[1:, :, :, 190:199], want[1:, :, :, 100:109])
    status.zero_()
    dst.zero_()
    sv.sharpv_kv_append(src, dst, pos.int().cuda(), _i32(offsets), _i32(begin), capacity=6, layer_begin=1, status_word=status)
    assert status.item() == sv.Status.ERR_CAPACITY
    assert torch.equal(dst[1:, :, :, :100], want[1:, :, :, :100]) and torch.equal(dst[1:, :, :, 100], want[1:, :, :, 100])
    assert bool((dst[1:, :, :, 101:] == 0).all())


def test_kv_append_token_major_destination_and_large():
    src = torch.randn((2, 2, 4, 5000, 128), device="cuda").to(torch.bfloat16)
    dst = torch.zeros((2, 9000, 2, 4, 128), device="cuda", dtype=torch.bfloat16).permute(0, 2, 3, 1, 4)
    offsets, begin = [0, 2000, 4999], [10, 4000]
    sv.sharpv_kv_append(src, dst, torch.arange(1, 5000, device="cuda", dtype=torch.int32), _i32(offsets), _i32(begin))
    assert torch.equal(dst[:, :, :, 10:2010], src[:, :, :, 1:2001]) and torch.equal(dst[:, :, :, 4000:6999], src[:, :, :, 2001:])
    assert bool((dst[:, :, :, 6999:] == 0).all())


# ------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decode_loop_over_a_pruned_cache(dtype):
    """A packed, compacted cache is spread over regions with room; every step attends a tree of drafts, commits a path,
    collects weight; when a sequence is over its budget rows are evicted and the cache compacted.  At every step the
    result is the attention over the tokens the cache should hold."""
    g = np.random.default_rng(11)
    L, H, G, D, B = 2, 2, 3, 64, 2
    dt, bf16 = DT[dtype], dtype == "bf16"
    kept = [37, 61]
    packed = torch.from_numpy(g.standard_normal((L, 2, H, 120, D), dtype=np.float32)).to(dt).cuda()
    positions = np.sort(g.permutation(120)[:98])
    room = 128
    cache = torch.full((L, 2, H, B * room, D), NAN, dtype=dt, device="cuda")
    begin = np.array([0, room])
    sv.sharpv_kv_append(packed, cache, _i32(positions), _i32([0, 37, 98]), _i32(begin))
    held = [packed[:, :, :, positions[:37]].cpu(), packed[:, :, :, positions[37:]].cpu()]
    length = np.array(kept)
    mass = torch.zeros(B * room, device="cuda")
    parents = [-1, 0, 0, 1, 3, 2]
    bits = np.zeros((6, 32), np.uint8)
    for i, p in enumerate(parents):
        if p >= 0:
            bits[i] = bits[p]
        bits[i, i] = 1
    tree = torch.from_numpy(np.packbits(np.tile(bits, (B, 1)), axis=1, bitorder="little").view("<i4").copy()).cuda()
    path, offsets = [0, 1, 3], [0, 6, 12]
    weight = torch.from_numpy(np.tile([1.0, 1.0, 0.0, 1.0, 0.0, 0.0], B).astype(np.float32)).cuda()
    budget = 64
    evicted = 0
    for step in range(6):
        draft = torch.from_numpy(g.standard_normal((L, 2, H, 12, D), dtype=np.float32)).to(dt).cuda()
        for layer in range(L):
            q = torch.from_numpy(g.standard_normal((12, H * G, D), dtype=np.float32)).to(dt).cuda()
            dk, dv = (draft[layer, i].transpose(0, 1).contiguous() for i in range(2))
            got = sv.sharpv_tree_attention(q, cache, layer, _i32(begin), _i32(length), _i32(offsets), dk, dv, tree)
            mass = sv.sharpv_attention_mass(q, got["lse"], cache, layer, _i32(begin), _i32(length), _i32(offsets),
                                            mass=mass, node_weight=weight, out=mass)
            kv = np.concatenate([_f64(x[layer]) for x in held], axis=2)
            at = np.array([0, held[0].shape[3]])
            o, lse, o_tol, lse_tol = ref.attention(_f64(q), kv[0], kv[1], at, length, offsets, _f64(dk), _f64(dv),
                                                   tree.cpu().numpy(), D ** -0.5, bf16)
            assert np.all(np.abs(_f64(got["out"]) - o) <= o_tol) and np.all(np.abs(_f64(got["lse"]) - lse) <= lse_tol)
        accepted = np.concatenate([path, np.array(path) + 6])
        sv.sharpv_kv_append(draft, cache, _i32(accepted), _i32([0, 3, 6]), _i32(begin + length))
        for b in range(B):
            held[b] = torch.cat([held[b], draft[:, :, :, accepted[3 * b:3 * b + 3]].cpu()], 3)
            mass[begin[b] + length[b]:begin[b] + length[b] + 3] = 0
        length = length + 3
        if (length > budget).any():
            m = mass.cpu().numpy()
            want, off = ref.evict(m, begin, length, [budget, budget], 2, 8)
            s = sv.sharpv_evict_select(mass, _i32(begin), _i32(length), _i32([budget, budget]), 2, 8)
            assert np.array_equal(s["kept_pos"].cpu().numpy()[:off[-1]], want)
            fresh = torch.full_like(cache, NAN)
            sv.sharpv_kv_append(cache, fresh, s["kept_pos"], s["kept_seq_offsets"], _i32(begin), capacity=int(off[-1]))
            # the packed form of the same cut, by the compaction
            packed = torch.zeros((L, 2, H, int(off[-1]), D), dtype=dt, device="cuda")
            sv.sharpv_kv_compact(cache, packed, s["kept_pos"], s["kept_seq_offsets"], capacity=int(off[-1]))
            for b in range(B):
                rows = want[off[b]:off[b + 1]]
                held[b] = held[b][:, :, :, rows - begin[b]]
                assert torch.equal(packed[:, :, :, off[b]:off[b + 1]].cpu(), held[b])
                mass[begin[b]:begin[b] + len(rows)] = s["mass"][off[b]:off[b + 1]]
            evicted += int((length - np.diff(off)).sum())
            cache, length = fresh, np.diff(off)
        for b in range(B):
            assert torch.equal(cache[:, :, :, begin[b]:begin[b] + length[b]].cpu(), held[b])
    assert evicted > 0

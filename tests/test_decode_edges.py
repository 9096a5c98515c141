"""Operators that decode over a cache, where keys are not finite, tables are long or query rows come in lots."""
import numpy as np
import pytest
import torch

import decode_reference as ref
from paper_2511_08003_b200 import binding as sv
from test_decode_ops import NAN, Case, _f64, _i32, _mass_case, _needs_capture

pytestmark = pytest.mark.gpu

# numbers of query rows a (sequence, KV head) that fill none of the kernels' blocks, for each kernel
UNEVEN = [(3, [3, 1]), (3, [1, 0]), (5, [41, 13]), (7, [150, 3])]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group,nodes", UNEVEN)
@pytest.mark.parametrize("weights", [False, True])
def test_attention_mass_of_keys_with_infinities(weights, group, nodes, dtype):
    """A key whose score is -inf for every row collects nothing, and does not touch the others."""
    c = Case(dtype, 2, group, 128, [70, 333], nodes, spare=0, seed=group)
    c.q[..., 0] = c.q[..., 0].abs() + 0.5
    at = [int(c.begin[0]), int(c.begin[0]) + 69, int(c.begin[1]) + 100]
    c.kv[c.layer, 0, :, at, 0] = float("-inf")
    got = sv.sharpv_tree_attention(c.q, c.kv, c.layer, *c.tables, c.dk, c.dv, c.tree)
    assert bool(torch.isfinite(got["lse"]).all()) and bool(torch.isfinite(got["out"]).all())
    g = np.random.default_rng(1)
    w = g.random(c.q.shape[0]).astype(np.float32) * (np.arange(c.q.shape[0]) % 3 != 1) if weights else None
    hist = torch.rand(c.kv.shape[3], device="cuda")
    mass = sv.sharpv_attention_mass(c.q, got["lse"], c.kv, c.layer, *c.tables, mass=hist, decay=0.75,
                                    node_weight=None if w is None else torch.from_numpy(w).cuda())
    with np.errstate(invalid="ignore"):
        want, tol = ref.attention_mass(_f64(c.q), _f64(got["lse"]), _f64(c.kv[c.layer, 0]), c.begin, c.length, c.offsets,
                                       c.D ** -0.5, w, 0.75, _f64(hist), c.kv.shape[3])
    fine = ~np.isnan(want)
    fine[at] = False
    assert fine.sum() == 400 and np.all(np.abs(_f64(mass) - want)[fine] <= tol[fine])
    assert torch.equal(mass[at], 0.75 * hist[at])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group,nodes", UNEVEN)
def test_attention_mass_of_rows_that_saw_nothing_over_any_keys(group, nodes, dtype):
    c = Case(dtype, 2, group, 128, [70, 333], nodes, spare=0)
    c.kv[c.layer, 0, :, int(c.begin[0]):int(c.begin[0]) + 9, 3] = float("inf")
    c.kv[c.layer, 0, :, int(c.begin[1]):int(c.begin[1]) + 200, 5] = NAN
    c.q[::2] = NAN
    lse = torch.full(c.q.shape[:2], float("-inf"), device="cuda")
    hist = torch.rand(c.kv.shape[3], device="cuda")
    mass = sv.sharpv_attention_mass(c.q, lse, c.kv, c.layer, *c.tables, mass=hist, decay=0.5)
    for b in range(2):
        rows = slice(int(c.begin[b]), int(c.begin[b] + c.length[b]))
        assert torch.equal(mass[rows], 0.5 * hist[rows])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_mass_without_nodes(dtype):
    """Without nodes, or with none that counts, a row gets decay * mass; rows outside the sequences stay."""
    c = Case(dtype, 2, 4, 128, [70, 0, 333], [0, 0, 0], spare=0, tree=None)
    hist = torch.rand(c.kv.shape[3], device="cuda")
    inside = torch.cat([torch.arange(b, b + n) for b, n in zip(c.begin, c.length)]).cuda()
    want = torch.full_like(hist, -3.0)
    want[inside] = 0.25 * hist[inside]
    out = torch.full_like(hist, -3.0)
    sv.sharpv_attention_mass(c.q, torch.empty((0, 8), device="cuda"), c.kv, c.layer, *c.tables, mass=hist, decay=0.25, out=out)
    assert torch.equal(out, want)
    for nodes in ([3, 1, 4], [90, 3, 70]):
        c = Case(dtype, 2, 4, 128, [70, 0, 333], nodes, spare=0, tree=None)
        lse = torch.zeros(c.q.shape[:2], device="cuda")
        out.fill_(-3.0)
        sv.sharpv_attention_mass(c.q, lse, c.kv, c.layer, *c.tables, mass=hist, decay=0.25, out=out,
                                 node_weight=torch.zeros(c.q.shape[0], device="cuda"))
        assert torch.equal(out, want)


# ------------------------------------------------------------------------------------------ many sequences, many lots
def _many(n, most_rows, most_nodes, seed):
    g = np.random.default_rng(seed)
    return [int(x) for x in g.integers(0, most_rows + 1, n)], [int(x) for x in g.integers(0, most_nodes + 1, n)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("n,H,G,D,nodes", [
    (40, 2, 2, 64, 4), (700, 1, 2, 128, 3),             # few query rows a sequence
    (40, 2, 7, 128, 25), (700, 1, 16, 64, 10),          # many
    (33, 2, 3, 256, 5),
])
def test_attention_mass_of_many_sequences(n, H, G, D, nodes, weights, dtype):
    """More sequences than lanes of a warp, some without rows, some without nodes."""
    lens, count = _many(n, 150, nodes, n + nodes)
    lens[0], count[0] = 700, nodes
    _mass_case(dtype, H, G, D, lens, count, 0.5, weights, seed=n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tree", ["random", None])
@pytest.mark.parametrize("n,H,G,D,nodes", [(40, 2, 7, 128, 20), (700, 1, 8, 64, 9), (33, 1, 4, 80, 70)])
def test_tree_attention_of_many_sequences(n, H, G, D, nodes, tree, dtype):
    """The same for the attention, with query rows enough for the tensor cores' kernel."""
    lens, count = _many(n, 150, nodes, n)
    lens[0], count[0] = 900, nodes
    Case(dtype, H, G, D, lens, count, seed=n, tree=tree, gap=1).check()


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("H,G,D,lens,nodes", [
    (8, 8, 256, [40, 500], [60, 5]),                    # lots of 24 query rows a head
    (8, 7, 256, [330], [31]),                           # that no whole number of nodes fills
    (2, 7, 256, [130, 0, 60], [70, 9, 0]),
    (30, 1, 256, [90, 33], [20, 9]),                    # lots of heads
    (30, 3, 200, [100], [7]),
    (40, 3, 128, [100], [20]),
    (1, 600, 136, [50, 7], [2, 1]),                     # a node's own rows in several lots
])
def test_attention_mass_in_lots_of_query_rows(H, G, D, lens, nodes, weights):
    _mass_case("bf16", H, G, D, lens, nodes, 0.75, weights, seed=D + H)


# ------------------------------------------------------------------------------------------ a whole step in a graph
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nodes", [[1, 1], [30, 41]])
def test_a_step_captured_and_replayed(nodes, dtype):
    """Attention, weight, append and eviction in one graph; replayed on other contents it does what the calls do."""
    _needs_capture()
    c = Case(dtype, 2, 5, 128, [700, 411], nodes, spare=0, gap=100, tree=None, layers=2, layer=0)
    T, N = c.kv.shape[3], sum(nodes)
    drafts = torch.stack([c.dk, c.dv]).unsqueeze(0).repeat(2, 1, 1, 1, 1).transpose(2, 3)
    pos, offsets, budget = _i32([0, N - 1]), _i32([0, 1, 2]), _i32([300, 200])
    mass = torch.zeros(T, device="cuda")
    fresh = torch.zeros_like(c.kv)
    c.kv[1].zero_()

    def step(cache, weight, into):
        begin, length, table = c.tables
        att = sv.sharpv_tree_attention(c.q, cache, 0, begin, length, table, c.dk, c.dv)
        sv.sharpv_attention_mass(c.q, att["lse"], cache, 0, begin, length, table, mass=weight, out=weight)
        sv.sharpv_kv_append(drafts, cache, pos, offsets, begin + length)
        kept = sv.sharpv_evict_select(weight, begin, length + 1, budget, 2, 16, capacity=500)
        sv.sharpv_kv_append(cache, into, kept["kept_pos"], kept["kept_seq_offsets"], begin)
        return {**att, "pos": kept["kept_pos"], "offsets": kept["kept_seq_offsets"], "kept_mass": kept["mass"]}

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(c.kv, mass, fresh)
    for lens in ([700, 411], [350, 500], [0, 250], [700, 411]):
        c.kv.copy_(torch.randn(c.kv.shape, device="cuda"))
        c.tables[1].copy_(_i32(lens))
        mass.copy_(torch.rand(T, device="cuda"))
        fresh.zero_()
        cache, weight, into = c.kv.clone(), mass.clone(), torch.zeros_like(fresh)
        graph.replay()
        want = step(cache, weight, into)
        kept = int(want["offsets"][-1])
        assert kept == min(lens[0] + 1, 300) + 200
        for key, t in got.items():
            n = kept if key in ("pos", "kept_mass") else None
            assert torch.equal(t[:n], want[key][:n]), key
        assert torch.equal(c.kv, cache) and torch.equal(mass, weight) and torch.equal(fresh, into)

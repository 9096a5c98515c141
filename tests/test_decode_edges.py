"""Operators that decode over a cache, where keys are not finite, tables are long or query rows come in lots."""
import numpy as np
import pytest
import torch

import decode_reference as ref
from paper_2511_08003_b200 import binding as sv
from test_decode_ops import NAN, Case, _f64

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

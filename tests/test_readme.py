"""README.md's decode step, run as it stands there."""
import os
import re
import textwrap

import numpy as np
import pytest
import torch

import decode_reference as ref
from paper_2511_08003_b200 import binding as sv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    with open(os.path.join(ROOT, "README.md")) as f:
        blocks = [textwrap.dedent(b) for b in re.findall(r"^ *```python\n(.*?)^ *```", f.read(), re.S | re.M)]
    return next(b for b in blocks if "sharpv_tree_attention" in b)


def test_the_example_compiles():
    compile(_example(), "README.md", "exec")


@pytest.mark.gpu
def test_the_decode_step_of_the_readme():
    """Six steps of two sequences of different lengths.  The host keeps every sequence's tokens and, by position in them,
    their weights; the example has to leave the same in the cache, in its tables and in `mass`."""
    step = compile(_example(), "README.md", "exec")
    g = np.random.default_rng(3)
    L, H, G, D, B, room, N = 2, 2, 3, 64, 2, 400, 12
    new = lambda *shape: torch.from_numpy(g.standard_normal(shape, dtype=np.float32)).bfloat16().cuda()
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")
    length, begin = np.array([150, 210]), np.array([0, room])
    cache = torch.full((L, 2, H, B * room, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    held = [new(L, 2, H, n, D) for n in length]
    for b in range(B):
        cache[:, :, :, begin[b]:begin[b] + length[b]] = held[b]
    weights = [torch.zeros(n, device="cuda") for n in length]
    parents = [-1, 0, 0, 1, 3, 2]
    bits = np.zeros((6, 32), np.uint8)
    for i, p in enumerate(parents):
        if p >= 0:
            bits[i] = bits[p]
        bits[i, i] = 1
    tree = torch.from_numpy(np.packbits(np.tile(bits, (B, 1)), axis=1, bitorder="little").view("<i4").copy()).cuda()
    budget = [140, 190]
    # rows that no sequence holds have whatever stood there
    env = {"torch": torch, "sv": sv, "layers": L, "cache": cache, "fresh": torch.full_like(cache, float("nan")),
           "mass": torch.rand(B * room + 1, device="cuda") * 100, "seq_begin": i32(begin), "seq_len": i32(length),
           "budget": i32(budget), "most": sum(budget), "node_offsets": i32([0, 6, 12]), "tree_mask": tree}
    for b in range(B):
        env["mass"][begin[b]:begin[b] + length[b]] = 0
    evicted = 0
    for turn in range(6):
        # keys and values of a node side by side, as a projection leaves them
        made = new(L, N, 2, H, D)
        env["draft_k"], env["draft_v"], env["drafts"] = made[:, :, 0], made[:, :, 1], made.permute(0, 2, 3, 1, 4)
        env["q"] = [new(N, H * G, D) for _ in range(L)]
        outs = {}
        env["outputs"] = outs.__setitem__
        nodes = [[0, 1, 3], [6, 8]] if turn % 2 else [[0], [6, 7, 9, 10]]
        on = np.isin(np.arange(N), np.concatenate(nodes)).astype(np.float32)
        env["verify"] = lambda: (torch.from_numpy(on).cuda(), i32(np.concatenate(nodes)), i32(np.cumsum([0] + [len(x) for x in nodes])))
        env["over_budget"] = lambda: turn % 2 == 1
        exec(step, env)
        # ---- the same on the host
        kv = [torch.cat(held, 3)[layer].double().cpu().numpy() for layer in range(L)]
        at, n = [0, held[0].shape[3]], [x.shape[3] for x in held]
        for layer in range(L):
            f64 = lambda t: t.double().cpu().numpy()
            o, lse, tol, _ = ref.attention(f64(env["q"][layer]), kv[layer][0], kv[layer][1], at, n, [0, 6, 12], f64(made[layer, :, 0]),
                                           f64(made[layer, :, 1]), tree.cpu().numpy(), D ** -0.5, True)
            assert np.all(np.abs(f64(outs[layer]) - o) <= tol)
            # weights as the kernel collects them, from tensors that hold a sequence each
            for b in range(B):
                rows = slice(6 * b, 6 * b + 6)
                sv.sharpv_attention_mass(env["q"][layer][rows], env["lse"][layer][rows], held[b], layer, i32([0]), i32([n[b]]), i32([0, 6]),
                                         mass=weights[b], node_weight=torch.from_numpy(on[rows]).cuda(), out=weights[b])
        for b in range(B):
            held[b] = torch.cat([held[b], made.permute(0, 2, 3, 1, 4)[:, :, :, nodes[b]]], 3)
            weights[b] = torch.cat([weights[b], torch.zeros(len(nodes[b]), device="cuda")])
        if turn % 2:
            for b in range(B):
                want, _ = ref.evict(weights[b].cpu().numpy(), [0], [len(weights[b])], [budget[b]], 4, 64)
                evicted += len(weights[b]) - len(want)
                held[b], weights[b] = held[b][:, :, :, want], weights[b][want]
        assert env["seq_len"].tolist() == [len(w) for w in weights]
        for b in range(B):
            rows = slice(begin[b], begin[b] + len(weights[b]))
            assert torch.equal(env["cache"][:, :, :, rows], held[b]), (turn, b)
            # one call for all sequences or one a sequence: the same terms in an order that may differ, 18 query rows a call and
            # 2 calls a step, so 216 at most, all positive: either sum is off by up to 216 u
            assert bool(((env["mass"][rows] - weights[b]).abs() <= 2 * 216 * ref.U * weights[b]).all()), (turn, b)
    assert evicted > 0

"""README.md's step over a cache in 8 bits, run as it stands there."""
import os
import re
import textwrap

import numpy as np
import pytest
import torch

import q8_reference as ref
from decode_reference import B16
from paper_2511_08003_b200 import binding as sv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    with open(os.path.join(ROOT, "README.md")) as f:
        blocks = [textwrap.dedent(b) for b in re.findall(r"^ *```python\n(.*?)^ *```", f.read(), re.S | re.M)]
    return next(b for b in blocks if "sharpv_tree_attention_q8" in b)


def test_the_example_compiles():
    compile(_example(), "README.md", "exec")


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["e4m3", "i8"])
def test_the_step_of_the_readme(kind):
    g = np.random.default_rng(4)
    L, H, HQ, D, N = 2, 2, 6, 64, 5
    new = lambda *s: torch.from_numpy(g.standard_normal(s, dtype=np.float32)).bfloat16().cuda()  # noqa: E731
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")  # noqa: E731
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    kept, offsets, begin = np.sort(g.permutation(400)[:250]), np.array([0, 150, 250]), np.array([0, 256])
    cache, qkv = new(L, 2, H, 400, D), new(L, N, HQ + 2 * H, D)
    positions, axis, nodes = g.integers(0, 3000, (3, N)), np.arange(32) % 3, np.array([0, 2, 5])
    accepted, accepted_off = np.array([0, 2, 3]), np.array([0, 1, 3])
    norms = [new(L, D), new(L, D)]
    made, outs = qkv.clone(), {}
    code = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}[kind]
    env = {"sv": sv, "layers": L, "heads": H, "q_heads": HQ, "cache": cache, "qkv": qkv, "kept": {"kept_pos": i32(kept), "kept_seq_offsets": i32(offsets)},
           "cache8": torch.zeros((L, 2, H, 512, D), dtype=code, device="cuda"), "scales": torch.zeros((L, 2, H, 8), dtype=torch.uint8, device="cuda"),
           "seq_begin": i32(begin), "positions": i32(positions), "pair_axis": [int(a) for a in axis], "q_norm": norms[0], "k_norm": norms[1],
           "node_offsets": i32(nodes), "tree_mask": None, "outputs": outs.__setitem__, "accepted_nodes": i32(accepted),
           "accepted_offsets": i32(accepted_off)}
    exec(compile(_example(), "README.md", "exec"), env)
    codes, scales = np.zeros((L, 2, H, 512, D), np.uint8), np.zeros((L, 2, H, 8), np.uint8)
    length = np.diff(offsets)
    for plane in np.ndindex(L, 2, H):
        for b in range(2):
            ref.append(f64(cache[plane])[kept[offsets[b]:offsets[b + 1]]], codes[plane], scales[plane], kind, 64, int(begin[b]))
    for layer in range(L):
        for part, weight in ((slice(0, HQ), norms[0]), (slice(HQ, HQ + H), norms[1])):
            o, tol = ref.norm_rope(f64(made[layer, :, part]), positions, axis, 1e6, f64(weight[layer]), float(np.float32(1e-6)), True, B16)
            assert np.all(np.abs(f64(qkv[layer, :, part]) - o) <= tol)
        o, _, tol, _ = ref.attention(f64(qkv[layer, :, :HQ]), codes[layer, 0], scales[layer, 0], codes[layer, 1], scales[layer, 1], kind, 64, begin,
                                     length, nodes, f64(qkv[layer, :, HQ:HQ + H]), f64(qkv[layer, :, HQ + H:]), None, D ** -0.5)
        assert np.all(np.abs(f64(outs[layer]) - o) <= tol)
    for l, kv, h in np.ndindex(L, 2, H):
        for b in range(2):
            rows = f64(qkv[l, :, HQ + kv * H + h])[accepted[accepted_off[b]:accepted_off[b + 1]]]
            ref.append(rows, codes[l, kv, h], scales[l, kv, h], kind, 64, int(begin[b] + length[b]))
    assert np.array_equal(env["cache8"].view(torch.uint8).cpu().numpy(), codes) and np.array_equal(env["scales"].cpu().numpy(), scales)
    assert env["seq_len"].tolist() == (length + np.diff(accepted_off)).tolist()

"""Calls of the operators round a cache in 8 bits on streams that are not the current one, next to each other, and far into memory."""
import numpy as np
import pytest
import torch

import q8_reference as ref
from decode_reference import B16
from paper_2511_08003_b200 import binding as sv
from test_q8_ops import Attn, Store, _bits, _f64, _i32, _needs_capture
from test_streams import _pool

pytestmark = pytest.mark.gpu


def _rope_call():
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k = torch.randn((50, 8, 64), generator=g, device="cuda"), torch.randn((50, 2, 64), generator=g, device="cuda")
    pos = _i32(np.arange(50)[None])
    return lambda s: sv.sharpv_qk_norm_rope(q, k, pos, bytes(32), 1e4, norm=True, stream=s)


def _attention_call(nodes=(2, 40)):
    c = Attn("e4m3", 16, 2, 4, 128, [700, 100], list(nodes), spare=0)
    return lambda s: sv.sharpv_tree_attention_q8(*c.args(), stream=s)


CALLS = {"qk_norm_rope": _rope_call, "tree_attention_q8": _attention_call, "tree_attention_q8_few": lambda: _attention_call((1, 2))}


@pytest.mark.parametrize("name", list(CALLS))
def test_memory_comes_from_the_pool_of_the_stream_of_the_call(name, monkeypatch):
    call = CALLS[name]()
    plain, scratch = sv._workspace, []
    monkeypatch.setattr(sv, "_workspace", lambda *a, **kw: scratch.append(plain(*a, **kw)) or scratch[-1])
    want = call(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    del scratch[:]
    got = call(side)
    torch.cuda.synchronize()
    assert set(got) == set(want)
    for key, t in got.items():
        assert _pool(t) == side.cuda_stream, key
        assert torch.equal(t, want[key]), key
    for ws in scratch:
        assert _pool(ws) == side.cuda_stream


def test_results_are_kept_for_what_the_current_stream_still_does_with_them():
    call = _rope_call()
    call(None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = call(side)
    torch.cuda.current_stream().wait_stream(side)
    at = {t.data_ptr(): t.numel() * t.element_size() for t in got.values()}
    torch.cuda._sleep(1 << 28)              # about 0.15 s
    read = [t.clone() for t in got.values()]
    del got
    with torch.cuda.stream(side):
        new = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in at.values() for _ in range(2)]
        busy = not torch.cuda.default_stream().query()
    assert busy and not any(x.data_ptr() in at for x in new)
    torch.cuda.synchronize()
    del read


def test_calls_on_two_streams_at_once():
    """Attention of different kernels and an append at the same time, with a workspace each."""
    a, b = Attn("i8", 32, 2, 7, 128, [9000, 300], [1, 1], seed=1, spare=0), Attn("e4m3", 16, 2, 7, 128, [9000, 411], [30, 60], seed=2, spare=0)
    want = [sv.sharpv_tree_attention_q8(*x.args()) for x in (a, b)]
    s = Store("bf16", "e4m3", 32, 2, 128, [5, 40, 0], [900, 9, 3000], layers=4)
    codes, scales = s.expected()
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(20):
        got = [sv.sharpv_tree_attention_q8(*x.args(), stream=y) for x, y in zip((a, b), streams)]
        s.call(stream=streams[2])
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g["out"], w["out"]) and torch.equal(g["lse"], w["lse"])
    # the same rows again leave what the first call left: scales do not grow a second time
    assert np.array_equal(_bits(s.dst), codes) and np.array_equal(s.dst_scales.cpu().numpy(), scales)


def test_a_captured_step_follows_its_tables():
    """Norm and rotation, attention and append in one graph; replayed with other tables it does what separate calls do."""
    _needs_capture()
    c = Attn("e4m3", 32, 2, 4, 128, [200, 90], [2, 3], spare=0, layers=1, layer=0, gap=96, tree=None)
    begin = np.array([0, 512])
    # regions with room, at borders of blocks
    kv = torch.zeros((1, 2, 2, 1024, 128), dtype=c.kv.dtype, device="cuda")
    scales = torch.zeros((1, 2, 2, 32), dtype=torch.uint8, device="cuda")
    n = 290
    sv.sharpv_kv_append_q8(torch.randn((1, 2, 2, n, 128), device="cuda").bfloat16(), kv, scales, 32, _i32(np.arange(n)), _i32([0, 200, 290]), _i32(begin))
    first_kv, first_scales = kv.clone(), scales.clone()
    q, k = torch.randn((5, 8, 128), device="cuda").bfloat16(), torch.randn((5, 2, 128), device="cuda").bfloat16()
    v = torch.randn((1, 2, 2, 5, 128), device="cuda").bfloat16()
    pos, at, length, to = _i32([[7, 8, 9, 10, 11]]), _i32(begin), _i32([200, 90]), _i32(begin + [200, 90])
    off, rows = _i32([0, 2, 5]), _i32(np.arange(5))
    ws = torch.empty(sv.sharpv_tree_attention_q8_workspace_bytes(2, 5, 8, 2, 128), dtype=torch.uint8, device="cuda")
    out = {"out": torch.empty_like(q), "lse": torch.empty((5, 8), device="cuda")}
    turned = {"q": torch.empty_like(q), "k": v[0, 0].transpose(0, 1)}

    def step():
        sv.sharpv_qk_norm_rope(q, k, pos, bytes(64), 1e4, norm=True, out=turned)
        sv.sharpv_tree_attention_q8(turned["q"], kv, scales, 32, 0, at, length, off, v[0, 0].transpose(0, 1).contiguous(), v[0, 1].transpose(0, 1).contiguous(),
                                    out=out, workspace=ws)
        sv.sharpv_kv_append_q8(v, kv, scales, 32, rows, off, to)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    kv.copy_(first_kv), scales.copy_(first_scales)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens, p in (([200, 90], 7), ([31, 64], 40000)):
        length.copy_(_i32(lens)), to.copy_(_i32(begin + lens)), pos.copy_(_i32([np.arange(p, p + 5)]))
        got = []
        for run in (graph.replay, step):
            kv.view(torch.uint8).copy_(first_kv.view(torch.uint8)), scales.copy_(first_scales)
            run()
            torch.cuda.synchronize()
            got.append([t.clone() for t in (out["out"], out["lse"], kv.view(torch.uint8), scales)])
        assert all(torch.equal(x, y) for x, y in zip(*got))


def test_far_into_a_large_cache():
    """Rows, scales and planes behind the first 4 GB."""
    L, H, T, D, block = 9, 4, 600000, 128, 64
    kv = torch.empty((L, 2, H, T, D), dtype=torch.int8, device="cuda")             # 5.5 GB
    scales = torch.zeros((L, 2, H, -(-T // block)), dtype=torch.uint8, device="cuda")
    src = torch.empty((L, 2, H, T // 2, D), dtype=torch.bfloat16, device="cuda")   # as much
    g = torch.Generator(device="cuda").manual_seed(0)
    n, at, layer = 200, T - 300 - (T - 300) % block, L - 1
    src[layer, :, :, -n:] = torch.randn((2, H, n, D), generator=g, device="cuda").bfloat16()
    sv.sharpv_kv_append_q8(src, kv, scales, block, _i32(np.arange(T // 2 - n, T // 2)), _i32([0, n]), _i32([at]), layer_begin=layer)
    codes, bytes_ = np.zeros((2, H, n, D), np.uint8), np.zeros((2, H, -(-n // block)), np.uint8)
    for plane in np.ndindex(2, H):
        ref.append(_f64(src[layer, plane[0], plane[1], -n:]), codes[plane], bytes_[plane], "i8", block, 0)
    assert np.array_equal(_bits(kv[layer, :, :, at:at + n].contiguous()), codes)
    assert np.array_equal(scales[layer, :, :, at // block:at // block + bytes_.shape[2]].cpu().numpy(), bytes_)
    for nodes in (1, 40):
        q, dk, dv = (torch.randn((nodes, h, D), generator=g, device="cuda").bfloat16() for h in (8, H, H))
        got = sv.sharpv_tree_attention_q8(q, kv, scales, block, layer, _i32([at]), _i32([n]), _i32([0, nodes]), dk, dv)
        o, lse, tol, ltol = ref.attention(_f64(q), codes[0], bytes_[0], codes[1], bytes_[1], "i8", block, np.array([0]), np.array([n]), np.array([0, nodes]),
                                          _f64(dk), _f64(dv), None, D ** -0.5)
        assert np.all(np.abs(_f64(got["out"]) - o) <= tol) and np.all(np.abs(_f64(got["lse"]) - lse) <= ltol)


def test_norm_and_rotation_of_tokens_far_apart():
    n, step = 2500, 1 << 20
    raw = torch.empty(n * step + 4096, dtype=torch.bfloat16, device="cuda")         # 5.2 GB, a token every 2 MB
    q = raw.as_strided((n, 3, 64), (step, 64, 1))
    q.copy_(torch.randn((n, 3, 64), device="cuda").bfloat16())
    dense = q.contiguous()
    pos = np.arange(n)[None]
    first = sv.sharpv_qk_norm_rope(q, dense, _i32(pos), bytes(32), 1e4, norm=True)
    assert torch.equal(first["q"], first["k"])
    got = sv.sharpv_qk_norm_rope(dense, q, _i32(pos), bytes(32), 1e4, norm=True, out={"q": torch.empty_like(dense), "k": q})
    o, tol = ref.norm_rope(_f64(dense), pos, np.zeros(32, int), 1e4, None, float(np.float32(1e-6)), True, B16)
    assert np.all(np.abs(_f64(got["q"]) - o) <= tol) and torch.equal(got["k"], got["q"])

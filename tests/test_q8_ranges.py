"""The operators round a cache in 8 bits at the ends of what their scales, queries and strides may be, on the GPU."""
import numpy as np
import pytest
import torch

import q8_reference as ref
from decode_reference import B16, U
from paper_2511_08003_b200 import binding as sv
from test_q8_ops import CODES, INF, Store, _bits, _f64, _i32

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------ scales of values far apart
def _attention(q, k8, ke, v8, ve, scale):
    """One head's queries q [rows, D] over keys and values of codes' values k8, v8 [n, D] and exponents ke, ve [n], in 64 bits: out
    and the bound that the header gives: weights off by 2^-8 of themselves or 2^-25 of the row's largest, out rounded to bf16,
    and scores, maximum and sums in fp32 (decode_reference: e_p; the values' exponents are added to the scores)."""
    k, v = k8 * 2.0 ** ke[:, None], v8 * 2.0 ** ve[:, None]
    n, D = k.shape
    out, tol = np.zeros((len(q), D)), np.zeros((len(q), D))
    for i, x in enumerate(q):
        s = scale * (k @ x)
        p = np.exp(s - s.max())
        l = p.sum()
        out[i] = p @ v / l
        e_s = (D + 2) * U * scale * (np.abs(k) @ np.abs(x)).max() + scale * 2.0 ** -39 * np.abs(x).max() * np.abs(k).sum(1).max()
        e_p = e_s + 8 * U * (np.abs(s).max() + abs(s.max() + np.log(l)) + np.abs(ve).max()) + 8 * U
        A = p @ np.abs(v) / l
        tol[i] = 1.1 * ((2 * e_p + 2 * n * U + B16) * A + 2.0 ** -25 * np.abs(v).sum(0) / l + B16 * np.abs(out[i]))
    return out, tol


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("heads,D", [(2, 64), (7, 128), (12, 64), (12, 128), (3, 256), (40, 64), (40, 128)])
@pytest.mark.parametrize("gap", [7, 12, 24, 31, 34, 60, 96])
def test_attention_next_to_a_block_of_far_larger_scale(gap, heads, D, kind):
    """A block of values whose scale is 2^gap of the others', where nothing of it is in most columns: codes of 0 but for one row of
    no weight.  What the other blocks hold in those columns is the result.  In the first, a middle and the last block, and
    in the same 16 keys as others (blocks of 8)."""
    g = np.random.default_rng(gap)
    n, least = 200, -48 if gap > 48 else -gap // 2
    for block, big in ((16, 0), (16, 5), (16, 12), (8, 1), (1, 70)):
        blocks = -(-n // block)
        of = np.arange(n) // block
        scales = np.full((1, 2, 1, blocks), 127, np.uint8)
        scales[0, 0] = 118
        scales[0, 1] = 127 + least + g.integers(0, 2, blocks)
        scales[0, 1, 0, big] = 127 + least + gap
        k = ref.nearest(g.standard_normal((n, D)) * 60, kind)
        v = ref.nearest(g.standard_normal((n, D)) * 60, kind)
        here = np.flatnonzero(of == big)
        v[here] = 0
        k[here[-1]] = ref.nearest(np.full(D, -100.0), kind)         # the row of no weight: queries are positive
        v[here[-1], :3] = ref.nearest(np.array([100.0, -7.0, 1.0]), kind)
        codes = np.stack([k, v])[None, :, None]
        q = torch.from_numpy(np.abs(g.standard_normal((1, heads, D))).astype(np.float32)).bfloat16().cuda()
        kv = torch.from_numpy(np.ascontiguousarray(codes)).cuda().view(CODES[kind])
        got = sv.sharpv_tree_attention_q8(q, kv, torch.from_numpy(scales).cuda(), block, 0, _i32([0]), _i32([n]), _i32([0, 1]))
        e = ref.clamped(scales[0, :, 0])
        want, tol = _attention(_f64(q)[0], ref.values_of(k, kind), e[0][of], ref.values_of(v, kind), e[1][of], D ** -0.5)
        worst = np.max(np.abs(_f64(got["out"])[0] - want) / tol)
        assert worst <= 1, f"blocks of {block}, the far one {big}: {worst:.3e} of the bound"


# ------------------------------------------------------------------------------------------ large queries, large scales
@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("heads,D", [(1, 64), (7, 128), (12, 64), (12, 128), (3, 256), (40, 128)])
def test_attention_of_large_queries_over_keys_of_zero_with_the_largest_scale(heads, D, kind):
    """All scores are 0 whatever a query's size times a key's scale is.  Every weight is 1: out is the values' mean, of whole numbers
    under 2^24, rounded once; their sum is divided by a power of two, or by multiplying with a reciprocal: 2 u more."""
    n = 61
    g = np.random.default_rng(D)
    v = g.integers(1, 9, (n, D)).astype(np.float64)
    kv = np.zeros((1, 2, 1, 64, D), np.uint8)
    kv[0, 1, 0, :n] = ref.nearest(v, kind)
    scales = torch.tensor([[[[175] * 4], [[127] * 4]]], dtype=torch.uint8, device="cuda")
    q = torch.full((1, heads, D), 1.5 * 2.0 ** 118, device="cuda").bfloat16()
    got = sv.sharpv_tree_attention_q8(q, torch.from_numpy(kv).cuda().view(CODES[kind]), scales, 16, 0, _i32([0]), _i32([n]), _i32([0, 1]))
    want = v.mean(0)
    assert np.all(np.abs(_f64(got["out"])[0] - want) <= (B16 + 8 * U) * want)
    assert np.all(np.abs(_f64(got["lse"]) - np.log(n)) <= 16 * U * np.log(n))


# ------------------------------------------------------------------------------------------ heads far apart
@pytest.mark.parametrize("n", [1, 2])
def test_norm_and_rotation_straight_into_a_long_cache(n):
    """Keys into a plane whose heads are 256 MB apart, one token and two."""
    cache = torch.zeros((8, 1 << 20, 128), dtype=torch.bfloat16, device="cuda")
    q, k = (torch.randn((n, 8, 128), device="cuda").bfloat16() for _ in range(2))
    want = sv.sharpv_qk_norm_rope(q, k, _i32(np.arange(n)[None] + 70000), [0] * 64, 1e6, norm=True)
    at = 1000003
    got = sv.sharpv_qk_norm_rope(q, k, _i32(np.arange(n)[None] + 70000), [0] * 64, 1e6, norm=True,
                                 out={"q": q, "k": cache[:, at:at + n].transpose(0, 1)})
    assert torch.equal(got["q"], want["q"]) and torch.equal(cache[:, at:at + n].transpose(0, 1), want["k"])
    assert not bool(cache[:, at - 1].any()) and not bool(cache[:, at + n].any())


def test_norm_and_rotation_refuse_outputs_that_overlap():
    """Refused before any launch: the values stay what they are.  Interleaving rows are taken."""
    qkv = torch.randn((50, 12, 64), device="cuda")
    before, pos = qkv.clone(), _i32(np.arange(50)[None])
    q, k = qkv[:, :8], qkv[:, 8:10]
    for out in ({"q": q, "k": q[:, :2]}, {"q": qkv[:, 1:9], "k": k}, {"q": q, "k": qkv[:, 9:11]}, {"q": torch.empty_like(q), "k": qkv[:, 7:9]},
                {"q": torch.empty((50, 1, 64), device="cuda").expand(50, 8, 64), "k": k}):
        with pytest.raises((sv.SharpVError, ValueError)):
            sv.sharpv_qk_norm_rope(q, k, pos, [0] * 32, 1e4, out=out)
        assert torch.equal(qkv, before)
    want = sv.sharpv_qk_norm_rope(q, k, pos, [0] * 32, 1e4)
    wide = torch.zeros((50, 14, 64), device="cuda")                 # outputs between each other's rows
    got = sv.sharpv_qk_norm_rope(q, k, pos, [0] * 32, 1e4, out={"q": wide[:, 3:11], "k": wide[:, 11:13]})
    assert torch.equal(got["q"], want["q"]) and torch.equal(got["k"], want["k"]) and not bool(wide[:, [0, 1, 2, 13]].any())
    got = sv.sharpv_qk_norm_rope(q, k, pos, [0] * 32, 1e4, out={"q": q, "k": qkv[:, 10:12]})       # keys where the values were
    assert torch.equal(got["q"], want["q"]) and torch.equal(got["k"], want["k"]) and torch.equal(k, before[:, 8:10])


# ------------------------------------------------------------------------------------------ codes and scales in one allocation
@pytest.mark.parametrize("kind", ["e4m3", "i8"])
def test_append_and_attention_with_codes_and_scales_layer_by_layer(kind):
    """Scales behind the codes of their layer: nothing overlaps, and all is as it is with the two apart.  A scale for all heads, or
    scales over codes, are refused and leave everything as it was."""
    L, H, T, D, block = 3, 2, 96, 64, 16
    layer = 2 * H * T * D + 2 * H * 16
    raw = torch.zeros(L * layer, dtype=torch.uint8, device="cuda")
    codes = raw.as_strided((L, 2, H, T, D), (layer, H * T * D, T * D, D, 1)).view(CODES[kind])
    scales = raw.as_strided((L, 2, H, T // block), (layer, 16 * H, 16, 1), 2 * H * T * D)
    src = torch.randn((L, 2, H, 50, D), device="cuda").bfloat16()
    apart, its = torch.zeros((L, 2, H, T, D), dtype=CODES[kind], device="cuda"), torch.zeros((L, 2, H, T // block), dtype=torch.uint8, device="cuda")
    lists = _i32(np.arange(50)), _i32([0, 20, 50]), _i32([0, 48])
    before = raw.clone()
    for bad in (scales[:, :, :1].expand(L, 2, H, T // block), raw.as_strided((L, 2, H, T // block), (layer, 16 * H, 16, 1))):
        with pytest.raises(sv.SharpVError):
            sv.sharpv_kv_append_q8(src, codes, bad, block, *lists)
        assert torch.equal(raw, before)
    sv.sharpv_kv_append_q8(src, codes, scales, block, *lists)
    sv.sharpv_kv_append_q8(src, apart, its, block, *lists)
    assert torch.equal(codes.view(torch.uint8), apart.view(torch.uint8)) and torch.equal(scales, its)
    q, dk = torch.randn((3, 6, D), device="cuda").bfloat16(), torch.randn((3, H, D), device="cuda").bfloat16()
    got, want = (sv.sharpv_tree_attention_q8(q, c, s, block, 1, _i32([0, 48]), _i32([20, 30]), _i32([0, 1, 3]), dk, dk)
                 for c, s in ((codes, scales), (apart, its)))
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])


# ------------------------------------------------------------------------------------------ lists with room behind them
@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("source", ["bf16", "i8"])
@pytest.mark.parametrize("lens,rows", [([2], [63]), ([2, 62], [64, 127]), ([0, 63, 17], [5, 0, 700]), ([40] * 40, [3] * 39 + [300])])
def test_append_with_a_list_that_has_room_behind(lens, rows, source, kind):
    """capacity over the rows there are (a kept list's usual form; what lies behind is no row at all), last sequences that begin late in a
    block and so need a tile more than their rows fill."""
    s = Store(source, kind, 64, 2, 128, lens, rows, seed=len(lens))
    for room in (1, 64, 5000):
        fresh = Store(source, kind, 64, 2, 128, lens, rows, seed=len(lens))
        fresh.pos = np.concatenate([s.pos, np.full(room, -7)])
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        fresh.call(status_word=status)
        fresh.pos = s.pos
        codes, scales = fresh.expected()
        assert status.item() == 0
        assert np.array_equal(fresh.dst_scales.cpu().numpy(), scales) and np.array_equal(_bits(fresh.dst), codes)


# ------------------------------------------------------------------------------------------ pairs
def test_norm_and_rotation_take_axes_by_value():
    """A list, bytes, an array or a tensor of whole numbers of any width say the same; more than a byte's is refused."""
    q = torch.randn((5, 4, 128), device="cuda")
    pos, axis = _i32(np.stack([np.arange(5), 3 * np.arange(5) + 1])), [0, 1, 1, 0, 1, 0, 0, 0]
    want = sv.sharpv_qk_norm_rope(q, q, pos, axis, 1e4)["q"]
    for same in (bytes(axis), bytearray(axis), tuple(axis), np.array(axis), np.array(axis, np.uint8), np.array(axis, np.int32), torch.tensor(axis)):
        assert torch.equal(sv.sharpv_qk_norm_rope(q, q, pos, same, 1e4)["q"], want)
    for bad in ([0] * 7 + [256], np.array([-1] * 8)):
        with pytest.raises(ValueError):
            sv.sharpv_qk_norm_rope(q, q, pos, bad, 1e4)


# ------------------------------------------------------------------------------------------ copies
def test_copies_of_int8_blocks_with_the_code_that_has_no_counterpart():
    """-128, which a negative infinity becomes, is past 127 * 2^e: a copy of its block has the next scale, and odd codes are rounded to
    even ones.  Blocks without it, odd codes and all, are the same values."""
    x = torch.randn((1, 2, 1, 64, 32), device="cuda")
    x[0, :, 0, 20, 3] = -INF
    one, two, scales, its = *(torch.zeros((1, 2, 1, 64, 32), dtype=torch.int8, device="cuda") for _ in range(2)), \
        *(torch.zeros((1, 2, 1, 4), dtype=torch.uint8, device="cuda") for _ in range(2))
    rows = _i32(np.arange(64)), _i32([0, 64]), _i32([0])
    sv.sharpv_kv_append_q8(x, one, scales, 16, *rows)
    sv.sharpv_kv_append_q8(one, two, its, 16, *rows, src_scales=scales)
    assert bool((one[0, :, 0, 20, 3] == -128).all())
    same = [0, 2, 3]
    assert torch.equal(its[..., same], scales[..., same]) and torch.equal(its[..., 1], scales[..., 1] + 1)
    a, b = one.view(1, 2, 1, 4, 16, 32), two.view(1, 2, 1, 4, 16, 32)
    assert torch.equal(a[:, :, :, same], b[:, :, :, same])
    codes = a[:, :, :, 1].cpu().numpy()
    assert np.any(codes % 2) and np.array_equal(b[:, :, :, 1].cpu().numpy(), np.rint(codes / 2).astype(np.int8))

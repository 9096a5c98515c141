"""Head norm with rotation, rows into a cache in 8 bits, and attention over such a cache, on the GPU."""
import numpy as np
import pytest
import torch

import q8_reference as ref
from decode_reference import B16, U
from helpers import Guarded
from paper_2511_08003_b200 import binding as sv

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
CODES = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}
NAN, INF = float("nan"), float("inf")


def _i32(v):
    return torch.tensor(np.asarray(v, dtype=np.int64).astype(np.int32), device="cuda")


def _f64(t):
    return t.detach().double().cpu().numpy()


def _bits(t):
    return t.view(torch.uint8).cpu().numpy()


def _needs_capture():
    if sv.lib().sharpv_version() >= 200 and sv.lib_path() != sv._build.LIB_PATH:
        pytest.skip("with the range-checking library every call is followed by a synchronise, which a capture refuses")


# ------------------------------------------------------------------------------------------ norm and rotation
def _axes(pairs, axes, mixed):
    return np.arange(pairs) % axes if mixed else np.sort(np.arange(pairs) % axes)


def _check_rope(dtype, N, HQ, H, D, rotary, axes=1, norm=True, weights=True, mixed=False, layout="fused", far=5000, eps=1e-6,
                base=1e6, seed=0, spread=1.0):
    g = np.random.default_rng(seed)
    dt = DT[dtype]
    x = torch.from_numpy(g.standard_normal((N, HQ + 2 * H, D), dtype=np.float32) * np.float32(spread)).to(dt).cuda()
    if layout == "fused":
        q, k = x[:, :HQ], x[:, HQ:HQ + H]
    elif layout == "head_major":
        q, k = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (x[:, :HQ], x[:, HQ:HQ + H]))
    else:
        q, k = x[:, :HQ].contiguous(), x[:, HQ:HQ + H].contiguous()
    axis = _axes(rotary // 2, axes, mixed)
    pos = g.integers(-far, far, (axes, N))
    w = [torch.from_numpy(1 + 0.5 * g.standard_normal(D).astype(np.float32)).to(dt).cuda() if weights and norm else None for _ in range(2)]
    mem = Guarded()
    out = {"q": mem.empty((N, HQ, D), dt), "k": mem.empty((N, H, D), dt)}
    want = [ref.norm_rope(_f64(t), pos, axis, base, None if y is None else _f64(y), float(np.float32(eps)), norm, U if dtype == "f32" else B16)
            for t, y in ((q, w[0]), (k, w[1]))]
    before = x.clone()
    got = sv.sharpv_qk_norm_rope(q, k, _i32(pos), [int(a) for a in axis], base, norm=norm, q_weight=w[0], k_weight=w[1], eps=eps, out=out)
    mem.check("norm and rotation")
    assert torch.equal(x, before)
    for name, (o, tol) in zip("qk", want):
        worst = np.max(np.abs(_f64(got[name]) - o) - tol, initial=-1.0)
        assert worst <= 0, f"{name} is {worst:.3e} past its bound"
    # in place, where the outputs are the inputs' own views
    same = sv.sharpv_qk_norm_rope(q, k, _i32(pos), bytes(int(a) for a in axis), base, norm=norm, q_weight=w[0], k_weight=w[1], eps=eps,
                                  out={"q": q, "k": k})
    assert torch.equal(same["q"], got["q"]) and torch.equal(same["k"], got["k"])
    if layout == "fused":
        assert torch.equal(x[:, HQ + H:], before[:, HQ + H:])       # the values beside them
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,HQ,H,D,rotary,axes", [
    (1, 1, 1, 16, 16, 1), (1, 28, 4, 128, 128, 3), (16, 28, 4, 128, 128, 3), (37, 14, 2, 64, 64, 2), (5, 6, 3, 80, 80, 3),
    (9, 3, 1, 96, 48, 2), (3, 64, 8, 256, 256, 3), (700, 28, 4, 128, 128, 3), (1203, 5, 1, 80, 32, 1), (2, 7, 1, 256, 64, 8),
    (4, 9, 2, 136, 112, 1), (3, 130, 2, 64, 64, 1), (1, 300, 20, 64, 64, 1),
])
def test_qk_norm_rope(N, HQ, H, D, rotary, axes, dtype):
    _check_rope(dtype, N, HQ, H, D, rotary, axes, seed=N + D)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("change", [dict(norm=False), dict(weights=False), dict(mixed=True, axes=3), dict(layout="head_major"),
                                    dict(layout="dense"), dict(rotary=0), dict(rotary=0, N=1), dict(far=2 ** 31 - 1), dict(eps=10.0),
                                    dict(base=1e4, rotary=32), dict(spread=1e-4), dict(spread=3e4)],
                         ids=lambda c: "-".join(c))
def test_qk_norm_rope_variants(change, dtype):
    _check_rope(dtype, **{**dict(N=50, HQ=8, H=2, D=128, rotary=128), **change})


def test_qk_norm_rope_rows_of_zeros_and_what_is_not_finite():
    q = torch.randn((3, 4, 64), device="cuda").bfloat16()
    q[1, 2] = 0
    q[0, 1, 5] = NAN
    got = sv.sharpv_qk_norm_rope(q, q[:, :1].clone(), _i32([[1, 2, 3]]), [0] * 32, 1e4, norm=True)["q"]
    assert bool((got[1, 2] == 0).all()) and bool(torch.isnan(got[0, 1]).all())
    rest = torch.ones((3, 4), dtype=torch.bool, device="cuda")
    rest[0, 1] = False
    assert bool(torch.isfinite(got[rest]).all())


def test_qk_norm_rope_no_tokens_and_outputs_with_strides():
    e = torch.empty((0, 4, 64), device="cuda")
    got = sv.sharpv_qk_norm_rope(e, e[:, :2], torch.empty((1, 0), dtype=torch.int32, device="cuda"), [0] * 32, 1e4)
    assert got["q"].shape == (0, 4, 64)
    # keys straight into a cache's plane: heads far apart, rows behind one another
    q, k = torch.randn((9, 4, 64), device="cuda"), torch.randn((9, 2, 64), device="cuda")
    pos = _i32(np.arange(9)[None])
    dense = sv.sharpv_qk_norm_rope(q, k, pos, [0] * 32, 1e4, norm=True)
    cache = torch.full((2, 20, 64), 7.0, device="cuda")
    sv.sharpv_qk_norm_rope(q, k, pos, [0] * 32, 1e4, norm=True, out={"q": torch.empty_like(q), "k": cache[:, 5:14].transpose(0, 1)})
    assert torch.equal(cache[:, 5:14].transpose(0, 1), dense["k"])
    assert bool((cache[:, :5] == 7).all()) and bool((cache[:, 14:] == 7).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 40, 700])
def test_qk_norm_rope_of_text_whose_axes_share_their_positions(N, dtype):
    """A text token's axes all hold the same number: a view without a stride between the axes will do."""
    q = torch.randn((N, 6, 64), device="cuda").to(DT[dtype])
    pos, axis = _i32(np.arange(N) * 7 - 3), [i % 3 for i in range(32)]
    want = sv.sharpv_qk_norm_rope(q, q[:, :2], pos.expand(3, N).contiguous(), axis, 1e6, norm=True)
    got = sv.sharpv_qk_norm_rope(q, q[:, :2], pos.expand(3, N), axis, 1e6, norm=True)
    assert torch.equal(got["q"], want["q"]) and torch.equal(got["k"], want["k"])


def test_qk_norm_rope_agrees_with_the_compaction():
    """Rotation to a position by this call is the rotation that sharpv_kv_compact_rope adds to keys at position 0."""
    n, D = 6, 64
    k = torch.randn((n, 1, D), device="cuda")
    got = sv.sharpv_qk_norm_rope(k, k, _i32(np.arange(n)[None]), [0] * 32, 1e4)["k"]
    kv = torch.zeros((1, 2, 1, 20, D), device="cuda")
    kv[0, 0, 0, 8:8 + n] = got[:, 0]
    dst = torch.zeros_like(kv)
    # the rows move from 8 .. to 0 ..: turned back by 8
    sv.sharpv_kv_compact_rope(kv, dst, _i32(np.arange(8, 8 + n)), _i32([0, n]), _i32([0, 20]), n, D, 1e4)
    back = sv.sharpv_qk_norm_rope(k, k, _i32(np.arange(n)[None] - 8), [0] * 32, 1e4)["k"]
    assert float((dst[0, 0, 0, :n] - back[:, 0]).abs().max()) <= 40 * U * float(k.abs().max())


# ------------------------------------------------------------------------------------------ rows into the cache
class Store:
    """A cache in 8 bits that has rows already, and a source for more."""

    def __init__(self, source, kind, block, H, D, lens, rows, seed=0, layers=2, spare=9, src_block=None, token_major=False, spread=1.0,
                 gap=0):
        g = np.random.default_rng(seed)
        self.kind, self.block, self.source, self.rows, self.lens = kind, block, source, np.asarray(rows), np.asarray(lens)
        room = [-(-(a + b + gap) // block) * block for a, b in zip(lens, rows)]
        self.begin = np.concatenate([[0], np.cumsum(room)])[:-1].astype(int)
        T, n = int(sum(room)) + 3, int(sum(rows))
        self.codes = g.integers(0, 256, (layers, 2, H, T, D)).astype(np.uint8)
        if kind == "e4m3":
            self.codes[(self.codes & 127) == 127] = 5
        self.scales = g.integers(118, 126, (layers, 2, H, -(-T // block))).astype(np.uint8)
        self.S = n + spare
        self.src_block = src_block or block
        if source in CODES:
            bits = g.integers(0, 256, (layers, 2, H, self.S, D)).astype(np.uint8)
            if source == "e4m3":
                bits[(bits & 127) == 127] = 3
            s = g.integers(115, 130, (layers, 2, H, -(-self.S // self.src_block))).astype(np.uint8)
            self.x = ref.values_of(bits, source) * 2.0 ** ref.clamped(s)[..., np.arange(self.S) // self.src_block][..., None]
            self.src, self.src_scales = torch.from_numpy(bits).cuda().view(CODES[source]), torch.from_numpy(s).cuda()
        else:
            x = g.standard_normal((layers, 2, H, self.S, D), dtype=np.float32) * np.float32(spread)
            x *= np.exp2(g.integers(-9, 3, (layers, 2, H, self.S, 1))).astype(np.float32)
            self.src = torch.from_numpy(x).to(DT[source]).cuda()
            self.x, self.src_scales = _f64(self.src), None
        self.pos = np.sort(g.permutation(self.S)[:n])
        self.offsets = np.concatenate([[0], np.cumsum(rows)]).astype(int)
        dst = torch.from_numpy(self.codes)
        if token_major:
            dst = dst.permute(0, 3, 1, 2, 4).contiguous().permute(0, 2, 3, 1, 4)
        self.dst = (dst.cuda() if not token_major else dst.permute(0, 3, 1, 2, 4).contiguous().cuda().permute(0, 2, 3, 1, 4)).view(CODES[kind])
        self.dst_scales = torch.from_numpy(self.scales.copy()).cuda()

    def call(self, **kw):
        return sv.sharpv_kv_append_q8(self.src, self.dst, self.dst_scales, self.block, _i32(self.pos), _i32(self.offsets),
                                      _i32(self.begin + self.lens), src_scales=self.src_scales,
                                      src_block_tokens=self.src_block if self.src_scales is not None else None, **kw)

    def expected(self, layers=None):
        codes, scales = self.codes.copy(), self.scales.copy()
        for l, kv, h in np.ndindex(codes.shape[:3]):
            if layers is not None and not layers[0] <= l < layers[1]:
                continue
            for b in range(len(self.rows)):
                if self.rows[b]:
                    x = self.x[l, kv, h][self.pos[self.offsets[b]:self.offsets[b + 1]]]
                    ref.append(x, codes[l, kv, h], scales[l, kv, h], self.kind, self.block, int(self.begin[b] + self.lens[b]))
        return codes, scales

    def check(self, **kw):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.call(status_word=status, **kw)
        assert status.item() == 0
        codes, scales = self.expected()
        assert np.array_equal(self.dst_scales.cpu().numpy(), scales)
        got = _bits(self.dst)
        assert np.array_equal(got, codes), f"{np.mean(got != codes):.2e} of the codes differ"
        return self


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("source", ["f32", "bf16", "e4m3", "i8"])
@pytest.mark.parametrize("block,H,D,lens,rows", [
    (16, 1, 16, [0], [1]),
    (64, 2, 128, [3, 0, 64, 70, 127], [2, 1, 5, 0, 3]),             # pieces of a warp, blocks begun before
    (32, 2, 64, [0, 0, 31, 17], [100, 0, 33, 900]),
    (1, 2, 80, [0, 5], [40, 7]),                                    # a scale a row
    (128, 1, 128, [100, 0], [400, 129]),
    (256, 2, 96, [10, 255], [700, 3]),                              # a block in two goes
    (256, 1, 256, [1, 0], [300, 600]),
    (16, 3, 112, [7, 0, 0], [90, 200, 1]),
    (2, 1, 16, [1, 0], [1500, 3]),                                  # more rows than a tile's list holds
])
def test_kv_append_q8(block, H, D, lens, rows, source, kind):
    Store(source, kind, block, H, D, lens, rows, seed=block + D).check()


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
def test_kv_append_q8_layouts_blocks_and_many_sequences(kind):
    Store("bf16", kind, 32, 2, 64, [5, 40], [100, 9], token_major=True).check()
    Store("i8", kind, 64, 2, 64, [5, 0], [100, 90], src_block=16).check()
    Store("e4m3", kind, 16, 1, 128, [0, 1], [100, 90], src_block=256).check()
    g = np.random.default_rng(1)
    Store("bf16", kind, 16, 1, 32, list(g.integers(0, 40, 600)), list(g.integers(0, 4, 600))).check()
    Store("bf16", kind, 16, 1, 32, [0] * 70, list(g.integers(0, 90, 70))).check()
    Store("f32", kind, 16, 1, 64, [3], [70], spread=1e-20).check()      # scales at their least
    Store("f32", kind, 16, 1, 64, [3], [70], spread=1e30).check()       # beyond their largest


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("source", ["f32", "bf16"])
def test_kv_append_q8_borders_ties_and_what_is_not_finite(source, kind):
    """Largest values on both sides of a scale's border, values half way between codes, zeros, infinities and NaN."""
    s = Store(source, kind, 16, 1, 64, [0], [16 * 24], spare=0, layers=1)
    x = np.zeros((16 * 24, 64), np.float32)
    g = np.random.default_rng(2)
    top = ref.TOP[kind]
    steps = np.arange(64) - 32
    for i in range(24):
        r = x[16 * i:16 * (i + 1)]
        if i < 8:                                   # the border itself, and a step of the source's type to each side
            border = np.float32(top * 2.0 ** (i - 4))
            step = 2.0 ** -7 if source == "bf16" else 2.0 ** -23
            r[3, 5] = [border, border * np.float32(1 - step), border * np.float32(1 + step)][i % 3]
            r[7] = g.standard_normal(64).astype(np.float32) * border / 8
        elif i < 16:                                # half way between codes, at every size
            r[0, 0] = top
            r[1] = steps + 0.5
            r[2] = (steps * 2 + 1) * 2.0 ** -4
            r[3] = (steps * 2 + 1) * 2.0 ** -10
            r[4] = (steps * 2 + 1) * 8
        elif i < 20:
            r[2, 1], r[5, 3], r[6, 0], r[9] = INF, -INF, NAN, g.standard_normal(64)
        elif i < 22:
            r[2, 1], r[5, 3] = INF, NAN             # nothing finite but zeros
        if i == 23:
            r[0, 0] = -0.0
    s.src = torch.from_numpy(x)[None, None, None].expand(1, 2, 1, -1, -1).contiguous().to(DT[source]).cuda()
    s.x = _f64(s.src)
    s.check()


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("source", ["e4m3", "i8"])
def test_kv_append_q8_scales_far_apart(source, kind):
    """Rows of a block whose scales differ by anything, rows of the smallest codes alone, and scales beyond what is used."""
    s = Store(source, kind, 16, 1, 64, [0, 5], [16 * 40, 70], spare=0, src_block=1)
    g = np.random.default_rng(7)
    bits = _bits(s.src).copy()
    far = g.integers(60, 200, s.src_scales.shape).astype(np.uint8)
    far[..., 200:400] = g.integers(120, 134, far[..., 200:400].shape)
    small = np.array([0, 1, 2, 0x81] if source == "e4m3" else [0, 1, 255, 0], np.uint8)
    bits[..., 100:140, :] = small[g.integers(0, 4, bits[..., 100:140, :].shape)]
    far[..., 112:128] = 127                     # a block of the smallest codes with one scale
    s.src, s.src_scales = torch.from_numpy(bits).cuda().view(CODES[source]), torch.from_numpy(far).cuda()
    s.x = ref.values_of(bits, source) * 2.0 ** ref.clamped(far)[..., None]
    s.check()


def test_kv_append_q8_layer_range_and_twice():
    s = Store("bf16", "e4m3", 32, 2, 64, [5, 40], [100, 9], layers=4)
    s.call(layer_begin=1, layer_end=3)
    codes, scales = s.expected((1, 3))
    assert np.array_equal(_bits(s.dst), codes) and np.array_equal(s.dst_scales.cpu().numpy(), scales)
    s.call(layer_begin=1, layer_end=3)              # the same rows again: nothing moves
    assert np.array_equal(_bits(s.dst), codes) and np.array_equal(s.dst_scales.cpu().numpy(), scales)


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
def test_kv_append_q8_copies_of_whole_blocks_are_the_same_values(kind):
    """Block by block onto the same borders, a cache in 8 bits is copied without another rounding."""
    s = Store("bf16", kind, 32, 2, 64, [0, 0], [96, 64], spare=0)
    s.check()
    n = 160
    new, scales = torch.zeros_like(s.dst), torch.zeros_like(s.dst_scales)
    # the copy of the copy (which has the least scales) is the copy
    sv.sharpv_kv_append_q8(s.dst, new, scales, 32, _i32(np.arange(n)), _i32([0, n]), _i32([0]), src_scales=s.dst_scales)
    value = lambda c, e: ref.values_of(_bits(c), kind)[..., :n, :] * 2.0 ** ref.clamped(e.cpu().numpy())[..., np.arange(n) // 32][..., None]  # noqa: E731
    assert np.array_equal(value(new, scales), value(s.dst, s.dst_scales))


def test_kv_append_q8_tables_that_reach_outside():
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    # a bad source row is left out, the others are as they would be
    s = Store("bf16", "e4m3", 16, 1, 64, [0], [40])
    s.pos[17] = s.S + 5
    s.call(status_word=status)
    assert status.item() == sv.Status.ERR_BOUNDS
    codes, scales = s.codes.copy(), s.scales.copy()
    for l, kv in np.ndindex(codes.shape[:2]):
        x = np.where((s.pos < s.S)[:, None], s.x[l, kv, 0][np.minimum(s.pos, s.S - 1)], 0.0)
        old = codes[l, kv, 0, 17].copy()
        ref.append(x, codes[l, kv, 0], scales[l, kv, 0], "e4m3", 16, 0)
        codes[l, kv, 0, 17] = old
    assert np.array_equal(_bits(s.dst), codes) and np.array_equal(s.dst_scales.cpu().numpy(), scales)
    # rows in front of the cache and behind it
    for at in (-20, None):
        status.zero_()
        s = Store("bf16", "i8", 16, 1, 64, [0], [40])
        to = at if at is not None else s.dst.shape[3] - 10
        sv.sharpv_kv_append_q8(s.src, s.dst, s.dst_scales, 16, _i32(s.pos), _i32([0, 40]), _i32([to]), status_word=status)
        assert status.item() == sv.Status.ERR_BOUNDS
        codes, scales = s.codes.copy(), s.scales.copy()
        cut = slice(20, 40) if at is not None else slice(0, 10)
        for l, kv in np.ndindex(codes.shape[:2]):
            ref.append(s.x[l, kv, 0][s.pos[cut]], codes[l, kv, 0], scales[l, kv, 0], "i8", 16, max(to, 0))
        assert np.array_equal(_bits(s.dst), codes) and np.array_equal(s.dst_scales.cpu().numpy(), scales)
    # more rows than capacity
    status.zero_()
    s = Store("bf16", "i8", 16, 1, 64, [0], [40])
    s.call(capacity=33, status_word=status)
    assert status.item() == sv.Status.ERR_CAPACITY
    codes, scales = s.codes.copy(), s.scales.copy()
    for l, kv in np.ndindex(codes.shape[:2]):
        ref.append(s.x[l, kv, 0][s.pos[:33]], codes[l, kv, 0], scales[l, kv, 0], "i8", 16, 0)
    assert np.array_equal(_bits(s.dst), codes) and np.array_equal(s.dst_scales.cpu().numpy(), scales)


# ------------------------------------------------------------------------------------------ attention
class Attn:
    """A cache in 8 bits whose rows and scales outside the sequences are what disturbs most, query nodes behind the last sequence."""

    def __init__(self, kind, block, H, G, D, lens, nodes, seed=0, layers=2, layer=1, gap=3, spare=2, spread=1.0, tree="random",
                 token_major=False, draft=True, wide=4, words=None):
        g = np.random.default_rng(seed)
        self.kind, self.block, self.H, self.G, self.D, self.layer = kind, block, H, G, D, layer
        self.length = np.asarray(lens)
        self.begin = np.concatenate([[0], np.cumsum(self.length + gap)])[:-1].astype(int) + gap
        self.offsets = np.concatenate([[0], np.cumsum(nodes)]).astype(int)
        T, N = int(self.begin[-1] + self.length[-1]) + gap, int(self.offsets[-1]) + spare
        codes = np.full((layers, 2, H, T, D), 0x7F if kind == "e4m3" else 0x80, np.uint8)
        scales = np.full((layers, 2, H, -(-T // block)), 255, np.uint8)
        for b, n in zip(self.begin, self.length):
            x = g.standard_normal((2, H, n, D))
            codes[layer, :, :, b:b + n] = ref.nearest(x * (90.0 if kind == "e4m3" else 30.0), kind)
            if n:
                blocks = np.arange(b // block, (b + n - 1) // block + 1)
                scales[layer, 0, :, blocks] = g.integers(121 - (kind == "e4m3"), 123 - (kind == "e4m3"), (len(blocks), H))
                scales[layer, 1, :, blocks] = g.integers(122 - wide, 122 + wide, (len(blocks), H))
        self.codes, self.scales = codes, scales
        t = torch.from_numpy(codes)
        self.kv = (t.permute(0, 3, 1, 2, 4).contiguous().cuda().permute(0, 2, 3, 1, 4) if token_major else t.cuda()).view(CODES[kind])
        self.sc = torch.from_numpy(scales).cuda()
        qkv = torch.from_numpy(g.standard_normal((N, H * G + 2 * H, D), dtype=np.float32))
        qkv[:, :H * G] *= spread
        qkv[self.offsets[-1]:] = NAN
        qkv = qkv.bfloat16().cuda()                                 # side by side, as a fused projection leaves them
        self.q, self.dk, self.dv = qkv[:, :H * G], qkv[:, H * G:H * G + H], qkv[:, H * G + H:]
        if not draft:
            self.dk = self.dv = None
        self.tree = None
        if tree == "random":
            words = words or (max(max(nodes), 1) + 31) // 32
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

    def args(self):
        return (self.q, self.kv, self.sc, self.block, self.layer, *self.tables, self.dk, self.dv, self.tree)

    def reference(self, scale):
        c, s = self.codes[self.layer], self.scales[self.layer]
        return ref.attention(_f64(self.q), c[0], s[0], c[1], s[1], self.kind, self.block, self.begin, self.length, self.offsets,
                             None if self.dk is None else _f64(self.dk), None if self.dv is None else _f64(self.dv),
                             None if self.tree is None else self.tree.cpu().numpy(), scale)

    def check(self, scale=None, what=""):
        mem = Guarded()
        N, HQ = self.q.shape[0], self.H * self.G
        out = {"out": mem.empty(self.q.shape, torch.bfloat16), "lse": mem.empty((N, HQ), torch.float32)}
        out["out"].fill_(7.0)
        out["lse"].fill_(7.0)
        ws = mem.empty(sv.sharpv_tree_attention_q8_workspace_bytes(len(self.length), N, HQ, self.H, self.D), torch.uint8)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = sv.sharpv_tree_attention_q8(*self.args(), scale=scale, out=out, workspace=ws, status_word=status)
        mem.check(what)
        assert status.item() == 0
        o, lse, o_tol, lse_tol = self.reference(self.D ** -0.5 if scale is None else scale)
        n = self.offsets[-1]
        assert bool((got["out"][n:] == 7).all()) and bool((got["lse"][n:] == 7).all()), "rows of no sequence were written"
        go, gl = _f64(got["out"])[:n], _f64(got["lse"])[:n]
        empty = np.isneginf(lse[:n])
        assert np.array_equal(np.isneginf(gl), empty)
        assert np.all(go[empty] == 0)
        assert np.all(np.isfinite(go)), what
        worst = np.max(np.abs(go - o[:n]) - o_tol[:n], initial=-1.0)
        assert worst <= 0, f"{what}: out is {worst:.3e} past its bound"
        worst = np.max(np.abs(gl[~empty] - lse[:n][~empty]) - lse_tol[:n][~empty], initial=-1.0)
        assert worst <= 0, f"{what}: lse is {worst:.3e} past its bound"
        return got


SHAPES = [
    # block, kv heads, group, head_dim, lens, nodes
    (32, 2, 7, 64, [100], [1]),
    (16, 1, 1, 16, [0, 1, 2], [1, 1, 1]),
    (64, 2, 3, 80, [33, 0, 257], [5, 2, 1]),
    (1, 1, 8, 128, [128, 31, 64, 65], [1, 0, 4, 2]),
    (128, 4, 7, 128, [700, 1], [9, 33]),
    (16, 3, 2, 256, [65, 190], [3, 20]),
    (256, 2, 1, 128, [129, 0, 511], [70, 40, 1]),
    (8, 1, 5, 96, [1030], [64]),
    (32, 2, 16, 64, [300, 20], [12, 1]),
    (64, 1, 7, 144, [77], [6]),
    (64, 1, 4, 128, [1500, 3], [130, 64]),
    (32, 1, 2, 64, [640], [300]),
    (16, 1, 100, 128, [200, 9], [2, 1]),
    (16, 1, 130, 64, [70, 300], [2, 3]),
]


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("tree", ["random", None])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "h%dx%d_d%d_%s" % (s[1], s[2], s[3], "-".join(map(str, s[5]))))
def test_tree_attention_q8(shape, tree, kind):
    block, H, G, D, lens, nodes = shape
    Attn(kind, block, H, G, D, lens, nodes, seed=sum(lens) + D, tree=tree).check()


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("name", ["token_major", "no_draft", "no_draft_empty", "peaked", "long", "few_words", "many", "long_chain", "wide",
                                  "one_in_many_parts", "far_scales", "alternating"])
def test_tree_attention_q8_layouts_and_ranges(name, kind):
    if name == "token_major":
        Attn(kind, 16, 2, 4, 64, [90, 210], [3, 7], token_major=True).check()
        Attn(kind, 16, 2, 4, 64, [90, 210], [30, 70], token_major=True).check()
    elif name == "no_draft":
        Attn(kind, 32, 2, 4, 128, [75, 300], [1, 3], draft=False, tree=None).check()
        Attn(kind, 32, 2, 4, 128, [75, 300], [9, 30], draft=False, tree=None).check()
    elif name == "no_draft_empty":          # rows without any key
        for nodes in ([2, 3, 1], [2, 30, 1]):
            got = Attn(kind, 16, 2, 4, 128, [0, 40, 0], nodes, draft=False, tree=None).check()
            assert bool((got["out"][:2] == 0).all()) and bool(torch.isneginf(got["lse"][:2]).all())
    elif name == "peaked":                  # the running maximum moves often and far
        Attn(kind, 16, 2, 7, 128, [900, 40], [2, 2], spread=40.0).check()
        Attn(kind, 16, 1, 7, 128, [900, 40], [50, 20], spread=40.0).check()
    elif name == "long":
        Attn(kind, 64, 1, 7, 128, [20011], [1]).check()
        Attn(kind, 64, 1, 4, 64, [9973, 12], [33, 1]).check()
    elif name == "few_words":
        Attn(kind, 16, 1, 2, 64, [50], [70], words=1).check()
    elif name == "many":
        g = np.random.default_rng(5)
        Attn(kind, 16, 1, 2, 64, list(g.integers(0, 40, 700)), list(g.integers(0, 3, 700)), gap=1).check()
    elif name == "long_chain":
        Attn(kind, 128, 2, 4, 128, [333], [700], tree=None).check()
    elif name == "wide":                    # values of blocks 2^16 apart
        Attn(kind, 16, 1, 4, 128, [700], [2], wide=8).check()
        Attn(kind, 16, 1, 4, 128, [700], [40], wide=8).check()
    elif name == "one_in_many_parts":
        Attn(kind, 64, 1, 2, 256, [12007], [1]).check()
        Attn(kind, 64, 1, 4, 128, [9000] + [70] * 39, [1] * 40).check()
    elif name == "far_scales":              # the ends of what scales may be, and bytes beyond them
        for nodes in ([2], [40]):
            c = Attn(kind, 16, 1, 4, 64, [300], nodes)
            c.scales[c.layer, 1, 0, ::2] = 79
            c.scales[c.layer, 1, 0, 1::4] = 0
            c.sc.copy_(torch.from_numpy(c.scales))
            c.check()
            c.scales[c.layer, 1, 0, 2] = 175
            c.scales[c.layer, 1, 0, 4] = 250
            c.scales[c.layer, 0, 0, 7] = 0
            c.sc.copy_(torch.from_numpy(c.scales))
            c.check()
    else:                                   # a row tile between the drafted tiles of others: every CTA alternates the two kinds
        Attn(kind, 16, 8, 3, 64, [70, 130, 1, 200, 64, 63, 190, 20] * 12, [3, 1, 5, 2, 4, 1, 2, 5] * 12).check()
        Attn(kind, 16, 2, 1, 256, [700], [600], tree=None).check()


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("nodes", [[3, 2], [90, 40]])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
def test_tree_attention_q8_ignores_what_is_not_seen(value, nodes, kind):
    c = Attn(kind, 16, 2, 4, 128, [100, 37], nodes, seed=5)
    last = [c.offsets[1] - 1, c.offsets[2] - 1]
    tree = c.tree.cpu().numpy()
    for b in range(2):                      # the last node of each sequence is seen by itself alone
        i = last[b] - c.offsets[b]
        rows = np.arange(c.offsets[b], c.offsets[b + 1])
        tree[rows, i // 32] &= np.int32(~(1 << (i % 32)) if i % 32 != 31 else 0x7fffffff)
        tree[last[b], i // 32] |= np.int32(1 << (i % 32)) if i % 32 != 31 else np.int32(-2 ** 31)
    c.tree.copy_(torch.from_numpy(tree))
    clean = c.check()
    c.dk[last], c.dv[last] = value, value
    got = sv.sharpv_tree_attention_q8(*c.args())
    keep = np.setdiff1d(np.arange(c.offsets[-1]), last)
    assert torch.equal(got["out"][keep], clean["out"][keep]) and torch.equal(got["lse"][keep], clean["lse"][keep])
    assert not bool(torch.isfinite(got["out"][last]).all())


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("HQ,D", [(1, 64), (7, 128), (12, 64), (12, 128), (3, 256)])
def test_tree_attention_q8_large_queries_over_small_scales(HQ, D, kind):
    """Few query rows that overflow with the codes alone, where the scale of the key brings the score back.  One key: its weight is
    relative to its own score, and out is its value.  (With many rows scores and maximum are scaled apart: at scores X a weight's
    exponent is off by u X, which is past any bound here, over a 16-bit cache as well.)  The products are whole multiples of one power
    of two and their sum is under 2^24 of them, so the score is rounded with the scale of the scores, with its own product and as
    lse: 4 u, and 4 more for the logarithms' base."""
    code, top = (0x7e, 448.0) if kind == "e4m3" else (0x70, 112.0)
    kv = torch.full((1, 2, 1, 16, D), code, dtype=torch.uint8, device="cuda").view(CODES[kind])
    scales = torch.full((1, 2, 1, 1), 127 - 48, dtype=torch.uint8, device="cuda")
    q = torch.full((1, HQ, D), 1.5 * 2.0 ** 118, device="cuda").bfloat16()
    got = sv.sharpv_tree_attention_q8(q, kv, scales, 16, 0, _i32([5]), _i32([1]), _i32([0, 1]))
    score = D ** -0.5 * D * 1.5 * 2.0 ** 118 * top * 2.0 ** -48
    assert bool((got["out"].double() == top * 2.0 ** -48).all())
    assert float((got["lse"].double() / score - 1).abs().max()) <= 8 * U


@pytest.mark.parametrize("nodes", [2, 50])
def test_tree_attention_q8_shows_what_is_seen(nodes):
    c = Attn("e4m3", 16, 1, 4, 128, [200], [nodes], tree=None, spare=0)
    c.kv.view(torch.uint8)[c.layer, 1, 0, c.begin[0] + 150, 5] = 0xFF       # NaN
    c.dv[0, 0, 9] = -INF
    got = sv.sharpv_tree_attention_q8(*c.args())["out"].float()
    assert bool(torch.isnan(got[:, :, 5]).all()) and bool(torch.isneginf(got[:, :, 9]).all())
    rest = [i for i in range(128) if i not in (5, 9)]
    assert bool(torch.isfinite(got[:, :, rest]).all())


def test_tree_attention_q8_empty_mask_rows_and_tables_outside():
    c = Attn("i8", 16, 2, 4, 64, [0, 60], [40, 4])
    c.tree[3] = 0
    c.tree[37] = 0
    got = c.check()
    assert bool(torch.isneginf(got["lse"][3]).all()) and bool((got["out"][37] == 0).all())
    for nodes in ([3, 1], [30, 40]):
        c = Attn("e4m3", 16, 2, 4, 64, [50, 60], nodes, gap=0)
        good = c.check()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        T = c.kv.shape[3]
        args = c.args()
        got = sv.sharpv_tree_attention_q8(*args[:5], _i32([c.begin[0], T - 10]), _i32([50, 1 << 30]), *args[7:], status_word=status)
        assert status.item() == sv.Status.ERR_BOUNDS
        assert torch.equal(got["out"][:nodes[0]], good["out"][:nodes[0]])
        status.zero_()
        sv.sharpv_tree_attention_q8(*args[:5], _i32([-5, 1 << 30]), _i32([50, -3]), _i32([0, nodes[0], 900]), *args[8:], status_word=status)
        assert status.item() == sv.Status.ERR_BOUNDS


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("nodes", [[1, 1], [20, 33], [200, 30]])
def test_tree_attention_q8_same_bits_again_captured_and_on_a_stream(nodes, kind):
    _needs_capture()
    c = Attn(kind, 32, 2, 7, 128, [3000, 411], nodes, spare=0)
    first = sv.sharpv_tree_attention_q8(*c.args())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = sv.sharpv_tree_attention_q8(*c.args())
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first["out"], again["out"]) and torch.equal(first["lse"], again["lse"])
    ws = torch.full((sv.sharpv_tree_attention_q8_workspace_bytes(2, sum(nodes), 14, 2, 128),), 0xFF, dtype=torch.uint8, device="cuda")
    out = {k: torch.zeros_like(v) for k, v in first.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sv.sharpv_tree_attention_q8(*c.args(), out=out, workspace=ws)
    for _ in range(2):
        out["out"].zero_()
        graph.replay()
        assert torch.equal(first["out"], out["out"])
    c.length[1] = 100                       # the captured call follows the tables' contents
    c.tables[1].copy_(_i32(c.length))
    graph.replay()
    assert torch.equal(out["out"], sv.sharpv_tree_attention_q8(*c.args())["out"])
    o, _, tol, _ = c.reference(c.D ** -0.5)
    assert np.all(np.abs(_f64(out["out"]) - o) <= tol)


# ------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("kind", ["e4m3", "i8"])
def test_a_pruned_prompt_and_decode_steps(kind):
    """A prompt's rows are normed and turned, pruned into an 8-bit cache, and decoded from: tokens attend and are appended, until
    half of the rows are moved to another cache.  Every attention is checked against the values that the cache stands for."""
    g = np.random.default_rng(11)
    L, H, G, D, block, prompt = 2, 2, 4, 128, 32, np.array([150, 260])
    pairs = [int(a) for a in _axes(D // 2, 3, True)]
    new = lambda *s: torch.from_numpy(g.standard_normal(s, dtype=np.float32)).bfloat16().cuda()  # noqa: E731
    wq, wk = new(D), new(D)
    T = int(prompt.sum())
    begin = np.array([0, 256])
    where = np.stack([np.arange(T) // 14, np.arange(T) % 14, np.arange(T) % 7])
    first = torch.zeros((L, 2, H, T, D), dtype=torch.bfloat16, device="cuda")
    for l in range(L):
        qkv = new(T, H * G + 2 * H, D)
        sv.sharpv_qk_norm_rope(qkv[:, :H * G], qkv[:, H * G:H * G + H], _i32(where), pairs, 1e6, norm=True, q_weight=wq, k_weight=wk,
                               out={"q": qkv[:, :H * G], "k": first[l, 0].transpose(0, 1)})
        first[l, 1] = qkv[:, H * G + H:].transpose(0, 1)
    kept = [np.sort(g.permutation(n)[:n * 2 // 3]) + o for n, o in zip(prompt, [0, prompt[0]])]
    offsets = np.concatenate([[0], np.cumsum([len(k) for k in kept])])
    cache = torch.zeros((L, 2, H, 512, D), dtype=CODES[kind], device="cuda")
    scales = torch.zeros((L, 2, H, 512 // block), dtype=torch.uint8, device="cuda")
    sv.sharpv_kv_append_q8(first, cache, scales, block, _i32(np.concatenate(kept)), _i32(offsets), _i32(begin))
    length = np.diff(offsets)
    codes, bytes_ = np.zeros((L, 2, H, 512, D), np.uint8), np.zeros((L, 2, H, 512 // block), np.uint8)
    for plane in np.ndindex(L, 2, H):
        for b in range(2):
            ref.append(_f64(first[plane])[kept[b]], codes[plane], bytes_[plane], kind, block, int(begin[b]))
    for turn in range(4):
        nodes = np.array([[1, 3], [4, 1], [2, 2], [1, 1]][turn])
        N, node_off = int(nodes.sum()), np.concatenate([[0], np.cumsum(nodes)])
        drafts = torch.zeros((L, 2, H, N, D), dtype=torch.bfloat16, device="cuda")
        for l in range(L):
            qkv = new(N, H * G + 2 * H, D)
            dk = drafts[l, 0].transpose(0, 1).contiguous()
            step = sv.sharpv_qk_norm_rope(qkv[:, :H * G], qkv[:, H * G:H * G + H], _i32(np.tile(np.arange(N) + 40, (3, 1))), pairs, 1e6, norm=True,
                                          q_weight=wq, k_weight=wk)
            dk, dv = step["k"], qkv[:, H * G + H:]
            got = sv.sharpv_tree_attention_q8(step["q"], cache, scales, block, l, _i32(begin), _i32(length), _i32(node_off), dk, dv)
            o, lse, tol, ltol = ref.attention(_f64(step["q"]), codes[l, 0], bytes_[l, 0], codes[l, 1], bytes_[l, 1], kind, block, begin, length,
                                              node_off, _f64(dk), _f64(dv), None, D ** -0.5)
            assert np.all(np.abs(_f64(got["out"]) - o) <= tol) and np.all(np.abs(_f64(got["lse"]) - lse) <= ltol), turn
            drafts[l, 0], drafts[l, 1] = dk.transpose(0, 1), dv.transpose(0, 1)
        sv.sharpv_kv_append_q8(drafts, cache, scales, block, _i32(np.arange(N)), _i32(node_off), _i32(begin + length))
        for plane in np.ndindex(L, 2, H):
            for b in range(2):
                ref.append(_f64(drafts[plane])[node_off[b]:node_off[b + 1]], codes[plane], bytes_[plane], kind, block, int(begin[b] + length[b]))
        length = length + nodes
        assert np.array_equal(_bits(cache), codes) and np.array_equal(scales.cpu().numpy(), bytes_)
        if turn == 1:                       # every second row moves to the start of its region of another cache
            stay = [np.arange(b, b + n, 2) for b, n in zip(begin, length)]
            off = np.concatenate([[0], np.cumsum([len(s) for s in stay])])
            fresh, fs = torch.zeros_like(cache), torch.zeros_like(scales)
            sv.sharpv_kv_append_q8(cache, fresh, fs, block, _i32(np.concatenate(stay)), _i32(off), _i32(begin), src_scales=scales)
            c2, b2 = np.zeros_like(codes), np.zeros_like(bytes_)
            for plane in np.ndindex(L, 2, H):
                x = ref.values_of(codes[plane], kind) * 2.0 ** ref.clamped(bytes_[plane])[np.arange(512) // block][:, None]
                for b in range(2):
                    ref.append(x[stay[b]], c2[plane], b2[plane], kind, block, int(begin[b]))
            cache, scales, codes, bytes_, length = fresh, fs, c2, b2, np.diff(off)

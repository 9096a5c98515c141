"""Refusals of the operators round a cache in 8 bits: nothing here needs a GPU, every call returns before any launch."""
import ctypes as C

import numpy as np
import pytest
import torch

import q8_reference as ref
from paper_2511_08003_b200 import binding as sv
from paper_2511_08003_b200 import build as svbuild

P, INF, NAN = 0x10000, float("inf"), float("nan")
S = sv.Status


@pytest.fixture(scope="module")
def L():
    svbuild.build()
    return sv.lib()


def _layout(layers=2, heads=4, d=128, dtype=sv.E4M3, **kw):
    lay = sv.KVLayout(layers, heads, d, dtype, 2 * heads * 100 * d, heads * 100 * d, 100 * d, d)
    for k, v in kw.items():
        setattr(lay, k, v)
    return lay


def _scales(block=16, **kw):
    s = sv.KVScales(block, 2 * 4 * 8, 4 * 8, 8)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


ROPE = dict(q=P, ldq=4608, hsq=128, k=P, ldk=4608, hsk=128, dtype=1, N=9, HQ=28, H=4, D=128, norm=1, qw=P, kw=P, eps=1e-6, pos=P,
            ldp=9, axes=3, pairs=bytes(64), rot=128, base=1e6, oq=P, ldoq=3584, hsoq=128, ok=P, ldok=512, hsok=128)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), S.ERR_INVALID_ARG), (dict(k=None), S.ERR_INVALID_ARG), (dict(oq=None), S.ERR_INVALID_ARG),
    (dict(ok=None), S.ERR_INVALID_ARG), (dict(pos=None), S.ERR_INVALID_ARG), (dict(pairs=None), S.ERR_INVALID_ARG),
    (dict(N=-1), S.ERR_INVALID_ARG), (dict(HQ=0), S.ERR_INVALID_ARG), (dict(H=0), S.ERR_INVALID_ARG), (dict(D=0), S.ERR_INVALID_ARG),
    (dict(rot=-2), S.ERR_INVALID_ARG), (dict(rot=130), S.ERR_INVALID_ARG), (dict(rot=63), S.ERR_INVALID_ARG),
    (dict(norm=2), S.ERR_INVALID_ARG), (dict(norm=0), S.ERR_INVALID_ARG), (dict(eps=-1.0), S.ERR_INVALID_ARG),
    (dict(eps=NAN), S.ERR_INVALID_ARG), (dict(eps=INF), S.ERR_INVALID_ARG), (dict(axes=0), S.ERR_INVALID_ARG),
    (dict(base=0.0), S.ERR_INVALID_ARG), (dict(base=-1.0), S.ERR_INVALID_ARG), (dict(base=NAN), S.ERR_INVALID_ARG),
    (dict(base=INF), S.ERR_INVALID_ARG), (dict(pairs=bytes([3] + [0] * 63)), S.ERR_INVALID_ARG), (dict(ldp=8), S.ERR_INVALID_ARG),
    (dict(rot=0, norm=0, qw=None, kw=None), S.ERR_INVALID_ARG), (dict(hsq=120), S.ERR_INVALID_ARG), (dict(ldok=120), S.ERR_INVALID_ARG),
    (dict(dtype=2), S.ERR_UNSUPPORTED), (dict(dtype=3), S.ERR_UNSUPPORTED), (dict(dtype=9), S.ERR_UNSUPPORTED),
    (dict(D=264, rot=128, hsq=264, hsk=264, hsoq=264, hsok=264), S.ERR_UNSUPPORTED), (dict(D=124, rot=64), S.ERR_UNSUPPORTED),
    (dict(rot=72), S.ERR_UNSUPPORTED), (dict(axes=9), S.ERR_UNSUPPORTED), (dict(HQ=4093), S.ERR_UNSUPPORTED),
    (dict(N=1 << 31), S.ERR_UNSUPPORTED), (dict(q=P + 8), S.ERR_UNSUPPORTED), (dict(ok=P + 2), S.ERR_UNSUPPORTED),
    (dict(qw=P + 8), S.ERR_UNSUPPORTED), (dict(ldq=4604), S.ERR_UNSUPPORTED), (dict(hsok=132), S.ERR_UNSUPPORTED),
    (dict(ldq=1 << 30), S.ERR_UNSUPPORTED), (dict(hsok=1 << 30), S.ERR_UNSUPPORTED), (dict(ldp=-1), S.ERR_INVALID_ARG),
    (dict(N=0), S.OK), (dict(N=0, q=None, pos=None), S.OK),
])
def test_qk_norm_rope_refusals(L, change, status):
    a = dict(ROPE, **change)
    assert L.sharpv_qk_norm_rope(a["q"], a["ldq"], a["hsq"], a["k"], a["ldk"], a["hsk"], a["dtype"], a["N"], a["HQ"], a["H"], a["D"],
                                 a["norm"], a["qw"], a["kw"], a["eps"], a["pos"], a["ldp"], a["axes"], a["pairs"], a["rot"], a["base"],
                                 a["oq"], a["ldoq"], a["hsoq"], a["ok"], a["ldok"], a["hsok"], None) == status


APPEND = dict(src=P, sl=_layout(dtype=sv.BF16), ss=None, ssl=None, st=100, dst=1 << 40, dl=_layout(), ds=1 << 41, dsl=_scales(), dt=100,
              lb=0, le=2, pos=P, off=P, begin=P, B=2, cap=10)
Q8 = dict(sl=_layout(), ss=1 << 42, ssl=_scales())


@pytest.mark.parametrize("change,status", [
    (dict(src=None), S.ERR_INVALID_ARG), (dict(dst=None), S.ERR_INVALID_ARG), (dict(sl=None), S.ERR_INVALID_ARG),
    (dict(dl=None), S.ERR_INVALID_ARG), (dict(ds=None), S.ERR_INVALID_ARG), (dict(dsl=None), S.ERR_INVALID_ARG),
    (dict(pos=None), S.ERR_INVALID_ARG), (dict(off=None), S.ERR_INVALID_ARG), (dict(begin=None), S.ERR_INVALID_ARG),
    (dict(cap=-1), S.ERR_INVALID_ARG), (dict(B=-1), S.ERR_INVALID_ARG), (dict(st=-1), S.ERR_INVALID_ARG), (dict(dt=-1), S.ERR_INVALID_ARG),
    (dict(lb=1, le=0), S.ERR_INVALID_ARG), (dict(le=3), S.ERR_INVALID_ARG), (dict(lb=-1), S.ERR_INVALID_ARG),
    (dict(dl=_layout(heads=2)), S.ERR_INVALID_ARG), (dict(dl=_layout(layers=3)), S.ERR_INVALID_ARG), (dict(dl=_layout(d=64)), S.ERR_INVALID_ARG),
    (dict(ss=P), S.ERR_INVALID_ARG), (dict(ssl=_scales()), S.ERR_INVALID_ARG),             # scales of a cache that has none
    (dict(Q8, ss=None), S.ERR_INVALID_ARG), (dict(Q8, ssl=None), S.ERR_INVALID_ARG),
    (dict(dst=P + 256), S.ERR_INVALID_ARG), (dict(Q8, ss=(1 << 41) + 16), S.ERR_INVALID_ARG),       # overlaps
    (dict(dsl=_scales(stride_head=-1)), S.ERR_INVALID_ARG),
    (dict(dl=_layout(dtype=sv.BF16)), S.ERR_UNSUPPORTED), (dict(dl=_layout(dtype=sv.U8)), S.ERR_UNSUPPORTED),
    (dict(sl=_layout(dtype=sv.U8)), S.ERR_UNSUPPORTED), (dict(sl=_layout(dtype=9)), S.ERR_UNSUPPORTED),
    (dict(dsl=_scales(0)), S.ERR_UNSUPPORTED), (dict(dsl=_scales(24)), S.ERR_UNSUPPORTED), (dict(dsl=_scales(512)), S.ERR_UNSUPPORTED),
    (dict(dsl=_scales(-16)), S.ERR_UNSUPPORTED), (dict(Q8, ssl=_scales(3)), S.ERR_UNSUPPORTED),
    (dict(sl=_layout(dtype=sv.BF16, d=120), dl=_layout(d=120)), S.ERR_UNSUPPORTED),
    (dict(sl=_layout(dtype=sv.BF16, d=1040), dl=_layout(d=1040)), S.ERR_UNSUPPORTED),
    (dict(src=P + 4), S.ERR_UNSUPPORTED), (dict(dst=(1 << 40) + 8), S.ERR_UNSUPPORTED), (dict(dl=_layout(stride_token=136)), S.ERR_UNSUPPORTED),
    (dict(st=1 << 31), S.ERR_UNSUPPORTED), (dict(dt=1 << 31), S.ERR_UNSUPPORTED), (dict(cap=1 << 31), S.ERR_UNSUPPORTED),
    (dict(cap=0), S.OK), (dict(B=0), S.OK), (dict(lb=1, le=1), S.OK), (dict(Q8, B=0), S.OK),
])
def test_kv_append_q8_refusals(L, change, status):
    a = dict(APPEND, **change)
    assert L.sharpv_kv_append_q8(a["src"], a["sl"], a["ss"], a["ssl"], a["st"], a["dst"], a["dl"], a["ds"], a["dsl"], a["dt"], a["lb"],
                                 a["le"], a["pos"], a["off"], a["begin"], a["B"], a["cap"], None, None) == status


ATTN = dict(q=P, ldq=28 * 128, dk=P, ldk=512, dv=P, ldv=512, hq=28, kv=P, lay=_layout(), sc=P, scl=_scales(), layer=0, tokens=100, B=2,
            begin=P, len=P, off=P, N=5, mask=None, words=0, scale=0.1, out=P, lse=P, ws=P, wsb=1 << 40)


@pytest.mark.parametrize("change,status", [
    (dict(kv=None), S.ERR_INVALID_ARG), (dict(lay=None), S.ERR_INVALID_ARG), (dict(q=None), S.ERR_INVALID_ARG),
    (dict(sc=None), S.ERR_INVALID_ARG), (dict(scl=None), S.ERR_INVALID_ARG), (dict(begin=None), S.ERR_INVALID_ARG),
    (dict(len=None), S.ERR_INVALID_ARG), (dict(off=None), S.ERR_INVALID_ARG), (dict(out=None), S.ERR_INVALID_ARG),
    (dict(lse=None), S.ERR_INVALID_ARG), (dict(ws=None), S.ERR_INVALID_ARG), (dict(layer=-1), S.ERR_INVALID_ARG),
    (dict(layer=2), S.ERR_INVALID_ARG), (dict(hq=0), S.ERR_INVALID_ARG), (dict(hq=27), S.ERR_INVALID_ARG),
    (dict(ldq=28 * 128 - 8), S.ERR_INVALID_ARG), (dict(B=-1), S.ERR_INVALID_ARG), (dict(N=-1), S.ERR_INVALID_ARG),
    (dict(tokens=-1), S.ERR_INVALID_ARG), (dict(scale=0.0), S.ERR_INVALID_ARG), (dict(scale=INF), S.ERR_INVALID_ARG),
    (dict(scale=NAN), S.ERR_INVALID_ARG), (dict(dk=None), S.ERR_INVALID_ARG), (dict(ldk=504), S.ERR_INVALID_ARG),
    (dict(mask=P, words=0), S.ERR_INVALID_ARG), (dict(scl=_scales(stride_kv=-8)), S.ERR_INVALID_ARG),
    (dict(lay=_layout(dtype=sv.BF16)), S.ERR_UNSUPPORTED), (dict(lay=_layout(dtype=sv.U8)), S.ERR_UNSUPPORTED),
    (dict(scl=_scales(0)), S.ERR_UNSUPPORTED), (dict(scl=_scales(48)), S.ERR_UNSUPPORTED), (dict(scl=_scales(512)), S.ERR_UNSUPPORTED),
    (dict(lay=_layout(d=272), ldq=28 * 272, ldk=1088, ldv=1088), S.ERR_UNSUPPORTED), (dict(lay=_layout(d=120)), S.ERR_UNSUPPORTED),
    (dict(lay=_layout(stride_head=12808)), S.ERR_UNSUPPORTED), (dict(kv=P + 8), S.ERR_UNSUPPORTED), (dict(q=P + 8), S.ERR_UNSUPPORTED),
    (dict(ldq=28 * 128 + 4), S.ERR_UNSUPPORTED), (dict(ldv=516), S.ERR_UNSUPPORTED), (dict(ws=P + 16), S.ERR_UNSUPPORTED),
    (dict(tokens=1 << 31), S.ERR_UNSUPPORTED), (dict(N=1 << 30), S.ERR_UNSUPPORTED), (dict(wsb=64), S.ERR_WORKSPACE),
    (dict(B=0), S.OK), (dict(N=0), S.OK),
])
def test_tree_attention_q8_refusals(L, change, status):
    a = dict(ATTN, **change)
    assert L.sharpv_tree_attention_q8(a["q"], a["ldq"], a["dk"], a["ldk"], a["dv"], a["ldv"], a["hq"], a["kv"], a["lay"], a["sc"], a["scl"],
                                      a["layer"], a["tokens"], a["B"], a["begin"], a["len"], a["off"], a["N"], a["mask"], a["words"],
                                      a["scale"], a["out"], a["lse"], a["ws"], a["wsb"], None, None) == status


def test_the_others_refuse_codes_with_scales(L):
    """sharpv_tree_attention, the weights and the rotation do not read codes without their scales."""
    for dtype in (sv.E4M3, sv.I8):
        lay = _layout(dtype=dtype)
        assert L.sharpv_tree_attention(P, 3584, None, 0, None, 0, 28, P, lay, 0, 100, 2, P, P, P, 5, None, 0, 0.1, P, P, P, 1 << 40, None,
                                       None) == S.ERR_UNSUPPORTED
        assert L.sharpv_attention_mass(P, 3584, P, None, 28, P, lay, 0, 100, 2, P, P, P, 5, 0.1, 1.0, None, P, P, 1 << 40, None,
                                       None) == S.ERR_UNSUPPORTED


def test_workspace_query(L):
    a = L.sharpv_tree_attention_q8_workspace_bytes(1, 1, 14, 2, 64)
    assert 0 < a <= L.sharpv_tree_attention_q8_workspace_bytes(1, 1, 14, 2, 128) <= L.sharpv_tree_attention_q8_workspace_bytes(1, 500, 14, 2, 128)
    assert a % 256 == 0


def test_wrappers_refuse_what_is_not_on_the_gpu():
    kv = torch.zeros((1, 2, 2, 32, 64), dtype=torch.int8)
    sc = torch.zeros((1, 2, 2, 2), dtype=torch.uint8)
    i, off = torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    x = torch.zeros((1, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        sv.sharpv_tree_attention_q8(x, kv, sc, 16, 0, i, i, off)
    with pytest.raises(ValueError):
        sv.sharpv_kv_append_q8(kv.float(), kv, sc, 16, i, off, i)
    with pytest.raises(ValueError):
        sv.sharpv_qk_norm_rope(x, x, i[None], [0] * 32, 1e4)


def test_the_reference_rounds_to_codes_as_torch_does():
    """e4m3 by its definition against torch's cast (which does not saturate) over every half-way point and random values."""
    v = np.sort(ref.e4m3_values()[:127])
    x = np.concatenate([v, (v[1:] + v[:-1]) / 2, np.nextafter((v[1:] + v[:-1]) / 2, 0), np.random.default_rng(0).uniform(0, 448, 20000)])
    x = np.concatenate([x, -x]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.nearest(x.astype(np.float64), "e4m3"), want)
    assert np.array_equal(ref.values_of(want, "e4m3"), torch.from_numpy(want).view(torch.float8_e4m3fn).double().numpy())
    for kind in ("e4m3", "i8"):
        for e in range(-20, 20):
            top = ref.TOP[kind] * 2.0 ** e
            assert ref.exponent(top, kind) == e and ref.exponent(np.nextafter(top, np.inf), kind) == e + 1

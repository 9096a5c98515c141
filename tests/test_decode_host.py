"""Refusals of the operators that decode over a cache: nothing here needs a GPU, every call returns before any launch."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2511_08003_b200 import binding as sv
from paper_2511_08003_b200 import build as svbuild

P, INF = 0x10000, float("inf")
S = sv.Status


@pytest.fixture(scope="module")
def L():
    svbuild.build()
    return sv.lib()


def _layout(layers=2, heads=4, d=128, dtype=1, **kw):
    lay = sv.KVLayout(layers, heads, d, dtype, 2 * heads * 100 * d, heads * 100 * d, 100 * d, d)
    for k, v in kw.items():
        setattr(lay, k, v)
    return lay


ATTN = dict(q=P, ldq=28 * 128, dk=P, ldk=512, dv=P, ldv=512, hq=28, kv=P, lay=_layout(), layer=0, tokens=100, B=2,
            begin=P, len=P, off=P, N=5, mask=None, words=0, scale=0.1, out=P, lse=P, ws=P, wsb=1 << 40, st=None, stream=None)
MASS = dict(q=P, ldq=28 * 128, lse=P, w=None, hq=28, kv=P, lay=_layout(), layer=0, tokens=100, B=2, begin=P, len=P, off=P,
            N=5, scale=0.1, decay=1.0, mass=None, out=P, ws=P, wsb=1 << 40, st=None, stream=None)
COMMON = [
    (dict(kv=None), S.ERR_INVALID_ARG), (dict(lay=None), S.ERR_INVALID_ARG), (dict(q=None), S.ERR_INVALID_ARG),
    (dict(begin=None), S.ERR_INVALID_ARG), (dict(len=None), S.ERR_INVALID_ARG), (dict(off=None), S.ERR_INVALID_ARG),
    (dict(out=None), S.ERR_INVALID_ARG), (dict(lse=None), S.ERR_INVALID_ARG), (dict(ws=None), S.ERR_INVALID_ARG),
    (dict(layer=-1), S.ERR_INVALID_ARG), (dict(layer=2), S.ERR_INVALID_ARG), (dict(hq=0), S.ERR_INVALID_ARG),
    (dict(hq=27), S.ERR_INVALID_ARG), (dict(ldq=28 * 128 - 8), S.ERR_INVALID_ARG), (dict(B=-1), S.ERR_INVALID_ARG),
    (dict(N=-1), S.ERR_INVALID_ARG), (dict(tokens=-1), S.ERR_INVALID_ARG), (dict(scale=0.0), S.ERR_INVALID_ARG),
    (dict(scale=-1.0), S.ERR_INVALID_ARG), (dict(scale=INF), S.ERR_INVALID_ARG), (dict(scale=float("nan")), S.ERR_INVALID_ARG),
    (dict(lay=_layout(stride_token=120)), S.ERR_INVALID_ARG), (dict(lay=_layout(layers=0)), S.ERR_INVALID_ARG),
    (dict(lay=_layout(dtype=2)), S.ERR_UNSUPPORTED), (dict(lay=_layout(dtype=9)), S.ERR_UNSUPPORTED),
    (dict(lay=_layout(d=264, heads=4), ldq=28 * 264, ldk=1056, ldv=1056), S.ERR_UNSUPPORTED),
    (dict(lay=_layout(d=100), ldq=28 * 100), S.ERR_UNSUPPORTED), (dict(lay=_layout(stride_head=12801)), S.ERR_UNSUPPORTED),
    (dict(kv=P + 2), S.ERR_UNSUPPORTED), (dict(q=P + 8), S.ERR_UNSUPPORTED), (dict(ldq=28 * 128 + 4), S.ERR_UNSUPPORTED),
    (dict(ws=P + 16), S.ERR_UNSUPPORTED), (dict(tokens=1 << 31), S.ERR_UNSUPPORTED), (dict(N=1 << 30), S.ERR_UNSUPPORTED),
    (dict(wsb=64), S.ERR_WORKSPACE), (dict(B=0), S.OK),
]


def _attn(L, **kw):
    a = dict(ATTN, **kw)
    return L.sharpv_tree_attention(a["q"], a["ldq"], a["dk"], a["ldk"], a["dv"], a["ldv"], a["hq"], a["kv"], a["lay"],
                                   a["layer"], a["tokens"], a["B"], a["begin"], a["len"], a["off"], a["N"], a["mask"],
                                   a["words"], a["scale"], a["out"], a["lse"], a["ws"], a["wsb"], a["st"], a["stream"])


def _mass(L, **kw):
    a = dict(MASS, **kw)
    return L.sharpv_attention_mass(a["q"], a["ldq"], a["lse"], a["w"], a["hq"], a["kv"], a["lay"], a["layer"], a["tokens"],
                                   a["B"], a["begin"], a["len"], a["off"], a["N"], a["scale"], a["decay"], a["mass"],
                                   a["out"], a["ws"], a["wsb"], a["st"], a["stream"])


@pytest.mark.parametrize("change,status", COMMON + [
    (dict(dk=None), S.ERR_INVALID_ARG), (dict(dv=None), S.ERR_INVALID_ARG), (dict(ldk=504), S.ERR_INVALID_ARG),
    (dict(mask=P, words=0), S.ERR_INVALID_ARG), (dict(words=-1), S.ERR_INVALID_ARG), (dict(dk=P + 2), S.ERR_UNSUPPORTED),
    (dict(ldv=516), S.ERR_UNSUPPORTED), (dict(out=P + 4), S.ERR_UNSUPPORTED), (dict(N=0), S.OK),
])
def test_tree_attention_refusals(L, change, status):
    assert _attn(L, **change) == status


@pytest.mark.parametrize("change,status", [c for c in COMMON if "ws" not in c[0] and "wsb" not in c[0]] + [
    (dict(lay=_layout(dtype=0, d=64), ldq=28 * 64, ws=None), S.ERR_INVALID_ARG),
    (dict(lay=_layout(dtype=0, d=64), ldq=28 * 64, ws=P + 16), S.ERR_UNSUPPORTED),
    (dict(lay=_layout(dtype=0, d=64), ldq=28 * 64, wsb=64), S.ERR_WORKSPACE),
    (dict(decay=-0.5), S.ERR_INVALID_ARG), (dict(decay=float("nan")), S.ERR_INVALID_ARG), (dict(decay=INF), S.ERR_INVALID_ARG),
    (dict(mass=P + 256), S.ERR_INVALID_ARG), (dict(tokens=0), S.OK),
])
def test_attention_mass_refusals(L, change, status):
    assert _mass(L, **change) == status


def test_workspace_queries(L):
    a = L.sharpv_tree_attention_workspace_bytes(1, 1, 14, 2, 64, 1)
    assert 0 < a <= L.sharpv_tree_attention_workspace_bytes(1, 1, 14, 2, 128, 1) <= L.sharpv_tree_attention_workspace_bytes(1, 500, 14, 2, 128, 1)
    assert a % 256 == 0
    assert L.sharpv_attention_mass_workspace_bytes(1000, 4, 0) >= 16000 and L.sharpv_attention_mass_workspace_bytes(1000, 4, 1) == 0


@pytest.mark.parametrize("change,status", [
    (dict(mass=None), S.ERR_INVALID_ARG), (dict(tokens=-1), S.ERR_INVALID_ARG), (dict(B=-1), S.ERR_INVALID_ARG),
    (dict(begin=None), S.ERR_INVALID_ARG), (dict(len=None), S.ERR_INVALID_ARG), (dict(budget=None), S.ERR_INVALID_ARG),
    (dict(sink=-1), S.ERR_INVALID_ARG), (dict(recent=-1), S.ERR_INVALID_ARG), (dict(pos=None), S.ERR_INVALID_ARG),
    (dict(off=None), S.ERR_INVALID_ARG), (dict(cap=-1), S.ERR_INVALID_ARG), (dict(out=P), S.ERR_INVALID_ARG),
    (dict(out=P + 396), S.ERR_INVALID_ARG), (dict(tokens=1 << 31), S.ERR_UNSUPPORTED), (dict(B=1 << 30), S.ERR_UNSUPPORTED),
])
def test_evict_select_refusals(L, change, status):
    a = dict(mass=P, tokens=100, B=2, begin=P, len=P, budget=P, sink=1, recent=2, pos=P, off=P, out=None, cap=50)
    a.update(change)
    assert L.sharpv_evict_select(a["mass"], a["tokens"], a["B"], a["begin"], a["len"], a["budget"], a["sink"], a["recent"],
                                 a["pos"], a["off"], a["out"], a["cap"], None, None) == status


@pytest.mark.parametrize("change,status", [
    (dict(src=None), S.ERR_INVALID_ARG), (dict(dst=None), S.ERR_INVALID_ARG), (dict(pos=None), S.ERR_INVALID_ARG),
    (dict(off=None), S.ERR_INVALID_ARG), (dict(begin=None), S.ERR_INVALID_ARG), (dict(cap=-1), S.ERR_INVALID_ARG),
    (dict(lb=1, le=0), S.ERR_INVALID_ARG), (dict(le=3), S.ERR_INVALID_ARG), (dict(B=-1), S.ERR_INVALID_ARG),
    (dict(dl=_layout(heads=2)), S.ERR_INVALID_ARG), (dict(dl=_layout(dtype=0)), S.ERR_INVALID_ARG),
    (dict(dst=P + 256), S.ERR_INVALID_ARG),                     # overlaps the source
    (dict(src=P + 4), S.ERR_UNSUPPORTED), (dict(sl=_layout(stride_token=129)), S.ERR_UNSUPPORTED),
    (dict(sl=_layout(dtype=5)), S.ERR_UNSUPPORTED), (dict(st=1 << 31), S.ERR_UNSUPPORTED),
    (dict(cap=0), S.OK), (dict(B=0), S.OK), (dict(lb=1, le=1), S.OK),
])
def test_kv_append_refusals(L, change, status):
    a = dict(src=P, sl=_layout(), st=100, dst=1 << 40, dl=_layout(), dt=100, lb=0, le=2, pos=P, off=P, begin=P, B=2, cap=10)
    a.update(change)
    assert L.sharpv_kv_append(a["src"], a["sl"], a["st"], a["dst"], a["dl"], a["dt"], a["lb"], a["le"], a["pos"], a["off"],
                              a["begin"], a["B"], a["cap"], None, None) == status


def test_wrappers_refuse_what_is_not_on_the_gpu():
    kv = torch.zeros((1, 2, 2, 8, 64))
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        sv.sharpv_tree_attention(torch.zeros((1, 2, 64)), kv, 0, i, i, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        sv.sharpv_attention_mass(torch.zeros((1, 2, 64)), torch.zeros((1, 2)), kv, 0, i, i, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        sv.sharpv_evict_select(torch.zeros(8), i, i, i)
    with pytest.raises(ValueError):
        sv.sharpv_kv_append(kv, kv.clone(), i, torch.zeros(2, dtype=torch.int32), i)


def test_workspace_sizes_that_are_kept_stay_few(L):
    sizes = {n: sv.sharpv_tree_attention_workspace_bytes(3, n, 28, 4, 128) for n in range(1, 3000)}
    assert sv.sharpv_tree_attention_workspace_bytes.cache_info().currsize <= 1000
    assert all(L.sharpv_tree_attention_workspace_bytes(3, n, 28, 4, 128, 1) == b for n, b in sizes.items())


def test_query_arrays_without_nodes_have_no_strides_that_matter():
    cpu, f32 = torch.device("cpu"), torch.float32
    for t in (torch.empty((5, 24, 64))[:0, 3:11], torch.from_numpy(np.zeros((0, 8, 64), np.float32)),    # strides of 0
              torch.empty((4, 64, 8)).transpose(1, 2)[:0]):
        assert sv._heads(t, "q", cpu, f32, None, None, 64) == 8 * 64
    with pytest.raises(ValueError):
        sv._heads(torch.empty((0, 8, 32)), "q", cpu, f32, None, None, 64)
    with pytest.raises(ValueError):
        sv._heads(torch.empty((8, 5, 64)).transpose(0, 1), "q", cpu, f32, None, None, 64)

"""What the operators round a cache in 8 bits take and refuse at the ends of their ranges: nothing here needs a GPU."""
import ctypes as C
import subprocess

import numpy as np
import pytest
import torch

from paper_2511_08003_b200 import binding as sv
from paper_2511_08003_b200 import build as svbuild


def test_one_token_in_a_plane_with_heads_far_apart():
    """A single token needs no token stride: none may come of a head stride that would be refused as one (2 GB)."""
    cache = torch.empty((8, 1 << 20, 128), dtype=torch.bfloat16, device="meta")
    for n in (1, 2, 9):
        address, token, head = sv._token_rows(cache[:, 7:7 + n].transpose(0, 1), n, 8, 128)
        assert (token, head) == (128, 128 << 20)
    assert sv._token_rows(cache[:1, 7:8].transpose(0, 1), 1, 1, 128)[1:] == (128, 128)
    assert sv._token_rows(cache[:, 7:8], 8, 1, 128)[1:] == (128 << 20, 128)


SHIM = r"""
#include "overlap.h"
#include <cstring>
using namespace sharpv;
static Runs runs(uintptr_t base, int64_t bytes, int dims, const int64_t* s, const int64_t* n) {
    Runs r = {base, bytes, dims, {}, {}};
    for (int k = 0; k < dims; ++k) { r.stride[k] = s[k]; r.count[k] = n[k]; }
    return r;
}
extern "C" int share(uintptr_t a, int64_t al, int ad, const int64_t* as, const int64_t* an, uintptr_t b, int64_t bl, int bd, const int64_t* bs,
                     const int64_t* bn) { return (int)share_bytes(runs(a, al, ad, as, an), runs(b, bl, bd, bs, bn)); }
extern "C" int own(uintptr_t a, int64_t al, int ad, const int64_t* as, const int64_t* an) { return (int)shares_own_bytes(runs(a, al, ad, as, an)); }
"""


@pytest.fixture(scope="module")
def overlap(tmp_path_factory):
    at = tmp_path_factory.mktemp("overlap")
    (at / "shim.cpp").write_text(SHIM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", svbuild.CSRC, "-o", str(at / "shim.so"), str(at / "shim.cpp")])
    L = C.CDLL(str(at / "shim.so"))
    words = lambda v: (C.c_int64 * max(len(v), 1))(*v)  # noqa: E731
    runs = lambda r: (C.c_size_t(r[0]), C.c_int64(r[1]), len(r[2]), words(r[2]), words(r[3]))  # noqa: E731
    return (lambda a, b: L.share(*runs(a), *runs(b))), (lambda a: L.own(*runs(a)))


def _bytes_of(r):
    base, length, strides, counts = r
    at = base + np.arange(length)[None]
    for s, n in zip(strides, counts):
        at = (at[:, None] + (np.arange(n) * s)[None, :, None]).reshape(-1, length)
    return at


def test_arrays_with_strides_that_share_bytes(overlap):
    """Against every byte of small arrays: 0 apart, 1 sharing."""
    share, own = overlap
    g = np.random.default_rng(0)

    def some():
        d = int(g.integers(0, 4))
        strides = g.choice([0, 1, 3, 4, 8, 12, 16, 24, 40, 64], d)
        return 1000 + int(g.integers(0, 60)), int(g.integers(1, 6)), [int(x) for x in strides], [int(x) for x in g.integers(1, 5, d)]

    seen = [0, 0, 0, 0]
    for _ in range(20000):
        a, b = some(), some()
        x, y = _bytes_of(a), _bytes_of(b)
        want = bool(np.intersect1d(x, y).size)
        assert share(a, b) == want, (a, b)
        alone = np.unique(x).size == x.size
        assert own(a) == (not alone), a
        seen[want] += 1
        seen[2 + alone] += 1
    assert min(seen) > 2000


def test_layouts_that_interleave(overlap):
    share, own = overlap
    D, HQ, H, N = 256, 28, 4, 50432
    fused = (HQ + 2 * H) * D
    q, k, v = ((4096 + o * D, D, [fused, D], [N, n]) for o, n in ((0, HQ), (HQ, H), (HQ + H, H)))
    for a, b in ((q, k), (q, v), (k, v)):
        assert share(a, b) == share(b, a) == 0
    assert own(q) == own(k) == 0 and share(q, q) == 1
    assert share(q, (4096 + (HQ - 1) * D, D, [fused, D], [N, 2])) == 1              # a head of q taken for k's
    assert share(q, (4096 + (HQ + 2) * D + fused * (N - 1), D, [fused, D], [1, H])) == 0
    plane = (4096, D, [D, D << 20], [N, H])                                         # a plane of a long cache
    assert own(plane) == 0 and share(plane, (4096 + N * D, D, [D, D << 20], [1 << 19, H])) == 0
    assert share(plane, (4096 + (N - 1) * D, D, [D, D << 20], [9, H])) == 1
    assert own((4096, D, [0, D], [2, 4])) == 1 and own((4096, D, [D, D], [2, 2])) == 1
    # codes and scales layer by layer in one allocation
    layer = 2 * 4 * 1000 * 128 + 2 * 4 * 16
    codes, scales = (0, 128, [layer, 4 * 128000, 128000, 128], [28, 2, 4, 1000]), (2 * 4 * 128000, 16, [layer, 64, 16], [28, 2, 4])
    assert share(codes, scales) == 0 and own(codes) == own(scales) == 0
    assert share(codes, (2 * 4 * 128000 - 1, 16, [layer, 64, 16], [28, 2, 4])) == 1
    assert own((0, 16, [layer, 64, 0], [28, 2, 4])) == 1 and own((0, 17, [layer, 64, 16], [28, 2, 4])) == 1


ROPE = dict(q=1 << 20, ldq=36 * 128, hsq=128, k=(1 << 20) + 28 * 256, ldk=36 * 128, hsk=128, N=9, qw=1 << 30, kw=1 << 30, pos=1 << 31, axes=3,
            oq=1 << 32, ldoq=28 * 128, hsoq=128, ok=1 << 33, ldok=4 * 128, hsok=128)


@pytest.mark.parametrize("change", [
    dict(oq=(1 << 20) + 256), dict(oq=1 << 20), dict(oq=(1 << 20) + 256 * 30, ldoq=36 * 128),      # q's rows elsewhere than they were
    dict(ok=1 << 20, ldok=36 * 128), dict(oq=1 << 20, ldoq=36 * 128, ok=1 << 20, ldok=36 * 128),   # k's rows over q's first heads
    dict(ok=(1 << 32) + 256 * 28 * 9 - 256), dict(ldoq=128), dict(hsok=512), dict(oq=(1 << 30) - 256), dict(ok=(1 << 31) + 16),
    dict(oq=1 << 20, ldoq=36 * 128, hsoq=256),
])
def test_norm_and_rotation_refuse_outputs_that_overlap(change):
    svbuild.build()
    a = dict(ROPE, **change)
    assert sv.lib().sharpv_qk_norm_rope(
        a["q"], a["ldq"], a["hsq"], a["k"], a["ldk"], a["hsk"], 1, a["N"], 28, 4, 128, 1, a["qw"], a["kw"], 1e-6, a["pos"], a["N"], a["axes"], bytes(64),
        128, 1e6, a["oq"], a["ldoq"], a["hsoq"], a["ok"], a["ldok"], a["hsok"], None) == sv.Status.ERR_INVALID_ARG


def _layout(dtype, **kw):
    lay = sv.KVLayout(2, 4, 128, dtype, 2 * 4 * 100 * 128, 4 * 100 * 128, 100 * 128, 128)
    for k, v in kw.items():
        setattr(lay, k, v)
    return lay


def _scales(**kw):
    s = sv.KVScales(16, 2 * 4 * 8, 4 * 8, 8)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


DST = 1 << 40


@pytest.mark.parametrize("change", [
    dict(dsl=_scales(stride_head=0)), dict(dsl=_scales(stride_kv=0)), dict(dsl=_scales(stride_layer=0)),       # planes with one scale
    dict(dsl=_scales(stride_head=6)),                                                                          # 7 blocks of 100 rows
    dict(dl=_layout(sv.E4M3, stride_head=0)), dict(dl=_layout(sv.E4M3, stride_layer=99 * 128)),                # planes with one another's rows
    dict(ds=DST), dict(ds=DST + 2 * 2 * 4 * 100 * 128 - 1), dict(ds=DST - 1), dict(ds=1 << 20), dict(ds=(1 << 20) - 1),    # scales over rows
    dict(sl=_layout(sv.I8), ss=DST + 128, ssl=_scales()),
])
def test_append_refuses_destinations_that_overlap(change):
    svbuild.build()
    a = dict(dict(sl=_layout(sv.BF16), ss=None, ssl=None, dl=_layout(sv.E4M3), ds=1 << 41, dsl=_scales()), **change)
    assert sv.lib().sharpv_kv_append_q8(1 << 20, a["sl"], a["ss"], a["ssl"], 100, DST, a["dl"], a["ds"], a["dsl"], 100, 0, 2, 1 << 16, 1 << 16, 1 << 16,
                                        2, 10, None, None) == sv.Status.ERR_INVALID_ARG

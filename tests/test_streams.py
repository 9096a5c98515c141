"""Calls on a stream that is not the current one: whose memory they take."""
import pytest
import torch

from helpers import DeviceWorkload
from paper_2511_08003_b200 import binding as sv
from paper_2511_08003_b200 import workloads

ENTRY_POINTS = ["score_frames", "select_tokens", "select_tokens_threshold", "prune_frames", "kv_calibrate_prune",
                "kv_calibrate_prune_noalloc", "kv_prune_layers", "kv_compact_rope", "tree_attention", "tree_attention_f32",
                "attention_mass", "attention_mass_f32", "evict_select"]


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _calls(name):
    """The entry point as a function of the stream, its inputs made on the current stream."""
    if name in ("score_frames", "select_tokens", "select_tokens_threshold", "prune_frames", "kv_calibrate_prune",
                "kv_calibrate_prune_noalloc", "kv_prune_layers"):
        wl = workloads.custom("streams", 7, workloads.F32, 6, 64, 3, [workloads.make_video_spec(7, 0.6, cuts=[5])], 0.0, 2, 3, 8)
        workloads.fill_tokens(wl)
        workloads.fill_hidden(wl)
        d = DeviceWorkload(wl)
        if name in ("score_frames", "prune_frames"):
            fn = getattr(sv, "sharpv_" + name)
            return lambda s: fn(d.tokens, d.video_frame_offsets, wl.total_frames, wl.f, stream=s)
        if name == "select_tokens":
            a = sv.sharpv_score_frames(d.tokens, d.video_frame_offsets, wl.total_frames, wl.f)
            return lambda s: sv.sharpv_select_tokens(a["importance"], a["k"], wl.total_frames, wl.f, d.tokens, stream=s)
        if name == "select_tokens_threshold":
            a = sv.sharpv_score_frames(d.tokens, d.video_frame_offsets, wl.total_frames, wl.f)
            return lambda s: sv.sharpv_select_tokens_threshold(a["importance"], 0.5, wl.total_frames, wl.f, d.tokens, stream=s)
        tables = (d.seq_offsets, d.vis_begin, d.vis_count, d.vis_offsets, int(wl.seq_offsets[-1]))
        if name == "kv_prune_layers":
            layers = torch.stack([d.hidden, d.hidden])
            return lambda s: sv.sharpv_kv_prune_layers(layers, d.tokens, *tables, None, None, want_mean_cos=True, stream=s)
        fn = getattr(sv, "sharpv_" + name)
        return lambda s: fn(d.hidden, d.tokens, *tables, want_mean_cos=True, stream=s)
    dt = torch.float32 if name.endswith("f32") else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(1)
    kv = torch.randn((1, 2, 2, 900, 64), device="cuda", generator=g).to(dt)
    if name == "kv_compact_rope":
        dst = torch.zeros_like(kv)
        pos = torch.arange(0, 900, 3, dtype=torch.int32, device="cuda")
        off, seq = _i32([0, 300]), _i32([0, 900])
        return lambda s: {"kv": sv.sharpv_kv_compact_rope(kv, dst, pos, off, seq, 300, 64, 10000.0, stream=s)}
    q = torch.randn((30, 6, 64), device="cuda", generator=g).to(dt)
    tables = (_i32([0, 500]), _i32([500, 380]), _i32([0, 10, 30]))
    if name.startswith("tree"):
        return lambda s: sv.sharpv_tree_attention(q, kv, 0, *tables, stream=s)
    lse = sv.sharpv_tree_attention(q, kv, 0, *tables)["lse"]
    if name.startswith("attention_mass"):
        return lambda s: {"mass": sv.sharpv_attention_mass(q, lse, kv, 0, *tables, stream=s)}
    mass = torch.rand(900, device="cuda", generator=g)
    budget = _i32([100, 70])
    return lambda s: sv.sharpv_evict_select(mass, tables[0], tables[1], budget, 2, 5, 170, stream=s)


def _pool(t):
    """The stream whose pool a tensor's memory comes from."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not the allocator's memory")


@pytest.mark.gpu
@pytest.mark.parametrize("name", ENTRY_POINTS)
def test_memory_comes_from_the_pool_of_the_stream_of_the_call(name, monkeypatch):
    """A block of the current stream's pool may still be written by what was queued there before it was freed, and nothing
    orders that before a call on another stream."""
    call = _calls(name)
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
        if key != "kv":                     # the caller's own
            assert _pool(t) == side.cuda_stream, key
    for ws in scratch:
        assert _pool(ws) == side.cuda_stream
    if name in ("tree_attention", "tree_attention_f32", "attention_mass", "attention_mass_f32", "evict_select", "kv_compact_rope"):
        for key, t in got.items():
            assert torch.equal(t, want[key]), key


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["prune_frames", "tree_attention", "attention_mass", "evict_select"])
def test_results_are_kept_for_what_the_current_stream_still_does_with_them(name):
    """A result that is freed while work on it is queued on the current stream is not handed out again on its own stream."""
    call = _calls(name)
    call(None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = call(side)
    torch.cuda.current_stream().wait_stream(side)
    at = {t.data_ptr(): (t.numel() * t.element_size()) for t in got.values()}
    torch.cuda._sleep(1 << 28)              # about 0.15 s
    read = [t.clone() for t in got.values()]
    del got
    with torch.cuda.stream(side):
        new = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in at.values() for _ in range(2)]
        busy = not torch.cuda.default_stream().query()
    assert busy and not any(x.data_ptr() in at for x in new)
    torch.cuda.synchronize()
    del read

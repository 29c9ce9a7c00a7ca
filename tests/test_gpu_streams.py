"""GPU: whatever a call with stream= allocates, workspace and outputs, comes from that stream's part of torch's allocator: blocks of the current
stream may still be in use there.  And what it returns is what the call on the current stream returns."""
import pytest
import torch

from paper_2512_09010_amd import binding as lv

pytestmark = pytest.mark.gpu


def calls():
    gen = torch.Generator(device="cuda").manual_seed(60)
    x4 = torch.randn((2, 24, 24, 64), generator=gen, device="cuda")
    key = torch.randn((2, 24, 24, 16), generator=gen, device="cuda")
    x3 = torch.randn((2, 576, 64), generator=gen, device="cuda")
    flat = torch.randn((576 + 300, 64), generator=gen, device="cuda")
    ones, scores = torch.ones((2, 576), dtype=torch.int32, device="cuda"), torch.rand((2, 576), generator=gen, device="cuda")
    half = [(1, 12), (0, 12)]
    return [x4, key, x3, flat, ones, scores], dict(
        oim_merge=lambda st: lv.luvc_oim_merge(x4, half, stream=st),
        oim_merge_wide=lambda st: lv.luvc_oim_merge_wide(x4, [(1, 2), (0, 2)], 0, stream=st),
        oim_merge_keyed=lambda st: lv.luvc_oim_merge_keyed(x4, key, half, stream=st),
        value_enhance=lambda st: lv.luvc_value_enhance(x3, ones, stream=st),
        spu_score=lambda st: lv.luvc_spu_score(x3, 40, stream=st),
        spu_score_static=lambda st: lv.luvc_spu_score_static(x3, 40, stream=st),
        spu_prune=lambda st: lv.luvc_spu_prune(x3, scores, 57, stream=st),
        spu_stage=lambda st: lv.luvc_spu_stage(x3, 40, 57, stream=st),
        spu_stage_of_nothing=lambda st: lv.luvc_spu_stage(x3, 40, 0, stream=st),
        oim_merge_ragged=lambda st: lv.luvc_oim_merge_ragged(flat, [(24, 24), (15, 20)], [half, [(1, 10)]], stream=st),
        spu_stage_ragged=lambda st: lv.luvc_spu_stage_ragged(flat, [576, 300], [40, 20], [57, 30], stream=st))


@pytest.mark.parametrize("name", ["oim_merge", "oim_merge_wide", "oim_merge_keyed", "value_enhance", "spu_score", "spu_score_static", "spu_prune",
                                  "spu_stage", "spu_stage_of_nothing", "oim_merge_ragged", "spu_stage_ragged"])
def test_buffers_of_a_call_on_another_stream_are_that_streams(name, monkeypatch):
    inputs, table = calls()
    run, nat, passed = table[name], lv._native(), []
    want = run(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    call = nat.call
    monkeypatch.setattr(nat, "call", lambda entry, *args: (passed.append(args), call(entry, *args))[1])
    got = run(side)
    torch.cuda.synchronize()
    segments = torch.cuda.memory_snapshot()
    given = {t.data_ptr() for t in inputs}
    of = lambda p: [s["stream"] for s in segments if s["address"] <= p < s["address"] + s["total_size"]]
    made = [s for args in passed for p in args if isinstance(p, int) and p not in given for s in of(p)]
    assert len(passed) == 1 and made and set(made) == {side.cuda_stream}
    got, want = (d if isinstance(d, dict) else dict(out=d) for d in (got, want))
    assert got.keys() == want.keys()
    for k, t in want.items():
        if name == "spu_stage_of_nothing":                  # launches nothing: what its tensors hold is nobody's
            assert got[k].shape == t.shape
        else:
            assert torch.equal(got[k], t) if isinstance(t, torch.Tensor) else got[k] == t, k


@pytest.mark.parametrize("name", ["oim_merge", "spu_score", "spu_stage_ragged"])
def test_calls_behind_waiting_work_of_the_current_stream(name):
    """Work that waits on the current stream reads blocks that are free by then; calls on another stream go ahead of it."""
    inputs, table = calls()
    run = table[name]
    want = run(None)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    blocks = [torch.full((1 << k,), 77, dtype=torch.uint8, device="cuda") for k in range(9, 24) for _ in range(2)]
    torch.cuda._sleep(100_000_000)
    late = [b.clone() for b in blocks]
    del blocks
    got = [run(side) for _ in range(3)]
    torch.cuda.synchronize()
    assert all(bool((t == 77).all()) for t in late)
    for g in got:
        for k, t in (want if isinstance(want, dict) else dict(out=want)).items():
            assert torch.equal(g[k] if isinstance(g, dict) else g, t), k

"""GPU: what luvc_kv_attend allocates for a call on another stream does not meet what the current stream still uses.  Each test holds one
stream back with a kernel that only waits, and lets the other one go ahead."""
import pytest
import torch

from paper_2512_09010_amd import binding as lv
from test_gpu_kv import Pool

pytestmark = pytest.mark.gpu

WAIT = 100_000_000                                          # clock ticks, some 50 ms


def setup(seqs, Hq):
    pool = Pool(50, [3000, 1, 700] + [1] * (seqs - 3), 2, 128, "bf16", 16)
    q = pool.tensor(seqs, Hq, 128)
    want = lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    return pool, q, want


def test_workspace_is_not_a_block_that_the_current_stream_still_reads():
    pool, q, want = setup(3, 8)
    need = lv.luvc_kv_attend_workspace_bytes(pool.cache, 3, 8, 16 * pool.width)
    out, side = torch.zeros_like(q), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    block = torch.full((need,), 77, dtype=torch.uint8, device="cuda")
    torch.cuda._sleep(WAIT)
    late = block.clone()                                    # read after the wait
    del block                                               # free for the current stream's next allocation
    lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, stream=side, out=out)
    torch.cuda.synchronize()
    assert bool((late == 77).all()) and torch.equal(out, want)


def test_output_is_not_a_block_that_the_current_stream_still_reads():
    pool, q, want = setup(1000, 16)
    ws = torch.empty(lv.luvc_kv_attend_workspace_bytes(pool.cache, 1000, 16, 16 * pool.width), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    block = torch.full_like(q, 77.0)
    torch.cuda._sleep(WAIT)
    late = block.clone()
    del block
    out = lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, workspace=ws, stream=side)
    torch.cuda.synchronize()
    assert bool((late == 77.0).all()) and torch.equal(out, want)


def test_output_used_on_the_current_stream_is_not_handed_out_again_before():
    pool, q, want = setup(1000, 16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(WAIT)
    late = out.clone()
    del out
    with torch.cuda.stream(side):
        noise = [torch.full_like(q, 9.0) for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(late, want) and all(bool((t == 9.0).all()) for t in noise)


def test_two_calls_without_a_workspace_on_two_streams(monkeypatch):
    """One on the current stream, one on another right behind it: a workspace for each, and for a third of either."""
    pool, q, want = setup(3, 8)
    nat, spaces = lv._native(), []
    call = nat.call

    def seen(entry, *args):
        if entry == nat.luvc_kv_attend:
            spaces.append(args[14])
        return call(entry, *args)
    monkeypatch.setattr(nat, "call", seen)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda._sleep(WAIT)
    outs = [lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, stream=st) for st in (None, side, None, side)]
    torch.cuda.synchronize()
    assert len(spaces) == 4 and not {spaces[0], spaces[2]} & {spaces[1], spaces[3]}
    assert all(torch.equal(o, want) for o in outs)


def test_the_current_stream_given_by_name():
    pool, q, want = setup(3, 8)
    assert torch.equal(lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, stream=torch.cuda.current_stream()), want)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, stream=side)
    side.synchronize()
    assert torch.equal(got, want)

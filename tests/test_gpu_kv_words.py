"""GPU: the arrival words of luvc_kv_attend, at the front of its workspace, serve one launch: nothing a launch leaves there, or left undone,
reaches the next one."""
import pytest
import torch

from paper_2512_09010_amd import binding as lv
from test_gpu_kv import Pool, check_attend

pytestmark = pytest.mark.gpu

# lengths, heads, words to a sequence and head: one, and where runs are joined in groups one for each group besides
SHAPES = [([3000, 1, 700, 0, 2900], 2, 1), ([30000], 1, 16)]


@pytest.mark.parametrize("lengths, H, each", SHAPES)
def test_words_that_a_launch_left_half_counted(lengths, H, each):
    S, n = len(lengths), len(lengths) * H * each
    pool = Pool(70, lengths, H, 128, "bf16", 16)
    q, most = pool.tensor(S, 4 * H, 128), 16 * pool.width
    ws = torch.zeros(lv.luvc_kv_attend_workspace_bytes(pool.cache, S, 4 * H, most), dtype=torch.uint8, device="cuda")
    words = ws[:8 * n].view(torch.int64)
    run = lambda: lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, max_tokens=most, enhance=True, workspace=ws, out=torch.full_like(q, 5.0))
    want = run()
    check_attend(pool, q, want, enhance=True)
    assert bool((ws != 0).any()), "no parts were written: the case joins no runs"
    for count in (0, 1, 2, 3, 65535, 1):
        assert bool((words == 0).all()), "a launch leaves no tag"
        words += count                                      # what runs that never came would have left
        assert torch.equal(run(), want)
        words.zero_()


@pytest.mark.parametrize("lengths, H, each", SHAPES)
def test_words_between_the_replays_of_a_graph(lengths, H, each):
    S, n = len(lengths), len(lengths) * H * each
    pool = Pool(71, lengths, H, 128, "bf16", 16)
    q, out, most = pool.tensor(S, 4 * H, 128), torch.zeros((S, 4 * H, 128), dtype=torch.bfloat16, device="cuda"), 16 * pool.width
    ws = torch.zeros(lv.luvc_kv_attend_workspace_bytes(pool.cache, S, 4 * H, most), dtype=torch.uint8, device="cuda")
    words = ws[:8 * n].view(torch.int64)
    run = lambda o: lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, max_tokens=most, workspace=ws, out=o)
    want = run(torch.empty_like(q))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(out)
    for left in (0, 1, 2, -1, 1 << 40, 7):
        words.fill_(left)
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        out.fill_(5.0)
        graph.replay()                                      # right behind one that completed
        assert torch.equal(run(torch.empty_like(q)), want)
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_numbers_beyond_32_bits_are_refused():
    """Layers, bounds and counts that would pass by their lower 32 bits."""
    pool = Pool(72, [40, 20], 2, 64, "bf16", 16)
    c, q, n, wide = pool.cache, pool.tensor(2, 4, 64), pool.tensor(2, 2, 64), 2 ** 32
    refs = torch.ones(pool.n_pages, dtype=torch.int32)
    refs[-4:] = 0
    before = pool.kt.view(torch.int16).clone(), refs.clone()
    for bad in (lambda: lv.luvc_kv_attend(c, wide, q, pool.tt, pool.lt), lambda: lv.luvc_kv_attend(c, 0, q, pool.tt, pool.lt, max_tokens=wide + 5),
                lambda: lv.luvc_kv_attend(c, 0, q, pool.tt, pool.lt, max_tokens=wide + 5, workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda")),
                lambda: lv.luvc_kv_attend_workspace_bytes(c, wide + 2, 4, 64), lambda: lv.luvc_kv_write(c, wide, n, n, pool.lt - 1, pool.tt),
                lambda: lv.luvc_kv_fork(c, refs, [0], 5, wide + 1)):
        with pytest.raises(lv.LuvcError) as e:
            bad()
        assert e.value.status == lv.LUVC_ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert torch.equal(pool.kt.view(torch.int16), before[0]) and torch.equal(refs, before[1])

"""GPU: attention over the cache where every block of tokens is an output channel (kv_blocks.py), in a workspace of just the size asked for."""
import numpy as np
import pytest
import torch

from gpu_util import to_host_f64
from kv_blocks import CASES, Blocks
from paper_2512_09010_amd import binding as lv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lengths, Hq, H, D, dtype, P, dead, most", CASES, ids=lambda v: str(v)[:24])
def test_every_block_has_its_share(lengths, Hq, H, D, dtype, P, dead, most):
    case = Blocks(lengths, Hq, H, D, P, dead)
    dt, S, most = torch.float32 if dtype == "f32" else torch.bfloat16, len(lengths), most or max(lengths)
    dev = lambda a: torch.from_numpy(a).cuda()
    cache = lv.KvCache(dev(case.k).to(dt)[None], dev(case.v).to(dt)[None], dev(case.sizes))
    need, room = lv.luvc_kv_attend_workspace_bytes(cache, S, Hq, most), 4096
    space = torch.full((need + 2 * room,), 165, dtype=torch.uint8, device="cuda")
    want, tol = case.want(), case.relative_tolerance(dtype, most)
    q, table, n = dev(case.q).to(dt), dev(case.table), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    first = None
    for again in range(2):
        out = lv.luvc_kv_attend(cache, 0, q, table, n, max_tokens=most, scale=1.0, workspace=space[room:room + need], out=torch.full_like(q, 9.0))
        got = to_host_f64(out)
        off = ~(np.abs(got - want) <= tol * want)
        assert not off.any(), (int(off.sum()), [(tuple(i), got[tuple(i)], want[tuple(i)]) for i in np.argwhere(off)[:5]])
        assert bool((space[:room] == 165).all()) and bool((space[room + need:] == 165).all())
        assert first is None or torch.equal(out, first)
        first = out

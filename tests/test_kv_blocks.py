"""The cases of kv_blocks.py show what they are meant to show: whatever a call could lose or take twice is more than their tolerance."""
import numpy as np
import pytest

from kv_blocks import CASES, Blocks


@pytest.mark.parametrize("lengths, Hq, H, D, dtype, P, dead, most", CASES, ids=lambda v: str(v)[:24])
def test_lost_and_repeated_tokens_exceed_the_tolerance(lengths, Hq, H, D, dtype, P, dead, most):
    case = Blocks(lengths, Hq, H, D, P, dead)
    tol = case.relative_tolerance(dtype, most or max(lengths))
    piece = 16 if dtype == "f32" else 32                    # a wavefront's step, the least that is taken or left as a whole
    for s in sorted(range(len(lengths)), key=lambda i: -lengths[i])[:6]:
        n, live = lengths[s], case.seqs[s][0]
        want = case.shares(s)
        ranges = [(n - 1, n)] + [(a, min(a + piece, n)) for a in range(0, n, piece)]
        if len(ranges) > 400:                               # every one of a long sequence takes minutes
            ranges = ranges[:100] + ranges[-100:] + ranges[100:-100:len(ranges) // 200]
        if H > 4:
            ranges = ranges[:6] + ranges[-2:]
        for a, b in ranges:
            if n == 0 or not live[a:b].any() or live.sum() == live[a:b].sum():
                continue
            for times in (0, 2):
                t = np.ones(n)
                t[a:b] = times
                off = np.abs(case.shares(s, t) - want) > tol * want
                assert off.any(axis=1).all(), (s, a, b, times)


def test_shares_are_attention():
    """The shares against attention from the definition on the case's own pages."""
    import kv_reference as ref
    case = Blocks([50, 0, 17], 6, 2, 12, 16, dead=0.3)
    k, v = case.k.astype(np.float64), case.v.astype(np.float64)
    out, _, _, _ = ref.attend(case.q.astype(np.float64), k, v, case.sizes, case.table, case.lengths, 1.0, False)
    assert np.allclose(out, case.want(), rtol=1e-12, atol=0)

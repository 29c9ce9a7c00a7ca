"""GPU: attention over the cache weighs values with the bits of fp32, whatever the cache's type."""
import numpy as np
import pytest
import torch

from gpu_util import to_host_f64
from paper_2512_09010_amd import binding as lv

pytestmark = pytest.mark.gpu


def bf16(x):
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()


@pytest.mark.parametrize("spare", [0, 40, 700])
@pytest.mark.parametrize("D", [8, 128, 256])
def test_weights_of_bf16_caches_keep_the_bits_of_fp32(D, spare):
    """Three tokens of weights p, 1, 1 (over p + 2) and values 1, -b1, -b2 with b1 + b2 = p but for 2^-17: what is left is as small as a weight
    in two bf16 terms is wrong.  `spare` further tokens of weight 2^-40 and less with values of zero: steps and runs of the same sum.

    In units of 2^-24 on p: the one product of a logit is exact, its scaling and the difference to the maximum are two roundings of an
    argument of at most 1.45 (times ln 2: 2 units), the exponential 2, nine products that are added 2 each, two joins 2 each: 26.
    The sum of weights and the last division act on what is left only."""
    rng = np.random.default_rng(40 + D + spare)
    S, P, H = 48, 16, 8
    n = 3 + spare
    width = -(-n // P)
    x = -bf16(rng.uniform(0.01, 1.0, (S, H)))               # logits of the first token; the other two have 0
    p = np.exp(x)
    b1 = bf16(p)
    b2 = bf16(p - b1)
    k, v = np.zeros((S * width, H, P, D), np.float32), np.zeros((S * width, H, P, D), np.float32)
    at = rng.permutation(n)[:3] if spare else np.arange(3)
    rows = np.arange(S) * width
    for s in range(S):
        for j in range(n):
            k[rows[s] + j // P, :, j % P, 0] = -28.0        # 2^-40 = exp(-27.7)
    for i, (logit, value) in enumerate(((x, np.ones_like(p)), (np.zeros_like(x), -b1), (np.zeros_like(x), -b2))):
        k[rows + at[i] // P, :, at[i] % P, 0] = logit
        v[rows + at[i] // P, :, at[i] % P, :] = value[:, :, None]
    dev = lambda a: torch.from_numpy(a).cuda().to(torch.bfloat16)
    cache = lv.KvCache(dev(k)[None], dev(v)[None])
    q = torch.zeros((S, H, D), dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = 1.0
    table = torch.arange(S * width, dtype=torch.int32, device="cuda").view(S, width)
    out = to_host_f64(lv.luvc_kv_attend(cache, 0, q, table, torch.full((S,), n, dtype=torch.int32, device="cuda"), scale=1.0))
    total = p + 2 + spare * np.exp(-28.0)
    want = ((p - b1 - b2) / total)[:, :, None]
    tol = 2.0 ** -8 * np.abs(want) + 26 * 2.0 ** -24 * (p / total)[:, :, None]
    off = np.abs(out - want) - tol
    assert (off <= 0).all(), (int((off > 0).sum()), off.size, float((np.abs(out - want) / (p / total)[:, :, None]).max() * 2 ** 24))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("up", [100, -60])
def test_magnitudes_of_values_and_logits(dtype, up):
    """Values times a power of two give the output times that power, bit for bit, and so do keys for queries divided by it: nothing on the way
    leaves the range of fp32 (256 times a sum of 900 values of 2^100 is 2^118)."""
    gen = torch.Generator(device="cuda").manual_seed(90)
    S, H, P, D, width = 2, 2, 16, 64, 57
    k, v = (torch.randn((1, S * width, H, P, D), generator=gen, device="cuda").clamp(-4, 4).to(dtype) for _ in range(2))
    q = torch.randn((S, 4, D), generator=gen, device="cuda").to(dtype)
    table = torch.arange(S * width, dtype=torch.int32, device="cuda").view(S, width)
    n = torch.tensor([900, 33], dtype=torch.int32, device="cuda")
    f = 2.0 ** up
    want = lv.luvc_kv_attend(lv.KvCache(k, v), 0, q, table, n)
    assert torch.equal(lv.luvc_kv_attend(lv.KvCache(k, v * f), 0, q, table, n), want * f)
    g = 2.0 ** (up // 2)
    assert torch.equal(lv.luvc_kv_attend(lv.KvCache(k * g, v), 0, q / g, table, n), want)

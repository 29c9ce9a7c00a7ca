"""GPU: the paged key-value cache against plain numpy in 64 bits (tests/kv_reference.py): attention of one token within derived
tolerances, everything that moves rows bit for bit."""
import numpy as np
import pytest
import torch

import kv_reference as ref
from gpu_util import to_host_f64
from paper_2512_09010_amd import binding as lv

pytestmark = pytest.mark.gpu

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


class Pool:
    """Pages in shuffled order; whatever is not a live token of a sequence holds NaN, infinities and sizes of any kind."""

    def __init__(self, seed, lengths, H, D, dtype, P, layers=1, extra=3, sized=True, dead=0.0, spread=1.0, max_pages=None):
        rng = self.rng = np.random.default_rng(seed)
        need = [-(-n // P) for n in lengths]
        self.n_pages, self.P, self.dtype = sum(need) + extra, P, dtype
        order = list(rng.permutation(self.n_pages))
        self.width = max(1, max(need)) if max_pages is None else max_pages
        self.table = np.full((len(lengths), self.width), -1, np.int32)
        self.table[:, 1:] = rng.choice(np.array([-1, -2 ** 31, self.n_pages, 2 ** 31 - 1], np.int64), (len(lengths), self.width - 1)).astype(np.int32)
        for i, n in enumerate(need):
            for j in range(n):
                self.table[i, j] = order.pop()
        self.free = order
        shape = (layers, self.n_pages, H, P, D)
        junk = rng.choice(np.array([np.nan, np.inf, -np.inf, 3e38], np.float32), shape)
        k, v = junk.copy(), np.roll(junk, 1)
        sizes = rng.choice(np.array([0, -1, 7, -2 ** 31, 2 ** 31 - 1], np.int64), (self.n_pages, P)).astype(np.int32)
        for s, n in enumerate(lengths):
            for j, page, r in ref.tokens_of(self.table[s], n, P, self.n_pages):
                if sized and rng.random() < dead:
                    sizes[page, r] = rng.choice([0, 0, -1, -2 ** 31])
                    continue
                sizes[page, r] = rng.integers(1, 100)
                k[:, page, :, r] = rng.standard_normal((layers, H, D)) * spread
                v[:, page, :, r] = rng.standard_normal((layers, H, D))
        self.kt, self.vt = torch.tensor(k).cuda().to(TORCH[dtype]), torch.tensor(v).cuda().to(TORCH[dtype])
        self.st = torch.tensor(sizes).cuda() if sized else None
        self.tt, self.lengths = torch.tensor(self.table).cuda(), lengths
        self.lt = torch.tensor(lengths, dtype=torch.int32).cuda()
        self.sizes = sizes if sized else None
        self.cache = lv.KvCache(self.kt, self.vt, self.st)

    def tensor(self, *shape):
        return torch.tensor(self.rng.standard_normal(shape).astype(np.float32)).cuda().to(TORCH[self.dtype])


def check_attend(pool, q, out, layer=0, scale=None, enhance=False, lengths=None, table=None):
    D = q.shape[2]
    k, v = to_host_f64(pool.kt[layer]), to_host_f64(pool.vt[layer])
    with np.errstate(invalid="ignore"):
        want, bulk, steep, live = ref.attend(to_host_f64(q), k, v, pool.sizes, pool.table if table is None else table,
                                             pool.lengths if lengths is None else lengths, D ** -0.5 if scale is None else scale, enhance)
    got = to_host_f64(out)
    assert np.isfinite(got).all()
    err, tol = np.abs(got - want), ref.tolerance(want, bulk, steep, live, D, pool.dtype)
    i = np.unravel_index(np.argmax(err - tol), err.shape)
    assert (err <= tol).all(), (int((err > tol).sum()), err.size, i, got[i], want[i], tol[i])
    assert (got[live == 0] == 0).all()


# lengths, query heads, heads, D, dtype, page, sizes
SHAPES = [
    ([1], 1, 1, 1, "f32", 16, "none"),
    ([1], 4, 4, 128, "bf16", 16, "none"),
    ([0, 1, 2, 15, 16, 17, 31, 32, 33], 8, 2, 64, "bf16", 16, "none"),
    ([0, 1, 2, 15, 16, 17, 31, 32, 33], 8, 2, 64, "f32", 16, "enhance"),
    ([127, 128, 129, 130, 0, 260], 28, 4, 128, "bf16", 32, "mask"),
    ([127, 128, 129, 130, 0, 260], 28, 4, 128, "f32", 32, "mask"),
    ([513, 1025, 77], 32, 8, 128, "bf16", 16, "enhance"),
    ([513, 1025, 77], 32, 32, 128, "f32", 16, "none"),
    ([300, 5], 16, 1, 128, "bf16", 64, "mask"),
    ([300, 5], 17, 1, 128, "bf16", 64, "none"),
    ([300, 5], 71, 1, 96, "bf16", 64, "enhance"),
    ([300, 5], 33, 1, 96, "f32", 64, "mask"),
    ([300, 900], 12, 3, 256, "bf16", 128, "enhance"),
    ([300, 900], 12, 3, 256, "f32", 128, "enhance"),
    ([300, 900], 40, 2, 192, "bf16", 256, "none"),
    ([200, 90], 6, 6, 80, "bf16", 16, "mask"),
    ([200, 90], 6, 3, 72, "f32", 16, "none"),
    ([200, 90], 6, 3, 33, "bf16", 16, "enhance"),
    ([200, 90], 6, 3, 127, "f32", 16, "mask"),
    ([200, 90], 4, 2, 250, "bf16", 1024, "none"),
    ([40, 90], 4, 2, 5, "bf16", 16, "none"),
    ([40, 90], 4, 2, 20, "f32", 16, "none"),
    ([1500], 8, 1, 32, "bf16", 16, "mask"),
    ([5000, 3, 2500], 8, 2, 128, "bf16", 16, "enhance"),
    ([5000, 3, 2500], 8, 2, 64, "f32", 64, "mask"),
    # runs that are joined in groups, next to sequences of a few runs, of one, of none
    ([40000, 3000, 100, 0], 4, 1, 64, "bf16", 16, "none"),
    ([30000, 2000, 700], 2, 1, 100, "bf16", 64, "enhance"),
    ([20000, 11, 9000], 1, 1, 128, "f32", 32, "mask"),
    ([25000], 19, 1, 24, "bf16", 256, "mask"),
]


@pytest.mark.parametrize("lengths, Hq, H, D, dtype, P, sizes", SHAPES)
def test_attend(lengths, Hq, H, D, dtype, P, sizes):
    pool = Pool(1, lengths, H, D, dtype, P, sized=sizes != "none", dead=0.3 if sizes != "none" else 0.0)
    q = pool.tensor(len(lengths), Hq, D) * 2
    out = lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, enhance=sizes == "enhance")
    check_attend(pool, q, out, enhance=sizes == "enhance")
    # a bound on the lengths that is not tight, and one that cuts them
    for most in (max(lengths) + 3 * P, max(1, max(lengths) - 7)):
        out = lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, max_tokens=most, enhance=sizes == "enhance")
        check_attend(pool, q, out, enhance=sizes == "enhance", lengths=[min(n, most) for n in lengths])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_without_a_live_token(dtype):
    lengths = [70, 33, 0, 48, 300]
    pool = Pool(2, lengths, 2, 64, dtype, 16, dead=1.0)
    pool.sizes[pool.table[4, 0], 3] = 5                     # one token of the last sequence
    pool.st.copy_(torch.tensor(pool.sizes))
    pool.kt[0, int(pool.table[4, 0]), :, 3], pool.vt[0, int(pool.table[4, 0]), :, 3] = 1.0, 2.0
    pool.table[3] = -1                                      # no pages at all
    pool.tt.copy_(torch.tensor(pool.table))
    q = pool.tensor(5, 6, 64)
    for enhance in (False, True):
        out = lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, enhance=enhance, out=torch.full_like(q, 9.0))
        check_attend(pool, q, out, enhance=enhance)


def test_attend_skips_places_without_a_page():
    lengths = [200, 130]
    pool = Pool(3, lengths, 2, 128, "bf16", 16, sized=False)
    pool.table[0, [0, 3, 4, 12]] = [-1, pool.n_pages, -2 ** 31, 2 ** 31 - 1]
    pool.tt.copy_(torch.tensor(pool.table))
    q = pool.tensor(2, 8, 128)
    check_attend(pool, q, lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt))
    # lengths beyond the table, negative ones
    pool.lt.copy_(torch.tensor([2 ** 31 - 1, -5]))
    pool.table[1] = pool.table[1][::-1].copy()
    pool.kt[:] = pool.tensor(*pool.kt.shape)
    pool.vt[:] = pool.tensor(*pool.vt.shape)
    out = lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, max_tokens=10 ** 6)
    check_attend(pool, q, out, lengths=[pool.width * 16, 0])


@pytest.mark.parametrize("dtype, spread, scale", [("bf16", 1.0, 0.5), ("bf16", 30.0, None), ("f32", 30.0, None), ("f32", 1.0, -1.0), ("bf16", 1.0, 0.0), ("f32", 300.0, None)])
def test_attend_scales_and_steep_softmax(dtype, spread, scale):
    """Logits of hundreds: one token takes all; a scale of zero: the mean of the values."""
    pool = Pool(4, [333, 64], 2, 128, dtype, 16, spread=spread)
    q = pool.tensor(2, 8, 128) * 3
    out = lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, scale=scale, enhance=True)
    check_attend(pool, q, out, scale=scale, enhance=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_strided_and_unaligned_tensors(dtype):
    D, Hq, H = 64, 6, 2
    pool = Pool(5, [100, 40, 77], H, D, dtype, 32, layers=3)
    wide = pool.tensor(3, (Hq + 2 * H) * D + 1)
    q = wide.as_strided((3, Hq, D), (wide.stride(0), D, 1), 1)
    buf = torch.full((3, Hq * D + 5), 7.0, dtype=TORCH[dtype], device="cuda")
    out = buf.as_strided((3, Hq, D), (buf.stride(0), D, 1), 3)
    lv.luvc_kv_attend(pool.cache, 2, q, pool.tt, pool.lt, out=out, enhance=True)
    check_attend(pool, q.contiguous(), out.contiguous(), layer=2, enhance=True)
    assert bool((buf[:, :3] == 7).all()) and bool((buf[:, 3 + Hq * D:] == 7).all())
    # a pool that starts at an odd element
    k1 = torch.empty(pool.kt.numel() + 1, dtype=TORCH[dtype], device="cuda")[1:].view(pool.kt.shape)
    k1.copy_(pool.kt)
    out = lv.luvc_kv_attend(lv.KvCache(k1, pool.vt, pool.st), 1, q, pool.tt, pool.lt)
    check_attend(pool, q.contiguous(), out, layer=1)


def test_attend_beyond_32_bits():
    """Keys and values of more than 2^32 elements each; the pages in use lie at both ends."""
    P, H, D = 1024, 8, 128
    n_pages = (1 << 32) // (P * H * D) + 4
    pool = Pool(6, [2050, 1000], H, D, "bf16", P, sized=False)
    k = torch.empty((1, n_pages, H, P, D), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    far = {p: (n_pages - 1 - p if p % 2 else p) for p in range(pool.n_pages)}
    for p, f in far.items():
        k[0, f], v[0, f] = pool.kt[0, p], pool.vt[0, p]
    table = torch.tensor([[far.get(int(p), -1) for p in row] for row in pool.table], dtype=torch.int32).cuda()
    q = pool.tensor(2, 16, D)
    cache = lv.KvCache(k, v)
    check_attend(pool, q, lv.luvc_kv_attend(cache, 0, q, table, pool.lt))
    # rows written there, a page copied there, a sequence compacted there
    new = pool.tensor(3, H, D)
    pos = torch.tensor([2050, 2051, 1000], dtype=torch.int32).cuda()
    lv.luvc_kv_write(cache, 0, new, new, pos, table, seq=torch.tensor([0, 0, 1], dtype=torch.int32).cuda())
    last = [int(table[0, 2]), int(table[0, 2]), int(table[1, 0])]
    for t, (page, row) in enumerate(zip(last, (2, 3, 1000))):
        assert torch.equal(k[0, page, :, row], new[t]) and torch.equal(v[0, page, :, row], new[t])
    lv.luvc_kv_copy_pages(cache, [last[0]], [n_pages // 2])
    assert torch.equal(k[0, n_pages // 2], k[0, last[0]]) or torch.equal(k[0, n_pages // 2].view(torch.int16), k[0, last[0]].view(torch.int16))
    out = torch.tensor([[n_pages - 6]], dtype=torch.int32).cuda()
    lv.luvc_kv_compact(cache, torch.tensor([2049], dtype=torch.int32).cuda(), [2052], [0], [2050], [1], table[:1].contiguous(), out)
    row0 = k[0, int(table[0, 2]), :, 1:4]
    assert torch.equal(k[0, n_pages - 6, :, :3].contiguous().view(torch.int16), row0.contiguous().view(torch.int16))
    del k, v, cache
    torch.cuda.empty_cache()


@pytest.mark.parametrize("long", [False, True])
def test_attend_with_stale_workspaces_streams_and_repeats(long):
    """Same bits whatever the workspace held, on other streams at once, call after call."""
    pool = Pool(7, [3000, 1, 700, 0, 2900, 64] if not long else [30000, 1, 700, 0, 2900, 64], 1 if long else 2, 128, "bf16", 16)
    q, most = pool.tensor(6, 8, 128), 16 * pool.width
    want = lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, enhance=True)
    check_attend(pool, q, want, enhance=True)
    need = lv.luvc_kv_attend_workspace_bytes(pool.cache, 6, 8, most)
    gen = torch.Generator(device="cuda").manual_seed(3)
    streams = [torch.cuda.Stream() for _ in range(3)]
    spaces = [torch.randint(0, 256, (need,), generator=gen, dtype=torch.uint8, device="cuda") for _ in streams]
    outs = [[torch.empty_like(q) for _ in range(8)] for _ in streams]
    torch.cuda.synchronize()
    for i in range(8):
        for st, ws, o in zip(streams, spaces, outs):
            lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, max_tokens=most, enhance=True, workspace=ws, out=o[i], stream=st)
    torch.cuda.synchronize()
    again = lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, max_tokens=most, enhance=True)
    for o in outs:
        for t in o:
            assert torch.equal(t, again)


def test_attend_on_another_stream_keeps_its_own_workspace():
    """A workspace that the binding allocates is not handed out again before the call on the other stream has ended."""
    pool = Pool(30, [3000, 1, 700], 2, 128, "bf16", 16)
    q, out = pool.tensor(3, 8, 128), torch.zeros((3, 8, 128), dtype=torch.bfloat16, device="cuda")
    need = lv.luvc_kv_attend_workspace_bytes(pool.cache, 3, 8, 16 * pool.width)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    want = lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt)             # leaves one free block of that size
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)                      # holds the call back while its workspace might be handed out
    lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, stream=side, out=out)
    noise = [torch.full((need,), 255, dtype=torch.uint8, device="cuda") for _ in range(16)]
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    assert all(bool((t == 255).all()) for t in noise)


def test_attend_in_a_graph_follows_lengths_and_tables():
    pool = Pool(8, [2000, 900, 40, 1], 2, 64, "bf16", 16)
    q, out = pool.tensor(4, 4, 64), torch.zeros((4, 4, 64), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(lv.luvc_kv_attend_workspace_bytes(pool.cache, 4, 4, 2000), dtype=torch.uint8, device="cuda")
    new_k, new_v = pool.tensor(4, 2, 64), pool.tensor(4, 2, 64)
    pos = pool.lt - 1
    run = lambda: (lv.luvc_kv_write(pool.cache, 0, new_k, new_v, pos, pool.tt),
                   lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, max_tokens=2000, enhance=True, workspace=ws, out=out))
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    sizes = pool.sizes
    for lengths in ([2000, 900, 40, 1], [1999, 1, 0, 1], [3, 899, 33, 0], [2000, 2, 1, 1]):
        pool.lt.copy_(torch.tensor(lengths, dtype=torch.int32))
        torch.sub(pool.lt, 1, out=pos)
        new_k.normal_()
        q.normal_()
        out.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        for s, n in enumerate(lengths):
            if n:
                sizes[pool.table[s, (n - 1) // 16], (n - 1) % 16] = 1
        eager = lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, max_tokens=2000, enhance=True)
        assert torch.equal(out, eager)
        check_attend(pool, q, out, enhance=True, lengths=lengths)


@pytest.mark.parametrize("S, most", [(70, 80), (300, 4096), (1024, 10 ** 5), (1025, 4096), (1100, 60)])
@pytest.mark.parametrize("dtype, Hq, H, D", [("bf16", 6, 2, 64), ("f32", 2, 2, 20)])
def test_attend_of_many_sequences(S, most, dtype, Hq, H, D):
    """Mostly short ones, with a long one first, last or between, and lengths of zero; the bound on them tight or far away."""
    rng = np.random.default_rng(20 + S)
    lengths = [int(n) for n in rng.integers(0, 40, S)]
    for i in (0, S // 2, S - 1):
        lengths[i] = int(rng.integers(60, 80) if most < 100 else rng.integers(1000, 3000))
    pool = Pool(21, lengths, H, D, dtype, 16, sized=False)
    q = pool.tensor(S, Hq, D)
    check_attend(pool, q, lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, max_tokens=most), lengths=[min(n, most) for n in lengths])


@pytest.mark.parametrize("lengths", [[0], [1], [17], [130], [4000], [20000]])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_of_one_sequence_within_a_distant_bound(lengths, dtype):
    pool = Pool(22, lengths, 4, 64, dtype, 64, dead=0.2, max_pages=2048)
    q = pool.tensor(1, 8, 64)
    check_attend(pool, q, lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, enhance=True), enhance=True)


@pytest.mark.parametrize("scale", [1e-300, 1e-44, -1e-20, 0.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_with_scales_next_to_zero(scale, dtype):
    """The mean of the values of the tokens that take part."""
    pool = Pool(23, [77, 3], 2, 64, dtype, 16, dead=0.3)
    q = pool.tensor(2, 4, 64)
    check_attend(pool, q, lv.luvc_kv_attend(pool.cache, 0, q, pool.tt, pool.lt, scale=scale), scale=scale)


@pytest.mark.parametrize("D, dtype", [(33, "bf16"), (96, "f32")])
def test_attend_strided_tensors_with_several_runs(D, dtype):
    pool = Pool(24, [3000, 0, 1200, 40], 4, D, dtype, 16, layers=2)
    wide = pool.tensor(4, 8 * D + 3)
    q = wide.as_strided((4, 8, D), (wide.stride(0), D, 1), 2)
    buf = torch.full((4, 8 * D + 5), 7.0, dtype=TORCH[dtype], device="cuda")
    out = buf.as_strided((4, 8, D), (buf.stride(0), D, 1), 3)
    lv.luvc_kv_attend(pool.cache, 1, q, pool.tt, pool.lt, max_tokens=10 ** 5, out=out)
    check_attend(pool, q.contiguous(), out.contiguous(), layer=1)
    assert bool((buf[:, :3] == 7).all()) and bool((buf[:, 3 + 8 * D:] == 7).all())


def test_attend_graphs_with_room_to_grow_on_one_workspace():
    """Captured for more tokens than the sequences have yet; a graph of four sequences, one of a single one and eager calls of three take
    turns on a workspace that was made for the largest of them."""
    most = 8192
    pool = Pool(25, [6000, 900, 40, 1], 4, 64, "bf16", 16, max_pages=most // 16)
    q = pool.tensor(4, 8, 64)
    outs = [torch.zeros((n, 8, 64), dtype=torch.bfloat16, device="cuda") for n in (4, 1)]
    ws = torch.empty(lv.luvc_kv_attend_workspace_bytes(pool.cache, 4, 8, most), dtype=torch.uint8, device="cuda")
    run = lambda o: lv.luvc_kv_attend(pool.cache, 0, q[:len(o)], pool.tt[:len(o)], pool.lt[:len(o)], max_tokens=most, enhance=True, workspace=ws, out=o)
    for o in outs:
        run(o)
    torch.cuda.synchronize()
    graphs = []
    for o in outs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            run(o)
    for lengths in ([6000, 900, 40, 1], [5999, 0, 40, 0], [1, 700, 3, 1], [0, 0, 0, 0], [2500, 899, 39, 1]):
        pool.lt.copy_(torch.tensor(lengths, dtype=torch.int32))
        q.normal_()
        for o in outs:
            o.fill_(5.0)
        graphs[0].replay()
        three = run(torch.empty_like(q[:3]))
        graphs[1].replay()
        torch.cuda.synchronize()
        check_attend(pool, q, outs[0], enhance=True, lengths=lengths)
        check_attend(pool, q[:3], three, enhance=True, lengths=lengths[:3], table=pool.table[:3])
        check_attend(pool, q[:1], outs[1], enhance=True, lengths=lengths[:1], table=pool.table[:1])


# ------------------------------------------------------------------ moving rows

def bits(t):
    return t.contiguous().view({torch.bfloat16: torch.int16, torch.float32: torch.int32, torch.int32: torch.int32}[t.dtype]).cpu().numpy()


MOVES = [("bf16", 128, 16, 4), ("f32", 128, 32, 8), ("bf16", 80, 64, 1), ("bf16", 33, 16, 3), ("f32", 5, 16, 2), ("bf16", 1, 16, 1), ("bf16", 4, 128, 7),
         ("f32", 256, 16, 2), ("bf16", 250, 32, 2)]


@pytest.mark.parametrize("dtype, D, P, H", MOVES)
@pytest.mark.parametrize("how", ["padded", "rows", "unsized", "slices"])
def test_write(dtype, D, P, H, how):
    pool = Pool(9, [40, 300, 1, 95], H, D, dtype, P, layers=2, sized=how != "unsized", max_pages=20)
    rng = np.random.default_rng(10)
    T = 4 if how == "rows" else 150
    places = [(s, p) for s, n in enumerate(pool.lengths) for p in range(n)]
    picked = [places[i] for i in rng.permutation(len(places))[:T]]
    if how == "rows":
        seq, pos = None, np.array([7, 299, 0, 94], np.int32)
    else:
        seq, pos = np.array([s for s, _ in picked], np.int32), np.array([p for _, p in picked], np.int32)
        if how == "padded":
            seq[::7], seq[3::31], pos[5::13], pos[6::29], pos[11::37] = -1, 4, -3, 20 * P, 2 ** 31 - 1
            pos[12::41] = 20 * P - 1                        # a place without a page
    if how == "slices":
        qkv = pool.tensor(T, 2 * H * D + 8 + H * D)
        nk = qkv.as_strided((T, H, D), (qkv.stride(0), D, 1), 8)
        nv = qkv.as_strided((T, H, D), (qkv.stride(0), D, 1), 8 + H * D)
    else:
        nk, nv = pool.tensor(T, H, D), pool.tensor(T, H, D)
    ns = torch.tensor(rng.integers(-2, 50, T).astype(np.int32)).cuda() if how in ("padded", "slices") else None
    k, v = bits(pool.kt).copy(), bits(pool.vt).copy()
    sizes = None if pool.sizes is None else pool.sizes.copy()
    ref.write(k[1], v[1], sizes, bits(nk), bits(nv), None if ns is None else ns.cpu().numpy(), seq, pos, pool.table)
    lv.luvc_kv_write(pool.cache, 1, nk, nv, torch.tensor(pos).cuda(), pool.tt, seq=None if seq is None else torch.tensor(seq).cuda(), sizes=ns)
    assert np.array_equal(bits(pool.kt), k) and np.array_equal(bits(pool.vt), v)
    assert sizes is None or np.array_equal(pool.st.cpu().numpy(), sizes)


@pytest.mark.parametrize("dtype, D, P, H", MOVES)
@pytest.mark.parametrize("sized", [True, False])
def test_compact(dtype, D, P, H, sized):
    lengths, first, span, keep = [40, 300, 1, 2 * P, 190, 70], [3, 2 * P + 1, 0, P, 190, 0], [30, 300 - 3 * P - 9, 1, P, 0, 70], [11, 20, 0, P, 0, 0]
    if 300 - 3 * P - 9 < 20:
        first[1], span[1] = 5, 250
    lengths[3], lengths[4] = 2 * P, 190
    pool = Pool(11, lengths, H, D, dtype, P, layers=3, sized=sized, extra=60)
    rng = np.random.default_rng(12)
    kept = np.concatenate([np.sort(rng.permutation(s)[:k]) for s, k in zip(span, keep)]).astype(np.int32)
    after = [n - s + k for n, s, k in zip(lengths, span, keep)]
    out = np.full((len(lengths), max(-(-n // P) for n in after) + 2), -1, np.int32)
    free = list(pool.free)
    for i, n in enumerate(after):
        stay = first[i] // P if i % 2 else 0                # every other sequence leaves the pages of its front where they are
        for j in range(-(-n // P)):
            out[i, j] = pool.table[i, j] if j < stay else free.pop()
    k, v = bits(pool.kt).copy(), bits(pool.vt).copy()
    sizes = None if not sized else pool.sizes.copy()
    want = ref.compact([k, v], sizes, kept, lengths, first, span, keep, pool.table, out)
    got = lv.luvc_kv_compact(pool.cache, torch.tensor(kept).cuda(), lengths, first, span, keep, pool.tt, torch.tensor(out).cuda())
    assert got == want == after
    assert np.array_equal(bits(pool.kt), k) and np.array_equal(bits(pool.vt), v)
    assert sizes is None or np.array_equal(pool.st.cpu().numpy(), sizes)


def test_compact_of_many_sequences_and_bad_entries():
    """150 sequences: more than one launch; positions and pages that are none move nothing."""
    P, H, D, S = 16, 2, 64, 150
    rng = np.random.default_rng(13)
    lengths = [int(n) for n in rng.integers(1, 120, S)]
    span = [int(rng.integers(0, n + 1)) for n in lengths]
    first = [int(rng.integers(0, n - s + 1)) for n, s in zip(lengths, span)]
    keep = [int(rng.integers(0, s + 1)) for s in span]
    pool = Pool(14, lengths, H, D, "bf16", P, sized=True, extra=1000)
    kept = np.concatenate([np.sort(rng.permutation(s)[:k]) for s, k in zip(span, keep)]).astype(np.int32)
    kept[rng.permutation(len(kept))[:9]] = [-1, 2 ** 31 - 1, -2 ** 31, 120, 500, -7, 10 ** 6, 121, 122]
    out = np.full((S, 8), -1, np.int32)
    for i in range(S):
        out[i] = [pool.free.pop() if rng.random() < 0.95 and len(pool.free) else int(rng.choice([-1, pool.n_pages, 2 ** 31 - 1])) for _ in range(8)]
    pool.table[7, 0], pool.table[140, 0] = -1, pool.n_pages
    pool.tt.copy_(torch.tensor(pool.table))
    k, v, sizes = bits(pool.kt).copy(), bits(pool.vt).copy(), pool.sizes.copy()
    want = ref.compact([k, v], sizes, kept, lengths, first, span, keep, pool.table, out)
    assert lv.luvc_kv_compact(pool.cache, torch.tensor(kept).cuda(), lengths, first, span, keep, pool.tt, torch.tensor(out).cuda()) == want
    assert np.array_equal(bits(pool.kt), k) and np.array_equal(bits(pool.vt), v) and np.array_equal(pool.st.cpu().numpy(), sizes)


@pytest.mark.parametrize("dtype, D, P, H", MOVES)
@pytest.mark.parametrize("pairs, sized", [(1, True), (7, False), (300, True)])
def test_copy_pages(dtype, D, P, H, pairs, sized):
    layers = 2 if pairs < 100 else 1
    pool = Pool(15, [P], H, D, dtype, P, layers=layers, sized=sized, extra=2 * pairs + 5)
    pool.kt.copy_(pool.tensor(*pool.kt.shape))
    pool.vt.copy_(pool.tensor(*pool.vt.shape))
    order = np.random.default_rng(16).permutation(pool.n_pages)
    src, dst = [int(order[i // 2]) for i in range(pairs)], [int(p) for p in order[pairs:2 * pairs]]       # a page may be read twice
    k, v = bits(pool.kt).copy(), bits(pool.vt).copy()
    for a, b in zip(src, dst):
        k[:, b], v[:, b] = k[:, a], v[:, a]
        if sized:
            pool.sizes[b] = pool.sizes[a]
    lv.luvc_kv_copy_pages(pool.cache, src, torch.tensor(dst, dtype=torch.int32))
    assert np.array_equal(bits(pool.kt), k) and np.array_equal(bits(pool.vt), v)
    assert not sized or np.array_equal(pool.st.cpu().numpy(), pool.sizes)
    lv.luvc_kv_copy_pages(pool.cache, [], [])


def test_layers_with_room_between_them():
    """A layer stride that is larger than a layer."""
    base = torch.zeros((3, 6, 2, 16, 32), dtype=torch.float32, device="cuda").normal_()
    k, v = base[:, :5], base[:, :5].clone()
    room = torch.empty((3, 6, 2, 16, 32), device="cuda").normal_()
    v = room[:, :5]
    keep_k, keep_v = base[:, 5].clone(), room[:, 5].clone()
    cache = lv.KvCache(k, v)
    wk, wv = k.clone(), v.clone()
    wk[:, 3], wv[:, 3] = wk[:, 1], wv[:, 1]
    lv.luvc_kv_copy_pages(cache, [1], [3])
    assert torch.equal(k, wk) and torch.equal(v, wv) and torch.equal(base[:, 5], keep_k) and torch.equal(room[:, 5], keep_v)
    with pytest.raises(AssertionError):
        lv.KvCache(k, v.contiguous())                       # one stride serves both


@pytest.mark.parametrize("dtype, D, P, H", MOVES)
@pytest.mark.parametrize("length, children", [(1, 1), (16, 3), (50, 2), (129, 5), (300, 600)])
def test_fork(dtype, D, P, H, length, children):
    used = -(-length // P)
    if children > 100 and D > 64:
        children = 20
    pool = Pool(17, [length], H, D, dtype, P, layers=2, sized=True, extra=children + 4)
    refs = torch.zeros(pool.n_pages, dtype=torch.int32)
    parent = pool.table[0, :used]
    refs[torch.tensor(parent).long()] = 2
    refs[pool.free[:3]] = 1
    rows, start = length % P, refs.clone()
    free = [p for p in range(pool.n_pages) if refs[p] == 0][:children]
    k, v = bits(pool.kt).copy(), bits(pool.vt).copy()
    want = np.tile(parent, (children, 1))
    if rows:
        for c, p in enumerate(free):
            want[c, -1] = p
            k[:, p, :, :rows], v[:, p, :, :rows] = k[:, parent[-1], :, :rows], v[:, parent[-1], :, :rows]
            pool.sizes[p, :rows] = pool.sizes[parent[-1], :rows]
    got = lv.luvc_kv_fork(pool.cache, refs, torch.tensor(parent), length, children)
    assert np.array_equal(got.numpy(), want)
    assert np.array_equal(bits(pool.kt), k) and np.array_equal(bits(pool.vt), v) and np.array_equal(pool.st.cpu().numpy(), pool.sizes)
    for p in range(pool.n_pages):
        assert int(refs[p]) == int(start[p]) + int((want == p).sum())
    lv.luvc_kv_release(refs, got)
    assert torch.equal(refs, start)


def test_compact_of_forks_that_share_a_prompt():
    """Three sequences read the same pages; two of them leave the pages of the front where they are, for both."""
    P, H, D, n, first, span = 16, 2, 64, 100, 35, 50
    pool = Pool(26, [n], H, D, "bf16", P, layers=2, extra=20)
    table = np.tile(pool.table[0], (3, 1))
    kept = np.concatenate([np.sort(np.random.default_rng(27 + i).permutation(span)[:k]) for i, k in enumerate((10, 0, 50))]).astype(np.int32)
    out = np.full((3, 7), -1, np.int32)
    for i, after in enumerate((60, 50, 100)):
        for j in range(-(-after // P)):
            out[i, j] = table[i, j] if i < 2 and j < first // P else pool.free.pop()
    k, v, sizes = bits(pool.kt).copy(), bits(pool.vt).copy(), pool.sizes.copy()
    want = ref.compact([k, v], sizes, kept, [n] * 3, [first] * 3, [span] * 3, [10, 0, 50], table, out)
    assert lv.luvc_kv_compact(pool.cache, torch.tensor(kept).cuda(), [n] * 3, [first] * 3, [span] * 3, [10, 0, 50], torch.tensor(table).cuda(), torch.tensor(out).cuda()) == want
    assert np.array_equal(bits(pool.kt), k) and np.array_equal(bits(pool.vt), v) and np.array_equal(pool.st.cpu().numpy(), sizes)


def test_captured_writes_copies_and_compactions():
    """The host lists of a captured call are those of the capture, whatever becomes of them; device arrays are read anew."""
    P, H, D, n = 16, 2, 80, 150
    pool = Pool(28, [n, n], H, D, "bf16", P, layers=2, extra=40)
    nk, nv = pool.tensor(6, H, D), pool.tensor(6, H, D)
    seq, pos = torch.tensor([0, 1, 0, 1, -1, 0], dtype=torch.int32).cuda(), torch.tensor([3, 149, 77, 0, 5, 16], dtype=torch.int32).cuda()
    kept = torch.arange(24, dtype=torch.int32).cuda()
    out = torch.tensor([[pool.free.pop() for _ in range(10)] for _ in range(2)], dtype=torch.int32).cuda()
    src, dst = torch.tensor(pool.table[0, :3]), torch.tensor([pool.free.pop() for _ in range(3)], dtype=torch.int32)
    spans = [torch.tensor(x, dtype=torch.int32) for x in ([n, n], [20, 0], [100, 140], [12, 12])]

    def run(spans, src, dst):
        lv.luvc_kv_write(pool.cache, 1, nk, nv, pos, pool.tt, seq=seq)
        lv.luvc_kv_compact(pool.cache, kept, *spans, pool.tt, out)
        lv.luvc_kv_copy_pages(pool.cache, src, dst)
    held = [list(map(int, t)) for t in spans], list(map(int, src)), list(map(int, dst))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        run(spans, src, dst)
    for t in (*spans, src, dst):
        t.fill_(0)
    start = pool.kt.clone(), pool.vt.clone(), pool.st.clone()
    for step in range(4):
        nk.normal_()
        pos[0] = 4 + step
        kept.copy_(torch.cat([torch.randperm(100)[:12].sort().values, torch.randperm(140)[:12].sort().values]).to(torch.int32))
        after = []
        for f in (graph.replay, lambda: run(*held)):
            for t, was in zip((pool.kt, pool.vt, pool.st), start):
                t.copy_(was)
            f()
            torch.cuda.synchronize()
            after.append((bits(pool.kt).copy(), bits(pool.vt).copy(), pool.st.cpu().numpy().copy()))
        assert all(np.array_equal(a, b) for a, b in zip(*after))
        assert not np.array_equal(after[0][0], bits(start[0]))


def test_calls_the_binding_refuses():
    pool = Pool(29, [40, 20], 2, 64, "bf16", 16)
    c, q, n = pool.cache, pool.tensor(2, 4, 64), pool.tensor(2, 2, 64)
    pos = pool.lt - 1
    before = bits(pool.kt).copy(), pool.st.clone()
    for bad in (lambda: lv.luvc_kv_attend(c, 0, q.float(), pool.tt, pool.lt), lambda: lv.luvc_kv_attend(c, 0, q.cpu(), pool.tt, pool.lt),
                lambda: lv.luvc_kv_attend(c, 0, q, pool.tt.cpu(), pool.lt), lambda: lv.luvc_kv_attend(c, 0, q, pool.tt, pool.lt.long()),
                lambda: lv.luvc_kv_attend(c, 0, q, pool.tt[:1], pool.lt), lambda: lv.luvc_kv_attend(c, 0, q.transpose(1, 2), pool.tt, pool.lt),
                lambda: lv.luvc_kv_attend(c, 0, q[:, :3], pool.tt, pool.lt), lambda: lv.luvc_kv_attend(c, 1, q, pool.tt, pool.lt),
                lambda: lv.luvc_kv_attend(c, 0, q, pool.tt, pool.lt, workspace=torch.empty(0, dtype=torch.uint8, device="cuda")),
                lambda: lv.luvc_kv_attend(c, 0, q, pool.tt, pool.lt, out=torch.empty(1, 4, 64, dtype=torch.bfloat16, device="cuda").expand(2, 4, 64)),
                lambda: lv.luvc_kv_attend(lv.KvCache(pool.kt, pool.vt), 0, q, pool.tt, pool.lt, enhance=True),
                lambda: lv.luvc_kv_write(c, 0, n, n[:1], pos, pool.tt), lambda: lv.luvc_kv_write(c, 0, n.cpu(), n.cpu(), pos, pool.tt),
                lambda: lv.luvc_kv_write(c, 0, n, n, pos[:1], pool.tt), lambda: lv.luvc_kv_write(c, -1, n, n, pos, pool.tt),
                lambda: lv.luvc_kv_write(lv.KvCache(pool.kt, pool.vt), 0, n, n, pos, pool.tt, sizes=pos),
                lambda: lv.luvc_kv_copy_pages(c, [0, 1], [2]), lambda: lv.luvc_kv_copy_pages(c, [0], [0]), lambda: lv.luvc_kv_copy_pages(c, [0], [pool.n_pages]),
                lambda: lv.luvc_kv_compact(c, pos, [40, 20], [0, 0], [30, 10], [1, 0], pool.tt, pool.tt),
                lambda: lv.luvc_kv_compact(c, pos, [40, 20], [0, 0], [30, 10], [1], pool.tt, pool.tt),
                lambda: lv.luvc_kv_fork(c, torch.ones(3, dtype=torch.int32), [0], 5, 1), lambda: lv.luvc_kv_fork(c, torch.ones(pool.n_pages, dtype=torch.int64), [0], 5, 1),
                lambda: lv.KvCache(pool.kt.cpu(), pool.vt.cpu()), lambda: lv.KvCache(pool.kt, pool.vt.float()), lambda: lv.KvCache(pool.kt, pool.vt, pool.st[:1])):
        with pytest.raises((AssertionError, lv.LuvcError)):
            bad()
    torch.cuda.synchronize()
    assert np.array_equal(bits(pool.kt), before[0]) and torch.equal(pool.st, before[1])


# ------------------------------------------------------------------ all of it, as a serving program uses it

@pytest.mark.parametrize("dtype, model, H, Hq, D", [("bf16", 512, 2, 8, 64), ("f32", 256, 2, 2, 128)])
def test_prompt_stage_compaction_and_forked_decoding(dtype, model, H, Hq, D):
    """Merge an image, write its tokens and the text around them into two layers, prune at the second, compact the first, fork the
    prompt, decode a few tokens of every continuation in each layer: outputs against attention over plain lists of tokens."""
    torch.manual_seed(0)
    dt, P, B, layers = TORCH[dtype], 16, 2, 2
    x = torch.randn(B, 12, 12, model, device="cuda").to(dt)
    merged = lv.luvc_oim_merge(x, [(1, 6), (0, 6)])
    N, before, after = 36, 21, 9
    tokens = merged["x"].view(B, N, model)
    n_pages = 64
    k = torch.full((layers, n_pages, H, P, D), float("nan"), dtype=dt, device="cuda")
    v, sizes = k.clone(), torch.zeros((n_pages, P), dtype=torch.int32, device="cuda")
    cache, refs = lv.KvCache(k, v, sizes), torch.zeros(n_pages, dtype=torch.int32)
    total = before + N + after
    pages = [lv.luvc_kv_take(refs, -(-total // P)) for _ in range(B)]
    table = torch.stack(pages).cuda()
    # the prompt: per token [q, k, v] of one projection, here of random weights
    w = torch.randn(layers, model, (Hq + 2 * H) * D, device="cuda") / model ** 0.5
    text = torch.randn(B, before + after, model, device="cuda").to(dt)
    prompt = torch.cat([text[:, :before], tokens, text[:, before:]], 1).reshape(B * total, model)
    size = torch.cat([torch.ones(B, before, device="cuda"), merged["sizes"].view(B, N), torch.ones(B, after, device="cuda")], 1).to(torch.int32).reshape(-1)
    seq = torch.arange(B, device="cuda", dtype=torch.int32).repeat_interleave(total)
    pos = torch.arange(total, device="cuda", dtype=torch.int32).repeat(B)
    held = [[] for _ in range(layers)]                     # [layer][sequence]: k, v, sizes of its tokens in order
    for l in range(layers):
        qkv = (prompt.float() @ w[l]).to(dt).view(B * total, Hq + 2 * H, D)
        nk, nv = qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
        lv.luvc_kv_write(cache, l, nk, nv, pos, table, seq=seq, sizes=size)
        for b in range(B):
            at = slice(b * total, (b + 1) * total)
            held[l].append((to_host_f64(nk[at]), to_host_f64(nv[at]), size[at].cpu().numpy()))
    stage = lv.luvc_spu_stage(tokens, 4, 10)
    new_pages = [lv.luvc_kv_take(refs, -(-(total - N + 10) // P)) for _ in range(B)]
    out_table = torch.full((B, 6), -1, dtype=torch.int32)
    for b in range(B):
        out_table[b, :len(new_pages[b])] = new_pages[b]
    lengths = lv.luvc_kv_compact(cache, stage["kept_idx"], [total] * B, [before] * B, [N] * B, [10] * B, table, out_table.cuda())
    for p in pages:
        lv.luvc_kv_release(refs, p)
    kept = stage["kept_idx"].cpu().numpy()
    for l in range(layers):
        for b in range(B):
            live = np.concatenate([np.arange(before), before + kept[b], np.arange(before + N, total)])
            held[l][b] = tuple(a[live] for a in held[l][b])
    assert lengths == [total - N + 10] * B
    # three continuations of the first prompt, the second as it is
    kids = lv.luvc_kv_fork(cache, refs, new_pages[0], lengths[0], 3)
    rows = [list(new_pages[0].tolist())] + kids.tolist() + [list(new_pages[1].tolist())]
    owner, S = [0, 0, 0, 0, 1], 5
    lines = [[list(held[l][o][i] for i in range(3)) for o in owner] for l in range(layers)]
    length = [lengths[o] for o in owner]
    for step in range(9):
        for r, n in zip(rows, length):
            if n % P == 0:
                r += lv.luvc_kv_take(refs, 1).tolist()
        tab = torch.full((S, 6), -1, dtype=torch.int32)
        for i, r in enumerate(rows):
            tab[i, :len(r)] = torch.tensor(r, dtype=torch.int32)
        tab = tab.cuda()
        at = torch.tensor(length, dtype=torch.int32).cuda()
        length = [n + 1 for n in length]
        now = torch.tensor(length, dtype=torch.int32).cuda()
        h = torch.randn(S, model, device="cuda")
        for l in range(layers):
            qkv = (h @ w[l]).to(dt).view(S, Hq + 2 * H, D)
            q, nk, nv = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
            lv.luvc_kv_write(cache, l, nk, nv, at, tab)
            got = to_host_f64(lv.luvc_kv_attend(cache, l, q, tab, now, max_tokens=6 * P, enhance=True))
            for i in range(S):
                lines[l][i] = [np.concatenate([a, b]) for a, b in zip(lines[l][i], (to_host_f64(nk[i:i + 1]), to_host_f64(nv[i:i + 1]), np.ones(1, int)))]
                kk, vv, ss = lines[l][i]
                n = len(ss)
                want, bulk, steep, live = ref.attend(to_host_f64(q[i:i + 1]), kk.transpose(1, 0, 2)[None], vv.transpose(1, 0, 2)[None], ss[None],
                                                     np.zeros((1, 1), int), [n], D ** -0.5, True)
                assert (np.abs(got[i:i + 1] - want) <= ref.tolerance(want, bulk, steep, live, D, dtype)).all(), (step, l, i)

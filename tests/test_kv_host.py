"""Host side of the paged key-value cache: counting of pages and refusals.  No GPU: every call fails its checks, or launches nothing."""
import ctypes
import random

import pytest
import torch

from paper_2512_09010_amd import binding as lv
from paper_2512_09010_amd import build as lvbuild

FAKE = ctypes.c_void_p(0x1000)          # never dereferenced


@pytest.fixture(scope="module")
def L():
    lvbuild.build(force=False)
    return lv.lib()


def cache(**kw):
    c = dict(k=0x10000, v=0x20000, sizes=0x30000, layer_stride=1 << 30, n_layers=2, n_pages=10, n_heads=4, page_tokens=16, D=64, dtype=lv.LUVC_BF16)
    c.update(kw)
    return lv.LuvcKvCache(*(c[f] for f, _ in lv.LuvcKvCache._fields_))


BAD_CACHES = [(dict(k=None), lv.LUVC_ERR_INVALID_ARG), (dict(v=None), lv.LUVC_ERR_INVALID_ARG), (dict(dtype=7), lv.LUVC_ERR_INVALID_ARG),
              (dict(n_layers=0), lv.LUVC_ERR_INVALID_ARG), (dict(n_pages=0), lv.LUVC_ERR_INVALID_ARG), (dict(n_heads=0), lv.LUVC_ERR_INVALID_ARG),
              (dict(D=0), lv.LUVC_ERR_INVALID_ARG), (dict(page_tokens=0), lv.LUVC_ERR_INVALID_ARG), (dict(k=0x10001), lv.LUVC_ERR_INVALID_ARG),
              (dict(dtype=lv.LUVC_F32, v=0x10002), lv.LUVC_ERR_INVALID_ARG), (dict(sizes=0x30002), lv.LUVC_ERR_INVALID_ARG),
              (dict(layer_stride=10 * 4 * 16 * 64 - 1), lv.LUVC_ERR_INVALID_ARG),
              (dict(page_tokens=24), lv.LUVC_ERR_UNSUPPORTED), (dict(page_tokens=8), lv.LUVC_ERR_UNSUPPORTED), (dict(page_tokens=2048), lv.LUVC_ERR_UNSUPPORTED),
              (dict(D=257), lv.LUVC_ERR_UNSUPPORTED), (dict(n_heads=1025), lv.LUVC_ERR_UNSUPPORTED)]


def i32(*v):
    return (ctypes.c_int32 * max(1, len(v)))(*v)


def calls(L, c):
    """Every entry point on cache c with arguments that pass wherever the cache does, so far as that launches nothing."""
    p = None if c is None else ctypes.byref(c)
    return [L.luvc_kv_write(p, 0, FAKE, 256, FAKE, 256, None, 0, None, FAKE, FAKE, 1, 1, None),
            L.luvc_kv_attend(p, 0, FAKE, 512, 8, 1, FAKE, 1, FAKE, 16, None, 0, FAKE, 512, None, 0, None),
            L.luvc_kv_compact(p, 1, i32(0), i32(0), i32(0), i32(0), None, FAKE, 1, FAKE, 1, None),
            L.luvc_kv_copy_pages(p, i32(), i32(), 0, None)]


@pytest.mark.parametrize("fields, status", BAD_CACHES, ids=lambda x: str(x))
def test_bad_caches_are_refused(L, fields, status):
    refs = i32(*[1] * 10)
    c = cache(**fields)
    assert calls(L, c) == [status] * 4, lv.last_error()
    assert L.luvc_kv_fork(ctypes.byref(c), refs, i32(0), 16, 1, i32(0), None) == status
    assert list(refs) == [1] * 10


def test_no_cache_and_good_cache(L):
    assert calls(L, None) == [lv.LUVC_ERR_INVALID_ARG] * 4
    assert calls(L, cache()) == [lv.LUVC_OK, lv.LUVC_ERR_WORKSPACE, lv.LUVC_OK, lv.LUVC_OK]
    assert calls(L, cache(sizes=None, dtype=lv.LUVC_F32))[1] == lv.LUVC_ERR_WORKSPACE


def test_write_refusals(L):
    c = cache()
    w = lambda **kw: L.luvc_kv_write(ctypes.byref(kw.get("c", c)), kw.get("layer", 0), kw.get("k", FAKE), kw.get("ks", 256), kw.get("v", FAKE), kw.get("vs", 256),
                                     kw.get("sizes"), kw.get("tokens", 3), None, kw.get("pos", FAKE), kw.get("table", FAKE), kw.get("seqs", 1), kw.get("mp", 1), None)
    for bad in (dict(layer=-1), dict(layer=2), dict(k=None), dict(v=None), dict(pos=None), dict(table=None), dict(ks=255), dict(vs=255),
                dict(tokens=-1), dict(seqs=0), dict(mp=0), dict(k=ctypes.c_void_p(0x1001)), dict(c=cache(sizes=None), sizes=FAKE)):
        assert w(**bad) == lv.LUVC_ERR_INVALID_ARG, bad
        assert lv.last_error()
    assert w(tokens=1 << 25) == lv.LUVC_ERR_UNSUPPORTED
    assert w(tokens=0, k=None, v=None, pos=None, table=None) == lv.LUVC_OK


def test_attend_refusals_and_workspace(L):
    c = cache()
    nan, one = ctypes.c_double(float("nan")), ctypes.c_double(1.0)
    a = lambda **kw: L.luvc_kv_attend(ctypes.byref(kw.get("c", c)), kw.get("layer", 0), kw.get("q", FAKE), kw.get("qs", 512), kw.get("hq", 8), kw.get("S", 2),
                                      kw.get("table", FAKE), kw.get("mp", 4), kw.get("lengths", FAKE), kw.get("most", 64), kw.get("scale"), kw.get("enhance", 0),
                                      kw.get("out", FAKE), kw.get("os", 512), kw.get("ws"), kw.get("wsb", 0), None)
    for bad in (dict(layer=2), dict(q=None), dict(table=None), dict(lengths=None), dict(out=None), dict(hq=0), dict(hq=6), dict(S=0), dict(mp=0), dict(most=0),
                dict(qs=511), dict(os=511), dict(q=ctypes.c_void_p(0x1001)), dict(out=ctypes.c_void_p(0x1001)), dict(scale=ctypes.byref(nan)),
                dict(c=cache(sizes=None), enhance=1)):
        assert a(**bad) == lv.LUVC_ERR_INVALID_ARG, bad
        assert lv.last_error()
    for beyond in (dict(S=1 << 21), dict(S=1 << 19), dict(most=1 << 30)):
        assert a(**beyond) == lv.LUVC_ERR_UNSUPPORTED, beyond
    need = L.luvc_kv_attend_workspace_bytes(ctypes.byref(c), 2, 8, 64)
    assert need >= 256 and need % 256 == 0
    assert a(scale=ctypes.byref(one)) == lv.LUVC_ERR_WORKSPACE
    assert a(ws=ctypes.c_void_p(0x10000), wsb=need - 1) == lv.LUVC_ERR_WORKSPACE
    assert a(ws=ctypes.c_void_p(0x10008), wsb=need + 256) == lv.LUVC_ERR_WORKSPACE
    q = lambda *args, **kw: L.luvc_kv_attend_workspace_bytes(ctypes.byref(cache(**kw)), *args)
    assert q(2, 8, 64, k=None, v=None, sizes=None) == need                  # of the pool itself nothing is looked at
    assert q(0, 8, 64) == q(2, 6, 64) == q(2, 8, 0) == q(2, 8, 64, D=300) == q(2, 8, 64, dtype=9) == 0
    assert L.luvc_kv_attend_workspace_bytes(None, 2, 8, 64) == 0


@pytest.mark.parametrize("hq, h, D, dtype", [(32, 8, 128, lv.LUVC_BF16), (28, 4, 128, lv.LUVC_BF16), (4, 1, 64, lv.LUVC_F32), (64, 64, 96, lv.LUVC_BF16), (40, 1, 256, lv.LUVC_F32),
                                             (1024, 1024, 8, lv.LUVC_BF16)])
def test_a_workspace_serves_fewer_sequences_and_shorter_ones(L, hq, h, D, dtype):
    c = cache(n_heads=h, D=D, dtype=dtype)
    seqs = [1, 2, 3, 7, 8, 16, 60, 64, 65, 128, 255, 256, 257, 500, 1023, 1024, 1025, 1100, 2048, 4000]
    tokens = [1, 16, 63, 64, 65, 127, 128, 129, 300, 512, 513, 1000, 2048, 4096, 4097, 5000, 8200, 30000, 65537, 10 ** 5, 10 ** 6, 2 ** 30 - 1]
    need = [[L.luvc_kv_attend_workspace_bytes(ctypes.byref(c), n, hq, t) for t in tokens] for n in seqs]
    for a, b in zip(need, need[1:]):
        assert all(0 < x <= y for x, y in zip(a, b) if y)   # 0: too many sequences
    for row in need:
        assert all(x <= y for x, y in zip(row, row[1:]))


def test_attend_refuses_scales_beyond_fp32(L):
    for v in (3e38, -3e38, 1e39, float("inf"), float("-inf")):
        s = ctypes.c_double(v)
        assert L.luvc_kv_attend(ctypes.byref(cache()), 0, FAKE, 512, 8, 2, FAKE, 4, FAKE, 64, ctypes.byref(s), 0, FAKE, 512, None, 0, None) == lv.LUVC_ERR_INVALID_ARG
        assert "scale" in lv.last_error()


def test_compact_refusals(L):
    c = cache()
    def call(lengths, first, span, keep, kept=FAKE, mi=4, mo=4, tin=FAKE, tout=FAKE):
        return L.luvc_kv_compact(ctypes.byref(c), len(lengths), i32(*lengths), i32(*first), i32(*span), i32(*keep), kept, tin, mi, tout, mo, None)
    for bad in (([20], [-1], [4], [2]), ([20], [0], [-1], [0]), ([20], [0], [4], [5]), ([20], [0], [4], [-1]), ([20], [17], [4], [2]), ([65], [0], [64], [2]),
                ([50, -1], [0, 0], [4, 0], [2, 0]), ([2 ** 31 - 1], [2 ** 31 - 1], [4], [2])):
        assert call(*bad) == lv.LUVC_ERR_INVALID_ARG, bad
    assert call([60], [0], [10], [9], mo=3) == lv.LUVC_ERR_INVALID_ARG                     # 59 tokens, 48 places
    assert call([20], [0], [4], [2], kept=None) == lv.LUVC_ERR_INVALID_ARG
    assert call([20], [0], [4], [2], tin=None) == lv.LUVC_ERR_INVALID_ARG
    assert call([20], [0], [4], [2], tout=None) == lv.LUVC_ERR_INVALID_ARG
    assert call([20], [0], [4], [2], mi=0) == lv.LUVC_ERR_INVALID_ARG
    assert call([1 << 29], [0], [4], [2], mi=1 << 26, mo=1 << 26) == lv.LUVC_ERR_UNSUPPORTED
    assert call([4], [0], [4], [0], kept=None) == lv.LUVC_OK                               # nothing survives: nothing is launched
    assert L.luvc_kv_compact(ctypes.byref(c), 0, i32(), i32(), i32(), i32(), None, FAKE, 1, FAKE, 1, None) == lv.LUVC_ERR_INVALID_ARG


def test_copy_refusals(L):
    c = cache()
    call = lambda src, dst: L.luvc_kv_copy_pages(ctypes.byref(c), i32(*src), i32(*dst), len(src), None)
    for src, dst in (([0], [10]), ([-1], [2]), ([10], [2]), ([0], [-1]), ([3], [3]), ([0, 1], [2, 2]), ([0, 2], [2, 3]), ([0, 1], [5, 0])):
        assert call(src, dst) == lv.LUVC_ERR_INVALID_ARG, (src, dst)
    assert L.luvc_kv_copy_pages(ctypes.byref(c), None, i32(1), 1, None) == lv.LUVC_ERR_INVALID_ARG
    assert L.luvc_kv_copy_pages(ctypes.byref(c), i32(1), i32(2), -1, None) == lv.LUVC_ERR_INVALID_ARG


def test_fork_of_full_pages_is_counting_only(L):
    """No partial page: nothing is copied, so the call runs without a GPU."""
    c = cache()
    refs, children = i32(*[1, 0, 2, 1] + [0] * 6), i32(*[-7] * 6)
    assert L.luvc_kv_fork(ctypes.byref(c), refs, i32(3, 2), 32, 3, children, None) == lv.LUVC_OK
    assert list(children) == [3, 2] * 3 and list(refs) == [1, 0, 5, 4] + [0] * 6


def test_fork_refusals_leave_the_counts(L):
    c = cache()
    start = [1, 0, 2, 1] + [1] * 5 + [0]
    refs = i32(*start)
    call = lambda pages, length, n: L.luvc_kv_fork(ctypes.byref(c), refs, i32(*pages), length, n, i32(*[0] * 100), None)
    assert call([0, 2], 0, 1) == lv.LUVC_ERR_INVALID_ARG
    assert call([0, 2], 20, 0) == lv.LUVC_ERR_INVALID_ARG
    assert call([0, 1], 20, 1) == lv.LUVC_ERR_INVALID_ARG                   # page 1 is free
    assert call([0, -1], 20, 1) == lv.LUVC_ERR_INVALID_ARG
    assert call([0, 10], 20, 1) == lv.LUVC_ERR_INVALID_ARG
    assert call([0] * 11, 161, 1) == lv.LUVC_ERR_INVALID_ARG                # more pages than there are
    assert call([0, 2], 20, 3) == lv.LUVC_ERR_WORKSPACE                     # three copies, two free pages
    assert list(refs) == start
    refs[0] = 2 ** 31 - 1
    assert call([0], 16, 1) == lv.LUVC_ERR_INVALID_ARG and refs[0] == 2 ** 31 - 1
    assert L.luvc_kv_fork(ctypes.byref(c), None, i32(0), 16, 1, i32(0), None) == lv.LUVC_ERR_INVALID_ARG


def test_take_and_release_against_a_model(L):
    rng = random.Random(5)
    refs, model, held = torch.zeros(37, dtype=torch.int32), [0] * 37, []
    for step in range(400):
        n = rng.randint(0, 9)
        if rng.random() < 0.55:
            free = [p for p in range(37) if model[p] == 0]
            if n > len(free):
                with pytest.raises(lv.LuvcError) as e:
                    lv.luvc_kv_take(refs, n)
                assert e.value.status == lv.LUVC_ERR_WORKSPACE
            else:
                got = lv.luvc_kv_take(refs, n).tolist()
                assert got == free[:n]
                for p in got:
                    model[p] += 1
                held += got
        else:
            rng.shuffle(held)
            back, held = held[:n], held[n:]
            lv.luvc_kv_release(refs, back)
            for p in back:
                model[p] -= 1
        assert refs.tolist() == model


@pytest.mark.parametrize("n_pages", [1, 15, 16, 17, 33, 1000, 4096])
def test_take_finds_the_last_free_pages(L, n_pages):
    rng = random.Random(n_pages)
    free = sorted(rng.sample(range(n_pages), min(n_pages, 5)) + ([n_pages - 1] if n_pages > 5 else []))
    free = sorted(set(free))
    refs = torch.ones(n_pages, dtype=torch.int32)
    refs[free] = 0
    with pytest.raises(lv.LuvcError):
        lv.luvc_kv_take(refs, len(free) + 1)
    assert lv.luvc_kv_take(refs, len(free)).tolist() == free and bool((refs == 1).all())


@pytest.mark.parametrize("pairs", [1, 2, 16, 17, 200])
def test_copy_refusals_at_any_place(L, pairs):
    c = cache(n_pages=500, layer_stride=1 << 30)
    for bad in range(0, pairs, max(1, pairs // 7)):
        src, dst = [i // 2 for i in range(pairs)], [200 + i for i in range(pairs)]
        for page in {src[-1], src[bad], dst[bad - 1] if pairs > 1 else src[0]}:
            broken = list(dst)
            broken[bad] = page
            assert L.luvc_kv_copy_pages(ctypes.byref(c), i32(*src), i32(*broken), pairs, None) == lv.LUVC_ERR_INVALID_ARG, (pairs, bad, page)
            assert "written to" in lv.last_error()


def test_release_refusals_leave_the_counts(L):
    refs = torch.tensor([2, 1, 0], dtype=torch.int32)
    for bad in ([0, 0, 0], [1, 2], [0, -1], [0, 3], [1, 1]):
        with pytest.raises(lv.LuvcError) as e:
            lv.luvc_kv_release(refs, bad)
        assert e.value.status == lv.LUVC_ERR_INVALID_ARG and refs.tolist() == [2, 1, 0]
    lv.luvc_kv_release(refs, [0, 1, 0])
    assert refs.tolist() == [0, 0, 0]
    for bad in (-1,):
        with pytest.raises(lv.LuvcError):
            lv.luvc_kv_take(refs, bad)
    assert lv.luvc_kv_take(refs, 0).numel() == 0
    with pytest.raises(AssertionError):
        lv.luvc_kv_take(refs.long(), 1)

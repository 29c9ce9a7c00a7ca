"""The paged key-value cache that the compressed tokens end in, as cases to be timed and compared.

Five kinds of case, each one pass through an operator the way a serving program calls it (buffers allocated once and reused,
everything on the current stream):

``attend``   attention of one new token per sequence over its pages; with the sizes of merged tokens, Eq. 3 of the paper,
             O = A (V + log s), and tokens of size 0 that take no part.
``write``    keys and values of new tokens, slices of one projection's output, go to their places in the pages.
``compact``  after a stage of the spectrum pruning: the kept visual tokens close up, the text around them stays.
``copy``     whole pages, all layers.
``fork``     further continuations of one prompt share its full pages and get a page of their own for the last, partial
             one; at the end they are released.

A pool holds ``[layers, pages, heads, page_tokens, D]`` keys and as many values, a table the pages of every sequence.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}
_NO_PAGE = -1                                               # entry of a table behind a sequence's last page


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # one fp32 image of 144 merged tokens and a short question, 4096 channels in 32 heads: one token's latency
        _attend("attend_image_208_f32", 1, 208, 208, 32, 32, 128, "f32", 16, "none", 0.0),
        # the batch of eight dynamic-resolution images: 1024 merged tokens each with their sizes, grouped heads of 3584 channels
        _attend("attend_images8_1100", 8, 1040, 1160, 28, 4, 128, "bf16", 16, "enhance", 0.0),
        # one long video with OIM off: a single sequence, which has to be split to fill the chip
        _attend("attend_video_100000", 1, 100001, 100001, 28, 4, 128, "bf16", 64, "none", 0.0),
        # a full serving batch, prompts from one token to whole documents, some tokens pruned in place
        _attend("attend_serving64_8200", 64, 1, 8200, 32, 8, 128, "bf16", 16, "mask", 0.125),
        # a decoding step's new tokens
        _write("write_step64", 64, 1, 1, 1500, 32, 8, 128, "bf16", 16, False),
        # the prompts of four videos, 8192 tokens each and some text, with the sizes of the merged tokens
        _write("write_prompts4_8300", 4, 8250, 8300, 0, 28, 4, 128, "bf16", 16, True),
        # a stage on one image whose token count has no convenient factors
        _compact("compact_image_729_f32", 1, 729, 729, 35, 21, 0.25, 2, 8, 128, "f32", 16, False),
        # a stage on four videos of 8192 tokens, in the layers below it
        _compact("compact_videos4_8192", 4, 8192, 8192, 40, 100, 0.10, 8, 4, 128, "bf16", 16, True),
        # a handful of pages of one layer, and a large part of a pool when sequences move
        _copy("copy_pages_8", 8, 1, 8, 128, "bf16", 16, False),
        _copy("copy_pages_1024", 1024, 8, 8, 128, "bf16", 16, True),
        # a second answer to one question, and a wide sampling of continuations in all layers
        _fork("fork_2_of_1000", 1000, 2, 2, 8, 128, "bf16", 16, False),
        _fork("fork_32_of_8200", 8200, 32, 28, 4, 128, "bf16", 64, True),
    ]


def draw(rng):
    costs, moved = {}, {}
    for case in listed():
        costs[case["kind"]] = max(costs.get(case["kind"], 0), _cost(case))
        moved[case["kind"]] = max(moved.get(case["kind"], 0), work(case)["bytes"])
    while True:
        kind = rng.choice(["attend", "attend", "attend", "attend", "write", "compact", "copy", "fork"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        D = rng.choice([32, 64, 64, 80, 96, 112, 128, 128, 128, 128, 192, 256, rng.randint(1, 256)])
        page = rng.choice([16, 16, 16, 32, 64, 128, 256])
        heads = rng.choice([1, 2, 4, 8, 8, rng.randint(1, 16)])
        q_heads = heads * rng.choice([1, 1, 2, 4, 7, 8, 12, 16, 32])
        sized = rng.random() < 0.5
        if kind == "attend":
            a, b = _log_int(rng, 1, 120000), _log_int(rng, 1, 120000)
            sizes = rng.choice(["none", "none", "mask", "enhance"])
            short = 0 if rng.random() < 0.1 else min(a, b)
            seqs = _log_int(rng, 1, 128)
            case = _attend("", seqs, short if seqs > 1 else max(a, b), max(a, b), q_heads, heads, D, dtype, page, sizes,
                           0.0 if sizes == "none" else round(rng.choice([0.0, rng.random()]), 3))
        elif kind == "write":
            a, b = _log_int(rng, 1, 16384), _log_int(rng, 1, 16384)
            if rng.random() < 0.4:
                a = b = 1
            case = _write("", _log_int(rng, 1, 128), min(a, b), max(a, b), rng.randint(0, 5000), q_heads, heads, D, dtype, page, sized)
        elif kind == "compact":
            a, b = _log_int(rng, 48, 8192), _log_int(rng, 48, 8192)
            seqs = _log_int(rng, 1, 100)
            case = _compact("", seqs, min(a, b) if seqs > 1 else max(a, b), max(a, b), rng.randint(0, 300), rng.randint(0, 300),
                            round(math.exp(rng.uniform(math.log(0.05), 0.0)), 3), _log_int(rng, 1, 28), heads, D, dtype, page, sized)
        elif kind == "copy":
            case = _copy("", _log_int(rng, 1, 2000), _log_int(rng, 1, 28), heads, D, dtype, page, sized)
        else:
            case = _fork("", _log_int(rng, 1, 16384), _log_int(rng, 1, 32), _log_int(rng, 1, 28), heads, D, dtype, page, sized)
        if _cost(case) <= costs[kind] and work(case)["bytes"] <= moved[kind]:
            del case["name"]
            return case


def _attend(name, seqs, shortest, longest, q_heads, heads, D, dtype, page, sizes, dead):
    """`sizes`: "none", "mask" (only tokens of size 1 and more take part) or "enhance" (and V + log s); `dead`: share of size 0."""
    return dict(name=name, kind="attend", seqs=seqs, shortest=shortest, longest=longest, q_heads=q_heads, heads=heads, D=D, dtype=dtype,
                page=page, sizes=sizes, dead=dead)


def _write(name, seqs, shortest, longest, past, q_heads, heads, D, dtype, page, sized):
    """`past` tokens of every sequence are in the cache already."""
    return dict(name=name, kind="write", seqs=seqs, shortest=shortest, longest=longest, past=past, q_heads=q_heads, heads=heads, D=D,
                dtype=dtype, page=page, sized=sized)


def _compact(name, seqs, shortest, longest, before, after, ratio, layers, heads, D, dtype, page, sized):
    """`before` text tokens, then visual tokens of which `ratio` are kept, then `after` text tokens."""
    return dict(name=name, kind="compact", seqs=seqs, shortest=shortest, longest=longest, before=before, after=after, ratio=ratio,
                layers=layers, heads=heads, D=D, dtype=dtype, page=page, sized=sized)


def _copy(name, pages, layers, heads, D, dtype, page, sized):
    return dict(name=name, kind="copy", pages=pages, layers=layers, heads=heads, D=D, dtype=dtype, page=page, sized=sized)


def _fork(name, length, children, layers, heads, D, dtype, page, sized):
    return dict(name=name, kind="fork", length=length, children=children, layers=layers, heads=heads, D=D, dtype=dtype, page=page, sized=sized)


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _lengths(case):
    """Tokens per sequence: the case's shortest and longest, the others spread between them on a logarithmic scale."""
    n, lo, hi = case["seqs"], case["shortest"], case["longest"]
    if n == 1 or lo == hi:
        return [hi] * n
    rng = random.Random("%d %d %d" % (n, lo, hi))
    out = [lo, hi] + [_log_int(rng, max(lo, 1), hi) for _ in range(n - 2)]
    rng.shuffle(out)
    return out


def _pages_of(case, tokens):
    return -(-tokens // case["page"])


def _keeps(case, lengths):
    return [min(n, max(1, int(math.floor(case["ratio"] * n + 0.5)))) for n in lengths]


def _dead_count(case, n):
    return min(n, int(round(case["dead"] * n)))


def _cost(case):
    """Bytes that a case occupies: cache, and where the plain form pads sequences to the longest, those too."""
    token = 2 * case["heads"] * case["D"] * _BYTES[case["dtype"]]
    if case["kind"] == "attend":
        return max(case["seqs"] * case["longest"] * token, case["seqs"] * case["longest"] * case["q_heads"] * 64)
    if case["kind"] == "write":
        return sum(_pages_of(case, case["past"] + n) for n in _lengths(case)) * case["page"] * token + case["seqs"] * case["longest"] * case["q_heads"] * case["D"]
    if case["kind"] == "compact":
        lengths = _lengths(case)
        pages = sum(_pages_of(case, case["before"] + n + case["after"]) + _pages_of(case, case["before"] + k + case["after"])
                    for n, k in zip(lengths, _keeps(case, lengths)))
        return pages * case["page"] * token * case["layers"]
    if case["kind"] == "copy":
        return 2 * case["pages"] * case["page"] * token * case["layers"]
    return (_pages_of(case, case["length"]) + case["children"]) * case["page"] * token * case["layers"]


def work(case):
    e, heads, D = _BYTES[case["dtype"]], case["heads"], case["D"]
    token = 2 * heads * D * e
    if case["kind"] == "attend":
        lengths = _lengths(case)
        live = sum(n - _dead_count(case, n) for n in lengths)
        sized = 0 if case["sizes"] == "none" else 4 * sum(lengths)
        table = 4 * sum(_pages_of(case, n) for n in lengths) + 4 * len(lengths)
        return {"bytes": live * token + sized + table + 2 * len(lengths) * case["q_heads"] * D * e, "flops": 4 * live * case["q_heads"] * D}
    if case["kind"] == "write":
        n = sum(_lengths(case))
        return {"bytes": n * (2 * token + 4 + (8 if case["sized"] else 0)), "flops": 0}
    if case["kind"] == "compact":
        # the pages of the text in front that are full stay where they are
        stay = case["before"] // case["page"] * case["page"]
        moved = sum(case["before"] + k + case["after"] - stay for k in _keeps(case, _lengths(case)))
        return {"bytes": moved * (2 * token * case["layers"] + (8 if case["sized"] else 0)) + 4 * sum(_keeps(case, _lengths(case))), "flops": 0}
    sized = 8 * case["page"] if case["sized"] else 0
    if case["kind"] == "copy":
        return {"bytes": case["pages"] * (case["page"] * 2 * token * case["layers"] + sized), "flops": 0}
    copied = case["children"] if case["length"] % case["page"] else 0
    table = 4 * _pages_of(case, case["length"]) * (1 + case["children"])
    # the children read one page between them
    rows = case["length"] % case["page"]
    return {"bytes": (copied + (1 if copied else 0)) * (rows * token * case["layers"] + (4 * rows if case["sized"] else 0)) + table, "flops": 0}


# ------------------------------------------------------------------------------------------------ inputs

def _inputs(case, seed):
    """What the program has in hand: pool, tables, new tokens.  The same for all forms of an operator."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = random.Random(seed)
    dt, dev = _TORCH[case["dtype"]], "cuda"
    randn = lambda *shape: torch.randn(shape, generator=gen, dtype=dt, device=dev)
    randint = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=gen, dtype=torch.int32, device=dev)
    kind, layers = case["kind"], case.get("layers", 1)
    if kind in ("copy", "fork"):
        used = case["pages"] if kind == "copy" else _pages_of(case, case["length"])
        extra = used if kind == "copy" else case["children"]
        n_pages = used + extra + 3
        order = list(range(n_pages))
        host.shuffle(order)
        s = {"pages": order[:used]}
        if kind == "copy":
            s["src"] = torch.tensor(order[:used], dtype=torch.int32)
            s["dst"] = torch.tensor(order[used:used + extra], dtype=torch.int32)
        else:
            s["refs"] = torch.zeros(n_pages, dtype=torch.int32)
            s["refs"][order[:used]] = 1
            s["refs"][order[used:used + 2]] = 1                 # two pages that others hold
            s["parent"] = torch.tensor(order[:used], dtype=torch.int32)
    else:
        lengths = _lengths(case)
        s = {"lengths": lengths}
        need = lengths
        if kind == "write":
            need = [case["past"] + n for n in lengths]
        if kind == "compact":
            keeps = _keeps(case, lengths)
            need = [case["before"] + n + case["after"] for n in lengths]
            after = [case["before"] + k + case["after"] for k in keeps]
        n_pages = sum(_pages_of(case, n) for n in need) + 3
        if kind == "compact":
            n_pages += sum(_pages_of(case, n) for n in after)
        order = list(range(n_pages))
        host.shuffle(order)

        def table(tokens, front=None):
            most = max(1, max(_pages_of(case, n) for n in tokens))
            rows = []
            for i, n in enumerate(tokens):
                row = list(front[i]) if front else []
                while len(row) < _pages_of(case, n):
                    row.append(order.pop())
                rows.append(row + [_NO_PAGE] * (most - len(row)))
            return rows

        rows = table(need)
        s["rows"], s["table"] = rows, torch.tensor(rows, dtype=torch.int32, device=dev)
        if kind == "compact":
            stay = case["before"] // case["page"]
            out_rows = table(after, [r[:stay] for r in rows])
            s["out_rows"], s["table_out"] = out_rows, torch.tensor(out_rows, dtype=torch.int32, device=dev)
            s["need"], s["keeps"], s["after"] = need, keeps, after
            s["kept_lists"] = [sorted(host.sample(range(n), k)) for n, k in zip(lengths, keeps)]
            s["kept_idx"] = torch.tensor([i for l in s["kept_lists"] for i in l], dtype=torch.int32, device=dev)
    shape = (layers, n_pages, case["heads"], case["page"], case["D"])
    s["k"], s["v"] = randn(*shape), randn(*shape)
    sized = case["sized"] if kind != "attend" else case["sizes"] != "none"
    s["sizes"] = randint(1, 17, n_pages, case["page"]) if sized else None
    if kind == "attend":
        s["device_lengths"] = torch.tensor(lengths, dtype=torch.int32, device=dev)
        # logits of a few units: attention that picks tokens out, as trained heads do
        s["q"] = randn(len(lengths), case["q_heads"], case["D"]) * 2
        if case["dead"] > 0.0:
            for row, n in zip(rows, lengths):
                if n:
                    at = torch.randperm(n, generator=gen, device=dev)[:_dead_count(case, n)]
                    pages = torch.tensor(row, device=dev)[at // case["page"]]
                    s["sizes"][pages, at % case["page"]] = 0
    if kind == "write":
        T = sum(lengths)
        qkv = randn(T, case["q_heads"] + 2 * case["heads"], case["D"])
        s["new_k"], s["new_v"] = qkv[:, case["q_heads"]:case["q_heads"] + case["heads"]], qkv[:, case["q_heads"] + case["heads"]:]
        s["new_sizes"] = randint(0, 17, T) if case["sized"] else None
        one_each = all(n == 1 for n in lengths)
        s["seq"] = None if one_each else torch.tensor([i for i, n in enumerate(lengths) for _ in range(n)], dtype=torch.int32, device=dev)
        s["pos"] = torch.tensor([case["past"] + j for n in lengths for j in range(n)], dtype=torch.int32, device=dev)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2512_09010_amd import binding as lv
        s["lv"] = lv
        s["cache"] = lv.KvCache(s["k"], s["v"], s["sizes"])
        if case["kind"] == "attend":
            s["most"] = max(1, max(s["lengths"]))
            need = lv.luvc_kv_attend_workspace_bytes(s["cache"], len(s["lengths"]), case["q_heads"], s["most"])
            s["workspace"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
            s["out"] = torch.empty_like(s["q"])
    return s


# ------------------------------------------------------------------------------------------------ passes

def run(state):
    return (_run_own if own else _run_plain)[state["case"]["kind"]](state)


def _pool(s):
    return (s["k"], s["v"]) if s["sizes"] is None else (s["k"], s["v"], s["sizes"])


def _own_attend(s):
    c = s["case"]
    return s["lv"].luvc_kv_attend(s["cache"], 0, s["q"], s["table"], s["device_lengths"], max_tokens=s["most"],
                                  enhance=c["sizes"] == "enhance", workspace=s["workspace"], out=s["out"])


def _own_write(s):
    s["lv"].luvc_kv_write(s["cache"], 0, s["new_k"], s["new_v"], s["pos"], s["table"], seq=s["seq"], sizes=s["new_sizes"])
    return _pool(s)


def _own_compact(s):
    c, n = s["case"], len(s["lengths"])
    after = s["lv"].luvc_kv_compact(s["cache"], s["kept_idx"], s["need"], [c["before"]] * n, s["lengths"], s["keeps"], s["table"], s["table_out"])
    return (torch.tensor(after, dtype=torch.int32),) + _pool(s)


def _own_copy(s):
    s["lv"].luvc_kv_copy_pages(s["cache"], s["src"], s["dst"])
    return _pool(s)


def _own_fork(s):
    c = s["case"]
    children = s["lv"].luvc_kv_fork(s["cache"], s["refs"], s["parent"], c["length"], c["children"])
    s["lv"].luvc_kv_release(s["refs"], children)
    return (children, s["refs"]) + _pool(s)


def _plain_attend(s):
    c, q, table = s["case"], s["q"], s["table"].long()
    S, P, heads, D = len(s["lengths"]), c["page"], c["heads"], c["D"]
    L = table.shape[1] * P
    pages = table.clamp(min=0)
    here = torch.arange(L, device=q.device) < s["device_lengths"][:, None]                     # [S, L]
    if s["sizes"] is not None:
        size = s["sizes"][pages].view(S, L)
        here = here & (size >= 1)
    k = s["k"][0][pages].float().permute(0, 2, 1, 3, 4).reshape(S, heads, L, D)
    v = s["v"][0][pages].float().permute(0, 2, 1, 3, 4).reshape(S, heads, L, D)
    if c["sizes"] == "enhance":
        v = v + torch.log(size.clamp(min=1).float())[:, None, :, None]
    v = torch.where(here[:, None, :, None], v, 0.0)
    logits = torch.matmul(q.float().view(S, heads, -1, D), k.transpose(2, 3).contiguous()) / math.sqrt(D)
    logits = torch.where(here[:, None, None, :], logits, -torch.inf)
    most = logits.amax(dim=-1, keepdim=True)
    p = torch.exp(logits - torch.where(most > -torch.inf, most, 0.0))
    total = p.sum(dim=-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    return out.view(S, -1, D).to(q.dtype)


def _plain_write(s):
    P = s["case"]["page"]
    pos = s["pos"].long()
    seq = torch.arange(pos.numel(), device=pos.device) if s["seq"] is None else s["seq"].long()
    page = s["table"].long()[seq, pos // P]
    s["k"][0][page, :, pos % P] = s["new_k"]
    s["v"][0][page, :, pos % P] = s["new_v"]
    if s["sizes"] is not None:
        s["sizes"][page, pos % P] = s["new_sizes"]
    return _pool(s)


def _plain_compact(s):
    c, P, dev = s["case"], s["case"]["page"], s["k"].device
    src, dst, at = [], [], 0
    for i, (n, keep, total) in enumerate(zip(s["lengths"], s["keeps"], s["need"])):
        first = c["before"]
        old = torch.cat([torch.arange(first, device=dev), first + s["kept_idx"][at:at + keep].long(), torch.arange(first + n, total, device=dev)])
        new = torch.arange(old.numel(), device=dev)
        at += keep
        src.append(s["table"][i].long()[old // P] * P + old % P)
        dst.append(s["table_out"][i].long()[new // P] * P + new % P)
    src, dst = torch.cat(src), torch.cat(dst)
    for pool in (s["k"], s["v"]):
        pool[:, dst // P, :, dst % P] = pool[:, src // P, :, src % P]
    if s["sizes"] is not None:
        s["sizes"][dst // P, dst % P] = s["sizes"][src // P, src % P]
    return (torch.tensor([t - n + k for t, n, k in zip(s["need"], s["lengths"], s["keeps"])], dtype=torch.int32),) + _pool(s)


def _plain_copy(s):
    src, dst = s["src"].long().to(s["k"].device), s["dst"].long().to(s["k"].device)
    for pool in (s["k"], s["v"]):
        pool[:, dst] = pool[:, src]
    if s["sizes"] is not None:
        s["sizes"][dst] = s["sizes"][src]
    return _pool(s)


def _plain_fork(s):
    c, refs, parent = s["case"], s["refs"], s["parent"].long()
    children = parent.repeat(c["children"], 1)
    full = parent[:c["length"] // c["page"]]
    refs[full] += c["children"]
    if full.numel() < parent.numel():
        new = torch.nonzero(refs == 0)[:c["children"], 0]
        refs[new] = 1
        children[:, -1] = new
        dst, src = new.to(s["k"].device), int(parent[-1])
        rows = c["length"] % c["page"]
        for pool in (s["k"], s["v"]):
            pool[:, dst, :, :rows] = pool[:, src, :, :rows][:, None]
        if s["sizes"] is not None:
            s["sizes"][dst, :rows] = s["sizes"][src, :rows]
        refs[new] -= 1
    refs[full] -= c["children"]
    return (children.to(torch.int32), refs) + _pool(s)


_run_own = {"attend": _own_attend, "write": _own_write, "compact": _own_compact, "copy": _own_copy, "fork": _own_fork}
_run_plain = {"attend": _plain_attend, "write": _plain_write, "compact": _plain_compact, "copy": _plain_copy, "fork": _plain_fork}


# ------------------------------------------------------------------------------------------------ from the definition, in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    P, kind = case["page"], case["kind"]
    if kind == "attend":
        return _exact_attend(case, s)
    pools = [s["k"].double(), s["v"].double()] + ([] if s["sizes"] is None else [s["sizes"][None, :, None, :, None].clone()])
    front = ()
    if kind == "write":
        t = 0
        news = [s["new_k"].double(), s["new_v"].double()] + ([] if s["sizes"] is None else [s["new_sizes"][:, None, None]])
        for row, n in zip(s["rows"], s["lengths"]):
            done = 0
            while done < n:                                 # the part of the sequence that lies in one page
                at = case["past"] + done
                take = min(n - done, P - at % P)
                for pool, new in zip(pools, news):
                    pool[0, row[at // P], :, at % P:at % P + take] = new[t + done:t + done + take].transpose(0, 1)
                done += take
            t += n
    elif kind == "compact":
        before = [pool.clone() for pool in pools]
        ends = []
        for row, out, kept, n, total in zip(s["rows"], s["out_rows"], s["kept_lists"], s["lengths"], s["need"]):
            first = case["before"]
            survivors = torch.tensor(list(range(first)) + [first + j for j in kept] + list(range(first + n, total)), device="cuda")
            ends.append(survivors.numel())
            held = torch.tensor(row[:_pages_of(case, total)], device="cuda")
            for pool, old in zip(pools, before):
                whole = old[:, held].transpose(1, 2).flatten(2, 3)[:, :, survivors]        # [layers, heads, tokens, D]
                for j in range(_pages_of(case, survivors.numel())):
                    part = whole[:, :, j * P:(j + 1) * P]
                    pool[:, out[j], :, :part.shape[2]] = part
        front = (torch.tensor(ends, dtype=torch.int32),)
    elif kind == "copy":
        for pool in pools:
            for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
                pool[:, b].copy_(pool[:, a])
    else:
        rows, parent = case["length"] % P, s["parent"].tolist()
        free = [p for p, r in enumerate(s["refs"].tolist()) if r == 0]
        children = []
        for c in range(case["children"]):
            children.append(parent[:-1] + [free[c]] if rows else parent)
            if rows:
                for pool in pools:
                    pool[:, free[c], :, :rows] = pool[:, parent[-1], :, :rows]
        front = (torch.tensor(children, dtype=torch.int32), s["refs"])
    if s["sizes"] is not None:
        pools[2] = pools[2][0, :, 0, :, 0]
    return front + tuple(pools)


def _exact_attend(case, s):
    P, heads, D = case["page"], case["heads"], case["D"]
    group = case["q_heads"] // heads
    out = torch.zeros(len(s["lengths"]), case["q_heads"], D, dtype=torch.float64, device="cuda")
    for i, n in enumerate(s["lengths"]):
        if n == 0:
            continue
        at = torch.arange(n, device="cuda")
        slot = s["table"][i].long()[at // P]
        if s["sizes"] is not None:
            size = s["sizes"][slot, at % P]
            at, slot, size = at[size > 0], slot[size > 0], size[size > 0].double()
            if at.numel() == 0:
                continue
        for h in range(heads):
            k, v = s["k"][0, slot, h, at % P].double(), s["v"][0, slot, h, at % P].double()
            if case["sizes"] == "enhance":
                v = v + size.log()[:, None]
            a = torch.softmax(s["q"][i, h * group:(h + 1) * group].double() @ k.T / D ** 0.5, dim=1)
            out[i, h * group:(h + 1) * group] = a @ v
    return out

"""Decode from a KV cache held in 8 bits, and the page tables of such a cache kept on the GPU, as cases to be measured.

Four kinds of pass, one for each operator:
  tables    rows that ended give their pages back, the others take pages for their new tokens: block table, slots,
            positions, page lists (`dag_kv_release`, `dag_kv_tables`)
  append    new keys, rotated at their positions, and values become 8-bit codes in the slots (`dag_kv_append_rope_q8`)
  decode    attention of live branches over the shared context of their group and their own pages (`dag_attn_decode_q8`)
  frontier  the same over contexts given as lists of segments, also for several new tokens of a node at once
            (`dag_attn_decode_segments_q8`)

The cache: pages of 16 tokens, codes in OCP e4m3, one scale for each (page, KV head) of K and of V,
    K codes [page][head][dim / 16][slot][dim % 16],  V codes [page][head][dim][slot],  scales [page][head] in 32 bits;
a code c stands for scale * c.  A page's scale is the smallest power of two (2^-100 at least) with which all its tokens so far
are within +-448; when it grows, the codes that are there are taken along (rounded again).  A token in slot 0 begins
the page: its scale is that of its new tokens alone and the slots behind them are 0.
Sizes are those of the library's decode benchmark (32 / 8 heads of 128, 16 groups of 8 branches), or generic.
"""
import math
import random

import numpy as np
import torch

own = False

PAGE = 16
TOP = 448.0        # largest e4m3
LEAST = -100       # of a scale's exponent
E4M3 = torch.float8_e4m3fn
LAYER = dict(hq=32, hkv=8, d=128)


def listed():
    return [
        # one step of a serving batch: most rows take a token, some of them a page, a few have ended
        dict(name="tables_step", kind="tables", rows=128, width=576, old=9216, new=1, ended=3, spare=64, lens=1),
        # prompts of very different lengths arrive together; the pool runs out before the last of them
        dict(name="tables_prompts", kind="tables", rows=777, width=640, old=2000, new=4099, ended=10, spare=-5000, lens=2),
        # the new tokens of one decode step
        dict(name="append_step", kind="append", rows=128, old=1040, new=1, dtype="bf16", theta=500000.0, hkv=8, d=128, lens=3),
        # step headers of a few tokens that continue partly filled pages, small heads, 32-bit inputs
        dict(name="append_headers_f32", kind="append", rows=67, old=300, new=41, dtype="f32", theta=10000.0, hkv=4, d=64, lens=4),
        # whole prompts after their prefill
        dict(name="append_prompts", kind="append", rows=16, old=0, new=8192, dtype="bf16", theta=500000.0, hkv=8, d=128, lens=5),
        # a single request with four branches: latency
        dict(name="decode_single", kind="decode", groups=1, branches=4, shared=1500, own=200, jitter=50, lens=6, **LAYER),
        # small heads, ragged contexts
        dict(name="decode_d64", kind="decode", groups=11, branches=5, shared=3777, own=517, jitter=300, lens=7, hq=16, hkv=8, d=64),
        # a full serving batch
        dict(name="decode_batch", kind="decode", groups=16, branches=8, shared=8192, own=1024, jitter=0, lens=8, **LAYER),
        # few requests with many siblings over a very long shared context
        dict(name="decode_wide", kind="decode", groups=2, branches=32, shared=32768, own=640, jitter=0, lens=9, hq=40, hkv=8, d=128),
        # one plan with three live branches behind a join: latency
        dict(name="frontier_single", kind="frontier", groups=1, mids=2, leaves=3, reads=2, new=1, root=600, mid=150, own=70,
             jitter=20, lens=10, **LAYER),
        # live leaves under two levels of shared nodes
        dict(name="frontier_batch", kind="frontier", groups=16, mids=2, leaves=4, reads=1, new=1, root=4096, mid=2048, own=1031,
             jitter=31, lens=11, **LAYER),
        # step headers of nine tokens go through the cache at once, each token seeing those before it
        dict(name="frontier_headers", kind="frontier", groups=8, mids=2, leaves=3, reads=2, new=9, root=2048, mid=700, own=90,
             jitter=40, lens=12, **LAYER),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {"tables": 1.6e7, "append": 4.5e8, "decode": 5.4e8, "frontier": 5.4e8}
    while True:
        kind = rng.choice(["tables", "append", "decode", "decode", "frontier", "frontier"])
        case = dict(kind=kind, lens=rng.randrange(1 << 30))
        if kind == "tables":
            case.update(rows=_log_int(rng, 1, 4000), old=_log_int(rng, 1, 10000), new=_log_int(rng, 1, 5000),
                        ended=rng.choice([0, 2, 15, 50]), spare=rng.choice([-2000, -30, 0, 100]))
            case["width"] = -(-(case["old"] + case["new"]) // PAGE) + rng.choice([-3, 0, 5])
            if case["width"] < 1:
                continue
        else:
            case.update(hkv=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128, 128]))
        if kind == "append":
            case.update(rows=_log_int(rng, 1, 500), old=rng.choice([0, _log_int(rng, 1, 3000)]), new=_log_int(rng, 1, 8192),
                        dtype=rng.choice(["bf16", "bf16", "f32"]), theta=rng.choice([10000.0, 500000.0, 1000000.0]))
        if kind in ("decode", "frontier"):
            case["hq"] = case["hkv"] * rng.choice([1, 2, 4, 4, 5, 6, 8])
            case.update(groups=_log_int(rng, 1, 20), jitter=rng.choice([0, 13, 39]), own=_log_int(rng, 1, 1500))
        if kind == "decode":
            case.update(branches=_log_int(rng, 1, 32), shared=_log_int(rng, 1, 32768))
        if kind == "frontier":
            case.update(mids=rng.randint(1, 3), leaves=rng.randint(1, 6), root=_log_int(rng, 16, 8192), mid=_log_int(rng, 16, 3000),
                        new=rng.choice([1, 1, 1, _log_int(rng, 2, 16)]))
            case["reads"] = rng.randint(1, case["mids"])
        if work(case)["bytes"] <= most[kind] and work(case)["flops"] <= 4.3e10 and _padded(case) <= 6.0e9:
            return case


# --------------------------------------------------------------------------- shapes
def _pages(n):
    return -(-n // PAGE)


def _rows(case):
    """(tokens stored, new tokens, whether it ended) of every row of a table, or of the rows that an append goes to."""
    rng = random.Random(case["lens"])
    got = []
    for _ in range(case["rows"]):
        old = rng.randint(0, case["old"])
        end = rng.random() * 100 < case.get("ended", 0)
        new = 1 if case["new"] == 1 else rng.randint(case["new"] // 4, case["new"])
        got.append((old, 0 if end else new, end))
    return got


def _contexts(case):
    """[tokens of each branch's own pages] and [(tokens, its readers)] of every shared stretch of context."""
    rng = random.Random(case["lens"])

    def vary(n):
        return max(1, n + rng.randint(-case["jitter"], case["jitter"]))

    live, shared = [], []
    for _ in range(case["groups"]):
        first = len(live)
        if case["kind"] == "decode":
            n = max(1, case["branches"] - (rng.randint(0, 2) if case["jitter"] else 0))
            live += [vary(case["own"]) for _ in range(n)]
            shared.append((vary(case["shared"]), list(range(first, len(live)))))
        else:
            live += [case["new"] - 1 + vary(case["own"]) for _ in range(case["mids"] * case["leaves"])]
            shared.append((vary(case["root"]), list(range(first, len(live)))))
            for m in range(case["mids"]):
                shared.append((vary(case["mid"]), [r for r in range(first, len(live))
                                                   if (m - (r - first) // case["leaves"]) % case["mids"] < case["reads"]]))
    return live, shared


def _padded(case):
    """Values in the largest arrays of the plain form, whose lists all have the longest one's length."""
    if case["kind"] in ("tables", "append"):
        return 0
    live, shared = _contexts(case)
    lists = [([n for n, _ in shared], max(len(r) for _, r in shared)), (live, 1)]
    if case["kind"] == "frontier":
        lists = [(live + lists[0][0], lists[0][1] * case["new"])]
    return sum(len(n) * max(n) * (2 * case["hkv"] * case["d"] + 2 * case["hq"] * rows) for n, rows in lists)


def _pool_pages(case):
    if case["kind"] in ("tables", "append"):
        return 0
    live, shared = _contexts(case)
    return sum(_pages(n) for n in live) + sum(_pages(n) for n, _ in shared)


def work(case):
    if case["kind"] == "tables":
        new = taken = kept = freed = 0
        for old, n, end in _rows(case):
            freed += _pages(old) if end else 0
            new += n
            taken += 0 if end else _pages(old + n) - _pages(old)
            kept += 0 if end else _pages(old + n)
        # a row: length, new tokens, position, flag read; length and two offsets written.  A slot and a position for each new
        # token; a page taken or given back is read and written, and so is one that is listed
        return {"bytes": 28 * case["rows"] + 8 * new + 8 * (taken + freed + kept), "flops": 0}
    hkv, d = case["hkv"], case["d"]
    if case["kind"] == "append":
        rows = _rows(case)
        new = sum(n for _, n, _ in rows)
        pages = sum(_pages(old + n) - old // PAGE for old, n, _ in rows)
        # K and V in 16 or 32 bits read, 8 bits written, scales, slot and position; rotation, division, maximum
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": new * (2 * hkv * d * (size + 1) + 8) + pages * hkv * 8, "flops": new * hkv * d * 10}
    live, shared = _contexts(case)
    new = case.get("new", 1)
    tokens = sum(live) + sum(n for n, _ in shared)
    rows = len(live) * new
    pairs = sum(n * new * len(readers) for n, readers in shared) + sum(new * n - new * (new - 1) // 2 for n in live)
    # codes of every token once, scales and page ids, q read, out written
    return {"bytes": 2 * hkv * d * tokens + _pool_pages(case) * (8 * hkv + 4) + 4 * case["hq"] * d * rows,
            "flops": 4 * d * case["hq"] * pairs}


# --------------------------------------------------------------------------- states
def _ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def _normal(gen, shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=gen)


def _pool(gen, n_pages, hkv, d):
    """A cache of pages in use: normal values whose size differs between heads, a page's scale from its largest."""
    size = torch.exp(0.7 * _normal(gen, (1, hkv)))
    out = {}
    for name, shape in (("k", (n_pages, hkv, d // PAGE, PAGE, PAGE)), ("v", (n_pages, hkv, d, PAGE))):
        x = torch.empty(shape, dtype=E4M3, device="cuda")
        for a in range(0, n_pages, 8192):
            part = _normal(gen, (min(8192, n_pages - a),) + shape[1:])
            x[a:a + 8192] = (part * 64.0).clamp_(-TOP, TOP).to(E4M3)
        out[name + "_pool"] = x
        out[name + "_scale"] = torch.exp2(torch.round(torch.log2(size / 64.0))).expand(n_pages, hkv).contiguous()
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    s = dict(case=case)
    if case["kind"] == "tables":
        rows = _rows(case)
        width = case["width"]
        held = [min(_pages(old), width) for old, _, _ in rows]
        need = sum(max(0, _pages(old + n) - _pages(old)) for old, n, _ in rows)
        n_free = max(1, need + case["spare"])
        n_pages = sum(held) + n_free
        perm = rng.permutation(n_pages).astype(np.int32)
        table = np.full((len(rows), width), -1, dtype=np.int32)
        at = 0
        for r, n in enumerate(held):
            table[r, :n] = perm[at:at + n]
            at += n
        free = np.full(n_pages, -1, dtype=np.int32)
        free[:n_free] = perm[at:]
        total = sum(n for _, n, _ in rows)
        s.update(table=_ints(table), row_len=_ints([min(old, width * PAGE) for old, _, _ in rows]), free_pages=_ints(free),
                 free_count=_ints([n_free]), new_len=_ints([n for _, n, _ in rows]), ended=_ints([int(e) for _, _, e in rows]),
                 pos0=_ints(rng.integers(0, 40000, len(rows))), total=total, any_ended=any(e for _, _, e in rows))
        s["out"] = {name: torch.full((n,), -1, dtype=torch.int32, device="cuda") for name, n in (
            ("len_between", len(rows)), ("count_between", 1), ("row_len", len(rows)), ("free_count", 1), ("new_off", len(rows) + 1),
            ("slots", total), ("pos", total), ("page_off", len(rows) + 1), ("pages", n_pages), ("refused", 1))}
        return s
    hkv, d = case["hkv"], case["d"]
    if case["kind"] == "append":
        rows = _rows(case)
        counts = [_pages(old + n) - old // PAGE for old, n, _ in rows]
        perm = rng.permutation(sum(counts)).astype(np.int64)
        ends = np.cumsum([0] + counts)
        slots, pos = [], []
        for r, (old, n, _) in enumerate(rows):
            t = old % PAGE + np.arange(n)
            slots.append(perm[ends[r] + t // PAGE] * PAGE + t % PAGE)
            pos.append(int(rng.integers(0, 3000)) + old + np.arange(n))
        s.update(_pool(gen, int(ends[-1]), hkv, d), slots=_ints(np.concatenate(slots)), pos=_ints(np.concatenate(pos)))
        dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        total = sum(n for _, n, _ in rows)
        # (the sizes of tokens differ, so that the scales of begun pages grow here and there)
        size = torch.exp(0.7 * _normal(gen, (total, 1, 1)))
        for name in ("k_new", "v_new"):
            s[name] = (_normal(gen, (total, hkv, d)) * size).to(dtype)
        return s
    live, shared = _contexts(case)
    new = case.get("new", 1)
    lens = [n for n, _ in shared] + live
    ends = np.cumsum([0] + [_pages(n) for n in lens])
    perm = rng.permutation(int(ends[-1])).astype(np.int32)
    s.update(_pool(gen, int(ends[-1]), hkv, d), q=_normal(gen, (len(live) * new, case["hq"], d), torch.bfloat16))
    s["out"] = torch.empty_like(s["q"])
    if case["kind"] == "decode":
        at, n = int(ends[len(shared)]), [len(r) for _, r in shared]
        s["desc"] = dict(
            group_branch_off=_ints(np.cumsum([0] + n)), shared_page_off=_ints(ends[:len(shared) + 1]), shared_pages=_ints(perm[:at]),
            shared_len=_ints(lens[:len(shared)]), branch_page_off=_ints(ends[len(shared):] - at), branch_pages=_ints(perm[at:]),
            branch_len=_ints(live), branch_pos=_ints(live))
        s["most"] = dict(n_groups=len(shared), n_live=len(live), max_shared_pages=max(_pages(n) for n, _ in shared),
                         max_branch_pages=max(map(_pages, live)), max_group_size=max(n))
        return s
    readers = [[r * new + i for r in rs for i in range(new)] for _, rs in shared] + [[r * new + i for i in range(new)] for r in range(len(live))]
    flat = [r for rs in readers for r in rs]
    entries = [[] for _ in range(len(live) * new)]
    for e, r in enumerate(flat):
        entries[r].append(e)
    sees = [n for n, rs in shared for _ in range(len(rs) * new)] + [n - new + 1 + i for n in live for i in range(new)]
    s["desc"] = dict(
        seg_page_off=_ints(ends), seg_pages=_ints(perm), seg_len=_ints(lens), seg_reader_off=_ints(np.cumsum([0] + [len(r) for r in readers])),
        seg_readers=_ints(flat), branch_entry_off=_ints(np.cumsum([0] + [len(e) for e in entries])),
        branch_entries=_ints([e for b in entries for e in b]), seg_reader_len=_ints(sees) if new > 1 else None)
    s["most"] = dict(n_live=len(live) * new, n_segments=len(lens), max_seg_pages=max(map(_pages, lens)),
                     max_readers=max(map(len, readers)), total_readers=len(flat))
    s["most_entries"] = max(map(len, entries))
    return s


# --------------------------------------------------------------------------- one pass
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"tables": _own_tables, "append": _own_append, "decode": _own_decode, "frontier": _own_frontier}[kind](s)
    return {"tables": _plain_tables, "append": _plain_append, "decode": _plain_decode, "frontier": _plain_frontier}[kind](s)


def _own_tables(s):
    from paper_2602_07529_amd import binding as B
    rows = s.get("rows")  # (the handles that a program keeps: the rows, the cache, the description with its workspace)
    if rows is None:
        rows = s["rows"] = B.KvRows(s["table"], s["free_pages"])
    o = s["out"]
    row_len, count = s["row_len"], s["free_count"]
    if s["any_ended"]:
        B.dag_kv_release(rows, s["ended"], row_len, o["len_between"], count, o["count_between"])
        row_len, count = o["len_between"], o["count_between"]
    B.dag_kv_tables(rows, s["new_len"], row_len, o["row_len"], count, o["free_count"], o["new_off"], o["slots"], pos0=s["pos0"], pos=o["pos"],
                    page_off=o["page_off"], pages=o["pages"], refused=o["refused"])
    return dict({n: o[n] for n in ("row_len", "free_count", "new_off", "slots", "pos", "page_off", "pages", "refused")},
                table=s["table"], free_pages=s["free_pages"])


def _cache(s, B):
    cache = s.get("cache")
    if cache is None:
        cache = s["cache"] = B.KvCacheQ8(s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"])
    return cache


def _own_append(s):
    from paper_2602_07529_amd import binding as B
    B.dag_kv_append_rope_q8(_cache(s, B), s["slots"], s["pos"], s["k_new"], s["v_new"], s["case"]["theta"])
    return {n: s[n] for n in ("k_pool", "v_pool", "k_scale", "v_scale")}


def _own_decode(s):
    from paper_2602_07529_amd import binding as B
    cache, plan = _cache(s, B), s.get("plan")
    if plan is None:
        desc = B.DecodeDesc.on_device(**s["most"], **s["desc"])
        plan = s["plan"] = desc, torch.empty(max(256, B.dag_decode_q8_workspace_bytes(desc, cache, s["q"].shape[1])), dtype=torch.uint8, device="cuda")
    B.dag_attn_decode_q8(plan[0], s["q"], cache, s["out"], plan[1])
    return s["out"]


def _own_frontier(s):
    from paper_2602_07529_amd import binding as B
    cache, plan = _cache(s, B), s.get("plan")
    if plan is None:
        desc = B.SegDecodeDesc.on_device(**s["most"], **s["desc"])
        plan = s["plan"] = desc, torch.empty(max(256, B.dag_decode_segments_q8_workspace_bytes(desc, cache, s["q"].shape[1])), dtype=torch.uint8, device="cuda")
    B.dag_attn_decode_segments_q8(plan[0], s["q"], cache, s["out"], plan[1])
    return s["out"]


# --------------------------------------------------------------------------- plain forms
def _before(x):  # sums of the values in front, and the sum of all behind them
    return torch.nn.functional.pad(torch.cumsum(x, 0), (1, 0))


def _plain_tables(s):
    table, free, count, old = s["table"].long(), s["free_pages"].long(), s["free_count"].long(), s["row_len"].long()
    n_rows, width = table.shape
    col = torch.arange(width, device="cuda")
    behind = free.numel()  # a place behind the list, for what is not written

    def put(to, mask, at, what):
        to = torch.cat([to.reshape(-1), to.new_zeros(1)])
        to.scatter_(0, torch.where(mask, at, to.numel() - 1).reshape(-1), what.expand(mask.shape).reshape(-1))
        return to[:-1]

    # pages of ended rows, in the order of rows and tokens
    gone = torch.where(s["ended"] > 0, (old + PAGE - 1) // PAGE, 0)
    first = _before(gone)
    free = put(free, col < gone[:, None], (count + first[:-1])[:, None] + col, table)
    count = count + first[-1]
    old = torch.where(s["ended"] > 0, 0, old)
    # pages for new tokens: from the end of the list
    want = s["new_len"].long()
    has = (old + PAGE - 1) // PAGE
    fits = old + want <= width * PAGE
    need = torch.where(fits, (old + want + PAGE - 1) // PAGE - has, 0)
    start = _before(need)[:-1]
    ok = fits & ((need == 0) | (start + need <= count))
    need = torch.where(ok, need, 0)
    k = col - has[:, None]
    taken = free[(count - 1 - start[:, None] - k).clamp(0, behind - 1)]
    mine = (k >= 0) & (k < need[:, None])
    table = torch.where(mine, taken, table)
    length = old + torch.where(ok, want, 0)
    left = count - torch.where(need > 0, start + need, 0).max()
    new_off = _before(want)
    t = torch.arange(s["total"], device="cuda")
    r = torch.searchsorted(new_off[1:], t, right=True)
    at = old[r] + t - new_off[r]
    slots = torch.where(ok[r], table[r, (at // PAGE).clamp(max=width - 1)] * PAGE + at % PAGE, -1)
    n = (length + PAGE - 1) // PAGE
    page_off = _before(n)
    pages = put(torch.full_like(free, -1), col < n[:, None], page_off[:-1, None] + col, table)
    refused = (~ok & (want > 0)).sum()
    got = dict(row_len=length, free_count=left, new_off=new_off, slots=slots, pos=s["pos0"].long()[r] + at, page_off=page_off, pages=pages,
               refused=refused[None], table=table, free_pages=free)
    return {name: x.to(torch.int32) for name, x in got.items()}


def _turned(x, pos, theta):
    """Pairs (m, m + d / 2) rotated by pos * theta^(-2 m / d), in 64 bits."""
    half = x.shape[-1] // 2
    angle = pos.double()[:, None, None] * theta ** (torch.arange(half, device="cuda", dtype=torch.float64) * (-1.0 / half))
    c, n, lo, hi = torch.cos(angle), torch.sin(angle), x[..., :half].double(), x[..., half:].double()
    return torch.cat([lo * c - hi * n, hi * c + lo * n], -1)


def _exponent(most):
    """The smallest k with most <= 448 * 2^k."""
    m, e = torch.frexp(most)
    return torch.where(most > 0, torch.where(m <= 0.875, e - 9, e - 8), LEAST).clamp(min=LEAST)


def _plain_append(s):
    case, slots = s["case"], s["slots"].long()
    n_pages, hkv = s["k_scale"].shape
    page, slot = slots // PAGE, slots % PAGE
    begun = torch.zeros(n_pages, dtype=torch.bool, device="cuda")
    begun[page[slot == 0]] = True
    out = {}
    for name, x in (("k", _turned(s["k_new"], s["pos"], case["theta"])), ("v", s["v_new"].double())):
        most = x.new_zeros(n_pages, hkv).scatter_reduce_(0, page[:, None].expand(-1, hkv), x.abs().amax(-1), "amax")
        touched = torch.zeros(n_pages, dtype=torch.bool, device="cuda")
        touched[page] = True
        old = s[name + "_scale"].double()
        scale = torch.ldexp(torch.ones_like(most), _exponent(most))
        scale = torch.where(begun[:, None], scale, torch.where(touched[:, None], torch.maximum(scale, old), old))
        keep = torch.where(begun[:, None], 0.0, old / scale)
        pool = s[name + "_pool"]
        codes = (pool.float() * keep.float()[(...,) + (None,) * (pool.dim() - 2)]).to(E4M3)
        mine = (x / scale[page][..., None]).float().to(E4M3)
        # (bytes: the codes are put where they belong as they are)
        flat = codes.view(torch.uint8)
        if name == "k":
            flat[page, :, :, slot] = mine.view(torch.uint8).reshape(len(page), hkv, -1, PAGE)
        else:
            flat[page, :, :, slot] = mine.view(torch.uint8)
        pool.copy_(codes)
        s[name + "_scale"].copy_(scale)
        out[name + "_pool"], out[name + "_scale"] = pool, s[name + "_scale"]
    return out


def _values(s, pages, offsets, most):
    """K and V of lists of pages, each filled up to `most` pages: [list][KV head][token][dim] in 32 bits."""
    at = (offsets[:-1, None].long() + torch.arange(most, device="cuda")).clamp(max=pages.numel() - 1)
    p = pages.long()[at]
    k = s["k_pool"][p].float() * s["k_scale"][p][..., None, None, None]  # [n][page][h][d / 16][slot][16]
    v = s["v_pool"][p].float() * s["v_scale"][p][..., None, None]        # [n][page][h][d][slot]
    n, _, h = k.shape[:3]
    k = k.permute(0, 2, 1, 4, 3, 5).reshape(n, h, most * PAGE, -1)
    return k, v.permute(0, 2, 1, 4, 3).reshape(n, h, most * PAGE, -1)


def _part(q, k, v, sees):
    """Largest score, sum of exponentials and their weighted values: q [n][row][query head][d], the leading `sees` [n][row] tokens."""
    n, r, hq, d = q.shape
    h = k.shape[1]
    g = hq // h
    x = q.float().reshape(n, r, h, g, d).transpose(1, 2).reshape(n, h, r * g, d)
    x = torch.matmul(x, k.transpose(2, 3).contiguous()) * d ** -0.5
    hidden = torch.arange(k.shape[2], device="cuda") >= sees[..., None]  # [n][row][token]
    x = x.masked_fill(hidden.repeat_interleave(g, 1)[:, None], -math.inf)
    m = x.amax(-1).clamp(min=-1e30)
    x = torch.exp(x - m[..., None])
    back = lambda y: y.reshape(n, h, r, g, *y.shape[3:]).transpose(1, 2).reshape(n, r, hq, *y.shape[3:])  # noqa: E731
    return back(m), back(x.sum(-1)), back(torch.matmul(x, v))


def _joined(m, l, o):  # parts in dimension 1
    w = torch.exp(m - m.amax(1, keepdim=True))
    total = (w * l).sum(1)[..., None]
    return torch.where(total > 0, (w[..., None] * o).sum(1) / total.clamp(min=1e-37), 0.0).to(torch.bfloat16)


def _plain_decode(s):
    c, most, q = s["desc"], s["most"], s["q"]
    first, length = c["group_branch_off"][:-1].long(), torch.diff(c["group_branch_off"]).long()
    col = torch.arange(most["max_group_size"], device="cuda")
    r = (first[:, None] + col).clamp(max=q.shape[0] - 1)
    sees = torch.where(col < length[:, None], c["shared_len"].long()[:, None], 0)
    a = _part(q[r], *_values(s, c["shared_pages"], c["shared_page_off"], most["max_shared_pages"]), sees)
    g = torch.searchsorted(c["group_branch_off"][1:].contiguous(), torch.arange(q.shape[0], device="cuda", dtype=torch.int32), right=True)
    j = torch.arange(q.shape[0], device="cuda") - first[g]
    b = _part(q[:, None], *_values(s, c["branch_pages"], c["branch_page_off"], most["max_branch_pages"]), c["branch_len"].long()[:, None])
    return _joined(*(torch.stack([x[g, j], y[:, 0]], 1) for x, y in zip(a, b)))


def _plain_frontier(s):
    c, most, q = s["desc"], s["most"], s["q"]
    first, length = c["seg_reader_off"][:-1].long(), torch.diff(c["seg_reader_off"]).long()
    col = torch.arange(most["max_readers"], device="cuda")
    e = (first[:, None] + col).clamp(max=most["total_readers"] - 1)  # [segment][reader]
    sees = c["seg_len"].long()[:, None].expand_as(e)
    if c["seg_reader_len"] is not None:
        sees = torch.minimum(sees, c["seg_reader_len"].long()[e])
    sees = torch.where(col < length[:, None], sees, 0)
    part = _part(q[c["seg_readers"].long()[e]], *_values(s, c["seg_pages"], c["seg_page_off"], most["max_seg_pages"]), sees)
    off = c["branch_entry_off"].long()
    n = torch.arange(s["most_entries"], device="cuda")
    mine = c["branch_entries"].long()[(off[:-1, None] + n).clamp(max=most["total_readers"] - 1)]  # [branch][entry]
    seg = torch.searchsorted(c["seg_reader_off"][1:].long(), mine, right=True)
    m, l, o = (x[seg, mine - first[seg]] for x in part)
    there = (n < torch.diff(off)[:, None])[..., None]
    return _joined(torch.where(there, m, -1e30), torch.where(there, l, 0.0), o)


# --------------------------------------------------------------------------- 64 bits, written apart
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "tables":
        return None
    return _exact_append(s) if case["kind"] == "append" else _exact_attention(s)


def _to_e4m3(x):
    """To the nearest of the type's values, ties to even: steps of 2^-3 of a value's power of two, of 2^-9 below 2^-6."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 1).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def _exact_append(s):
    case = s["case"]
    hkv, d = case["hkv"], case["d"]
    slots, pos = s["slots"].cpu().numpy().astype(np.int64), s["pos"].double()
    half = d // 2
    x = s["k_new"].double()
    z = torch.complex(x[..., :half], x[..., half:])
    freq = torch.tensor([case["theta"] ** (-2.0 * m / d) for m in range(half)], dtype=torch.float64, device="cuda")
    z = z * torch.polar(torch.ones_like(x[:, :1, :half]), pos[:, None, None] * freq)
    fresh = {"k": torch.cat([z.real, z.imag], -1), "v": s["v_new"].double()}
    # the pages that tokens go to, each with its tokens by slot
    page, place = np.unique(slots // PAGE, return_inverse=True)
    token = np.full((len(page), PAGE), -1, dtype=np.int64)
    token[place, slots % PAGE] = np.arange(len(slots))
    token = torch.from_numpy(token).cuda()
    page = torch.from_numpy(page).cuda()
    out = {}
    for name in ("k", "v"):
        old = s[name + "_pool"][page].double()
        if name == "k":
            old = old.transpose(2, 3).reshape(len(page), hkv, PAGE, d)
        else:
            old = old.transpose(2, 3)
        there = (token >= 0)[:, None, :, None]
        x = torch.where(there, fresh[name][token.clamp(min=0)].transpose(1, 2), 0.0)
        most = x.abs().amax((2, 3))
        k = torch.ceil(torch.log2(most / TOP))
        k = torch.where(torch.exp2(k - 1) * TOP >= most, k - 1, torch.where(torch.exp2(k) * TOP < most, k + 1, k)).clamp(min=float(LEAST))
        before, begun = s[name + "_scale"][page].double(), (token[:, 0] >= 0)[:, None]
        scale = torch.where(begun, torch.exp2(k), torch.maximum(torch.exp2(k), before))
        kept = torch.where(begun[..., None, None], 0.0, old * (before / scale)[..., None, None])
        codes = _to_e4m3(torch.where(there, x / scale[..., None, None], kept))
        if name == "k":
            codes = codes.reshape(len(page), hkv, PAGE, d // PAGE, PAGE).transpose(2, 3)
        else:
            codes = codes.transpose(2, 3)
        pool, scales = s[name + "_pool"].double(), s[name + "_scale"].double()
        pool[page], scales[page] = codes, scale
        out[name + "_pool"], out[name + "_scale"] = pool, scales
    return out


def _exact_attention(s):
    case, c = s["case"], {n: x.cpu().numpy() for n, x in s["desc"].items() if x is not None}
    hkv, d, n_live = case["hkv"], case["d"], s["q"].shape[0]
    g = case["hq"] // hkv
    if case["kind"] == "decode":
        lists = [("shared_pages", "shared_page_off", "shared_len"), ("branch_pages", "branch_page_off", "branch_len")]
        off = c["group_branch_off"]
        readers = [list(range(off[i], off[i + 1])) for i in range(len(off) - 1)] + [[r] for r in range(n_live)]
        sees = None
    else:
        lists = [("seg_pages", "seg_page_off", "seg_len")]
        off = c["seg_reader_off"]
        readers = [list(c["seg_readers"][off[i]:off[i + 1]]) for i in range(len(off) - 1)]
        sees = [c["seg_reader_len"][off[i]:off[i + 1]] for i in range(len(off) - 1)] if "seg_reader_len" in c else None
    stretches = [(c[p][c[o][i]:c[o][i] + _pages(int(n))], int(n)) for p, o, ln in lists for i, n in enumerate(c[ln])]
    top = torch.full((n_live, hkv, g), -math.inf, dtype=torch.float64, device="cuda")
    total, acc = torch.zeros_like(top), torch.zeros((n_live, hkv, g, d), dtype=torch.float64, device="cuda")
    q = s["q"].double().reshape(n_live, hkv, g, d)
    for i, ((pages, n), rs) in enumerate(zip(stretches, readers)):
        if not n or not rs:
            continue
        p, r = torch.from_numpy(pages.astype(np.int64)).cuda(), torch.tensor(rs, dtype=torch.int64, device="cuda")
        k = s["k_pool"][p].double() * s["k_scale"][p].double()[:, :, None, None, None]
        k = k.permute(1, 0, 3, 2, 4).reshape(hkv, -1, d)[:, :n]
        v = s["v_pool"][p].double() * s["v_scale"][p].double()[:, :, None, None]
        v = v.permute(1, 0, 3, 2).reshape(hkv, -1, d)[:, :n]
        x = torch.matmul(q[r].transpose(0, 1).reshape(hkv, -1, d), k.transpose(1, 2).contiguous()) / math.sqrt(d)
        x = x.reshape(hkv, len(rs), g, n)
        if sees is not None:
            lim = torch.from_numpy(sees[i].astype(np.int64)).cuda()
            x = torch.where(torch.arange(n, device="cuda") < lim[None, :, None, None], x, -math.inf)
        m = torch.maximum(top[r], x.amax(-1).transpose(0, 1))
        ref = torch.where(torch.isinf(m), 0.0, m)
        e, keep = torch.exp(x - ref.transpose(0, 1)[..., None]), torch.exp(top[r] - ref)
        total[r] = total[r] * keep + e.sum(-1).transpose(0, 1)
        acc[r] = acc[r] * keep[..., None] + torch.matmul(e.reshape(hkv, -1, n), v.contiguous()).reshape(hkv, len(rs), g, d).transpose(0, 1)
        top[r] = m
    return torch.where(total[..., None] > 0, acc / total[..., None], 0.0).reshape(n_live, case["hq"], d)

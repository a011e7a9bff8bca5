"""Chunks of new tokens over a KV cache in 8 bits, forks and compaction of its pages, and general rotary positions, as cases to be measured.

Four kinds of pass, one for each operator:
  chunk     attention of the new tokens of nodes over the pages of their contexts, their own last (`dag_attn_prefill_paged_q8`)
  fork      rows that become copies of others: full pages by reference, the last partly filled one copied
            (`dag_kv_fork`, `dag_kv_copy_pages_q8`)
  compact   ended rows give back what nobody else holds, then the pages in use move to the front of the pool
            (`dag_kv_release_shared`, `dag_kv_compact`, `dag_kv_copy_pages_q8`)
  rotary    rotary positions in either pair layout, for part of a head, with stretched frequencies, forward and transposed
            (`dag_rope_apply`), or on the way into the cache (`dag_kv_append_rotary_q8`)

The cache: pages of 16 tokens, codes in OCP e4m3, one scale for each (page, KV head) of K and of V,
    K codes [page][head][dim / 16][slot][dim % 16],  V codes [page][head][dim][slot],  scales [page][head] in 32 bits;
a code c stands for scale * c.  Sizes are those of the library's decode and prefill benchmarks (32 / 8 heads of 128), or generic.
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
        # one token of each of a few dozen nodes, every context a list of its own: the form for single tokens
        dict(name="chunk_tokens", kind="chunk", groups=5, nodes=7, new=1, shared=900, segs=2, own=77, jitter=60, lens=1, hq=16, hkv=8, d=64),
        # a single request: three step headers of nine tokens behind one context; latency
        dict(name="chunk_headers", kind="chunk", groups=1, nodes=3, new=9, shared=1500, segs=2, own=40, jitter=30, lens=2, **LAYER),
        # the next piece of one long prompt
        dict(name="chunk_prompt", kind="chunk", groups=1, nodes=1, new=1024, shared=0, segs=0, own=31000, jitter=0, lens=3, hq=40, hkv=8, d=128),
        # join prompts of a full serving batch, ragged
        dict(name="chunk_joins", kind="chunk", groups=16, nodes=4, new=131, shared=6000, segs=3, own=20, jitter=19, lens=4, **LAYER),
        # prompts of a batch behind a common document
        dict(name="chunk_batch", kind="chunk", groups=4, nodes=4, new=2048, shared=8192, segs=1, own=0, jitter=0, lens=5, **LAYER),
        # four branches of a request are forked from its best one
        dict(name="fork_few", kind="fork", rows=9, forks=4, parents=1, width=130, old=1900, spare=40, lens=6, hkv=8, d=128),
        # a sampling step of a batch: every prompt gets its samples
        dict(name="fork_batch", kind="fork", rows=1100, forks=768, parents=96, width=96, old=1400, spare=1000, lens=7, hkv=8, d=128),
        # a small pool after a request has ended
        dict(name="compact_few", kind="compact", rows=24, forks=6, parents=3, width=64, old=700, spare=300, ended=20, lens=8, hkv=4, d=64),
        # a large pool of which half is given back
        dict(name="compact_batch", kind="compact", rows=640, forks=256, parents=64, width=96, old=900, spare=1500, ended=50, lens=9, hkv=8, d=128),
        # the new tokens of one decode step: pairs next to each other, a quarter of the head, 32 bits
        dict(name="rotary_step_f32", kind="rotary", to="rows", tokens=128, back=False, dtype="f32", hq=32, hkv=8, d=128, rotary=32, layout="pairs",
             theta=10000.0, stretch=1.0, original=0.0, factor=1.0, fused=True, far=30000, lens=10),
        # gradients of the packed training batch of the prefill benchmark, frequencies stretched by parts
        dict(name="rotary_gradients", kind="rotary", to="rows", tokens=18432, back=True, dtype="bf16", hq=32, hkv=8, d=128, rotary=128, layout="halves",
             theta=500000.0, stretch=8.0, original=8192.0, factor=1.0, fused=False, far=40000, lens=11),
        # prompts go from the fused projection's output into the cache, half of the head rotated
        dict(name="rotary_append", kind="rotary", to="cache", tokens=20000, rows=7, old=0, back=False, dtype="bf16", hq=32, hkv=8, d=128, rotary=64,
             layout="pairs", theta=10000.0, stretch=4.0, original=4096.0, factor=1.1, fused=True, far=90000, lens=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {w["kind"]: (0.0, 0.0) for w in listed()}
    for case in listed():
        w, kind = work(case), case["kind"]
        most[kind] = max(most[kind][0], w["bytes"]), max(most[kind][1], w["flops"])
    while True:
        kind = rng.choice(["chunk", "chunk", "chunk", "fork", "compact", "rotary", "rotary"])
        case = dict(kind=kind, lens=rng.randrange(1 << 30), hkv=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128, 128]))
        if kind == "chunk":
            case.update(hq=case["hkv"] * rng.choice([1, 2, 3, 4, 4, 5, 7, 8]), groups=_log_int(rng, 1, 20), nodes=_log_int(rng, 1, 20),
                        new=_log_int(rng, 1, 4096), segs=rng.randint(0, 3), own=rng.choice([0, _log_int(rng, 1, 32768)]), jitter=rng.choice([0, 11, 47]))
            case["shared"] = _log_int(rng, 16, 20000) if case["segs"] else 0
        if kind in ("fork", "compact"):
            rows = _log_int(rng, 3, 1100)
            case.update(rows=rows, parents=_log_int(rng, 1, max(1, rows // 3)), width=_log_int(rng, 2, 200), spare=rng.choice([0, 5, 300, 2000]))
            case["forks"] = rng.randint(1, rows - case["parents"])
            case["old"] = rng.randint(1, case["width"] * PAGE)
            if kind == "fork" and rng.random() < 0.3:
                case["spare"] = -rng.randint(1, case["forks"])  # too few pages for all
            if kind == "compact":
                case["ended"] = rng.choice([0, 5, 30, 80])
            if _pool_pages(case) * case["hkv"] * case["d"] * 32 > 1.2e9:
                continue
        if kind == "rotary":
            case.update(hq=case["hkv"] * rng.choice([1, 2, 4, 5, 8]), to=rng.choice(["rows", "rows", "cache"]), tokens=_log_int(rng, 1, 20000),
                        dtype=rng.choice(["bf16", "bf16", "f32"]), layout=rng.choice(["pairs", "halves"]), fused=rng.random() < 0.5,
                        theta=rng.choice([10000.0, 500000.0, 1000000.0]), stretch=rng.choice([1.0, 4.0, 32.0]),
                        original=rng.choice([0.0, 4096.0]), factor=rng.choice([1.0, 1.1, 1.35]), far=_log_int(rng, 100, 200000))
            case["rotary"] = rng.choice([32, 64, case["d"]])
            case["back"] = case["to"] == "rows" and rng.random() < 0.4
            if case["to"] == "cache":
                case.update(rows=rng.randint(1, min(200, case["tokens"])), old=rng.choice([0, _log_int(rng, 1, 500)]))
        w = work(case)
        if w["bytes"] <= most[kind][0] and w["flops"] <= most[kind][1]:
            return case


# --------------------------------------------------------------------------- shapes
def _pages(n):
    return -(-n // PAGE)


def _contexts(case):
    """Lengths of the shared stretches, and of every node: (its stretches, tokens of its own pages, new ones among them)."""
    rng = random.Random(case["lens"])

    def vary(n):
        return max(0, n + rng.randint(-case["jitter"], case["jitter"]))

    stretches, nodes = [], []
    for _ in range(case["groups"]):
        first = len(stretches)
        stretches += [max(1, vary(case["shared"] // case["segs"])) for _ in range(case["segs"])]
        for _ in range(case["nodes"]):
            new = 1 if case["new"] == 1 else max(1, case["new"] - rng.randint(0, min(case["jitter"], case["new"] // 2)))
            nodes.append((list(range(first, len(stretches))), vary(case["own"]) + new, new))
    return stretches, nodes


def _family(case):
    """Tokens of the parents' rows and of the other rows in use; (parent, tokens) of every fork; the rows that end."""
    rng = random.Random(case["lens"])
    lens = [rng.randint(max(1, case["old"] // 3), case["old"]) for _ in range(case["rows"] - case["forks"])]
    forks = []
    for _ in range(case["forks"]):
        p = rng.randrange(case["parents"])
        forks.append((p, lens[p] if rng.random() < 0.7 else rng.randint(0, lens[p])))
    ended = [rng.random() * 100 < case.get("ended", 0) for _ in range(case["rows"])]
    return lens, forks, ended


def _pool_pages(case):
    lens, forks, _ = _family(case)
    held = sum(map(_pages, lens))
    return held + max(0, sum(1 for _, n in forks if n % PAGE) + case["spare"])


def _stored(case):
    """(tokens stored, new tokens) of the rows that an append goes to."""
    rng = random.Random(case["lens"])
    cuts = sorted(rng.sample(range(1, case["tokens"]), case["rows"] - 1))
    new = [b - a for a, b in zip([0] + cuts, cuts + [case["tokens"]])]
    return [(rng.randint(0, case["old"]), n) for n in new]


def work(case):
    kind, hkv, d = case["kind"], case["hkv"], case["d"]
    if kind == "chunk":
        stretches, nodes = _contexts(case)
        tokens = sum(stretches) + sum(n for _, n, _ in nodes)
        rows = sum(new for _, _, new in nodes)
        listed_pages = sum(_pages(n) + sum(_pages(stretches[i]) for i in c) for c, n, _ in nodes)
        pool = sum(map(_pages, stretches)) + sum(_pages(n) for _, n, _ in nodes)
        pairs = sum(new * (sum(stretches[i] for i in c) + n) - new * (new - 1) // 2 for c, n, new in nodes)
        # codes of every token once, scales, page ids and lengths; q read, out and the logarithm written
        return {"bytes": 2 * hkv * d * tokens + pool * 8 * hkv + 8 * listed_pages + rows * case["hq"] * (4 * d + 4), "flops": 4 * d * case["hq"] * pairs}
    if kind in ("fork", "compact"):
        lens, forks, ended = _family(case)
        page = 2 * hkv * (d * PAGE + 4)
        if kind == "fork":
            # a fork: row, length and page pair; a shared page: entry read and written, holders read and written; a copied page
            shared = sum(n // PAGE for _, n in forks)
            copied = max(0, sum(1 for _, n in forks if n % PAGE) + min(0, case["spare"]))
            return {"bytes": 8 * case["rows"] + 24 * len(forks) + 16 * shared + copied * 2 * page, "flops": 0}
        lens = lens + [n for _, n in forks]
        kept = sum(_pages(n) for n, e in zip(lens, ended) if not e)
        gone = sum(_pages(n) for n, e in zip(lens, ended) if e)
        used, n_pages = _in_use(case)
        moves = _moves(case, used, n_pages)
        # pages given back: entry and holders; pages of the pool: holders, free list, new place; table entries; the moves
        return {"bytes": 12 * case["rows"] + 16 * gone + 20 * n_pages + 8 * kept + moves * 2 * page, "flops": 0}
    size = 4 if case["dtype"] == "f32" else 2
    if case["to"] == "rows":
        elements = case["tokens"] * (case["hq"] + hkv) * d
        return {"bytes": 2 * size * elements + 4 * case["tokens"], "flops": case["tokens"] * (case["hq"] + hkv) * case["rotary"] * 3}
    pages = sum(_pages(old % PAGE + n) for old, n in _stored(case))
    return {"bytes": case["tokens"] * (2 * hkv * d * (size + 1) + 8) + pages * hkv * 8, "flops": case["tokens"] * hkv * (3 * case["rotary"] + 4 * d)}


def _holders(case):
    """Ids of the pages of every row, in a pool where they lie in order; forks hold their parents' full pages and one of their own."""
    lens, forks, ended = _family(case)
    at, lines = 0, []
    for n in lens:
        lines.append(list(range(at, at + _pages(n))))
        at += _pages(n)
    for p, n in forks:
        lines.append(lines[p][:n // PAGE] + ([at] if n % PAGE else []))
        at += 1 if n % PAGE else 0
    return lines, lens + [n for _, n in forks], ended


def _in_use(case):
    lines, _, ended = _holders(case)
    return len({p for line, e in zip(lines, ended) if not e for p in line}), _pool_pages(case)


def _moves(case, used, n_pages):  # on average: the pages lie anywhere
    return used * (n_pages - used) // n_pages


# --------------------------------------------------------------------------- states
def _ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def _normal(gen, shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=gen)


def _pool(gen, n_pages, hkv, d):
    """A cache of pages in use: normal values whose size differs between heads and a little between pages."""
    size = torch.exp(0.7 * _normal(gen, (1, hkv)))
    out = {}
    for name, shape in (("k", (n_pages, hkv, d // PAGE, PAGE, PAGE)), ("v", (n_pages, hkv, d, PAGE))):
        x = torch.empty(shape, dtype=E4M3, device="cuda")
        for a in range(0, n_pages, 8192):
            part = _normal(gen, (min(8192, n_pages - a),) + shape[1:])
            x[a:a + 8192] = (part * 64.0).clamp_(-TOP, TOP).to(E4M3)
        out[name + "_pool"] = x
        grown = torch.where(_normal(gen, (n_pages, hkv)) > 1.5, 1.0, 0.0)
        out[name + "_scale"] = torch.exp2(torch.round(torch.log2(size / 64.0)) + grown - (0.4 if name == "k" else 0.0))
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    return {"chunk": _prepare_chunk, "fork": _prepare_rows, "compact": _prepare_rows, "rotary": _prepare_rotary}[case["kind"]](case, gen, rng)


def _prepare_chunk(case, gen, rng):
    hkv, d = case["hkv"], case["d"]
    stretches, nodes = _contexts(case)
    lens = stretches + [n for _, n, _ in nodes]
    ends = np.cumsum([0] + [_pages(n) for n in lens])
    perm = rng.permutation(int(ends[-1])).astype(np.int32)
    s = dict(case=case, **_pool(gen, int(ends[-1]), hkv, d))
    lists = [c + [len(stretches) + i] for i, (c, _, _) in enumerate(nodes)]
    q_off = np.cumsum([0] + [new for _, _, new in nodes])
    page_off = np.cumsum([0] + [sum(_pages(lens[i]) for i in c) for c in lists])
    s["desc"] = dict(
        q_off=_ints(q_off), ctx_page_off=_ints(page_off), ctx_pages=_ints(np.concatenate([perm[ends[i]:ends[i + 1]] for c in lists for i in c])),
        ctx_page_len=_ints([min(PAGE, lens[i] - PAGE * j) for c in lists for i in c for j in range(_pages(lens[i]))]),
        own_page=_ints([sum(_pages(lens[i]) for i in c[:-1]) for c in lists]), own_len=_ints([n for _, n, _ in nodes]))
    s["most"] = dict(n_nodes=len(nodes), max_new=int(np.diff(q_off).max()), max_ctx_pages=int(np.diff(page_off).max()))
    s["sizes"] = list(zip(np.diff(q_off).tolist(), np.diff(page_off).tolist()))
    s["q"] = _normal(gen, (int(q_off[-1]), case["hq"], d), torch.bfloat16)
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    return s


def _prepare_rows(case, gen, rng):
    lens, forks, ended = _family(case)
    n_rows, width, n_pages = case["rows"], case["width"], _pool_pages(case)
    lines, all_lens, _ = _holders(case)
    perm = rng.permutation(n_pages).astype(np.int32)
    order = rng.permutation(n_rows)  # rows of the table that parents, others and children have
    s = dict(case=case, **_pool(gen, n_pages, case["hkv"], case["d"]))
    table = np.full((n_rows, width), -1, dtype=np.int32)
    row_len = np.zeros(n_rows, dtype=np.int32)
    extra = np.full(n_pages, -1, dtype=np.int32)
    there = len(lines) if case["kind"] == "compact" else len(lens)
    for i in range(there):
        mine = perm[lines[i]]
        table[order[i], :len(mine)] = mine
        row_len[order[i]] = all_lens[i]
        np.add.at(extra, mine, 1)
    free = np.flatnonzero(extra < 0)
    extra = np.maximum(extra, 0)
    stack = np.full(n_pages, -1, dtype=np.int32)
    stack[:len(free)] = rng.permutation(free)
    s.update(table=_ints(table), free_pages=_ints(stack), free_count=_ints([len(free)]), row_len=_ints(row_len), extra=_ints(extra))
    if case["kind"] == "fork":
        s.update(parent=_ints([order[p] for p, _ in forks]), child=_ints(order[len(lens):]), fork_len=_ints([n for _, n in forks]))
        s["most_shared"] = max(n for _, n in forks) // PAGE
        sizes = dict(row_len=n_rows, extra=n_pages, free_count=1, copy_src=len(forks), copy_dst=len(forks), refused=1)
    else:
        flag = np.zeros(n_rows, dtype=np.int32)
        flag[order] = ended
        s["ended"] = _ints(flag)
        sizes = dict(row_len=n_rows, extra_between=n_pages, extra=n_pages, free_count=1, free_pages=n_pages, page_map=n_pages,
                     copy_src=n_pages // 2, copy_dst=n_pages // 2, n_copies=1)
        s["table_out"] = torch.full_like(s["table"], -1)
    s["out"] = {name: torch.full((n,), -1, dtype=torch.int32, device="cuda") for name, n in sizes.items()}
    return s


def _prepare_rotary(case, gen, rng):
    hq, hkv, d, tokens = case["hq"], case["hkv"], case["d"], case["tokens"]
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    s = dict(case=case)
    heads = (hq, hkv, hkv)
    if case["fused"]:  # the output of a projection: query, key and value heads of a token side by side
        s["q"], s["k"], s["v"] = _normal(gen, (tokens, sum(heads), d), dtype).split(heads, 1)
    else:
        s["q"], s["k"], s["v"] = (_normal(gen, (tokens, h, d), dtype) for h in heads)
    if case["to"] == "rows":
        s["pos"] = _ints(rng.integers(0, case["far"], tokens))
        s["q_out"], s["k_out"] = (torch.empty((tokens, h, d), dtype=dtype, device="cuda") for h in (hq, hkv))
        return s
    rows = _stored(case)
    counts = [_pages(old % PAGE + n) for old, n in rows]
    perm = rng.permutation(sum(counts)).astype(np.int64)
    ends = np.cumsum([0] + counts)
    slots, pos = [], []
    for r, (old, n) in enumerate(rows):
        t = old % PAGE + np.arange(n)
        slots.append(perm[ends[r] + t // PAGE] * PAGE + t % PAGE)
        pos.append(int(rng.integers(0, case["far"])) + np.arange(n))
    s.update(_pool(gen, int(ends[-1]), hkv, d), slots=_ints(np.concatenate(slots)), pos=_ints(np.concatenate(pos)))
    for name in ("k_scale", "v_scale"):  # (the scales of an append are powers of two)
        s[name] = torch.exp2(torch.round(torch.log2(s[name])))
    return s


# --------------------------------------------------------------------------- one pass
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"chunk": _own_chunk, "fork": _own_fork, "compact": _own_compact, "rotary": _own_rotary}[kind](s)
    return {"chunk": _plain_chunk, "fork": _plain_fork, "compact": _plain_compact, "rotary": _plain_rotary}[kind](s)


POOLS = ("k_pool", "v_pool", "k_scale", "v_scale")


def _cache(s, B):  # (the handles that a program keeps: the cache, the rows, the description with its workspace, the frequencies)
    if "cache" not in s:
        s["cache"] = B.KvCacheQ8(*(s[n] for n in POOLS))
    return s["cache"]


def _own_chunk(s):
    from paper_2602_07529_amd import binding as B
    cache, plan = _cache(s, B), s.get("plan")
    if plan is None:
        desc = B.PagedPrefillDesc.on_device(**s["most"], **s["desc"])
        need = B.dag_prefill_paged_q8_workspace_bytes(desc, cache, s["q"].shape[0], s["q"].shape[1])
        plan = s["plan"] = desc, torch.empty(max(256, need), dtype=torch.uint8, device="cuda")
    B.dag_attn_prefill_paged_q8(plan[0], s["q"], cache, s["out"], plan[1], lse=s["lse"])
    return s["out"], s["lse"]


def _own_fork(s):
    from paper_2602_07529_amd import binding as B
    cache, o = _cache(s, B), s["out"]
    if "rows" not in s:
        s["rows"] = B.KvRows(s["table"], s["free_pages"])
    B.dag_kv_fork(s["rows"], s["parent"], s["child"], s["row_len"], o["row_len"], s["extra"], o["extra"], s["free_count"], o["free_count"],
                  o["copy_src"], o["copy_dst"], fork_len=s["fork_len"], refused=o["refused"])
    B.dag_kv_copy_pages_q8(cache, o["copy_src"], o["copy_dst"])
    return dict(o, table=s["table"], **{n: s[n] for n in POOLS})


def _own_compact(s):
    from paper_2602_07529_amd import binding as B
    cache, o = _cache(s, B), s["out"]
    if "rows" not in s:
        s["rows"] = B.KvRows(s["table"], s["free_pages"])
        s["rows_out"] = B.KvRows(s["table_out"], o["free_pages"])
    B.dag_kv_release_shared(s["rows"], s["ended"], s["row_len"], o["row_len"], s["extra"], o["extra_between"], s["free_count"], o["free_count"])
    B.dag_kv_compact(s["rows"], s["rows_out"], o["row_len"], o["extra_between"], o["extra"], o["free_count"], o["page_map"], o["copy_src"],
                     o["copy_dst"], o["n_copies"])
    B.dag_kv_copy_pages_q8(cache, o["copy_src"], o["copy_dst"], count=o["n_copies"])
    return dict(o, table=s["table_out"], **{n: s[n] for n in POOLS})


def _own_rotary(s):
    from paper_2602_07529_amd import binding as B
    case, rope = s["case"], s.get("rope")
    if rope is None:
        rope = s["rope"] = B.Rope(case["rotary"], case["theta"], "cuda", layout=B.ROPE_PAIRS if case["layout"] == "pairs" else B.ROPE_HALVES,
                                  stretch=case["stretch"], original=case["original"], factor=case["factor"])
    if case["to"] == "cache":
        B.dag_kv_append_rotary_q8(_cache(s, B), s["slots"], s["pos"], s["k"], s["v"], rope)
        return {n: s[n] for n in POOLS}
    B.dag_rope_apply(rope, s["pos"], s["q"], s["k"], s["q_out"], s["k_out"], transposed=case["back"])
    return s["q_out"], s["k_out"]


# --------------------------------------------------------------------------- plain forms
def _plain_chunk(s):
    """Nodes next to each other together, their lists filled up to the longest one's length, as many as make 10^9 scores."""
    case, c = s["case"], s["desc"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    g = hq // hkv
    at = 0
    while at < len(s["sizes"]):
        end, new, most = at, 0, 0
        while end < len(s["sizes"]):
            n, m = max(new, s["sizes"][end][0]), max(most, s["sizes"][end][1])
            if end > at and (end + 1 - at) * hq * n * m * PAGE > 1e9:
                break
            end, new, most = end + 1, n, m
        off, first = c["ctx_page_off"][at:end + 1].long(), c["q_off"][at:end + 1].long()
        col = torch.arange(most, device="cuda")
        e = (off[:-1, None] + col).clamp(max=c["ctx_pages"].numel() - 1)
        held = torch.where(col < torch.diff(off)[:, None], c["ctx_page_len"].long()[e], 0)  # [node][page]
        p = c["ctx_pages"].long()[e]
        k = s["k_pool"][p].float() * s["k_scale"][p][..., None, None, None]  # [node][page][h][d / 16][slot][16]
        v = s["v_pool"][p].float() * s["v_scale"][p][..., None, None]        # [node][page][h][d][slot]
        n = end - at
        k = k.permute(0, 2, 3, 5, 1, 4).reshape(n, hkv, d, most * PAGE)
        v = v.permute(0, 2, 1, 4, 3).reshape(n, hkv, most * PAGE, d)
        there = (torch.arange(PAGE, device="cuda") < held[..., None]).reshape(n, most * PAGE)
        i = torch.arange(new, device="cuda")
        last = (c["own_page"][at:end].long() * PAGE + c["own_len"][at:end].long() - torch.diff(first))[:, None] + i  # [node][row]
        sees = there[:, None] & (torch.arange(most * PAGE, device="cuda") <= last[..., None])  # [node][row][slot]
        r = (first[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
        q = s["q"][r].float().reshape(n, new, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, g * new, d)
        x = torch.matmul(q, k).mul_(d ** -0.5).reshape(n, hkv, g, new, most * PAGE)
        x.masked_fill_(~sees[:, None, None], -math.inf)
        m = x.amax(-1, keepdim=True).clamp(min=-1e30)
        x = x.sub_(m).exp_()
        total = x.sum(-1)
        o = torch.matmul(x.reshape(n, hkv, g * new, -1), v).reshape(n, hkv, g, new, d)
        o = torch.where(total[..., None] > 0, o / total[..., None].clamp(min=1e-37), 0.0)
        lse = torch.where(total > 0, m[..., 0] + torch.log(total.clamp(min=1e-37)), -math.inf)
        mine = i < torch.diff(first)[:, None]
        s["out"][r[mine]] = o.permute(0, 3, 1, 2, 4).reshape(n, new, hq, d)[mine].to(torch.bfloat16)
        s["lse"][r[mine]] = lse.permute(0, 3, 1, 2).reshape(n, new, hq)[mine]
        at = end
    return s["out"], s["lse"]


def _put(to, mask, at, what):  # (a place behind the list for what is not written)
    to = torch.cat([to.reshape(-1), to.new_zeros(1)])
    to.scatter_(0, torch.where(mask, at, to.numel() - 1).reshape(-1), what.expand(mask.shape).reshape(-1))
    return to[:-1]


def _copied(s, src, dst):
    src, dst = src[src >= 0], dst[dst >= 0]
    for name in POOLS:
        x = s[name].view(torch.uint8) if s[name].dtype == E4M3 else s[name]
        x[dst] = x[src]
    return {n: s[n] for n in POOLS}


def _plain_fork(s):
    parent, child, old, count = s["parent"].long(), s["child"].long(), s["row_len"].long(), s["free_count"].long()
    table, free = s["table"].long(), s["free_pages"].long()
    n = torch.minimum(s["fork_len"].long(), old[parent])
    need = (n % PAGE > 0).long()
    start = torch.cumsum(need, 0) - need
    ok = (need == 0) | (start < count)
    fresh = free[(count - 1 - start).clamp(min=0)]
    col = torch.arange(table.shape[1], device="cuda")
    line = table[parent]
    shared = ok[:, None] & (col < (n // PAGE)[:, None])
    copied = ok & (need > 0)
    src = line.gather(1, (n // PAGE).clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    line = torch.where(shared, line, torch.where(copied[:, None] & (col == (n // PAGE)[:, None]), fresh[:, None], table[child]))
    extra = torch.nn.functional.pad(s["extra"].long(), (0, 1))
    extra.scatter_add_(0, torch.where(shared, line, extra.numel() - 1).reshape(-1), torch.ones_like(line).reshape(-1))
    s["table"][child] = line.int()
    row_len = old.clone()
    row_len[child] = torch.where(ok, n, old[child])
    src, dst = torch.where(copied, src, -1), torch.where(copied, fresh, -1)
    got = dict(row_len=row_len, extra=extra[:-1], free_count=count - copied.sum(), copy_src=src, copy_dst=dst, refused=(~ok).sum()[None], table=s["table"])
    return dict({name: x.int() for name, x in got.items()}, **_copied(s, src, dst))


def _plain_compact(s):
    table, free, count, old, extra = (s[n].long() for n in ("table", "free_pages", "free_count", "row_len", "extra"))
    n_rows, width = table.shape
    n_pages = free.numel()
    col = torch.arange(width, device="cuda")
    held = torch.where(s["ended"] > 0, (old + PAGE - 1) // PAGE, 0)
    gone = col < held[:, None]
    # how often a page is given back, and the last of the places where it is
    to = torch.where(gone, table, n_pages).reshape(-1)
    place = torch.arange(to.numel(), device="cuda")
    times = torch.zeros(n_pages + 1, dtype=torch.int64, device="cuda").scatter_add_(0, to, torch.ones_like(to))
    last = torch.full((n_pages + 1,), -1, dtype=torch.int64, device="cuda").scatter_reduce_(0, to, place, "amax")
    freed = (gone.reshape(-1)) & (last[to] == place) & (times[to] > torch.nn.functional.pad(extra, (0, 1))[to])
    at = torch.cumsum(freed.long(), 0) - 1 + count
    free = _put(free, freed, at, table.reshape(-1))
    s["free_pages"].copy_(free)
    left = count + freed.sum()
    between = (extra - times[:-1]).clamp(min=0)
    row_len = torch.where(s["ended"] > 0, 0, old)
    # pages in use from the number of them on go to the free places in front, both in ascending order
    is_free = torch.zeros(n_pages + 1, dtype=torch.bool, device="cuda")
    is_free[torch.where(torch.arange(n_pages, device="cuda") < left, free, n_pages)] = True
    is_free = is_free[:-1]
    ids = torch.arange(n_pages, device="cuda")
    front = ids < n_pages - left
    src, dst = ids[~is_free & ~front], ids[is_free & front]
    page_map = torch.where(is_free, -1, ids)
    page_map[src] = dst
    new_extra = torch.where(is_free | ~front, 0, between)
    new_extra[dst] = between[src]
    mine = col < ((row_len + PAGE - 1) // PAGE)[:, None]
    s["table_out"].copy_(torch.where(mine, page_map[table.clamp(min=0)], s["table_out"].long()))
    o = s["out"]
    list_out = torch.where(ids < left, n_pages - 1 - ids, o["free_pages"].long())
    pad = lambda x, name: torch.cat([x, o[name][x.numel():].long()])  # noqa: E731
    got = dict(row_len=row_len, extra_between=between, extra=new_extra, free_count=left, free_pages=list_out, page_map=page_map,
               copy_src=pad(src, "copy_src"), copy_dst=pad(dst, "copy_dst"), n_copies=torch.full((1,), src.numel(), device="cuda"), table=s["table_out"])
    return dict({name: x.int() for name, x in got.items()}, **_copied(s, src, dst))


def _frequencies(case):
    """theta^(-2 m / R), divided by the stretch where a pair turns less than once over the original length, as it is where it turns 32 times, and
    in between in proportion (all of them divided if no original length is given)."""
    r = case["rotary"]
    f = case["theta"] ** (torch.arange(r // 2, device="cuda", dtype=torch.float64) * (-2.0 / r))
    keep = torch.zeros_like(f)
    if case["original"] > 0:
        keep = ((case["original"] * f / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
    return keep * f + (1 - keep) * f / case["stretch"]


def _turned(x, pos, case, sign=1.0):
    r = case["rotary"]
    angle = pos.double()[:, None, None] * _frequencies(case) * sign
    c, n = torch.cos(angle) * case["factor"], torch.sin(angle) * case["factor"]
    x = x.double()
    if case["layout"] == "pairs":
        lo, hi = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([lo * c - hi * n, hi * c + lo * n], -1).flatten(-2)
    else:
        lo, hi = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([lo * c - hi * n, hi * c + lo * n], -1)
    return torch.cat([y, x[..., r:]], -1)


def _plain_rotary(s):
    case = s["case"]
    if case["to"] == "cache":
        return _plain_store(s)
    sign = -1.0 if case["back"] else 1.0
    s["q_out"].copy_(_turned(s["q"], s["pos"], case, sign))
    s["k_out"].copy_(_turned(s["k"], s["pos"], case, sign))
    return s["q_out"], s["k_out"]


def _plain_store(s):
    slots = s["slots"].long()
    n_pages, hkv = s["k_scale"].shape
    page, slot = slots // PAGE, slots % PAGE
    begun = torch.zeros(n_pages, dtype=torch.bool, device="cuda")
    begun[page[slot == 0]] = True
    touched = torch.zeros_like(begun)
    touched[page] = True
    for name, x in (("k", _turned(s["k"], s["pos"], s["case"])), ("v", s["v"].double())):
        most = x.new_zeros(n_pages, hkv).scatter_reduce_(0, page[:, None].expand(-1, hkv), x.abs().amax(-1), "amax")
        m, e = torch.frexp(most)  # the smallest k with most <= 448 * 2^k
        e = torch.where(most > 0, torch.where(m <= 0.875, e - 9, e - 8), LEAST).clamp(min=LEAST)
        scale, old = torch.ldexp(torch.ones_like(most), e), s[name + "_scale"].double()
        scale = torch.where(begun[:, None], scale, torch.where(touched[:, None], torch.maximum(scale, old), old))
        keep = torch.where(begun[:, None], 0.0, old / scale)
        pool = s[name + "_pool"]
        codes = (pool.float() * keep.float()[(...,) + (None,) * (pool.dim() - 2)]).to(E4M3)
        mine = (x / scale[page][..., None]).float().to(E4M3).view(torch.uint8)
        codes.view(torch.uint8)[page, :, :, slot] = mine.reshape(len(page), hkv, -1, PAGE) if name == "k" else mine
        pool.copy_(codes)
        s[name + "_scale"].copy_(scale)
    return {n: s[n] for n in POOLS}


# --------------------------------------------------------------------------- 64 bits, written apart
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("fork", "compact"):
        return None
    if case["kind"] == "chunk":
        return _exact_chunk(s)
    return _exact_store(s) if case["to"] == "cache" else _exact_rows(s)


def _exact_chunk(s):
    case, c = s["case"], {n: x.cpu().numpy() for n, x in s["desc"].items()}
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    g = hq // hkv
    out, lse = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for node in range(len(c["own_len"])):
        a, b = int(c["q_off"][node]), int(c["q_off"][node + 1])
        pages, held = (c[n][c["ctx_page_off"][node]:c["ctx_page_off"][node + 1]] for n in ("ctx_pages", "ctx_page_len"))
        at = np.concatenate([PAGE * j + np.arange(n) for j, n in enumerate(held)])  # places of the tokens that are there
        token = torch.from_numpy(at).cuda()
        first = int(c["own_page"][node]) * PAGE + int(c["own_len"][node]) - (b - a)
        p = torch.from_numpy(pages.astype(np.int64)).cuda()
        for h in range(hkv):
            k = (s["k_pool"][p, h].double() * s["k_scale"][p, h].double()[:, None, None, None]).transpose(1, 2).reshape(-1, d)[token]
            v = (s["v_pool"][p, h].double() * s["v_scale"][p, h].double()[:, None, None]).transpose(1, 2).reshape(-1, d)[token]
            kt = k.t().contiguous()
            for r0 in range(a, b, 512):
                r1 = min(b, r0 + 512)
                q = s["q"][r0:r1, h * g:(h + 1) * g].double()
                x = torch.matmul(q.reshape(-1, d), kt).reshape(r1 - r0, g, -1) / math.sqrt(d)
                hidden = token[None] > first + torch.arange(r0 - a, r1 - a, device="cuda")[:, None]
                x = x.masked_fill(hidden[:, None], -math.inf)
                total = torch.logsumexp(x, -1)
                e = torch.nan_to_num(torch.exp(x - total[..., None]), nan=0.0)
                out[r0:r1, h * g:(h + 1) * g] = torch.matmul(e.reshape(-1, e.shape[-1]), v).reshape(r1 - r0, g, d)
                lse[r0:r1, h * g:(h + 1) * g] = total
    return out, lse


def _exact_turned(x, pos, case, back=False):
    """Every pair as a complex number, times factor * e^(i angle)."""
    r, x = case["rotary"], x.double().clone()
    for m in range(r // 2):
        f = case["theta"] ** (-2.0 * m / r)
        if case["stretch"] != 1.0:
            turns = case["original"] * f / (2.0 * math.pi)
            part = min(max((turns - 1.0) / (32.0 - 1.0), 0.0), 1.0) if case["original"] > 0 else 0.0
            f = f * (part + (1.0 - part) / case["stretch"])
        i, j = (2 * m, 2 * m + 1) if case["layout"] == "pairs" else (m, m + r // 2)
        z = torch.polar(torch.full_like(pos, case["factor"], dtype=torch.float64), pos.double() * (-f if back else f))[:, None]
        y = torch.complex(x[..., i].contiguous(), x[..., j].contiguous()) * z
        x[..., i], x[..., j] = y.real, y.imag
    return x


def _exact_rows(s):
    return tuple(_exact_turned(s[n], s["pos"], s["case"], s["case"]["back"]) for n in ("q", "k"))


def _to_e4m3(x):
    """To the nearest of the type's values, ties to even: steps of 2^-3 of a value's power of two, of 2^-9 below 2^-6."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 1).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def _exact_store(s):
    case = s["case"]
    hkv, d = case["hkv"], case["d"]
    slots = s["slots"].cpu().numpy().astype(np.int64)
    fresh = {"k": _exact_turned(s["k"], s["pos"], case), "v": s["v"].double()}
    # the pages that tokens go to, each with its tokens by slot
    page, place = np.unique(slots // PAGE, return_inverse=True)
    token = np.full((len(page), PAGE), -1, dtype=np.int64)
    token[place, slots % PAGE] = np.arange(len(slots))
    token, page = torch.from_numpy(token).cuda(), torch.from_numpy(page).cuda()
    out = {}
    for name in ("k", "v"):
        old = s[name + "_pool"][page].double()
        old = old.transpose(2, 3).reshape(len(page), hkv, PAGE, d) if name == "k" else old.transpose(2, 3)
        there = (token >= 0)[:, None, :, None]
        x = torch.where(there, fresh[name][token.clamp(min=0)].transpose(1, 2), 0.0)
        most = x.abs().amax((2, 3))
        k = torch.ceil(torch.log2(most / TOP))
        k = torch.where(torch.exp2(k - 1) * TOP >= most, k - 1, torch.where(torch.exp2(k) * TOP < most, k + 1, k)).clamp(min=float(LEAST))
        before, begun = s[name + "_scale"][page].double(), (token[:, 0] >= 0)[:, None]
        scale = torch.where(begun, torch.exp2(k), torch.maximum(torch.exp2(k), before))
        kept = torch.where(begun[..., None, None], 0.0, old * (before / scale)[..., None, None])
        codes = _to_e4m3(torch.where(there, x / scale[..., None, None], kept))
        codes = codes.reshape(len(page), hkv, PAGE, d // PAGE, PAGE).transpose(2, 3) if name == "k" else codes.transpose(2, 3)
        pool, scales = s[name + "_pool"].double(), s[name + "_scale"].double()
        pool[page], scales[page] = codes, scale
        out[name + "_pool"], out[name + "_scale"] = pool, scales
    return out

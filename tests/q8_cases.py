"""Contexts over an 8-bit cache for the tests: a pool of random codes, page lists of given lengths, and what the oracle says of them.

How far a kernel may be off: probabilities are rounded to bf16 before the second product (half a step, 2^-8, of every term, so
2^-8 of the result with |V| in the place of V), and so is the result; scores are sums of d products in 32 bits, off by at most
(d + 4) 2^-24 of the sum of their magnitudes, which moves a probability by that much, twice (its sum too); exponentials, the rescaling
and the partial sums add a few 2^-24 each per slice of the context: 2^-17 has room for 32 of them."""
import numpy as np
import torch

from oracle import q8_oracle as q8
from paper_2602_07529_amd import binding as B
from tests.gpu_util import DEV

PAGE = 16


def pages_of(n):
    return -(-int(n) // PAGE)


def ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32).reshape(-1), device=DEV)


def pool(rng, n_pages, hkv, d, scales="powers"):
    """Random codes (every bit pattern of a number), scales of a few magnitudes."""
    x = {}
    for name, shape in (("k", (n_pages, hkv, d // 16, PAGE, 16)), ("v", (n_pages, hkv, d, PAGE))):
        codes = torch.from_numpy((rng.standard_normal(shape) * 60).clip(-448, 448).astype(np.float32)).to(torch.float8_e4m3fn)
        size = 2.0 ** rng.integers(-8, -5, size=(n_pages, hkv)) if scales == "powers" else np.exp(rng.uniform(-6, -4, size=(n_pages, hkv)))
        x[name + "_pool"], x[name + "_scale"] = codes.to(DEV), torch.from_numpy(size.astype(np.float32)).to(DEV)
    return B.KvCacheQ8(x["k_pool"], x["v_pool"], x["k_scale"], x["v_scale"])


def junk_behind(cache, pages, n):
    """Codes that are no number in the slots behind the last token."""
    if n % PAGE:
        cache.k_pool.view(torch.uint8)[int(pages[-1]), :, :, n % PAGE:] = 0x7f
        cache.v_pool.view(torch.uint8)[int(pages[-1]), :, :, n % PAGE:] = 0xff


def values(cache):
    k, v = q8.tokens_of_pools(cache.k_pool.float().cpu().numpy(), cache.v_pool.float().cpu().numpy())
    return k * cache.k_scale.double().cpu().numpy()[..., None, None], v * cache.v_scale.double().cpu().numpy()[..., None, None]


def check(out, q, contexts, cache, scale=None, rows=None):
    d = q.shape[-1]
    rows = range(q.shape[0]) if rows is None else rows
    ref, mass, size = q8.attention(q.double().cpu().numpy()[rows], [contexts[r] for r in rows], *values(cache), d ** -0.5 if scale is None else scale)
    got = out.double().cpu().numpy()[rows]
    assert np.isfinite(got).all()
    room = mass * (2.0 ** -8 + 2 * (d + 4) * 2.0 ** -24 * size + 2.0 ** -17)
    room += 2.0 ** -8 * (np.abs(ref) + room)
    worst = (np.abs(got - ref) / np.maximum(room, 1e-300)).max()
    assert worst <= 1.0, "off by %.3g of what the roundings allow" % worst
    # the roundings are independent of each other: their sum is far below the bound
    norm = np.linalg.norm(ref)
    assert norm == 0 or np.linalg.norm(got - ref) <= 2.0 ** -8 * np.linalg.norm(np.maximum(mass, np.abs(ref)))
    for r, n in enumerate(rows):
        if not any(t > 0 for _, t in contexts[n]):
            assert (got[r] == 0).all()


class Cascade:
    """Sibling groups: [(tokens of the shared context, [tokens of each branch])]."""

    def __init__(self, groups, hq, hkv, d, seed=0, scales="powers", spare=0):
        rng = np.random.default_rng(seed)
        shared, own = [s for s, _ in groups], [n for _, b in groups for n in b]
        counts = [pages_of(n) for n in shared + own]
        ends = np.cumsum([0] + counts)
        perm = rng.permutation(int(ends[-1]) + 1).astype(np.int32)
        self.cache = pool(rng, len(perm), hkv, d, scales)
        lists = [perm[ends[i]:ends[i + 1]] for i in range(len(counts))]
        for pages, n in zip(lists, shared + own):
            junk_behind(self.cache, pages, n)
        g = np.repeat(np.arange(len(groups)), [len(b) for _, b in groups])
        self.contexts = [[(lists[g[r]], shared[g[r]]), (lists[len(shared) + r], own[r])] for r in range(len(own))]
        at = ends[len(shared)]
        most = lambda x: max(list(x) + [0])  # noqa: E731
        self.desc = B.DecodeDesc.on_device(
            len(groups), len(own), most(counts[:len(shared)]) + spare, most(counts[len(shared):]) + spare, most(len(b) for _, b in groups),
            ints(np.cumsum([0] + [len(b) for _, b in groups])), ints(ends[:len(shared) + 1]), ints(perm[:at + 1]), ints(shared),
            ints(ends[len(shared):] - at), ints(perm[at:]), ints(own), ints(own))
        self.q = torch.from_numpy(rng.standard_normal((len(own), hq, d)).astype(np.float32)).to(torch.bfloat16).to(DEV)
        self.out = torch.full_like(self.q, float("nan"))
        self.ws = torch.full((max(256, B.dag_decode_q8_workspace_bytes(self.desc, self.cache, hq)),), 0xff, dtype=torch.uint8, device=DEV)

    def call(self, **kw):
        B.dag_attn_decode_q8(self.desc, self.q, self.cache, self.out, self.ws, **kw)


class Segments:
    """Segments [(tokens, [(reader, tokens it sees)])] of n_live branches."""

    def __init__(self, n_live, segments, hq, hkv, d, seed=0, scales="powers", spare=0, limits=True, shuffle=False):
        rng = np.random.default_rng(seed)
        counts = [pages_of(n) for n, _ in segments]
        ends = np.cumsum([0] + counts)
        perm = rng.permutation(int(ends[-1]) + 1).astype(np.int32)
        self.cache = pool(rng, len(perm), hkv, d, scales)
        self.contexts, entries, flat, sees = [[] for _ in range(n_live)], [[] for _ in range(n_live)], [], []
        for i, (n, readers) in enumerate(segments):
            pages = perm[ends[i]:ends[i + 1]]
            junk_behind(self.cache, pages, n)
            for r, m in readers:
                self.contexts[r].append((pages, min(max(m, 0), n)))
                entries[r].append(len(flat))
                flat.append(r)
                sees.append(m)
        if shuffle:
            for e in entries:
                rng.shuffle(e)
        most = lambda x: max(list(x) + [0])  # noqa: E731
        self.desc = B.SegDecodeDesc.on_device(
            n_live, len(segments), most(counts) + spare, most(len(r) for _, r in segments) + spare, len(flat) + spare, ints(ends), ints(perm),
            ints([n for n, _ in segments]), ints(np.cumsum([0] + [len(r) for _, r in segments])), ints(flat + [0] * (1 + spare)),
            ints(np.cumsum([0] + [len(e) for e in entries])), ints([e for b in entries for e in b] + [0]),
            ints(sees + [0] * (1 + spare)) if limits else None)
        self.q = torch.from_numpy(rng.standard_normal((n_live, hq, d)).astype(np.float32)).to(torch.bfloat16).to(DEV)
        self.out = torch.full_like(self.q, float("nan"))
        self.ws = torch.full((max(256, B.dag_decode_segments_q8_workspace_bytes(self.desc, self.cache, hq)),), 0xff, dtype=torch.uint8, device=DEV)

    def call(self, **kw):
        B.dag_attn_decode_segments_q8(self.desc, self.q, self.cache, self.out, self.ws, **kw)

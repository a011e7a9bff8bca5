"""Chunks of new tokens over an 8-bit cache for the tests: nodes whose contexts are lists of partly filled pages, and what the oracle says."""
import numpy as np
import torch

from paper_2602_07529_amd import binding as B
from tests.gpu_util import DEV
from tests.q8_cases import PAGE, check, ints, pages_of, pool, values


class Chunks:
    """nodes: (tokens of each page in front of the node's own, tokens of its own pages, new ones among them).  With `idle` the q and
    out have that many rows behind the last node's; `spare` is added to the host's bounds."""

    def __init__(self, nodes, hq, hkv, d, seed=0, scales="free", idle=0, spare=0, shared=False, junk=True, q_scale=1.0):
        rng = np.random.default_rng(seed)
        lens = [list(front) + [min(PAGE, own - PAGE * j) for j in range(pages_of(own))] for front, own, _ in nodes]
        total = sum(map(len, lens))
        perm = rng.permutation(total + 3).astype(np.int32)
        if shared:  # all nodes read the pages of the first one in front of their own (lens have to be alike)
            front = len(nodes[0][0])
            at, lists = front, []
            for ln in lens:
                lists.append(np.concatenate([perm[:front], perm[at:at + len(ln) - front]]))
                at += len(ln) - front
        else:
            ends = np.cumsum([0] + [len(x) for x in lens])
            lists = [perm[ends[i]:ends[i + 1]] for i in range(len(nodes))]
        self.cache = pool(rng, total + 3, hkv, d, scales)
        self.lists, self.lens = lists, lens
        for pages, ln in zip(lists, lens):
            for p, n in zip(pages, ln):
                if junk and n < PAGE:
                    self.cache.k_pool.view(torch.uint8)[int(p), :, :, n:] = 0x7f
                    self.cache.v_pool.view(torch.uint8)[int(p), :, :, n:] = 0xff
                if junk and n == 0:
                    self.cache.k_scale[int(p)] = float("nan")
                    self.cache.v_scale[int(p)] = float("inf")
        self.contexts = []
        for (front, own, new), pages, ln in zip(nodes, lists, lens):
            start = PAGE * len(front) + own - new
            for i in range(new):
                self.contexts.append([([int(p)], max(0, min(n, start + i - PAGE * j + 1))) for j, (p, n) in enumerate(zip(pages, ln))])
        q_off = np.cumsum([0] + [new for _, _, new in nodes])
        self.n = int(q_off[-1])
        flat_pages = np.concatenate([np.asarray(x, np.int32) for x in lists] + [np.zeros(1, np.int32)])
        flat_lens = np.concatenate([np.asarray(x, np.int32) for x in lens] + [np.zeros(1, np.int32)])
        self.desc = B.PagedPrefillDesc.on_device(
            len(nodes), max([new for _, _, new in nodes] + [0]) + spare, max([len(x) for x in lens] + [0]) + spare, ints(q_off),
            ints(np.cumsum([0] + [len(x) for x in lens])), ints(flat_pages), ints(flat_lens), ints([len(f) for f, _, _ in nodes]),
            ints([own for _, own, _ in nodes]))
        self.q = (torch.from_numpy(rng.standard_normal((self.n + idle, hq, d)).astype(np.float32)) * q_scale).to(torch.bfloat16).to(DEV)
        self.out = torch.full_like(self.q, 7.0)
        self.lse = torch.full(self.q.shape[:2], 7.0, dtype=torch.float32, device=DEV)
        self.ws = torch.full((max(256, B.dag_prefill_paged_q8_workspace_bytes(self.desc, self.cache, self.n + idle, hq)),), 0xff, dtype=torch.uint8,
                             device=DEV)

    def call(self, **kw):
        kw.setdefault("lse", self.lse)
        B.dag_attn_prefill_paged_q8(self.desc, self.q, self.cache, self.out, self.ws, **kw)

    def check(self, scale=None, rows=None):
        """Against the oracle; rows behind the last node's have to be as they were."""
        rows = list(range(self.n)) if rows is None else list(rows)
        for x in (self.out, self.lse):
            assert (x[self.n:] == 7.0).all()
        check(self.out, self.q, self.contexts, self.cache, scale, rows)
        self.check_lse(scale, rows)

    def check_lse(self, scale, rows):
        """A score is a sum of d products in 32 bits; the sum of the probabilities and its logarithm add a few 2^-24 per stretch, and
        the result, a sum of two terms of its size or less, is rounded."""
        k, _ = values(self.cache)
        d, hkv = self.q.shape[-1], k.shape[1]
        q, got = self.q.double().cpu().numpy(), self.lse.double().cpu().numpy()
        scale = d ** -0.5 if scale is None else scale
        for r in rows:
            for h in range(hkv):
                keys = np.concatenate([k[p, h].reshape(-1, d)[:n] for p, n in self.contexts[r]] + [np.zeros((0, d))])
                for j in range(h * q.shape[1] // hkv, (h + 1) * q.shape[1] // hkv):
                    if not len(keys):
                        assert got[r, j] == -np.inf
                        continue
                    s = keys @ q[r, j] * scale
                    want = s.max() + np.log(np.exp(s - s.max()).sum())
                    size = (np.abs(keys) @ np.abs(q[r, j])).max() * abs(scale)
                    room = (d + 4) * 2.0 ** -24 * size + 2.0 ** -17 + 2.0 ** -22 * (abs(want) + abs(s).max())
                    assert abs(got[r, j] - want) <= room, (r, j, got[r, j], want)

"""Example drivers of the execution phase for ONE attention layer (run_plan, Fork).  run_plan: the host-side scheduler
(dag_sched_*) decides the live transitions of every step, this loop uploads its descriptions and
calls dag_kv_append_rope and dag_attn_decode_segments on the tokens it names.  The "model" is a
table of per-token q / k / v rows (synthetic), so the loop shows the data flow of the engine, not
a language model.  Argument marshalling only: positions, pages, frontiers come from the scheduler,
attention from the kernels."""
import numpy as np
import torch

from . import binding as B


def run_plan(parents, node_len, q_tok, k_tok, v_tok, theta, n_pages=None, chunk=None, softmax_scale=None,
             on_step=None, cache=None, tiled=None):
    """Generates every node of the plan (tokens stored node after node in q_tok [T][hq][d],
    k_tok / v_tok [T][hkv][d], bf16 on the GPU; q already rotated, k rotated by the append at the
    adaptive position).  With `cache` (a KvCacheQ8) the keys and values are held there in 8 bits; n_pages is then its
    number of pages, and steps in which some node has `tiled` new tokens or more (never without it) go through dag_attn_prefill_paged_q8.
    Returns (out [T][hq][d], number of steps, k_pool, v_pool)."""
    dev = q_tok.device
    T, hq, d = q_tok.shape
    hkv = k_tok.shape[1]
    node_len = np.asarray(node_len, dtype=np.int64)
    node_start = np.concatenate([[0], np.cumsum(node_len)])
    if cache is not None:
        n_pages, k_pool, v_pool = cache.c.n_pages, cache.k_pool, cache.v_pool
    else:
        if n_pages is None:
            n_pages = int(np.sum((node_len + 15) // 16))
        k_pool = torch.zeros((n_pages, hkv, d // 8, 16, 8), dtype=q_tok.dtype, device=dev)
        v_pool = torch.zeros((n_pages, hkv, d, 16), dtype=q_tok.dtype, device=dev)
    out = torch.zeros_like(q_tok)
    sch = B.Scheduler(parents, node_len, n_pages, chunk)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=dev)
    n_steps = 0
    zero = np.zeros(1, dtype=np.int32)
    while True:
        st = sch.step()
        if st is None:
            break
        idx = torch.from_numpy(node_start[st["live_node"]] + st["live_token"]).to(dev)
        q, k_new, v_new = q_tok.index_select(0, idx), k_tok.index_select(0, idx), v_tok.index_select(0, idx)
        if cache is not None:
            last = st["branch_len"] - 1
            slots = st["branch_pages"][st["branch_page_off"][:-1] + last // 16] * 16 + last % 16
            B.dag_kv_append_rope_q8(cache, torch.from_numpy(slots).to(dev), torch.from_numpy(st["branch_pos"]).to(dev), k_new,
                                    v_new, theta)
        append = None if cache is not None else dict(n_groups=0, n_live=st["n_live"], page_size=16, group_branch_off=zero, shared_page_off=zero,
                      shared_pages=zero, shared_len=zero, branch_page_off=st["branch_page_off"],
                      branch_pages=st["branch_pages"], branch_len=st["branch_len"], branch_pos=st["branch_pos"])
        if append is not None:
            B.dag_kv_append_rope(B.DecodeDesc(append, dev), k_new, v_new, k_pool, v_pool, theta)
        o = torch.empty_like(q)
        if cache is not None and tiled is not None and np.bincount(st["live_node"]).max() >= tiled:
            pd, order = _paged_of_step(st, dev)
            need = B.dag_prefill_paged_q8_workspace_bytes(pd, cache, len(order), hq)
            if need > ws.numel():
                ws = torch.empty(need, dtype=torch.uint8, device=dev)
            by_node = torch.from_numpy(order).to(dev)
            o_node = torch.empty_like(q)
            B.dag_attn_prefill_paged_q8(pd, q.index_select(0, by_node), cache, o_node, ws, softmax_scale=softmax_scale)
            o.index_copy_(0, by_node, o_node)
            out.index_copy_(0, idx, o)
            n_steps += 1
            if on_step is not None:
                on_step(st)
            continue
        sd = B.SegDecodeDesc(st, dev)
        need = (B.dag_decode_segments_workspace_bytes(sd, hq, hkv, d) if cache is None else
                B.dag_decode_segments_q8_workspace_bytes(sd, cache, hq))
        if need > ws.numel():
            ws = torch.empty(need, dtype=torch.uint8, device=dev)
        if cache is None:
            B.dag_attn_decode_segments(sd, q, k_pool, v_pool, o, ws, softmax_scale=softmax_scale)
        else:
            B.dag_attn_decode_segments_q8(sd, q, cache, o, ws, softmax_scale=softmax_scale)
        out.index_copy_(0, idx, o)
        n_steps += 1
        if on_step is not None:
            on_step(st)
    sch.close()
    return out, n_steps, k_pool, v_pool


def _paged_of_step(st, device):
    """A step of the scheduler as the description of dag_attn_prefill_paged(_q8): a node's context is what its first new token
    reads, its own segment last.  Returns it and the step's entries in the order of its rows."""
    nodes = list(dict.fromkeys(st["live_node"].tolist()))
    rows, pages, lens, page_off, own_page, own_len = [], [], [], [0], [], []
    seg_of_entry = np.repeat(np.arange(st["n_segments"]), np.diff(st["seg_reader_off"]))
    for node in nodes:
        mine = np.flatnonzero(st["live_node"] == node)
        mine = mine[np.argsort(st["live_token"][mine], kind="stable")]
        rows.append(mine)
        r = mine[0]
        segs = [int(seg_of_entry[e]) for e in st["branch_entries"][st["branch_entry_off"][r]:st["branch_entry_off"][r + 1]]]
        segs.sort(key=lambda s: int(st["seg_node"][s]) == node)  # (stable: own pages last)
        for s in segs:
            if int(st["seg_node"][s]) == node:
                own_page.append(len(pages) - page_off[-1])
                own_len.append(int(st["seg_len"][s]))
            ids = st["seg_pages"][st["seg_page_off"][s]:st["seg_page_off"][s + 1]]
            pages += ids.tolist()
            lens += [min(B.PAGE, int(st["seg_len"][s]) - B.PAGE * j) for j in range(len(ids))]
        page_off.append(len(pages))
    desc = dict(page_size=B.PAGE, q_off=np.cumsum([0] + [len(r) for r in rows]), ctx_page_off=page_off, ctx_pages=pages, ctx_page_len=lens,
                own_page=own_page, own_len=own_len)
    return B.PagedPrefillDesc(desc, device), np.concatenate(rows)


class Fork:
    """Sibling branches behind one shared prefix over an 8-bit cache, one layer: pages, slots, positions and descriptions stay on the
    GPU, so that a step is a fixed sequence of calls, captured once (capture=True) and replayed for every token.

    `cache` holds the prefix (appended here: k / v [tokens][hkv][d]) and up to max_len tokens of each of the n_branches; pages are
    handed out from its last one down.  `theta`: of the plain rotation, or a binding.Rope."""

    def __init__(self, cache, k, v, n_branches, max_len, hq, theta, softmax_scale=None, capture=False):
        dev = cache.k_pool.device
        self.cache, self.scale, self.n = cache, softmax_scale, n_branches
        self.rope, self.theta = (theta, None) if isinstance(theta, B.Rope) else (None, float(theta))
        prefix, self.max_len = k.shape[0], max_len
        need = (prefix + 15) // 16 + n_branches * ((max_len + 15) // 16)
        if need > cache.c.n_pages:  # (so no step is ever refused a page)
            raise ValueError("the cache has %d pages, not the %d of the prefix and its branches" % (cache.c.n_pages, need))
        width = max((prefix + 15) // 16, (max_len + 15) // 16)
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
        # row 0 holds the prefix, row 1 + b branch b, whose first position is the fork's
        self.rows = B.KvRows(torch.zeros((1 + n_branches, width), dtype=torch.int32, device=dev),
                             torch.arange(cache.c.n_pages, dtype=torch.int32, device=dev))
        self.len, self.free = ints([0] * (1 + n_branches)), ints([cache.c.n_pages])
        self.pos0, self.one = ints([0] + [prefix] * n_branches), ints([0] + [1] * n_branches)
        self.off, self.slots, self.pos = ints([0] * (2 + n_branches)), ints([0] * n_branches), ints([0] * n_branches)
        self.refused = ints([0])
        self.extra, self.prefix = torch.zeros(cache.c.n_pages, dtype=torch.int32, device=dev), prefix  # (holders of a page besides the first)
        if prefix > 0:
            slots, pos = ints([0] * prefix), ints([0] * prefix)
            B.dag_kv_tables(self.rows, ints([prefix] + [0] * n_branches), self.len, self.len, self.free, self.free, self.off, slots,
                            pos0=self.pos0, pos=pos, refused=self.refused)
            self._append(slots, pos, k, v)
        line = torch.arange(1 + n_branches, dtype=torch.int32, device=dev) * width
        self.desc = B.DecodeDesc.on_device(
            1, n_branches, (prefix + 15) // 16, (max_len + 15) // 16, n_branches, ints([0, n_branches]),
            ints([0, (prefix + 15) // 16]), self.rows.table[0], self.len[:1], line, self.rows.table[1:].reshape(-1), self.len[1:],
            self.pos)
        d = cache.head_dim
        new = lambda h: torch.zeros((n_branches, h, d), dtype=torch.bfloat16, device=dev)  # noqa: E731
        self.q, self.k, self.v, self.out = new(hq), new(cache.hkv), new(cache.hkv), new(hq)
        self.ws = torch.empty(max(256, B.dag_decode_q8_workspace_bytes(self.desc, cache, hq)), dtype=torch.uint8, device=dev)
        self.graph, self.tokens = None, 0
        if capture:
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph):
                self._calls()

    def _append(self, slots, pos, k, v):
        if self.rope is not None:
            B.dag_kv_append_rotary_q8(self.cache, slots, pos, k, v, self.rope)
        else:
            B.dag_kv_append_rope_q8(self.cache, slots, pos, k, v, self.theta)

    def _calls(self):
        B.dag_kv_tables(self.rows, self.one, self.len, self.len, self.free, self.free, self.off, self.slots, pos0=self.pos0,
                        pos=self.pos, refused=self.refused)
        self._append(self.slots, self.pos, self.k, self.v)
        B.dag_attn_decode_q8(self.desc, self.q, self.cache, self.out, self.ws, softmax_scale=self.scale)

    def step(self, q, k, v):
        """One token of every branch: q (rotated) [n][hq][d], k / v [n][hkv][d].  Returns the attention's output, which the next
        step overwrites."""
        if self.tokens == self.max_len:
            raise ValueError("the branches are full")
        if q.shape != self.q.shape or k.shape != self.k.shape or v.shape != self.v.shape:
            raise ValueError("q is %s, k and v are %s" % (list(self.q.shape), list(self.k.shape)))
        self.tokens += 1
        self.q.copy_(q)
        self.k.copy_(k)
        self.v.copy_(v)
        if self.graph is not None:
            self.graph.replay()
        else:
            self._calls()
        return self.out

    def extend(self, q, k, v):
        """Several tokens of every branch at once (a step header): q (rotated) [n][tokens][hq][d], k / v [n][tokens][hkv][d].
        Returns the attention's output [n][tokens][hq][d]."""
        n, m = q.shape[:2]
        if n != self.n or q.shape[2:] != self.q.shape[1:] or k.shape != (n, m) + self.k.shape[1:] or v.shape != k.shape:
            raise ValueError("q is %s, k and v are %s, for the tokens of each branch" % (list(self.q.shape), list(self.k.shape)))
        if self.tokens + m > self.max_len:
            raise ValueError("the branches are full")
        dev = q.device
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
        slots, pos = ints([0] * (n * m)), ints([0] * (n * m))
        B.dag_kv_tables(self.rows, self.one * m, self.len, self.len, self.free, self.free, self.off, slots, pos0=self.pos0, pos=pos,
                        refused=self.refused)
        self._append(slots, pos, k.reshape(n * m, *k.shape[2:]), v.reshape(n * m, *v.shape[2:]))
        self.tokens += m
        # the context of a branch: the pages of the prefix, then its own line of the table
        front, width = (self.prefix + 15) // 16, (self.max_len + 15) // 16
        table = self.rows.table
        pages = torch.cat([table[:1, :front].expand(n, front), table[1:, :width]], 1).contiguous()
        room = torch.cat([self.len[:1].expand(n)[:, None] - ints(range(0, 16 * front, 16)), self.len[1:, None] - ints(range(0, 16 * width, 16))], 1)
        step = front + width
        desc = B.PagedPrefillDesc.on_device(n, m, step, ints(range(0, n * m + 1, max(m, 1)) if m else [0] * (n + 1)), ints(range(0, n * step + 1, step)),
                                            pages.reshape(-1), room.clamp(0, 16).reshape(-1), ints([front] * n), self.len[1:])
        rows, out = q.reshape(n * m, *q.shape[2:]).contiguous(), torch.empty((n * m,) + q.shape[2:], dtype=q.dtype, device=dev)
        ws = torch.empty(max(256, B.dag_prefill_paged_q8_workspace_bytes(desc, self.cache, n * m, q.shape[2])), dtype=torch.uint8, device=dev)
        B.dag_attn_prefill_paged_q8(desc, rows, self.cache, out, ws, softmax_scale=self.scale)
        return out.reshape(q.shape)

    def select(self, parents):
        """Branch b goes on as a copy of branch parents[b]; a branch that others copy has to be its own parent."""
        if len(parents) != self.n or any(not 0 <= p < self.n or parents[p] != p for p in parents):
            raise ValueError("parents are %d branches that are kept" % self.n)
        child = [b for b, p in enumerate(parents) if p != b]
        if not child:
            return
        dev = self.len.device
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
        B.dag_kv_release_shared(self.rows, ints([0] + [int(p != b) for b, p in enumerate(parents)]), self.len, self.len, self.extra, self.extra,
                                self.free, self.free)
        src, dst = ints([0] * len(child)), ints([0] * len(child))
        B.dag_kv_fork(self.rows, ints([1 + parents[b] for b in child]), ints([1 + b for b in child]), self.len, self.len, self.extra, self.extra,
                      self.free, self.free, src, dst, refused=self.refused)
        B.dag_kv_copy_pages_q8(self.cache, src, dst)

    def compact(self):
        """Moves the pages in use to the front of the cache.  Returns the new place of every page (-1: free)."""
        n, dev = self.cache.c.n_pages, self.len.device
        new = lambda m: torch.zeros(m, dtype=torch.int32, device=dev)  # noqa: E731
        page_map, src, dst, count = new(n), new(n // 2), new(n // 2), new(1)
        B.dag_kv_compact(self.rows, self.rows, self.len, self.extra, self.extra, self.free, page_map, src, dst, count)
        B.dag_kv_copy_pages_q8(self.cache, src, dst, count=count)
        return page_map

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
             on_step=None, cache=None):
    """Generates every node of the plan (tokens stored node after node in q_tok [T][hq][d],
    k_tok / v_tok [T][hkv][d], bf16 on the GPU; q already rotated, k rotated by the append at the
    adaptive position).  With `cache` (a KvCacheQ8) the keys and values are held there in 8 bits; n_pages is then its
    number of pages.  Returns (out [T][hq][d], number of steps, k_pool, v_pool)."""
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
        sd = B.SegDecodeDesc(st, dev)
        need = (B.dag_decode_segments_workspace_bytes(sd, hq, hkv, d) if cache is None else
                B.dag_decode_segments_q8_workspace_bytes(sd, cache, hq))
        if need > ws.numel():
            ws = torch.empty(need, dtype=torch.uint8, device=dev)
        o = torch.empty_like(q)
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


class Fork:
    """Sibling branches behind one shared prefix over an 8-bit cache, one layer: pages, slots, positions and descriptions stay on the
    GPU, so that a step is a fixed sequence of calls, captured once (capture=True) and replayed for every token.

    `cache` holds the prefix (appended here: k / v [tokens][hkv][d]) and up to max_len tokens of each of the n_branches; pages are
    handed out from its last one down."""

    def __init__(self, cache, k, v, n_branches, max_len, hq, theta, softmax_scale=None, capture=False):
        dev = cache.k_pool.device
        self.cache, self.theta, self.scale, self.n = cache, float(theta), softmax_scale, n_branches
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
        if prefix > 0:
            slots, pos = ints([0] * prefix), ints([0] * prefix)
            B.dag_kv_tables(self.rows, ints([prefix] + [0] * n_branches), self.len, self.len, self.free, self.free, self.off, slots,
                            pos0=self.pos0, pos=pos, refused=self.refused)
            B.dag_kv_append_rope_q8(cache, slots, pos, k, v, self.theta)
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

    def _calls(self):
        B.dag_kv_tables(self.rows, self.one, self.len, self.len, self.free, self.free, self.off, self.slots, pos0=self.pos0,
                        pos=self.pos, refused=self.refused)
        B.dag_kv_append_rope_q8(self.cache, self.slots, self.pos, self.k, self.v, self.theta)
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

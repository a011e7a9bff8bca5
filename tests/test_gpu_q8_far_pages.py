"""Pages that lie more than 4 GiB into a pool: copies there and back, chunks of few and of many pairs, appends with general rotary positions."""
import numpy as np
import pytest
import torch

from paper_2602_07529_amd import binding as B
from tests.gpu_util import DEV
from tests.q8_cases import ints
from tests.q8_chunk_cases import Chunks

pytestmark = pytest.mark.gpu

POOLS = ("k_pool", "v_pool", "k_scale", "v_scale")


def raw(x):
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def test_copies_and_chunks():
    hkv, d, n_pages = 8, 128, 290000  # 16 KiB a page
    assert (n_pages - 1000) * hkv * d * 16 > 2 ** 32
    c = Chunks([([16] * 5, 40, 1), ([16, 9] * 9, 33, 20), ([16] * 70 + [3], 90, 80), ([], 300, 300)], 32, hkv, d, seed=31)
    small, n = c.cache, c.cache.c.n_pages
    c.call()
    want, want_lse = c.out.clone(), c.lse.clone()
    cache = B.KvCacheQ8.empty(n_pages, hkv, d, DEV)
    near, far = ints(np.arange(n) + 3), ints(n_pages - 1 - 2 * np.arange(n))
    for name in POOLS:
        raw(getattr(cache, name))[3:3 + n] = raw(getattr(small, name))
    B.dag_kv_copy_pages_q8(cache, near, far)
    for name in POOLS:
        assert torch.equal(raw(getattr(cache, name))[far.long()], raw(getattr(small, name)))
        raw(getattr(cache, name))[3:3 + n].zero_()
    c.cache = cache
    pages = c.desc.t["ctx_pages"]
    pages.copy_(far[pages.clamp(0, n - 1).long()])
    c.out.fill_(7.0), c.lse.fill_(7.0)
    c.call()
    assert torch.equal(c.out, want) and torch.equal(c.lse, want_lse)
    B.dag_kv_copy_pages_q8(cache, far, near)
    for name in POOLS:
        assert torch.equal(raw(getattr(cache, name))[3:3 + n], raw(getattr(small, name)))
    # appends: the same tokens near and far
    rope = B.Rope(64, 10000.0, DEV, layout=B.ROPE_PAIRS, factor=1.1)
    at = np.arange(700)
    k, v = (torch.randn((700, hkv, d), device=DEV).to(torch.bfloat16) for _ in range(2))
    pos = ints(at * 3)
    slots = near.cpu().numpy()[at // 16] * 16 + at % 16, far.cpu().numpy()[at // 16].astype(np.int64) * 16 + at % 16
    for s in slots:
        B.dag_kv_append_rotary_q8(cache, ints(s), pos, k, v, rope)
    used = at[-1] // 16 + 1
    for name in POOLS:
        assert torch.equal(raw(getattr(cache, name))[near[:used].long()], raw(getattr(cache, name))[far[:used].long()])


def test_copies_of_bf16_pages():
    hkv, d, n_pages = 8, 128, 140000  # 32 KiB a page
    k = torch.zeros((n_pages, hkv, d // 8, 16, 8), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros((n_pages, hkv, d, 16), dtype=torch.bfloat16, device=DEV)
    k[:40].normal_(), v[:40].normal_()
    near, far = ints(np.arange(40)), ints(n_pages - 1 - np.arange(40))
    B.dag_kv_copy_pages(k, v, near, far)
    for x in (k, v):
        assert torch.equal(x[far.long()], x[:40]) and int(torch.count_nonzero(x[40:200])) == 0

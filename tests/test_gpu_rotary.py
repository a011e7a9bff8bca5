"""dag_rope_apply and dag_kv_append_rotary_q8 against the oracle.

The angle is a product in 64 bits, its cosine and sine are rounded to 32 (half a step, 2^-24 each, and 2^-24 more with the factor), the two
products and their difference in 32 bits add at most 3 x 2^-24 of |x| + |x'|, times the factor: 6 x 2^-24 has room; then the rounding to the type."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as q8
from paper_2602_07529_amd import binding as B
from tests.gpu_util import DEV
from tests.q8_cases import ints

pytestmark = pytest.mark.gpu

SCALED = [dict(theta=10000.0), dict(theta=500000.0, stretch=8.0, original=8192.0, factor=1.2), dict(theta=10000.0, stretch=4.0),
          dict(theta=1e6, stretch=32.0, original=4096.0, low=1.0, high=4.0)]


def oracle_of(x, pos, rotary, pairs, kind, transposed=False):
    kind = dict(kind)
    factor = kind.pop("factor", 1.0)
    return q8.rotary(x.double().cpu().numpy(), pos.cpu().numpy(), q8.frequencies(rotary, **kind), pairs, factor, transposed)


def near(got, x, want, factor):
    size = np.abs(x.double().cpu().numpy())
    room = 6 * 2.0 ** -24 * 2 * size.max(-1, keepdims=True) * max(factor, 1.0)
    room = room + np.abs(want) * (2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24)
    assert (np.abs(got.double().cpu().numpy() - want) <= room).all()


@pytest.mark.parametrize("layout", [B.ROPE_HALVES, B.ROPE_PAIRS])
@pytest.mark.parametrize("d,rotary", [(128, 128), (128, 32), (64, 48), (80, 16), (256, 256)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,hq,hkv", [(1, 3, 1), (77, 5, 2), (2500, 4, 1)])
def test_rotary(layout, d, rotary, dtype, n, hq, hkv):
    kind = SCALED[(d + n + hq) % len(SCALED)]
    gen = torch.Generator(device=DEV).manual_seed(n + d)
    q, k = (torch.randn((n, h, d), device=DEV, generator=gen).to(dtype) for h in (hq, hkv))
    pos = torch.randint(0, 200000, (n,), device=DEV, dtype=torch.int32, generator=gen)
    pos[0] = 0 if n > 1 else 123456789
    rope = B.Rope(rotary, device=DEV, layout=layout, **kind)
    for transposed in (False, True):
        q_out, k_out = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
        B.dag_rope_apply(rope, pos, q, k, q_out, k_out, transposed=transposed)
        for x, y in ((q, q_out), (k, k_out)):
            near(y, x, oracle_of(x, pos, rotary, layout == B.ROPE_PAIRS, kind, transposed), kind.get("factor", 1.0))
            assert torch.equal(y[..., rotary:], x[..., rotary:])
    again, alone = q.clone(), k.clone()
    B.dag_rope_apply(rope, pos, again, None)  # in place, one at a time
    B.dag_rope_apply(rope, pos, None, alone, transposed=True)
    B.dag_rope_apply(rope, pos, q, None, q_out)
    assert torch.equal(again, q_out) and torch.equal(alone, k_out)


def test_parts_of_a_fused_projection():
    n, hq, hkv, d = 300, 4, 2, 64
    x = torch.randn((n, hq + 2 * hkv, d), device=DEV).to(torch.bfloat16)
    keep = x.clone()
    q, k, v = x.split((hq, hkv, hkv), 1)
    pos = torch.arange(n, device=DEV, dtype=torch.int32) * 7
    rope = B.Rope(32, 10000.0, DEV, layout=B.ROPE_PAIRS)
    q_out, k_out = torch.empty((n, hq, d), device=DEV, dtype=x.dtype), torch.empty((n, hkv, d), device=DEV, dtype=x.dtype)
    B.dag_rope_apply(rope, pos, q, k, q_out, k_out)
    assert torch.equal(x, keep)
    B.dag_rope_apply(rope, pos, q, k)
    assert torch.equal(q, q_out) and torch.equal(k, k_out) and torch.equal(v, keep[:, hq + hkv:])


@pytest.mark.parametrize("layout", [B.ROPE_HALVES, B.ROPE_PAIRS])
def test_gradient(layout):
    """Of sum(y . w) with respect to x: the transposed rotation of w; and against differences of the forward call."""
    n, h, d, rotary = 20, 2, 64, 32
    x, w = (torch.randn((n, h, d), device=DEV) for _ in range(2))
    pos = torch.randint(0, 5000, (n,), device=DEV, dtype=torch.int32)
    rope = B.Rope(rotary, 10000.0, DEV, layout=layout, factor=1.5)
    grad = torch.empty_like(w)
    B.dag_rope_apply(rope, pos, w, None, grad, transposed=True)
    for i in (0, 1, 15, 16, 31, 32, 63):
        a, b = x.clone(), x.clone()
        a[..., i] += 1.0
        b[..., i] -= 1.0
        ya, yb = torch.empty_like(x), torch.empty_like(x)
        B.dag_rope_apply(rope, pos, a, None, ya)
        B.dag_rope_apply(rope, pos, b, None, yb)
        diff = ((ya.double() - yb.double()) * w.double()).sum(-1) / 2  # (the call is linear in x)
        room = 2.0 ** -20 * 1.5 * (1 + x.double().abs().max()) * w.double().abs().sum(-1)
        assert ((diff - grad[..., i].double()).abs() <= room).all()


def test_as_the_plain_rotation():
    """Halves of the whole head at a plain table: what dag_rope_qk computes, up to the last bit of an angle's cosine."""
    n, h, d = 500, 3, 128
    x = torch.randn((n, h, d), device=DEV)
    pos = torch.randint(0, 30000, (n,), device=DEV, dtype=torch.int32)
    a, b = x.clone(), x.clone()
    B.dag_rope_qk(pos, a, None, 500000.0)
    B.dag_rope_apply(B.Rope(d, 500000.0, DEV), pos, b, None)
    assert ((a - b).abs() <= 6 * 2.0 ** -24 * 2 * x.abs().amax(-1, keepdim=True)).all()


def test_frequencies_that_the_caller_has():
    n, d = 40, 64
    x = torch.randn((n, 1, d), device=DEV)
    pos = torch.arange(n, device=DEV, dtype=torch.int32)
    freq = np.linspace(2.0, 0.001, 16)
    y = torch.empty_like(x)
    B.dag_rope_apply(B.Rope(32, 1.0, DEV, freq=freq), pos, x, None, y)
    near(y, x, q8.rotary(x.double().cpu().numpy(), pos.cpu().numpy(), freq, False), 1.0)


@pytest.mark.parametrize("layout", [B.ROPE_HALVES, B.ROPE_PAIRS])
@pytest.mark.parametrize("d,rotary", [(128, 128), (128, 64), (128, 32), (64, 32), (64, 64)])
@pytest.mark.parametrize("dtype,n", [(torch.bfloat16, 40), (torch.float32, 40), (torch.bfloat16, 2100)])
def test_append(layout, d, rotary, dtype, n):
    """Rotated keys in the cache: runs over pages, single tokens, partly filled pages, dropped slots."""
    hkv, rng = 3, np.random.default_rng(d + n)
    n_pages = n // 16 + 8
    perm = rng.permutation(n_pages)
    cache = B.KvCacheQ8.empty(n_pages, hkv, d, DEV)
    x = torch.randn((n, 2 * hkv, d), device=DEV).to(dtype)
    k, v = x.split(hkv, 1)
    kind = dict(theta=10000.0, stretch=4.0, original=2048.0, factor=1.1)
    rope = B.Rope(rotary, device=DEV, layout=layout, **kind)
    at = np.arange(n) + 5
    slots = perm[at // 16] * 16 + at % 16
    slots[6] = -1  # left out (the last of its page in its call)
    pos = rng.integers(0, 100000, n).astype(np.int32)
    for a, b in ((0, 7), (11, 27), (27, 28), (28, n)):  # a partly filled first page, whole pages, one token, the rest
        B.dag_kv_append_rotary_q8(cache, ints(slots[a:b]), ints(pos[a:b]), k[a:b], v[a:b], rope)
    codes = {m: np.zeros((n_pages, hkv, 16, d)) for m in "kv"}
    scales = {m: np.ones((n_pages, hkv)) for m in "kv"}
    kr = q8.rotary(k.double().cpu().numpy(), pos, q8.frequencies(rotary, 10000.0, 4.0, 2048.0), layout == B.ROPE_PAIRS, 1.1)
    vr = v.double().cpu().numpy()
    for a, b in ((0, 7), (11, 27), (27, 28), (28, n)):
        q8.append(codes["k"], scales["k"], kr[a:b], slots[a:b])
        q8.append(codes["v"], scales["v"], vr[a:b], slots[a:b])
    got_k, got_v = q8.tokens_of_pools(cache.k_pool.float().cpu().numpy(), cache.v_pool.float().cpu().numpy())
    assert np.array_equal(cache.v_scale.double().cpu().numpy(), scales["v"]) and np.array_equal(got_v, codes["v"])
    assert np.array_equal(cache.k_scale.double().cpu().numpy(), scales["k"])
    # a key whose exact value lies next to a border of two codes may be either
    off = np.abs(got_k - codes["k"])
    step = 2.0 ** np.maximum(np.floor(np.log2(np.maximum(np.abs(codes["k"]), 2.0 ** -6))) - 3, -9) * 1.0001
    assert (off <= 2 * step).all() and (off > 0).mean() < 1e-3


def test_append_as_the_plain_one():
    """Halves of the whole head without a factor: the same codes as dag_kv_append_rope_q8, up to borders."""
    n, hkv, d = 100, 2, 128
    k, v = (torch.randn((n, hkv, d), device=DEV).to(torch.bfloat16) for _ in range(2))
    slots, pos = ints(np.arange(n)), ints(np.arange(n) * 11)
    a, b = (B.KvCacheQ8.empty(7, hkv, d, DEV) for _ in range(2))
    B.dag_kv_append_rope_q8(a, slots, pos, k, v, 500000.0)
    B.dag_kv_append_rotary_q8(b, slots, pos, k, v, B.Rope(d, 500000.0, DEV))
    assert torch.equal(a.v_pool.view(torch.uint8), b.v_pool.view(torch.uint8)) and torch.equal(a.k_scale, b.k_scale)
    assert (a.k_pool.view(torch.uint8) != b.k_pool.view(torch.uint8)).float().mean() < 1e-3

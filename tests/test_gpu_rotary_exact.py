"""What the rotations of 32-bit tensors, and those on the way into the 8-bit cache, do in 64 bits: angles, rotation and factor, then one rounding.

The angle pos * f is off by a few 2^-53 of itself (the table's f and its turns, the product with the position; the oracle's own too: 2^-50 has room), its
cosine and sine by 2e-14 of the series more; that times |x| + |x'| and the factor, and the rounding to 32 bits, 2^-24 of the result."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as q8
from paper_2602_07529_amd import binding as B
from tests.gpu_util import DEV
from tests.q8_cases import ints

pytestmark = pytest.mark.gpu


def in_64_bits(x, pos, freq, pairs, factor):
    """How far the rotation may be off in front of its rounding, per element."""
    half = len(freq)
    i = 2 * np.arange(half) if pairs else np.arange(half)
    j = i + 1 if pairs else i + half
    size = np.abs(x)
    room = np.zeros(x.shape)
    off = (np.abs(np.asarray(pos, dtype=np.float64))[:, None, None] * freq * 2.0 ** -50 + 3e-14) * factor
    room[..., i] = room[..., j] = (size[..., i] + size[..., j]) * off
    return room


@pytest.mark.parametrize("layout", [B.ROPE_HALVES, B.ROPE_PAIRS])
@pytest.mark.parametrize("d,rotary,kind", [(128, 128, dict(theta=10000.0)), (128, 32, dict(theta=500000.0, stretch=8.0, original=8192.0, factor=1.2)),
                                           (64, 48, dict(theta=10000.0, stretch=4.0, factor=1.35)), (256, 256, dict(theta=1e6))])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("n", [1, 500, 2500])
def test_rows_of_32_bits_are_rounded_once(layout, d, rotary, kind, transposed, n):
    gen = torch.Generator(device=DEV).manual_seed(n + d)
    x = torch.randn((n, 3, d), device=DEV, generator=gen)
    pos = torch.randint(0, 200000, (n,), device=DEV, dtype=torch.int32, generator=gen)
    y = torch.empty_like(x)
    B.dag_rope_apply(B.Rope(rotary, device=DEV, layout=layout, **kind), pos, x, None, y, transposed=transposed)
    kind = dict(kind)
    factor = kind.pop("factor", 1.0)
    freq, pairs, a, at = q8.frequencies(rotary, **kind), layout == B.ROPE_PAIRS, x.double().cpu().numpy(), pos.cpu().numpy()
    want = q8.rotary(a, at, freq, pairs, factor, transposed)
    assert (np.abs(y.double().cpu().numpy() - want) <= np.abs(want) * 2.0 ** -24 + in_64_bits(a, at, freq, pairs, factor)).all()


@pytest.mark.parametrize("layout", [B.ROPE_HALVES, B.ROPE_PAIRS])
@pytest.mark.parametrize("d,rotary", [(128, 64), (64, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_codes_are_those_of_the_exact_rotation(layout, d, rotary, dtype):
    """Whole pages, parts of pages and single tokens in one call.  A code may only be another one where a border between two codes lies within the
    rounding to 32 bits (2^-24 of the value) and what the rotation in 64 bits is off by."""
    hkv, factor, rng = 8, 1.1, np.random.default_rng(d)
    slots = np.concatenate([np.arange(64 * 16), 64 * 16 + np.arange(60) // 7 * 16 + np.arange(60) % 7, (80 + np.arange(300)) * 16])
    n = len(slots)
    pos = rng.integers(0, 100000, n).astype(np.int32)
    x = torch.randn((n, 2 * hkv, d), device=DEV, generator=torch.Generator(device=DEV).manual_seed(d)).to(dtype)
    k, v = x.split(hkv, 1)
    cache = B.KvCacheQ8.empty(380, hkv, d, DEV)
    rope = B.Rope(rotary, 10000.0, DEV, layout=layout, stretch=4.0, original=2048.0, factor=factor)
    B.dag_kv_append_rotary_q8(cache, ints(slots), ints(pos), k, v, rope)
    pairs, freq, a = layout == B.ROPE_PAIRS, q8.frequencies(rotary, 10000.0, 4.0, 2048.0), k.double().cpu().numpy()
    exact = q8.rotary(a, pos, freq, pairs, factor)
    off = np.abs(exact) * 2.0 ** -24 + in_64_bits(a, pos, freq, pairs, factor)
    off[..., rotary:] = 0.0  # (these stay as they are, and bf16 values do lie on borders)
    got, _ = q8.tokens_of_pools(cache.k_pool.float().cpu().numpy(), cache.v_pool.float().cpu().numpy())
    scale = cache.k_scale.double().cpu().numpy()[slots // 16]  # [token][head]
    got = got[slots // 16, :, slots % 16]
    most = np.zeros((380, hkv))
    np.maximum.at(most, slots // 16, np.abs(exact).max(-1))
    assert all(scale[t, h] == q8.scale_for(most[slots[t] // 16, h]) for t in range(n) for h in range(hkv))
    lo, hi = (q8.e4m3(np.clip((exact + s * off) / scale[..., None], -448, 448)) for s in (-1, 1))
    assert ((lo <= got) & (got <= hi)).all()
    assert (lo != hi).mean() < 1e-5

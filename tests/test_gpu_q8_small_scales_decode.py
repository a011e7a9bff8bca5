"""Decode over an 8-bit cache whose pages have tiny value scales (see the cases of chunks for the pages).  What a sum could lose of keys on pages of zeros
cannot show: a slice has 256 pages at most, so 2^12 keys 2^-26 of the largest, 2^-14 of a result that is rounded to bf16."""
import numpy as np
import pytest
import torch

from paper_2602_07529_amd import binding as B
from tests.gpu_util import DEV
from tests.q8_cases import ints
from tests.test_gpu_q8_small_scales import NOTHING, SCALE, SMALL, SMALL_ROOM, TOP_OF_SMALL, cache_of, close, counts, of_small, pages_of, queries

pytestmark = pytest.mark.gpu


def decode(form, cache, pages, hq, d, spare=0):
    """One branch that reads the list, and a token of its own that does not count."""
    q, n = queries(1, hq, d), len(pages)
    out = torch.full_like(q, 7.0)
    both = ints(np.concatenate([pages, [NOTHING]]))
    if form == "cascade":
        desc = B.DecodeDesc.on_device(1, 1, n + spare, 1 + spare, 1, ints([0, 1]), ints([0, n]), both, ints([16 * n]), ints([0, 1]), ints([NOTHING]), ints([1]),
                                      ints([0]))
        need, call = B.dag_decode_q8_workspace_bytes, B.dag_attn_decode_q8
    else:
        desc = B.SegDecodeDesc.on_device(1, 2, n + spare, 1, 2, ints([0, n, n + 1]), both, ints([16 * n, 1]), ints([0, 1, 2]), ints([0, 0]), ints([0, 2]),
                                         ints([0, 1]), ints([16 * n, 1]) if form == "limits" else None)
        need, call = B.dag_decode_segments_q8_workspace_bytes, B.dag_attn_decode_segments_q8
    ws = torch.full((max(256, need(desc, cache, hq)),), 0xff, dtype=torch.uint8, device=DEV)
    call(desc, q, cache, out, ws, softmax_scale=SCALE)
    return out[0].double().cpu().numpy()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", ["cascade", "segments", "limits"])
@pytest.mark.parametrize("spare", [0, 100000])  # (one launch, or slices and a merge)
def test_decode_over_tiny_values(form, d, spare):
    cache = cache_of(d)
    pages = pages_of(10, SMALL, TOP_OF_SMALL, 10)
    out = decode(form, cache, pages, 4, d, spare)
    want = of_small(*counts(pages, SMALL, 160))
    close(out, want, want * SMALL_ROOM)

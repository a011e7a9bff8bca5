"""CPU: every array that a call over the 8-bit cache reads is on the device that is looked at, whichever of them the description has."""
import pytest
import torch

from paper_2602_07529_amd import binding as B


class Seen(Exception):
    pass


def _ints(n):
    return torch.zeros(n, dtype=torch.int32)


SHARED = dict(group_branch_off=_ints(2), shared_page_off=_ints(2), shared_pages=_ints(4), shared_len=_ints(1))
OWN = dict(branch_page_off=_ints(4), branch_pages=_ints(4), branch_len=_ints(3))
SEGMENTS = dict(seg_page_off=_ints(2), seg_pages=_ints(4), seg_len=_ints(1), seg_reader_off=_ints(2), seg_readers=_ints(3))
ENTRIES = dict(branch_entry_off=_ints(4), branch_entries=_ints(3))
NONE = dict.fromkeys(SEGMENTS)


@pytest.mark.parametrize("arrays", [{**SHARED, **OWN}, OWN, SHARED, {**SEGMENTS, **ENTRIES}, {**NONE, **ENTRIES}], ids=["both", "own", "shared", "segments", "entries"])
def test_an_array_of_the_description_is_looked_at(arrays, monkeypatch):
    def here(*tensors):
        raise Seen([x.data_ptr() for x in tensors])

    monkeypatch.setattr(B, "_here", here)
    if "branch_entry_off" in arrays:
        desc, call = B.SegDecodeDesc.on_device(3, 1 if arrays["seg_len"] is not None else 0, 1, 3, 3, **arrays), B.dag_attn_decode_segments_q8
    else:
        shared, own = "shared_len" in arrays, "branch_len" in arrays
        desc, call = B.DecodeDesc.on_device(int(shared), 3, int(shared), int(own), 3, **arrays), B.dag_attn_decode_q8
    q = torch.zeros((3, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(Seen) as seen:
        call(desc, q, B.KvCacheQ8.empty(4, 2, 64, "cpu"), q.clone(), torch.zeros(256, dtype=torch.uint8))
    assert set(seen.value.args[0]) & {x.data_ptr() for x in arrays.values() if x is not None}

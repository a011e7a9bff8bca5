"""CPU: batches of very many nodes that one launch still holds are taken, more are refused."""
import pytest

from paper_2602_07529_amd import binding as B
from tests.test_q8_more_refusals import FAKE, chunk, kv


@pytest.mark.parametrize("nodes,new,rows,hq,hkv,taken", [
    (2 ** 18, 100, 2 ** 18, 8, 8, True), (2 ** 18, 1, 2 ** 18, 32, 8, True), (2 ** 20, 1, 2 ** 20, 8, 8, True), (2 ** 18 + 1, 129, 2 ** 18, 8, 8, False),
    (2 ** 18, 200, 2 ** 26, 8, 8, True), (2 ** 10, 2 ** 18, 2 ** 28, 8, 8, False)])
def test_very_many_nodes(nodes, new, rows, hq, hkv, taken):
    """(Without queries: what is taken is refused for these.)"""
    assert B.lib().dag_attn_prefill_paged_q8(chunk(nodes=nodes, new=new, pages=10), kv(hkv=hkv, d=64), 0, rows, FAKE, 0, hq, 0.1, FAKE, 2 ** 62,
                                             None) == (-1 if taken else -7)

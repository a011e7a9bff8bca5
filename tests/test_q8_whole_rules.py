"""CPU: which 8-bit decode steps take one launch where siblings share pages: every branch reads them for itself then."""
import pytest

from paper_2602_07529_amd import binding as B
from tests import q8_rules


def whole(groups, live, shared, own, size, hq, hkv, d):
    return bool(q8_rules.plan(B.dag_decode_desc_t(groups, live, 16, shared, own, size), hq, hkv, d).whole)


@pytest.mark.parametrize("groups,live,shared,own,size,hq,hkv,d,taken", [
    (1, 256, 90, 5, 256, 4, 1, 128, False), (64, 256, 90, 5, 4, 4, 1, 128, False), (32, 128, 90, 5, 4, 8, 2, 128, False),  # three to six times the pages
    (2, 32, 90, 5, 16, 8, 8, 128, False), (1, 32, 90, 5, 32, 8, 8, 64, False),                                            # a merge of few rows
    (8, 32, 90, 5, 4, 32, 8, 128, True), (32, 128, 90, 5, 4, 16, 2, 128, True),                                           # siblings meet in an L2, a large merge
    (256, 256, 90, 5, 1, 4, 1, 128, True), (0, 128, 0, 95, 0, 8, 2, 128, True), (32, 128, 50, 50, 4, 8, 2, 128, True),    # hardly anything shared
    (32, 128, 36, 5, 4, 8, 2, 128, True), (1, 16, 36, 5, 16, 8, 2, 128, True),                                            # few pages
    (64, 256, 36, 5, 4, 8, 2, 64, False), (16, 256, 20, 2, 16, 8, 2, 64, True), (4, 64, 36, 5, 16, 32, 8, 64, True), (4, 64, 36, 5, 16, 8, 8, 64, False)])
def test_steps_whose_siblings_share_pages(groups, live, shared, own, size, hq, hkv, d, taken):
    assert whole(groups, live, shared, own, size, hq, hkv, d) is taken


@pytest.mark.parametrize("live,segments,pages,readers,total,hkv,d,taken", [
    (32, 64, 128, 1, 64, 8, 128, False), (32, 64, 128, 1, 64, 8, 64, False), (3, 18, 63, 1, 18, 8, 128, False),  # one branch has most of the segments
    (32, 64, 31, 1, 64, 8, 128, True), (3, 6, 39, 3, 12, 8, 128, True), (32, 41, 63, 32, 128, 8, 128, True), (16, 11, 80, 16, 48, 8, 128, True),
    (1, 4, 64, 1, 4, 8, 128, True), (1, 5, 64, 1, 5, 8, 128, False), (1, 64, 6, 1, 64, 1, 64, True)])
def test_frontiers_with_a_branch_of_many_segments(live, segments, pages, readers, total, hkv, d, taken):
    assert q8_rules.segments_whole(B.dag_decode_seg_desc_t(live, segments, 16, pages, readers, total), hkv, d) is taken

"""Host-side check of dip_sample's workspace: it goes by the rows' length, not by the longest list alone."""
import paper_2412_01380_amd as D


def test_workspace_goes_by_the_vocabulary():
    # (a row's list has no more words than the row)
    one = lambda v: D.dip_sample_workspace_bytes(1000, v) / 1000
    assert one(40) <= one(4096) - 8 * (4096 - 40) + 1 and one(4096) <= one(8192) - 8 * 4096 + 1
    assert one(40) < 10000

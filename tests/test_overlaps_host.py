"""Arrays of a selection or a compaction that may not lie over each other: refused on the host, before any launch."""
import pytest

import paper_2405_03917_amd as cq
from test_bounded_host import E, select

KEPT_END = 4 * 2 * 4 * 100


@pytest.mark.parametrize("t", [300, 20000])
def test_selection_in_arrays_that_overlap(t):
    a = dict(w=0x1000000, kept=0x2000000, lens=0x3000000, ws=0x4000000, seq=0x5000000, t=t, stride=20480)
    w_end, ws_end = 4 * (7 * 20480 + t), cq.cq_select_workspace_bytes(2, 4, t)

    def refused(**kw):
        return select(**{**a, **kw}) == E

    assert refused(lens=a["seq"])                           # lengths are not updated in place: other workgroups still read them
    assert refused(seq=a["lens"] + 4)
    assert refused(kept=a["w"])
    assert refused(kept=a["w"] + w_end - 16)
    assert refused(kept=a["w"] - KEPT_END + 16)
    assert refused(lens=a["w"] + w_end - 16)
    assert refused(lens=a["kept"] + KEPT_END - 16)
    assert refused(seq=a["kept"] + KEPT_END - 4)
    if t > 8192:                                            # (shorter streams use no workspace)
        for name, size in (("w", w_end), ("kept", KEPT_END), ("lens", 8), ("seq", 8)):
            assert refused(ws=a[name] - (ws_end - 16) // 16 * 16)
            assert refused(ws=a[name] + (size - 1) // 16 * 16), name

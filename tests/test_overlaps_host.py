"""Arrays of a selection or a compaction that may not lie over each other: refused on the host, before any launch."""
import pytest

import paper_2405_03917_amd as cq
from test_bounded_host import COMPACT, E, compact, fmt_of, select

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


def test_compaction_in_arrays_that_overlap():
    size, out = cq.cq_cache_bytes(fmt_of(), 2, 512), cq.cq_cache_bytes(fmt_of(), 2, 128)
    ends = dict(k=size, v=size, w=4 * (7 * 512 + 300), kept=4 * 2 * 4 * 100, lens=8, k2=out, v2=out, w2=4 * (7 * 512 + 128))
    a = {name: COMPACT[name] for name in ends}
    work = cq.cq_compact_workspace_bytes(fmt_of(), 2, 100)
    for write, used in (("k2", out), ("v2", out), ("w2", ends["w2"])):
        for name, end in ends.items():
            if name != write:
                assert compact(**{write: a[name] + (end - 1) // 16 * 16}) == E, (write, name)
                assert compact(**{write: a[name] - (used - 1) // 16 * 16}) == E, (write, name)
    # in place: the workspace and everything else
    in_place = dict(k2=a["k"], v2=a["v"], w2=a["w"], cap2=512)
    for name in ("k", "v", "w", "kept", "lens"):
        assert compact(**in_place, ws=a[name] + (ends[name] - 1) // 16 * 16) == E, name
        assert compact(**in_place, ws=a[name] - (work - 1) // 16 * 16) == E, name
    for name, end in (("kept", ends["kept"]), ("lens", 8)):
        for over in ("k", "v", "w"):
            assert compact(**in_place, **{name: a[over] + (ends[over] - 1) // 16 * 16}) == E, (name, over)

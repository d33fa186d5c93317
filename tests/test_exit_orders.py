"""What the kernels do with their barriers when a bounded wait runs out for some warps and not for others, played through on the CPU for every
choice of warps: each order of barriers has to end.  (A wait that runs out belongs to a warp: the next warp may see the phase end in time.)"""
import itertools

import pytest


def play(warps):
    """warps: {(cta, warp): generator of barriers}.  A generator yields ("bar", id, warps, vote) or ("cluster",) and is sent whether any vote at
    that barrier was true; a cluster's barrier opens when every warp that has not exited stands at it.  True: all of them end."""
    at = {}
    for k, g in list(warps.items()):
        at[k] = next(g, None)
    while True:
        live = {k: b for k, b in at.items() if b is not None}
        if not live:
            return True
        groups = {}
        for k, b in live.items():
            groups.setdefault(("cluster",) if b[0] == "cluster" else (k[0], b[1]), []).append(k)
        opened = [(g, ks) for g, ks in groups.items() if (len(ks) == len(live) if g == ("cluster",) else len(ks) == at[ks[0]][2])]
        if not opened:
            return False
        for g, ks in opened:
            vote = g != ("cluster",) and any(at[k][3] for k in ks)
            for k in ks:
                try:
                    at[k] = warps[k].send(vote)
                except StopIteration:
                    at[k] = None


def leave_cluster(ok, n):
    if (yield ("bar", 2, n, not ok)):
        yield ("cluster",)


def leave_by_oneself(ok, n):
    """The order that does not end: every warp decides for itself."""
    if not ok:
        yield ("cluster",)
    yield ("bar", 2, n, False)


def exits(leave, first, second):
    n = len(first)
    return play({(c, w): leave(ok, n) for c, oks in enumerate((first, second)) for w, ok in enumerate(oks)})


def test_a_cluster_is_left_whoever_gave_up():
    for first in itertools.product([True, False], repeat=4):
        for second in itertools.product([True, False], repeat=4):
            assert exits(leave_cluster, first, second), (first, second)


def test_deciding_by_oneself_does_not_end():
    assert exits(leave_by_oneself, (True,) * 4, (True,) * 4) and exits(leave_by_oneself, (False,) * 4, (True,) * 4)
    assert not exits(leave_by_oneself, (True, False, True, True), (True,) * 4)


def epilogue(fails_at, tiles, n, stay):
    """The epilogue warps of the GEMM kernels: two barriers around the staging of a tile's column terms, then a wait."""
    ok = True
    for tile in range(tiles):
        yield ("bar", 1, n, False)
        yield ("bar", 1, n, False)
        ok = ok and tile != fails_at
        if not ok and not stay:
            break
    yield ("bar", 0, n, False)


@pytest.mark.parametrize("tiles", [1, 3])
def test_epilogue_warps_meet_whoever_gave_up(tiles):
    for fails in itertools.product([None] + list(range(tiles)), repeat=4):
        assert play({(0, w): epilogue(f, tiles, 4, True) for w, f in enumerate(fails)}), fails


def test_leaving_the_loop_of_tiles_does_not_end():
    assert play({(0, w): epilogue(0, 3, 4, False) for w in range(4)})
    assert not play({(0, w): epilogue(0 if w == 2 else None, 3, 4, False) for w in range(4)})

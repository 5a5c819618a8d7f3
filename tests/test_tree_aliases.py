"""Lengths that a call writes while others of its workgroups still read: refused on the host."""
import ctypes as C

import pytest

from paper_2512_01278_amd import binding as pb
from tests.test_abi import FAKE, good_kv, lib  # noqa: F401  (a fixture)

APART = [FAKE * k for k in range(2, 12)]


def around(address, span, mine):
    """Places of `mine` bytes that share at least one entry of four bytes with `span` bytes at `address`: its first, middle and last, and all of it."""
    return [address, address - mine + 4, address + span - 4, address + (span - mine) // 8 * 4]


@pytest.mark.parametrize("batch,M", [(1, 1), (2, 5), (7, 64)])
def test_commit_writes_over_nothing_that_it_reads(lib, batch, M):  # noqa: F811
    """Head 0 leaves the new length of a request while the workgroups of other heads read the request's length, tree size, path and its length."""
    sizes, path, lens, now, seq = APART[:5]
    kv = good_kv(batch=batch, seq_lens=seq)

    def tc(now, sizes=sizes, m=M):
        return lib.pillar_tree_commit(C.byref(kv), sizes, 8, path, lens, m, now, None, 0, None)
    mine = 4 * batch
    for address, span in ((seq, mine), (sizes, mine), (lens, mine), (path, mine * M)):
        for place in around(address, span, mine):
            assert tc(place) == pb.PILLAR_EINVAL, (hex(address), place - address)


@pytest.mark.parametrize("batch", [2, 3, 64])
def test_eviction_writes_over_whole_arrays_or_none(lib, batch):  # noqa: F811
    """New lengths may replace the lengths, the old lengths or the budgets, but not those of other requests."""
    old, budgets, now, seq = APART[:4]
    kv = good_kv(batch=batch, seq_lens=seq)

    def ev(now):
        return lib.pillar_evict_kv(C.byref(kv), FAKE, 1024, 0.5, old, budgets, 4, 64, FAKE, FAKE, 1024, now, FAKE, 1 << 40, None)
    for address in (old, budgets, seq):
        for step in (4, 4 * batch - 4, 2 * batch):
            assert ev(address + step) == ev(address - step) == pb.PILLAR_EINVAL, (hex(address), step)

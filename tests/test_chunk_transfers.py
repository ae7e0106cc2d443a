"""CPU model of where the chunk attention's tile transfers read, restated from
its description (no code is shared with the kernel).

An item's keys [kb, ke) come in 32-key blocks; a stage j of the ring takes K of
tile j and V of tile j - 1, dealt to the waves in (matrix, 32-key half) units,
also for tiles that the item does not have (the ring starts full, and the last
stage has V alone).  A unit reads 32 rows from the place of its block's first
key in that key's page on; blocks behind the item's last one stand where that
one does.  Checked: the 32 rows lie in one page, one that the item's request has,
whatever the buffer's bounds leave out of them."""
import random

import pytest


def reads(kb, ke, page, tile, waves, first_key, stages=2):
    """(logical page, first row in it) of every unit of every stage."""
    halves = tile // 32
    units = 2 * halves // waves
    ntiles = -(-(ke - kb) // tile)
    before = [(0, 0)] * waves              # a second unit reads where the first one read last
    for j in range(max(ntiles + 1, stages)):
        for w in range(waves):
            is_v, half = divmod(w * units, halves)
            block = halves * max(j - 1 if is_v else j, 0) + half
            t = first_key(kb + 32 * block, ke)
            now = (t // page, t % page)
            yield now
            if units > 1:
                yield before[w]
            before[w] = now


@pytest.mark.parametrize("tile,waves", [(64, 4), (32, 1)])
def test_every_transfer_stays_in_a_page_of_the_request(tile, waves):
    rng = random.Random(5)
    for _ in range(3000):
        page = 32 * rng.randint(1, 8)
        keys = rng.choice([1, rng.randint(1, 70), rng.randint(1, 3000)])
        kb = 64 * rng.randint(0, (keys - 1) // 64)
        ke = min(keys, kb + 64 * rng.randint(1, 50))
        for pg, row in reads(kb, ke, page, tile, waves, lambda t, ke: min(t, (ke - 1) & ~31)):
            assert 0 <= pg <= (keys - 1) // page and 0 <= row and row + 32 <= page, (page, kb, ke, pg, row)


def test_blocks_behind_the_end_at_the_last_key_would_leave_the_page():
    """What the rule is for: 60 keys in pages of 64, the blocks behind them
    standing at key 59 and not at key 32."""
    far = [row + 32 for _, row in reads(0, 60, 64, 64, 4, lambda t, ke: min(t, ke - 1))]
    assert max(far) > 64

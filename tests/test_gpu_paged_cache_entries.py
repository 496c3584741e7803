"""Entries of the paged cache's calls that are padding, or that say less than an extend before them."""
import pytest
import torch

from paged_model import D
from test_gpu_paged_cache import Pair, _refused, ints, offsets, tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", ["fork", "copy"])
def test_an_entry_without_a_source_leaves_its_target_to_others(what):
    """Padding may name any target: it is passed over, and the entry behind it that names the same one is not a second one."""
    p = Pair(n_layers=2, n_kv=2, max_seqs=6, max_ctx=256, n_pages=40)
    p.grow([0, 1], [100, 37])
    call = getattr(p.c, what)
    call(ints([-1, 0, -1, 1, 0, -1]), ints([2, 2, 3, 3, -1, 0]))
    getattr(p.m, what)([0, 1], [2, 3])
    p.check_tables()                                     # (and nothing is reported)
    p.check_contents()
    call(ints([0, -1, 1]), ints([4, 4, 4]))              # twice all the same
    getattr(p.m, what)([0], [4])
    _refused(p, "passed over")
    p.check_tables()
    p.check_contents()


def test_rows_that_bring_none_of_the_tokens_they_have_room_for_are_reported():
    """An extend made room for tokens and the append's offsets leave them out: some rows, all of them, behind the last token that there is."""
    p = Pair(n_layers=2, n_kv=2, max_seqs=4, max_ctx=256, n_pages=40)
    p.grow([0, 1], [40, 20])
    p.c.extend(ints([0, 1, 2]), offsets([4, 33, 2]))
    assert p.m.extend([0, 1, 2], [4, 33, 2])
    k, v = tokens(p.gen, 39, 2, "bf16")
    none = k[:0].cuda()
    for cu, n in (([0, 4, 37, 37], 37), ([0, 0, 33, 35], 35), ([0, 0, 0, 0], 0), ([0, 0, 0, 0], 39), ([0, 4, 40, 40], 4)):
        p.c.append(1, ints([0, 1, 2]), k[:n].cuda() if n else none, v[:n].cuda() if n else none, ints(cu))
        _refused(p, "passed over")
        # (a row that was right has its tokens in this layer now: the same ones again with another extend)
        p.c.free(ints([0, 1, 2])), p.m.free([0, 1, 2])
        p.grow([0, 1], [40, 20])
        p.c.extend(ints([0, 1, 2]), offsets([4, 33, 2]))
        assert p.m.extend([0, 1, 2], [4, 33, 2])
    for layer in range(2):
        p.c.append(layer, ints([0, 1, 2]), k.cuda(), v.cuda(), offsets([4, 33, 2]))
        p.m.append(layer, [0, 1, 2], [4, 33, 2], k, v)
    p.check_tables()
    p.check_contents()


def test_rows_without_tokens_are_nothing_to_report():
    """Room for none, asked for or not; padding; a slot that another call has made room for."""
    p = Pair(n_layers=1, n_kv=2, max_seqs=4, max_ctx=256, n_pages=40)
    p.grow([0, 1, 2], [40, 0, 5])
    p.grow([0, 2], [0, 0])
    k, v = tokens(p.gen, 3, 2, "bf16")
    p.c.extend(ints([3, 0, -1, 1]), offsets([0, 3, 0, 0]))
    assert p.m.extend([0], [3])
    p.c.append(0, ints([3, 0, -1, 1]), k.cuda(), v.cuda(), offsets([0, 3, 0, 0]))
    p.m.append(0, [0], [3], k, v)
    p.c.append(0, ints([1, 2, 0]), k[:0].cuda(), k[:0].cuda(), offsets([0, 0, 0]))      # (slot 0 has been row 1)
    p.c.read(0, ints([0, 1]), k[:0].cuda(), k[:0].cuda(), offsets([0, 0]))
    p.check_tables()
    p.check_contents()
    p.c.append(0, ints([77]), k[:0].cuda(), k[:0].cuda(), offsets([0]))
    _refused(p, "passed over")

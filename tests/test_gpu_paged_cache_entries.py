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

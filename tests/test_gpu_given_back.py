"""Chunks under a window in blocks of 128 columns: pages that no token sees make no difference, whether they are there or none."""
import numpy as np
import pytest
import torch

import test_gpu_prefix as prefix
from test_gpu_decoder import BF16, Cached, pop  # noqa: F401  (pop: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks", [(100, 4), (100, 17), (37, 1), (101, 33), (64, 0), (90, 0), (300, 47)])
@pytest.mark.parametrize("heads,n_kv,d,page,context,new", [
    (6, 2, 64, 16, [1630, 640, 333], [70, 64, 5]), (8, 8, 128, 16, [1300, 700], [150, 129]), (8, 2, 128, 32, [1900, 65], [130, 65]), (3, 3, 64, 64, [1500], [97])])
def test_pages_that_are_given_back_change_nothing(pop, heads, n_kv, d, page, context, new, window, sinks):  # noqa: F811
    """Bit for bit: they do not take the steps over the pages that are there from the path for steps that are seen whole, which takes maxima at
    other times (and twice as long: every step is masked, and looks its pages up again)."""
    rng = np.random.default_rng(window + d)
    c = Cached(pop, rng, context, n_kv, d, page)
    start = prefix.starts_of(new)
    q = prefix.queries(rng, start[-1], heads, d, BF16)
    prefix.assert_in_blocks(pop, c, len(q), heads, window)
    table = prefix.given_back(c, start, window, sinks)
    assert (table != c.table).any()
    # (without: in the place of the pages that are given back stands another one, as a table may)
    other = np.where((table < 0) & (c.table >= 0), c.table[0, 0], c.table)
    entry = dict(entry="sinks" if sinks else "plain", **prefix.IN_BLOCKS)
    y = prefix.attend(pop, c, q, start, BF16, BF16, heads, d ** -0.5, window, sinks, table=table, **entry)
    prefix.check(c, y, q, start, BF16, d ** -0.5, window, sinks)
    for with_pages in (c.table, other):
        assert torch.equal(y, prefix.attend(pop, c, q, start, BF16, BF16, heads, d ** -0.5, window, sinks, table=with_pages, **entry))

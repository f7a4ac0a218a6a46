"""The paged cache where contents that no sequence owns, or extreme contents, could reach a result."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from paged_util import Paged, attention_bound, f64

pytestmark = pytest.mark.gpu


def check(c, got, q=None, scale=None):
    q = c.q if q is None else q
    scale = c.hd ** -0.5 if scale is None else scale
    want, weight, delta = P.attend(*c.host(), c.starts_h, c.lens_h, c.table_h, f64(q), scale)
    bound = attention_bound(c.kind, want, weight, delta, c.lens_h, c.starts_h, c.hd)
    rows = ~np.isnan(want).all(axis=(1, 2))
    off = np.abs(f64(got) - want)[rows]
    assert (off <= bound[rows]).all(), (off / bound[rows]).max()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("number", [float("nan"), float("inf"), float("-inf")])
def test_missing_pages_are_zeros_whatever_the_scales_of_a_page_of_nobody(hd, number):
    """Page numbers out of range, in single rows, drafts, chunks and a context that is split, beside a page 0 that nothing was
    ever appended to: its scales are what the allocation held."""
    for seqs, starts in (([(20, 90), (1, 64), (130, 140), (2, 5000), (60, 3000), (3, 0)], True), ([(1, 64), (1, 700), (1, 9000), (1, 0)], False)):
        c = Paged("e4m3", 4, 2, hd, 16, seqs, seed=hd, starts=starts)
        used = {int(x) for b, n in enumerate(c.lens_h) for x in c.table_h[b][:-(-n // 16)]}
        spare = next(x for x in range(1, len(c.k)) if x not in used)
        c.table_h[c.table_h == 0] = spare
        c.ks[0], c.vs[0] = number, number
        for b, n in enumerate(c.lens_h):
            for t in range(0, -(-n // 16), 3):
                c.table_h[b, t] = (-1, len(c.k), -(1 << 31), (1 << 31) - 1)[(b + t) % 4]
        c.bind()
        got = c.attend()
        c.ks[0], c.vs[0] = 1.0, 1.0                              # (the oracle's zeros take no scale; its arrays have to be numbers)
        check(c, got)

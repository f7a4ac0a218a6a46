"""The paged cache's calls at sizes where whole numbers grow large, on sampled rows."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from paged_util import Paged, attention_bound, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_attention_whose_count_of_work_passes_2_39(kind):
    """1024 rows of 1024 heads behind 131072 positions: each of the 256 workgroups has a part of more than 2^31.  No row may be
    missed."""
    new, length, hq, hd = 1024, 131072 + 1024, 1024, 64
    c = Paged(kind, hq, 1, hd, 128, [(new, length)], seed=30)
    out = c.attend(out=torch.full((new, hq, hd), float("nan"), dtype=torch.bfloat16, device="cuda"))
    assert torch.isfinite(out).all()
    k, v, ks, vs = c.host()
    for r, h in ((0, 0), (0, 1023), (1, 77), (300, 500), (511, 3), (767, 1000), (1022, 0), (1023, 1023)):
        # the row alone, as the newest of the positions that it sees
        n = length - new + r + 1
        want, weight, delta = P.attend(k, v, ks, vs, [0, 1], [n], c.table_h, f64(c.q[r:r + 1, h:h + 1]), hd ** -0.5)
        bound = attention_bound(kind, want, weight, delta, [n], [0, 1], hd)
        assert (np.abs(f64(out[r:r + 1, h:h + 1]) - want) <= bound).all(), (r, h)

"""The paged cache's calls at sizes where whole numbers grow large, on sampled rows."""
import numpy as np
import pytest
import torch

import paper_2603_04716_amd as pd
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


def test_append_of_codes_in_more_than_one_launch():
    """4096 sequences of 1024 kv heads have more workgroups than one launch takes.  Only the first and the last sequences have pages, the
    others' page numbers are out of range; queries come behind the pages' workgroups and are all there."""
    n, hkv, hd, ps, kept = 4096, 1024, 64, 16, 24
    g = torch.Generator("cuda")
    g.manual_seed(31)
    rows = torch.randn(n, 3 * hkv, hd, generator=g, device="cuda", dtype=torch.bfloat16)
    q, k, v = rows[:, :hkv], rows[:, hkv:2 * hkv], rows[:, 2 * hkv:]
    pool = [(torch.randn(2 * kept, hkv, ps, hd, generator=g, device="cuda") * 64).clamp(-448, 448).to(torch.float8_e4m3fn) for _ in range(2)]
    scales = [2.0 ** torch.randint(-10, -4, (2 * kept, hkv), generator=g, device="cuda").float() for _ in range(2)]
    has = list(range(kept)) + list(range(n - kept, n))
    table = np.full((n, 1), -1, np.int32)
    table[has, 0] = np.arange(2 * kept)[::-1]
    lens = np.arange(n, dtype=np.int32) % ps + 1
    before = [f64(t) for t in pool + scales]
    kv = pd.make_paged_kv(*pool, *scales)
    seqs = pd.make_paged_seqs(torch.from_numpy(lens).cuda(), torch.from_numpy(table).cuda(), torch.arange(n + 1, dtype=torch.int32, device="cuda"), n)
    q_out = torch.full((n, hkv, hd), float("nan"), dtype=torch.bfloat16, device="cuda")
    pd.pd_paged_append(kv, seqs, k, v, 0.0, q, q_out)
    assert torch.equal(q_out, q)
    want = P.append(*before, np.arange(2 * kept + 1), lens[has], table[has], f64(k[has]), f64(v[has]), 0.0)
    for got, w in zip(pool + scales, want):
        np.testing.assert_array_equal(f64(got), w)

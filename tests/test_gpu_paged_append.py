"""pd_paged_append against the float64 definition in oracle/paged.py.

Bounds.  A rotated element y = x0 c - x1 s: cosine and sine are within 4e-7 (the angle, at most pi, is rounded to fp32,
2^-23, and the functions' own error), products and sum add 2^-23, so y is within 6e-7 (|x0| + |x1|), and what is stored is
rounded once.  Values are not computed with: they are equal, and so are their codes and scales."""
import numpy as np
import pytest
import torch

import paper_2603_04716_amd as pd
from oracle import paged as P
from paged_util import HALF_STEP, Paged, f64

pytestmark = pytest.mark.gpu
BASE = 10000.0

# (new rows, positions held with them): fresh, mid-page, across pages, page ends, none, more rows than positions, empty slot
RAGGED = [(1, 1), (3, 20), (40, 40), (17, 64), (0, 9), (130, 131), (4, 2), (1, 0), (1, 128), (33, 161), (2, 17)]


def rotation_bound(x):
    half = x.shape[-1] // 2
    a = np.abs(x[..., :half]) + np.abs(x[..., half:])
    return 6e-7 * np.concatenate([a, a], -1)


def check(c, before, base, with_q=True, q_out=None):
    """Everything that an append of c's rows may change, against the oracle on the state before it."""
    kp, vp, ks, vs = before
    q, k, v = (f64(t) for t in c.parts())
    want = P.append(kp, vp, ks, vs, c.starts_h, c.lens_h, c.table_h, k, v, base)
    gk, gv, gks, gvs = c.host()
    step = HALF_STEP["f32" if c.kind == "f32" else "bf16"]
    err = np.zeros_like(want[0])                                  # fp32 error of a new key, in units of the page's elements
    for r, (b, p) in enumerate(P.positions(c.starts_h, c.lens_h, c.n_rows)):
        if b >= 0 and 0 <= c.table_h[b][p // c.ps] < len(kp):
            err[c.table_h[b][p // c.ps], :, p % c.ps] = rotation_bound(k[r]) if base else 0.0
    if c.kind == "e4m3":
        np.testing.assert_array_equal(gks, want[2])
        np.testing.assert_array_equal(gvs, want[3])
        np.testing.assert_array_equal(gv, want[1])
        # one code further where the error carries a key over the middle between two codes: a whole step instead of half of one
        err = err / want[2][:, :, None, None]
        whole = np.maximum(np.abs(want[0]) * 2.0 ** -3, 2.0 ** -9)
        same = gk == want[0]
        assert ((err > 0) | same | np.isnan(want[0])).all()
        assert np.nanmax(np.where(same, 0.0, np.abs(gk - want[0]) - whole)) <= 0
        assert (~same & ~np.isnan(want[0])).sum() <= 8 + 1e-4 * same.size
    else:
        np.testing.assert_array_equal(gv, f64(torch.from_numpy(want[1]).to(c.v.dtype)))
        changed = err > 0
        np.testing.assert_array_equal(gk[~changed], f64(torch.from_numpy(want[0]).to(c.k.dtype))[~changed])
        assert (np.abs(gk - want[0])[changed] <= (err + step * np.abs(want[0]))[changed]).all()
    if with_q:
        got = f64(q_out)
        for r, (b, p) in enumerate(P.positions(c.starts_h, c.lens_h, c.n_rows)):
            if b < 0:
                assert (got[r] == 7.0).all()                      # rows without a position are left alone
            else:
                w = P.rotate(q[r], p, base)
                assert (np.abs(got[r] - w) <= rotation_bound(q[r]) + step * np.abs(w)).all(), r


@pytest.mark.parametrize("kind", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("hq,hkv,hd,ps", [(4, 2, 128, 64), (5, 1, 64, 16), (8, 8, 64, 128), (10, 2, 128, 32), (2, 2, 128, 16), (3, 3, 128, 128)])
def test_ragged_rows(kind, hq, hkv, hd, ps):
    c = Paged(kind, hq, hkv, hd, ps, RAGGED, pad=3, seed=hq + ps)
    before = c.host()
    q, k, v = c.parts()
    q_out = torch.full((c.n_rows, hq, hd), 7.0, dtype=q.dtype, device="cuda")
    pd.pd_paged_append(c.kv, c.seqs, k, v, BASE, q, q_out)
    check(c, before, BASE, True, q_out)


@pytest.mark.parametrize("kind", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("n", [1, 7, 65, 300])
def test_one_row_each_without_starts(kind, n):
    rng = np.random.default_rng(n)
    c = Paged(kind, 4, 2, 128, 64, [(1, int(x)) for x in rng.integers(0, 300, n)], seed=n, starts=False)
    before = c.host()
    q, k, v = c.parts()
    q_out = torch.full((c.n_rows, 4, 128), 7.0, dtype=q.dtype, device="cuda")
    pd.pd_paged_append(c.kv, c.seqs, k, v, BASE, q, q_out)
    check(c, before, BASE, True, q_out)


@pytest.mark.parametrize("kind", ["bf16", "f32", "e4m3"])
def test_many_rows_four_to_a_workgroup(kind):
    """More than 1024 rows; keys and values alone, and unrotated."""
    for base in (BASE, 0.0):
        c = Paged(kind, 2, 2, 64, 32, [(700, 1400), (1, 77), (0, 3), (600, 600), (513, 520)], pad=5, seed=3)
        before = c.host()
        _, k, v = c.parts()
        pd.pd_paged_append(c.kv, c.seqs, k, v, base)
        check(c, before, base, False)


def test_4096_sequences():
    rng = np.random.default_rng(5)
    new = rng.integers(0, 3, 4096)
    c = Paged("e4m3", 1, 1, 64, 16, [(int(n), int(n + rng.integers(0, 20))) for n in new], seed=5)
    before = c.host()
    q, k, v = c.parts()
    q_out = torch.full((c.n_rows, 1, 64), 7.0, dtype=q.dtype, device="cuda")
    pd.pd_paged_append(c.kv, c.seqs, k, v, BASE, q, q_out)
    check(c, before, BASE, True, q_out)


def test_queries_in_place_and_separate_tensors():
    c = Paged("bf16", 4, 2, 128, 64, [(5, 70), (3, 3)], seed=6)
    before = c.host()
    q, k, v = c.parts()
    mine = q.contiguous()
    pd.pd_paged_append(c.kv, c.seqs, k.contiguous(), v.contiguous(), BASE, mine, mine)
    check(c, before, BASE, True, mine)


@pytest.mark.parametrize("kind", ["bf16", "f32", "e4m3"])
def test_far_positions(kind):
    """Angles of positions near 10^6 and 2^29: the bound is the same as near 0."""
    for length in (1_000_003, (1 << 29) - 5):
        c = Paged(kind, 2, 1, 64, 128, [(3, 130)], seed=7)
        wide = np.zeros((1, -(-length // 128)), np.int32)
        wide[0, -1], wide[0, -2] = c.table_h[0, 0], c.table_h[0, 1]
        c.table_h, c.lens_h = wide, [length]
        c.bind()
        before = c.host()
        q, k, v = c.parts()
        q_out = torch.full((c.n_rows, 2, 64), 7.0, dtype=q.dtype, device="cuda")
        pd.pd_paged_append(c.kv, c.seqs, k, v, BASE, q, q_out)
        check(c, before, BASE, True, q_out)


def test_scale_follows_the_page():
    """Token by token: the scale is the largest that any token needed, older codes follow it, a new page starts afresh."""
    c = Paged("e4m3", 1, 2, 64, 16, [(1, 1)], seed=8, extra_width=3, starts=False, spare=4)
    c.table_h[0, :4] = [3, 0, 2, 1]
    rng = np.random.default_rng(8)
    for t in range(40):
        c.lens_h = [t + 1]
        c.qkv = torch.from_numpy(rng.standard_normal((1, 5, 64)) * 2.0 ** rng.integers(-12, 12)).cuda().to(torch.bfloat16)
        c.bind()
        before = c.host()
        _, k, v = c.parts()
        pd.pd_paged_append(c.kv, c.seqs, k, v, 0.0)
        check(c, before, 0.0, False)


def test_extreme_elements_of_codes():
    """Zeros only, the border 448 s itself, one bf16 step above it, the smallest and largest numbers, infinities and NaN."""
    rows = torch.zeros(12, 3, 64)
    rows[1, 1:, 5], rows[2, 1:, 5], rows[3, 1:, 5] = 448.0, 450.0, 446.0
    rows[4, 1:, 0], rows[5, 1:, 0] = 2.0 ** -120, 3e38
    rows[6, 1:, :4] = torch.tensor([float("inf"), float("-inf"), float("nan"), 3.0])
    rows[7, 1:, :] = float("inf")
    rows[8, 1:, :] = float("nan")
    rows[9, 1:, :] = torch.linspace(-1, 1, 64)
    rows[10, 1:, 7], rows[11, 1:, 63] = 1.75 * 2.0 ** -52, -1.7578125 * 2.0 ** -52
    c = Paged("e4m3", 1, 1, 64, 16, [(1, 1)] * 12, seed=9, starts=False)
    c.qkv = rows.to(torch.bfloat16).cuda()
    before = c.host()
    _, k, v = c.parts()
    pd.pd_paged_append(c.kv, c.seqs, k, v, 0.0)
    want = P.append(*before, c.starts_h, c.lens_h, c.table_h, f64(k), f64(v), 0.0)
    for got, w in zip(c.host(), want):
        np.testing.assert_array_equal(got, w)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_page_numbers_and_lengths_out_of_range(kind):
    """Nothing is stored for a page that is not there; lengths beyond the table and starts beyond the rows count as the bound."""
    c = Paged(kind, 2, 2, 64, 16, [(20, 40), (5, 5), (3, 30)], seed=10)
    c.table_h[0, 1], c.table_h[2, 1] = -1, len(c.k)
    c.bind()
    before = c.host()
    q, k, v = c.parts()
    q_out = torch.full((c.n_rows, 2, 64), 7.0, dtype=q.dtype, device="cuda")
    pd.pd_paged_append(c.kv, c.seqs, k, v, BASE, q, q_out)
    check(c, before, BASE, True, q_out)

    c = Paged(kind, 2, 2, 64, 16, [(2, 48)], seed=11)
    c.lens_h = [1000]
    c.bind()
    c.lens_h = [48]                                               # three pages of 16
    before = c.host()
    q, k, v = c.parts()
    pd.pd_paged_append(c.kv, c.seqs, k, v, BASE)
    check(c, before, BASE, False)


def test_pool_of_more_than_4_gib():
    """Offsets that do not fit 32 bits: pages at the end of a 4.5 GiB pool."""
    n_pages, ps, hkv, hd = 37000, 128, 8, 128
    k = torch.zeros(n_pages, hkv, ps, hd, dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(k)
    ks, vs = (torch.ones(n_pages, hkv, device="cuda") for _ in range(2))
    assert k.numel() > 1 << 32
    kv = pd.make_paged_kv(k, v, ks, vs)
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([130], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 130], dtype=torch.int32, device="cuda")
    seqs = pd.make_paged_seqs(lens, table, starts, 130)
    rows = torch.randn(130, 2 * hkv, hd, device="cuda").to(torch.bfloat16)
    pd.pd_paged_append(kv, seqs, rows[:, :hkv], rows[:, hkv:])
    got = torch.cat([v[n_pages - 1].transpose(0, 1), v[n_pages - 2, :, :2].transpose(0, 1)]).view(torch.float8_e4m3fn).float()
    scale = torch.cat([vs[n_pages - 1].expand(128, -1), vs[n_pages - 2].expand(2, -1)])[:, :, None]
    x = rows[:, hkv:].float()
    assert ((got * scale - x).abs() <= x.abs() * 2.0 ** -4 + scale * 2.0 ** -10).all()
    out = torch.empty(130, hkv, hd, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(pd.pd_paged_attention_workspace(kv, seqs, hkv), dtype=torch.uint8, device="cuda")
    pd.pd_paged_attention(kv, seqs, rows[:, :hkv], out, ws)
    # the first row sees itself alone: its value, as the page holds it
    torch.testing.assert_close(out[0].float(), (got * scale)[0].to(torch.bfloat16).float(), rtol=0, atol=0)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("starts", [True, False])
def test_full_pages_whose_scales_grow(hd, starts):
    """One row in the last slots of pages, whose scales are too small by up to 2^20: every older code is rounded again."""
    for ps in (16, 64, 128):
        lens = [ps, ps - 1, 2 * ps, 3 * ps - 1, ps // 2 + 1, 2]
        c = Paged("e4m3", 2, 2, hd, ps, [(1, n) for n in lens], seed=ps + hd, starts=starts)
        rng = np.random.default_rng(ps + hd)
        for s in (c.ks, c.vs):
            s *= torch.from_numpy(2.0 ** -rng.integers(0, 21, tuple(s.shape))).float().cuda()
        c.bind()
        before = c.host()
        q, k, v = c.parts()
        q_out = torch.full((c.n_rows, 2, hd), 7.0, dtype=q.dtype, device="cuda")
        pd.pd_paged_append(c.kv, c.seqs, k, v, BASE, q, q_out)
        check(c, before, BASE, True, q_out)

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


@pytest.mark.parametrize("kind", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("q_log,k_log,scale", [(2, 3, 0.3), (20, 13, 0.3), (20, 13, 0.7), (60, 40, 0.3), (67, 60, float(np.float32(np.log(2.0))))])
def test_scores_of_any_size(kind, sign, q_log, k_log, scale):
    """Scores of up to 3.2e38 (the softmax in base 2): equal ones share a row's weight, and a larger one has all of it.  One channel
    makes the score, so that it is one exact product, the same for all keys but one."""
    # rows of both kernels, contexts that are split, and single rows
    for seqs, starts in (([(1, 40), (3, 700), (100, 130), (150, 6000), (2, 9000), (5, 2)], True), ([(1, 300), (1, 9000), (1, 1)], False)):
        c = Paged(kind, 4, 2, 64, 32, seqs, seed=q_log, starts=starts)
        q = torch.zeros_like(c.q)
        q[:, :, 0] = sign * 2.0 ** q_log
        some, one = (1.875, 0.9375) if sign < 0 else (0.9375, 1.875)
        if kind == "e4m3":
            c.ks.fill_(2.0 ** k_log)
        else:
            some, one = some * 2.0 ** k_log, one * 2.0 ** k_log
        c.k[:, :, :, 0] = torch.tensor(some).to(c.k.dtype).cuda()
        for b, n in enumerate(c.lens_h):
            if b % 2 and n > 2:
                c.k[int(c.table_h[b, (n - 2) // 32]), :, (n - 2) % 32, 0] = torch.tensor(one).to(c.k.dtype).cuda()
        got = c.attend(q=q, scale=scale)
        want, weight, delta = P.attend(*c.host(), c.starts_h, c.lens_h, c.table_h, f64(q), scale)
        if q_log > 2:
            delta[:] = 0.0                                       # the scores are exact but for one rounding that all share
        bound = attention_bound(kind, want, weight, delta, c.lens_h, c.starts_h, 64)
        assert (np.abs(f64(got) - want) <= bound).all()


@pytest.mark.parametrize("hd", [64, 128])
def test_key_codes_that_are_not_numbers(hd):
    """A NaN code among a sequence's keys: the rows that see it are NaN in the heads that read it, no other element changes."""
    c = Paged("e4m3", 4, 2, hd, 32, [(100, 130), (3, 700), (1, 90), (60, 5000), (40, 40)], seed=32)
    clean = c.attend()
    check(c, clean)
    x = c.k.view(torch.uint8)
    hit = torch.zeros_like(clean, dtype=torch.bool)
    for b, p, g, code in ((0, 70, 0, 0x7F), (1, 650, 1, 0xFF), (2, 0, 0, 0x7F), (3, 1234, 1, 0xFF), (4, 39, 0, 0x7F)):
        x[int(c.table_h[b, p // 32]), g, p % 32, 5] = code
        first = int(c.starts_h[b]) + max(p - (c.lens_h[b] - c.new[b]), 0)
        hit[first:int(c.starts_h[b + 1]), 2 * g:2 * g + 2] = True
    got = c.attend()
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], clean[~hit])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_infinite_keys_in_chunks_and_prompts(kind):
    """Scores of -infinity weigh nothing, rows that see no other score are 0 / 0, a score of infinity makes the rows that see it NaN: in
    chunks whose rows see different keys, and in a context that is split."""
    c = Paged(kind, 4, 2, 64, 16, [(100, 100), (70, 400), (40, 6000), (3, 60)], seed=33)
    q = c.q.clone()
    q[:, :, 0] = 1.0
    for b, keys in ((0, [0, 1, 2, 50, 99]), (1, list(range(0, 400, 7))), (2, list(range(0, 2000))), (3, [0, 59])):
        for p in keys:
            c.k[int(c.table_h[b, p // 16]), :, p % 16, 0] = float("-inf")
    scale = 64 ** -0.5

    def held_to(got):
        with np.errstate(invalid="ignore"):
            want, weight, _ = P.attend(*c.host(), c.starts_h, c.lens_h, c.table_h, f64(q), scale)
        k = c.k.clone()
        k[..., 0] = torch.where(torch.isfinite(k[..., 0]), k[..., 0], 0.0)
        _, _, delta = P.attend(f64(k), f64(c.v), None, None, c.starts_h, c.lens_h, c.table_h, f64(q), scale)
        g, nan = f64(got), np.isnan(want)
        assert (np.isnan(g) == nan).all()
        bound = attention_bound(kind, want, weight, delta, c.lens_h, c.starts_h, 64)
        assert (np.abs(g - want)[~nan] <= bound[~nan]).all()
        return nan

    nan = held_to(c.attend(q=q))
    assert nan[:3].all() and not nan[3:].any()
    for b, p in ((0, 60), (1, 350), (2, 5990)):
        c.k[int(c.table_h[b, p // 16]), :, p % 16, 0] = float("inf")
    nan = held_to(c.attend(q=q))
    # (rows 170 .. 209 are positions 5960 .. 5999 of the third sequence)
    assert nan[60:100].all() and not nan[3:60].any() and not nan[170:200].any() and nan[200:210].all() and not nan[210:].any()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_values_that_are_not_finite_in_long_parts(kind):
    """Parts of more than 512 tiles of keys, sequences that read the same pages: infinities and NaN in a few of the tiles reach the
    rows that see them, in their channels, and nothing else; a NaN in a query or a key reaches the rows that it makes."""
    hkv, new, length = 32, 40, 45000
    c = Paged(kind, 8 * hkv, hkv, 64, 128, [(new, length)] + [(new, 1)] * 7, seed=34, extra_width=0)
    c.table_h[:] = c.table_h[0]
    c.lens_h = [length] * 8
    c.bind()
    clean = c.attend()
    assert torch.isfinite(clean).all()
    x, odd = (c.v.view(torch.uint8), 0x7F) if kind == "e4m3" else (c.v, float("nan"))
    hit = torch.zeros_like(clean, dtype=torch.bool)
    for p, g, ch in ((0, 0, 5), (63, 0, 6), (64, 3, 7), (20000, 3, 8), (33000, 31, 63), (length - new - 1, 30, 0), (length - 7, 30, 1), (length - 1, 30, 2)):
        x[int(c.table_h[0, p // 128]), g, p % 128, ch] = odd
        for b in range(8):
            hit[b * new + max(p - (length - new), 0):(b + 1) * new, 8 * g:8 * g + 8, ch] = True
    got = c.attend()
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], clean[~hit])
    q = c.q.clone()
    q[77, 100, 3] = float("nan")
    hit[77, 100] = True
    got = c.attend(q=q)
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], clean[~hit])
    (c.k.view(torch.uint8) if kind == "e4m3" else c.k)[int(c.table_h[0, 100]), 7, 3, 9] = odd
    hit[:, 56:64] = True
    got = c.attend(q=q)
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], clean[~hit])


@pytest.mark.parametrize("hd", [64, 128])
def test_values_of_the_largest_scale(hd):
    """At a scale of 2^120 the codes of 256 and more are infinite: rows behind them are that, rows before them as without."""
    for seqs, starts, at in (([(3, 40), (100, 130), (40, 9000)], True, (38, 118, 8980)), ([(1, 40), (1, 5000)], False, (38, 4000))):
        c = Paged("e4m3", 2, 1, hd, 16, seqs, seed=35, starts=starts)
        for b, p in enumerate(at):
            page = int(c.table_h[b, p // 16])
            c.v.view(torch.uint8)[page] = 0
            c.vs[page] = 2.0 ** 120
        clean = c.attend()
        check(c, clean)
        for code, value in ((0x7E, float("inf")), (0xF8, float("-inf")), (0x7F, float("nan"))):
            hit = torch.zeros_like(clean, dtype=torch.bool)
            for b, p in enumerate(at):
                c.v.view(torch.uint8)[int(c.table_h[b, p // 16]), 0, p % 16, 5] = code
                hit[int(c.starts_h[b]) + max(p - (c.lens_h[b] - c.new[b]), 0):int(c.starts_h[b + 1]), :, 5] = True
            got = c.attend()
            assert torch.equal(got[~hit], clean[~hit])
            assert torch.isnan(got[hit]).all() if value != value else (got[hit] == value).all()

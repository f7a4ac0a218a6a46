"""pd_paged_attention against the float64 definition in oracle/paged.py; the bounds are derived in paged_util.attention_bound."""
import numpy as np
import pytest
import torch

import paper_2603_04716_amd as pd
from oracle import paged as P
from paged_util import Paged, attention_bound, f64

pytestmark = pytest.mark.gpu

KINDS = ["bf16", "f32", "e4m3"]
# (new rows, positions held with them): one token, drafts, page and step ends, a prompt, none, more rows than positions, an empty slot
RAGGED = [(1, 1), (1, 2), (3, 33), (8, 64), (1, 65), (0, 9), (70, 70), (4, 2), (1, 0), (2, 129), (5, 300), (1, 257), (33, 161)]


def check(c, got, q=None, scale=None, host=None):
    q = c.q if q is None else q
    want, weight, delta = P.attend(*(c.host() if host is None else host), c.starts_h, c.lens_h, c.table_h, f64(q),
                                   c.hd ** -0.5 if scale is None else scale)
    bound = attention_bound(c.kind, want, weight, delta, c.lens_h, c.starts_h, c.hd)
    g = f64(got)
    rows = ~np.isnan(want).all(axis=(1, 2))
    owned = np.zeros(c.n_rows, bool)
    owned[:c.starts_h[-1]] = True
    assert (g[~owned] == 7.0).all()                              # rows behind the last sequence
    off = np.abs(g - want)[rows & owned]
    assert (off <= bound[rows & owned]).all(), (off / bound[rows & owned]).max()
    return want


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv,hd,ps", [(4, 2, 128, 64), (5, 1, 64, 16), (8, 8, 64, 128), (10, 2, 128, 16), (2, 2, 128, 32), (32, 2, 64, 32),
                                          (17, 1, 128, 128), (40, 1, 64, 64)])
def test_ragged_rows(kind, hq, hkv, hd, ps):
    c = Paged(kind, hq, hkv, hd, ps, RAGGED, pad=3, seed=hq + ps)
    check(c, c.attend())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv", [(4, 1), (16, 1), (6, 3), (34, 2), (1, 1)])
@pytest.mark.parametrize("n", [1, 5, 70])
def test_one_row_each_without_starts(kind, hq, hkv, n):
    rng = np.random.default_rng(n + hq)
    lens = [int(x) for x in rng.integers(0, 400, n)]
    lens[0] = 700
    c = Paged(kind, hq, hkv, 128, 32, [(1, x) for x in lens], seed=n, starts=False)
    check(c, c.attend())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("length", [1, 15, 16, 17, 255, 256, 257, 2000, 9001])
def test_lengths_of_one_sequence(kind, length):
    """From one key to many chunks, joined by the merge."""
    for hd in (64, 128):
        c = Paged(kind, 4, 2, hd, 64, [(1, length)], seed=length, starts=False)
        check(c, c.attend())
        c = Paged(kind, 4, 2, hd, 16, [(2, length)], seed=length)
        check(c, c.attend())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new,length", [(100, 100), (129, 700), (300, 300), (257, 2500), (65, 5000)])
def test_prompts_and_chunks(kind, new, length):
    for hq, hkv, hd in ((4, 2, 128), (3, 1, 64)):
        c = Paged(kind, hq, hkv, hd, 64, [(new, length), (1, 100), (new // 2, new // 2 + 3)], pad=2, seed=new)
        check(c, c.attend())


@pytest.mark.parametrize("kind", KINDS)
def test_long_and_short_sequences_together(kind):
    """Chunks are sized for the whole call: a long sequence is divided, short ones beside it are not."""
    c = Paged(kind, 8, 2, 128, 64, [(1, 20000), (1, 3), (1, 700), (1, 0), (1, 5000)], seed=1, starts=False)
    check(c, c.attend())
    c = Paged(kind, 8, 2, 64, 16, [(2, 9000), (3, 3), (40, 4000), (0, 0), (1, 5)], seed=2)
    check(c, c.attend())


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_4096_sequences(kind):
    rng = np.random.default_rng(4)
    c = Paged(kind, 2, 1, 64, 16, [(int(n), int(n + x)) for n, x in zip(rng.integers(0, 3, 4096), rng.integers(0, 30, 4096))], seed=4)
    check(c, c.attend())


@pytest.mark.parametrize("kind", KINDS)
def test_strided_queries_other_scales_and_large_scores(kind):
    c = Paged(kind, 4, 2, 128, 64, [(3, 200), (40, 90), (1, 600)], seed=5)
    q = c.parts()[0]                                             # part of a wider row
    for scale in (1e-30, 0.3, 1.5):                              # scores up to some hundred: one key takes all
        check(c, c.attend(q=q, scale=scale), q, scale)


@pytest.mark.parametrize("kind", KINDS)
def test_what_a_row_does_not_see_does_not_reach_it(kind):
    """Infinities and NaN behind a sequence's end, in later positions of its own rows (keys and values), and in pages of nobody."""
    for hq, hkv, hd, ps, seqs in ((4, 2, 128, 16, [(9, 40), (1, 50), (100, 130), (1, 1)]), (2, 2, 64, 64, [(70, 90), (3, 3), (200, 777)])):
        c = Paged(kind, hq, hkv, hd, ps, seqs, seed=6)
        clean = c.attend()
        check(c, clean)

        bad = torch.tensor([float("nan"), float("inf"), float("-inf")], device="cuda")
        codes = torch.tensor([0x7F, 0xFF, 0x7F], dtype=torch.uint8, device="cuda")
        used = set()
        for b, n in enumerate(c.lens_h):
            for t in range(-(-n // ps)):
                used.add((int(c.table_h[b][t]), min(ps, n - t * ps)))
        held = dict(used)

        def spoil(pool, page, slots):
            x = pool.view(torch.uint8) if kind == "e4m3" else pool
            m = x[page, :, slots].shape
            fill = (codes if kind == "e4m3" else bad)[torch.randint(0, 3, m, device="cuda")]
            x[page, :, slots] = fill.to(x.dtype)

        for page in range(len(c.k)):
            for pool in (c.k, c.v):
                spoil(pool, page, slice(held.get(page, 0), ps))
        got = c.attend()
        assert torch.equal(got, clean)
        # the last row of every sequence is spoiled too: the rows before it do not change, it itself is not a number
        late = []
        for b, n in enumerate(c.lens_h):
            if c.new[b] > 1:
                page, slot = int(c.table_h[b][(n - 1) // ps]), (n - 1) % ps
                spoil(c.v, page, slice(slot, slot + 1))
                late.append(int(c.starts_h[b + 1]) - 1)
        got = c.attend()
        keep = [r for r in range(c.n_rows) if r not in late]
        assert torch.equal(got[keep], clean[keep])
        assert not torch.isfinite(got[late].float()).any()
        for b, n in enumerate(c.lens_h):
            if c.new[b] > 1:
                page, slot = int(c.table_h[b][(n - 1) // ps]), (n - 1) % ps
                spoil(c.k, page, slice(slot, slot + 1))
        got = c.attend()
        assert torch.equal(got[keep], clean[keep])



@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_infinite_values_that_a_row_sees(kind):
    """An infinite value in a visible place gives that infinity, two of both signs give NaN, also where other rows do not see it."""
    c = Paged(kind, 2, 1, 128, 16, [(20, 40), (90, 100)], seed=7)
    page = lambda b, p: (int(c.table_h[b][p // 16]), 0, p % 16)  # noqa: E731
    c.v[page(0, 25)][3] = float("inf")
    c.v[page(0, 30)][3] = float("-inf")
    c.v[page(0, 33)][70] = float("-inf")
    c.v[page(1, 60)][9] = float("nan")
    got = c.attend()[:, 0].float().cpu().numpy()
    for r in range(20):
        p = 20 + r
        assert np.isfinite(got[r, 3]) if p < 25 else got[r, 3] == np.inf if p < 30 else np.isnan(got[r, 3]), p
        assert np.isfinite(got[r, 70]) if p < 33 else got[r, 70] == -np.inf, p
        assert np.isfinite(np.delete(got[r], [3, 70])).all()
    for r in range(90):
        p = 10 + r
        assert np.isnan(got[20 + r, 9]) == (p >= 60) and np.isfinite(np.delete(got[20 + r], 9)).all()


@pytest.mark.parametrize("kind", KINDS)
def test_keys_that_are_not_finite(kind):
    """Scores of -infinity weigh nothing; a row all of whose scores are -infinity is 0 / 0."""
    c = Paged(kind, 1, 1, 64, 16, [(1, 100), (1, 40)], seed=8, starts=False)
    if kind == "e4m3":
        return
    q = c.q.clone()
    q[:, :, 0] = 1.0
    for p in range(0, 100, 3):
        c.k[int(c.table_h[0][p // 16]), 0, p % 16, 0] = float("-inf")
    for p in range(40):
        c.k[int(c.table_h[1][p // 16]), 0, p % 16, 0] = float("-inf")
    got = c.attend(q=q)
    assert torch.isnan(got[1]).all()
    k = c.k[torch.from_numpy(c.table_h[0][:7]).cuda().long(), 0].reshape(-1, 64)[:100].double()
    v = c.v[torch.from_numpy(c.table_h[0][:7]).cuda().long(), 0].reshape(-1, 64)[:100].double()
    w = torch.softmax((k * q[0, 0].double()).sum(1) / 8.0, 0)
    want = (w[:, None] * v).sum(0)
    tol = (2.0 ** -7 if kind == "bf16" else 1e-4) * (w[:, None] * v.abs()).sum(0) + 1e-6
    assert ((got[0, 0].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("kind", KINDS)
def test_pages_that_are_not_there_read_as_zeros(kind):
    c = Paged(kind, 4, 2, 64, 16, [(20, 90), (1, 64), (130, 140)], seed=9)
    c.table_h[0, 2], c.table_h[1, 0], c.table_h[1, 3], c.table_h[2, 5], c.table_h[2, 8] = -1, len(c.k), -(1 << 31), (1 << 31) - 1, -5
    c.bind()
    check(c, c.attend())


def test_lengths_and_starts_out_of_range():
    c = Paged("bf16", 4, 2, 64, 16, [(2, 48), (3, 20)], seed=10)
    c.lens_h = [1000, -7]
    c.bind()
    got = c.attend()
    c.lens_h = [48, 0]                                           # three pages of 16
    check(c, got)
    # rows that overlap: no such call, nothing is written
    c.row_starts = torch.tensor([0, 5, 0], dtype=torch.int32, device="cuda")
    three = pd.make_paged_seqs(torch.tensor([48, 48, 48], dtype=torch.int32, device="cuda"), c.table[[0, 0, 0]].contiguous(),
                               torch.tensor([0, 5, 0, 5], dtype=torch.int32, device="cuda"), 5)
    out = torch.full((5, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(pd.pd_paged_attention_workspace(c.kv, three, 4), dtype=torch.uint8, device="cuda")
    pd.pd_paged_attention(c.kv, three, c.q, out, ws)
    assert (out == 7.0).all()


def test_shared_pages_and_no_rows():
    """Two sequences that share their first pages; sequences without rows alone; calls of nothing."""
    c = Paged("bf16", 4, 2, 128, 16, [(1, 70), (3, 75)], seed=11)
    c.table_h[1, :4] = c.table_h[0, :4]
    c.bind()
    check(c, c.attend())
    c = Paged("bf16", 4, 2, 128, 16, [(0, 70), (0, 3)], pad=4, seed=12)
    check(c, c.attend())
    none = pd.make_paged_seqs(torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, 1, dtype=torch.int32, device="cuda"))
    assert pd.pd_paged_attention_workspace(c.kv, none, 4) == 0
    q = torch.empty(0, 4, 128, dtype=torch.bfloat16, device="cuda")
    pd.pd_paged_attention(c.kv, none, q, q, torch.empty(0, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("kind", KINDS)
def test_same_bits_every_time_and_the_workspace_is_enough(kind):
    c = Paged(kind, 8, 2, 128, 64, [(1, 6000), (20, 3000), (1, 100), (90, 1500)], seed=13)
    need = pd.pd_paged_attention_workspace(c.kv, c.seqs, 8)
    assert need > 0
    ws = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    first = c.attend(ws=ws[:need])
    assert (ws[need:] == 0x5A).all()
    for _ in range(5):
        assert torch.equal(first, c.attend(ws=ws[:need]))
    ws.fill_(0xFF)
    assert torch.equal(first, c.attend(ws=ws[:need]))
    with pytest.raises(pd.PdError) as e:
        c.attend(ws=ws[:need - 1])
    assert e.value.status == pd.PD_ERR_INVALID_ARG


def test_two_streams_at_once():
    calls = [Paged("bf16", 8, 2, 128, 64, [(1, 5000), (1, 900)], seed=14, starts=False), Paged("e4m3", 8, 2, 128, 64, [(30, 4000), (1, 9)], seed=15)]
    want = [c.attend() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = []
    for _ in range(3):
        for c, s in zip(calls, streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(c.attend())
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert torch.equal(g, want[i % 2])


@pytest.mark.parametrize("kind", KINDS)
def test_steps_replayed_from_a_graph_while_sequences_grow(kind):
    """A captured decode step (append, attention, lengths + 1) replayed: every replay equals the eager step on a twin's state, over
    page borders and from one key chunk to several.  Two graphs share a workspace, one after the other."""
    lens = [1, 15, 250, 600, 0]
    mk = lambda: Paged(kind, 4, 2, 128, 16, [(1, n) for n in lens], seed=16, starts=False, extra_width=8, spare=64)  # noqa: E731
    a, b = mk(), mk()
    for c in (a, b):                                             # pages for what is to come, nobody else's
        taken = {int(x) for s, n in enumerate(lens) for x in c.table_h[s][:-(-n // 16)]}
        free = [p for p in range(len(c.k)) if p not in taken]
        for s, n in enumerate(lens):
            for t in range(-(-n // 16), c.table_h.shape[1]):
                if t < -(-n // 16) + 6:
                    c.table_h[s, t] = free.pop()
        c.bind()
    grow = torch.tensor([1, 1, 1, 1, 0], dtype=torch.int32, device="cuda")
    ws = a.workspace()

    def step(c, qkv, q_out, out):
        c.lens += grow
        pd.pd_paged_append(c.kv, c.seqs, qkv[:, 4:6], qkv[:, 6:], 10000.0, qkv[:, :4], q_out)
        pd.pd_paged_attention(c.kv, c.seqs, q_out, out, ws)

    qkv = a.qkv.clone()
    q_out, out, out2 = torch.zeros_like(a.q), torch.zeros_like(a.q), torch.zeros_like(a.q)
    eager_q, eager = torch.zeros_like(a.q), torch.zeros_like(a.q)
    torch.cuda.synchronize()
    kept = (a.lens.clone(), a.k.clone(), a.v.clone(), *(t.clone() for t in (a.ks, a.vs) if t is not None))
    graphs = []
    for o in (out, out2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(a, qkv, q_out, o)
        graphs.append((g, o))
    for t, old in zip((a.lens, a.k, a.v, a.ks, a.vs), kept):
        t.copy_(old)
    for i in range(60):
        qkv.copy_(torch.randn_like(qkv, dtype=torch.float32) * (1 + i % 7))
        g, o = graphs[i % 2]
        g.replay()
        step(b, qkv, eager_q, eager)
        torch.cuda.synchronize()
        assert torch.equal(o[:4], eager[:4]) and torch.equal(a.k.view(torch.uint8), b.k.view(torch.uint8)), i
        assert (o[4] == 0).all() and torch.equal(a.lens, b.lens)
    a.lens_h = a.lens.tolist()
    last, weight, delta = P.attend(*a.host(), a.starts_h, a.lens_h, a.table_h, f64(q_out), 128 ** -0.5)
    bound = attention_bound(kind, last, weight, delta, a.lens_h, a.starts_h, 128)
    assert (np.abs(f64(graphs[1][1]) - last) <= bound).all()


@pytest.mark.parametrize("kind", KINDS)
def test_a_prompt_in_any_division_is_the_same_prompt(kind):
    """Append and attention as a server uses them: a prompt in one call, in chunks, and token by token leave the same pages (8-bit
    ones up to the rounding of codes that a growing scale rounds again) and outputs within the bound of the whole prompt's."""
    n, hq, hkv, hd, ps = 150, 4, 2, 64, 16
    x = Paged(kind, hq, hkv, hd, ps, [(n, n)], seed=17).qkv
    results = []
    for sizes in ([n], [64, 64, 22], [1] * 20 + [100] + [1] * 30):
        c = Paged(kind, hq, hkv, hd, ps, [(n, n)], seed=18)
        outs, at = [], 0
        for m in sizes:
            at += m
            c.starts_h, c.lens_h, c.n_rows = np.array([0, m], np.int32), [at], m
            c.bind()
            rows = x[at - m:at]
            q = torch.empty(m, hq, hd, dtype=rows.dtype, device="cuda")
            pd.pd_paged_append(c.kv, c.seqs, rows[:, hq:hq + hkv], rows[:, hq + hkv:], 10000.0, rows[:, :hq], q)
            outs.append((q, c.attend(q=q)))
        c.starts_h, c.n_rows = np.array([0, n], np.int32), n
        results.append((c, torch.cat([q for q, _ in outs]), torch.cat([o for _, o in outs]), sizes[-1]))
    c0, q0, o0, _ = results[0]
    check(c0, o0, q0)
    for c, q, o, m in results[1:]:
        assert torch.equal(q, q0)
        if kind != "e4m3":
            assert torch.equal(c.k, c0.k) and torch.equal(c.v, c0.v)
            check(c, o, q)
        else:
            assert torch.equal(c.ks, c0.ks) and torch.equal(c.vs, c0.vs)
            # rows of the last call read the final pages
            want, weight, delta = P.attend(*c.host(), [0, n], [n], c.table_h, f64(q), hd ** -0.5)
            bound = attention_bound(kind, want, weight, delta, [n], [0, n], hd)
            assert (np.abs(f64(o) - want)[-m:] <= bound[-m:]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv,hd,ps", [(64, 16, 64, 16), (16, 8, 128, 32)])
def test_more_units_than_a_workgroup_lists(kind, hq, hkv, hd, ps):
    """Hundreds of short chunks in one call, with a long one among them; then with infinities and NaN where nobody looks."""
    rng = np.random.default_rng(19)
    n = 5000 // hkv
    seqs = [(int(a), int(a + b)) for a, b in zip(rng.integers(9, 20, n), rng.integers(0, 30, n))]
    seqs[n // 3] = (200, 2600)
    c = Paged(kind, hq, hkv, hd, ps, seqs, pad=5, seed=19)
    clean = c.attend()
    check(c, clean)
    x = c.v.view(torch.uint8) if kind == "e4m3" else c.v
    for b in range(0, n, 3):                                     # the last page's slots behind the sequence's end
        m = c.lens_h[b]
        if m % ps:
            x[int(c.table_h[b, m // ps]), :, m % ps:] = 0x7F if kind == "e4m3" else float("inf")
    assert torch.equal(c.attend(), clean)


@pytest.mark.parametrize("kind", KINDS)
def test_rows_about_the_border_of_the_kernels(kind):
    """31 to 33 (token, head) rows, whole tiles of 256 and one more, in one call and with a length of zero."""
    c = Paged(kind, 3, 3, 64, 16, [(31, 60), (32, 500), (33, 33), (256, 300), (257, 257), (255, 900), (40, 0)], seed=20)
    check(c, c.attend())
    c = Paged(kind, 8, 1, 128, 128, [(4, 900), (5, 900), (32, 200), (33, 4000), (64, 64)], pad=1, seed=21)
    check(c, c.attend())


@pytest.mark.parametrize("kind", KINDS)
def test_more_rows_than_positions(kind):
    """Whole tiles of rows that see nothing are zeros, beside rows that see keys and sequences that hold none."""
    c = Paged(kind, 4, 2, 128, 16, [(300, 20), (700, 300), (90, 0), (20, 900)], pad=2, seed=22)
    check(c, c.attend())
    got = c.attend()
    assert (got[:280] == 0).all() and (got[300:700] == 0).all() and (got[1000:1090] == 0).all()
    c = Paged(kind, 4, 2, 64, 64, [(50, 0), (1, 0), (300, 0)], seed=23)
    assert (c.attend() == 0).all()


@pytest.mark.parametrize("kind", KINDS)
def test_prompts_of_one_length(kind):
    """Equal prompts, whose tiles the workgroups share without splitting one, and so many rows that all have several."""
    c = Paged(kind, 16, 4, 64, 64, [(1000, 1000), (1000, 1000), (1000, 1000)], seed=24)
    check(c, c.attend())


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_a_value_that_is_not_a_number_in_a_split_unit(kind):
    """A chunk behind a long past, whose keys many workgroups share: one NaN in the past makes its channel NaN in all rows, and no
    other element changes."""
    c = Paged(kind, 8, 2, 128, 32, [(40, 20000)], seed=25)
    clean = c.attend()
    check(c, clean)
    x = c.v.view(torch.uint8) if kind == "e4m3" else c.v
    x[int(c.table_h[0, 5000 // 32]), 1, 5000 % 32, 77] = 0x7F if kind == "e4m3" else float("nan")
    got = c.attend()
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[:, 4:, 77] = True
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], clean[~hit])


def test_tensors_elsewhere_are_refused():
    c = Paged("bf16", 4, 2, 64, 16, [(2, 20)], seed=26)
    q, k, v = c.parts()
    host = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    ws = c.workspace()
    for bad in ((host, torch.zeros_like(c.q), ws), (c.q, host, ws), (c.q, torch.zeros_like(c.q), ws.cpu())):
        with pytest.raises(ValueError):
            pd.pd_paged_attention(c.kv, c.seqs, *bad)
    with pytest.raises(ValueError):
        pd.pd_paged_append(c.kv, c.seqs, k.cpu(), v)
    with pytest.raises(ValueError):
        pd.pd_paged_append(c.kv, c.seqs, k, v, 0.0, q, host)
    with pytest.raises(ValueError):
        pd.pd_paged_append(c.kv, c.seqs, k, v, 0.0, q)
    with pytest.raises(ValueError):
        pd.pd_paged_attention(pd.make_paged_kv(c.k.cpu(), c.v.cpu()), c.seqs, c.q, torch.zeros_like(c.q), ws)
    with pytest.raises(ValueError):
        pd.make_paged_kv(c.k, c.v.cpu())
    with pytest.raises(ValueError):
        pd.make_paged_seqs(c.lens, c.table.cpu())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv", [(300, 1), (1024, 1), (99, 3)])
def test_large_groups(kind, hq, hkv):
    """A token's heads fill a tile of rows, or several."""
    c = Paged(kind, hq, hkv, 64, 16, [(1, 90), (1, 700), (1, 0)], seed=27, starts=False)
    check(c, c.attend())
    c = Paged(kind, hq, hkv, 64, 16, [(3, 90), (1, 900), (2, 1), (7, 7)], pad=1, seed=28)
    check(c, c.attend())


@pytest.mark.parametrize("kind", KINDS)
def test_chunks_replayed_from_a_graph(kind):
    """A captured call of chunks, drafts and single rows, replayed while starts, lengths and page numbers change on the device: each replay
    equals the eager call, with eager work between the replays."""
    steps = [[(100, 300), (1, 700), (9, 9), (40, 1500)], [(1, 301), (140, 840), (5, 14), (4, 1504)], [(0, 301), (1, 841), (149, 163), (0, 0)]]
    c = Paged(kind, 8, 2, 128, 32, [(n, 1600) for n in (50, 50, 25, 25)], seed=29)
    out = torch.zeros_like(c.q)
    ws = c.workspace()
    k, v = c.parts()[1:]
    pages = [t.clone() for t in (c.k, c.v, c.ks, c.vs) if t is not None]

    def call(q_out, out):
        pd.pd_paged_append(c.kv, c.seqs, k, v, 10000.0, c.q, q_out)
        pd.pd_paged_attention(c.kv, c.seqs, q_out, out, ws)

    def reset(step):
        for t, kept in zip([t for t in (c.k, c.v, c.ks, c.vs) if t is not None], pages):
            t.copy_(kept)
        c.row_starts.copy_(torch.tensor([0] + list(np.cumsum([n for n, _ in step])), dtype=torch.int32))
        c.lens.copy_(torch.tensor([m for _, m in step], dtype=torch.int32))
        c.table.copy_(c.table[[1, 2, 3, 0]])

    q_out = torch.zeros_like(c.q)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(q_out, out)
    for i in range(6):
        reset(steps[i % 3])
        out.fill_(7.0)
        graph.replay()
        got, got_k = out.clone(), c.k.clone()
        table = c.table.clone()
        reset(steps[i % 3])
        c.table.copy_(table)
        eager_q, eager = torch.zeros_like(c.q), torch.full_like(out, 7.0)
        call(eager_q, eager)
        torch.cuda.synchronize()
        assert torch.equal(got, eager) and torch.equal(got_k.view(torch.uint8), c.k.view(torch.uint8)), i
        assert torch.isfinite(eager.float()).all()

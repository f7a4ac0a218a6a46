"""The paged cache without a GPU: its oracle against library routines, and what the entry points refuse before they touch a
device (the non-NULL pointers below are never dereferenced)."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2603_04716_amd as pd
from oracle import paged as P


def test_oracle_codes_are_the_librarys():
    x = torch.arange(0x8000, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = torch.cat([x, -x]).float()
    x = x[x.abs() <= 448]
    want = x.to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(P.nearest_code(x.double().numpy()), want)
    rng = np.random.default_rng(0)
    y = (rng.standard_normal(200000) * 2.0 ** rng.integers(-14, 9, 200000)).astype(np.float32).clip(-448, 448)
    np.testing.assert_array_equal(P.nearest_code(y), torch.from_numpy(y).to(torch.float8_e4m3fn).double().numpy())
    assert P.nearest_code([1e9, -np.inf, np.inf])[0] == 448 and np.isnan(P.nearest_code(np.nan))


def test_oracle_scale():
    assert P.scale_for([0.0]) == 2.0 ** -60 and P.scale_for([448.0]) == 1.0 and P.scale_for([-448.5]) == 2.0
    assert P.scale_for([1.75 * 2.0 ** -40]) == 2.0 ** -48 and P.scale_for([np.inf, np.nan, 3.0]) == 2.0 ** -7


@pytest.mark.parametrize("ps", [16, 64])
def test_oracle_append_then_attend_is_attention_over_the_sequence(ps):
    """Prompts appended to an empty pool in two chunks, against torch's attention in float64 on rows rotated as complex numbers."""
    torch.manual_seed(0)
    hq, hkv, hd = 6, 2, 32
    lens, first = [37, 5, 80], [20, 5, 16]
    width = -(-max(lens) // ps)
    table = np.random.default_rng(1).permutation(len(lens) * width).reshape(len(lens), width)
    pool = [np.full((len(lens) * width, hkv, ps, hd), np.nan) for _ in range(2)]
    x = [torch.randn(n, hq + 2 * hkv, hd, dtype=torch.float64) for n in lens]

    def turned(t):
        a = torch.arange(t.shape[0], dtype=torch.float64)[:, None] * 500.0 ** (-torch.arange(0, hd, 2, dtype=torch.float64) / hd)
        z = torch.complex(t[..., :hd // 2], t[..., hd // 2:]) * torch.polar(torch.ones_like(a), a)[:, None]
        return torch.cat([z.real, z.imag], -1)

    for lo, hi in ((0, first), (first, lens)):
        lo = [0] * len(lens) if lo == 0 else lo
        rows = torch.cat([t[a:b] for t, a, b in zip(x, lo, hi)]).numpy()
        starts = np.concatenate([[0], np.cumsum([b - a for a, b in zip(lo, hi)])])
        pool[0], pool[1], _, _ = P.append(pool[0], pool[1], None, None, starts, hi, table, rows[:, hq:hq + hkv], rows[:, hq + hkv:], 500.0)
        q = np.concatenate([turned(t[:, :hq])[a:b].numpy() for t, a, b in zip(x, lo, hi)])
        got, weight, _ = P.attend(pool[0], pool[1], None, None, starts, hi, table, q, hd ** -0.5)
        for b, t in enumerate(x):
            m = t[:hi[b]]
            want = torch.nn.functional.scaled_dot_product_attention(
                turned(m[:, :hq]).transpose(0, 1), turned(m[:, hq:hq + hkv]).repeat_interleave(hq // hkv, 1).transpose(0, 1),
                m[:, hq + hkv:].repeat_interleave(hq // hkv, 1).transpose(0, 1), is_causal=True).transpose(0, 1)[lo[b]:]
            np.testing.assert_allclose(got[starts[b]:starts[b + 1]], want.numpy(), rtol=1e-10, atol=1e-12)
            assert (weight[starts[b]:starts[b + 1]] >= np.abs(want.numpy()) - 1e-12).all()


def kv_of(**over):
    f = dict(k=0x1000, v=0x2000, k_scales=0x3000, v_scales=0x4000, n_pages=8, page_size=64, n_kv_heads=2, head_dim=128, dtype=pd.PD_BF16, e4m3=0)
    f.update(over)
    return pd.pd_paged_kv(**f)


def seqs_of(**over):
    f = dict(n_seqs=3, n_rows=7, row_starts=0x5000, lens=0x6000, page_table=0x7000, table_width=4)
    f.update(over)
    return pd.pd_paged_seqs(**f)


def rows_of(**over):
    f = dict(k=0x8000, v=0x9000, q=0xA000, q_out=0xB000, k_stride=1024, v_stride=1024, q_stride=1024, q_out_stride=512, n_q_heads=4, rope_base=1e4)
    f.update(over)
    return pd.pd_paged_rows(**f)


BAD_KV = [(dict(k=None), pd.PD_ERR_INVALID_ARG), (dict(v=None), pd.PD_ERR_INVALID_ARG), (dict(k=0x1008), pd.PD_ERR_INVALID_ARG),
          (dict(e4m3=1, k_scales=None), pd.PD_ERR_INVALID_ARG), (dict(e4m3=1, v_scales=None), pd.PD_ERR_INVALID_ARG),
          (dict(e4m3=1, dtype=pd.PD_F32), pd.PD_ERR_DTYPE), (dict(dtype=2), pd.PD_ERR_DTYPE), (dict(page_size=48), pd.PD_ERR_SHAPE),
          (dict(page_size=8), pd.PD_ERR_SHAPE), (dict(page_size=256), pd.PD_ERR_SHAPE), (dict(head_dim=96), pd.PD_ERR_SHAPE), (dict(n_pages=0), pd.PD_ERR_SHAPE),
          (dict(n_kv_heads=0), pd.PD_ERR_SHAPE)]
BAD_SEQS = [(dict(lens=None), pd.PD_ERR_INVALID_ARG), (dict(page_table=None), pd.PD_ERR_INVALID_ARG), (dict(n_seqs=-1), pd.PD_ERR_INVALID_ARG),
            (dict(n_seqs=4097), pd.PD_ERR_INVALID_ARG), (dict(n_rows=-1), pd.PD_ERR_INVALID_ARG), (dict(n_rows=(1 << 24) + 1), pd.PD_ERR_INVALID_ARG),
            (dict(table_width=0), pd.PD_ERR_SHAPE), (dict(table_width=(1 << 24) + 1), pd.PD_ERR_SHAPE), (dict(row_starts=None, n_rows=2), pd.PD_ERR_SHAPE)]


def append(kv=None, seqs=None, rows=None):
    return pd.lib.pd_paged_append(C.byref(kv or kv_of()), C.byref(seqs or seqs_of()), C.byref(rows or rows_of()), None)


def attention(kv=None, seqs=None, q=0xA000, stride=1024, heads=4, scale=0.1, out=0xB000, ws=0xC000, ws_bytes=1 << 40):
    return pd.lib.pd_paged_attention(C.byref(kv or kv_of()), C.byref(seqs or seqs_of()), q, stride, heads, scale, out, ws, ws_bytes, None)


def workspace(kv=None, seqs=None, heads=4):
    n = C.c_int64(-1)
    st = pd.lib.pd_paged_attention_workspace(C.byref(kv or kv_of()), C.byref(seqs or seqs_of()), heads, C.byref(n))
    return st, n.value


def test_refusals():
    for over, status in BAD_KV:
        assert append(kv=kv_of(**over)) == attention(kv=kv_of(**over)) == status, over
        assert workspace(kv=kv_of(**over)) == (status, -1)
    for over, status in BAD_SEQS:
        assert append(seqs=seqs_of(**over)) == attention(seqs=seqs_of(**over)) == status, over
        assert workspace(seqs=seqs_of(**over)) == (status, -1)
    for over, status in [(dict(k=None), 1), (dict(v=0x9004), 1), (dict(q_out=None), 1), (dict(k_stride=248), 2), (dict(v_stride=260), 2),
                         (dict(q_stride=0), 2), (dict(q_out_stride=-512), 2), (dict(n_q_heads=3), 2), (dict(n_q_heads=0), 2),
                         (dict(rope_base=-1.0), 1), (dict(rope_base=float("nan")), 1), (dict(rope_base=float("inf")), 1)]:
        assert append(rows=rows_of(**over)) == status, over
    for over, status in [(dict(q=None), 1), (dict(q=0xA002), 1), (dict(stride=511), 2), (dict(stride=504), 2), (dict(heads=5), 2), (dict(heads=2048), 2),
                         (dict(scale=float("nan")), 1), (dict(scale=0.0), 1), (dict(scale=-0.1), 1), (dict(scale=float("inf")), 1), (dict(out=None), 1), (dict(out=0xB008), 1)]:
        assert attention(**over) == status, over
    st, need = workspace(seqs=seqs_of(table_width=64))
    assert st == pd.PD_OK and need > 0
    for over in (dict(ws=None), dict(ws=0xC004), dict(ws_bytes=need - 1)):
        assert attention(seqs=seqs_of(table_width=64), **over) == pd.PD_ERR_INVALID_ARG, over
    assert b"workspace" in pd.lib.pd_last_error()
    assert pd.lib.pd_paged_append(None, None, None, None) == pd.PD_ERR_INVALID_ARG
    assert pd.lib.pd_paged_attention_workspace(C.byref(kv_of()), C.byref(seqs_of()), 4, None) == pd.PD_ERR_INVALID_ARG
    assert append(seqs=seqs_of(n_rows=1 << 24), rows=rows_of(n_q_heads=1024, q_stride=1 << 17, q_out_stride=1 << 17)) == pd.PD_ERR_SHAPE


def test_calls_of_nothing_are_calls():
    for over in (dict(n_seqs=0), dict(n_rows=0), dict(n_seqs=0, n_rows=0, row_starts=None, lens=None, page_table=None)):
        assert append(seqs=seqs_of(**over)) == attention(seqs=seqs_of(**over), ws=None, ws_bytes=0) == pd.PD_OK
        assert workspace(seqs=seqs_of(**over)) == (pd.PD_OK, 0)


def test_workspace_is_bounded():
    """It does not grow with the table behind a few chunks, nor with the rows behind the items that a launch aims for."""
    big = workspace(seqs=seqs_of(n_seqs=4096, n_rows=1 << 20, table_width=1 << 20))[1]
    assert 0 < workspace(seqs=seqs_of(table_width=64))[1] <= big < 256 << 20
    assert workspace(seqs=seqs_of(n_seqs=1, n_rows=1, row_starts=None, table_width=1))[1] == 0


def test_descriptors_refuse_other_tensors():
    pages = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    scales = torch.zeros(4, 2)
    for bad in ((pages.half(), pages.half()), (pages, pages.float()), (pages, pages[:, :, :8]), (pages, pages.transpose(1, 2)), (pages, pages, scales, scales),
                (pages.to(torch.uint8), pages.to(torch.uint8)), (pages.to(torch.uint8), pages.to(torch.uint8), scales, scales.double())):
        with pytest.raises(ValueError):
            pd.make_paged_kv(*bad)
    kv = pd.make_paged_kv(pages, pages.clone())
    lens, table, starts = torch.zeros(3, dtype=torch.int32), torch.zeros(3, 5, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    for bad in ((lens.long(), table), (lens, table.t()), (lens, table[:2]), (lens, table, starts), (lens, table, starts[:3], 7)):
        with pytest.raises(ValueError):
            pd.make_paged_seqs(*bad)
    seqs = pd.make_paged_seqs(lens, table, starts, 7)
    rows = torch.zeros(7, 8, 64, dtype=torch.bfloat16)
    for bad in (rows[:6, :2], rows[:, :3], rows[:, :2].float(), rows[:, ::4], rows[:, :2, ::2]):
        with pytest.raises(ValueError):
            pd.pd_paged_append(kv, seqs, bad, rows[:, 2:4])
    with pytest.raises(ValueError):
        pd.pd_paged_attention(kv, seqs, rows[:, :4].contiguous(), rows[:, :4], rows)


def test_sizes_set_in_a_descriptor_are_the_sizes_that_tensors_are_held_to():
    """A program that sets a descriptor's n_rows for its next call may not have a kernel read rows that its tensors do not have."""
    kv = pd.make_paged_kv(torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16))
    seqs = pd.make_paged_seqs(torch.zeros(3, dtype=torch.int32), torch.zeros(3, 5, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), 7)
    rows = torch.zeros(7, 4, 64, dtype=torch.bfloat16)
    seqs.n_rows = 9
    with pytest.raises(ValueError):
        pd.pd_paged_append(kv, seqs, rows[:, :2], rows[:, 2:])
    with pytest.raises(ValueError):
        pd.pd_paged_attention(kv, seqs, rows, torch.zeros_like(rows), rows)
    seqs.n_rows = 7
    kv.n_kv_heads = 3
    with pytest.raises(ValueError):
        pd.pd_paged_append(kv, seqs, rows[:, :2], rows[:, 2:])
    kv.n_kv_heads, kv.head_dim = 2, 128
    with pytest.raises(ValueError):
        pd.pd_paged_attention(kv, seqs, rows, torch.zeros_like(rows), rows)

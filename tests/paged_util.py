"""Pools, page tables and calls of the paged key/value cache for its tests, and the bounds that its outputs are held to."""
import numpy as np
import torch

import paper_2603_04716_amd as pd

ROW = {"bf16": torch.bfloat16, "e4m3": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}       # of a rounding to the type, relative to the value


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


class Paged:
    """A pool with random contents, and sequences given as (new rows, positions held with them)."""

    def __init__(self, kind, hq, hkv, hd, ps, seqs, pad=0, seed=0, spare=2, extra_width=0, starts=True):
        rng = np.random.default_rng(seed)
        g = torch.Generator("cuda")
        g.manual_seed(seed)
        self.kind, self.hq, self.hkv, self.hd, self.ps = kind, hq, hkv, hd, ps
        self.new = [n for n, _ in seqs]
        self.lens_h = [length for _, length in seqs]
        self.starts_h = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.n_rows = int(self.starts_h[-1]) + pad
        pages = [-(-length // ps) for length in self.lens_h]
        n_pages = sum(pages) + spare
        width = max(pages + [1]) + extra_width
        order = rng.permutation(n_pages)
        self.table_h = rng.integers(0, n_pages, (len(seqs), width)).astype(np.int32)
        at = 0
        for b, n in enumerate(pages):
            self.table_h[b, :n] = order[at:at + n]
            at += n

        def normal(*shape):
            return torch.randn(*shape, generator=g, device="cuda")

        shape = (n_pages, hkv, ps, hd)
        if kind == "e4m3":
            self.k, self.v = ((normal(*shape) * 64).clamp(-448, 448).to(torch.float8_e4m3fn) for _ in range(2))
            self.ks, self.vs = (2.0 ** torch.randint(-8, -4, shape[:2], generator=g, device="cuda").float() for _ in range(2))
        else:
            self.k, self.v = (normal(*shape).to(ROW[kind]) for _ in range(2))
            self.ks = self.vs = None
        self.qkv = (normal(self.n_rows, hq + 2 * hkv, hd) * torch.exp(0.7 * normal(self.n_rows, 1, 1))).to(ROW[kind])
        self.q = (1.5 * normal(self.n_rows, hq, hd)).to(ROW[kind])
        self.starts = starts
        self.bind()

    def bind(self):
        """Device arrays and descriptors of what the host fields say now."""
        self.lens = torch.tensor(self.lens_h, dtype=torch.int32, device="cuda")
        self.table = torch.from_numpy(self.table_h).cuda()
        self.row_starts = torch.from_numpy(self.starts_h).cuda() if self.starts else None
        self.kv = pd.make_paged_kv(self.k, self.v, self.ks, self.vs)
        self.seqs = pd.make_paged_seqs(self.lens, self.table, self.row_starts, self.n_rows)

    def host(self):
        """k, v, k_scales, v_scales as float64 arrays."""
        return tuple(None if t is None else f64(t) for t in (self.k, self.v, self.ks, self.vs))

    def parts(self):
        return self.qkv[:, :self.hq], self.qkv[:, self.hq:self.hq + self.hkv], self.qkv[:, self.hq + self.hkv:]

    def workspace(self, slack=0):
        n = pd.pd_paged_attention_workspace(self.kv, self.seqs, self.hq)
        return torch.full((n + slack,), 0xA5, dtype=torch.uint8, device="cuda")       # no initial value is needed

    def attend(self, q=None, out=None, ws=None, scale=None):
        q = self.q if q is None else q
        out = torch.full((self.n_rows, self.hq, self.hd), 7.0, dtype=q.dtype, device="cuda") if out is None else out
        pd.pd_paged_attention(self.kv, self.seqs, q, out, self.workspace() if ws is None else ws, scale)
        return out


def attention_bound(kind, out, weight, delta, lens, starts, hd):
    """|got - exact| allowed per element.  A score's error is at most hd roundings of its partial sums (2^-24 each, of the sum
    of magnitudes delta) and three more for scale, log2 e and the subtraction, and the exponential's own 2^-21, in all
    e(delta); both numerator and denominator change by that share.  Sums over L keys add L 2^-24.  In bf16 each
    exponential is rounded once (2^-8), and every type's output once."""
    e = (hd + 8) * 2.0 ** -24 * delta + 2.0 ** -21
    keys = np.zeros(out.shape[0])
    for b, n in enumerate(lens):
        keys[starts[b]:starts[b + 1]] = n
    share = 2 * e[:, :, None] + 2 * keys[:, None, None] * 2.0 ** -24
    if kind != "f32":
        share = share + 2.0 ** -8
    return share * weight + HALF_STEP["f32" if kind == "f32" else "bf16"] * np.abs(out) * (1 + share) + 1e-30

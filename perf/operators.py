"""The paged key/value cache as measurable cases: appending rows to it (rotated on the way, in the rows' own type or as E4M3
codes with a scale per page and kv head) and attention over it.

A case is a dict of plain values.  `layout` fixes the sequences' lengths, the seed everything else.
  op        append | attend
  kind      bf16 | f32: pages in the rows' type; e4m3: bf16 rows, pages of E4M3 codes
  seqs      sequences; each holds past positions (past_lo .. past_hi) and brings new rows (new_lo .. new_hi)
  idle      how many of them are empty slots of a fixed-size batch: length 0, one row that sees nothing
  pad       rows behind the last sequence (a fixed-size chunk that is not full)
"""
import math
import random

import torch

own = False

ROPE_BASE = 500000.0
SMALLEST_SCALE = 2.0 ** -60


def _case(name, op, kind, **over):
    c = dict(op=op, kind=kind, hq=32, hkv=8, hd=128, ps=64, seqs=1, past_lo=0, past_hi=0, new_lo=1, new_hi=1, idle=0, pad=0, layout=1)
    c.update(over)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user's stream: the smallest call there is, all latency
        _case("append_b1", "append", "bf16", past_lo=517, past_hi=517),
        # a full decode batch on 8-bit pages, some slots of the captured batch empty
        _case("append_b256_e4m3", "append", "e4m3", seqs=256, past_lo=1, past_hi=600, idle=6),
        # a step of ragged chunks: prompts' pieces beside running sequences, five query heads per kv head, small pages
        _case("append_chunks", "append", "bf16", hq=40, ps=16, seqs=24, past_lo=0, past_hi=1500, new_lo=1, new_hi=700, pad=37, layout=2),
        # four prompts of 2048 tokens stored in 8 bits
        _case("append_4x2048_e4m3", "append", "e4m3", seqs=4, new_lo=2048, new_hi=2048),
        # the fp32 two-layer configuration that a deployment is checked with
        _case("append_f32", "append", "f32", hq=4, hkv=4, hd=64, ps=32, seqs=8, past_lo=3, past_hi=200, new_lo=1, new_hi=150, layout=3),
        # one user's stream again: one query row per head over a short context
        _case("attend_b1", "attend", "bf16", past_lo=700, past_hi=700),
        # an ordinary decode batch caught mid-generation
        _case("attend_b64", "attend", "bf16", seqs=64, past_lo=100, past_hi=8000, layout=4),
        # throughput decode on 8-bit pages
        _case("attend_b256_e4m3", "attend", "e4m3", seqs=256, past_lo=1500, past_hi=2600, idle=5, layout=5),
        # one long document, one token at a time
        _case("attend_b1_long", "attend", "bf16", ps=128, past_lo=131000, past_hi=131000),
        # the headline prefill call: four prompts of 2048 tokens, matrix-bound
        _case("attend_4x2048", "attend", "bf16", seqs=4, new_lo=2048, new_hi=2048),
        # chunks of prompts and running sequences in one call on 8-bit pages
        _case("attend_mixed_e4m3", "attend", "e4m3", seqs=12, past_lo=0, past_hi=6000, new_lo=1, new_hi=700, pad=19, layout=6),
        # the fp32 check configuration: short ragged chunks
        _case("attend_f32", "attend", "f32", hq=4, hkv=4, hd=64, ps=16, seqs=9, past_lo=0, past_hi=900, new_lo=1, new_hi=60, layout=7),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["append", "attend", "attend"])
    kind = rng.choice(["bf16", "bf16", "e4m3", "e4m3", "f32"])
    hq, hkv = rng.choice([(32, 8), (32, 8), (4, 4), (16, 2), (40, 8), (8, 1), (12, 4)])
    hd, ps = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128])
    step = rng.choice(["decode", "decode", "draft", "chunk"])
    if step == "chunk":
        seqs = log(1, 12)
        new_hi = log(2, 8192 // seqs)
        new_lo = rng.choice([1, new_hi])
    else:
        seqs = log(1, 256)
        new_lo, new_hi = (1, 1) if step == "decode" else (1, rng.randint(2, 8))
    past_hi = log(1, 8192)
    # no dearer than the listed cases: elements of the cache, and of the scores of a padded batch
    past_hi = min(past_hi, (1 << (28 if op == "attend" and kind != "f32" else 27)) // (seqs * hkv * hd))
    if op == "attend":
        most = 400_000_000 if kind != "f32" else 100_000_000
        new_hi = max(1, min(new_hi, int(math.sqrt(most / (seqs * hq)))))
        new_lo = min(new_lo, new_hi)
        past_hi = max(0, min(past_hi, most // (seqs * hq * new_hi) - new_hi))
    idle = rng.randint(0, 3) if step == "decode" and seqs >= 8 else 0
    pad = rng.randint(1, 50) if step != "decode" and rng.random() < 0.3 else 0
    return _case(None, op, kind, hq=hq, hkv=hkv, hd=hd, ps=ps, seqs=seqs, past_lo=rng.choice([0, past_hi // 2, past_hi]), past_hi=past_hi,
                 new_lo=new_lo, new_hi=new_hi, idle=idle, pad=pad, layout=rng.randrange(1 << 20))


def lengths(case):
    """(new rows, positions held with them) of every sequence."""
    r = random.Random(case["layout"])
    both = []
    for b in range(case["seqs"]):
        past, new = r.randint(case["past_lo"], case["past_hi"]), r.randint(case["new_lo"], case["new_hi"])
        both.append((1, 0) if b >= case["seqs"] - case["idle"] else (new, past + new))
    return both


def work(case):
    hq, hkv, hd, both = case["hq"], case["hkv"], case["hd"], lengths(case)
    e = 4 if case["kind"] == "f32" else 2
    ep = 1 if case["kind"] == "e4m3" else e
    rows = sum(n for n, length in both if length)
    if case["op"] == "append":
        return {"bytes": rows * hd * ((hq + 2 * hkv) * e + hq * e + 2 * hkv * ep), "flops": 6 * rows * (hq + hkv) * hd // 2}
    held = sum(length for _, length in both)
    seen = sum(n * length - n * (n - 1) // 2 for n, length in both if length)
    return {"bytes": held * 2 * hkv * hd * ep + 2 * rows * hq * hd * e, "flops": 4 * hd * hq * seen}


def prepare(case, seed):
    hq, hkv, hd, ps, kind = case["hq"], case["hkv"], case["hd"], case["ps"], case["kind"]
    g = torch.Generator("cuda")
    g.manual_seed(seed)
    both = lengths(case)
    starts = [0]
    for n, _ in both:
        starts.append(starts[-1] + n)
    rows = starts[-1] + case["pad"]
    most = max(1, max(-(-length // ps) for _, length in both))
    used = sum(-(-length // ps) for _, length in both)
    n_pages = used + 3
    # a table row's unused entries point anywhere, as a scheduler leaves them
    order = torch.randperm(n_pages, generator=g, device="cuda")
    table = torch.randint(0, n_pages, (case["seqs"], most), generator=g, device="cuda", dtype=torch.int32)
    held = torch.tensor([-(-length // ps) for _, length in both], device="cuda")
    mine = torch.arange(most, device="cuda")[None, :] < held[:, None]
    table[mine] = order[:used].to(torch.int32)
    dtype = torch.float32 if kind == "f32" else torch.bfloat16

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = dict(case=case, both=both, rows=rows, most_new=max(n for n, _ in both),
             starts=torch.tensor(starts, device="cuda", dtype=torch.int32),
             lens=torch.tensor([length for _, length in both], device="cuda", dtype=torch.int32), table=table)
    if kind == "e4m3":
        for name in ("k", "v"):
            s[name + "_pages"] = torch.empty(n_pages, hkv, ps, hd, device="cuda", dtype=torch.float8_e4m3fn)
            for i in range(0, n_pages, 4096):
                part = s[name + "_pages"][i:i + 4096]
                part.copy_((normal(*part.shape) * 64.0).clamp(-448.0, 448.0))
            s[name + "_scales"] = 2.0 ** torch.randint(-7, -5, (n_pages, hkv), generator=g, device="cuda").float()
    else:
        for name in ("k", "v"):
            s[name + "_pages"] = normal(n_pages, hkv, ps, hd).to(dtype)
            s[name + "_scales"] = None
    if case["op"] == "append":
        # rows as the projection leaves them: q, k and v of a row side by side; some rows much larger than the rest
        size = torch.exp(0.7 * normal(rows, 1, 1))
        s["qkv"] = (normal(rows, hq + 2 * hkv, hd) * size).to(dtype)
        s["q_out"] = torch.zeros(rows, hq, hd, device="cuda", dtype=dtype)
    else:
        s["q"] = (1.5 * normal(rows, hq, hd)).to(dtype)
        s["out"] = torch.zeros(rows, hq, hd, device="cuda", dtype=dtype)
    if own:                                  # what the program keeps beside its tensors: two descriptors and a workspace
        import paper_2603_04716_amd as pd
        s["kv"] = pd.make_paged_kv(s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"])
        one_row_each = s["most_new"] == 1 and rows == case["seqs"]
        s["seqs"] = pd.make_paged_seqs(s["lens"], table, None if one_row_each else s["starts"], rows)
        if case["op"] == "attend":
            s["ws"] = torch.empty(pd.pd_paged_attention_workspace(s["kv"], s["seqs"], hq), device="cuda", dtype=torch.uint8)
    return s


def run(s):
    if s["case"]["op"] == "append":
        if own:
            import paper_2603_04716_amd as pd
            hq, hkv = s["case"]["hq"], s["case"]["hkv"]
            q, k, v = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hkv], s["qkv"][:, hq + hkv:]
            pd.pd_paged_append(s["kv"], s["seqs"], k, v, ROPE_BASE, q, s["q_out"])
        else:
            _append(s)
        out = {"q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"]}
        if s["k_scales"] is not None:
            out.update(k_scales=s["k_scales"], v_scales=s["v_scales"])
        return out
    if own:
        import paper_2603_04716_amd as pd
        pd.pd_paged_attention(s["kv"], s["seqs"], s["q"], s["out"], s["ws"])
        return s["out"]
    return _attend(s)


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _append(s):
    case, starts, lens = s["case"], s["starts"].long(), s["lens"].long()
    hq, hkv, hd, ps = case["hq"], case["hkv"], case["hd"], case["ps"]
    row = torch.arange(s["rows"], device="cuda")
    seq = torch.searchsorted(starts[1:], row, right=True).clamp(max=case["seqs"] - 1)
    pos = lens[seq] - (starts[seq + 1] - row)
    keep = ((row < starts[-1]) & (pos >= 0)).nonzero()[:, 0]
    seq, pos = seq[keep], pos[keep]
    page, slot = s["table"][seq, pos // ps].long(), pos % ps
    x = s["qkv"][keep].float()
    turn = pos.double()[:, None] * ROPE_BASE ** (-2.0 * torch.arange(hd // 2, device="cuda", dtype=torch.float64) / hd)
    c, n = torch.cos(turn).float()[:, None], torch.sin(turn).float()[:, None]

    def rotated(y):
        a, b = y[..., :hd // 2], y[..., hd // 2:]
        return torch.cat([a * c - b * n, a * n + b * c], -1)

    s["q_out"][keep] = rotated(x[:, :hq]).to(s["q_out"].dtype)
    k, v = rotated(x[:, hq:hq + hkv]), x[:, hq + hkv:]
    if s["k_scales"] is None:
        s["k_pages"][page, :, slot] = k.to(s["k_pages"].dtype)
        s["v_pages"][page, :, slot] = v.to(s["v_pages"].dtype)
        return
    n_pages = s["k_pages"].shape[0]
    first = torch.full((n_pages,), ps, device="cuda").scatter_reduce(0, page, slot, "amin")
    _append_codes(s["k_pages"], s["k_scales"], k, page, slot, first)
    _append_codes(s["v_pages"], s["v_scales"], v, page, slot, first)


def _append_codes(pages, scales, x, page, slot, first):
    n_pages, hkv, ps, _ = pages.shape
    most = torch.zeros(n_pages, hkv, device="cuda").scatter_reduce(0, page[:, None].expand(-1, hkv), x.abs().amax(-1), "amax")
    m, e = torch.frexp(most.double() / 448.0)
    need = torch.where(most > 0, torch.ldexp(torch.ones_like(m), torch.where(m == 0.5, e - 1, e)).float(), 0.0).clamp(min=SMALLEST_SCALE)
    new = torch.where(first[:, None] == 0, need, torch.maximum(need, scales))
    hit = torch.unique(page)
    old = pages[hit].float()
    again = (old * (scales[hit] / new[hit])[:, :, None, None]).clamp(-448.0, 448.0)
    before = torch.arange(ps, device="cuda")[None, None, :, None] < first[hit][:, None, None, None]
    pages[hit] = torch.where(before, again, old).to(pages.dtype)
    scales[hit] = new[hit]
    pages.view(torch.uint8)[page, :, slot] = (x / new[page][:, :, None]).clamp(-448.0, 448.0).to(pages.dtype).view(torch.uint8)


def _attend(s):
    case, starts, lens = s["case"], s["starts"].long(), s["lens"].long()
    hq, hkv, hd, seqs, most = case["hq"], case["hkv"], case["hd"], case["seqs"], s["most_new"]
    table = s["table"].long()

    def dense(pages, scales):
        x = pages[table].float() if scales is None else pages[table].float() * scales[table][..., None, None]
        return x.transpose(1, 2).reshape(seqs, hkv, -1, hd)

    k, v = dense(s["k_pages"], s["k_scales"]), dense(s["v_pages"], s["v_scales"])
    i = torch.arange(most, device="cuda")
    new = starts[1:] - starts[:-1]
    row = (starts[:-1, None] + i).clamp(max=s["rows"] - 1)
    pos = torch.where(i < new[:, None], lens[:, None] - new[:, None] + i, -1)
    q = s["q"][row].float().reshape(seqs, most, hkv, hq // hkv, hd).permute(0, 2, 3, 1, 4).reshape(seqs, hkv, -1, hd)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(hd))
    score = score.view(seqs, hkv, hq // hkv, most, -1)
    score.masked_fill_(torch.arange(score.shape[-1], device="cuda") > pos[:, None, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(seqs, hkv, -1, p.shape[-1]), v).view(seqs, hkv, hq // hkv, most, hd)
    o = (o / torch.where(total == 0, 1.0, total)).permute(0, 3, 1, 2, 4).reshape(seqs, most, hq, hd).to(s["q"].dtype)
    out = torch.zeros(s["rows"], hq, hd, device="cuda", dtype=s["q"].dtype)
    mine = i < new[:, None]
    out[row[mine]] = o[mine]
    return out


# ---- the definitions in 64 bits, sequence by sequence ----------------------------------------------------------------

def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    return _exact_append(s) if case["op"] == "append" else _exact_attend(s)


def _exact_attend(s):
    case = s["case"]
    hq, hkv, hd, ps = case["hq"], case["hkv"], case["hd"], case["ps"]
    out = torch.zeros(s["rows"], hq, hd, device="cuda", dtype=torch.float64)
    at = 0
    for b, (n, length) in enumerate(s["both"]):
        if length:
            pages = s["table"][b, :-(-length // ps)].long()
            for h in range(hkv):
                k, v = s["k_pages"][pages, h].double(), s["v_pages"][pages, h].double()
                if s["k_scales"] is not None:
                    k, v = k * s["k_scales"][pages, h].double()[:, None, None], v * s["v_scales"][pages, h].double()[:, None, None]
                k, v = k.reshape(-1, hd)[:length], v.reshape(-1, hd)[:length]
                for j in range(hq // hkv):
                    w = s["q"][at:at + n, h * (hq // hkv) + j].double() @ k.t() / math.sqrt(hd)
                    w = w + torch.full((n, length), -math.inf, device="cuda", dtype=torch.float64).triu(length - n + 1)
                    out[at:at + n, h * (hq // hkv) + j] = torch.softmax(w, -1) @ v
        at += n
    return out


def _power_of_two(e):
    return torch.tensor([math.ldexp(1.0, i) for i in range(-200, 200)], device="cuda", dtype=torch.float64)[e.long() + 200]


def _nearest_code(x):
    """The value of the E4M3 code nearest to x, ties to the even mantissa, at most 448."""
    step = _power_of_two(torch.frexp(x)[1].clamp(min=-5) - 4)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _exact_append(s):
    case = s["case"]
    hq, hkv, hd, ps = case["hq"], case["hkv"], case["hd"], case["ps"]
    half = hd // 2
    pages = {"k": s["k_pages"].double(), "v": s["v_pages"].double()}
    scales = {"k": s["k_scales"], "v": s["v_scales"]}
    if s["k_scales"] is not None:
        scales = {name: t.double() for name, t in scales.items()}
    q_out = s["q_out"].double()
    power = torch.tensor([math.pow(ROPE_BASE, -2.0 * c / hd) for c in range(half)], device="cuda", dtype=torch.float64)
    at = 0
    for b, (n, length) in enumerate(s["both"]):
        if length:
            x = s["qkv"][at:at + n].double()
            p0 = length - n
            z = torch.polar(torch.ones(n, half, device="cuda", dtype=torch.float64),
                            torch.arange(p0, length, device="cuda", dtype=torch.float64)[:, None] * power)[:, None]
            y = torch.complex(x[:, :hq + hkv, :half], x[:, :hq + hkv, half:]) * z
            y = torch.cat([y.real, y.imag], -1)
            q_out[at:at + n] = y[:, :hq]
            new = {"k": y[:, hq:], "v": x[:, hq + hkv:]}
            numbers = s["table"][b].tolist()
            for name in ("k", "v"):
                for t in range(p0 // ps, (length - 1) // ps + 1):
                    page, lo, hi = numbers[t], max(p0, t * ps), min(length, t * ps + ps)
                    part = new[name][lo - p0:hi - p0].transpose(0, 1)
                    slot = lo - t * ps
                    if s["k_scales"] is not None:
                        m, e = torch.frexp(part.abs().amax((1, 2)) / 448.0)
                        need = _power_of_two(torch.where(m == 0.5, e - 1, e).clamp(min=-60))
                        if slot:
                            old = scales[name][page].clone()
                            need = torch.maximum(need, old)
                            pages[name][page, :, :slot] = _nearest_code(pages[name][page, :, :slot] * (old / need)[:, None, None])
                        scales[name][page] = need
                        part = _nearest_code(part / need[:, None, None])
                    pages[name][page, :, slot:slot + hi - lo] = part
        at += n
    out = {"q": q_out, "k": pages["k"], "v": pages["v"]}
    if s["k_scales"] is not None:
        out.update(k_scales=scales["k"], v_scales=scales["v"])
    return out

"""Plain float64 definitions of the paged key/value cache: pd_paged_append and pd_paged_attention of include/pd.h, row by
row in numpy, with bounds on the error of one rounding per stored element where a test needs them."""
import numpy as np

MIN_SCALE = 2.0 ** -60


def positions(row_starts, lens, n_rows):
    """(sequence, position) of every row, (-1, -1) where it has none."""
    out = [(-1, -1)] * n_rows
    for b in range(len(lens)):
        s, e = int(row_starts[b]), int(row_starts[b + 1])
        for r in range(s, e):
            p = int(lens[b]) - (e - s) + r - s
            if p >= 0:
                out[r] = (b, p)
    return out


def rotate(x, pos, base):
    """x [..., hd] at position pos; base 0: unchanged."""
    x = np.asarray(x, np.float64)
    if base == 0:
        return x
    half = x.shape[-1] // 2
    a = pos * np.power(float(base), -2.0 * np.arange(half) / x.shape[-1])
    c, s = np.cos(a), np.sin(a)
    lo, hi = x[..., :half], x[..., half:]
    return np.concatenate([lo * c - hi * s, lo * s + hi * c], -1)


def nearest_code(x):
    """Value of the E4M3 code nearest to x: ties to the even mantissa, saturating at 448, NaN stays NaN."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore"):
        c = np.clip(x, -448.0, 448.0)
        _, e = np.frexp(c)
        step = np.ldexp(1.0, np.maximum(e, -5) - 4)
        return np.where(np.isnan(x), np.nan, np.clip(np.round(c / step) * step, -448.0, 448.0))


def scale_for(values):
    """Smallest power of two s >= 2^-60 with every finite magnitude of values <= 448 s."""
    v = np.abs(np.asarray(values, np.float64))
    v = v[np.isfinite(v)]
    s = MIN_SCALE
    while v.size and v.max() > 448.0 * s:
        s *= 2.0
    return s


def append(k_pages, v_pages, k_scales, v_scales, row_starts, lens, table, k, v, base):
    """New (k_pages, v_pages, k_scales, v_scales) as float64: values, or the codes' values beside scales (None: plain pages, not
    rounded).  Pages are [n_pages, Hkv, ps, hd]."""
    kp, vp = np.array(k_pages, np.float64), np.array(v_pages, np.float64)
    ks = None if k_scales is None else np.array(k_scales, np.float64)
    vs = None if v_scales is None else np.array(v_scales, np.float64)
    n_pages, _, ps, _ = kp.shape
    todo = {}                                    # page -> [(slot, row, position)]
    for r, (b, p) in enumerate(positions(row_starts, lens, len(k))):
        if b >= 0:
            page = int(table[b][p // ps])
            if 0 <= page < n_pages:
                todo.setdefault(page, []).append((p % ps, r, p))
    for page, items in todo.items():
        slots = [i[0] for i in items]
        kn = np.stack([rotate(k[r], p, base) for _, r, p in items], 1)            # [Hkv, n, hd]
        vn = np.stack([np.asarray(v[r], np.float64) for _, r, _ in items], 1)
        if ks is None:
            kp[page][:, slots], vp[page][:, slots] = kn, vn
            continue
        first = min(slots)
        for pages, scales, new in ((kp, ks, kn), (vp, vs, vn)):
            for h in range(pages.shape[1]):
                need = scale_for(new[h])
                if first > 0:
                    old = scales[page, h]
                    need = max(need, old)
                    if need > old:
                        pages[page, h, :first] = nearest_code(pages[page, h, :first] * (old / need))
                scales[page, h] = need
                pages[page, h, slots] = nearest_code(new[h] / need)
    return kp, vp, ks, vs


def attend(k_pages, v_pages, k_scales, v_scales, row_starts, lens, table, q, scale):
    """(out, weight, delta): out [n_rows, Hq, hd] (NaN rows where a row has no sequence), weight = sum p |v| / sum p, and delta, the
    largest sum of |scale q_c k_c| over a visible key: what the error bounds of the tests are made of."""
    n_pages, hkv, ps, hd = k_pages.shape
    q = np.asarray(q, np.float64)
    n_rows, hq, _ = q.shape
    out = np.full((n_rows, hq, hd), np.nan)
    weight, delta = np.zeros((n_rows, hq, hd)), np.zeros((n_rows, hq))
    g = hq // hkv
    for b in range(len(lens)):
        s, e, n = int(row_starts[b]), int(row_starts[b + 1]), int(lens[b])
        if e == s:
            continue
        kk, vv = np.zeros((hkv, n, hd)), np.zeros((hkv, n, hd))
        for j0 in range(0, n, ps):
            page, m = int(table[b][j0 // ps]), min(ps, n - j0)
            if 0 <= page < n_pages:
                fk = 1.0 if k_scales is None else np.asarray(k_scales[page], np.float64)[:, None, None]
                fv = 1.0 if v_scales is None else np.asarray(v_scales[page], np.float64)[:, None, None]
                kk[:, j0:j0 + m] = np.asarray(k_pages[page][:, :m], np.float64) * fk
                vv[:, j0:j0 + m] = np.asarray(v_pages[page][:, :m], np.float64) * fv
        for r in range(s, e):
            p = n - (e - s) + r - s
            for h in range(hq):
                if p < 0:
                    out[r, h] = 0.0
                    continue
                x = kk[h // g, :p + 1] @ q[r, h] * scale
                w = np.exp(x - x.max())
                w /= w.sum()
                out[r, h] = w @ vv[h // g, :p + 1]
                weight[r, h] = w @ np.abs(vv[h // g, :p + 1])
                delta[r, h] = (np.abs(kk[h // g, :p + 1]) @ np.abs(q[r, h])).max() * abs(scale)
    return out, weight, delta

"""Plain models of the 8-bit sequence cache for the tests: e4m3 by a table of its values, pages as
arrays on the CPU, appends block by block, attention in fp64.  Nothing here is shared with the
library."""
import math

import numpy as np
import torch

import seq_oracle

NAN_CODE = 0x7f


def _value(code):
    e, m = code >> 3 & 15, code & 7
    if e == 15 and m == 7:
        return math.nan
    return (8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9


VALUES = torch.tensor([(-1 if c & 128 else 1) * _value(c) for c in range(256)], dtype=torch.float64)
_UP = VALUES[:127].numpy()   # 0 .. 448, ascending: code c is value c


def values(codes):
    """uint8 codes as fp64 numbers."""
    return VALUES[codes.long()]


def codes(x):
    """fp64 numbers as uint8 codes: nearest, ties to the even code; what is not finite is NaN."""
    x = x.double().numpy()
    fine = np.isfinite(x)
    a = np.where(fine, np.abs(x), 0.0)
    assert a.max(initial=0.0) <= 448
    hi = np.searchsorted(_UP, a).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    below, above = a - _UP[lo], _UP[hi] - a
    c = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    c = np.where(np.signbit(x), c + 128, c)
    return torch.from_numpy(np.where(fine, c, NAN_CODE).astype(np.uint8))


def same_codes(a, b):
    """Whether two uint8 tensors hold the same codes, NaNs of either sign alike."""
    a, b = a.cpu(), b.cpu()
    nan_a, nan_b = a & 127 == 127, b & 127 == 127
    return bool(((a == b) | (nan_a & nan_b)).all())


def needed(x):
    """The exponent of the scale that values x need."""
    a = x[torch.isfinite(x)].abs()
    most = float(a.max()) if a.numel() else 0.0
    e = -110
    while most > 448 * 2.0 ** e:
        e += 1
    return e


def append(k, v, scales, table, lens, new_k, new_v, starts, S):
    """omnimem_append_kv_quant on CPU tensors: k, v uint8 [P, H, B, d], scales [P, H, 2] fp32, changed in place."""
    P, H, B, _ = k.shape
    N, M = len(table), len(table[0]) if table else 0
    T = new_k.shape[0]
    cap = seq_oracle.capacity(M, S, B) if table else 0
    starts = list(range(N + 1)) if starts is None else [min(max(s, 0), T) for s in starts]
    for i in range(N):
        blocks = {}
        for row in range(starts[i], starts[i + 1]):
            t = lens[i] - (starts[i + 1] - row)
            if 0 <= t < cap:
                b, slot = seq_oracle.place(t, S, B)
                blocks.setdefault(b, []).append((slot, row))
        for b, rows in blocks.items():
            page = table[i][b]
            if not 0 <= page < P:
                continue
            slots, rows = [s for s, _ in rows], [r for _, r in rows]
            begin = min(slots)
            for which, (pool, new) in enumerate(((k, new_k), (v, new_v))):
                x = new[rows].double()                       # [m, H, d]
                for h in range(H):
                    e = needed(x[:, h])
                    if begin > 0:
                        own = float(scales[page, h, which])
                        own = min(own, 2.0 ** 120) if own >= 2.0 ** -110 else 2.0 ** -110
                        e = max(e, math.ceil(math.log2(own)))
                        if own != 2.0 ** e:
                            pool[page, h, :begin] = codes(values(pool[page, h, :begin]) * (own / 2.0 ** e))
                    pool[page, h, slots] = codes(x[:, h] / 2.0 ** e)
                    scales[page, h, which] = 2.0 ** e


def read(k, v, scales, table, lens, tokens, starts, first, S, out_k, out_v):
    """omnimem_read_kv_quant on CPU tensors, into out_k and out_v (fp64)."""
    P, H, B, _ = k.shape
    N, M = len(table), len(table[0])
    cap = seq_oracle.capacity(M, S, B)
    starts = list(range(N + 1)) if starts is None else [min(max(s, 0), tokens) for s in starts]
    for i in range(N):
        for row in range(starts[i], starts[i + 1]):
            t = lens[i] - (starts[i + 1] - row) if first is None else first[i] + row - starts[i]
            out_k[row] = out_v[row] = 0
            if 0 <= t < min(lens[i], cap):
                b, slot = seq_oracle.place(t, S, B)
                page = table[i][b]
                if 0 <= page < P:
                    out_k[row] = values(k[page, :, slot]) * scales[page, :, :1].double()
                    out_v[row] = values(v[page, :, slot]) * scales[page, :, 1:].double()


def decode(q, k_pages, v_pages, scales, table, lens, B, S, window, scale):
    """fp64 outputs and elementwise error bounds of the library's arithmetic: (O, lse, O bound, lse bound).

    The bounds, with u = 2^-24: a score is a sum of d products of a query and a code (fp32 queries: 3 d
    products of its pieces), each sum's step u off, then scaled by a factor of two roundings and
    shifted: at most e = u ((n d + 3) A + 6 |s|max) off, n 1 or 3, A the sum of |q k| scale; the exponential
    adds 2^-22 relative; sums over n keys and their rescales n u for each piece of P, and V's scale
    in P one u more.  bf16: P's first piece is cut below 2^-7 of it, the second rounded by 2^-8 of
    that; the output is 2^-8 off.  fp32: P's pieces hold all of it; the output is u off."""
    N, Hq, d = q.shape
    H = k_pages.shape[1]
    G = Hq // H
    cap = seq_oracle.capacity(table.shape[1], S, B)
    u = 2.0 ** -24
    bf16 = q.dtype == torch.bfloat16
    O = torch.zeros((N, Hq, d), dtype=torch.float64)
    lse = torch.full((Hq, N), -np.inf, dtype=torch.float64)
    ob, lb = torch.zeros_like(O), torch.zeros_like(lse)
    rows = table.tolist()
    used = sorted({p for r in rows for p in r if 0 <= p < k_pages.shape[0]})
    at = {p: n for n, p in enumerate(used)}
    rows = [[at.get(p, -1) for p in r] for r in rows]
    pick = torch.tensor(used, dtype=torch.long, device=k_pages.device)
    sc = scales[pick].cpu().double()
    kd = values(k_pages.view(torch.uint8)[pick].cpu()) * sc[:, :, 0, None, None]
    vd = values(v_pages.view(torch.uint8)[pick].cpu()) * sc[:, :, 1, None, None]
    for i in range(N):
        end = min(max(int(lens[i]), 0), cap)
        begin = max(0, end - window) if window else 0
        k = seq_oracle.tokens_of(kd, rows[i], begin, end, S, B)
        v = seq_oracle.tokens_of(vd, rows[i], begin, end, S, B)
        n = k.shape[0]
        if n == 0:
            continue
        qi = q[i].double().cpu()
        for h in range(Hq):
            s = scale * (k[:, h // G] @ qi[h])
            mag = scale * (k[:, h // G].abs() @ qi[h].abs()).max()
            top = s.max()
            p = torch.exp(s - top)
            total = p.sum()
            lse[h, i] = top + torch.log(total)
            w = (p / total)[:, None]
            O[i, h] = (w * v[:, h // G]).sum(0)
            spread = (w * v[:, h // G].abs()).sum(0)
            e = u * (((1 if bf16 else 3) * d + 3) * mag + 6 * s.abs().max()) + 2.0 ** -22 + (n + 80) * u
            ob[i, h] = spread * (2 * e + (2 * n * u + 2.0 ** -15 if bf16 else 3 * n * u)) + O[i, h].abs() * (2.0 ** -8 if bf16 else u)
            lb[h, i] = e + 4 * u * lse[h, i].abs()
    return O, lse, ob, lb

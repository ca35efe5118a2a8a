"""Plain models of the sequence cache for the tests: tables as Python lists, attention in
fp64 token by token.  Nothing here is shared with the library."""
import numpy as np
import torch


def place(t, S, B):
    """(block, slot) of token t."""
    c, r = divmod(t, S)
    return c * -(-S // B) + r // B, r % B


def blocks(t, S, B):
    return place(t - 1, S, B)[0] + 1 if t > 0 else 0


def capacity(M, S, B):
    bpc = -(-S // B)
    return M // bpc * S + min(M % bpc * B, S)


def update(table, lens, P, B, S, parent, keep, grow):
    """omnimem_seq_update on lists: (rows, lens, copies, info)."""
    N, M = len(table), len(table[0])
    cap = capacity(M, S, B)
    rows, kept, want, tails = [], [], [], []
    for i, p in enumerate(parent):
        have = min(max(lens[p], 0), cap) if 0 <= p < N else 0
        k = have if keep is None else min(max(keep[i], 0), have)
        g = 0 if grow is None else max(grow[i], 0)
        row = [e if 0 <= e < P else -1 for e in table[p][:blocks(k, S, B)]] if k else []
        begun = k > 0 and place(k - 1, S, B)[0] == place(k, S, B)[0]   # the next token goes into a begun block
        kept.append(k)
        want.append(g)
        rows.append(row)
        tails.append(row[-1] if g > 0 and begun else -1)
    users = {}
    for i, row in enumerate(rows):
        for b, page in enumerate(row):
            if page >= 0:
                users.setdefault(page, []).append((i, tails[i] == page and b == len(row) - 1))
    free = [p for p in range(P) if p not in users]
    in_use = len(users)
    over = [k + g > cap for k, g in zip(kept, want)]
    asks = []
    for i in range(len(rows)):
        copy = False
        if tails[i] >= 0 and not over[i]:
            u = users[tails[i]]
            copy = not all(w for _, w in u) or min(j for j, w in u) != i
        more = 0 if over[i] else blocks(kept[i] + want[i], S, B) - blocks(kept[i], S, B)
        asks.append((copy, more))
    need = sum(c + m for c, m in asks)
    short = max(0, need - len(free))
    if short or any(over):
        return [r + [-1] * (M - len(r)) for r in rows], kept, [], [0, in_use, short, sum(over)]
    copies = []
    for i, (copy, more) in enumerate(asks):
        if copy:
            to = free.pop(0)
            copies.append((tails[i], to))
            rows[i][-1] = to
        rows[i] = rows[i] + [free.pop(0) for _ in range(more)]
    lens = [k + g for k, g in zip(kept, want)]
    return [r + [-1] * (M - len(r)) for r in rows], lens, copies, [len(copies), in_use + need, 0, 0]


def compact(table, lens, P, B, S):
    """omnimem_seq_compact on lists: (rows, moves, info)."""
    M = len(table[0]) if table else 0
    cap = capacity(M, S, B) if table else 0
    rows = [[e if 0 <= e < P else -1 for e in r[:blocks(min(max(t, 0), cap), S, B)]] for r, t in zip(table, lens)]
    used = sorted({e for r in rows for e in r if e >= 0})
    gaps = [p for p in range(len(used)) if p not in set(used)]
    moves = list(zip([p for p in used if p >= len(used)], gaps))
    to = dict(moves)
    return [[to.get(e, e) for e in r] + [-1] * (M - len(r)) for r in rows], moves, [len(moves), len(used), 0, 0]


def tokens_of(pool, row, t0, t1, S, B):
    """Tokens [t0, t1) on resident pages of a table row, [n, H, d]."""
    P = pool.shape[0]
    at = [(row[b], s) for b, s in (place(t, S, B) for t in range(t0, t1)) if 0 <= row[b] < P]
    if not at:
        return pool.new_zeros((0, pool.shape[1], pool.shape[3]))
    page, slot = (torch.tensor(x, device=pool.device) for x in zip(*at))
    return pool[page, :, slot]


def decode(q, k_pages, v_pages, table, lens, B, S, window, scale):
    """fp64 outputs and elementwise error bounds of the library's arithmetic: (O, lse, O bound, lse bound).

    The bounds, with u = 2^-24: a score is a sum of d fp32 products, then scaled and shifted:
    at most e = u ((d + 3) A + 4 |s|max) off, A the sum of |q k| scale; the exponential adds 2^-22
    relative; sums of n terms and their rescales n u.  P rounded to bf16 is 2^-8 off, and so is
    a bf16 output (fp32: u)."""
    N, Hq, d = q.shape
    H = k_pages.shape[1]
    G = Hq // H
    cap = capacity(table.shape[1], S, B)
    u = 2.0 ** -24
    bf16 = q.dtype == torch.bfloat16
    O = torch.zeros((N, Hq, d), dtype=torch.float64)
    lse = torch.full((Hq, N), -np.inf, dtype=torch.float64)
    ob, lb = torch.zeros_like(O), torch.zeros_like(lse)
    rows = table.tolist()
    for i in range(N):
        end = min(max(int(lens[i]), 0), cap)
        begin = max(0, end - window) if window else 0
        k = tokens_of(k_pages, rows[i], begin, end, S, B).double().cpu()
        v = tokens_of(v_pages, rows[i], begin, end, S, B).double().cpu()
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
            e = u * ((d + 3) * mag + 4 * s.abs().max()) + 2.0 ** -22 + (n + 80) * u
            ob[i, h] = spread * (2 * e + (2.0 ** -8 if bf16 else 0.0)) + O[i, h].abs() * (2.0 ** -8 if bf16 else u)
            lb[h, i] = e + 4 * u * lse[h, i].abs()
    return O, lse, ob, lb

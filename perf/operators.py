"""The operators of the sequence cache, as they are measured: attention of one new token per
sequence over paged keys and values, the appending of new tokens' keys and values, and the
copying, forking, freeing and compacting of pages.

A case names one operator and its sizes.  `listed` holds the fixed ones, `draw` makes more of
the same ranges, `prepare` builds what a program that generates many sequences has in hand
before the call, `run` makes one pass (the plain form in elementary torch operations, or the
library's entry points where `own` is true), and `exact` computes the same outputs in 64 bits.

A page holds one block of B tokens for every key/value head, [num_pages][H][B][d]; sequence i
has a row of the page table [N][M] and a length.  Its tokens come in chunks of S: token t lies
in block (t div S) * ceil(S / B) + (t mod S) div B, slot (t mod S) mod B, so that S = B is a
contiguous sequence and S = 4,680 a history of video chunks.
"""
import math

import torch

own = False
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
DEV = "cuda"

# op: decode = one query token per sequence; append = new tokens' K and V into the pages;
# copy = pages by a list of (source, target); update = the new table of a step that forks,
# frees, shortens and lengthens sequences; compact = the table and moves that bring the pages
# in use to the front of the pool.
# N = sequences, Hq / H = query heads / key-value heads, d = head size, B = tokens of a page,
# S = tokens of a chunk, lo..hi = the shortest and longest sequence, window = only the last so
# many tokens (0: all), n = new tokens of a sequence (append: 0 = ragged, 1..hi; update: the
# longest prompt of a newly admitted sequence), layers and pairs = of a copy, extra = pool
# pages to a page in use.


def _case(name, op, dtype="bf16", N=1, Hq=12, H=12, d=128, B=64, S=64, lo=64, hi=64, window=0, n=1, layers=1, pairs=0,
          extra=1.1):
    c = {"op": op, "dtype": dtype, "N": N, "Hq": Hq, "H": H, "d": d, "B": B, "S": S, "lo": lo, "hi": hi, "window": window,
         "n": n, "layers": layers, "pairs": pairs, "extra": extra}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the smallest call: one short sequence of a two-head fp32 layer, all launch latency
        _case("decode_tiny_fp32", "decode", "fp32", N=1, Hq=2, H=2, d=64, lo=300, hi=300),
        # four rollouts of a 1.3B-shaped layer, 10 to 20 cached chunks each: the largest stream
        _case("decode_1.3b_chunks", "decode", N=4, S=4680, lo=46800, hi=93600),
        # a serving batch: 40 query heads over 8 key-value heads, lengths over two decades
        _case("decode_gqa_ragged", "decode", N=48, Hq=40, H=8, lo=100, hi=16000),
        # reference precision, small heads, eight query heads a key head, the last frame only
        _case("decode_fp32_window", "decode", "fp32", N=16, Hq=16, H=2, d=64, B=128, S=128, lo=1000, hi=6000, window=1560),
        # one new token for each sequence of a batch, between two decoding steps
        _case("append_token", "append", N=64, lo=100, hi=16000, n=1),
        # the chunk just generated, for eight rollouts of a 1.3B-shaped layer
        _case("append_chunk", "append", N=8, S=4680, lo=4680, hi=46800, n=4680),
        # the private copies that sixteen forked sequences need before they append
        _case("copy_fork", "copy", N=16, lo=64, hi=64, pairs=16, extra=4.0),
        # the moves of a compaction, six layers of a 1.3B-shaped model at once
        _case("copy_moves", "copy", layers=6, pairs=300, extra=2.0),
        # a beam search's step: sixteen rows of a thousand tokens choose their parents
        _case("update_beams", "update", N=16, lo=900, hi=1100, n=0, extra=1.5),
        # a serving batch's step: rows end, fork, start with a prompt, or get one more token
        _case("update_serving", "update", N=256, lo=100, hi=30000, n=4000, extra=1.5),
        # a small pool, a third of it in use
        _case("compact_small", "compact", N=16, lo=900, hi=1100, extra=3.0),
        # a large pool after many sequences have ended
        _case("compact_pool", "compact", N=256, lo=100, hi=30000, extra=1.7),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["decode", "decode", "decode", "append", "append", "copy", "update", "compact"])
        H = rng.choice([1, 2, 3, 4, 8, 8, 12, 12, 16, 40])
        B = rng.choice([64, 64, 128])
        S = rng.choice([B, B, B, 4680, 1560, log(B, 5000)])
        hi = log(30, 100000)
        lo = min(hi, log(1, hi))
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        d = rng.choice([64, 128, 128])
        if op == "decode":
            c = _case(None, op, dtype, N=log(1, 128), Hq=H * rng.choice([1, 1, 2, 4, 5, 7, 8, 16, 24]), H=H, d=d, B=B, S=S, lo=lo,
                      hi=hi, window=rng.choice([0, 0, 0, log(1, hi)]))
        elif op == "append":
            c = _case(None, op, dtype, N=log(1, 128), H=H, d=d, B=B, S=S, lo=lo, hi=hi, n=rng.choice([1, 0, 0, log(1, lo)]))
        elif op == "copy":
            c = _case(None, op, dtype, H=H, d=d, B=B, layers=rng.choice([1, 1, 2, 5]), pairs=log(1, 1000),
                      extra=rng.choice([2.0, 3.0, 4.0]))
        else:
            c = _case(None, op, N=log(1, 256), B=B, S=S, lo=lo, hi=hi, n=rng.choice([0, log(1, 4000)]) if op == "update" else 1,
                      extra=rng.choice([1.2, 1.7, 3.0]))
        pool = _pool_pages(c) * c["layers"] * c["H"] * B * d * (2 if dtype == "bf16" else 4) * 2
        f = work(c)
        if c["op"] in ("update", "compact") and c["N"] * _max_blocks(c) > 130000:
            continue
        if c["op"] in ("decode", "append", "copy") and (pool > 6e9 or f["bytes"] > 1.5e9 or c["N"] * _max_blocks(c) * H * B * d > 8e8):
            continue
        return c


# ------------------------------------------------------------------------- sizes


def _bpc(case):
    return -(-case["S"] // case["B"])


def _blocks(case, t):
    """Blocks of a sequence of t tokens (a number or a tensor)."""
    S, B = case["S"], case["B"]
    return t // S * _bpc(case) + (t % S + B - 1) // B


def _lens(case):
    """The N lengths in ascending order, evenly spaced on a logarithmic scale."""
    lo, hi, N = case["lo"], case["hi"], case["N"]
    return [int(round(lo * (hi / lo) ** ((i + 0.5) / N))) for i in range(N)]


def _max_blocks(case):
    return _blocks(case, case["hi"] + max(case["n"], 1)) + 1


def _pool_pages(case):
    if case["op"] == "copy":
        return max(2, int(case["pairs"] * case["extra"]))
    used = sum(_blocks(case, t) for t in _lens(case))
    if case["op"] == "update":
        used += case["N"] * 2 + case["N"] // 8 * _blocks(case, max(case["n"], 1))
    return max(2, int(used * case["extra"]))


def work(case):
    eb = 2 if case["dtype"] == "bf16" else 4
    N, H, d, Hq = case["N"], case["H"], case["d"], case["Hq"]
    lens, M = _lens(case), _max_blocks(case)
    if case["op"] == "decode":
        read = sum(min(t, case["window"] or t) for t in lens)
        return {"bytes": 2 * read * H * d * eb + 2 * N * Hq * d * eb + 4 * N * Hq + 4 * sum(_blocks(case, t) for t in lens),
                "flops": 4 * read * Hq * d}
    if case["op"] == "append":
        new = sum(_news(case))
        return {"bytes": 4 * new * H * d * eb, "flops": 0}
    if case["op"] == "copy":
        return {"bytes": 4 * case["layers"] * case["pairs"] * H * case["B"] * d * eb, "flops": 0}
    entries = sum(_blocks(case, t) for t in lens)
    if case["op"] == "update":
        return {"bytes": 4 * (entries + N * M + 8 * N), "flops": 0}
    return {"bytes": 4 * (entries + N * M + N + _pool_pages(case) // 2 * 2), "flops": 0}


def _news(case):
    """New tokens of each sequence of an append, of the lengths in ascending order."""
    lens = _lens(case)
    return [min(case["n"], t) if case["n"] else 1 + (t * 7919) % t for t in lens]


# ------------------------------------------------------------------------- inputs


class _State:
    pass


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    st = _State()
    st.case = case
    N, H, d, B, M, P = case["N"], case["H"], case["d"], case["B"], _max_blocks(case), _pool_pages(case)
    dt = DTYPES[case["dtype"]]

    def randint(hi, shape):
        return torch.randint(0, max(int(hi), 1), shape, generator=g, device=DEV)

    if case["op"] == "copy":
        shape = (case["layers"], P, H, B, d)
        st.k = torch.randn(shape, generator=g, device=DEV, dtype=dt)
        st.v = torch.randn(shape, generator=g, device=DEV, dtype=dt)
        ids = torch.randperm(P, generator=g, device=DEV)
        n = case["pairs"]
        targets, sources = ids[:n], ids[n:]
        # forked sequences share a source now and then; a target is written once
        st.pairs = torch.stack([sources[randint(sources.numel(), (n,))], targets], 1).int().contiguous()
        st.count = torch.full((4,), n, dtype=torch.int32, device=DEV)
        return st

    order = torch.randperm(N, generator=g, device=DEV)
    lens = torch.tensor(_lens(case), device=DEV)[order]
    nb = _blocks(case, lens)
    col = torch.arange(M, device=DEV)
    here = col[None] < nb[:, None]
    ids = torch.randperm(P, generator=g, device=DEV)
    at = torch.cumsum(here.flatten().int(), 0).view(N, M) - 1
    st.table = torch.where(here, ids[at.clamp(0, P - 1)], -1).int().contiguous()
    st.lens = lens.int()
    st.P = P
    if case["op"] in ("update", "compact"):
        # half of the rows go back to a common prompt: they share its full blocks with the row before
        if N > 1:
            share = torch.arange(N, device=DEV) % 2 == 1
            prev = torch.arange(N, device=DEV) - share.long()
            common = torch.minimum(lens, lens[prev]) // 2 // case["S"] * _bpc(case)
            st.table = torch.where(share[:, None] & (col[None] < common[:, None]), st.table[prev], st.table).contiguous()
        if case["op"] == "update":
            rows = torch.arange(N, device=DEV)
            kind = torch.rand(N, generator=g, device=DEV)
            parent = torch.where(kind < 0.3, randint(N, (N,)), rows)     # forks, beside the rows that go on
            if case["n"] == 0:
                parent = randint(N, (N,))                                  # a beam search: every row chooses
            fresh = (rows % 8 == 7) & (case["n"] > 0)                      # ended rows, whose place a prompt takes
            st.parent = torch.where(fresh, -1, parent).int().contiguous()
            st.keep = torch.where(kind < 0.1, lens[parent] - randint(B, (N,)), lens[parent]).clamp(min=0).int().contiguous()
            st.grow = torch.where(fresh, 1 + randint(case["n"], (N,)), 1).int().contiguous()
        return st

    st.k = torch.randn((P, H, B, d), generator=g, device=DEV, dtype=dt)
    st.v = torch.randn((P, H, B, d), generator=g, device=DEV, dtype=dt)
    if case["op"] == "append":
        new = torch.tensor(_news(case), device=DEV)[order]
        st.starts = torch.cat([new.new_zeros(1), torch.cumsum(new, 0)]).int()
        T = sum(_news(case))
        # K and V as a fused projection leaves them: rows of [3, H, d], Q first
        qkv = torch.randn((T, 3, H, d), generator=g, device=DEV, dtype=dt)
        st.new_k, st.new_v = qkv[:, 1], qkv[:, 2]
        if case["n"] == 1:
            st.starts = None
        return st
    # a query looks for one of its sequence's tokens, which its score then lifts over the others
    G = case["Hq"] // H
    t = (torch.rand(N, generator=g, device=DEV) * lens).long()
    S = case["S"]
    page = st.table[torch.arange(N, device=DEV), t // S * _bpc(case) + t % S // B].long()
    seek = st.k[page, :, t % S % B].float().repeat_interleave(G, 1)
    st.q = (torch.randn((N, case["Hq"], d), generator=g, device=DEV) + 0.6 * seek).to(dt)
    return st


# ------------------------------------------------------------------------- one pass


def run(st):
    case = st.case
    if own:
        return _own(st)
    return {"decode": _plain_decode, "append": _plain_append, "copy": _plain_copy, "update": _plain_update,
            "compact": _plain_compact}[case["op"]](st)


def _own(st):
    from paper_2605_30519_amd import (SeqKVCache, omnimem_append_kv, omnimem_copy_pages, omnimem_decode_attn,
                                      omnimem_seq_compact, omnimem_seq_update)
    case = st.case
    if case["op"] == "copy":
        omnimem_copy_pages(st.k, st.v, st.pairs, st.count)
        return st.k, st.v
    if case["op"] == "update":
        u = omnimem_seq_update(st.table, st.lens, st.P, case["B"], st.parent, st.keep, st.grow, chunk_tokens=case["S"])
        return u.page_table, u.seq_lens, u.copies, u.info
    if case["op"] == "compact":
        u = omnimem_seq_compact(st.table, st.lens, st.P, case["B"], chunk_tokens=case["S"])
        return u.page_table, u.copies, u.info
    cache = SeqKVCache(st.k, st.v, st.table, st.lens, case["S"])
    if case["op"] == "append":
        omnimem_append_kv(cache, st.new_k, st.new_v, st.starts)
        return st.k, st.v
    return omnimem_decode_attn(cache, st.q, window=case["window"])


def _tokens(case, M):
    """Token number of every slot of a row's M blocks [M * B], and whether the slot is one."""
    S, B = case["S"], case["B"]
    at = torch.arange(M * B, device=DEV)
    block, slot = at // B, at % B
    inside = block % _bpc(case) * B + slot
    return block // _bpc(case) * S + inside, inside < S


def _plain_decode(st):
    case = st.case
    N, Hq, d = st.q.shape
    P, H, B, _ = st.k.shape
    M = st.table.shape[1]
    tok, real = _tokens(case, M)
    last = st.lens.long()[:, None]
    ok = real & (tok < last)
    if case["window"]:
        ok = ok & (tok >= last - case["window"])
    ok = ok & ((st.table >= 0) & (st.table < P)).repeat_interleave(B, 1)
    pages = st.table.long().clamp(0, P - 1)
    ok4 = ok[:, None, :, None]
    k = st.k[pages].transpose(1, 2).reshape(N, H, M * B, d).float()
    v = st.v[pages].transpose(1, 2).reshape(N, H, M * B, d).float().masked_fill(~ok4, 0.0)
    q = st.q.float().view(N, H, Hq // H, d)
    s = torch.matmul(k, q.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
    s = s.masked_fill(~ok4, -math.inf)
    top = s.amax(2, keepdim=True)
    p = torch.exp(s - top.clamp(min=-3e38))
    total = p.sum(2, keepdim=True)
    o = torch.matmul(p.transpose(2, 3).contiguous(), v) / total.transpose(2, 3).clamp(min=1e-30)
    lse = (top + torch.log(total)).view(N, Hq)
    return o.view(N, Hq, d).to(st.q.dtype), lse.t().contiguous()


def _plain_append(st):
    case = st.case
    P, H, B, d = st.k.shape
    S, T = case["S"], st.new_k.shape[0]
    N, M = st.table.shape
    starts = torch.arange(N + 1, device=DEV) if st.starts is None else st.starts.long()
    row = torch.arange(T, device=DEV)
    seq = torch.searchsorted(starts, row, right=True) - 1
    t = st.lens.long()[seq] - starts[seq + 1] + row
    t0 = t.clamp(min=0)
    block = t0 // S * _bpc(case) + t0 % S // B
    page = st.table[seq, block.clamp(max=M - 1)].long()
    put = (t >= 0) & (block < M) & (page >= 0) & (page < P)
    page, slot = page[put], (t0 % S % B)[put]
    st.k[page, :, slot] = st.new_k[put]
    st.v[page, :, slot] = st.new_v[put]
    return st.k, st.v


def _plain_copy(st):
    P = st.k.shape[1]
    src, dst = st.pairs.long().unbind(1)
    take = (torch.arange(src.numel(), device=DEV) < st.count[0]) & (src >= 0) & (src < P) & (dst >= 0) & (dst < P)
    src, dst = src[take], dst[take]
    st.k[:, dst] = st.k[:, src]
    st.v[:, dst] = st.v[:, src]
    return st.k, st.v


def _capacity(case, M):
    return M // _bpc(case) * case["S"] + min(M % _bpc(case) * case["B"], case["S"])


def _plain_update(st):
    case, P = st.case, st.P
    S, B = case["S"], case["B"]
    N, M = st.table.shape
    R = st.parent.numel()
    cap = _capacity(case, M)
    rows, col = torch.arange(R, device=DEV), torch.arange(M, device=DEV)
    parent = st.parent.long()
    known = (parent >= 0) & (parent < N)
    parent = parent.clamp(0, N - 1)
    have = torch.where(known, st.lens.long()[parent].clamp(0, cap), 0)
    keep = torch.minimum(st.keep.long().clamp(min=0), have)
    grow = st.grow.long().clamp(min=0)
    nk, over = _blocks(case, keep), keep + grow > cap
    nt = torch.where(over, nk, _blocks(case, keep + grow))
    old = st.table.long()[parent]
    old = torch.where((col < nk[:, None]) & (old >= 0) & (old < P), old, -1)
    tail = (nk - 1).clamp(min=0)
    tail_page = old[rows, tail]
    writes = (grow > 0) & (keep % S % B != 0) & (tail_page >= 0)
    mine = writes[:, None] & (col == tail[:, None])
    held = torch.zeros(P + 1, dtype=torch.bool, device=DEV)
    held[torch.where(mine | (old < 0), P, old).flatten()] = True
    first = torch.full((P + 1,), R, device=DEV)
    first.scatter_reduce_(0, torch.where(writes, tail_page, P), rows, "amin")
    copy = writes & (held[tail_page] | (first[tail_page] != rows)) & ~over
    used = (held | (first < R))[:P]
    want = copy.long() + nt - nk
    need, room = want.sum(), P - used.sum()
    short = (need - room).clamp(min=0)
    done = (short == 0) & ~over.any()
    free = ~used
    spare = torch.full((P + 1,), -1, device=DEV)
    spare[torch.where(free, torch.cumsum(free, 0) - 1, P)] = torch.arange(P, device=DEV)
    off = torch.cumsum(want, 0) - want
    at = off[:, None] + torch.where(col >= nk[:, None], copy.long()[:, None] + col - nk[:, None], 0)
    fresh = (mine & copy[:, None]) | ((col >= nk[:, None]) & (col < nt[:, None]))
    table = torch.where(fresh & done, spare[at.clamp(0, P)], old).int()
    copy = copy & done
    pairs = torch.full((R + 1, 2), -1, dtype=torch.int32, device=DEV)
    pairs[torch.where(copy, torch.cumsum(copy, 0) - 1, R)] = torch.stack([tail_page, table[rows, tail].long()], 1).int()
    info = torch.stack([copy.sum(), used.sum() + torch.where(done, need, 0), short, over.sum()]).int()
    lens = torch.where(done, keep + grow, keep).int()
    pairs[R] = -1
    return table, lens, torch.where(rows[:, None] < info[0], pairs[:R], -1), info


def _plain_compact(st):
    case, P = st.case, st.P
    N, M = st.table.shape
    col = torch.arange(M, device=DEV)
    nb = _blocks(case, st.lens.long().clamp(0, _capacity(case, M)))
    old = st.table.long()
    old = torch.where((col < nb[:, None]) & (old >= 0) & (old < P), old, -1)
    used = torch.zeros(P + 1, dtype=torch.bool, device=DEV)
    used[torch.where(old < 0, P, old).flatten()] = True
    used = used[:P]
    ids, U = torch.arange(P, device=DEV), used.sum()
    moves, gaps = used & (ids >= U), ~used & (ids < U)
    half = max(1, P // 2)
    pairs = torch.full((half + 1, 2), -1, device=DEV)
    pairs[torch.where(moves, torch.cumsum(moves, 0) - 1, half), 0] = ids
    pairs[torch.where(gaps, torch.cumsum(gaps, 0) - 1, half), 1] = ids
    pairs[half] = -1
    target = torch.where(moves, pairs[(torch.cumsum(moves, 0) - 1).clamp(0, half), 1], ids)
    table = torch.where(old >= 0, target[old.clamp(min=0)], -1).int()
    info = torch.stack([moves.sum(), U, torch.zeros_like(U), torch.zeros_like(U)]).int()
    return table, pairs[:half].int(), info


# ------------------------------------------------------------------------- in 64 bits


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "decode":
        return _exact_decode(st)
    if op == "append":
        return _exact_append(st)
    if op == "copy":
        n, P = int(st.count[0]), st.k.shape[1]
        k, v = st.k.double(), st.v.double()
        for s, t in st.pairs[:n].tolist():
            if 0 <= s < P and 0 <= t < P:
                k[:, t], v[:, t] = st.k[:, s].double(), st.v[:, s].double()
        return k, v
    return None   # page numbers and counts: no value in 64 bits


def _exact_decode(st):
    """Sequence by sequence: its tokens' rows gathered one chunk after another, a two-pass softmax."""
    case = st.case
    N, Hq, d = st.q.shape
    P, H, B, _ = st.k.shape
    S, bpc = case["S"], _bpc(case)
    out = torch.zeros((N, Hq, d), dtype=torch.float64, device=DEV)
    lse = torch.full((Hq, N), -math.inf, dtype=torch.float64, device=DEV)
    for i, t in enumerate(st.lens.tolist()):
        keys, values = [], []
        for c in range(-(-t // S)):
            size = min(S, t - c * S)
            pages = st.table[i, c * bpc:c * bpc + -(-size // B)].long()
            keys.append(st.k[pages].permute(0, 2, 1, 3).reshape(-1, H, d)[:size])
            values.append(st.v[pages].permute(0, 2, 1, 3).reshape(-1, H, d)[:size])
        if not keys:
            continue
        k, v = torch.cat(keys), torch.cat(values)
        if case["window"]:
            k, v = k[-case["window"]:], v[-case["window"]:]
        for h in range(H):
            heads = slice(h * (Hq // H), (h + 1) * (Hq // H))
            s = k[:, h].double() @ st.q[i, heads].double().t().contiguous() / math.sqrt(d)
            lse[heads, i] = torch.logsumexp(s, 0)
            out[i, heads] = torch.softmax(s, 0).t().contiguous() @ v[:, h].double()
    return out, lse


def _exact_append(st):
    case = st.case
    P, H, B, d = st.k.shape
    k, v = st.k.double(), st.v.double()
    starts = list(range(case["N"] + 1)) if st.starts is None else st.starts.tolist()
    for i, t in enumerate(st.lens.tolist()):
        n = starts[i + 1] - starts[i]
        at = t - n
        while at < t:   # one block after another
            c, inside = divmod(at, case["S"])
            slot = inside % B
            m = min(B - slot, case["S"] - inside, t - at)
            page = int(st.table[i, c * _bpc(case) + inside // B])
            row = starts[i] + at - (t - n)
            k[page, :, slot:slot + m] = st.new_k[row:row + m].double().transpose(0, 1)
            v[page, :, slot:slot + m] = st.new_v[row:row + m].double().transpose(0, 1)
            at += m
    return k, v

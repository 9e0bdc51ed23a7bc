"""Attention with a sliding window and first tokens that stay visible, and the operators on the blocks
of the cache that a program with such a window (or with several samples of one prompt) needs beside it.

A case is one pass of one path, over the paged cache of ``include/coopt_attn.h`` (tiles in matrix-core
operand order, E4M3 / E5M2 codes with a scale per token and head, or fp16).  The sizes are the repository's
(40 query heads of 128 dims over 8 or 40 KV heads; 64 dims in the small ones) and generic ones around them.

Operations (`op`):
  decode   one new token per sequence attends to its last `window` tokens and the first `sinks`
  prefill  a chunk of new rows per sequence, every row with its own window
  fork     sequences that go on from another's tokens: full blocks shared, the last one copied, all layers
  compact  finished sequences freed, the blocks in use moved to the front of the pool, all layers
  roll     one step's bookkeeping: finished sequences freed, blocks behind the window freed, blocks and
           slots for the new tokens of every sequence

Blocks behind the window are no longer in the pool in the decode cases (their table entries are -1), as
in a program that frees them; in the prefill cases they still are.  The block operators work on tables,
lengths, reference counts and the map of free blocks; a pass begins by setting these back to where it starts
(they are one buffer), so that every pass does the same work.
"""
import math

import torch

own = False

BLOCK = 16
_CODE = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_MAX = {"e4m3": 448.0, "e5m2": 57344.0}


def _coopt():
    import paper_2602_09323_amd
    return paper_2602_09323_amd


def _attention(name, op, cache, seqs, q_heads, kv_heads, dim, window, sinks, ctx_lo, ctx_hi, chunk_lo=0, chunk_hi=0):
    """ctx_*: tokens in front of the new ones; chunk_*: new rows of a prefill."""
    return dict(name=name, op=op, cache=cache, seqs=seqs, q_heads=q_heads, kv_heads=kv_heads, dim=dim, window=window,
                sinks=sinks, ctx_lo=ctx_lo, ctx_hi=ctx_hi, chunk_lo=chunk_lo, chunk_hi=chunk_hi)


def _blocks(name, op, cache, seqs, kv_heads, dim, layers, ctx_lo, ctx_hi, samples=0, window=0, sinks=0, chunk=1):
    return dict(name=name, op=op, cache=cache, seqs=seqs, kv_heads=kv_heads, dim=dim, layers=layers, ctx_lo=ctx_lo,
                ctx_hi=ctx_hi, samples=samples, window=window, sinks=sinks, chunk=chunk)


def listed():
    return [
        # one user of a small window: launches and memory round trips count
        _attention("decode_one", "decode", "e4m3", 1, 40, 8, 128, 512, 4, 1500, 1500),
        # a small model's batch, sequences shorter and longer than an odd window, the shortest with one token
        _attention("decode_odd", "decode", "e5m2", 13, 32, 8, 64, 1021, 13, 0, 9000),
        # a full serving batch far beyond the window
        _attention("decode_batch", "decode", "e4m3", 64, 40, 8, 128, 4096, 4, 600, 32000),
        # the last chunk of one prompt
        _attention("prefill_tail", "prefill", "e4m3", 1, 40, 8, 128, 1024, 4, 3000, 3000, 77, 77),
        # fresh prompts of different lengths over an uncompressed cache
        _attention("prefill_ragged", "prefill", "fp16", 5, 32, 8, 64, 500, 7, 0, 0, 100, 1777),
        # large chunks of long prompts, where the products count
        _attention("prefill_long", "prefill", "e4m3", 4, 40, 8, 128, 4096, 4, 8192, 8192, 2048, 2048),
        # eight samples of one prompt
        _blocks("fork_samples", "fork", "e4m3", 1, 8, 128, 40, 700, 700, samples=8),
        # four beams of each of a batch's sequences
        _blocks("fork_beams", "fork", "fp16", 32, 8, 128, 40, 100, 4000, samples=4),
        # a small pool with every second sequence gone
        _blocks("compact_small", "compact", "e5m2", 24, 2, 64, 4, 1, 900),
        # a large one
        _blocks("compact_large", "compact", "e4m3", 128, 8, 128, 16, 500, 3500),
        # a step of a small batch: one token each
        _blocks("roll_decode", "roll", "e4m3", 16, 8, 128, 1, 40, 3000, window=512, sinks=4),
        # a step of a large batch in which every eighth sequence brings a chunk of its prompt
        _blocks("roll_mixed", "roll", "e4m3", 1024, 8, 128, 1, 600, 32000, window=4096, sinks=4, chunk=512),
    ]


def _spread(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99)))))))


def draw(rng):
    op = rng.choice(["decode", "decode", "prefill", "prefill", "fork", "compact", "roll"])
    cache = rng.choice(["e4m3", "e4m3", "e5m2", "fp16"])
    dim = rng.choice([64, 128])
    kv = rng.choice([1, 2, 4, 8, 16, 40])
    if op in ("decode", "prefill"):
        heads = kv * rng.choice([g for g in (1, 2, 4, 5, 8, 16) if kv * g <= 40] or [1])
        window = _spread(rng, 16, 4096)
        sinks = rng.choice([0, 1, 4, rng.randint(0, 64)])
        seqs = _spread(rng, 1, 64 if op == "decode" else 8)
        ctx = sorted(rng.choice([0, 1]) + _spread(rng, 1, 32000 if op == "decode" else 8192) for _ in range(2))
        chunk = sorted(_spread(rng, 1, 2048) for _ in range(2)) if op == "prefill" else [0, 0]
        c = _attention("", op, cache, seqs, heads, kv, dim, window, sinks, ctx[0], ctx[1], *chunk)
        most = next(x for x in listed() if x["name"] == ("decode_batch" if op == "decode" else "prefill_long"))
        unit = "bytes" if op == "decode" else "flops"
        while work(c)[unit] > work(most)[unit]:
            c["seqs"] = (c["seqs"] + 1) // 2
            c["window"] = (c["window"] + 1) // 2
    else:
        kv = min(kv, 16)
        ctx = sorted(_spread(rng, 1, 4000 if op != "roll" else 32000) for _ in range(2))
        seqs = _spread(rng, *{"fork": (1, 32), "compact": (2, 128), "roll": (1, 1024)}[op])
        c = _blocks("", op, cache, seqs, kv, dim, 1 if op == "roll" else _spread(rng, 1, 16), ctx[0], ctx[1],
                    samples=rng.randint(1, 8) if op == "fork" else 0, window=_spread(rng, 16, 4096) if op == "roll" else 0,
                    sinks=rng.choice([0, 4, rng.randint(0, 64)]) if op == "roll" else 0,
                    chunk=_spread(rng, 1, 512) if op == "roll" else 1)
        most = next(x for x in listed() if x["name"] == {"fork": "fork_beams", "compact": "compact_large", "roll": "roll_mixed"}[op])
        while work(c)["bytes"] > work(most)["bytes"] or _pool_bytes(c) > _pool_bytes(most):
            c["seqs"], c["layers"] = max((c["seqs"] + 1) // 2, 2 if op == "compact" else 1), (c["layers"] + 1) // 2
    del c["name"]
    return c


# ---- lengths and pages: plain whole numbers, the same on both sides

def _even(lo, hi, n):
    return [lo + (hi - lo) * i // max(n - 1, 1) for i in range(n)]


def _ceil(n, by):
    return -(-n // by)


def _lengths(case):
    """(tokens in front, new rows) of every sequence, in the order of their lengths."""
    before = _even(case["ctx_lo"], case["ctx_hi"], case["seqs"])
    new = [1] * case["seqs"] if case["op"] == "decode" else _even(case["chunk_lo"], case["chunk_hi"], case["seqs"])
    return list(zip(before, new))


def _row_bytes(case):
    return 4 * case["dim"] if case["cache"] == "fp16" else 2 * case["dim"] + 8          # K and V of a token and head


def _visible(t, window, sinks):
    """Tokens that the last of t sees."""
    return min(t, window) + min(sinks, max(t - window, 0))


def _block_case(case):
    """Lengths, what is finished, and which entries of a row are no longer held, of a case on blocks."""
    S, op = case["seqs"], case["op"]
    lens = _even(case["ctx_lo"], case["ctx_hi"], S)
    rows = S * (1 + case["samples"])
    gone = list(range(1, S, 2)) if op == "compact" else list(range(7, S, 64)) if op == "roll" else []
    return lens, rows, gone


def _new_tokens(case):
    """New tokens of every sequence of a roll; a finished one has none."""
    return [0 if i % 64 == 7 else case["chunk"] if i % 8 == 3 else 1 for i in range(case["seqs"])]


def _pool_blocks(case):
    lens, rows, _ = _block_case(case)
    held = sum(_ceil(t, BLOCK) for t in lens)
    if case["op"] == "roll":
        held = sum(_ceil(min(t, case["window"] + case["sinks"] + case["chunk"] + 3 * BLOCK), BLOCK) for t in lens)
        held += sum(_ceil(n, BLOCK) + 1 for n in _new_tokens(case))
    return held + held // 8 + rows + 33


def _pool_bytes(case):
    return _pool_blocks(case) * BLOCK * case["kv_heads"] * _row_bytes(case) * case["layers"] if case["op"] != "roll" else 0


def work(case):
    op = case["op"]
    if op in ("decode", "prefill"):
        heads, kv, d, w, s = (case[k] for k in ("q_heads", "kv_heads", "dim", "window", "sinks"))
        read = pairs = rows = tables = 0
        for before, new in _lengths(case):
            t = before + new
            first = max(before + 1 - w, 0)                              # of the first new row's window
            tokens = t - first + min(s, first)
            read += tokens * kv * _row_bytes(case)
            tables += _ceil(tokens, BLOCK) * 4 + 8
            rows += new
            pairs += sum(_visible(before + 1 + i, w, s) for i in range(new))
        return {"bytes": read + tables + 2 * rows * heads * d * 2, "flops": 4 * pairs * heads * d}
    lens, _, gone = _block_case(case)
    block = BLOCK * case["kv_heads"] * _row_bytes(case) * case["layers"]
    if op == "fork":
        partial = sum(1 for t in lens if t % BLOCK) * case["samples"]
        full = sum(t // BLOCK for t in lens) * case["samples"]
        return {"bytes": 2 * partial * block + full * 12 + (len(lens) + 2) * case["samples"] * 8, "flops": 0}
    if op == "compact":
        kept = [_ceil(t, BLOCK) for i, t in enumerate(lens) if i not in set(gone)]
        freed = sum(_ceil(t, BLOCK) for t in lens) - sum(kept)
        # (blocks lie anywhere in the pool: of those in use, the share that lies behind the front moves)
        moved = int(sum(kept) * (1 - sum(kept) / _pool_blocks(case)))
        return {"bytes": 2 * moved * block + 8 * moved + 12 * freed + 8 * sum(kept), "flops": 0}
    new = _new_tokens(case)
    fresh = sum(_ceil(t + n, BLOCK) - _ceil(t, BLOCK) for t, n in zip(lens, new) if n)
    freed = sum(min(_ceil(t, BLOCK), _ceil(case["window"] + case["sinks"], BLOCK) + 1) for i, t in enumerate(lens) if i in set(gone))
    return {"bytes": sum(new) * 8 + case["seqs"] * 12 + (2 * fresh + freed) * 12 + _pool_blocks(case) // 8, "flops": 0}


# ---- inputs

def _to_tiles(x, e, value):
    """Rows [NB, H, 16, d] in the order of the pool's K or V tiles, e elements per 16 bytes."""
    nb, h, _, d = x.shape
    if value:
        return x.view(nb, h, 4, 4, d // (4 * e), e // 4, 16).permute(0, 1, 4, 2, 6, 5, 3).reshape(nb, h, BLOCK * d)
    return x.view(nb, h, BLOCK, d // e, e).permute(0, 1, 3, 2, 4).reshape(nb, h, BLOCK * d)


def _pool(case, nb, gen):
    """A pool of N(0, 1) rows: K, V and their scales (None for fp16)."""
    made, e = [], 8 if case["cache"] == "fp16" else 16
    for value in (False, True):
        x = torch.randn((nb, case["kv_heads"], BLOCK, case["dim"]), generator=gen, device="cuda").half()
        scale = None
        if case["cache"] != "fp16":
            top = _MAX[case["cache"]]
            scale = x.float().abs().amax(-1) / top
            x = (x.float() / scale[..., None]).clamp(-top, top).to(_CODE[case["cache"]]).view(torch.uint8)
        made.append((_to_tiles(x, e, value).contiguous(), scale))
    return made[0][0], made[1][0], made[0][1], made[1][1]


def _prepare_attention(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    lengths = _lengths(case)
    order = torch.randperm(len(lengths), generator=host).tolist()
    lengths = [lengths[i] for i in order]
    S, decode = len(lengths), case["op"] == "decode"
    total = [b + n for b, n in lengths]
    width = max(1, max(_ceil(t, BLOCK) for t in total))
    held = []
    for t in total:
        row = list(range(_ceil(t, BLOCK)))
        if decode:
            row = [b for b in row if b * BLOCK < case["sinks"] or (b + 1) * BLOCK > t - case["window"]]
        held.append(row)
    nb = sum(len(r) for r in held) + 5
    pages = torch.randperm(nb, generator=host).tolist()
    tables = torch.full((S, width), -1, dtype=torch.int32)
    at = 0
    for s, row in enumerate(held):
        tables[s, torch.tensor(row, dtype=torch.long)] = torch.tensor(pages[at:at + len(row)], dtype=torch.int32)
        at += len(row)
    k, v, ks, vs = _pool(case, nb, gen)
    new = [n for _, n in lengths]
    rows = sum(new)
    starts = torch.tensor([sum(new[:i]) for i in range(S + 1)], dtype=torch.int32)
    q = torch.randn((rows, case["q_heads"], case["dim"]), generator=gen, device="cuda").half()
    return {"op": case["op"], "k": k, "v": v, "ks": ks, "vs": vs, "q": q, "tables": tables.cuda(),
            "lens": torch.tensor(total, dtype=torch.int32).cuda(), "starts": starts.cuda(), "rows": rows,
            "longest": max(new), "out": torch.zeros_like(q), "case": case, "scale": case["dim"] ** -0.5, "kept": {}}


def _prepare_blocks(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    lens, rows, gone = _block_case(case)
    S, op, nb = case["seqs"], case["op"], _pool_blocks(case)
    new = _new_tokens(case) if op == "roll" else [0] * S
    width = max(1, max(_ceil(t + n, BLOCK) for t, n in zip(lens, new)))
    tables = torch.full((rows, width), -1, dtype=torch.int32)
    refs = torch.zeros(nb, dtype=torch.int32)
    pages = torch.randperm(nb, generator=host)
    at = 0
    for s, t in enumerate(lens):
        held = torch.arange(_ceil(t, BLOCK))
        if op == "roll":
            # blocks behind the window went in earlier steps; the last step's tokens are not taken into account yet
            was = t - (case["chunk"] if s % 8 == 3 else 1)
            held = held[(held * BLOCK < case["sinks"]) | ((held + 1) * BLOCK > was - case["window"])]
            # of four sequences, the blocks of the first tokens are the same
            lead = s - s % 4
            common = held[(held * BLOCK < case["sinks"]) & ((held + 1) * BLOCK <= lens[lead])] if s % 4 else held[:0]
            tables[s, common] = tables[lead, common]
            held = held[common.numel():]
            refs[tables[s, common].long()] += 1
        tables[s, held] = pages[at:at + held.numel()].int()
        refs[tables[s, held].long()] += 1
        at += held.numel()
    bits = torch.zeros(_ceil(nb, 32) * 32, dtype=torch.int64)
    bits[:nb] = (refs == 0).long()
    words = (bits.view(-1, 32) << torch.arange(32)).sum(1)
    free = torch.where(words >= 2 ** 31, words - 2 ** 32, words).int()
    lengths = torch.tensor(lens + [0] * (rows - S), dtype=torch.int32)
    parts = [tables.reshape(-1), lengths, refs, free]
    start = torch.cat(parts).cuda()
    live = start.clone()
    views = live.split([p.numel() for p in parts])
    st = {"op": op, "case": case, "start": start, "live": live, "tables": views[0].view(rows, width), "lens": views[1],
          "refs": views[2], "free": views[3], "nb": nb, "result": torch.zeros(1, dtype=torch.int32, device="cuda"), "kept": {}}
    if op == "fork":
        parents = torch.arange(S).repeat_interleave(case["samples"])
        children = S + torch.randperm(rows - S, generator=host)
        st["parents"], st["children"] = parents.int().cuda(), children.int().cuda()
        st["copies"] = torch.zeros((rows - S, 2), dtype=torch.int32, device="cuda")
    if op == "compact":
        st["copies"] = torch.zeros((max(nb // 2, 1), 2), dtype=torch.int32, device="cuda")
    if op != "fork":
        st["gone"] = torch.tensor(gone, dtype=torch.int32).cuda()
    if op == "roll":
        st["starts"] = torch.tensor([sum(new[:i]) for i in range(S + 1)], dtype=torch.int32).cuda()
        st["rows"] = sum(new)
        st["slots"] = torch.zeros(sum(new), dtype=torch.int64, device="cuda")
    else:
        e = 2 if case["cache"] == "fp16" else 1
        size = (case["layers"], nb, case["kv_heads"], BLOCK * case["dim"])
        # (any finite values do: nothing is computed from them)
        top = 0x78 if e == 1 else 0x7800
        for name in ("k", "v"):
            x = torch.randint(0, top, size, generator=gen, device="cuda", dtype=torch.uint8 if e == 1 else torch.int16)
            st[name] = x.view(torch.float16) if e == 2 else x
            st[name + "s"] = None if e == 2 else torch.rand((*size[:3], BLOCK), generator=gen, device="cuda")
    return st


def prepare(case, seed):
    return _prepare_attention(case, seed) if case["op"] in ("decode", "prefill") else _prepare_blocks(case, seed)


# ---- the plain forms

def _rows_of(st, name, block, token):
    """K or V rows [S, n, H, d] in 32 bits of the tokens in (block, place) [S, n]."""
    case = st["case"]
    tiles, d = st[name], case["dim"]
    nb, h, e = tiles.shape[0], tiles.shape[1], 8 if case["cache"] == "fp16" else 16
    if name == "v":
        x = tiles.view(nb, h, d // (4 * e), 4, 16, e // 4, 4).permute(0, 3, 6, 1, 2, 5, 4)[block, token // 4, token % 4]
    else:
        x = tiles.view(nb, h, d // e, BLOCK, e).permute(0, 3, 1, 2, 4)[block, token]
    x = x.reshape(*block.shape, h, d)
    if case["cache"] == "fp16":
        return x.float()
    scale = st[name + "s"].permute(0, 2, 1)[block, token]
    return x.view(_CODE[case["cache"]]).float() * scale[..., None]


def _plain_attention(st):
    """Every sequence's keys as one row of columns: the first tokens, then those of all its new rows' windows."""
    case, lens, starts = st["case"], st["lens"].long(), st["starts"].long()
    w, sinks, S, R, C = case["window"], case["sinks"], lens.shape[0], st["rows"], st["longest"]
    kv, heads, d = case["kv_heads"], case["q_heads"], case["dim"]
    tables = st["tables"].long()
    most = tables.shape[1] * BLOCK
    new = starts[1:] - starts[:-1]
    before = lens - new
    first = (before + 1 - w).clamp(min=0)                               # of the first row's window
    cols = torch.arange(min(w - 1 + C, most), device="cuda")
    pos = torch.cat([torch.arange(sinks, device="cuda").expand(S, -1), first[:, None] + cols], 1)
    there = torch.cat([(pos[:, :sinks] < first[:, None]), pos[:, sinks:] < lens[:, None]], 1)
    at = torch.where(there, pos, 0)
    block = tables.gather(1, at // BLOCK).clamp(min=0)
    k, v = _rows_of(st, "k", block, at % BLOCK), _rows_of(st, "v", block, at % BLOCK)
    # rows, each sequence's padded to the longest
    i = torch.arange(C, device="cuda")
    row = (starts[:-1, None] + i).clamp(max=max(R - 1, 0))
    q = st["q"][row].float().view(S, C, kv, heads // kv, d).permute(0, 2, 3, 1, 4).reshape(S, kv, -1, d)
    z = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) * st["scale"]                 # [S, kv, g C, n]
    p = (before[:, None] + i)[:, :, None]                                                # position of row i
    seen = there[:, None] & (pos[:, None] <= p) & ((pos[:, None] < sinks) | (pos[:, None] > p - w))
    z = z.view(S, kv, heads // kv, C, -1).masked_fill(~seen[:, None, None], float("-inf"))
    z = torch.exp(z - z.amax(-1, keepdim=True).clamp(min=-3e38))
    total = z.sum(-1, keepdim=True)
    o = torch.matmul(z.view(S, kv, -1, z.shape[-1]), v.permute(0, 2, 1, 3).contiguous()).view(S, kv, heads // kv, C, d)
    o = (o / torch.where(total > 0, total, 1)).permute(0, 3, 1, 2, 4).reshape(S * C, heads, d)
    r = torch.arange(R, device="cuda")
    seq = torch.searchsorted(starts, r, right=True) - 1
    st["out"].copy_(o[seq * C + r - starts[seq]])
    return st["out"]


def _bits(words, n):
    return ((words[:, None] >> torch.arange(32, device="cuda")) & 1).view(-1)[:n]


def _words(free):
    n = free.shape[0]
    bits = torch.nn.functional.pad(free.long(), (0, -n % 32)).view(-1, 32)
    return (bits << torch.arange(32, device="cuda")).sum(1).to(torch.int32)


def _nth(mask, ranks):
    """The places of the ranks-th (from 0) true ones of a mask."""
    return torch.searchsorted(torch.cumsum(mask.long(), 0), ranks + 1)


def _count(st, blocks, held, by):
    """`by` references to every held entry's block.  (The others add nothing, each to a place of its own.)"""
    blocks, held = blocks.reshape(-1).long(), held.reshape(-1)
    st["refs"].scatter_add_(0, torch.where(held, blocks, torch.arange(blocks.shape[0], device="cuda") % st["nb"]), by * held.int())


def _release(st, entries, held):
    """One reference less to every held entry's block; the map where none is left."""
    _count(st, entries, held, -1)
    st["free"].copy_(_words(st["refs"] == 0))


def _plain_free(st, seqs):
    tables, lens = st["tables"], st["lens"]
    b = torch.arange(tables.shape[1], device="cuda")
    rows = tables[seqs.long()]
    _release(st, rows, (rows >= 0) & (b * BLOCK < lens[seqs.long()][:, None]))
    lens[seqs.long()] = 0


def _plain_behind_window(st):
    case, tables, lens = st["case"], st["tables"], st["lens"]
    b = torch.arange(tables.shape[1], device="cuda")
    out = (tables >= 0) & (b * BLOCK >= case["sinks"]) & ((b + 1) * BLOCK <= lens[:, None] - case["window"])
    _release(st, tables, out)
    tables.masked_fill_(out, -1)


def _plain_reserve(st):
    tables, lens, starts = st["tables"], st["lens"], st["starts"].long()
    old = lens.long()
    total = old + starts[1:] - starts[:-1]
    have, need = (old + BLOCK - 1) // BLOCK, (total + BLOCK - 1) // BLOCK
    rank = torch.cumsum(need - have, 0) - (need - have)                          # of a sequence's first new block
    free = _bits(st["free"], st["nb"])
    b = torch.arange(tables.shape[1], device="cuda")
    fresh = (b >= have[:, None]) & (b < need[:, None])
    page = _nth(free, rank[:, None] + b - have[:, None]).clamp(max=st["nb"] - 1)
    tables.copy_(torch.where(fresh, page.int(), tables))
    _count(st, page, fresh, 1)
    st["free"].copy_(_words(st["refs"] == 0))
    lens.copy_(total)
    r = torch.arange(st["rows"], device="cuda")
    seq = torch.searchsorted(starts, r, right=True) - 1
    pos = old[seq] + r - starts[seq]
    st["slots"].copy_(tables[seq, pos // BLOCK].long() * BLOCK + pos % BLOCK)
    st["result"].zero_()


def _plain_fork(st):
    tables, lens, parents, children = st["tables"], st["lens"], st["parents"].long(), st["children"].long()
    t = lens[parents].long()
    full, partial = t // BLOCK, t % BLOCK > 0
    b = torch.arange(tables.shape[1], device="cuda")
    rows = tables[parents]
    shared = (b < full[:, None]) & (rows >= 0)
    _count(st, rows, shared, 1)
    page = _nth(_bits(st["free"], st["nb"]), torch.cumsum(partial.long(), 0) - partial.long()).clamp(max=st["nb"] - 1).int()
    source = rows.gather(1, full[:, None].clamp(max=rows.shape[1] - 1))[:, 0]
    last = (b == full[:, None]) & partial[:, None]
    rows = torch.where(last, page[:, None], torch.where(b < full[:, None], rows, tables[children]))
    tables[children] = rows
    lens[children] = t.int()
    _count(st, page, partial, 1)
    st["free"].copy_(_words(st["refs"] == 0))
    st["copies"].copy_(torch.where(partial[:, None], torch.stack([source, page], 1), -1))
    st["result"].zero_()


def _plain_compact(st):
    tables, lens, nb = st["tables"], st["lens"], st["nb"]
    used = st["refs"] > 0
    n = used.sum()
    at = torch.arange(nb, device="cuda")
    k = torch.arange(st["copies"].shape[0], device="cuda")
    moved = (used & (at >= n)).sum()
    src = _nth(used & (at >= n), k).clamp(max=nb - 1)
    dst = _nth(~used & (at < n), k).clamp(max=nb - 1)
    st["copies"].copy_(torch.where((k < moved)[:, None], torch.stack([src, dst], 1), -1))
    st["result"].copy_(moved)
    to = at.clone()
    to.scatter_reduce_(0, src, torch.where(k < moved, dst, nb), "amin")
    b = torch.arange(tables.shape[1], device="cuda")
    held = (tables >= 0) & (b * BLOCK < lens[:, None])
    tables.copy_(torch.where(held, to[tables.clamp(min=0).long()].int(), tables))
    old = st["refs"].clone()
    st["refs"].masked_fill_(at >= n, 0)
    st["refs"].scatter_add_(0, torch.where(k < moved, dst, 0), torch.where(k < moved, old[src], 0))
    st["free"].copy_(_words(at >= n))


def _plain_copy(st):
    """(A pair that is none copies the pool's last block, which no pair writes, to itself.)"""
    none = st["nb"] - 1
    src, dst = (torch.where(st["copies"][:, i] >= 0, st["copies"][:, i], none).long() for i in (0, 1))
    for pool in (st["k"], st["v"], st["ks"], st["vs"]):
        if pool is not None:
            words = pool.view(torch.int64)
            words[:, dst] = words[:, src]


def _plain(st):
    if st["op"] in ("decode", "prefill"):
        return _plain_attention(st)
    if st["op"] == "fork":
        _plain_fork(st)
        _plain_copy(st)
    elif st["op"] == "compact":
        _plain_free(st, st["gone"])
        _plain_compact(st)
        _plain_copy(st)
    else:
        _plain_free(st, st["gone"])
        _plain_behind_window(st)
        _plain_reserve(st)
    return None


# ---- the framework's calls

def _shape(st):
    coopt, case = _coopt(), st["case"]
    return coopt.Shape(st["tables"].shape[0], case.get("q_heads", case["kv_heads"]), case["kv_heads"], case["dim"], BLOCK,
                       st["k"].shape[-3] if "k" in st else st["nb"], st["tables"].shape[1],
                       {"e4m3": coopt.COOPT_KV_E4M3, "e5m2": coopt.COOPT_KV_E5M2, "fp16": coopt.COOPT_KV_FP16}[case["cache"]],
                       case["dim"] ** -0.5)


def _keep(st):
    """The shape, the layers' pools and the workspace, which a program makes once."""
    kept = st["kept"]
    if not kept:
        coopt, case = _coopt(), st["case"]
        kept["shape"] = shape = _shape(st)
        if st["op"] == "decode":
            need = coopt.decode_window_workspace_bytes(shape, case["window"], case["sinks"])
        elif st["op"] == "prefill":
            need = coopt.prefill_window_workspace_bytes(shape, st["longest"], case["window"], case["sinks"])
        else:
            need = coopt.kv_blocks_workspace_bytes(shape)
            kept["pools"] = [list(st[n].unbind(0)) if st.get(n) is not None else None for n in ("k", "v", "ks", "vs")]
        kept["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    return kept["shape"], kept["workspace"], kept.get("pools")


def _own(st):
    coopt, case = _coopt(), st["case"]
    shape, workspace, pools = _keep(st)
    if st["op"] == "decode":
        coopt.paged_gqa_decode_window(st["q"], st["k"], st["v"], st["ks"], st["vs"], st["tables"], st["lens"], case["window"],
                                      case["sinks"], st["out"], workspace, shape)
        return st["out"]
    if st["op"] == "prefill":
        coopt.paged_gqa_prefill_chunk_window(st["q"], st["k"], st["v"], st["ks"], st["vs"], st["tables"], st["lens"], st["starts"],
                                             st["rows"], st["longest"], case["window"], case["sinks"], st["out"], workspace, shape)
        return st["out"]
    pages = st["tables"], st["lens"], st["refs"], st["free"]
    if st["op"] == "fork":
        coopt.kv_blocks_fork(st["parents"], st["children"], *pages, st["copies"], st["result"], workspace, shape)
        coopt.kv_cache_copy_blocks(*pools, st["copies"], None, shape)
    elif st["op"] == "compact":
        coopt.kv_blocks_free(st["gone"], *pages, shape)
        coopt.kv_blocks_compact(*pages, st["copies"], st["result"], workspace, shape)
        coopt.kv_cache_copy_blocks(*pools, st["copies"], st["result"], shape)
    else:
        coopt.kv_blocks_free(st["gone"], *pages, shape)
        coopt.kv_blocks_free_outside_window(*pages, case["window"], case["sinks"], shape)
        coopt.kv_blocks_reserve(st["starts"], st["rows"], *pages, st["slots"], st["result"], workspace, shape)
    return None


def run(state):
    attention = state["op"] in ("decode", "prefill")
    if not attention:
        state["live"].copy_(state["start"])
    out = _own(state) if own else _plain(state)
    if attention:
        return out
    outputs = {n: state[n] for n in ("tables", "lens", "refs", "free", "result")}
    if state["op"] == "fork":
        outputs["copies"] = state["copies"]
    if state["op"] == "roll":
        outputs["slots"] = state["slots"]
    else:
        for n in ("k", "v"):
            codes = state["case"]["cache"] != "fp16"
            outputs[n] = state[n].view(_CODE[state["case"]["cache"]]) if codes else state[n]
            if codes:
                outputs[n + "s"] = state[n + "s"]
    return outputs


# ---- the definition in 64 bits

def exact(case, seed):
    """Row by row of the definition; the block operators compute no numbers."""
    if case["op"] not in ("decode", "prefill"):
        return None
    st = prepare(case, seed)
    d, h, e = case["dim"], case["kv_heads"], 8 if case["cache"] == "fp16" else 16
    g = case["q_heads"] // h
    tok, dim = (x.cuda() for x in torch.meshgrid(torch.arange(BLOCK), torch.arange(d), indexing="ij"))
    c, n, wide = dim // 16, dim % 16, e // 4
    place = {"k": (dim // e * BLOCK + tok) * e + dim % e, "v": (((c // wide * 4 + tok // 4) * 16 + n) * wide + c % wide) * 4 + tok % 4}
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    starts, lens = st["starts"].tolist(), st["lens"].tolist()
    for s, t in enumerate(lens):
        rows = range(starts[s], starts[s + 1])
        before = t - len(rows)
        low = max(before + 1 - case["window"], 0)
        keys = torch.tensor(sorted(set(range(min(case["sinks"], t))) | set(range(low, t))), device="cuda")
        block = st["tables"][s].long()[keys // BLOCK]
        side = {}
        for name in ("k", "v"):
            x = st[name][block]                                                     # [keys, h, 16 d]
            x = x.gather(2, place[name][keys % BLOCK][:, None].expand(-1, h, -1))
            x = x.double() if case["cache"] == "fp16" else x.view(_CODE[case["cache"]]).double() * st[name + "s"][block][torch.arange(len(keys), device="cuda"), :, keys % BLOCK].double()[..., None]
            side[name] = x.permute(1, 0, 2).contiguous()
        for r0 in range(0, len(rows), 512):
            r1 = min(r0 + 512, len(rows))
            p = torch.arange(before + r0, before + r1, device="cuda")[:, None]
            seen = (keys <= p) & ((keys > p - case["window"]) | (keys < case["sinks"]))
            for a in range(h):
                q = st["q"][rows[0] + r0:rows[0] + r1, a * g:(a + 1) * g].double().permute(1, 0, 2)
                z = torch.matmul(q, side["k"][a].T.contiguous()) * st["scale"]
                z = torch.softmax(z.masked_fill(~seen, float("-inf")), -1)
                out[rows[0] + r0:rows[0] + r1, a * g:(a + 1) * g] = torch.matmul(z, side["v"][a]).permute(1, 0, 2)
    return out

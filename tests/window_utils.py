"""A plain restatement, in 64 bits, of attention through a sliding window with the first tokens visible, and
workloads whose hidden tokens are poisoned: whatever a launch reads of them must not show."""
import numpy as np
import torch

import workloads
from helpers import k_tile_index, oracle_fill, v_tile_index


CODES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


class Rows:
    """K and V [H_k, keys, d] in 64 bits of a sequence's tokens, from the cache's bytes."""
    def __init__(self, w, cache):
        self.w = w
        self.where = "cuda" if torch.cuda.is_available() else "cpu"
        self.cache = [None if x is None else torch.from_numpy(x).to(self.where) for x in cache]
        E = 8 if w.kv_dtype == "fp16" else 16
        self.places = [torch.from_numpy(f(w.d, E, w.B)).to(self.where) for f in (k_tile_index, v_tile_index)]

    def of(self, s, keys):
        w = self.w
        block = torch.from_numpy(w.block_tables[s, keys // w.B].astype(np.int64)).to(self.where)
        place = torch.from_numpy(keys % w.B).to(self.where)
        out = []
        for data, scale, at in ((self.cache[0], self.cache[2], self.places[0]), (self.cache[1], self.cache[3], self.places[1])):
            x = data[block].gather(2, at[place][:, None].expand(-1, w.H_k, -1))
            if scale is None:
                x = x.double()
            else:
                one = scale[block].gather(2, place[:, None, None].expand(-1, w.H_k, 1))
                x = x.view(CODES[w.kv_dtype]).double() * one.double()
            out.append(x.permute(1, 0, 2).contiguous())
        return out


def seen_keys(p, window, sinks):
    """The tokens that the one at position p sees."""
    j = np.arange(p + 1)
    return j[(j > p - window) | (j < sinks)]


def window_attention(w, cache, q, lens, starts, window, sinks):
    """[rows, H_q, d] float64: sequence s's rows starts[s] .. starts[s+1]-1 are its last tokens."""
    G, rows = w.H_q // w.H_k, Rows(w, cache)
    where = rows.where
    out = torch.zeros(q.shape, dtype=torch.float64, device=where)
    for s in range(len(lens)):
        C = int(starts[s + 1] - starts[s])
        t = int(lens[s])
        if t == 0 or C == 0:
            continue
        first = max(t - C + 1 - window, 0)                 # of the first row's window
        keys = np.union1d(np.arange(min(sinks, t)), np.arange(first, t))
        K, V = rows.of(s, keys)
        x = torch.from_numpy(q[starts[s]:starts[s + 1]]).to(where).double().view(C, w.H_k, G, w.d)
        x = x.permute(1, 2, 0, 3).reshape(w.H_k, G * C, w.d)
        p = np.arange(t - C, t)[:, None]
        seen = torch.from_numpy((keys <= p) & ((keys > p - window) | (keys < sinks))).to(where)
        for g in range(w.H_k):
            z = torch.matmul(x[g], K[g].T.contiguous()).view(G, C, -1) * w.softmax_scale
            z = torch.softmax(z.masked_fill(~seen, -np.inf), -1).view(G * C, -1)
            o = torch.matmul(z, V[g]).view(G, C, w.d)
            out[starts[s]:starts[s + 1], g * G:(g + 1) * G] = o.permute(1, 0, 2)
    return out.cpu().numpy()


def poisoned(oracle, w, hidden):
    """The workload's cache and block tables with nothing to be had from hidden tokens: hidden(s) gives
    sequence s's; their codes and scales are NaN, and the table entries of blocks that are wholly hidden, or beyond
    the sequence, name a block of NaN (the pool's last)."""
    cache = oracle_fill(oracle, w)
    nan = {"e4m3": 0x7F, "e5m2": 0x7F, "fp16": np.float16(np.nan)}[w.kv_dtype]
    bad = w.NB - 1
    assert bad not in w.block_tables
    for x, value in zip(cache, (nan, nan, np.nan, np.nan)):
        if x is not None:
            x[bad] = value
    tables = w.block_tables.copy()
    blocks, places = [], []
    for s in range(w.S):
        t = int(w.context_lens[s])
        gone = np.zeros(w.max_blocks * w.B, bool)
        gone[t:] = True
        gone[hidden(s)] = True
        j = np.flatnonzero(gone[:t])
        blocks.append(tables[s, j // w.B])
        places.append(j % w.B)
        tables[s][gone.reshape(-1, w.B).all(axis=1)] = bad
    blocks, places = np.concatenate(blocks), np.concatenate(places)
    heads, E = np.arange(w.H_k)[:, None], 8 if w.kv_dtype == "fp16" else 16
    for x, f in ((cache[0], k_tile_index), (cache[1], v_tile_index)):
        x[blocks[:, None, None], heads, f(w.d, E, w.B)[places][:, None]] = nan
    for x in cache[2:]:
        if x is not None:
            x[blocks, :, places] = np.nan
    return cache, tables


def random_workload(name, seed, kv_dtype, H_q, H_k, d, lens, new_per_seq=1, slack=8, max_blocks=None):
    """One block of the pool at least is nobody's (its last)."""
    need = sum(-(-int(t) // 16) for t in lens)
    w = workloads.make_custom(name, seed=seed, S=len(lens), H_q=H_q, H_k=H_k, d=d, B=16, NB=need + slack,
                              context_lens=lens, kv_dtype=kv_dtype, new_per_seq=new_per_seq, max_blocks=max_blocks)
    # the last block out of use: swapped with one that is
    last = w.NB - 1
    if last in w.block_tables:
        free = next(b for b in range(w.NB) if b not in w.block_tables)
        w.slots[w.slots // 16 == last] += (free - last) * 16
        w.block_tables[w.block_tables == last] = free
    return w


def ragged_rows(w, chunks, seed=5):
    """The last `chunks[s]` tokens of every sequence as a prefill's rows: q [rows, H_q, d] and starts."""
    starts = np.concatenate([[0], np.cumsum(chunks)]).astype(np.int32)
    rng = np.random.default_rng(seed)
    return rng.standard_normal((int(starts[-1]), w.H_q, w.d), dtype=np.float32).astype(np.float16), starts

"""A plain restatement, in 64 bits, of attention through a sliding window with the first tokens visible, and
workloads whose hidden tokens are poisoned: whatever a launch reads of them must not show."""
import numpy as np
import torch

import workloads
from helpers import k_logical, k_store_logical, oracle_fill, v_logical, v_store_logical


def _values(w):
    """The value of every code, or None for an fp16 cache."""
    if w.kv_dtype == "fp16":
        return None
    code = torch.float8_e4m3fn if w.kv_dtype == "e4m3" else torch.float8_e5m2
    return torch.arange(256, dtype=torch.uint8).view(code).to(torch.float64).numpy()


def rows_of(w, cache, s, keys):
    """K and V [len(keys), H_k, d] float64 of sequence s's tokens `keys`."""
    block, place = w.block_tables[s, keys // w.B], keys % w.B
    table = _values(w)
    out = []
    for logical, data, scale in ((k_logical, cache[0], cache[2]), (v_logical, cache[1], cache[3])):
        x = logical(_Part(w, len(block)), data[block])[np.arange(len(block)), :, place]
        out.append(x.astype(np.float64) if table is None
                   else table[x] * scale[block, :, place].astype(np.float64)[:, :, None])
    return out


class _Part:
    """The workload's tile layout over a pool of n blocks."""
    def __init__(self, w, n):
        self.NB, self.H_k, self.B, self.d, self.kv_dtype = n, w.H_k, w.B, w.d, w.kv_dtype


def seen_keys(p, window, sinks):
    """The tokens that the one at position p sees."""
    j = np.arange(p + 1)
    return j[(j > p - window) | (j < sinks)]


def window_attention(w, cache, q, lens, starts, window, sinks):
    """[rows, H_q, d] float64: sequence s's rows starts[s] .. starts[s+1]-1 are its last tokens."""
    G, where = w.H_q // w.H_k, "cuda" if torch.cuda.is_available() else "cpu"
    out = np.zeros(q.shape)
    for s in range(len(lens)):
        C = int(starts[s + 1] - starts[s])
        t = int(lens[s])
        if t == 0 or C == 0:
            continue
        first = max(t - C + 1 - window, 0)                 # of the first row's window
        keys = np.union1d(np.arange(min(sinks, t)), np.arange(first, t))
        K, V = (torch.from_numpy(x.transpose(1, 0, 2).copy()).to(where) for x in rows_of(w, cache, s, keys))
        x = q[starts[s]:starts[s + 1]].astype(np.float64).reshape(C, w.H_k, G, w.d).transpose(1, 2, 0, 3)
        x = torch.from_numpy(x.reshape(w.H_k, G * C, w.d).copy()).to(where)
        p = np.arange(t - C, t)[:, None]
        seen = torch.from_numpy((keys <= p) & ((keys > p - window) | (keys < sinks))).to(where)
        for g in range(w.H_k):
            z = torch.matmul(x[g], K[g].T.contiguous()).view(G, C, -1) * w.softmax_scale
            z = torch.softmax(z.masked_fill(~seen, -np.inf), -1).view(G * C, -1)
            o = torch.matmul(z, V[g]).view(G, C, w.d)
            out[starts[s]:starts[s + 1], g * G:(g + 1) * G] = o.permute(1, 0, 2).cpu().numpy()
    return out


def poisoned(oracle, w, hidden):
    """The workload's cache and block tables with nothing to be had from hidden tokens: hidden(s) gives
    sequence s's; their codes and scales are NaN, and the table entries of blocks that are wholly hidden, or beyond
    the sequence, name a block of NaN (the pool's last)."""
    cache = oracle_fill(oracle, w)
    nan = {"e4m3": 0x7F, "e5m2": 0x7F, "fp16": np.float16(np.nan)}[w.kv_dtype]
    bad = w.NB - 1
    assert bad not in w.block_tables
    kl, vl = k_logical(w, cache[0]), v_logical(w, cache[1])
    kl[bad] = vl[bad] = nan
    if cache[2] is not None:
        cache[2][bad] = cache[3][bad] = np.nan
    tables = w.block_tables.copy()
    for s in range(w.S):
        t = int(w.context_lens[s])
        gone = np.zeros(w.max_blocks * w.B, bool)
        gone[t:] = True
        gone[hidden(s)] = True
        for j in np.flatnonzero(gone[:t]):
            b, place = tables[s, j // w.B], j % w.B
            kl[b, :, place] = vl[b, :, place] = nan
            if cache[2] is not None:
                cache[2][b, :, place] = cache[3][b, :, place] = np.nan
        tables[s][gone.reshape(-1, w.B).all(axis=1)] = bad
    k_store_logical(w, cache[0], kl)
    v_store_logical(w, cache[1], vl)
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

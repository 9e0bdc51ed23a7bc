"""GPU: the forms of the windowed launches that test_gpu_window.py's cases leave out -- whole streams of 64 dims, of few
tiles a pair -- and every form again over pools of more than 2 GiB per tensor, whose tiles are read, and whose new tokens
are stored, with 64-bit offsets.  test_window_forms.py asks the rule which launch every case is."""
import numpy as np
import pytest
import torch

import paper_2602_09323_amd as coopt
from gpu_utils import assert_close, cache_to_dev, dev, shape_of
from test_gpu_window import FORM_HEADS, hidden_from, hip_prefill_window, workspace_for
from window_utils import poisoned, ragged_rows, random_workload, window_attention

pytestmark = pytest.mark.gpu

# q heads, KV heads, chunks, lengths, window, sinks
WHOLE = {"stream16": (10, 2, [700] * 5, [1200, 700, 2000, 701, 1111], 500, 7),
         "stream8": (16, 8, [64] * 20, [64 + 37 * s for s in range(20)], 500, 4)}
KINDS = sorted({(kv, d) for kv, _, _, d in FORM_HEADS})


@pytest.mark.parametrize("form", WHOLE)
@pytest.mark.parametrize("kv,d", KINDS)
def test_whole_streams(oracle_mod, kv, d, form):
    H_q, H_k, chunks, lens, window, sinks = WHOLE[form]
    w = random_workload("window_whole", 71, kv, H_q, H_k, d, lens)
    q, starts = ragged_rows(w, chunks)
    cache, tables = poisoned(oracle_mod, w, hidden_from(w, chunks, window, sinks))
    ref = window_attention(w, cache, q, w.context_lens, starts, window, sinks)
    assert_close(hip_prefill_window(w, cache_to_dev(cache), tables, q, starts, window, sinks), ref, form)


# The forms over a large pool, for every cache and head size
BIG_PREFILL = {"tile1": (32, 8, [200], [300], 16, 0), "tile2": (40, 8, [30, 7], [800, 90], 130, 4), "tile4": (40, 8, [16], [700], 500, 4),
               "tile1of32": (32, 8, [500] * 5, [500, 700, 512, 501, 999], 33, 4), **WHOLE,
               "stream16parts": (40, 8, [700], [2000], 1500, 4), "stream8parts": (40, 8, [16, 16], [4300, 60], 4000, 7)}
# lengths, window, sinks of 40 heads over 8; whether the call needs a workspace (320 pairs of 64 dims are few enough for parts)
BIG_DECODE = {"one launch": ([300, 1025, 47, 16], 200, 4, False), "parts": ([2500, 1, 0, 2097], 2048, 20, True),
              "balanced": ([17, 100, 113, 1, 0, 129, 64, 200, 33, 97] * 7, 64, 4, True)}


def _large(w, cache, tables):
    """The cache dealt over a pool beyond 2 GiB per tensor, every byte of other blocks NaN codes: shape, device cache,
    table, and the place of every block."""
    shape = shape_of(w)
    tile = w.H_k * 16 * w.d * (2 if w.kv_dtype == "fp16" else 1)
    shape.num_blocks = NB = 3 * (1 << 30) // tile
    spread = np.sort(np.random.default_rng(72).permutation(NB)[:w.NB])
    spread[-2:] = NB - 2, NB - 1
    assert (spread[np.maximum(tables, 0)].astype(np.int64) * tile).max() > 1 << 31
    at = torch.from_numpy(spread).cuda()
    dcache = []
    for part in cache_to_dev(cache):
        if part is None:
            dcache.append(None)
            continue
        big = torch.empty((NB, *part.shape[1:]), dtype=part.dtype, device="cuda")
        big.view(torch.uint8).fill_(0x7F)
        big[at] = part
        dcache.append(big)
    return shape, dcache, spread[np.maximum(tables, 0)].astype(np.int32), spread


@pytest.mark.parametrize("form", BIG_PREFILL)
@pytest.mark.parametrize("kv,d", KINDS)
def test_prefill_beyond_2_gib(oracle_mod, kv, d, form):
    H_q, H_k, chunks, lens, window, sinks = BIG_PREFILL[form]
    w = random_workload("window_large", 73, kv, H_q, H_k, d, lens)
    q, starts = ragged_rows(w, chunks)
    cache, tables = poisoned(oracle_mod, w, hidden_from(w, chunks, window, sinks))
    ref = window_attention(w, cache, q, w.context_lens, starts, window, sinks)
    shape, dcache, far, _ = _large(w, cache, tables)
    out = torch.full(q.shape, -7.0, dtype=torch.float16, device="cuda")
    ws = workspace_for(coopt.prefill_window_workspace_bytes(shape, max(chunks), window, sinks))
    coopt.paged_gqa_prefill_chunk_window(dev(q.view(np.uint16)), *dcache, dev(far), dev(w.context_lens), dev(starts), len(q), max(chunks),
                                         window, sinks, out, ws, shape)
    torch.cuda.synchronize()
    assert_close(out.cpu().numpy().astype(np.float64), ref, form)


@pytest.mark.parametrize("form", BIG_DECODE)
@pytest.mark.parametrize("kv,d", KINDS)
def test_decode_and_step_beyond_2_gib(oracle_mod, kv, d, form):
    lens, window, sinks, workspace = BIG_DECODE[form]
    w = random_workload("window_large", 74, kv, 40, 8, d, lens)
    cache, tables = poisoned(oracle_mod, w, hidden_from(w, [1] * w.S, window, sinks))
    ref = window_attention(w, cache, w.q, w.context_lens, np.arange(w.S + 1), window, sinks)
    shape, dcache, far, spread = _large(w, cache, tables)
    need = coopt.decode_window_workspace_bytes(shape, window, sinks)
    assert (need > 0) == workspace
    out = torch.full((w.S, 40, d), -7.0, dtype=torch.float16, device="cuda")
    tail = dev(far), dev(w.context_lens), window, sinks, out, workspace_for(need), shape
    coopt.paged_gqa_decode_window(dev(w.q.view(np.uint16)), *dcache, *tail)
    torch.cuda.synchronize()
    assert_close(out.cpu().numpy().astype(np.float64), ref, f"decode, {form}")
    # the fused step: the appended tokens' blocks hold nothing of them (sequences whose last block holds no other token)
    last = np.asarray(w.seq_start[1:]) - 1
    some = np.array([s for s in range(w.S) if lens[s] > 0])
    slots = np.full(w.S, -1, np.int64)
    slots[some] = spread[w.slots[last[some]] // 16].astype(np.int64) * 16 + w.slots[last[some]] % 16
    new = np.zeros((2, w.S, 8, d), np.float16)
    new[0, some], new[1, some] = w.k_ctx[last[some]], w.v_ctx[last[some]]
    alone = [s for s in some if lens[s] % 16 == 1]
    assert alone
    before = [None if x is None else x[torch.from_numpy(spread).cuda()].clone() for x in dcache]
    for x in dcache:
        if x is not None:
            for s in alone:
                x[int(slots[s]) // 16].view(torch.uint8).fill_(0x7F)
    out.fill_(-7.0)
    coopt.paged_gqa_decode_window_step(dev(new[0].view(np.uint16)), dev(new[1].view(np.uint16)), dev(slots), dev(w.q.view(np.uint16)),
                                       *dcache, *tail)
    torch.cuda.synchronize()
    assert_close(out.cpu().numpy().astype(np.float64), ref, f"step, {form}")
    for s in alone:                                            # the rest of such a block is as it was made: NaN codes
        b = int(np.searchsorted(spread, slots[s] // 16))
        for x, y in zip(before, dcache):
            if x is not None:
                got, want = y[int(slots[s]) // 16].view(torch.uint8), x[b].view(torch.uint8)
                kept = (got == want) | (got == 0x7F)
                assert bool(kept.all()) and bool((got != 0x7F).any())

"""GPU: the fused step through a window in its three forms (one launch, in parts, balanced), for batches whose appended
tokens are not in the cache at all: their places hold NaN, so a launch that took them from there would show, and so would
one that did not store them."""
import numpy as np
import pytest
import torch

import paper_2602_09323_amd as coopt
from gpu_utils import assert_close, cache_to_dev, dev, shape_of
from helpers import k_tile_index, v_tile_index
from test_gpu_window import HEADS, hidden_from, workspace_for
from window_utils import poisoned, random_workload, window_attention

pytestmark = pytest.mark.gpu

MIXED = [17, 100, 113, 1, 0, 129, 64, 200, 33, 97, 48, 145]
# lengths (of H_k heads), window, sinks; whether the call needs a workspace
CASES = {"one launch": (lambda H_k: MIXED, 64, 4, False),
         "parts": (lambda H_k: [2500, 1, 0, 2097, 700], 2048, 20, True),
         # (more than 512 pairs and more than 64 sequences)
         "balanced": (lambda H_k: (MIXED * 60)[:max(520 // H_k + 1, 75)], 64, 4, True),
         "balanced, longer": (lambda H_k: ([620, 625, 17, 609] * 200)[:max(520 // H_k + 1, 75)], 512, 4, True)}


def _stale(w, cache, slots):
    """The cache without these tokens: NaN codes and scales at their places."""
    out = [None if x is None else x.copy() for x in cache]
    nan = {"e4m3": 0x7F, "e5m2": 0x7F, "fp16": np.float16(np.nan)}[w.kv_dtype]
    heads, E = np.arange(w.H_k)[:, None], 8 if w.kv_dtype == "fp16" else 16
    blocks, places = slots // 16, slots % 16
    for x, f in ((out[0], k_tile_index), (out[1], v_tile_index)):
        x[blocks[:, None, None], heads, f(w.d, E, w.B)[places][:, None]] = nan
    for x in out[2:]:
        if x is not None:
            x[blocks, :, places] = np.nan
    return out


@pytest.mark.parametrize("form", CASES)
@pytest.mark.parametrize("kv,H_q,H_k,d", HEADS)
def test_appended_tokens_are_nowhere_else(oracle_mod, kv, H_q, H_k, d, form):
    lens, window, sinks, workspace = CASES[form]
    lens = lens(H_k)
    w = random_workload("window_step_stale", 61, kv, H_q, H_k, d, lens)
    cache, tables = poisoned(oracle_mod, w, hidden_from(w, [1] * w.S, window, sinks))
    ref = window_attention(w, cache, w.q, w.context_lens, np.arange(w.S + 1), window, sinks)
    last = np.asarray(w.seq_start[1:]) - 1
    some = np.array([s for s in range(w.S) if lens[s] > 0 and s % 3 != 2])
    slots = np.full(w.S, -1, np.int64)
    slots[some] = w.slots[last[some]]
    stale = _stale(w, cache, slots[some])
    # what a launch gives that leaves the new tokens out: no number, of just these sequences
    without = np.isnan(window_attention(w, stale, w.q, w.context_lens, np.arange(w.S + 1), window, sinks))
    assert without[some].all() and not np.delete(without, some, axis=0).any()
    new = np.full((2, w.S, H_k, d), np.nan, np.float16)        # (rows of sequences that append nothing are not read)
    new[0, some], new[1, some] = w.k_ctx[last[some]], w.v_ctx[last[some]]
    dcache, shape = cache_to_dev(stale), shape_of(w)
    out = torch.full((w.S, H_q, d), -7.0, dtype=torch.float16, device="cuda")
    need = coopt.decode_window_workspace_bytes(shape, window, sinks)
    assert (need > 0) == workspace
    coopt.paged_gqa_decode_window_step(dev(new[0].view(np.uint16)), dev(new[1].view(np.uint16)), dev(slots), dev(w.q.view(np.uint16)),
                                       *dcache, dev(tables), dev(w.context_lens), window, sinks, out, workspace_for(need), shape)
    torch.cuda.synchronize()
    assert_close(out.cpu().numpy().astype(np.float64), ref, form)
    for name, got, want in zip(("k_cache", "v_cache", "k_scale", "v_scale"), dcache, cache):
        if got is not None:
            assert np.array_equal(got.cpu().numpy().view(np.uint8), want.view(np.uint8)), name

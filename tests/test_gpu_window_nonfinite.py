"""GPU: queries and keys that are infinite or NaN, through a sliding window.  The rows that are no number are those that
see one, in 64 bits, and no others: rows in front of a bad key keep their values, and so do rows whose windows have left it
behind; in both launches of the prefill, and in decode."""
import numpy as np
import pytest
import torch

from gpu_utils import assert_close, cache_to_dev
from helpers import oracle_fill
from test_gpu_window import hip_decode_window, hip_prefill_window
from window_utils import ragged_rows, random_workload, window_attention

pytestmark = pytest.mark.gpu

SHAPES = [("e4m3", 10, 2, 128), ("e5m2", 16, 8, 64), ("fp16", 16, 8, 128), ("fp16", 10, 2, 64)]
# (chunks, lengths, window, sinks): one tile a workgroup; whole streams and streams in parts
CASES = [([70, 33], [110, 33], 40, 3), ([200], [700], 90, 0), ([1700, 30], [2500, 30], 700, 5), ([1100], [6000], 4500, 16)]


def _compare(got, ref, expected, what):
    bad = ~np.isfinite(ref).all(axis=2)
    assert not np.isfinite(ref[bad]).any() and expected(bad), "the rows are not those that the test is about"
    assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all(), what
    assert_close(np.where(bad[..., None], 0.0, got), np.where(bad[..., None], 0.0, ref), what)


def _place(w, position):
    return int(w.block_tables[0, position // 16]), position % 16


def _spoil(w, cache, position, value):
    """An element of a key (fp16), or a key's scale, of KV head 1 and the first sequence."""
    block, at = _place(w, position)
    if w.kv_dtype == "fp16":
        cache[0].reshape(w.NB, w.H_k, w.d // 8, 16, 8)[block, 1, 2, at, 5] = value
    else:
        cache[2][block, 1, at] = np.nan


@pytest.mark.parametrize("chunks,lens,window,sinks", CASES)
@pytest.mark.parametrize("kv,H_q,H_k,d", SHAPES)
def test_query_rows(oracle_mod, kv, H_q, H_k, d, chunks, lens, window, sinks):
    w = random_workload("window_bad_q", 31, kv, H_q, H_k, d, lens)
    q, starts = ragged_rows(w, chunks)
    q[5, 1, 3], q[8, 0, d - 1], q[17, 1, 0] = np.nan, np.inf, -np.inf
    cache = oracle_fill(oracle_mod, w)
    ref = window_attention(w, cache, q, w.context_lens, starts, window, sinks)
    _compare(hip_prefill_window(w, cache_to_dev(cache), w.block_tables, q, starts, window, sinks), ref,
             lambda bad: bad.sum() == 3 and bad[5, 1] and bad[8, 0] and bad[17, 1], f"{kv} {H_q}/{H_k}")


@pytest.mark.parametrize("chunks,lens,window,sinks", CASES)
@pytest.mark.parametrize("kv,H_q,H_k,d", SHAPES)
def test_keys(oracle_mod, kv, H_q, H_k, d, chunks, lens, window, sinks):
    w = random_workload("window_bad_k", 32, kv, H_q, H_k, d, lens)
    q, starts = ragged_rows(w, chunks)
    G, before = H_q // H_k, lens[0] - chunks[0]
    heads = slice(G, 2 * G)
    for position in (before + 11, max(before - window + 30, sinks)):
        cache = oracle_fill(oracle_mod, w)
        _spoil(w, cache, position, np.nan)
        ref = window_attention(w, cache, q, w.context_lens, starts, window, sinks)
        p = before + np.arange(chunks[0])
        sees = (p >= position) & (p < position + window)

        def expected(bad):
            return (bad[:chunks[0], heads] == sees[:, None]).all() and not bad[chunks[0]:].any() and bad[:, heads].sum() == bad.sum()
        _compare(hip_prefill_window(w, cache_to_dev(cache), w.block_tables, q, starts, window, sinks), ref, expected,
                 f"{kv} {H_q}/{H_k} key {position}")
        # decode: the last row alone, and one whose window has just left the key behind
        for t in (lens[0], position + window, position + window + 1):
            if not position < t <= lens[0]:
                continue
            one = np.array([t] + lens[1:], np.int32)
            rows = q[np.concatenate([[chunks[0] - 1], starts[2:] - 1]).astype(int)]
            ref1 = window_attention(w, cache, rows, one, np.arange(w.S + 1), window, sinks)
            seen = position > t - 1 - window
            _compare(hip_decode_window(w, cache_to_dev(cache), w.block_tables, window, sinks, q=rows, lens=one), ref1,
                     lambda bad: bad[0, heads].all() == seen and bad.sum() == (G if seen else 0), f"decode at {t}, key {position}")


@pytest.mark.parametrize("chunks,lens,window,sinks", CASES)
@pytest.mark.parametrize("H_q,H_k,d", [(16, 8, 128), (10, 2, 64)])
def test_an_infinite_key(oracle_mod, H_q, H_k, d, chunks, lens, window, sinks):
    """No weight where its product with the query is negative, else no number."""
    w = random_workload("window_inf_k", 33, "fp16", H_q, H_k, d, lens)
    q, starts = ragged_rows(w, chunks)
    q[..., 21] = np.where(q[..., 21] == 0, 1, q[..., 21])                    # (0 * inf is none either)
    position = lens[0] - chunks[0] + 20
    cache = oracle_fill(oracle_mod, w)
    _spoil(w, cache, position, np.inf)
    ref = window_attention(w, cache, q, w.context_lens, starts, window, sinks)
    G, last = H_q // H_k, min(chunks[0], 20 + window)
    _compare(hip_prefill_window(w, cache_to_dev(cache), w.block_tables, q, starts, window, sinks), ref,
             lambda bad: 0.2 < bad[20:last, G:2 * G].mean() < 0.8 and bad.sum() == bad[20:last, G:2 * G].sum(), f"{H_q}/{H_k}")

"""GPU: attention through a sliding window with the first tokens visible, decode and chunked prefill, against
the definition in 64 bits.  Every token that no row of a call sees is NaN in the cache, and blocks of such tokens
alone are a block of NaN in the table, so a read of them that reaches a result shows.  Lengths on both sides of
block, group and window borders; windows of one token to more than the context; sinks inside a block, at its end,
beyond the window and beyond the context."""
import numpy as np
import pytest
import torch

import paper_2602_09323_amd as coopt
from gpu_utils import assert_close, cache_to_dev, dev, shape_of
from window_utils import poisoned, ragged_rows, random_workload, seen_keys, window_attention

pytestmark = pytest.mark.gpu

HEADS = [("e4m3", 40, 8, 128), ("e4m3", 4, 4, 64), ("e5m2", 32, 2, 128), ("e5m2", 8, 2, 64), ("fp16", 6, 2, 128),
         ("fp16", 16, 1, 64)]
# (window, sinks)
WINDOWS = [(1, 0), (1, 1), (5, 3), (16, 0), (16, 16), (17, 4), (31, 17), (32, 40), (100, 4), (333, 33), (700, 0), (1 << 30, 7)]
LENS = [1, 2, 0, 15, 16, 17, 18, 31, 32, 33, 49, 64, 96, 115, 116, 117, 118, 333, 400, 704, 705, 1033]


def workspace_for(need, byte=0xFF):
    return torch.full((need,), byte, dtype=torch.uint8, device="cuda") if need else None


def hip_decode_window(w, dcache, tables, window, sinks, q=None, lens=None, stream=None):
    shape = shape_of(w)
    out = torch.full((w.S, w.H_q, w.d), -7.0, dtype=torch.float16, device="cuda")
    ws = workspace_for(coopt.decode_window_workspace_bytes(shape, window, sinks))
    coopt.paged_gqa_decode_window(dev((w.q if q is None else q).view(np.uint16)), *dcache, dev(tables),
                                  dev(w.context_lens if lens is None else lens), window, sinks, out, ws, shape)
    torch.cuda.synchronize()
    return out.cpu().numpy().astype(np.float64)


def hip_prefill_window(w, dcache, tables, q, starts, window, sinks, longest=None):
    shape = shape_of(w)
    out = torch.full(q.shape, -7.0, dtype=torch.float16, device="cuda")
    longest = int(np.diff(starts).max()) if longest is None else longest
    ws = workspace_for(coopt.prefill_window_workspace_bytes(shape, longest, window, sinks))
    coopt.paged_gqa_prefill_chunk_window(dev(q.view(np.uint16)), *dcache, dev(tables), dev(w.context_lens), dev(starts),
                                         int(starts[-1]), longest, window, sinks, out, ws, shape)
    torch.cuda.synchronize()
    return out.cpu().numpy().astype(np.float64)


def hidden_from(w, chunks, window, sinks):
    """hidden(s): tokens that none of sequence s's last chunks[s] rows sees."""
    def hidden(s):
        t, C = int(w.context_lens[s]), int(chunks[s])
        first = max(t - max(C, 1) + 1 - window, 0)
        j = np.arange(t)
        return j[(j >= sinks) & (j < first)]
    return hidden


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("kv,H_q,H_k,d", HEADS)
def test_decode(oracle_mod, kv, H_q, H_k, d, window, sinks):
    w = random_workload("window_decode", 11, kv, H_q, H_k, d, LENS)
    cache, tables = poisoned(oracle_mod, w, hidden_from(w, [1] * w.S, window, sinks))
    ref = window_attention(w, cache, w.q, w.context_lens, np.arange(w.S + 1), window, sinks)
    assert_close(hip_decode_window(w, cache_to_dev(cache), tables, window, sinks), ref, f"window {window} sinks {sinks}")


@pytest.mark.parametrize("lens,window,sinks", [([2500, 1], 2048, 4), ([9000, 4097, 130, 3], 4096, 13),
                                               ([620] * 70 + [5] * 3, 512, 4), ([6000], 512, 4), ([150] * 150, 128, 0)])
@pytest.mark.parametrize("kv,H_q,H_k,d", [("e4m3", 40, 8, 128), ("fp16", 8, 8, 64)])
def test_decode_of_longer_contexts(oracle_mod, kv, H_q, H_k, d, lens, window, sinks):
    """Batches and contexts large enough for every way of cutting the work."""
    w = random_workload("window_long", 12, kv, H_q, H_k, d, lens)
    cache, tables = poisoned(oracle_mod, w, hidden_from(w, [1] * w.S, window, sinks))
    ref = window_attention(w, cache, w.q, w.context_lens, np.arange(w.S + 1), window, sinks)
    assert_close(hip_decode_window(w, cache_to_dev(cache), tables, window, sinks), ref, f"window {window} sinks {sinks}")


@pytest.mark.parametrize("lens,window,sinks", [(LENS, 1, 0), (LENS, 17, 4), (LENS, 333, 33), ([2500, 1, 0, 700], 2048, 4),
                                               ([620] * 70 + [5] * 3, 512, 4)])
@pytest.mark.parametrize("kv,H_q,H_k,d", HEADS)
def test_fused_step(oracle_mod, kv, H_q, H_k, d, lens, window, sinks):
    """The write of the new tokens and the attention in one call: every third sequence's slot is negative (nothing
    written, its last token read from the cache).  Cache bytes as the separate write leaves them."""
    w = random_workload("window_step", 21, kv, H_q, H_k, d, lens)
    cache, tables = poisoned(oracle_mod, w, hidden_from(w, [1] * w.S, window, sinks))
    ref = window_attention(w, cache, w.q, w.context_lens, np.arange(w.S + 1), window, sinks)
    last = np.asarray(w.seq_start[1:]) - 1
    some = [s for s in range(w.S) if lens[s] > 0 and s % 3 != 2]
    slots = np.full(w.S, -1, np.int64)
    slots[some] = w.slots[last[some]]
    new = np.zeros((2, w.S, H_k, d), np.float16)
    new[0, some], new[1, some] = w.k_ctx[last[some]], w.v_ctx[last[some]]
    dcache, shape = cache_to_dev(cache), shape_of(w)
    before = [None if x is None else x.clone() for x in dcache]
    for x in dcache:                                   # the rows that the step brings: not there yet
        if x is not None:
            y = x.view(torch.uint8).view(w.NB, -1)
            for s in some:
                if lens[s] % 16 == 1:                  # the block's first token: the whole block is stale
                    y[int(slots[s]) // 16] = 0x7F
    out = torch.full((w.S, H_q, d), -7.0, dtype=torch.float16, device="cuda")
    ws = workspace_for(coopt.decode_window_workspace_bytes(shape, window, sinks))
    coopt.paged_gqa_decode_window_step(dev(new[0].view(np.uint16)), dev(new[1].view(np.uint16)), dev(slots), dev(w.q.view(np.uint16)),
                                       *dcache, dev(tables), dev(w.context_lens), window, sinks, out, ws, shape)
    torch.cuda.synchronize()
    assert_close(out.cpu().numpy().astype(np.float64), ref, f"step window {window} sinks {sinks}")
    # what the separate write leaves, over the same stale bytes
    want = [None if x is None else x.clone() for x in before]
    for x in want:
        if x is not None:
            y = x.view(torch.uint8).view(w.NB, -1)
            for s in some:
                if lens[s] % 16 == 1:
                    y[int(slots[s]) // 16] = 0x7F
    rows = dev(new[0].view(np.uint16)), dev(new[1].view(np.uint16)), dev(slots)
    if kv == "fp16":
        coopt.kv_cache_write_fp16(*rows, want[0], want[1], shape)
    else:
        coopt.kv_cache_write_fp8(*rows, *want, shape)
    torch.cuda.synchronize()
    for name, a, b in zip(("k_cache", "v_cache", "k_scale", "v_scale"), dcache, want):
        if a is not None:
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), name


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("kv,H_q,H_k,d", HEADS)
def test_prefill(oracle_mod, kv, H_q, H_k, d, window, sinks):
    """Chunks of no rows to more than a window, behind histories of none to many tokens."""
    chunks = [1, 17, 0, 33, 64, 1, 160, 300, 5, 16]
    lens = [1, 17, 40, 50, 64, 333, 161, 700, 600, 1040]
    w = random_workload("window_prefill", 13, kv, H_q, H_k, d, lens)
    q, starts = ragged_rows(w, chunks)
    cache, tables = poisoned(oracle_mod, w, hidden_from(w, chunks, window, sinks))
    ref = window_attention(w, cache, q, w.context_lens, starts, window, sinks)
    got = hip_prefill_window(w, cache_to_dev(cache), tables, q, starts, window, sinks)
    assert_close(got, ref, f"window {window} sinks {sinks}")


@pytest.mark.parametrize("chunks,lens,window,sinks", [([700], [5000], 1024, 4), ([513, 20, 1300], [513, 4020, 1300], 500, 7),
                                                      ([300] * 9, [2300] * 9, 2000, 64), ([77], [3077], 1024, 4)])
@pytest.mark.parametrize("kv,H_q,H_k,d", [("e4m3", 40, 8, 128), ("e5m2", 16, 2, 64), ("fp16", 8, 8, 128)])
def test_prefill_of_longer_chunks(oracle_mod, kv, H_q, H_k, d, chunks, lens, window, sinks):
    w = random_workload("window_chunks", 14, kv, H_q, H_k, d, lens)
    q, starts = ragged_rows(w, chunks)
    cache, tables = poisoned(oracle_mod, w, hidden_from(w, chunks, window, sinks))
    ref = window_attention(w, cache, q, w.context_lens, starts, window, sinks)
    assert_close(hip_prefill_window(w, cache_to_dev(cache), tables, q, starts, window, sinks), ref, f"{chunks} window {window}")


# (chunks, lengths, window, sinks) that between them reach every form of the launch, for every cache and head size: the
# number of wavefronts a tile, whole streams, streams in parts, short chunks (test_window_view.py asks the rule)
FORM_HEADS = [("e4m3", 40, 8, 128), ("e4m3", 32, 8, 64), ("e5m2", 40, 8, 128), ("e5m2", 32, 8, 64), ("fp16", 16, 8, 128), ("fp16", 32, 8, 64)]
FORM_CASES = [([30, 7], [800, 90], 130, 4), ([16], [700], 500, 4), ([16], [2500], 2400, 4), ([16, 16], [4300, 60], 4000, 7),
              ([40] * 10 + [5], [40] * 10 + [5], 16, 0), ([1500, 40], [3500, 2500], 900, 20), ([700], [5000], 4100, 4),
              ([500] * 5, [500] * 5, 33, 4), ([200], [300], 16, 0)]


@pytest.mark.parametrize("chunks,lens,window,sinks", FORM_CASES)
@pytest.mark.parametrize("kv,H_q,H_k,d", FORM_HEADS)
def test_prefill_in_every_form(oracle_mod, kv, H_q, H_k, d, chunks, lens, window, sinks):
    w = random_workload("window_forms", 22, kv, H_q, H_k, d, lens)
    q, starts = ragged_rows(w, chunks)
    cache, tables = poisoned(oracle_mod, w, hidden_from(w, chunks, window, sinks))
    ref = window_attention(w, cache, q, w.context_lens, starts, window, sinks)
    assert_close(hip_prefill_window(w, cache_to_dev(cache), tables, q, starts, window, sinks), ref, f"{chunks[:3]} window {window}")


@pytest.mark.parametrize("kv,H_q,H_k,d", HEADS + [("e4m3", 3, 3, 64), ("fp16", 24, 24, 64)])
def test_mixed_batches(oracle_mod, kv, H_q, H_k, d):
    """A chunk or two among many sequences of one row, of none, or of a few, as a server's step has them: in any order, and
    more of them than a wavefront has lanes, more than lanes squared."""
    rng = np.random.default_rng(23)
    for S, longest, window, sinks in ((70, 200, 64, 4), (200, 130, 33, 0), (5000, 40, 16, 1)):
        if S > 1000 and (H_q, d) != (16, 64):
            continue
        chunks = [int(x) for x in rng.choice([1, 1, 1, 1, 0, 2, 5], size=S)]
        chunks[S // 3], chunks[S - 1], chunks[0] = longest, 1, 0
        lens = [c + int(rng.integers(0, 150 if S < 1000 else 20)) for c in chunks]
        w = random_workload("window_mixed", 24, kv, H_q, H_k, d, lens)
        q, starts = ragged_rows(w, chunks)
        cache, tables = poisoned(oracle_mod, w, hidden_from(w, chunks, window, sinks))
        ref = window_attention(w, cache, q, w.context_lens, starts, window, sinks)
        assert_close(hip_prefill_window(w, cache_to_dev(cache), tables, q, starts, window, sinks), ref, f"{S} sequences")


@pytest.mark.parametrize("kv,H_q,H_k,d", HEADS[:2])
def test_a_window_of_the_whole_context_is_plain_attention(oracle_mod, kv, H_q, H_k, d):
    w = random_workload("window_all", 15, kv, H_q, H_k, d, [700, 33, 1, 512])
    cache, tables = poisoned(oracle_mod, w, lambda s: np.zeros(0, int))
    ref = oracle_mod.paged_gqa_decode(w.q, *cache, tables, w.context_lens, H_q=H_q, H_k=H_k, d=d, B=16, softmax_scale=w.softmax_scale)
    for window in (700, 1 << 20, 0x7fffffff):
        assert_close(hip_decode_window(w, cache_to_dev(cache), tables, window, 0x7fffffff if window == 700 else 0), ref, f"{window}")


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_other_softmax_scales(oracle_mod, scale):
    w = random_workload("window_scale", 16, "e4m3", 10, 2, 128, [700, 33, 130])
    w.softmax_scale = float(np.float32(scale))
    cache, tables = poisoned(oracle_mod, w, hidden_from(w, [1] * 3, 100, 4))
    dcache = cache_to_dev(cache)
    ref = window_attention(w, cache, w.q, w.context_lens, np.arange(4), 100, 4)
    assert_close(hip_decode_window(w, dcache, tables, 100, 4), ref, f"scale {scale}")
    q, starts = ragged_rows(w, [40, 33, 1])
    cache, tables = poisoned(oracle_mod, w, hidden_from(w, [40, 33, 1], 100, 4))
    ref = window_attention(w, cache, q, w.context_lens, starts, 100, 4)
    assert_close(hip_prefill_window(w, cache_to_dev(cache), tables, q, starts, 100, 4), ref, f"prefill scale {scale}")


def test_rows_of_a_chunk_longer_than_announced(oracle_mod):
    """Some heads' rows of the sequence may be left as they were; every other row is right."""
    w = random_workload("window_announced", 17, "e4m3", 10, 2, 128, [200, 90])
    q, starts = ragged_rows(w, [100, 40])
    cache, tables = poisoned(oracle_mod, w, hidden_from(w, [100, 40], 64, 4))
    ref = window_attention(w, cache, q, w.context_lens, starts, 64, 4)
    got = hip_prefill_window(w, cache_to_dev(cache), tables, q, starts, 64, 4, longest=48)
    assert_close(got[100:], ref[100:], "the other sequence")
    left = np.all(got[:100] == -7.0, axis=2)                 # of some heads, as the deal has it
    assert_close(got[:100][~left], ref[:100][~left], "rows that were written")


def test_pool_beyond_2_gib(oracle_mod):
    """Tiles behind the 2 GiB mark are read with 64-bit offsets."""
    NB = 3 << 16
    lens = [300, 1025, 47, 16]
    w = random_workload("window_big", 18, "e4m3", 40, 8, 128, lens)
    cache, tables = poisoned(oracle_mod, w, hidden_from(w, [16] * 4, 200, 4))
    shape = shape_of(w)
    shape.num_blocks = NB
    spread = np.sort(np.random.default_rng(3).permutation(NB)[:w.NB])
    spread[-1] = NB - 1
    at = torch.from_numpy(spread).cuda()
    dcache = []
    for part in cache_to_dev(cache):
        big = torch.zeros((NB, *part.shape[1:]), dtype=part.dtype, device="cuda")
        big[at] = part
        dcache.append(big)
    far = spread[np.maximum(tables, 0)].astype(np.int32)
    q, starts = ragged_rows(w, [16] * 4)
    ref = window_attention(w, cache, q, w.context_lens, starts, 200, 4)
    out = torch.full(q.shape, -7.0, dtype=torch.float16, device="cuda")
    ws = workspace_for(coopt.prefill_window_workspace_bytes(shape, 16, 200, 4))
    coopt.paged_gqa_prefill_chunk_window(dev(q.view(np.uint16)), *dcache, dev(far), dev(w.context_lens), dev(starts), 64, 16, 200, 4,
                                         out, ws, shape)
    torch.cuda.synchronize()
    assert_close(out.cpu().numpy().astype(np.float64), ref, "prefill")
    last = starts[1:] - 1
    ws = workspace_for(coopt.decode_window_workspace_bytes(shape, 200, 4))
    out = torch.full((4, w.H_q, w.d), -7.0, dtype=torch.float16, device="cuda")
    coopt.paged_gqa_decode_window(dev(q[last].view(np.uint16)), *dcache, dev(far), dev(w.context_lens), 200, 4, out, ws, shape)
    torch.cuda.synchronize()
    assert_close(out.cpu().numpy().astype(np.float64), ref[last], "decode")


def test_captured_replays_and_another_stream(oracle_mod):
    """Decode and prefill captured into one graph with a shared workspace each, replayed with eager work between."""
    w = random_workload("window_graph", 19, "e4m3", 40, 8, 128, [700, 33, 1500, 64])
    cache, tables = poisoned(oracle_mod, w, hidden_from(w, [33] * 4, 300, 4))
    dcache, shape = cache_to_dev(cache), shape_of(w)
    q, starts = ragged_rows(w, [33] * 4)
    bt, lens, qs, dq = dev(tables), dev(w.context_lens), dev(starts), dev(q.view(np.uint16))
    one = dev(np.ascontiguousarray(q[starts[1:] - 1]).view(np.uint16))
    ws_d = workspace_for(coopt.decode_window_workspace_bytes(shape, 300, 4))
    ws_p = workspace_for(coopt.prefill_window_workspace_bytes(shape, 33, 300, 4))

    def call(out_d, out_p):
        coopt.paged_gqa_decode_window(one, *dcache, bt, lens, 300, 4, out_d, ws_d, shape)
        coopt.paged_gqa_prefill_chunk_window(dq, *dcache, bt, lens, qs, 132, 33, 300, 4, out_p, ws_p, shape)

    def outs():
        return (torch.full((4, w.H_q, w.d), -7.0, dtype=torch.float16, device="cuda"),
                torch.full(q.shape, -7.0, dtype=torch.float16, device="cuda"))
    eager, kept = outs(), outs()
    call(*eager)
    torch.cuda.synchronize()
    ref = window_attention(w, cache, q, w.context_lens, starts, 300, 4)
    assert_close(eager[1].cpu().numpy().astype(np.float64), ref, "prefill")
    assert_close(eager[0].cpu().numpy().astype(np.float64), ref[starts[1:] - 1], "decode")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            call(*kept)
    for _ in range(3):
        for o in kept:
            o.fill_(-5.0)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(kept, eager):
            assert torch.equal(got, want)
        scratch = outs()
        with torch.cuda.stream(side):
            call(*scratch)
        torch.cuda.synchronize()
        for got, want in zip(scratch, eager):
            assert torch.equal(got, want)


def test_the_reference_hides_what_it_should():
    assert list(seen_keys(9, 3, 2)) == [0, 1, 7, 8, 9]
    assert list(seen_keys(2, 3, 2)) == [0, 1, 2]
    assert list(seen_keys(5, 1, 0)) == [5]

"""GPU: decode over keys that are infinite or NaN, in batches large enough for the balanced form and in the other forms: where a
group of 32 tokens, or all that a window shows of one, has only scores of minus infinity, the row is the one over
the other tokens, as it is in 64 bits; where all of a row's scores are, or one is no number, it is no number."""
import numpy as np
import pytest
import torch

import paper_2602_09323_amd as coopt
import workloads
from gpu_utils import assert_close, cache_to_dev, hip_decode, planned, shape_of
from helpers import oracle_fill
from test_gpu_partitioned import _hip_partitioned
from test_gpu_scheduled import _prepare, _run
from test_gpu_window import hip_decode_window
from window_utils import random_workload, window_attention

pytestmark = pytest.mark.gpu

ELEMENT = 21


def _infinite(w, cache, s, head, positions, value=np.inf):
    """An element of these keys of sequence s (K blocks of fp16: [dim / 8][token][8])."""
    keys = cache[0].reshape(w.NB, w.H_k, w.d // 8, 16, 8)
    for p in positions:
        keys[w.block_tables[s, p // 16], head, ELEMENT // 8, p % 16, ELEMENT % 8] = value


def _signs(w):
    """Every second head's query is negative there, so that an infinite key has no weight for it."""
    w.q[:, :, ELEMENT] = np.where(np.arange(w.H_q) % 2, 1, -1)


def _check(got, ref, what):
    bad = np.isnan(ref).all(axis=2)
    assert np.isfinite(ref[~bad]).all()
    assert np.isnan(got[bad]).all(), f"{what}: rows that are no number"
    assert_close(np.where(bad[..., None], 0.0, got), np.where(bad[..., None], 0.0, ref), what)


def _oracle(oracle, w, cache):
    with np.errstate(invalid="ignore"):
        return oracle.paged_gqa_decode(w.q, *cache, w.block_tables, w.context_lens, H_q=w.H_q, H_k=w.H_k, d=w.d, B=w.B,
                                       softmax_scale=w.softmax_scale)


# sequences, whose pairs are too many for anything but the balanced form; one launch; in parts
@pytest.mark.parametrize("S,extra", [(70, 0), (4, 0), (3, 1000)], ids=["balanced", "one launch", "parts"])
@pytest.mark.parametrize("H_q,H_k,d", [(16, 8, 128), (32, 8, 64)])
def test_through_a_window(oracle_mod, H_q, H_k, d, S, extra):
    """One sink, and a window that begins at the last place of its block: the first 32 tokens of the view show two."""
    window, sinks = 50 + extra, 1
    lens = [97 + extra + 16 * (s % 4) - extra % 16 for s in range(S)]
    lens = [t + (15 - (t - window)) % 16 for t in lens]
    w = random_workload("window_infinite", 51, "fp16", H_q, H_k, d, lens)
    _signs(w)
    cache = oracle_fill(oracle_mod, w)
    for s, t in enumerate(lens):
        assert (t - window) % 16 == 15 and t - window > 32
        _infinite(w, cache, s, 1, [0, t - window])
    _infinite(w, cache, S - 1, 2, [0] + list(range(lens[-1] - window, lens[-1])))         # all that one sees
    _infinite(w, cache, 0, 3, [lens[0] - 3], np.nan)
    _infinite(w, cache, 1, 3, [lens[1] - window - 1], np.nan)                             # seen no more
    ref = window_attention(w, cache, w.q, w.context_lens, np.arange(S + 1), window, sinks)
    G = H_q // H_k
    bad = np.isnan(ref).all(axis=2)
    assert bad[:, G + 1:2 * G:2].all() and not bad[:, G:2 * G:2].any() and bad[S - 1, 2 * G:3 * G].all()
    assert bad[0, 3 * G:4 * G].all() and not bad[1, 3 * G:4 * G].any()
    need = coopt.decode_window_workspace_bytes(shape_of(w), window, sinks)
    assert (need == 0) == (S == 4)
    _check(hip_decode_window(w, cache_to_dev(cache), w.block_tables, window, sinks), ref, f"{S} sequences")


def _whole(oracle_mod, S, H_q=16, H_k=8, d=128):
    lens = [200 + 7 * (s % 5) for s in range(S)]
    w = workloads.make_custom("infinite", seed=52, S=S, H_q=H_q, H_k=H_k, d=d, B=16, NB=sum(-(-t // 16) for t in lens) + 2,
                              context_lens=lens, kv_dtype="fp16")
    _signs(w)
    cache = oracle_fill(oracle_mod, w)
    for s in range(S):
        _infinite(w, cache, s, 1, range(32))                   # a group, at the start of the stream
        _infinite(w, cache, s, 2, range(64, 128))              # groups, and a whole partition of 64 tokens
    _infinite(w, cache, S - 1, 3, range(lens[-1]))             # a whole sequence
    _infinite(w, cache, 0, 3, [70], np.nan)
    ref, G = _oracle(oracle_mod, w, cache), H_q // H_k
    bad = np.isnan(ref).all(axis=2)
    for head in (1, 2):
        assert bad[:, head * G + 1:(head + 1) * G:2].all() and not bad[:, head * G:(head + 1) * G:2].any()
    assert bad[S - 1, 3 * G:4 * G].all() and bad[0, 3 * G:4 * G].all() and not bad[1:S - 1, 3 * G:4 * G].any()
    return w, cache, ref


@pytest.mark.parametrize("plan", [None, {"softmax_reduction": 1}, {"tokens_per_group": 32, "grid_waves": 4096}])
@pytest.mark.parametrize("H_q,H_k,d", [(16, 8, 128), (32, 8, 64)])
def test_balanced(oracle_mod, H_q, H_k, d, plan):
    """Shares that begin with such a group, and shares that hold nothing else (32 tokens each)."""
    w, cache, ref = _whole(oracle_mod, 70, H_q, H_k, d)
    if plan:
        planned.set_plan(**plan)
    dcache = cache_to_dev(cache)
    _check(hip_decode(w, dcache), ref, f"plan {plan}")
    _check(_run(w, dcache, _prepare(w)), ref, f"prepared, plan {plan}")


def test_without_a_workspace(oracle_mod):
    w, cache, ref = _whole(oracle_mod, 70)
    _check(hip_decode(w, cache_to_dev(cache), split=False), ref, "no workspace")


@pytest.mark.parametrize("P", [32, 64, 512])
@pytest.mark.parametrize("waves", [1, 4])
def test_partitions(oracle_mod, P, waves):
    """Partitions that begin with such a group, of nothing else, and wavefronts of a partition that see nothing else."""
    w, cache, ref = _whole(oracle_mod, 6)
    planned.set_plan(waves_per_group=waves)
    out, tmp, ml, es = _hip_partitioned(w, cache_to_dev(cache), P, -(-int(w.context_lens.max()) // P))
    _check(out, ref, f"partitions of {P}")
    if P == 64:                                                # of tokens 64 .. 127, heads that give them no weight
        G = w.H_q // w.H_k
        none = slice(2 * G, 3 * G, 2)
        assert (es[:, none, 1] == 0).all() and (tmp[:, none, 1] == 0).all() and np.isfinite(ml[:, none, 1]).all()

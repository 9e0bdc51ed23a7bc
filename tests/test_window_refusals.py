"""The workspaces of the windowed calls, before any launch (nothing is read through these pointers): missing, too small and
misaligned ones are refused, of shapes that do need one."""
import ctypes

import pytest

from test_abi import _shape, lib  # noqa: F401


def _calls(lib, shape, longest, window, sinks):  # noqa: F811
    one, size, sh = ctypes.c_void_p(16), ctypes.c_size_t, ctypes.byref(shape)
    return {"decode": (lib.coopt_decode_window_workspace_bytes(sh, window, sinks),
                       lambda ws, n: lib.coopt_paged_gqa_decode_window(one, one, one, one, one, one, one, window, sinks, one, ws, size(n), sh, None)),
            "step": (lib.coopt_decode_window_workspace_bytes(sh, window, sinks),
                     lambda ws, n: lib.coopt_paged_gqa_decode_window_step(one, one, one, one, one, one, one, one, one, one, window, sinks, one,
                                                                          ws, size(n), sh, None)),
            "prefill": (lib.coopt_prefill_window_workspace_bytes(sh, longest, window, sinks),
                        lambda ws, n: lib.coopt_paged_gqa_prefill_chunk_window(one, one, one, one, one, one, one, one, shape.num_seqs * longest,
                                                                               longest, window, sinks, one, ws, size(n), sh, None))}


@pytest.mark.parametrize("call", ["decode", "step", "prefill"])
@pytest.mark.parametrize("kv", [0, 1, 2])
def test_workspaces(lib, kv, call):  # noqa: F811
    shape = _shape(num_seqs=64, num_q_heads=8, num_kv_heads=2, head_dim=128, max_blocks_per_seq=2048, kv_dtype=kv)
    need, enter = _calls(lib, shape, 64, 4096, 4)[call]
    assert need > 0
    assert enter(None, 0) == -1 and enter(None, need) == -1
    for at, n in ((16, need - 1), (16, 0), (8, need), (24, need), (17, need)):
        assert enter(ctypes.c_void_p(at), n) == -3, (at, n)


def test_sizes_of_what_is_needed(lib):  # noqa: F811
    """No more for a longer table than the window needs, more for a longer window or more sequences, none for what is refused."""
    def sizes(num_seqs=64, width=2048, window=4096, sinks=4, **fields):
        shape = _shape(num_seqs=num_seqs, num_q_heads=8, num_kv_heads=2, head_dim=128, max_blocks_per_seq=width, kv_dtype=1, **fields)
        return [need for need, _ in _calls(lib, shape, 64, window, sinks).values()]
    base = sizes()
    assert all(n > 0 for n in base) and sizes(width=1 << 20) == base
    assert all(a > b for a, b in zip(sizes(num_seqs=72), base)) and all(a >= b for a, b in zip(sizes(window=8192), base))
    assert sizes(window=0) == sizes(sinks=-1) == sizes(num_seqs=0) == sizes(block_size=32) == [0, 0, 0]

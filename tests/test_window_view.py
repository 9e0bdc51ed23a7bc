"""What a windowed launch takes of a sequence (csrc/window.hpp, compiled here for the CPU), for every small window,
number of sinks, length and number of rows: the view holds every token that a row sees at the place the kernels look
for it, hides the others, has no two blocks in a row without a token in sight, and never names a table entry of a
block that no row sees.  And the host's refusals of the windowed entry points."""
import ctypes
import subprocess
from pathlib import Path

import pytest

import paper_2602_09323_amd as coopt
from test_abi import _shape, lib  # noqa: F401

ROOT = Path(__file__).resolve().parent.parent

SOURCE = r"""
#include <cstdio>
#include <initializer_list>
#define __device__
#define __forceinline__ inline
#include "window.hpp"
using namespace coopt;
int main()
{
    int bad = 0;
    auto fail = [&](const char* what, int w, int s, int t, int rows) {
        if (++bad < 10) printf("%s: window %d sinks %d tokens %d rows %d\n", what, w, s, t, rows);
    };
    for (int window : {1, 2, 15, 16, 17, 30, 31, 32, 33, 47, 48, 100, 400})
        for (int sinks : {0, 1, 4, 15, 16, 17, 31, 32, 33, 64, 300})
            for (int t = 1; t < 260; ++t)
                for (int rows : {1, 2, 16, 40}) {
                    if (rows > t) continue;
                    const Window w{window, sinks};
                    const int first = t - rows + 1 - window;          // of the first row's window
                    const WindowView v = rows == 1 ? WindowView(w, t) : WindowView(w, t, first);
                    auto seen = [&](int j) { return j < sinks || j >= first; };
                    int at = 0;                                      // tokens found so far
                    const int nb = (v.t + 15) / 16;
                    int in_sight = 0;
                    for (int b = 0; b < nb; ++b) {
                        const int real = v.block(b);
                        bool any = false;
                        if (real < 0 || real >= (t + 15) / 16) fail("a block that is none", window, sinks, t, rows);
                        for (int i = 0; i < 16 && 16 * b + i < v.t; ++i) {
                            const int j = 16 * real + i, vj = 16 * b + i;
                            const bool shown = !(vj >= v.lo && vj < v.hi);
                            if (shown != seen(j)) fail("a token", window, sinks, t, rows);
                            at += shown;
                            any = any || shown;
                        }
                        if (!any) fail("a block without a seen token", window, sinks, t, rows);
                        if (b % 2 == 0) in_sight = 0;
                        in_sight += any;
                        if ((b % 2 == 1 || b == nb - 1) && !in_sight) fail("a pair of blocks without one", window, sinks, t, rows);
                    }
                    int want = 0;
                    for (int j = 0; j < t; ++j) want += seen(j);
                    if (at != want) fail("the number of tokens", window, sinks, t, rows);
                    if (v.hi - v.lo > 30) fail("a long gap", window, sinks, t, rows);
                    // the table of a window is as wide as the widest view
                    coopt_shape sh = {1, 1, 1, 64, 16, 1, (t + 15) / 16, 0, 1.0f};
                    const coopt_shape narrow = window_shape(&sh, window_of(&sh, window, sinks), rows);
                    if (nb > narrow.max_blocks_per_seq || narrow.max_blocks_per_seq > sh.max_blocks_per_seq) fail("the width", window, sinks, t, rows);
                }
    return 0;
}
"""


def test_views(tmp_path):
    src, exe = tmp_path / "view.cpp", tmp_path / "view"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", f"-I{ROOT / 'paper_2602_09323_amd' / 'csrc'}", f"-I{ROOT / 'include'}",
                    str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout == ""


TILES = r"""
#include <cstdio>
#include <initializer_list>
#define __device__
#define __forceinline__ inline
using std::max;
using std::min;
template <class T> T wave_uniform(T v) { return v; }
#include "window_tile.hpp"
using namespace coopt;
int main()
{
    // every wavefront's blocks fit its lanes, whatever the rule says, and the workspace is asked for by the same rule
    for (int kv : {0, 1, 2})
        for (int d : {64, 128})
            for (int hk : {1, 2, 7, 8, 40})
                for (int g : {1, 5, 16})
                    for (int seqs : {1, 3, 64, 1 << 16})
                        for (int chunk : {1, 16, 77, 2000})
                            for (int window : {1, 16, 100, 1024, 5000, 1 << 28})
                                for (int sinks : {0, 4, 5000})
                                    for (int width : {1, 70, 1 << 20}) {
                                        const coopt_shape sh = {seqs, hk * g, hk, d, 16, 1, width, kv, 1.0f};
                                        const Window w = window_of(&sh, window, sinks);
                                        int sets = 1;
                                        const int waves = window_tile_waves(&sh, -1, chunk, w, &sets);
                                        if (sets < 1 || sets > 2 || (sets == 2 && (waves != 1 || (kv == 0 && d == 128)))) printf("%d sets\n", sets);
                                        const int groups = (window_shape(&sh, w, 16 * sets).max_blocks_per_seq + 1) / 2;
                                        if (waves < 0 || waves > 4 || (waves & (waves - 1))) printf("%d wavefronts\n", waves);
                                        if (waves && (groups + waves - 1) / waves > kWindowTileGroups) printf("%d groups for %d\n", groups, waves);
                                    }
    return 0;
}
"""

# what the cases of test_gpu_window.py reach: (kv, q heads, kv heads, dim, sequences, longest chunk, table, window, sinks, rows)
FORMS = r"""
int main()
{
    int a[10];
    while (scanf("%d %d %d %d %d %d %d %d %d %d", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6, a + 7, a + 8, a + 9) == 10) {
        const coopt_shape sh = {a[4], a[1], a[2], a[3], 16, 1, a[6], a[0], 1.0f};
        const Window w = window_of(&sh, a[7], a[8]);
        int sets = 1;
        const int waves = window_tile_waves(&sh, a[9], a[5], w, &sets);
        const PrefillLaunchPlan plan(&sh, a[5], true, window_row_tokens(&sh, w));
        if (waves) printf("tile%d%s\n", waves, sets == 2 ? "of32" : "");
        else printf("stream%d%s\n", plan.wg_tiles, plan.parts > 1 ? "parts" : "");
    }
    return 0;
}
"""


def _program(tmp_path, source, name):
    src, exe = tmp_path / f"{name}.cpp", tmp_path / name
    src.write_text("#include <algorithm>\n" + source)
    subprocess.run(["g++", "-std=c++17", "-O1", f"-I{ROOT / 'paper_2602_09323_amd' / 'csrc'}", f"-I{ROOT / 'include'}",
                    str(src), "-o", str(exe)], check=True)
    return str(exe)


def test_the_rule_of_the_tiles(tmp_path):
    assert subprocess.run([_program(tmp_path, TILES, "tiles")], check=True, capture_output=True, text=True).stdout == ""


def test_every_form_has_its_cases(tmp_path):
    import test_gpu_window as cases
    program = _program(tmp_path, TILES[:TILES.index("int main")] + FORMS, "forms")
    kinds = {"fp16": 0, "e4m3": 1, "e5m2": 2}
    lines = []
    for kv, H_q, H_k, d in cases.FORM_HEADS:
        for chunks, lens, window, sinks in cases.FORM_CASES:
            lines.append((kinds[kv], H_q, H_k, d, len(lens), max(chunks), -(-max(lens) // 16), window, sinks, sum(chunks)))
    said = subprocess.run([program], input="\n".join(" ".join(map(str, x)) for x in lines), check=True, capture_output=True,
                          text=True).stdout.split()
    for kv in range(3):
        for d in (64, 128):
            found = {s for s, x in zip(said, lines) if x[0] == kv and x[3] == d}
            assert {"tile1", "tile2", "tile4"} <= found, (kv, d, found)
            assert "tile1of32" in found or (kv == 0 and d == 128), (kv, d, found)
            assert {x[:8] for x in found} >= {"stream16"} and {x[:7] for x in found} >= {"stream8"}, (kv, d, found)
    assert {"stream16", "stream16parts", "stream8parts"} <= set(said)


def test_refusals(lib):  # noqa: F811
    """Before any launch: nothing is read through these pointers."""
    one, size = ctypes.c_void_p(16), ctypes.c_size_t
    sh = _shape(num_seqs=64, max_blocks_per_seq=2048)

    def decode(*, window=100, sinks=4, out=one, ws=None, nbytes=0, shape=sh, q=one, ks=one):
        return lib.coopt_paged_gqa_decode_window(q, one, one, ks, one, one, one, window, sinks, out, ws, size(nbytes),
                                                 ctypes.byref(shape), None)

    def prefill(*, window=100, sinks=4, rows=64, longest=64, ws=None, nbytes=0, shape=sh, qs=one, vs=one):
        return lib.coopt_paged_gqa_prefill_chunk_window(one, one, one, one, vs, one, one, qs, rows, longest, window, sinks, one,
                                                        ws, size(nbytes), ctypes.byref(shape), None)
    for call in (decode, prefill):
        assert call(window=0) == -2 and call(window=-5) == -2 and call(sinks=-1) == -2
        assert call(shape=_shape(head_dim=96)) == -2 and call(shape=_shape(kv_dtype=7)) == -2
        assert call(shape=_shape(num_seqs=0)) == 0
    step = lib.coopt_paged_gqa_decode_window_step
    wide = _shape(num_seqs=64, max_blocks_per_seq=2048)
    need = lib.coopt_decode_window_workspace_bytes(ctypes.byref(wide), 4096, 4)
    for k, v, slots in ((None, one, one), (one, None, one), (one, one, None)):
        assert step(k, v, slots, one, one, one, one, one, one, one, 4096, 4, one, one, size(need), ctypes.byref(wide), None) == -1
    assert step(one, one, one, one, one, one, one, one, one, one, 0, 4, one, one, size(need), ctypes.byref(wide), None) == -2
    assert decode(q=None) == -1 and decode(out=None) == -1 and decode(ks=None) == -1
    assert prefill(qs=None) == -1 and prefill(vs=None) == -1
    assert prefill(rows=-1) == -2 and prefill(longest=-1) == -2 and prefill(rows=0) == 0 and prefill(longest=0) == 0
    # workspaces: none, too small, misaligned
    need = lib.coopt_decode_window_workspace_bytes(ctypes.byref(sh), 4096, 4)
    if need:
        assert decode(window=4096) == -1
        assert decode(window=4096, ws=one, nbytes=need - 1) == -3
        assert decode(window=4096, ws=ctypes.c_void_p(8), nbytes=need) == -3
    need = lib.coopt_prefill_window_workspace_bytes(ctypes.byref(sh), 64, 4096, 4)
    if need:
        assert prefill(window=4096) == -1
        assert prefill(window=4096, ws=one, nbytes=need - 1) == -3
        assert prefill(window=4096, ws=ctypes.c_void_p(8), nbytes=need) == -3
    # sizes: nothing for what is refused, and no more for a longer table than the window needs
    for bytes_of in (lambda s, w, k: lib.coopt_decode_window_workspace_bytes(ctypes.byref(s), w, k),
                     lambda s, w, k: lib.coopt_prefill_window_workspace_bytes(ctypes.byref(s), 64, w, k)):
        assert bytes_of(sh, 0, 4) == 0 and bytes_of(sh, 16, -1) == 0 and bytes_of(_shape(head_dim=96), 16, 0) == 0
        wide = _shape(num_seqs=64, max_blocks_per_seq=1 << 20)
        assert bytes_of(sh, 4096, 4) == bytes_of(wide, 4096, 4)


@pytest.mark.parametrize("call", ["paged_gqa_decode_window", "paged_gqa_prefill_chunk_window"])
def test_the_binding_refuses_host_tensors(lib, call):  # noqa: F811
    import torch
    x = torch.zeros(1 << 16, dtype=torch.uint8)
    args = [x] * 7 + ([100, 4, x, None] if "decode" in call else [x, 64, 64, 100, 4, x, None])
    with pytest.raises(coopt.CooptError, match="not a device tensor"):
        getattr(coopt, call)(*args, _shape())

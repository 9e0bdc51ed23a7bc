"""Which launch the cases of the GPU tests of windowed prefill are, by the rule itself (csrc/window_tile.hpp, compiled here for
the CPU): every form, by its exact name, for every cache and head size, in pools below and beyond 2 GiB; and what the rule
and the workspace have to agree on."""
import subprocess

import test_gpu_window as cases
import test_gpu_window_forms as more
from test_window_view import FORMS, TILES, _program

ALL = {"tile1", "tile2", "tile4", "tile1of32", "stream16", "stream16parts", "stream8", "stream8parts"}
KV = {"fp16": 0, "e4m3": 1, "e5m2": 2}


def _forms(tmp_path, calls):
    """calls: (cache, q heads, KV heads, dim, chunks, lengths, window, sinks)"""
    program = _program(tmp_path, TILES[:TILES.index("int main")] + FORMS, "forms")
    lines = [(KV[kv], H_q, H_k, d, len(lens), max(chunks), -(-max(lens) // 16), window, sinks, sum(chunks))
             for kv, H_q, H_k, d, chunks, lens, window, sinks in calls]
    return subprocess.run([program], input="\n".join(" ".join(map(str, x)) for x in lines), check=True, capture_output=True,
                          text=True).stdout.split()


def _reachable(kv, d):
    return ALL - {"tile1of32"} if (kv, d) == ("fp16", 128) else ALL


def test_every_form_by_name(tmp_path):
    calls = [(kv, H_q, H_k, d, *case) for kv, H_q, H_k, d in cases.FORM_HEADS for case in cases.FORM_CASES]
    calls += [(kv, H_q, H_k, d, *case) for kv, d in more.KINDS for H_q, H_k, *case in more.WHOLE.values()]
    said = _forms(tmp_path, calls)
    for kv, d in more.KINDS:
        assert {s for s, x in zip(said, calls) if (x[0], x[3]) == (kv, d)} >= _reachable(kv, d), (kv, d)


def test_every_form_in_a_large_pool(tmp_path):
    for kv, d in more.KINDS:
        calls = [(kv, H_q, H_k, d, *case) for H_q, H_k, *case in more.BIG_PREFILL.values()]
        assert set(_forms(tmp_path, calls)) >= _reachable(kv, d), (kv, d, dict(zip(more.BIG_PREFILL, _forms(tmp_path, calls))))


KNOWN = r"""
int main()
{
    // A caller asks for a workspace with the longest chunk alone: where that says tiles there is none, so a call of
    // whatever number of rows has to be tiles too (or, of more than a grid holds, whole streams, which take none), and
    // where it says streams what the plan of the call takes fits it.
    for (int kv : {0, 1, 2})
        for (int d : {64, 128})
            for (int hk : {1, 2, 8, 40})
                for (int g : {1, 5, 16})
                    for (int seqs : {1, 3, 64, 1 << 16})
                        for (int chunk : {1, 16, 77, 2000})
                            for (int window : {1, 100, 1024, 5000, 1 << 28})
                                for (int sinks : {0, 5000})
                                    for (int width : {1, 70, 1 << 20}) {
                                        const coopt_shape sh = {seqs, hk * g, hk, d, 16, 1, width, kv, 1.0f};
                                        const Window w = window_of(&sh, window, sinks);
                                        const long long all = (long long)seqs * chunk;
                                        const int announced = window_tile_waves(&sh, -1, chunk, w);
                                        const size_t need = announced > 0 ? 0 : PrefillLaunchPlan(&sh, chunk, true, window_row_tokens(&sh, w)).workspace_bytes(&sh);
                                        for (long long rows : {1LL, (all + 3) / 4, all - 1, all, all + 100}) {
                                            if (rows < 1) continue;
                                            int sets = 1;
                                            const int waves = window_tile_waves(&sh, rows, chunk, w, &sets);
                                            const long long most = window_tiles(&sh, std::min(rows, all), chunk, 16 * window_tile_sets(&sh));
                                            if (announced > 0 && waves == 0 && most <= kMaxWorkgroups) printf("tiles announced, none of %lld rows\n", rows);
                                            if (waves == 0 && PrefillLaunchPlan(&sh, chunk, need > 0, window_row_tokens(&sh, w)).workspace_bytes(&sh) > need)
                                                printf("a larger workspace of %lld rows\n", rows);
                                        }
                                    }
    return 0;
}
"""


def test_no_call_needs_what_was_not_announced(tmp_path):
    program = _program(tmp_path, TILES[:TILES.index("int main")] + KNOWN, "known")
    assert subprocess.run([program], check=True, capture_output=True, text=True).stdout == ""

"""GPU: the native entry points of the windowed calls and of the block operators take what the binding's Python path
takes, with the same results, and refuse what it refuses, with the same message."""
import pytest
import torch

import paper_2602_09323_amd as coopt
from paper_2602_09323_amd import binding

pytestmark = pytest.mark.gpu

S, HQ, HK, D, NB, WIDTH = 3, 8, 2, 64, 40, 12


def _state(kv):
    g = torch.Generator(device="cuda").manual_seed(5)
    shape = coopt.Shape(S, HQ, HK, D, 16, NB, WIDTH, kv, 0.125)
    code = 2 if kv == coopt.COOPT_KV_FP16 else 1

    def ints(*x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")
    a = {"kc": torch.randint(0, 100, (NB, HK, 16 * D * code), dtype=torch.uint8, device="cuda", generator=g),
         "vc": torch.randint(0, 100, (NB, HK, 16 * D * code), dtype=torch.uint8, device="cuda", generator=g),
         "ks": torch.rand(NB, HK, 16, device="cuda", generator=g) if code == 1 else None,
         "vs": torch.rand(NB, HK, 16, device="cuda", generator=g) if code == 1 else None,
         "q": torch.randn(7, HQ, D, device="cuda", generator=g).half(),
         "new": torch.randn(S, HK, D, device="cuda", generator=g).half(),
         "bt": torch.arange(S * WIDTH, dtype=torch.int32, device="cuda").view(S, WIDTH),
         "cl": ints(100, 20, 0), "starts": ints(0, 5, 7, 7), "out": torch.zeros(7, HQ, D, dtype=torch.float16, device="cuda"),
         "newslots": torch.tensor([6 * 16 + 3, WIDTH * 16 + 16 + 3, -1], device="cuda"),
         "refs": torch.zeros(NB, dtype=torch.int32, device="cuda"), "map": torch.zeros(2, dtype=torch.int32, device="cuda"),
         "slots": torch.zeros(9, dtype=torch.int64, device="cuda"), "result": ints(-9), "copies": torch.zeros(NB // 2, 2, dtype=torch.int32, device="cuda"),
         "some": ints(1, -1), "parents": ints(0, 1), "children": ints(2, -1),
         "bws": torch.empty(coopt.kv_blocks_workspace_bytes(shape), dtype=torch.uint8, device="cuda")}
    a["kcs"], a["vcs"] = [a["kc"], a["kc"].clone()], [a["vc"], a["vc"].clone()]
    a["kss"], a["vss"] = ([a["ks"], a["ks"].clone()], [a["vs"], a["vs"].clone()]) if code == 1 else (None, None)
    for name, need in (("ws", coopt.decode_window_workspace_bytes(shape, 64, 4)),
                       ("pws", coopt.prefill_window_workspace_bytes(shape, 5, 64, 4))):
        a[name] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    coopt.kv_blocks_init(a["bt"], a["cl"], a["refs"], a["map"], shape)
    return a, shape


CALLS = [("paged_gqa_decode_window", "q kc vc ks vs bt cl 64 4 out ws"),
         ("paged_gqa_decode_window_step", "new new newslots q kc vc ks vs bt cl 64 4 out ws"),
         ("paged_gqa_prefill_chunk_window", "q kc vc ks vs bt cl starts 7 5 64 4 out pws"),
         ("kv_blocks_fork", "parents children bt cl refs map copies result bws"),
         ("kv_cache_copy_blocks", "kcs vcs kss vss copies result"),
         ("kv_cache_copy_blocks", "kc vc ks vs copies none"),
         ("kv_blocks_reserve", "starts 9 bt cl refs map slots result bws"),
         ("kv_blocks_reserve", "none 9 bt cl refs map slots result bws"),
         ("kv_blocks_free", "some bt cl refs map"),
         ("kv_blocks_free_outside_window", "bt cl refs map 64 4"),
         ("kv_blocks_compact", "bt cl refs map copies result bws"),
         ("kv_cache_copy_blocks", "kcs vcs kss vss copies result")]


def _args(names, a):
    return [int(n) if n.isdigit() else None if n == "none" else a[n] for n in names.split()]


@pytest.mark.parametrize("kv", [coopt.COOPT_KV_E4M3, coopt.COOPT_KV_FP16], ids=["e4m3", "fp16"])
def test_native_and_python_path_agree(kv, monkeypatch):
    coopt.load_library()
    native = binding._fast()
    assert native is not None, "the native part is not built"
    results = []
    for path in (native, False):
        monkeypatch.setattr(binding, "_native", path)
        a, shape = _state(kv)
        got = []
        for name, names in CALLS:
            getattr(coopt, name)(*_args(names, a), shape)
            for key, t in a.items():
                if key not in ("ws", "pws", "bws"):            # (scratch)
                    got += [x.clone() for x in (t if isinstance(t, list) else [t]) if x is not None]
        torch.cuda.synchronize()
        results.append(got)
    assert len(results[0]) == len(results[1])
    for x, y in zip(*results):
        assert x.shape == y.shape and torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_the_native_part_takes_them(monkeypatch):
    """(not declining, which would leave every call to the slower path)"""
    coopt.load_library()
    assert binding._fast() is not None
    a, shape = _state(coopt.COOPT_KV_E4M3)
    monkeypatch.setattr(binding, "_sizes", lambda *_: pytest.fail("left to Python"))
    for name, names in CALLS:
        getattr(coopt, name)(*_args(names, a), shape)
    torch.cuda.synchronize()


@pytest.mark.parametrize("kv", [coopt.COOPT_KV_E4M3, coopt.COOPT_KV_FP16], ids=["e4m3", "fp16"])
def test_both_refuse_the_same(kv, monkeypatch):
    """Every tensor argument in turn missing, on the host, strided, of another type, too small."""
    coopt.load_library()
    native, refused = binding._fast(), 0
    a, shape = _state(kv)
    for name, names in CALLS:
        args = _args(names, a)
        for i, t in enumerate(args):
            one = t[1] if isinstance(t, list) else t
            if not isinstance(one, torch.Tensor):
                continue
            wide = torch.stack([one, one], dim=-1)[..., 0]
            other = one.double() if one.dtype != torch.uint8 else one[:1]
            for bad in (None, one.cpu(), wide, other, one.flatten()[:0]):
                said = []
                bad = [t[0], bad] if isinstance(t, list) else bad
                for path in (native, False):
                    monkeypatch.setattr(binding, "_native", path)
                    try:
                        getattr(coopt, name)(*args[:i], bad, *args[i + 1:], shape)
                        said.append("taken")
                    except Exception as e:  # noqa: BLE001
                        said.append(f"{type(e).__name__}: {e}")
                torch.cuda.synchronize()
                assert said[0] == said[1], (name, i, said)
                refused += said[0] != "taken"
    assert refused > 150


def test_layers_of_different_numbers(monkeypatch):
    a, shape = _state(coopt.COOPT_KV_E4M3)
    for path in (binding._fast(), False):
        monkeypatch.setattr(binding, "_native", path)
        with pytest.raises(coopt.CooptError, match="v_caches: 1 layers, expected 2"):
            coopt.kv_cache_copy_blocks(a["kcs"], a["vcs"][:1], a["kss"], a["vss"], a["copies"], None, shape)
        with pytest.raises(coopt.CooptError, match="k_scales"):
            coopt.kv_cache_copy_blocks(a["kcs"], a["vcs"], None, a["vss"], a["copies"], None, shape)
        with pytest.raises(coopt.CooptError, match="k_scales: 1 layers, expected 2"):
            coopt.kv_cache_copy_blocks(a["kcs"], a["vcs"], a["kss"][:1], a["vss"], a["copies"], None, shape)

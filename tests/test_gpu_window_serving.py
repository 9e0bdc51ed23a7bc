"""GPU: the windowed calls and the block operators together, as a server uses them: prompts in chunks, steps (fused and as
separate calls), samples that go on from one prompt, ends, blocks behind the window given back and taken again by
others, the pool compacted, in a pool with little room to spare and two layers.  Every output row is held to attention in
64 bits over the tokens that the sequence was given, quantised by the rule of the write."""
import numpy as np
import pytest
import torch

import paper_2602_09323_amd as coopt
from gpu_utils import assert_close

pytestmark = pytest.mark.gpu

S, WIDTH, WINDOW, SINKS, LAYERS = 10, 24, 70, 20, 2


def stored(x, kv):
    """What the cache gives back for fp16 rows [n, H, d], in 64 bits."""
    if kv == coopt.COOPT_KV_FP16:
        return x.double()
    code, top = (torch.float8_e4m3fn, 448.0) if kv == coopt.COOPT_KV_E4M3 else (torch.float8_e5m2, 57344.0)
    # (on the CPU: two correctly rounded divisions, which torch's division by a number is not on a GPU)
    x = x.float().cpu().numpy()
    scale = np.abs(x).max(axis=-1, keepdims=True) / np.float32(top)
    codes = torch.from_numpy(np.clip(x / scale, -top, top)).to(code)
    return (codes.double() * torch.from_numpy(scale).double()).cuda()


class Server:
    def __init__(self, kv, H_q, H_k, d, NB, seed):
        self.shape = coopt.Shape(S, H_q, H_k, d, 16, NB, WIDTH, kv, d ** -0.5)
        self.kv, self.H_q, self.H_k, self.d = kv, H_q, H_k, d
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        es = 2 if kv == coopt.COOPT_KV_FP16 else 1
        def pools(n):
            return [torch.full((NB, H_k, n), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(LAYERS)]
        self.k, self.v = pools(16 * d * es), pools(16 * d * es)
        self.ks, self.vs = (pools(64), pools(64)) if es == 1 else (None, None)
        self.tables = torch.full((S, WIDTH), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(S, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(NB, dtype=torch.int32, device="cuda")
        self.map = torch.zeros((NB + 31) // 32, dtype=torch.int32, device="cuda")
        self.result = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws = torch.empty(coopt.kv_blocks_workspace_bytes(self.shape), dtype=torch.uint8, device="cuda")
        self.copies = torch.zeros((NB, 2), dtype=torch.int32, device="cuda")
        coopt.kv_blocks_init(*self.state, self.shape)
        self.given = [[[] for _ in range(S)] for _ in range(LAYERS)]          # (k, v) of every token, as stored
        self.worst = 0.0

    @property
    def state(self):
        return self.tables, self.lens, self.refs, self.map

    def cache(self, layer):
        return self.k[layer], self.v[layer], *((self.ks[layer], self.vs[layer]) if self.ks else (None, None))

    def rows(self, n, heads):
        return torch.randn((n, heads, self.d), generator=self.gen, device="cuda").half()

    def write(self, layer, k, v, slots):
        if self.kv == coopt.COOPT_KV_FP16:
            coopt.kv_cache_write_fp16(k, v, slots, *self.cache(layer)[:2], self.shape)
        elif self.kv == coopt.COOPT_KV_E4M3:
            coopt.kv_cache_write_fp8(k, v, slots, *self.cache(layer), self.shape)
        else:
            coopt.kv_cache_write_fp8_scaled(k, v, slots, *self.cache(layer), self.shape, coopt.COOPT_SCALE_TOKEN)

    def remember(self, layer, k, v, owner):
        sk, sv = stored(k, self.kv), stored(v, self.kv)
        for i, s in enumerate(owner):
            if s >= 0:
                self.given[layer][s].append((sk[i], sv[i]))

    def check(self, layer, q, out, owner, what):
        """owner[i]: the sequence of row i (-1: none); a sequence's rows are its last tokens."""
        total = {s: sum(1 for o in owner if o == s) for s in set(owner)}
        seen = {s: 0 for s in total}
        want = torch.zeros(out.shape, dtype=torch.float64, device="cuda")
        G = self.H_q // self.H_k
        for i, s in enumerate(owner):
            if s < 0:
                continue
            given = self.given[layer][s]
            p = len(given) - total[s] + seen[s]
            seen[s] += 1
            keys = [j for j in range(p + 1) if j > p - WINDOW or j < SINKS]
            K, V = (torch.stack([given[j][x] for j in keys]) for x in (0, 1))       # [n, H, d]
            for h in range(self.H_q):
                z = (K[:, h // G] * q[i, h].double()).sum(-1) * self.shape.softmax_scale
                want[i, h] = (torch.softmax(z, 0)[:, None] * V[:, h // G]).sum(0)
        self.worst = max(self.worst, assert_close(out.double().cpu().numpy(), want.cpu().numpy(), what))

    def prompts(self, chunks, what):
        owner = [s for s, n in enumerate(chunks) for _ in range(n)]
        starts = torch.tensor(np.concatenate([[0], np.cumsum(chunks)]), dtype=torch.int32, device="cuda")
        slots = torch.full((len(owner),), -1, dtype=torch.int64, device="cuda")
        coopt.kv_blocks_reserve(starts, len(owner), *self.state, slots, self.result, self.ws, self.shape)
        if int(self.result):
            assert bool((slots == -1).all())
            return False
        for layer in range(LAYERS):
            k, v, q = self.rows(len(owner), self.H_k), self.rows(len(owner), self.H_k), self.rows(len(owner), self.H_q)
            self.write(layer, k, v, slots)
            self.remember(layer, k, v, owner)
            out = torch.full_like(q, -7.0)
            need = coopt.prefill_window_workspace_bytes(self.shape, max(chunks), WINDOW, SINKS)
            ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
            coopt.paged_gqa_prefill_chunk_window(q, *self.cache(layer), self.tables, self.lens, starts, len(owner), max(chunks),
                                                 WINDOW, SINKS, out, ws, self.shape)
            self.check(layer, q, out, owner, f"{what}, layer {layer}")
        return True

    def step(self, what):
        before = self.lens.tolist()
        slots = torch.full((S,), -5, dtype=torch.int64, device="cuda")
        coopt.kv_blocks_reserve(None, S, *self.state, slots, self.result, self.ws, self.shape)
        if int(self.result):
            return False
        owner = [s if t > 0 else -1 for s, t in enumerate(before)]
        need = coopt.decode_window_workspace_bytes(self.shape, WINDOW, SINKS)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        for layer in range(LAYERS):
            k, v, q = self.rows(S, self.H_k), self.rows(S, self.H_k), self.rows(S, self.H_q)
            out = torch.full_like(q, -7.0)
            where = self.tables, self.lens, WINDOW, SINKS, out, ws, self.shape
            if layer:
                self.write(layer, k, v, slots)
                coopt.paged_gqa_decode_window(q, *self.cache(layer), *where)
            else:
                coopt.paged_gqa_decode_window_step(k, v, slots, q, *self.cache(layer), *where)
            self.remember(layer, k, v, owner)
            self.check(layer, q, out, owner, f"{what}, layer {layer}")
        return True

    def copy(self, count):
        coopt.kv_cache_copy_blocks(self.k, self.v, self.ks, self.vs, self.copies, count, self.shape)

    def fork(self, parents, children):
        ints = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (parents, children)]
        copies = torch.empty((len(parents), 2), dtype=torch.int32, device="cuda")
        coopt.kv_blocks_fork(*ints, *self.state, copies, self.result, self.ws, self.shape)
        coopt.kv_cache_copy_blocks(self.k, self.v, self.ks, self.vs, copies, None, self.shape)
        if int(self.result):
            return False
        for layer in range(LAYERS):
            for p, c in zip(parents, children):
                self.given[layer][c] = list(self.given[layer][p])
        return True

    def end(self, seqs):
        coopt.kv_blocks_free(torch.tensor(seqs, dtype=torch.int32, device="cuda"), *self.state, self.shape)
        for layer in range(LAYERS):
            for s in seqs:
                self.given[layer][s] = []

    def trim(self):
        coopt.kv_blocks_free_outside_window(*self.state, WINDOW, SINKS, self.shape)

    def compact(self):
        coopt.kv_blocks_compact(*self.state, self.copies[:self.shape.num_blocks // 2], self.result, self.ws, self.shape)
        self.copy(self.result)


@pytest.mark.parametrize("kv,H_q,H_k,d,NB", [(coopt.COOPT_KV_E4M3, 4, 2, 64, 70), (coopt.COOPT_KV_FP16, 3, 3, 64, 61),
                                             (coopt.COOPT_KV_E5M2, 5, 1, 128, 83)], ids=["e4m3", "fp16", "e5m2"])
def test_a_servers_life(kv, H_q, H_k, d, NB):
    rng = np.random.default_rng(7 + NB)
    server = Server(kv, H_q, H_k, d, NB, 3)
    did = {"prompts": 0, "step": 0, "fork": 0, "compact": 0, "refused": 0}
    assert server.prompts([130, 0, 37, 0, 16, 0, 0, 1, 0, 0], "first prompts")
    for n in range(30):
        lens = server.lens.tolist()
        idle, busy = [s for s in range(S) if lens[s] == 0], [s for s in range(S) if 0 < lens[s] < WIDTH * 16 - 40]
        kind = rng.integers(0, 8)
        if kind == 0 and idle:
            chunks = [0] * S
            for s in list(idle[:2]) + list(busy[:1]):
                chunks[s] = int(rng.integers(1, 90))
            ok, name = server.prompts(chunks, f"prompts at {n}"), "prompts"
        elif kind == 1 and idle and busy:
            k = int(rng.integers(1, len(idle) + 1))
            ok, name = server.fork([int(x) for x in rng.choice(busy, k)], [int(x) for x in rng.permutation(idle)[:k]]), "fork"
        elif kind == 2:
            server.compact()
            ok, name = True, "compact"
        else:
            over = [s for s in range(S) if lens[s] >= WIDTH * 16 - 2]
            if over:
                server.end(over)
            ok, name = server.step(f"step at {n}"), "step"
        server.trim()
        if ok:
            did[name] += 1
        else:                                     # no room: the longest sequence ends
            did["refused"] += 1
            server.end([int(np.argmax(lens))])
    assert did["prompts"] and did["step"] > 5 and did["fork"] and did["compact"], did
    # the counts and the map are what the tables say
    refs, free = server.refs.clone(), server.map.clone()
    coopt.kv_blocks_init(*server.state, server.shape)
    assert torch.equal(refs, server.refs) and torch.equal(free, server.map)
    server.end(list(range(S)))
    assert int(server.refs.abs().sum()) == 0

"""GPU: the operators on the pool's blocks against a model of lists and loops, every table entry, length, reference
count, map word, slot and pair exactly, and what they must leave alone left alone: entries that no sequence holds are
filled with numbers that name no block."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2602_09323_amd as coopt
from blocks_model import Pool, ceil

pytestmark = pytest.mark.gpu

GARBAGE = [-7, 1 << 30, -(1 << 31), 0x7FFFFFFF]


def make(seed, S, NB, width, lens, kv_heads=2, dim=64, kv=coopt.COOPT_KV_E4M3, shared=0):
    """A pool whose sequences hold random blocks; with `shared`, every second sequence's first blocks are the one's
    before it."""
    rng = np.random.default_rng(seed)
    tables = rng.choice(GARBAGE, size=(S, width)).astype(np.int64)
    perm, at = rng.permutation(NB), 0
    for s, t in enumerate(lens):
        n, first = ceil(t), 0
        if shared and s % 2:
            first = min(shared, n, lens[s - 1] // 16)
            tables[s, :first] = tables[s - 1, :first]
        tables[s, first:n] = perm[at:at + n - first]
        at += n - first
        assert at <= NB
    shape = coopt.Shape(S, kv_heads, kv_heads, dim, 16, NB, width, kv, 0.125)
    return Pool(tables, lens, NB), Device(tables, lens, shape)


class Device:
    def __init__(self, tables, lens, shape):
        self.shape = shape
        self.tables = torch.from_numpy(tables.astype(np.int32)).cuda()
        self.lens = torch.tensor(np.asarray(lens), dtype=torch.int32).cuda()
        self.refs = torch.full((shape.num_blocks,), -99, dtype=torch.int32, device="cuda")
        self.free = torch.full((ceil(shape.num_blocks, 32),), -1, dtype=torch.int32, device="cuda")
        self.ws = torch.full((coopt.kv_blocks_workspace_bytes(shape),), 0xEE, dtype=torch.uint8, device="cuda")
        self.result = torch.full((1,), -55, dtype=torch.int32, device="cuda")
        coopt.kv_blocks_init(*self.state, shape)

    @property
    def state(self):
        return self.tables, self.lens, self.refs, self.free

    def check(self, pool, what):
        torch.cuda.synchronize()
        assert np.array_equal(self.tables.cpu().numpy(), pool.tables), f"{what}: tables"
        assert self.lens.cpu().tolist() == pool.lens, f"{what}: lengths"
        assert self.refs.cpu().tolist() == pool.refs, f"{what}: references"
        assert np.array_equal(self.free.cpu().numpy().view(np.uint32), pool.free_map()), f"{what}: map"

    def reserve(self, pool, starts, num_rows, what="reserve"):
        before = np.full(num_rows, -77, np.int64)
        slots = torch.from_numpy(before).cuda()
        want, want_slots = pool.reserve(starts, num_rows, before)
        qs = None if starts is None else torch.tensor(np.asarray(starts), dtype=torch.int32).cuda()
        coopt.kv_blocks_reserve(qs, num_rows, *self.state, slots, self.result, self.ws, self.shape)
        self.check(pool, what)
        assert int(self.result) == want, what
        assert np.array_equal(slots.cpu().numpy(), want_slots), f"{what}: slots"
        return want

    def fork(self, pool, parents, children, what="fork"):
        copies = torch.full((len(parents), 2), -66, dtype=torch.int32, device="cuda")
        want, want_copies = pool.fork(parents, children)
        lists = [torch.tensor(np.asarray(x), dtype=torch.int32).cuda() for x in (parents, children)]
        coopt.kv_blocks_fork(*lists, *self.state, copies, self.result, self.ws, self.shape)
        self.check(pool, what)
        assert int(self.result) == want, what
        assert np.array_equal(copies.cpu().numpy(), want_copies), f"{what}: copies"
        return copies

    def free_seqs(self, pool, seqs, what="free"):
        pool.free(seqs)
        coopt.kv_blocks_free(torch.tensor(np.asarray(seqs), dtype=torch.int32).cuda(), *self.state, self.shape)
        self.check(pool, what)

    def outside(self, pool, window, sinks):
        pool.free_outside_window(window, sinks)
        coopt.kv_blocks_free_outside_window(*self.state, window, sinks, self.shape)
        self.check(pool, f"outside the window of {window}, {sinks} sinks")

    def compact(self, pool):
        want = pool.compact()
        copies = torch.full((max(pool.nb // 2, 1), 2), -66, dtype=torch.int32, device="cuda")
        count = torch.full((1,), -5, dtype=torch.int32, device="cuda")
        coopt.kv_blocks_compact(*self.state, copies, count, self.ws, self.shape)
        self.check(pool, "compact")
        assert int(count) == len(want)
        got = copies.cpu().numpy()
        assert [tuple(x) for x in got[:len(want)]] == want
        assert (got[len(want):] == -66).all()
        return copies, count


@pytest.mark.parametrize("S,NB,width,most,shared", [(1, 1, 1, 16, 0), (3, 33, 9, 100, 2), (40, 700, 30, 450, 3), (7, 64, 40, 140, 0),
                                                    (1500, 4001, 5, 40, 1), (5, 9000, 2500, 28000, 7)])
def test_init_and_free(S, NB, width, most, shared):
    rng = np.random.default_rng(NB)
    lens = [min(int(x), width * 16) for x in rng.integers(0, most, size=S)]
    pool, dev = make(1, S, NB, width, lens, shared=shared)
    dev.check(pool, "init")
    seqs = [int(s) for s in rng.permutation(S)[:max(S // 2, 1)]]
    dev.free_seqs(pool, seqs + seqs[:1] + [-1, S, 1 << 30, -(1 << 31)])
    dev.free_seqs(pool, seqs, "freed again")
    dev.free_seqs(pool, list(range(S)), "all")
    assert len(pool.free_blocks()) == NB


@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 16), (17, 3), (100, 4), (1000, 40), (1 << 30, 0), (5, 1 << 30), (200, 0)])
def test_outside_a_window(window, sinks):
    lens = [0, 1, 16, 17, 33, 100, 116, 117, 500, 2000, 2064, 4800]
    pool, dev = make(2, len(lens), 1000, 300, lens, shared=4)
    dev.outside(pool, window, sinks)
    dev.outside(pool, window, sinks)
    for step in range(20):                                     # growing sequences: what each step leaves behind
        dev.reserve(pool, None, len(lens)) if step % 4 else dev.reserve(pool, [0] + list(np.cumsum([min(37, 4800 - t) for t in pool.lens])), 600)
        dev.outside(pool, window, sinks)


@pytest.mark.parametrize("S,NB,width,most", [(1, 3, 2, 30), (13, 400, 40, 300), (1024, 3000, 6, 60), (2500, 9000, 6, 60)])
def test_reserve(S, NB, width, most):
    rng = np.random.default_rng(S)
    lens = [int(x) for x in rng.integers(0, min(most, width * 16 - 3), size=S)]
    pool, dev = make(3, S, NB, width, lens)
    assert dev.reserve(pool, None, S + 3, "one each") == 0
    chunks = [int(rng.integers(0, width * 16 - t + 1)) if rng.random() < 0.3 else min(1, width * 16 - t) for t in pool.lens]
    starts = [0] + list(np.cumsum(chunks))
    dev.reserve(pool, starts, int(starts[-1]) + 5, "chunks")


def test_reserve_of_whole_prompts():
    """More rows than one workgroup gives slots to, more new blocks than it keeps in LDS."""
    chunks = [70000, 0, 17, 5000, 1, 3333]
    pool, dev = make(4, 6, 6000, 4400, [3, 0, 16, 0, 40, 15])
    assert dev.reserve(pool, [0] + list(np.cumsum(chunks)), sum(chunks)) == 0
    assert dev.reserve(pool, [0] + list(np.cumsum(chunks)), sum(chunks), "pool too small or row too short") != 0
    dev.free_seqs(pool, [0, 3])
    assert dev.reserve(pool, [0, 0, 40, 40, 40, 40, 40], 5000, "behind freed ones") == 0


def test_reserve_refusals():
    """Nothing changes and the slots leave everything out."""
    pool, dev = make(5, 4, 40, 10, [100, 0, 159, 16])
    assert dev.reserve(pool, [0, 400, 400, 400, 400], 400) == -1              # a row too short
    assert dev.reserve(pool, [0, 0, 0, 2, 2], 2) == -1
    assert dev.reserve(pool, [0, 1, 0, 1, 1], 5) == -1                        # not increasing
    assert dev.reserve(pool, [0, 1, 1, 1, 9], 5) == -1                        # more rows than announced
    assert dev.reserve(pool, [1, 1, 1, 1, 2], 5) == -1                        # not from 0
    assert dev.reserve(pool, [0, 60, 150, 150, 290], 300) == 0
    pool, dev = make(6, 2, 10, 100, [20, 0])
    assert dev.reserve(pool, [0, 0, 129], 129) == 1                           # 9 blocks, 8 free
    assert dev.reserve(pool, [0, 1000, 1500], 5000) == ceil(1020) - 2 + ceil(500) - 8
    assert dev.reserve(pool, [0, 12, 140], 140) == 0 and not pool.free_blocks()
    assert dev.reserve(pool, None, 2) == 2
    dev.free_seqs(pool, [1])
    assert dev.reserve(pool, None, 2) == 0


def test_fork():
    lens = [100, 32, 0, 1, 0, 0, 0, 0, 0, 16, 0, 0]
    pool, dev = make(7, len(lens), 60, 12, lens, shared=1)
    dev.fork(pool, [0, 0, 1, 3, 9, -1, 2], [2, 4, 5, 6, 7, 8, 8])              # (the last: a parent that is a child here)
    assert int(dev.result) == 0
    dev.fork(pool, [0, 4], [10, 11])
    assert int(dev.result) == 0
    for parents, children in [([0], [0]), ([0], [1]), ([0, 1], [8, 8]), ([12], [8]), ([0], [12]), ([1 << 30, 0], [8, 8]),
                              ([0, 1, 3], [8, 0, 8])]:
        dev.fork(pool, parents, children, f"refused {parents} {children}")
        assert int(dev.result) == -1
    dev.fork(pool, [-1, -5], [3, 1 << 30], "none")
    dev.fork(pool, [], [], "empty")
    dev.free_seqs(pool, [0, 2])
    dev.outside(pool, 20, 16)
    dev.fork(pool, [4], [0], "of a sequence with blocks behind its window")
    assert int(dev.result) == 0


def test_no_sequences_and_no_forks():
    """What is then not needed may be NULL, and nothing is read through it."""
    lib, none = coopt.load_library(), ctypes.c_void_p(None)
    shape = coopt.Shape(3, 2, 2, 64, 16, 4000, 10, coopt.COOPT_KV_E4M3, 0.125)
    ws = torch.empty(coopt.kv_blocks_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    result = torch.tensor([7, 7], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    ptr = [ctypes.c_void_p(t.data_ptr()) for t in (ws, result, result[1:], starts[1:])]

    def reserve(starts_at, rows):
        shape.num_seqs = 0
        assert lib.coopt_kv_blocks_reserve(starts_at, rows, none, none, none, none, none, ptr[1], ptr[0],
                                           ctypes.c_size_t(ws.numel()), ctypes.byref(shape), stream) == 0
        return int(result[0])
    assert reserve(none, 0) == 0 and reserve(none, 9) == 0 and reserve(none, 9000) == 0
    assert reserve(ptr[3], 9) == -1 and reserve(ptr[3], 9000) == -1                          # (does not begin at 0)
    shape.num_seqs = 3
    assert lib.coopt_kv_blocks_fork(none, none, 0, none, none, none, none, none, ptr[2], ptr[0],
                                    ctypes.c_size_t(ws.numel()), ctypes.byref(shape), stream) == 0
    assert int(result[1]) == 0


def test_fork_without_room():
    pool, dev = make(8, 12, 8, 8, [100] + [0] * 11)
    dev.fork(pool, [0, 0], [1, 2], "two of one")
    assert int(dev.result) == 1
    dev.fork(pool, [0], [5])
    assert int(dev.result) == 0 and not pool.free_blocks()


def test_many_forks():
    """More than a workgroup's threads, and more new blocks than LDS keeps."""
    S = 6000
    pool, dev = make(9, S, 9000, 40, [600, 33, 500] + [0] * (S - 3))
    rng = np.random.default_rng(1)
    dev.fork(pool, [int(x) for x in rng.integers(0, 3, size=S - 3)], [int(x) for x in 3 + rng.permutation(S - 3)])
    assert int(dev.result) == 0
    dev.reserve(pool, None, S)
    dev.free_seqs(pool, list(range(0, S, 2)))
    dev.compact(pool)


@pytest.mark.parametrize("S,NB,width,most", [(1, 1, 1, 16), (2, 31, 9, 100), (30, 1000, 40, 600), (9, 32, 4, 50), (400, 70001, 40, 640)])
def test_compact(S, NB, width, most):
    rng = np.random.default_rng(NB)
    lens = [int(x) for x in rng.integers(0, min(most, width * 16), size=S)]
    pool, dev = make(10, S, NB, width, lens, shared=2)
    dev.free_seqs(pool, list(range(0, S, 2)))
    dev.outside(pool, 300, 4)
    dev.compact(pool)
    used = pool.nb - len(pool.free_blocks())
    assert all(pool.refs[b] > 0 for b in range(used)) and not any(pool.refs[used:])
    dev.compact(pool)                                          # nothing left to do
    dev.free_seqs(pool, list(range(S)))
    dev.compact(pool)


@pytest.mark.parametrize("kv,heads,dim,layers", [(coopt.COOPT_KV_E4M3, 8, 128, 3), (coopt.COOPT_KV_FP16, 3, 64, 1),
                                                 (coopt.COOPT_KV_E5M2, 1, 64, 70), (coopt.COOPT_KV_FP16, 40, 128, 2)])
def test_copying(kv, heads, dim, layers):
    NB, es = 50, 2 if kv == coopt.COOPT_KV_FP16 else 1
    shape = coopt.Shape(1, heads, heads, dim, 16, NB, 1, kv, 0.125)
    gen = torch.Generator(device="cuda").manual_seed(3)
    sizes = [heads * 16 * dim * es] * 2 + [heads * 64] * 2
    pools = [[torch.randint(0, 256, (NB, n), generator=gen, device="cuda", dtype=torch.uint8) for _ in range(layers)] for n in sizes]
    want = [[x.clone() for x in p] for p in pools]
    pairs = [(3, 7), (-1, 4), (3, 49), (5, -1), (0, 1), (50, 2), (9, 50), (-1, -1), (48, 8), (1 << 30, 6), (10, 11)]
    copies = torch.tensor(pairs, dtype=torch.int32).cuda()
    scaled = kv != coopt.COOPT_KV_FP16

    def copy(n):
        ks, vs = (pools[2], pools[3]) if scaled else (None, None)
        coopt.kv_cache_copy_blocks(pools[0], pools[1], ks, vs, copies, n, shape)

    def expect(n):
        for src, dst in pairs[:n]:
            if 0 <= src < NB and 0 <= dst < NB:
                for p in want[:4 if scaled else 2]:
                    for x in p:
                        x[dst] = x[src]
        torch.cuda.synchronize()
        for p, w in zip(pools, want):
            for x, y in zip(p, w):
                assert torch.equal(x, y)
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    copy(zero)
    expect(0)
    copy(zero + 5)
    expect(5)
    copy(zero + 1000)
    expect(len(pairs))
    copy(None)
    expect(len(pairs))
    # one layer, given as a tensor
    coopt.kv_cache_copy_blocks(pools[0][0], pools[1][0], pools[2][0] if scaled else None, pools[3][0] if scaled else None, copies[:1] * 0 + 12,
                               zero, shape)
    expect(0)


def test_steps_drawn_at_random():
    """A server's life: prompts, steps, samples, ends, windows, compactions, in any order."""
    rng = np.random.default_rng(17)
    S, NB, width = 24, 300, 30
    pool, dev = make(11, S, NB, width, [0] * S)
    for step in range(120):
        kind = rng.integers(0, 7)
        if kind <= 1:
            dev.reserve(pool, None, S, f"step {step}")
        elif kind == 2:
            chunks = [int(rng.integers(0, 90)) if rng.random() < 0.2 else 0 for _ in range(S)]
            dev.reserve(pool, [0] + list(np.cumsum(chunks)), sum(chunks), f"step {step}")
        elif kind == 3:
            idle = [s for s in range(S) if pool.lens[s] == 0]
            busy = [s for s in range(S) if pool.lens[s] > 0]
            if idle and busy:
                n = int(rng.integers(1, len(idle) + 1))
                dev.fork(pool, [int(x) for x in rng.choice(busy, n)], [int(x) for x in rng.permutation(idle)[:n]], f"step {step}")
        elif kind == 4:
            dev.free_seqs(pool, [int(x) for x in rng.integers(0, S, size=4)], f"step {step}")
        elif kind == 5:
            dev.outside(pool, 70, 20)
        else:
            dev.compact(pool)


def test_captured_replays():
    """A step's calls captured; every replay continues from where the one before left the pool."""
    lens = [100, 17, 0, 31, 640, 48]
    pool, dev = make(12, 6, 90, 60, lens, shared=1)
    slots = torch.zeros(6, dtype=torch.int64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            coopt.kv_blocks_reserve(None, 6, *dev.state, slots, dev.result, dev.ws, dev.shape)
            coopt.kv_blocks_free_outside_window(*dev.state, 64, 4, dev.shape)
    torch.cuda.synchronize()
    dev.check(pool, "captured, not run")
    for step in range(40):
        want, want_slots = pool.reserve(None, 6, np.zeros(6, np.int64))
        pool.free_outside_window(64, 4)
        graph.replay()
        dev.check(pool, f"replay {step}")
        assert int(dev.result) == want and slots.cpu().tolist() == list(want_slots)
        if step % 10 == 9:
            dev.free_seqs(pool, [step // 10])
            dev.compact(pool)

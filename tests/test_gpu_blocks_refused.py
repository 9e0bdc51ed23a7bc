"""GPU: a reservation that is refused leaves no slot that names a place, whatever an earlier step left in the buffer and
however many rows it has: the write that takes the slots then leaves the pool as it was.  Slots that are negative already, and
the rows behind the last sequence of a reservation that is made, stay as they were."""
import numpy as np
import pytest
import torch

import paper_2602_09323_amd as coopt
from test_gpu_blocks import make

pytestmark = pytest.mark.gpu

# (lengths, blocks, width of the table, query_start, rows)
REFUSED = [([100, 0, 159, 16], 40, 10, [0, 1, 0, 1, 1], 5),                      # not increasing
           ([100, 0, 159, 16], 40, 10, [0, 1, 1, 1, -3], 5),                     # ends below 0
           ([100, 0, 159, 16], 40, 10, [0, 1, 1, 1, 9], 5),                      # more rows than announced
           ([100, 0, 159, 16], 40, 10, [2, 2, 2, 3, 4], 7),                      # does not begin at 0
           ([100, 0, 159, 16], 40, 10, [0, 0, 0, 2, 2], 6),                      # a sequence outgrows its row
           ([20, 0], 10, 100, [0, 0, 129], 140),                                 # too few blocks
           ([20, 0, 5], 3, 100, None, 9)]                                        # ... and one row a sequence


@pytest.mark.parametrize("more", [0, 5000])                  # rows in the planning launch, and in one of their own
@pytest.mark.parametrize("lens,NB,width,starts,rows", REFUSED)
def test_no_slot_names_a_place(lens, NB, width, starts, rows, more):
    if starts is None:
        lens = [16 if t else 0 for t in lens]
    if starts is not None and starts[-1] > rows:             # (with more rows announced, as much beyond them)
        starts = starts[:-1] + [starts[-1] + more]
    pool, dev = make(41, len(lens), NB, width, lens)
    rows += more
    said, _ = pool.reserve(starts, rows, np.zeros(rows, np.int64))
    assert said != 0
    old = torch.arange(rows, dtype=torch.int64, device="cuda") % (16 * NB)
    old[::4] = -9
    slots = old.clone()
    qs = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
    coopt.kv_blocks_reserve(qs, rows, *dev.state, slots, dev.result, dev.ws, dev.shape)
    dev.check(pool, "refused")
    assert int(dev.result) == said
    assert bool((slots < 0).all())
    last = len(lens) if starts is None else min(max(starts[-1], 0), rows)
    assert bool((slots[:last] == -1).all())
    assert torch.equal(slots[last:], torch.where(old[last:] >= 0, -1, old[last:]))
    # what takes them does nothing
    g = torch.Generator(device="cuda").manual_seed(2)
    cache = [torch.randint(0, 256, (NB, 2, n), generator=g, device="cuda", dtype=torch.uint8) for n in (1024, 1024, 64, 64)]
    before = [x.clone() for x in cache]
    new = torch.randn(rows, 2, 64, generator=g, device="cuda").half()
    coopt.kv_cache_write_fp8(new, new, slots, *cache, dev.shape)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(cache, before))


@pytest.mark.parametrize("more", [0, 5000])
def test_rows_behind_the_last_sequence(more):
    """Of a reservation that is made: as they were."""
    pool, dev = make(42, 3, 40, 10, [20, 0, 16])
    slots = torch.arange(20 + more, dtype=torch.int64, device="cuda")
    old = slots.clone()
    want, want_slots = pool.reserve([0, 1, 7, 7], 20 + more, old.cpu().numpy())
    coopt.kv_blocks_reserve(torch.tensor([0, 1, 7, 7], dtype=torch.int32, device="cuda"), 20 + more, *dev.state, slots, dev.result,
                            dev.ws, dev.shape)
    dev.check(pool, "made")
    assert want == int(dev.result) == 0
    assert np.array_equal(slots.cpu().numpy(), want_slots) and torch.equal(slots[7:], old[7:])


@pytest.mark.parametrize("rows", [9, 9000])
def test_no_sequences(rows):
    shape = coopt.Shape(0, 2, 2, 64, 16, 40, 10, coopt.COOPT_KV_E4M3, 0.125)
    ws = torch.empty(coopt.kv_blocks_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    ints = torch.zeros(40, dtype=torch.int32, device="cuda")
    result = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    for first, said in ((5, -1), (0, 0)):
        slots = torch.arange(rows, dtype=torch.int64, device="cuda")
        coopt.kv_blocks_reserve(torch.tensor([first], dtype=torch.int32, device="cuda"), rows, ints, ints, ints, ints, slots, result, ws,
                                shape)
        torch.cuda.synchronize()
        assert int(result) == said
        assert bool((slots == -1).all()) if said else torch.equal(slots, torch.arange(rows, device="cuda"))

"""surel_cache_plan on the GPU against the same bookkeeping in plain Python, and surel_cache_store."""
import random

import pytest
import torch

from cache_cases import bookkeeping, plan
from paper_2202_13538_amd import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.check() == 0
    c.close()


def check(ctx, args, page_rows, n_rows, flags=0, want=None):
    length, added, pages, ring, turn = args
    want = want or plan(*(x.cpu() for x in args), page_rows, n_rows)
    kept = [x.clone() for x in (length, added, turn)]
    for _ in range(2):   # the second time with the pages and the ring of the first
        got = binding.cache_plan(ctx, length, added, pages, ring, turn, page_rows, n_rows)
        assert ctx.check() == flags
        for name, x, y in zip(("off", "slots", "length", "turn", "pages", "ring"), (*got, pages, ring), want, strict=True):
            assert torch.equal(x.cpu(), torch.tensor(y, dtype=x.dtype).view(x.shape)), name
    assert all(torch.equal(x, y) for x, y in zip(kept, (length, added, turn)))
    return got


SHAPES = [  # lengths, added, rows of a page, pages of a sequence, rows beyond the last
    ([0], [1], 1, 1, 0), ([0], [0], 4, 3, 0), ([5], [-1], 2, 3, 4), ([0, 0, 0], [0, 7, 0], 4, 2, 1),
    ([16, 15, 17, 0], [1, 1, 1, 1], 16, 3, 0), ([3, 8, 1], [-1, -5, -1], 3, 4, 2), ([1] * 70, [1] * 70, 2, 1, 3),
    ([7, 0, 30], [33, 100, -1], 24, 5, 5), ([9, 0, 9, 9], [0, -1, 0, 0], 8, 2, 0), ([0, 0], [4099, 1], 7, 600, 0),
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x)[:20] for x in s))
def test_small_steps(ctx, shape):
    lengths, added, page_rows, width, beyond = shape
    args = bookkeeping(lengths, added, page_rows, width, spare=2)
    check(ctx, args, page_rows, sum(max(a, 0) for a in added) + beyond)


@pytest.mark.parametrize("seqs,most,page_rows", [(1000, 3, 4), (4095, 40, 16), (4096, 1, 1), (4097, 9, 24), (9001, 2, 8),
                                                 (20_000, 5, 3)])
def test_many_sequences(ctx, seqs, most, page_rows):
    rng = random.Random(seqs)
    lengths = [rng.randint(0, 50) for _ in range(seqs)]
    added = [rng.choice([-1, 0, 1, rng.randint(0, most)]) for _ in range(seqs)]
    args = bookkeeping(lengths, added, page_rows, -(-(50 + most) // page_rows), spare=5, seed=seqs)
    check(ctx, args, page_rows, sum(max(a, 0) for a in added) + 9)


def test_one_long_prompt_among_many_sequences(ctx):
    lengths = [10] * 5000
    added = [0] * 5000
    added[4321] = 100_003
    args = bookkeeping(lengths, added, 32, 3200, seed=1)
    check(ctx, args, 32, 100_003)


def test_no_sequences(ctx):
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    ring, turn = torch.arange(6, dtype=torch.int32, device="cuda"), torch.tensor([0, 6], device="cuda")
    check(ctx, (empty, empty, torch.empty((0, 3), dtype=torch.int32, device="cuda"), ring, turn), 4, 5,
          want=([0], [-1] * 5, [], [0, 6], [], list(range(6))))


def test_pages_that_run_out(ctx):
    # 5 pages for 9 that are needed: the first sequences get them, one of them in part
    lengths, added = [3, 0, 4, 0], [2, 9, 20, 5]
    args = bookkeeping(lengths, added, 4, 7, spare=-4, seed=2)
    check(ctx, args, 4, 36, flags=binding.DEV_NO_PAGE)
    got = binding.cache_plan(ctx, *args, 4, 36)
    assert got[2].tolist()[3] == 0 and ctx.check() == binding.DEV_NO_PAGE


def test_rows_that_do_not_fit_are_not_added(ctx):
    args = bookkeeping([0, 7, 0], [5, 100, 3], 4, 3, spare=3, seed=3)
    check(ctx, args, 4, 108, flags=binding.DEV_CAPACITY)        # the second sequence's pages
    args = bookkeeping([0, 7, 0, 1], [5, 6, 3, 1], 4, 5, spare=3, seed=4)
    check(ctx, args, 4, 8, flags=binding.DEV_CAPACITY)          # the list of slots


def test_pages_and_lengths_that_are_none(ctx):
    # a length that does not fit: nothing is done for its sequence
    length, added, pages, ring, turn = bookkeeping([4, 0, 4], [1, 1, -1], 4, 2, spare=2, seed=5)
    length[1] = 9
    off, slots, after, _ = binding.cache_plan(ctx, length, added, pages, ring, turn, 4, 3)
    assert ctx.check() == binding.DEV_BAD_LENGTH
    assert off.tolist() == [0, 1, 1, 1] and after.tolist() == [5, 0, 0] and slots.tolist()[1:] == [-1, -1]
    length[1] = -1
    binding.cache_plan(ctx, length, added, pages, ring, turn, 4, 3)
    assert ctx.check() == binding.DEV_BAD_LENGTH
    # a last page that is none: its rows have no place
    length, added, pages, ring, turn = bookkeeping([3, 3], [2, 1], 4, 2, spare=2, seed=6)
    pages[0, 0] = ring.numel()
    _, slots, _, _ = binding.cache_plan(ctx, length, added, pages, ring, turn, 4, 3)
    assert ctx.check() == binding.DEV_BAD_PAGE and slots[0] == -1 and slots[1] >= 0 and slots[2] >= 0
    # a page in the ring that is none
    length, added, pages, ring, turn = bookkeeping([0, 0], [2, 2], 4, 2, seed=7)
    ring[int(turn[0]) % ring.numel()] = -3
    _, slots, _, _ = binding.cache_plan(ctx, length, added, pages, ring, turn, 4, 4)
    assert ctx.check() == binding.DEV_BAD_PAGE and slots.tolist()[:2] == [-1, -1] and min(slots.tolist()[2:]) >= 0
    assert pages[0, 0] == -1
    # a ring that counts more than it has
    for bad in ([0, 99], [5, 4], [-1, 0]):
        length, added, pages, ring, turn = bookkeeping([4], [1], 4, 2, spare=2, seed=8)
        _, slots, after, turn_after = binding.cache_plan(ctx, length, added, pages, ring, torch.tensor(bad, device="cuda"), 4, 1)
        assert ctx.check() == binding.DEV_BAD_PAGE | binding.DEV_NO_PAGE
        assert slots.tolist() == [-1] and after.tolist() == [4] and turn_after.tolist() == bad


def test_slots_that_start_anywhere(ctx):
    # (the binding's own lists start on a line; from C they may start at any word)
    lengths, added = [1, 5, 0, 2], [3, 0, 9, 2]
    length, add, pages, ring, turn = bookkeeping(lengths, added, 4, 4, spare=1, seed=9)
    want = plan(length.cpu(), add.cpu(), pages.cpu(), ring.cpu(), turn.cpu(), 4, 15)
    for skip in (1, 2, 3):
        room = torch.full((24,), 77, dtype=torch.int32, device="cuda")
        off = torch.empty(5, dtype=torch.int64, device="cuda")
        after, turn_after = torch.empty_like(length), torch.empty_like(turn)
        rc = binding.load().surel_cache_plan(
            ctx.handle, length.data_ptr(), add.data_ptr(), 4, ring.numel(), 4, 4, 15, pages.data_ptr(), ring.data_ptr(),
            turn.data_ptr(), off.data_ptr(), room[skip:].data_ptr(), after.data_ptr(), turn_after.data_ptr())
        assert rc == binding.OK and ctx.check() == 0
        assert room.tolist() == [77] * skip + want[1] + [77] * (24 - 15 - skip)


def test_a_cache_from_its_first_row_to_its_last(ctx):
    """Steps of a server: prompts, single rows, ends; pages are never held twice and none is lost."""
    rng = random.Random(5)
    n_seqs, n_pages, page_rows, width = 12, 40, 4, 8
    length = torch.zeros(n_seqs, dtype=torch.int32, device="cuda")
    pages = torch.full((n_seqs, width), -1, dtype=torch.int32, device="cuda")
    ring, turn = torch.arange(n_pages, dtype=torch.int32, device="cuda"), torch.tensor([0, n_pages], device="cuda")
    seen_full = False
    for step in range(60):
        now = length.tolist()
        added = [-1 if x > 20 or (x and rng.random() < 0.1) else rng.randint(1, 9) if x == 0 else 1 for x in now]
        flags = 0
        free = int(turn[1] - turn[0])
        need = sum(0 if a < 0 else -(-(x + a) // page_rows) - -(-x // page_rows) for x, a in zip(now, added))
        if need > free:
            flags, seen_full = binding.DEV_NO_PAGE, True
        args = (length, torch.tensor(added, dtype=torch.int32, device="cuda"), pages, ring, turn)
        _, _, length, turn = check(ctx, args, page_rows, 120, flags=flags)
        held = [pages[s, j].item() for s, x in enumerate(length.tolist()) for j in range(-(-x // page_rows))]
        left = [ring[i % n_pages].item() for i in range(int(turn[0]), int(turn[1]))]
        assert sorted(held + left) == list(range(n_pages)), step
    assert seen_full


def test_a_stream_of_its_own_and_a_graph(ctx):
    lengths, added = [3, 0, 17, 5], [1, 9, -1, 1]
    args = bookkeeping(lengths, added, 4, 6, spare=3, seed=11)
    side = torch.cuda.Stream()
    own = binding.Context(0, stream=side)
    length, add, pages, ring, turn = args
    side.wait_stream(torch.cuda.current_stream())
    want = plan(*(x.cpu() for x in args), 4, 14)
    with torch.cuda.stream(side):
        binding.cache_plan(own, *args, 4, 14)   # (grows what it needs)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = binding.cache_plan(own, *args, 4, 14)
        for lens in (lengths, [2, 3, 4, 20], [0, 0, 0, 0]):
            now = bookkeeping(lens, added, 4, 6, spare=9, seed=12)
            if now[3].numel() > ring.numel():
                continue
            n = ring.numel()
            length.copy_(now[0])
            # pages of the same numbers for everybody: the ring's own length stays
            table = torch.arange(24, dtype=torch.int32, device="cuda").view(4, 6) % n
            pages.copy_(table), ring.copy_(torch.arange(n, dtype=torch.int32, device="cuda")), turn.copy_(torch.tensor([1, 1 + n - 10]))
            want = plan(length.cpu(), add.cpu(), pages.cpu(), ring.cpu(), turn.cpu(), 4, 14)
            graph.replay()
            side.synchronize()
            own.check()
            for x, y in zip((*got, pages, ring), want, strict=True):
                assert torch.equal(x.cpu(), torch.tensor(y, dtype=x.dtype).view(x.shape))
    own.close()


# ------------------------------------------------------------------ stores


def stored(k, v, slots, k_pages, v_pages):
    want = [k_pages.cpu().clone(), v_pages.cpu().clone()]
    P = k_pages.shape[1]
    for r, s in enumerate(slots.tolist()):
        if s >= 0:
            want[0][s // P, s % P], want[1][s // P, s % P] = k[r].cpu(), v[r].cpu()
    return want


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,kv_heads,dim,page_rows,heads_first,packed", [
    (1, 1, 8, 1, False, True), (7, 3, 40, 5, True, False), (300, 2, 128, 16, False, False), (65, 8, 64, 4, True, True),
    (1000, 1, 24, 100, False, True), (9, 130, 128, 2, True, False), (3, 1000, 16, 3, False, True)])
def test_store(ctx, rows, kv_heads, dim, page_rows, heads_first, packed, dtype):
    g = torch.Generator().manual_seed(rows)
    n_pages = -(-rows // page_rows) + 3
    bits = lambda *s: torch.randint(-2 ** 15, 2 ** 15, s, generator=g, dtype=torch.int16).view(dtype).cuda()  # noqa: E731  any bits, NaN too
    if packed:
        qkv = bits(rows, 3, kv_heads, dim)
        k, v = qkv[:, 1], qkv[:, 2]
    else:
        k, v = bits(rows, kv_heads, dim), bits(kv_heads, rows, dim).transpose(0, 1)
    shape = (n_pages, kv_heads, page_rows, dim) if heads_first else (n_pages, page_rows, kv_heads, dim)
    k_pages, v_pages = (bits(*shape).transpose(1, 2) if heads_first else bits(*shape) for _ in range(2))
    slots = torch.randperm(n_pages * page_rows, generator=g)[:rows].int()
    slots[torch.rand(rows, generator=g) < 0.1] = -1
    as_bits = lambda t: t.cpu().contiguous().view(torch.int16)  # noqa: E731
    want = stored(k, v, slots, k_pages, v_pages)
    binding.cache_store(ctx, k, v, slots.cuda(), k_pages, v_pages)
    assert ctx.check() == 0
    assert torch.equal(as_bits(k_pages), as_bits(want[0])) and torch.equal(as_bits(v_pages), as_bits(want[1]))


def test_store_leaves_out_slots_that_are_none(ctx):
    k = torch.arange(4 * 16, device="cuda").view(4, 1, 16).bfloat16()
    pages = torch.zeros(2, 3, 1, 16, device="cuda").bfloat16()
    for bad in (6, -2, 2 ** 31 - 1, -2 ** 31):
        k_pages, v_pages = pages.clone(), pages.clone()
        slots = torch.tensor([5, bad, -1, 0], dtype=torch.int32, device="cuda")
        binding.cache_store(ctx, k, k, slots, k_pages, v_pages)
        assert ctx.check() == binding.DEV_BAD_PAGE
        want = pages.clone()
        want[1, 2], want[0, 0] = k[0], k[3]
        assert torch.equal(k_pages, want) and torch.equal(v_pages, want)
    binding.cache_store(ctx, k[:0], k[:0], slots[:0], k_pages, v_pages)   # nothing
    assert ctx.check() == 0 and torch.equal(k_pages, want)


def test_one_page_only_may_have_any_stride(ctx):
    k = torch.randn(3, 1, 8, device="cuda").half()
    room = torch.zeros(40, device="cuda").half()
    pages = room.as_strided((1, 4, 1, 8), (3, 8, 5, 1))
    binding.cache_store(ctx, k, k, torch.tensor([2, 0, 3], dtype=torch.int32, device="cuda"), pages, pages)
    assert ctx.check() == 0
    assert torch.equal(room[:32].view(4, 8), torch.stack([k[1, 0], torch.zeros_like(k[0, 0]), k[0, 0], k[2, 0]]))

"""What the calls of a paged cache refuse before they touch a device, and how its keys are shared out."""
import ctypes
import math
import random
import types

import pytest
import torch

from paper_2202_13538_amd import binding
from test_rules_host import evaluate_list

P = 0x10000  # an aligned address that nothing reads: every call here is refused
R, N, C = binding.E_RANGE, binding.E_NULL, binding.E_CTX


def cache(**changes):
    a = dict(d_k=P, d_v=P, page=2048, row=128, head=64, n_pages=9, page_rows=16, type=binding.BF16, kv_heads=2, dim=64)
    assert set(changes) <= set(a)
    return binding.Cache(**(a | changes))


CACHE = [
    (R, dict(type=2)), (R, dict(type=-1)), (R, dict(n_pages=0)), (R, dict(n_pages=binding.MAX_ROWS)), (R, dict(page_rows=0)),
    (R, dict(page_rows=binding.MAX_ROWS, n_pages=2)), (R, dict(dim=0)), (R, dict(dim=12)), (R, dict(dim=136)),
    (R, dict(kv_heads=0)), (R, dict(kv_heads=65536)), (R, dict(page=2044)), (R, dict(page=2 ** 40 + 8)), (R, dict(row=-8)),
    (R, dict(row=binding.MAX_STRIDE + 8)), (R, dict(head=63)), (N, dict(d_k=None)), (N, dict(d_v=None)),
    (R, dict(d_k=P + 8)), (R, dict(d_v=P + 2)), (C, {}),
    (C, dict(n_pages=1, page=3)), (C, dict(page_rows=1, row=5)), (C, dict(kv_heads=1, head=7)),
]


def store(lib, ctx, c, k=P, v=P, k_row=128, k_head=64, v_row=128, v_head=64, slots=P, rows=5):
    return lib.surel_cache_store(ctx, None if c is None else ctypes.byref(c), k, v, k_row, k_head, v_row, v_head, slots, rows)


@pytest.mark.parametrize("status,changes", CACHE, ids=str)
def test_caches_that_are_none(status, changes):
    lib, c = binding.load(), cache(**changes)
    assert store(lib, None, c) == status
    args = attention()
    if c.page_rows == binding.MAX_ROWS:
        args.max_pages = 1
    if c.kv_heads > 65535:
        args.heads = c.kv_heads
    assert lib.surel_cache_attention(None, ctypes.byref(c), ctypes.byref(args), P, P) == status


@pytest.mark.parametrize("status,changes", [
    (R, dict(rows=-1)), (R, dict(rows=binding.MAX_ROWS + 1)), (R, dict(k_row=-8)), (R, dict(k_head=4)), (R, dict(v_row=9)),
    (R, dict(v_head=binding.MAX_STRIDE + 8)), (N, dict(k=None)), (N, dict(v=None)), (N, dict(slots=None)), (R, dict(k=P + 8)),
    (R, dict(v=P + 4)), (C, {}), (C, dict(rows=0, k=None, v=None, slots=None)), (C, dict(rows=1, k_row=3))], ids=str)
def test_store_refuses(status, changes):
    assert store(binding.load(), None, cache(), **changes) == status
    assert store(binding.load(), None, None, **changes) == N


def attention(**changes):
    a = dict(d_q=P, q_row=256, q_head=64, d_pages=P, d_length=P, n_seqs=3, max_pages=4, heads=4, scale=0.125, d_bias=None,
             d_bucket=None, n_buckets=0, reach=0)
    assert set(changes) <= set(a)
    return binding.CacheAttentionArgs(**(a | changes))


@pytest.mark.parametrize("status,changes", [
    (R, dict(n_seqs=-1)), (R, dict(n_seqs=binding.MAX_SEQS + 1)), (R, dict(max_pages=0)), (R, dict(max_pages=binding.MAX_ROWS)),
    (R, dict(heads=0)), (R, dict(heads=3)), (R, dict(heads=65536)), (R, dict(q_row=-8)), (R, dict(q_head=4)),
    (R, dict(q_row=binding.MAX_STRIDE + 8)), (R, dict(scale=0.0)), (R, dict(scale=-1.0)), (R, dict(scale=math.nan)),
    (R, dict(scale=math.inf)), (N, dict(d_bias=P)), (N, dict(d_bucket=P)), (R, dict(d_bias=P, d_bucket=P, n_buckets=0)),
    (R, dict(d_bias=P, d_bucket=P, n_buckets=4, reach=-1)),
    (R, dict(d_bias=P, d_bucket=P, n_buckets=4, reach=binding.MAX_REACH + 1)),
    (R, dict(n_seqs=binding.MAX_SEQS, max_pages=2 ** 25)), (N, dict(d_q=None)), (N, dict(d_pages=None)),
    (N, dict(d_length=None)), (R, dict(d_q=P + 8)), (C, {}), (C, dict(n_seqs=0, d_q=None, d_pages=None, d_length=None)),
    (C, dict(n_seqs=1, q_row=5)), (C, dict(d_bias=P, d_bucket=P, n_buckets=4, reach=0))], ids=str)
def test_cache_attention_refuses(status, changes):
    lib = binding.load()
    assert lib.surel_cache_attention(None, ctypes.byref(cache()), ctypes.byref(attention(**changes)), P, P) == status


def test_cache_attention_refuses_missing_outputs_and_arguments():
    lib, c, a = binding.load(), cache(), attention()
    assert lib.surel_cache_attention(None, None, ctypes.byref(a), P, P) == N
    assert lib.surel_cache_attention(None, ctypes.byref(c), None, P, P) == N
    assert lib.surel_cache_attention(None, ctypes.byref(c), ctypes.byref(a), None, P) == N
    assert lib.surel_cache_attention(None, ctypes.byref(c), ctypes.byref(a), P, None) == N
    assert lib.surel_cache_attention(None, ctypes.byref(c), ctypes.byref(a), P + 8, P) == R


PLAN = dict(length=P, added=P, seqs=5, n_pages=9, page_rows=16, max_pages=4, rows=7, pages=P, ring=P, turn=P, off=P, slots=P,
            after=2 * P, turn_after=2 * P)


@pytest.mark.parametrize("status,changes", [
    (R, dict(seqs=-1)), (R, dict(seqs=binding.MAX_SEQS + 1)), (R, dict(n_pages=0)), (R, dict(page_rows=0)),
    (R, dict(max_pages=0)), (R, dict(rows=-1)), (R, dict(rows=binding.MAX_ROWS + 1)), (R, dict(n_pages=2 ** 30)),
    (R, dict(max_pages=2 ** 27)), (N, dict(length=None)), (N, dict(added=None)), (N, dict(pages=None)), (N, dict(after=None)),
    (N, dict(ring=None)), (N, dict(turn=None)), (N, dict(off=None)), (N, dict(slots=None)), (N, dict(turn_after=None)),
    (R, dict(after=P)), (R, dict(turn_after=P)), (C, {}), (C, dict(rows=0, slots=None)),
    (C, dict(seqs=0, length=None, added=None, pages=None, after=None))], ids=str)
def test_plan_refuses(status, changes):
    assert binding.load().surel_cache_plan(None, *(PLAN | changes).values()) == status


def test_binding_refuses_tensors_that_do_not_fit():
    ctx = types.SimpleNamespace(handle=None, device=torch.device("cuda", 0), stream=None)
    pages, q = torch.zeros(3, 16, 2, 32).half(), torch.zeros(4, 2, 32).half()
    table, length = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError, match="bfloat16 or torch.float16"):
        binding.cache_attention(ctx, q, pages.float(), pages.float(), table, length)
    with pytest.raises(TypeError, match="v_pages"):
        binding.cache_store(ctx, q, q, length, pages, pages.bfloat16())
    with pytest.raises(ValueError, match="GPU"):
        binding.cache_attention(ctx, q, pages, pages, table, length)
    with pytest.raises(ValueError, match="GPU"):
        binding.cache_store(ctx, q, q, length, pages, pages)
    for bad in ((length, length[:3], table), (length[:3], length[:3], table), (length, length, table[0])):
        with pytest.raises(ValueError):
            binding.cache_plan(ctx, *bad, length, torch.tensor([0, 4]), 16, 5)
    for ring, turn in ((table, torch.tensor([0, 4])), (length, torch.tensor([0]))):
        with pytest.raises(ValueError):
            binding.cache_plan(ctx, length, length, table, ring, turn, 16, 5)
    with pytest.raises(ValueError, match="context's cuda:0"):
        binding.cache_plan(ctx, length, length, table, length, torch.tensor([0, 4]), 16, 5)


def test_division_by_a_page(tmp_path):
    rng = random.Random(0)
    cases = []
    for d in [1, 2, 3, 5, 7, 15, 16, 17, 100, 255, 1000, 65535, 2 ** 20 + 1, 2 ** 29 + 1, 2 ** 30 - 1, 2 ** 30]:
        xs = [0, 1, d - 1, d, d + 1, 2 ** 31 - 1, 2 ** 31 - 2, (2 ** 31 - 1) // d * d, (2 ** 31 - 1) // d * d - 1]
        cases += [(d, x) for x in xs + [rng.randrange(2 ** 31) for _ in range(20)] if 0 <= x < 2 ** 31]
    source = "(x[0] == 1 ? x[1] : (long long)(((unsigned long long)(unsigned)x[1] * Divisor(x[0]).m >> 32) >> Divisor(x[0]).shift))"
    # the constants as the host makes them, the multiplication as the device does it
    header = tmp_path / "divisor.h"
    text = open(binding._PKG_DIR + "/csrc/cache.h").read()
    begin, end = text.index("struct Divisor {"), text.index("    __device__", text.index("struct Divisor {"))
    header.write_text("#include <stdint.h>\nnamespace surel {\n" + text[begin:end] + "};\n}\n")
    got = evaluate_list(tmp_path, [str(header)], source, cases)
    assert got == [x // d for d, x in cases]


def shared_out(tmp_path, lists):
    """Parts of lists of tile counts, by the rules that the kernel uses: [(first tile, end)] with cuts moved."""
    out = []
    for counts, waves in lists:
        total = sum(counts)
        (parts,) = evaluate_list(tmp_path, ["cache_share.h"], "parts_of(x[0], x[1])", [(total, waves)])
        begins = evaluate_list(tmp_path, ["cache_share.h"], "part_begin(x[0], x[1], x[2])",
                               [(total, parts, n) for n in range(parts + 1)])
        starts, place = [], []
        at = 0
        for n in counts:
            place.append((at, n))
            at += n
        ask = []
        for b in begins[:-1]:
            s, n = next((s, n) for s, n in place if s <= b < s + n)
            ask.append((b - s, n))
        tiles = sorted({random.Random(2).randrange(total) for _ in range(40)} | {0, total - 1})
        own = evaluate_list(tmp_path, ["cache_share.h"], "part_with(x[0], x[1], x[2])", [(total, parts, t) for t in tiles])
        assert all(begins[n] <= t < begins[n + 1] for n, t in zip(own, tiles))
        backs = evaluate_list(tmp_path, ["cache_share.h"], "moves_back(x[0], x[1])", ask)
        starts = [b - m for b, m in zip(begins, backs)] + [total]
        out.append((parts, place, starts))
    return out


def test_keys_are_shared_out_whole(tmp_path):
    rng = random.Random(1)
    lists = [([1], 1), ([1], 512), ([17], 512), ([8] * 30, 7), ([2048], 1280), ([5, 2000, 1, 1, 40] * 3, 100)]
    lists += [([rng.choice([1, 2, 8, 9, 33, 300]) for _ in range(rng.randint(1, 60))], rng.choice([1, 3, 64, 1024]))
              for _ in range(12)]
    for (counts, waves), (parts, place, starts) in zip(lists, shared_out(tmp_path, lists), strict=True):
        assert 1 <= parts <= waves and starts[0] == 0 and starts == sorted(starts)
        for s, n in place:
            cuts = [b for b in set(starts) if s < b < s + n]
            assert not cuts or n > 16                        # only long pairs are cut
        most = max(b - a for a, b in zip(starts, starts[1:]))
        assert most <= -(-sum(counts) // parts) + 16         # a part's own tiles and one short pair


def test_lists_that_are_looked_through_are_short(tmp_path):
    sizes = [(n,) for n in (1, 64, 4096, 4097, 5000, 262144, 262145, 10 ** 6, 2 ** 24)]
    each = evaluate_list(tmp_path, ["cache_share.h"], "seqs_of_an_entry(x[0])", sizes)
    for (n,), e in zip(sizes, each, strict=True):
        assert 1 <= e <= 4096 and -(-n // e) <= 4096 and (e == 1) == (n <= 4096)

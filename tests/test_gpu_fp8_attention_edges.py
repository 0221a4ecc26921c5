"""Attention over the 8-bit cache where an item of query rows has no tokens: shares of it that end before its first tile, and sequences that
hold nothing at all."""
import numpy as np
import pytest
import torch

from fp8_reference import to64
from paper_2410_16926_b200 import pvq
from test_gpu_fp8_attention import check, compare, filled, queries
from test_gpu_fp8_cache import I32, ints, tables

pytestmark = pytest.mark.gpu

ROWS, UNITS, BLOCKS, TILE = 256, 6, 148, 128  # of the kernel for many rows: rows of an item, what its beginning counts, thread blocks, tokens of a tile


def shares_without_tiles(group, kv, lengths, new, causal):
    """How many shares of the work end before the first tile of an item that has some."""
    tiles = []
    for length, n in zip(lengths, new):
        of_head = []
        for q0 in range(0, n * group, ROWS):
            last = (min(q0 + ROWS, n * group) - 1) // group
            hi = min(length, length - n + last + 1) if causal else length
            of_head.append(max(0, -(-hi // TILE)))
        tiles += of_head * kv
    ends = np.cumsum([UNITS + t for t in tiles])
    blocks = min(BLOCKS, max(1, ends[-1] // (UNITS + 2)))
    each, larger = divmod(int(ends[-1]), blocks)
    found = 0
    for c in range(1, blocks):
        cut = each * c + min(c, larger)
        i = int(np.searchsorted(ends, cut, side="right"))
        into = cut - (ends[i] - UNITS - tiles[i])
        found += tiles[i] > 0 and 0 < into <= UNITS
    return found


@pytest.mark.parametrize("group,kv,lengths,new,causal", [(1, 8, [900, 1500, 700, 333], [900, 500, 700, 333], True), (4, 4, [2100, 300], [2100, 300], True),
                                                         (2, 16, [700, 512, 40], [333, 500, 40], False), (8, 2, [1000] * 6, [100] * 6, True)])
def test_shares_that_end_before_the_first_tile(group, kv, lengths, new, causal):
    assert shares_without_tiles(group, kv, lengths, new, causal) >= 3
    dim, page = 64, 32
    rng = np.random.default_rng(sum(new))
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, kv, page, dim)
    starts = [0] + [int(x) for x in np.cumsum(new)]
    q = queries(rng, starts[-1], group * kv, dim)
    first = check(q, cache, table, lengths, starts, page, causal=causal)
    for _ in range(5):
        again = pvq.fp8_attention(q, cache, ints(table), ints(lengths), ints(starts), causal=causal, lse=True)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,empty", [(1, 700), (1, 20), (3, 400), (40, 60), (300, 40)])
def test_sequences_that_hold_nothing(n, empty, causal):
    """A batch padded with sequences of length 0, many in a row: zeros and -inf, whatever their queries hold, and nothing of it in the others."""
    group, kv, dim, page = 4, 2, 64, 32
    rng = np.random.default_rng(n + empty)
    lengths = [0] * empty + [n + 200] + [0] * empty + [n + 3000, 0, n]
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, kv, page, dim)
    starts = None if n == 1 else [n * i for i in range(len(lengths) + 1)]
    q = queries(rng, n * len(lengths), group * kv, dim)
    args = ints(table), ints(lengths), None if starts is None else ints(starts)
    first = check(q, cache, table, lengths, starts, page, causal=causal)
    nothing = torch.tensor([length == 0 for length in lengths], device="cuda").repeat_interleave(n)
    for odd in (0.0, float("nan"), float("inf"), -3e38):
        q[nothing] = odd
        status = torch.zeros(1, dtype=I32, device="cuda")
        out, lse = pvq.fp8_attention(q, cache, *args, causal=causal, lse=True, status=status)
        assert bool((out[nothing] == 0).all()) and bool((lse[nothing] == -float("inf")).all())
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
        assert int(status) == pvq.STATUS_BAD_PAGE  # (lengths below their rows are told)


@pytest.mark.parametrize("n,group,length", [(20, 1, 5), (20, 4, 5), (100, 4, 10), (300, 1, 200), (300, 1, 0)])
def test_rows_that_see_nothing_beside_rows_that_see(n, group, length):
    """Rows in front of their sequence's beginning get zeros and -inf, whatever their queries hold."""
    kv, dim, page, seqs = 2, 64, 32, 5
    rng = np.random.default_rng(n + group)
    lengths = [length, n, length, 3 * n, length]
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, kv, page, dim)
    starts = [n * i for i in range(seqs + 1)]
    q = queries(rng, n * seqs, group * kv, dim)
    first = check(q, cache, table, lengths, starts, page)
    nothing = torch.cat([torch.arange(n, device="cuda") < n - x for x in lengths])
    for odd in (float("nan"), -float("inf")):
        q[nothing] = odd
        out, lse = pvq.fp8_attention(q, cache, ints(table), ints(lengths), ints(starts), lse=True)
        assert bool((out[nothing] == 0).all()) and bool((lse[nothing] == -float("inf")).all())
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("odd", [[2, 1, 0], [0, 2, 1], [1, 0, 2], [2 ** 31 - 1, 0, 2], [0, 2, -1]])
def test_starts_that_descend_are_told_and_nothing_is_written(odd, n):
    kv, dim, page, lengths = 2, 64, 32, [100, 300]
    rng = np.random.default_rng(n)
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, kv, page, dim)
    q = queries(rng, 2 * n, 8, dim)
    out = torch.full_like(q, float("nan"))
    status = torch.zeros(1, dtype=I32, device="cuda")
    pvq.fp8_attention(q, cache, ints(table), ints(lengths), ints([x * n if abs(x) < 9 else x for x in odd]), out=out, status=status)
    assert bool(torch.isnan(out).all()) and int(status) == pvq.STATUS_BAD_PAGE
    status.zero_()
    for fine in ([0, n, 2 * n], [0, 0, 2 * n], [-5, n, 2 ** 31 - 1]):  # (ends beyond the rows are cut off)
        out.fill_(float("nan"))
        pvq.fp8_attention(q, cache, ints(table), ints(lengths), ints(fine), out=out, status=status)
        assert int(status) == 0 and bool(torch.isfinite(out).all())


@pytest.mark.parametrize("heads,kv", [(32, 8), (64, 1)])  # few rows and many
def test_overlapping_sequences_of_more_than_2_to_31_tiles(heads, kv):
    """Every second sequence claims all rows, over tables of 2^20 tokens: what one sequence after another may have is fewer, all together are not."""
    dim, page, seqs, rows, width = 64, 128, 1024, 4096, 8192
    cache = pvq.alloc_fp8_cache(1, kv, page, dim)
    for c in cache:
        c.view(torch.uint8).fill_(0x38)
    table = torch.zeros((seqs, width), dtype=I32, device="cuda")
    lengths = torch.full((seqs,), width * page, dtype=I32, device="cuda")
    starts = torch.arange(seqs + 1, dtype=I32, device="cuda") % 2 * rows
    assert seqs // 2 * (rows * heads // kv // 256) * kv * width >= 2 ** 31
    q = torch.zeros((rows, heads, dim), dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 3.0)
    status = torch.zeros(1, dtype=I32, device="cuda")
    pvq.fp8_attention(q, cache, table, lengths, starts, out=out, status=status)
    assert bool((out == 3.0).all()) and int(status) == pvq.STATUS_BAD_PAGE


@pytest.mark.parametrize("scale", [None, 3e38])
@pytest.mark.parametrize("size", [1e25, 1e30, 3e38])
@pytest.mark.parametrize("n", [1, 8, 60])
def test_keys_of_zero_under_factors_beyond_fp32(n, size, scale):
    """Query values times the scale times a page's scale beyond fp32: a score of zero stays zero, and one that is far below takes no part."""
    heads, kv, dim, page, length = 8, 2, 64, 32, 300
    rng = np.random.default_rng(n)
    table, pool = tables(rng, [length], page)
    cache = filled(rng, table, [length], pool, kv, page, dim)
    keys = cache.k.view(torch.uint8)
    keys.fill_(0)
    keys[int(table[0][2])] = 0xb8  # -1
    cache.k_scales.view(torch.uint8).fill_(127 + 40)
    q = torch.full((n, heads, dim), size, dtype=torch.bfloat16, device="cuda")
    out, lse = pvq.fp8_attention(q, cache, ints(table), ints([length]), ints([0, n]), causal=False, lse=True, **({} if scale is None else dict(scale=scale)))
    kept = [t for t in range(length) if not 2 * page <= t < 3 * page]
    for h in range(kv):
        ids = torch.from_numpy(np.ascontiguousarray(table[0])).cuda()
        v = cache.v.view(torch.uint8)[ids, h].view(torch.float8_e4m3fn).double() * torch.exp2(cache.v_scales.view(torch.uint8)[ids, h].double() - 127)[:, None, None]
        v = v.flatten(0, 1)[kept]
        got = out[:, h * 4:h * 4 + 4].double()
        # equal weights: off by 2^-8 of themselves, the result by as much again
        assert bool(((got - v.mean(dim=0)).abs() <= 2.0 ** -7 * v.abs().mean(dim=0)).all())
    assert bool(((lse.double() - np.log(len(kept))).abs() <= 2.0 ** -18).all())


@pytest.mark.parametrize("n", [1, 3, 60])
@pytest.mark.parametrize("length,window", [(2 ** 31 - 1, 2 ** 30), (2 ** 31 - 1, 2 ** 31 - 200), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 40), (2 ** 30 + 200, 2 ** 30),
                                           (700, 2 ** 30 - 1), (700, 2 ** 31 - 1), (700, 2 ** 62)])
def test_windows_of_any_size(n, length, window):
    """Lengths beyond the table: what lies behind the window is not seen, however wide it is."""
    heads, kv, dim, page, held = 4, 2, 64, 32, 704
    rng = np.random.default_rng(n)
    table, pool = tables(rng, [held], page)
    cache = filled(rng, table, [held], pool, kv, page, dim)
    q = queries(rng, n, heads, dim)
    out, lse = pvq.fp8_attention(q, cache, ints(table), ints([length]), ints([0, n]), window=window, lse=True)
    for i in range(n):
        at = length - n + i
        low, high = max(0, at - window + 1), min(held, at + 1)
        if low >= high:
            assert bool((out[i] == 0).all()) and bool((lse[i] == -float("inf")).all())
            continue
        # the same row as the last of a sequence that ends with it, or with the table, and a window of what it sees
        want = pvq.fp8_attention(q[i:i + 1], cache, ints(table), ints([high]), window=high - low, lse=True)
        # each call off by 2^-8 of its result, its weights by 2^-8 of themselves and less for their scores: 2^-7 of the largest value in all, that is
        # 448 times the largest scale
        largest = 448.0 * 2.0 ** (int(cache.v_scales.view(torch.uint8).max()) - 127)
        assert bool(((out[i:i + 1].float() - want[0].float()).abs() <= 2.0 ** -7 * want[0].float().abs() + 2.0 ** -6 * largest).all())
        assert bool(((lse[i:i + 1] - want[1]).abs() <= 2.0 ** -10).all())


def test_steps_without_rows_or_sequences_are_refused():
    cache = pvq.alloc_fp8_cache(2, 2, 16, 32)
    for c in cache:
        c.view(torch.uint8).fill_(0x38)
    kept = [c.view(torch.uint8).clone() for c in cache]
    x, q = torch.zeros(0, 2, 32, device="cuda"), torch.zeros(0, 4, 32, device="cuda", dtype=torch.bfloat16)
    nothing = torch.zeros((0, 1), dtype=I32, device="cuda"), ints([])
    for step in ((ints([[0], [1]]), ints([0, 0]), ints([0, 0, 0])), (*nothing, None), (*nothing, ints([0])), (ints([[], []]), ints([1, 1]), ints([0, 0, 0]))):
        for call in (lambda: pvq.fp8_cache_write(x, x, cache, *step), lambda: pvq.fp8_cache_read(cache, *step, rows=0), lambda: pvq.fp8_attention(q, cache, *step)):
            with pytest.raises(pvq.PvqError):
                call()
    torch.cuda.synchronize()
    assert all(torch.equal(c.view(torch.uint8), k) for c, k in zip(cache, kept))


def test_items_of_few_rows_that_take_long():
    """Sequences of 2^20 tokens and 100 rows, one after another in a thread block, before one of 300 rows: its second tile of rows has nothing to do for
    a third of a second, which is no reason to give up.  All values are ones."""
    page, width, per, dim = 128, 8192, 22, 64
    new, lengths = [], []
    for _ in range(150):  # more than there are thread blocks
        new += [100] * per + [300]
        lengths += [width * page] * per + [300]
    cache = pvq.alloc_fp8_cache(1, 1, page, dim)
    for c, byte in zip(cache, (0x38, 0x38, 127, 127)):
        c.view(torch.uint8).fill_(byte)
    table = torch.zeros((len(new), width), dtype=I32, device="cuda")
    q = queries(np.random.default_rng(1), sum(new), 1, dim)
    status = torch.zeros(1, dtype=I32, device="cuda")
    out = pvq.fp8_attention(q, cache, table, ints(lengths), ints([0] + [int(x) for x in np.cumsum(new)]), status=status)
    assert int(status) == 0 and bool((out == 1).all())

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

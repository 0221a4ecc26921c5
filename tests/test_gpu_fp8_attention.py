"""Attention over the 8-bit cache against its definition."""
import numpy as np
import pytest
import torch

import fp8_cache_reference as ref
from fp8_reference import to64
from paper_2410_16926_b200 import pvq
from test_gpu_fp8_cache import I32, ints, tables

pytestmark = pytest.mark.gpu


def filled(rng, table, lengths, pool, heads, page, dim, spread=2, garbage=0x7f):
    """A cache with random tokens; what is behind the sequences' ends, and pages of none, hold `garbage` (NaN)."""
    codes, scales = [], []
    for _ in range(2):
        c = torch.full((pool, heads, page, dim), garbage, dtype=torch.uint8)
        e = torch.from_numpy(rng.integers(-7 - spread, -6 + spread, (pool, heads)))
        for s, length in enumerate(lengths):
            for i in range(-(-max(0, min(length, table.shape[1] * page)) // page)):
                n, pid = min(page, length - i * page), table[s][i]
                if 0 <= pid < pool:
                    x = torch.from_numpy(rng.standard_normal((heads, n, dim)) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
                    c[pid, :, :n] = x.view(torch.uint8)
        codes.append(c.cuda().view(torch.float8_e4m3fn))
        scales.append((e + 127).to(torch.uint8).cuda().view(torch.float8_e8m0fnu))
    return pvq.Fp8Cache(*codes, *scales)


def queries(rng, rows, heads, dim, scale=1.0):
    return torch.from_numpy(rng.standard_normal((rows, heads, dim)) * scale).to(torch.bfloat16).cuda()


def check(q, cache, table, lengths, starts, page, **how):
    out, lse = pvq.fp8_attention(q, cache, ints(table), ints(lengths), None if starts is None else ints(starts), lse=True, **how)
    compare(out, lse, q, cache, table, lengths, starts, page, **how)
    return out, lse


def compare(out, lse, q, cache, table, lengths, starts, page, **how):
    codes, exponents = ref.held(cache)
    want, want_lse, slack, slack_lse = ref.attention(to64(q), codes, exponents, np.asarray(table), lengths, starts, page, **how)
    mine = ~np.isnan(want_lse)
    got, got_lse = to64(out), to64(lse)
    assert np.isfinite(got[mine]).all()
    assert (np.abs(got - want)[mine] <= slack[mine]).all(), "off by %g of what it may be" % (np.abs(got - want)[mine] / np.maximum(slack[mine], 1e-300)).max()
    empty = mine & np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(got_lse) & mine, empty)
    some = mine & ~empty
    assert (np.abs(got_lse[some] - want_lse[some]) <= slack_lse[some]).all()


SHAPES = [  # query heads, cache heads, dim, page, lengths, new tokens of each (None: one row a sequence)
    (4, 1, 128, 64, [1], None),
    (4, 1, 128, 64, [127, 128, 129, 0, 1, 500], None),
    (8, 8, 64, 16, [15, 16, 17, 300], None),
    (32, 8, 128, 128, [3000], None),
    (7, 1, 96, 32, [1000, 1, 33], None),
    (40, 2, 16, 16, [260, 128], None),            # 20 query heads for each of the cache's
    (64, 1, 128, 64, [400, 70], None),            # 64
    (16, 4, 128, 64, [300, 40, 5, 700], [4, 3, 5, 1]),
    (6, 2, 80, 16, [129, 257, 0, 64], [9, 2, 0, 64]),
    (8, 2, 128, 32, [700, 10, 300], [100, 10, 1]),
    (4, 4, 64, 128, [513, 129], [513, 1]),
    (3, 1, 48, 16, [200, 3], [150, 7]),           # shorter than its rows
]


@pytest.mark.parametrize("how", [dict(), dict(causal=False), dict(window=1), dict(window=37), dict(window=400, scale=0.3)], ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[:4])))
def test_attention(shape, how):
    heads, kv, dim, page, lengths, new = shape
    rng = np.random.default_rng(heads + dim + len(lengths))
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, kv, page, dim)
    starts, rows = None, len(lengths)
    if new is not None:
        starts = [1]
        for n in new:
            starts.append(starts[-1] + n)
        rows = starts[-1] + 2
    check(queries(rng, rows, heads, dim), cache, table, lengths, starts, page, **how)


@pytest.mark.parametrize("heads,lengths,new", [(32, [40000], None), (8, [9000, 1, 20000, 130], None), (16, [70000], [3]), (8, [6000, 300], [500, 300])])
def test_long_sequences_are_shared_by_many_blocks(heads, lengths, new):
    kv, dim, page = 2, 128, 64
    rng = np.random.default_rng(heads)
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, kv, page, dim)
    starts = None if new is None else [0] + list(np.cumsum(new))
    rows = len(lengths) if new is None else starts[-1]
    q = queries(rng, rows, heads, dim, 2.0)
    first = check(q, cache, table, lengths, starts, page)
    again = pvq.fp8_attention(q, cache, ints(table), ints(lengths), None if starts is None else ints(starts), lse=True)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("n", [1, 3, 70])
def test_scales_far_apart(n):
    """Pages whose scales lie 2^60 apart, the ends of the range among them: values as small as the rest of a sum do not vanish where a large
    page has no weight."""
    heads, kv, dim, page, lengths = 4, 2, 64, 16, [200]
    rng = np.random.default_rng(11)
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, kv, page, dim)
    e = torch.full((pool, kv), 127 - 10, dtype=torch.uint8)
    e[::3] = 127 - 40
    e[1::3] = 127 + 20
    cache.v_scales.view(torch.uint8).copy_(e)
    cache.k_scales.view(torch.uint8).copy_(torch.from_numpy(rng.integers(127 - 40, 127 - 5, (pool, kv))).to(torch.uint8))
    q = queries(rng, n, heads, dim, 5.0)
    check(q, cache, table, lengths, [0, n], page)
    # the pages with large scales hidden by their scores
    x = cache.k.float()
    x[1::3, :, :, 0] = -448.0
    cache.k.copy_(x.to(torch.float8_e4m3fn))
    cache.k_scales.view(torch.uint8).fill_(127 - 2)
    q[:, :, 0] = 100.0
    check(q, cache, table, lengths, [0, n], page)


@pytest.mark.parametrize("n", [1, 40])
def test_queries_of_any_size(n):
    """Tiny and huge values, zeros, one outlier; rows that are not finite give NaN and touch no other row."""
    heads, kv, dim, page, lengths = 4, 1, 128, 64, [150]
    rng = np.random.default_rng(12)
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, kv, page, dim)
    q = queries(rng, n, heads, dim)
    q[:, 0] *= 1e-30
    q[:, 1] = 0.0
    q[:, 2, 3] = 300.0
    check(q, cache, table, lengths, [0, n], page)
    q[:, 0] *= 1e33
    check(q, cache, table, lengths, [0, n], page, scale=1e-4)
    clean, _ = pvq.fp8_attention(q, cache, ints(table), ints(lengths), ints([0, n]), lse=True)
    q[0, 2, 5], q[0, 3, 7] = float("nan"), float("inf")
    out, lse = pvq.fp8_attention(q, cache, ints(table), ints(lengths), ints([0, n]), lse=True)
    assert torch.isnan(out[0, 2:]).all() and torch.isnan(lse[0, 2:]).all()
    assert torch.equal(out[0, :2], clean[0, :2]) and torch.equal(out[1:], clean[1:])


@pytest.mark.parametrize("n", [1, 5, 60])
def test_nan_in_keys_stays_where_it_is_seen(n):
    """A key that is NaN makes NaN of the rows that see it, and of no other; where no row sees a token, neither matters."""
    heads, kv, dim, page, length = 2, 1, 64, 32, 200
    rng = np.random.default_rng(13)
    table, pool = tables(rng, [length], page)
    cache = filled(rng, table, [length], pool, kv, page, dim)
    q = queries(rng, n, heads, dim)
    args = ints(table), ints([length]), ints([0, n])
    clean = pvq.fp8_attention(q, cache, *args, window=64)
    def spoil(c, at):
        c.view(torch.uint8)[table[0][at // page], 0, at % page, 3] = 0xff
    spoil(cache.k, length - n - 64)
    spoil(cache.v, length - n - 64)  # the first row's window begins behind it
    assert torch.equal(pvq.fp8_attention(q, cache, *args, window=64), clean)
    spoil(cache.k, length - 1)  # the last row's own
    out = pvq.fp8_attention(q, cache, *args, window=64)
    assert torch.isnan(out[-1]).all() and torch.equal(out[:-1], clean[:-1])


def test_pages_that_are_not_there():
    """Numbers outside the pool are told, and count as zeros; so is a table that is too short."""
    heads, kv, dim, page = 4, 2, 64, 16
    rng = np.random.default_rng(14)
    table, pool = tables(rng, [100, 100], page)
    cache = filled(rng, table, [100, 100], pool, kv, page, dim)
    status = torch.zeros(1, dtype=I32, device="cuda")
    for n in (1, 30):
        q = queries(rng, 2 * n, heads, dim)
        bad = table.copy()
        bad[0, 2], bad[1, 0] = pool, -3
        starts = [0, n, 2 * n]
        status.zero_()
        out, lse = pvq.fp8_attention(q, cache, ints(bad), ints([100, 100]), ints(starts), lse=True, status=status)
        assert int(status) == pvq.STATUS_BAD_PAGE
        compare(out, lse, q, cache, bad, [100, 100], starts, page)
        status.zero_()
        pvq.fp8_attention(q, cache, ints(table), ints([100, 100]), ints(starts), status=status)
        assert int(status) == 0
        out, lse = pvq.fp8_attention(q, cache, ints(table[:, :3]), ints([100, 100]), ints(starts), lse=True, causal=False, status=status)
        compare(out, lse, q, cache, table[:, :3], [100, 100], starts, page, causal=False)
        assert int(status) == pvq.STATUS_BAD_PAGE
        for odd in ([7, 2, 5], [-1, 2 ** 31 - 1, 3], [2 * n, 2 * n, 2 * n]):
            pvq.fp8_attention(q, cache, ints(table), ints([100, -4]), ints(odd))
    torch.cuda.synchronize()


def test_views_other_rows_and_orders():
    """Queries inside one product's result, outputs with steps, pages with tokens first; rows of no sequence stay as they were."""
    heads, kv, dim, page, lengths, starts = 6, 2, 64, 32, [70, 300], [2, 5, 45]
    rng = np.random.default_rng(15)
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, kv, page, dim)
    both = queries(rng, 50, heads + 2 * kv, dim)
    q = both[:, :heads]
    out = torch.full((50, heads + 1, 2 * dim), 3.0, dtype=torch.bfloat16, device="cuda")
    other = pvq.Fp8Cache(*(c.transpose(1, 2).contiguous().transpose(1, 2) for c in cache[:2]), *cache[2:])
    got, lse = pvq.fp8_attention(q, other, ints(table), ints(lengths), ints(starts), lse=True, out=out[:, 1:, dim:])
    compare(out[:, 1:, dim:], lse, q, cache, table, lengths, starts, page)
    assert (out[:, :1] == 3.0).all() and (out[:, :, :dim] == 3.0).all() and (out[:2] == 3.0).all() and (out[45:] == 3.0).all()
    plain = pvq.fp8_attention(q.contiguous(), cache, ints(table), ints(lengths), ints(starts))
    assert torch.equal(plain[2:45], out[2:45, 1:, dim:])


@pytest.mark.parametrize("new", [1, 20])
def test_write_and_attend_captured_and_replayed(new):
    """A step of a layer, captured once and replayed as the sequences grow; two graphs at once on two streams."""
    heads, kv, dim, page, seqs, steps = 8, 2, 64, 16, 3, 4
    rng = np.random.default_rng(16 + new)
    start = [5, 0, 90]
    final = [x + new * steps for x in start]
    table, pool = tables(rng, final, page)
    starts = None if new == 1 else ints([i * new for i in range(seqs + 1)])
    sides = []
    for i in range(2):
        cache = filled(np.random.default_rng(40 + i), table, start, pool, kv, page, dim)
        both = queries(rng, seqs * new, heads + 2 * kv, dim)
        side = dict(cache=cache, both=both, lengths=ints([x + new for x in start]), table=ints(table), stream=torch.cuda.Stream())

        def step(side=side, both=both):
            q, k, v = both[:, :heads], both[:, heads:heads + kv], both[:, heads + kv:]
            pvq.fp8_cache_write(k, v, side["cache"], side["table"], side["lengths"], starts)
            return pvq.fp8_attention(q, side["cache"], side["table"], side["lengths"], starts, lse=True)

        kept = [c.clone() for c in cache]
        with torch.cuda.stream(side["stream"]):
            step()
        torch.cuda.synchronize()
        for c, k in zip(cache, kept):
            c.view(torch.uint8).copy_(k.view(torch.uint8))
        side["graph"] = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(side["graph"], stream=side["stream"]):
            side["result"] = step()
        sides.append(side)
    host_starts = None if new == 1 else [i * new for i in range(seqs + 1)]
    for n in range(steps):
        lengths = [x + new * (n + 1) for x in start]
        befores = []
        for side in sides:
            side["both"].copy_(queries(rng, seqs * new, heads + 2 * kv, dim, 1.0 + n))
            side["lengths"].copy_(ints(lengths))
            befores.append(ref.held(side["cache"]))
        torch.cuda.synchronize()
        for side in sides:
            with torch.cuda.stream(side["stream"]):
                side["graph"].replay()
        torch.cuda.synchronize()
        for side, (codes, exponents) in zip(sides, befores):
            both = side["both"]
            for i, x in enumerate((both[:, heads:heads + kv], both[:, heads + kv:])):
                ref.write(codes[i], exponents[i], to64(x), table, lengths, host_starts, page)
            got, e = ref.held(side["cache"])
            for i in range(2):
                assert np.array_equal(got[i], codes[i], equal_nan=True) and np.array_equal(e[i], exponents[i])
            compare(*side["result"], both[:, :heads], side["cache"], table, lengths, host_starts, page)


def test_many_sequences():
    """More sequences than a block has threads, most of them short or empty."""
    heads, kv, dim, page, seqs = 2, 1, 32, 16, 700
    rng = np.random.default_rng(18)
    lengths = [int(x) for x in rng.integers(0, 40, seqs)]
    lengths[500] = 5000
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, kv, page, dim)
    check(queries(rng, seqs, heads, dim), cache, table, lengths, None, page)
    new = [int(x) for x in rng.integers(0, 4, seqs)]
    starts = [0] + [int(x) for x in np.cumsum(new)]
    lengths = [max(a, b) for a, b in zip(lengths, new)]
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, kv, page, dim)
    check(queries(rng, starts[-1], heads, dim), cache, table, lengths, starts, page)


def test_a_pool_beyond_32_bits():
    pages, kv, page, dim, heads = 270000, 1, 128, 128, 4  # 4.4 GB
    rng = np.random.default_rng(19)
    cache = pvq.alloc_fp8_cache(pages, kv, page, dim)
    table = np.array([[pages - 1, 0, 262143, 262145]])
    few = filled(rng, np.array([[0, 1, 2, 3]]), [450], 4, kv, page, dim)
    for big, c in zip(cache, few):
        for i, pid in enumerate(table[0]):
            big.view(torch.uint8)[pid] = c.view(torch.uint8)[i]
    for n in (1, 70):
        q = queries(rng, n, heads, dim)
        assert torch.equal(pvq.fp8_attention(q, cache, ints(table), ints([450]), ints([0, n])),
                           pvq.fp8_attention(q, few, ints([[0, 1, 2, 3]]), ints([450]), ints([0, n])))

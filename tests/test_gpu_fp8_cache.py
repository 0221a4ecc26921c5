"""The 8-bit key and value cache against its definition: writing and reading it."""
import numpy as np
import pytest
import torch

import fp8_cache_reference as ref
from fp8_reference import to64
from paper_2410_16926_b200 import pvq

pytestmark = pytest.mark.gpu
I32 = torch.int32


def ints(x):
    return torch.tensor(x, dtype=I32, device="cuda")


def new_cache(pages, heads, page, dim, fill=0x35, tokens_first=False):
    """Pages full of what is not to be touched; `tokens_first`: laid out [pages][page][heads][dim]."""
    def codes():
        shape = (pages, page, heads, dim) if tokens_first else (pages, heads, page, dim)
        c = torch.full(shape, fill, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        return c.transpose(1, 2) if tokens_first else c
    return pvq.Fp8Cache(codes(), codes(), *(torch.full((pages, heads), 130, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu) for _ in range(2)))


def tables(rng, lengths, page, spare=2):
    """A table with pages in disorder, -7 behind each sequence's last, and the size of the pool."""
    counts = [-(-n // page) for n in lengths]
    pool = sum(counts) + spare
    order = list(rng.permutation(pool))
    t = np.full((len(lengths), max(1, max(counts))), -7)
    for s, n in enumerate(counts):
        t[s, :n] = [order.pop() for _ in range(n)]
    return t, pool


def same(cache, codes, exponents):
    got, e = ref.held(cache)
    for i in range(2):
        assert np.array_equal(e[i], exponents[i]), "scales"
        assert np.array_equal(got[i], codes[i], equal_nan=True), "codes"


def values(rng, shape, dtype, scale):
    x = rng.standard_normal(shape) * scale
    return torch.from_numpy(x).to(dtype).cuda()


STEPS = [  # page, dim, heads, dtype, new tokens of each sequence in each step
    (16, 128, 8, torch.bfloat16, [[1, 17, 40, 0, 3], [1, 1, 1, 1, 1], [16, 0, 5, 2, 33]]),
    (32, 64, 3, torch.float32, [[5, 31, 32, 33], [27, 1, 0, 64], [1, 1, 1, 1]]),
    (64, 16, 1, torch.bfloat16, [[100, 1], [28, 63], [1, 1], [200, 130]]),
    (128, 96, 2, torch.float32, [[127, 128, 129, 1], [1, 1, 1, 1], [2, 300, 0, 127]]),
    (128, 128, 4, torch.bfloat16, [[1], [126], [1], [1], [256]]),
]


@pytest.mark.parametrize("tokens_first", [False, True])
@pytest.mark.parametrize("page,dim,heads,dtype,steps", STEPS)
def test_steps_of_writing_and_reading(page, dim, heads, dtype, steps, tokens_first):
    rng = np.random.default_rng(page + dim)
    final = [sum(s[i] for s in steps) for i in range(len(steps[0]))]
    table, pool = tables(rng, final, page)
    cache = new_cache(pool, heads, page, dim, tokens_first=tokens_first)
    codes, exponents = ref.held(cache)
    lengths = [0] * len(final)
    for n, step in enumerate(steps):
        lengths = [a + b for a, b in zip(lengths, step)]
        starts = [3]  # rows in front of the first sequence and behind the last belong to none
        for b in step:
            starts.append(starts[-1] + b)
        rows = starts[-1] + 2
        # scales go up and down from step to step: pages that are half full have to be rounded again, or keep what they have
        k, v = values(rng, (rows, heads, dim), dtype, 10.0 ** (n % 3)), values(rng, (rows, heads, dim), dtype, 0.1 * 30.0 ** (-n))
        single = all(b == 1 for b in step) and n % 2 == 1
        if single:
            k, v, starts = k[3:3 + len(step)], v[3:3 + len(step)], None
        status = torch.zeros(1, dtype=I32, device="cuda")
        pvq.fp8_cache_write(k, v, cache, ints(table), ints(lengths), None if single else ints(starts), status=status)
        for x, c, e in zip((k, v), codes, exponents):
            ref.write(c, e, to64(x), table, lengths, starts, page)
        same(cache, codes, exponents)
        assert int(status) == 0
    starts = [0]
    for b in final:
        starts.append(starts[-1] + b)
    for out_dtype in (torch.float32, torch.bfloat16):
        got = pvq.fp8_cache_read(cache, ints(table), ints(lengths), ints(starts), rows=starts[-1], dtype=out_dtype)
        for x, c, e in zip(got, codes, exponents):
            want = np.concatenate([ref.sequence(c, e, table[s], lengths[s], page).transpose(1, 0, 2) for s in range(len(final))])
            assert x.dtype == out_dtype and np.array_equal(to64(x), want)


def test_a_growing_scale_rounds_what_the_page_holds():
    rng = np.random.default_rng(5)
    table, lengths = np.array([[1]]), 0
    cache = new_cache(2, 2, 64, 32)
    codes, exponents = ref.held(cache)
    for scale in (0.0, 1e-9, 1e-9, 3e-7, 0.0, 5.0, 1e3, 2.0, 1e15, 1.0):  # (what is written first is zeros; codes become subnormal, then 0)
        lengths += 1
        k, v = values(rng, (1, 2, 32), torch.float32, scale), values(rng, (1, 2, 32), torch.float32, scale * 7)
        pvq.fp8_cache_write(k, v, cache, ints(table), ints([lengths]))
        ref.write(codes[0], exponents[0], to64(k), table, [lengths], None, 64)
        ref.write(codes[1], exponents[1], to64(v), table, [lengths], None, 64)
        same(cache, codes, exponents)


def test_what_is_not_finite_or_out_of_the_range():
    table = ints([[0]])
    cache = new_cache(1, 1, 16, 16)
    x = torch.zeros(3, 1, 16, device="cuda")
    x[0, 0, :6] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38, -3e38, 1.0])
    y = torch.full((3, 1, 16), 1e-30, device="cuda")
    y[1, 0, 0] = 448.0 * 2.0 ** -41
    pvq.fp8_cache_write(x, y, cache, table, ints([3]), ints([0, 3]))
    codes, e = ref.held(cache)
    assert e[0][0, 0] == 40 and e[1][0, 0] == -40
    assert np.isnan(codes[0][0, 0, 0, :3]).all() and list(codes[0][0, 0, 0, 3:6]) == [448.0, -448.0, 0.0]
    assert codes[1][0, 0, 1, 0] == 224.0 and (codes[1][0, 0, 0] == 0).all()
    # a NaN that the page holds stays one where the scale grows, and does not make it grow
    cache = new_cache(1, 1, 16, 16)
    pvq.fp8_cache_write(x[2:] + float("nan"), x[2:], cache, table, ints([1]))
    pvq.fp8_cache_write(x[2:] + 5.0, x[2:], cache, table, ints([2]))
    codes, e = ref.held(cache)
    assert e[0][0, 0] == -6 and np.isnan(codes[0][0, 0, 0]).all() and (codes[0][0, 0, 1] == 320.0).all()


def test_positions_without_a_place_are_left_out_and_told():
    """Page numbers outside the pool, lengths beyond the table, below the rows and below zero, starts that go back or beyond."""
    rng = np.random.default_rng(6)
    page, heads, dim = 16, 2, 32
    cases = [  # table, lengths, starts, rows, told
        ([[0, 99], [1, -1]], [20, 20], [0, 20, 40], 40, True),
        ([[0, 1]], [40], [0, 40], 40, True),
        ([[0, 1]], [5], [0, 9], 9, True),
        ([[0, 1], [2, 3]], [-5, 3], [0, 2, 5], 5, True),
        ([[0, 1], [2, 3]], [0, 3], [0, 0, 3], 3, False),
        ([[0, 1]], [2 ** 31 - 1], [0, 7], 7, True),
    ]
    for table, lengths, starts, rows, told in cases:
        cache = new_cache(4, heads, page, dim)
        codes, exponents = ref.held(cache)
        k, v = values(rng, (rows, heads, dim), torch.float32, 1.0), values(rng, (rows, heads, dim), torch.float32, 2.0)
        status = torch.zeros(1, dtype=I32, device="cuda")
        pvq.fp8_cache_write(k, v, cache, ints(table), ints(lengths), ints(starts), status=status)
        for x, c, e in zip((k, v), codes, exponents):
            ref.write(c, e, to64(x), np.array(table), lengths, starts, page)
        same(cache, codes, exponents)
        assert (int(status) == pvq.STATUS_BAD_PAGE) == told
        status.zero_()
        out = tuple(torch.full((rows, heads, dim), 7.0, device="cuda") for _ in range(2))
        pvq.fp8_cache_read(cache, ints(table), ints(lengths), ints(starts), rows=rows, dtype=torch.float32, out=out, status=status)
        assert (int(status) == pvq.STATUS_BAD_PAGE) == told
        have = {r: (pid, t) for r, pid, t, _ in ref.places(np.array(table), lengths, starts, rows, page) if 0 <= pid < 4}
        for x, c, e in zip(out, codes, exponents):
            for r in range(rows):
                want = c[have[r][0], :, have[r][1]] * np.exp2(e[have[r][0]].astype(float))[:, None] if r in have else np.zeros((heads, dim))
                assert np.array_equal(to64(x[r]), want)
    # starts that make no sense: nothing outside is touched (what is written is not defined)
    cache = new_cache(4, heads, page, dim)
    for starts in ([5, 2, 9], [-4, 100, 3], [9, 9, 9], [2 ** 31 - 1, 0, 2 ** 31 - 1]):
        pvq.fp8_cache_write(k[:9].expand(9, -1, -1) if k.shape[0] >= 9 else values(rng, (9, heads, dim), torch.float32, 1.0),
                            values(rng, (9, heads, dim), torch.float32, 1.0), cache, ints([[0], [1]]), ints([9, 3]), ints(starts))
        pvq.fp8_cache_read(cache, ints([[0], [1]]), ints([9, 3]), ints(starts), rows=9)
    torch.cuda.synchronize()
    assert (cache.k[2:].view(torch.uint8) == 0x35).all() and (cache.v_scales[2:].view(torch.uint8) == 130).all()


def test_views_and_rows_of_no_sequence():
    """Keys and values as parts of one product's result, a cache that is a part of a larger one, outputs with steps."""
    rng = np.random.default_rng(7)
    heads, dim, page = 2, 48, 32
    both = values(rng, (20, 3 * heads, dim), torch.bfloat16, 1.0)
    k, v = both[:, :heads], both[:, heads:2 * heads]
    pool = new_cache(4, 5, page, 80)
    cache = pvq.Fp8Cache(pool.k[1:3, 1:3, :, 16:64], pool.v[1:3, 1:3, :, 16:64], pool.k_scales[1:3, 1:3], pool.v_scales[1:3, 1:3])
    codes, exponents = ref.held(pool)
    table, lengths, starts = np.array([[1], [0]]), [9, 7], [2, 11, 18]
    pvq.fp8_cache_write(k, v, cache, ints(table), ints(lengths), ints(starts))
    for x, c, e in zip((k, v), codes, exponents):
        ref.write(c[1:3, 1:3, :, 16:64], e[1:3, 1:3], to64(x), table, lengths, starts, page)
    same(pool, codes, exponents)
    out = torch.full((2, 20, 3, 64), 5.0, device="cuda", dtype=torch.bfloat16)
    got = pvq.fp8_cache_read(cache, ints(table), ints(lengths), ints(starts), rows=20, out=(out[0, :, 1:, 8:56], out[1, :, 1:, 8:56]))
    assert got[0].data_ptr() == out[0, :, 1:, 8:56].data_ptr()
    want = to64(out) * 0 + 5.0
    for i in range(2):
        for s in range(2):
            seq = ref.sequence(codes[i][1:3, 1:3, :, 16:64], exponents[i][1:3, 1:3], table[s], lengths[s], page)
            want[i, starts[s]:starts[s + 1], 1:, 8:56] = seq.transpose(1, 0, 2)
    assert np.array_equal(to64(out), want)


def test_a_pool_beyond_32_bits():
    """Pages whose codes lie more than 2^32 bytes into the pool, and whose rows lie more than 2^31 elements into theirs."""
    pages, heads, page, dim = 270000, 1, 128, 128  # 4.4 GB
    cache = pvq.alloc_fp8_cache(pages, heads, page, dim)
    table = np.array([[pages - 1, 0, 262143, 262145]])
    rng = np.random.default_rng(8)
    big = torch.zeros((400, 2, 3000000), dtype=torch.bfloat16, device="cuda")
    k = big[:, :1, 1000:1128]
    k.copy_(values(rng, (400, 1, dim), torch.bfloat16, 1.0))
    pvq.fp8_cache_write(k, k, cache, ints(table), ints([450]), ints([0, 400]))
    got = pvq.fp8_cache_read(cache, ints(table), ints([450]), ints([0, 400]), rows=400, dtype=torch.float32)
    x = to64(k)
    for g in got:
        for a, b in ((0, 78), (78, 206), (206, 334), (334, 400)):  # (the first page held 50 tokens of whatever: its scale may be larger)
            e = ref.page_scale(np.abs(x[a:b]).max())
            if a:
                assert np.array_equal(to64(g[a:b]), ref.clamped(x[a:b], e) * 2.0 ** e)


def test_what_does_not_fit_together_is_refused():
    cache, table, lengths, starts = new_cache(4, 2, 16, 32), ints([[0], [1]]), ints([3, 4]), ints([0, 3, 7])
    x = torch.zeros(7, 2, 32, device="cuda")
    q = torch.zeros(7, 4, 32, device="cuda", dtype=torch.bfloat16)
    good = dict(cache=cache, table=table, lengths=lengths, starts=starts)

    def refused(error, x=x, y=x, q=q, **change):
        a = {**good, **change}
        for call in (lambda: pvq.fp8_cache_write(x, y, a["cache"], a["table"], a["lengths"], a["starts"]),
                     lambda: pvq.fp8_cache_read(a["cache"], a["table"], a["lengths"], a["starts"], rows=7),
                     lambda: pvq.fp8_attention(q, a["cache"], a["table"], a["lengths"], a["starts"])):
            with pytest.raises(error):
                call()

    refused(ValueError, table=ints([[0]]))
    refused(ValueError, lengths=ints([3]))
    refused(ValueError, starts=ints([0, 7]))
    refused(ValueError, starts=None)                                   # seven rows, two sequences
    refused(TypeError, table=table.long())
    refused(TypeError, lengths=lengths.float())
    refused(ValueError, table=ints([0, 1]))
    refused(ValueError, table=ints([[0, 1], [2, 3]]).t())
    refused(ValueError, lengths=lengths.cpu())
    refused(TypeError, cache=cache._replace(k=cache.k.view(torch.uint8)))
    refused(TypeError, cache=cache._replace(v_scales=cache.v_scales.view(torch.uint8)))
    refused(ValueError, cache=cache._replace(v=cache.v[:3]))
    refused(ValueError, cache=cache._replace(k_scales=cache.k_scales[:, :1]))
    refused(ValueError, cache=cache._replace(v=new_cache(4, 2, 16, 32, tokens_first=True).v))
    refused(ValueError, cache=cache._replace(k=cache.k.transpose(2, 3), v=cache.v.transpose(2, 3)))
    refused(pvq.PvqError, cache=pvq.Fp8Cache(cache.k[:, :, :15], cache.v[:, :, :15], *cache[2:]))
    with pytest.raises(TypeError):
        pvq.fp8_cache_write(x, x.bfloat16(), cache, table, lengths, starts)
    with pytest.raises(ValueError):
        pvq.fp8_cache_write(x, x[:6], cache, table, lengths, starts)
    with pytest.raises(ValueError):
        pvq.fp8_cache_write(x[:, :, :16], x[:, :, :16], cache, table, lengths, starts)
    with pytest.raises(ValueError):
        pvq.fp8_cache_write(x.requires_grad_(), x, cache, table, lengths, starts)
    with pytest.raises(ValueError):
        pvq.fp8_cache_read(cache, table, lengths, starts)               # how many rows?
    with pytest.raises(TypeError):
        pvq.fp8_cache_read(cache, table, lengths, starts, rows=7, out=(x.detach(), None))
    with pytest.raises(TypeError):
        pvq.fp8_attention(q.float(), cache, table, lengths, starts)
    with pytest.raises(ValueError):
        pvq.fp8_attention(q[:, :3], cache, table, lengths, starts)
    with pytest.raises(ValueError):
        pvq.fp8_attention(q, cache, table, lengths, starts, out=q[:6])
    with pytest.raises(ValueError):
        pvq.fp8_attention(q.clone().requires_grad_(), cache, table, lengths, starts)
    for wrong in (dict(window=-1), dict(window=3, causal=False), dict(scale=0.0), dict(scale=float("nan"))):
        with pytest.raises(pvq.PvqError):
            pvq.fp8_attention(q, cache, table, lengths, starts, **wrong)
    version = cache.k._version
    pvq.fp8_cache_write(x.detach(), x.detach(), cache, table, lengths, starts)
    assert cache.k._version > version

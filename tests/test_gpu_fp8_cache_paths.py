"""The operators of the 8-bit cache on every path that their sizes choose, the path itself asserted, so that a change of the rules cannot
take a path away from its tests; every dim, group of heads and page; calls in which a long prompt meets single tokens."""
import re

import numpy as np
import pytest
import torch
from cuda.bindings import driver

import fp8_cache_reference as ref
from fp8_reference import to64
from paper_2410_16926_b200 import pvq
from test_gpu_fp8_attention import check, filled, queries
from test_gpu_fp8_cache import I32, ints, new_cache, same, tables, values

pytestmark = pytest.mark.gpu


def kernels(call):
    """[(name, first template argument)] of a call's launches."""
    def done(r):
        assert r[0] == driver.CUresult.CUDA_SUCCESS, r[0]
        return r[1] if len(r) == 2 else r[1:]

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        kept = call()
    raw = driver.CUgraph(graph.raw_cuda_graph())
    nodes = done(driver.cuGraphGetNodes(raw, done(driver.cuGraphGetNodes(raw, 0))[1]))[0]
    found = []
    for node in nodes:
        p = done(driver.cuGraphKernelNodeGetParams(node))
        name = done(driver.cuFuncGetName(p.func) if int(p.func) else driver.cuKernelGetName(p.kern)).decode()
        base, rest = re.search(r"\d+([a-z_]+_kernel)(.*)", name).groups()
        first = re.match(r"ILi(\d+)E|I(f)E|I13(__nv_bfloat16)E", rest)
        found.append((base, (first.group(1) or first.group(2) or first.group(3)) if first else None))
    del kept
    return sorted(found)


@pytest.mark.parametrize("heads,kv,n,rows", [(2, 2, 1, 4), (8, 2, 1, 4), (4, 1, 2, 8), (16, 4, 3, 16), (13, 1, 1, 16), (32, 2, 2, 32), (32, 1, 1, 32), (8, 2, 9, 256),
                                             (33, 1, 1, 256), (128, 1, 1, 256), (4, 4, 40, 256), (10, 2, 70, 256)])
@pytest.mark.parametrize("lengths", [[300, 41, 130], [5000, 129, 0], [40000, 129, 500]])
def test_attention(heads, kv, n, rows, lengths):
    dim, page = 128, 32
    lengths = [max(n, length) for length in lengths]
    rng = np.random.default_rng(heads + n)
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, kv, page, dim)
    starts = None if n == 1 else [n * i for i in range(len(lengths) + 1)]
    q = queries(rng, n * len(lengths), heads, dim)
    device = ints(table), ints(lengths), None if starts is None else ints(starts)
    expected = {("attention_many_kernel", None) if rows == 256 else ("attention_few_kernel", str(rows))}
    if n > 1 or rows > 16 or lengths[0] > 16 * 8 * 128:  # (otherwise an item for a cluster)
        expected.add(("attention_join_kernel", str(rows)))
    assert set(kernels(lambda: pvq.fp8_attention(q, cache, *device))) == expected
    check(q, cache, table, lengths, starts, page)


@pytest.mark.parametrize("group,seqs,kv,length", [(4, 1, 1, 100), (1, 1, 1, 200), (7, 1, 2, 500), (16, 1, 3, 900), (4, 1, 30, 2000), (2, 1, 31, 2000), (8, 33, 2, 1000),
                                                   (5, 67, 1, 1000), (16, 148, 1, 300), (3, 148, 2, 700), (4, 148, 2, 1), (1, 1, 296, 300)])
def test_single_tokens_in_clusters(group, seqs, kv, length):
    """Clusters of one, two, four and eight blocks, some of which may have no tile; sequences of every length."""
    rng = np.random.default_rng(seqs + kv + group)
    dim, page = 64, 32
    lengths = [length] + [int(x) for x in rng.integers(0, length, seqs - 1)]
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, kv, page, dim)
    q = queries(rng, seqs, group * kv, dim)
    device = ints(table), ints(lengths)
    assert [name for name, _ in kernels(lambda: pvq.fp8_attention(q, cache, *device))] == ["attention_few_kernel"]
    check(q, cache, table, lengths, None, page)
    check(q, cache, table, lengths, None, page, window=130)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dim", range(16, 129, 16))
def test_every_dim_and_page(dim, page):
    rng = np.random.default_rng(dim * page)
    lengths = [page * 3 + 1, 259, 128]
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, 2, page, dim)
    check(queries(rng, 3, 6, dim), cache, table, lengths, None, page)
    for heads, n in ((6, 1), (10, 6), (4, 30)):
        check(queries(rng, 3 * n, heads, dim), cache, table, lengths, [0, n, 2 * n, 3 * n], page)
        check(queries(rng, 3 * n, heads, dim), cache, table, lengths, [0, n, 2 * n, 3 * n], page, window=100)


@pytest.mark.parametrize("group", [1, 2, 3, 5, 7, 12, 31, 64, 100, 128])
def test_every_group_of_heads(group):
    rng = np.random.default_rng(group)
    lengths, page, dim = [290, 77], 64, 64
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, 2, page, dim)
    check(queries(rng, 2, 2 * group, dim), cache, table, lengths, None, page)
    for starts in ([0, 1, 2], [0, 5, 8], [0, 77, 130]):
        check(queries(rng, starts[-1], 2 * group, dim), cache, table, lengths, starts, page)


@pytest.mark.parametrize("how", [dict(), dict(window=50), dict(causal=False)], ids=str)
def test_long_prompts_and_single_tokens_in_one_call(how):
    """What the rule takes for few rows has a sequence of many, and the other way round."""
    rng = np.random.default_rng(3)
    page, dim = 16, 64
    for new in ([300] + [1] * 40, [2] * 3 + [90], [1, 0, 600, 0, 1]):
        lengths = [n + int(x) for n, x in zip(new, rng.integers(0, 300, len(new)))]
        table, pool = tables(rng, lengths, page)
        cache = filled(rng, table, lengths, pool, 1, page, dim)
        starts = [0] + [int(x) for x in np.cumsum(new)]
        check(queries(rng, starts[-1], 4, dim), cache, table, lengths, starts, page, **how)


def test_one_page_in_two_tables():
    """A prefix that two sequences share is read by both."""
    rng = np.random.default_rng(4)
    page, dim, lengths = 32, 64, [70, 90]
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, 2, page, dim)
    table[1, :2] = table[0, :2]
    for n in (1, 20):
        check(queries(rng, 2 * n, 4, dim), cache, table, lengths, [0, n, 2 * n], page)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new,few", [(None, True), ([1, 2, 3], True), ([8, 8, 8], True), ([9, 9, 9], False), ([20, 1, 1], True), ([200, 3, 1], False)])
def test_writing(new, few, dtype, page):
    rng = np.random.default_rng(page)
    heads, dim, before = 3, 80, [5, page - 1, 3 * page]
    counts = [1, 1, 1] if new is None else new
    lengths = [a + b for a, b in zip(before, counts)]
    table, pool = tables(rng, lengths, page)
    cache = new_cache(pool, heads, page, dim)
    codes, exponents = ref.held(cache)
    for grow in (1.0, 30.0, 0.01):  # (the second time the pages' scales grow)
        starts = None if new is None else [0] + [int(x) for x in np.cumsum(counts)]
        k, v = values(rng, (sum(counts), heads, dim), dtype, 1000.0 * grow), values(rng, (sum(counts), heads, dim), dtype, grow)
        k[-1, 1, 3], v[0, 2, 79] = float("nan"), -float("inf")
        args = ints(table), ints(lengths), None if starts is None else ints(starts)
        pvq.fp8_cache_write(k, v, cache, *args)
        for x, c, e in zip((k, v), codes, exponents):
            ref.write(c, e, to64(x), table, lengths, starts, page)
        same(cache, codes, exponents)
    spare = new_cache(pool, heads, page, dim)
    name = "cache_write_few_kernel" if few else "cache_write_kernel"
    assert kernels(lambda: pvq.fp8_cache_write(k, v, spare, *args)) == [(name, "f" if dtype == torch.float32 else "__nv_bfloat16")]


@pytest.mark.parametrize("rows", [1, 7, 300, 5000, 40000])
def test_reading(rows):
    """Blocks of each number of rows; many empty sequences among them."""
    rng = np.random.default_rng(rows)
    page, heads, dim = 16, 2, 48
    cuts = np.sort(rng.integers(0, rows + 1, 60))
    lengths = [int(x) for x in np.diff(np.concatenate([[0], cuts, [rows]]))]
    lengths[10:20] = [0] * 10
    total = sum(lengths)
    table, pool = tables(rng, lengths, page)
    cache = filled(rng, table, lengths, pool, heads, page, dim)
    starts = [0] + [int(x) for x in np.cumsum(lengths)]
    if total == 0:
        return
    codes, exponents = ref.held(cache)
    for dtype in (torch.bfloat16, torch.float32):
        for got, c, e in zip(pvq.fp8_cache_read(cache, ints(table), ints(lengths), ints(starts), rows=total, dtype=dtype), codes, exponents):
            want = np.concatenate([ref.sequence(c, e, table[s], n, page).transpose(1, 0, 2) for s, n in enumerate(lengths) if n])
            assert np.array_equal(to64(got), want)

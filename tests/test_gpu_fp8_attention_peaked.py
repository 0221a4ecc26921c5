"""Attention over the 8-bit cache for rows that one token leads by far: what the others hold together counts, however many they are and however small
each weight is; and values beside a channel that is much larger.  Against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2410_16926_b200 import pvq
from test_gpu_fp8_cache import ints, tables

pytestmark = pytest.mark.gpu
TILE = 128  # tokens that a row's weights are computed for at a time


def sequence(codes, scales, pages, length):
    """[head][token][dim] of a sequence in 64 bits, and the exponents of its tokens' scales, [head][token]."""
    e = scales.view(torch.uint8)[pages].double() - 127
    x = codes.view(torch.uint8)[pages].view(torch.float8_e4m3fn).double() * torch.exp2(e)[:, :, None, None]
    e = e[:, :, None].expand(-1, -1, codes.shape[2])
    return x.transpose(0, 1).flatten(1, 2)[:, :length], e.transpose(0, 1).flatten(1, 2)[:, :length]


def worst(out, lse, q, cache, table, lengths, n, scale):
    """The largest share of what each result may be off that it is off.

    What it may be off: a score by 2^-17 of the row's largest query value times the sum of the key's magnitudes (queries are two codes), by dim + 32 steps of 2^-23 of
    the products' magnitudes, and, as an exponent of two, by four roundings of at most its magnitude + 128; 2^x by 2^-21 of itself; a weight by 2^-8 of itself;
    or, up to 32 rows of a sequence and head, by 2^-22 of the largest weight times its page's scale among the tile's 128 tokens, beyond by 2^-32 of the row's
    largest one; sums of c weights by (c / 32 + 64) 2^-23 of their magnitudes; the result by 2^-8 of itself.  No term goes by the largest value."""
    heads, kv, dim = q.shape[1], cache.k.shape[1], q.shape[2]
    group, most = heads // kv, 0.0
    for s, length in enumerate(lengths):
        pages = torch.as_tensor(np.ascontiguousarray(table[s][:-(-length // cache.k.shape[2])])).cuda()
        (k, _), (v, e) = sequence(cache.k, cache.k_scales, pages, length), sequence(cache.v, cache.v_scales, pages, length)
        rows = q[s * n:(s + 1) * n].double()
        seen = torch.arange(length, device="cuda")[None, :] <= torch.arange(length - n, length, device="cuda")[:, None]
        for h in range(heads):
            x, kh, vh, eh = rows[:, h], k[h // group], v[h // group], e[h // group]
            w = (scale * (x @ kh.T)).masked_fill(~seen, -math.inf)
            want_lse = torch.logsumexp(w, dim=1)
            p = torch.exp(w - want_lse[:, None])
            want = p @ vh
            off = scale * (2.0 ** -17 * x.abs().amax(dim=1)[:, None] * kh.abs().sum(dim=1) + (dim + 32) * 2.0 ** -23 * (x.abs() @ kh.abs().T))
            off = (off + (w.abs().masked_fill(~seen, 0.0) + 128) * 2.0 ** -22 + 2.0 ** -21).masked_fill(~seen, 0.0).amax(dim=1)
            at = p * torch.exp2(eh)  # weights as the products have them
            if n * group <= 32:
                tiles = torch.nn.functional.pad(at, (0, -length % TILE)).unflatten(1, (-1, TILE)).amax(dim=2)
                least = 2.0 ** -22 * tiles.repeat_interleave(TILE, dim=1)[:, :length]
            else:
                least = 2.0 ** -32 * at.amax(dim=1, keepdim=True).expand(-1, length)
            absolute = (least * torch.exp2(-eh)).masked_fill(~seen, 0.0) @ vh.abs()
            relative = 2.0 ** -8 + 2 * off + 2 * (length / 32 + 64) * 2.0 ** -23
            slack = 2.0 ** -8 * want.abs() + relative[:, None] * (p @ vh.abs()) + absolute + 2.0 ** -130
            most = max(most, float(((out[s * n:(s + 1) * n, h].double() - want).abs() / slack).max()))
            slack_lse = off + (length / 32 + 64) * 2.0 ** -23 + 2.0 ** -22 * want_lse.abs() + 2.0 ** -21
            most = max(most, float(((lse[s * n:(s + 1) * n, h].double() - want_lse).abs() / slack_lse).max()))
    return most


def led(rng, seqs, length, kv, page, dim, lead, spread, first=0):
    """Sequences whose token `first` leads a query of `lead` in its last dim by that, and has values of zero; the others' values have a mean of one."""
    lengths = [length] * seqs
    table, pool = tables(rng, lengths, page)
    g = torch.Generator(device="cuda").manual_seed(int(rng.integers(1 << 30)))
    rand = lambda: torch.randn((pool, kv, page, dim), generator=g, device="cuda")  # noqa: E731
    k, v = (rand() * spread * 64).to(torch.float8_e4m3fn), ((1 + 0.25 * rand()) * 64).to(torch.float8_e4m3fn)
    k.view(torch.uint8)[..., -1] = 0
    for s in range(seqs):
        at = table[s][first // page], slice(None), first % page
        k.view(torch.uint8)[at] = 0
        k.view(torch.uint8)[at + (-1,)] = 0x68  # 64
        v.view(torch.uint8)[at] = 0
    scales = [torch.full((pool, kv), 127 - 6, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu) for _ in range(2)]
    return pvq.Fp8Cache(k, v, *scales), table, lengths


def attended(rng, cache, table, lengths, n, heads, lead):
    dim = cache.k.shape[3]
    q = torch.from_numpy(rng.standard_normal((n * len(lengths), heads, dim)) / math.sqrt(dim)).to(torch.bfloat16).cuda()
    q[:, :, -1] = lead
    starts = None if n == 1 else ints([n * i for i in range(len(lengths) + 1)])
    return (q, *pvq.fp8_attention(q, cache, ints(table), ints(lengths), starts, scale=1.0, lse=True))


# sequences, tokens, heads of the cache: items in clusters, in many parts, and in a part or two (so that one has 30 000 tokens and more)
SIZES = [(1, 1500, 2), (2, 9000, 2), (64, 8200, 8), (40, 33000, 8)]


@pytest.mark.parametrize("spread", [0.0, 0.5])  # of the others' scores: the same for all, or normal
@pytest.mark.parametrize("lead", [4.0, 9.0, 12.3125, 13.0, 15.0, 18.0])
@pytest.mark.parametrize("n", [1, 4, 40])
@pytest.mark.parametrize("seqs,length,kv", SIZES)
def test_a_token_that_leads(seqs, length, kv, n, lead, spread):
    rng = np.random.default_rng(length + n)
    cache, table, lengths = led(rng, seqs, length, kv, 64, 32, lead, spread)
    q, out, lse = attended(rng, cache, table, lengths, n, 4 * kv, lead)
    shown = [0, seqs - 1] if seqs > 2 else range(seqs)  # (the others are alike)
    part = torch.cat([torch.arange(s * n, (s + 1) * n) for s in shown]).cuda()
    assert worst(out[part], lse[part], q[part], cache, table[list(shown)], [length] * len(shown), n, 1.0) <= 1.0


@pytest.mark.parametrize("first", [5000, 8199])  # the row's largest comes late: what was summed before stays
@pytest.mark.parametrize("n", [1, 2, 8, 40])
def test_a_token_that_leads_late(n, first):
    rng = np.random.default_rng(n)
    cache, table, lengths = led(rng, 40, 8200 + n, 8, 16, 64, 13.0, 0.5, first=first)
    q, out, lse = attended(rng, cache, table, lengths, n, 32, 13.0)
    assert worst(out[:n], lse[:n], q[:n], cache, table[:1], lengths[:1], n, 1.0) <= 1.0


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("n", [1, 4, 40])
def test_a_channel_that_leads(n, page):
    """One page has one value 2^9 times the others': the other channels, and the other pages, keep theirs."""
    rng = np.random.default_rng(page + n)
    cache, table, lengths = led(rng, 3, 3000, 2, page, 64, 0.0, 0.5)
    for s in range(3):
        at = table[s][1000 // page]
        cache.v_scales.view(torch.uint8)[at] += 9
        x = cache.v.view(torch.uint8)[at].view(torch.float8_e4m3fn).float() / 512  # (subnormal codes: 1/8 of 64 is left)
        x[:, 1000 % page, 7] = 400.0
        cache.v.view(torch.uint8)[at] = x.to(torch.float8_e4m3fn).view(torch.uint8)
    q, out, lse = attended(rng, cache, table, lengths, n, 8, 0.0)
    assert worst(out, lse, q, cache, table, lengths, n, 1.0) <= 1.0

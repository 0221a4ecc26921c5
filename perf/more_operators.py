"""What the operators of an 8-bit key and value cache are measured on.

The cache holds the keys and values of many sequences in pages of 16 to 128 tokens: e4m3 codes and one power-of-two
scale (e8m0) for each page and head, keys and values apart.  The operators that make and read it:

  - write: the new tokens' keys and values, quantised into the pages of their sequences; a page that is half full already
    keeps its scale, or takes a larger one, to which the codes that it holds are rounded again;
  - read: the values of a sequence's tokens;
  - attention: softmax(q k^T) v of the new tokens over everything their sequences hold, straight from the codes, for single
    tokens, a few tokens and prompts.

A case is one call.  All take the same description of a step: a table of pages for each sequence, its length with the
tokens of this step, and where its tokens begin among the step's rows (None: one token a sequence).
Heads are those of `inputs.py`'s decoder layer (32 heads of 128, 8 of them for keys and values), and others around it.
With `own` false everything is computed by elementary torch operations in 32 bits.
"""
import math

import torch

own = False

LARGEST = 448.0  # of e4m3
LEAST, MOST = -40, 40  # exponents of a page's scale


def listed():
    layer = dict(heads=32, kv=8, dim=128)
    return [
        # one decoded token of one conversation: what a call costs
        dict(name="write one token", op="write", seqs=1, new=1, length=1000, page=64, ragged=False, dtype="bf16", **layer),
        # a decoded token of each of many conversations
        dict(name="write a batch's tokens", op="write", seqs=256, new=1, length=2048, page=16, ragged=True, dtype="bf16", **layer),
        # prompts, behind what their conversations held before
        dict(name="write prompts", op="write", seqs=7, new=4001, length=6000, page=64, ragged=True, dtype="bf16", **layer),
        # a short prefix read back
        dict(name="read a prefix", op="read", seqs=1, new=777, length=777, page=32, ragged=False, dtype="f32", **layer),
        # all conversations of a batch read back, for instance to move them
        dict(name="read a batch", op="read", seqs=16, new=8192, length=8192, page=64, ragged=True, dtype="bf16", **layer),
        # one decoded token, short conversation: latency
        dict(name="attend one token", op="attend", seqs=1, new=1, length=1000, page=64, ragged=False, window=0, causal=True, lse=False, **layer),
        # a decoded token of each conversation of a batch
        dict(name="attend a batch's tokens", op="attend", seqs=64, new=1, length=8192, page=64, ragged=True, window=0, causal=True, lse=False, **layer),
        # one decoded token behind a very long document, to be joined with another part
        dict(name="attend far back", op="attend", seqs=1, new=1, length=200001, page=128, ragged=False, window=0, causal=True, lse=True, **layer),
        # a few drafted tokens of each conversation, sliding window
        dict(name="attend drafts", op="attend", seqs=33, new=5, length=3000, page=16, ragged=True, window=1024, causal=True, lse=False, **layer),
        # a prompt from its beginning
        dict(name="attend a prompt", op="attend", seqs=1, new=8192, length=8192, page=64, ragged=False, window=0, causal=True, lse=False, **layer),
        # pieces of prompts behind what was written before, of several conversations
        dict(name="attend pieces", op="attend", seqs=5, new=700, length=7000, page=32, ragged=True, window=0, causal=True, lse=False, **layer),
        # decoder rows over an encoder's states, which all of them see; a head of its own for each
        dict(name="attend an encoder's states", op="attend", seqs=12, new=333, length=1500, page=64, ragged=True, window=0, causal=False, lse=False,
             heads=16, kv=16, dim=64),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = ((32, 8, 128), (32, 8, 128), (32, 32, 128), (16, 16, 64), (8, 1, 128), (24, 8, 128), (28, 4, 128), (40, 8, 96), (12, 4, 80))


def draw(rng):
    heads, kv, dim = rng.choice(HEADS)
    case = dict(op=rng.choice(("write", "read", "attend", "attend", "attend", "attend")), page=rng.choice((16, 32, 64, 128)), ragged=rng.random() < 0.7,
                heads=heads, kv=kv, dim=dim)
    width = kv * dim / 1024  # of the layer's keys
    if case["op"] == "write":
        case["seqs"] = _log_uniform(rng, 1, 256)
        case["new"] = 1 if rng.random() < 0.4 else _log_uniform(rng, 2, 28000 / case["seqs"] / max(1, width) + 2)
        case["length"] = case["new"] + _log_uniform(rng, 1, 2048)
        case["dtype"] = rng.choice(("bf16", "bf16", "f32"))
    elif case["op"] == "read":
        case["seqs"] = _log_uniform(rng, 1, 64)
        case["length"] = case["new"] = _log_uniform(rng, 1, 60000 / case["seqs"] / max(1, width) + 2)
        case["dtype"] = rng.choice(("bf16", "f32"))
    else:
        case["seqs"] = _log_uniform(rng, 1, 128)
        kind = rng.random()
        if kind < 0.4:  # single tokens
            case["new"], most = 1, 320000
        elif kind < 0.6:  # a few
            case["new"], most = rng.randint(2, 16), 200000
        else:
            case["new"], most = _log_uniform(rng, 17, 4096), 60000
        case["seqs"] = min(case["seqs"], max(1, 8192 // case["new"]))
        pairs = 8192 * 8192 * 32 * 128 // (2 * case["heads"] * dim * case["seqs"] * case["new"])  # (all that the longest one has)
        case["length"] = max(case["new"], min(_log_uniform(rng, 64, 32768), int(most / case["seqs"] / max(1, width)), pairs))
        case["causal"] = rng.random() < 0.75
        case["window"] = _log_uniform(rng, 16, 4096) if case["causal"] and rng.random() < 0.25 else 0
        case["lse"] = rng.random() < 0.3
    return case


def _spread(most, count, ragged):
    """Lengths from a quarter of the longest up to it, the first the longest."""
    return [max(1, round(most * (1 - 0.75 * ((0.618034 * i) % 1.0)))) if ragged else most for i in range(count)]


def _sizes(case):
    """(length, new tokens) of each sequence."""
    lengths, new = _spread(case["length"], case["seqs"], case["ragged"]), _spread(case["new"], case["seqs"], case["ragged"])
    if case["op"] == "read":
        return [(n, n) for n in lengths]
    return [(max(a, b), b) for a, b in zip(lengths, new)]


def _dtype(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


# ---- inputs ---------------------------------------------------------------------------

def _exponent(amax):
    """Of the smallest power of two s with amax <= 448 s, within the format's range."""
    mantissa, exponent = torch.frexp(amax)  # amax = mantissa 2^exponent, mantissa in [1/2, 1): 448 is 0.875 2^9
    return torch.where(amax > 0, torch.clamp(exponent - 9 + (mantissa > 0.875).int(), LEAST, MOST), LEAST)


def _features(g, shape):
    """Normal values, one channel in fifty four times as large."""
    x = torch.randn(shape, generator=g, device="cuda")
    return x.mul_(torch.where(torch.rand((shape[1], 1, shape[3]), generator=g, device="cuda") < 0.02, 4.0, 1.0))


def _held(g, pages, case):
    x = _features(g, (pages, case["kv"], case["page"], case["dim"]))
    e = _exponent(x.abs().amax(dim=(2, 3)))
    codes = torch.ldexp(x, -e[:, :, None, None]).to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    sizes, page = _sizes(case), case["page"]
    counts = [-(-length // page) for length, _ in sizes]
    pages = sum(counts) + 3
    order = torch.randperm(pages, generator=g, device="cuda").int()
    table = torch.zeros((case["seqs"], max(counts)), dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(counts):
        table[s, :n] = order[at:at + n]
        at += n
    state = dict(case=case, table=table, lengths=_ints([length for length, _ in sizes]), rows=sum(n for _, n in sizes), most=max(n for _, n in sizes))
    starts = [0]
    for _, n in sizes:
        starts.append(starts[-1] + n)
    state["starts"] = _ints(starts) if case["new"] > 1 else None
    k, ks = _held(g, pages, case)
    v, vs = _held(g, pages, case)
    state["cache"] = (k, v, ks, vs)
    if case["op"] != "read":  # one product's result holds queries, keys and values side by side
        heads, kv, dim = case["heads"], case["kv"], case["dim"]
        both = torch.randn((state["rows"], heads + 2 * kv, dim), generator=g, device="cuda").mul_(1.5).to(_dtype(case))
        state["q"], state["k"], state["v"] = both[:, :heads], both[:, heads:heads + kv], both[:, heads + kv:]
    return state


# ---- the operators in plain form ---------------------------------------------------------

def _rows(state):
    """For each row of the step its sequence, its place among the sequence's rows, and its position."""
    rows = torch.arange(state["rows"], device="cuda")
    if state["starts"] is None:
        return rows, torch.zeros_like(rows), state["lengths"].long() - 1
    starts = state["starts"].long()
    s = torch.searchsorted(starts, rows, right=True) - 1
    i = rows - starts[s]
    return s, i, state["lengths"].long()[s] - (starts[s + 1] - starts[s]) + i


def _write_one(x, codes, scales, state, rows):
    table, page = state["table"].long(), codes.shape[2]
    s, i, position = rows
    pid, slot = table[s, position // page], position % page
    pages, kv = codes.shape[:2]
    x = x.float()
    amax = torch.zeros((pages, kv), device="cuda").index_reduce_(0, pid, x.abs().amax(dim=2), "amax")
    need, had = _exponent(amax), scales.view(torch.uint8).int() - 127
    written = torch.zeros(pages, dtype=torch.bool, device="cuda").index_fill_(0, pid, True)
    # the first page of each sequence's rows may hold tokens before them
    first = position[i == 0] if state["starts"] is not None else position
    first_pid = table[torch.arange(len(first), device="cuda"), first // page]
    kept = torch.zeros(pages, dtype=torch.bool, device="cuda").index_put_((first_pid,), first % page > 0)
    e = torch.where(written[:, None], torch.where(kept[:, None], torch.maximum(need, had), need), had)
    again = torch.ldexp(codes[first_pid].float(), (had - e)[first_pid][:, :, None, None])
    hold = (torch.arange(page, device="cuda")[None, :] < (first % page)[:, None])[:, None, :, None]
    codes[first_pid] = torch.where(hold, again, codes[first_pid].float()).to(torch.float8_e4m3fn)
    new = torch.clamp(torch.ldexp(x, -e[pid][:, :, None]), -LARGEST, LARGEST)
    codes.view(torch.uint8)[pid, :, slot] = new.to(torch.float8_e4m3fn).view(torch.uint8)
    scales.view(torch.uint8).copy_(e + 127)


def _values(codes, scales, pages):
    """The values of these pages: [..., heads, tokens of a page, dim]."""
    e = scales.view(torch.uint8)[pages].int() - 127
    return torch.ldexp(codes[pages].float(), e[..., None, None])


def _sequences(codes, scales, table):
    """Everything the tables name: [sequences][heads][tokens][dim]."""
    x = _values(codes, scales, table.long()).transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[4])


def _attend(state):
    case = state["case"]
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    k, v, ks, vs = state["cache"]
    keys, values = _sequences(k, ks, state["table"]), _sequences(v, vs, state["table"])
    s, i, position = _rows(state)
    seqs, most, group = case["seqs"], state["most"], heads // kv
    q = torch.zeros((seqs, most, kv, group, dim), device="cuda")
    q[s, i] = state["q"].float().reshape(-1, kv, group, dim)
    q = q.permute(0, 2, 3, 1, 4).reshape(seqs, kv, group * most, dim)
    w = (q @ keys.transpose(2, 3)).mul_(1 / math.sqrt(dim)).view(seqs, kv, group, most, -1)
    at = torch.zeros((seqs, most), dtype=torch.long, device="cuda")
    at[s, i] = position
    token = torch.arange(w.shape[4], device="cuda")
    hidden = (token >= state["lengths"][:, None, None]).expand(seqs, most, -1)
    if case["causal"]:
        hidden = hidden | (token > at[:, :, None])
    if case["window"]:
        hidden = hidden | (token <= at[:, :, None] - case["window"])
    w.masked_fill_(hidden[:, None, None], -math.inf)
    top = w.amax(dim=4, keepdim=True)
    w.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = w.sum(dim=4, keepdim=True)
    out = (w.view(seqs, kv, group * most, -1) @ values).view(seqs, kv, group, most, dim)
    out = torch.where(total > 0, out / total, 0.0).permute(0, 3, 1, 2, 4).reshape(seqs, most, heads, dim)[s, i].to(torch.bfloat16)
    if not case["lse"]:
        return out
    return out, (top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(seqs, most, heads)[s, i]


def _plain(state):
    case = state["case"]
    k, v, ks, vs = state["cache"]
    if case["op"] == "write":
        rows = _rows(state)
        _write_one(state["k"], k, ks, state, rows)
        _write_one(state["v"], v, vs, state, rows)
        return k, v, ks, vs
    if case["op"] == "read":
        s, _, position = _rows(state)
        pid, slot = state["table"].long()[s, position // case["page"]], position % case["page"]
        return tuple(torch.ldexp(codes.view(torch.uint8)[pid, :, slot].view(torch.float8_e4m3fn).float(),
                                 (scales.view(torch.uint8)[pid].int() - 127)[:, :, None]).to(_dtype(case)) for codes, scales in ((k, ks), (v, vs)))
    return _attend(state)


# ---- the framework's -----------------------------------------------------------------------

def _own(state):
    from paper_2410_16926_b200 import pvq
    case, cache = state["case"], pvq.Fp8Cache(*state["cache"])
    if case["op"] == "write":
        pvq.fp8_cache_write(state["k"], state["v"], cache, state["table"], state["lengths"], state["starts"])
        return tuple(cache)
    if case["op"] == "read":
        return pvq.fp8_cache_read(cache, state["table"], state["lengths"], state["starts"], rows=state["rows"], dtype=_dtype(case))
    return pvq.fp8_attention(state["q"], cache, state["table"], state["lengths"], state["starts"], causal=case["causal"], window=case["window"],
                             lse=case["lse"])


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without -----------------------------------------------------------

def work(case):
    sizes, kv, dim, page = _sizes(case), case["kv"], case["dim"], case["page"]
    rows = sum(n for _, n in sizes)
    if case["op"] in ("write", "read"):
        size = 4 if case["dtype"] == "f32" else 2
        pages = sum((length - 1) // page - (length - n) // page + 1 for length, n in sizes)
        return dict(bytes=2 * kv * (rows * dim * (size + 1) + pages), flops=4 * rows * kv * dim)
    held = pairs = 0
    for length, n in sizes:
        if case["window"]:  # position p sees min(p + 1, window)
            short = max(0, min(n, case["window"] - (length - n)))
            pairs += short * (length - n) + short * (short + 1) // 2 + (n - short) * case["window"]
            held += min(length, case["window"] + n - 1)
        else:
            pairs += n * (length - n) + n * (n + 1) // 2 if case["causal"] else n * length
            held += length
    return dict(bytes=2 * kv * held * dim + rows * case["heads"] * (4 * dim + (4 if case["lse"] else 0)), flops=4 * pairs * case["heads"] * dim)


# ---- the same in 64 bits ---------------------------------------------------------------------

def _e4m3_64(v):
    """The nearest e4m3 value (ties to the even one), the largest beyond it."""
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), torch.clamp(e - 1, min=-6) - 3)
    return (torch.round(v / step) * step).clamp(-LARGEST, LARGEST)  # (torch.round: halves to even)


def _scale_64(top):
    s = torch.exp2(torch.ceil(torch.log2(top / LARGEST)))
    s = torch.where(top > s * LARGEST, s * 2, torch.where(top <= s * LARGEST / 2, s / 2, s))
    return torch.where(top > 0, s, torch.zeros_like(s)).clamp(2.0 ** LEAST, 2.0 ** MOST)


def _write_64(x, codes, scales, state, sizes):
    codes, scales, page = codes.double(), scales.double(), codes.shape[2]
    table, row = state["table"].tolist(), 0
    for s, (length, n) in enumerate(sizes):
        position = length - n
        while position < length:  # a page at a time
            pid, begin = table[s][position // page], position % page
            end = min(page, begin + length - position)
            new = x[row:row + end - begin].double().transpose(0, 1)  # [heads][tokens][dim]
            scale = _scale_64(new.abs().amax(dim=(1, 2)))
            if begin:
                scale = torch.maximum(scale, scales[pid])
                codes[pid, :, :begin] = _e4m3_64(codes[pid, :, :begin] * (scales[pid] / scale)[:, None, None])
            codes[pid, :, begin:end] = _e4m3_64(new / scale[:, None, None])
            scales[pid] = scale
            position, row = position + end - begin, row + end - begin
    return codes, scales


def _sequence_64(codes, scales, table, length):
    """[heads][tokens][dim] of one sequence."""
    pages = table[:-(-length // codes.shape[2])].long()
    x = codes.view(torch.uint8)[pages].view(torch.float8_e4m3fn).double() * scales.view(torch.uint8)[pages].view(torch.float8_e8m0fnu).double()[:, :, None, None]
    return x.transpose(0, 1).reshape(codes.shape[1], -1, codes.shape[3])[:, :length]


def exact(case, seed):
    state = prepare(case, seed)
    sizes = _sizes(case)
    k, v, ks, vs = state["cache"]
    if case["op"] == "write":
        (k, ks), (v, vs) = _write_64(state["k"], k, ks, state, sizes), _write_64(state["v"], v, vs, state, sizes)
        return k, v, ks, vs
    parts, sums, row = [], [], 0
    for s, (length, n) in enumerate(sizes):
        keys, values = (_sequence_64(c, x, state["table"][s], length) for c, x in ((k, ks), (v, vs)))
        if case["op"] == "read":
            parts.append(keys[:, length - n:].transpose(0, 1))
            sums.append(values[:, length - n:].transpose(0, 1))
            continue
        q = state["q"][row:row + n].double().view(n, case["kv"], -1, case["dim"])
        row += n
        place = torch.arange(length - n, length, device="cuda")[:, None, None]
        token = torch.arange(length, device="cuda")
        seen = torch.ones((n, 1, length), dtype=torch.bool, device="cuda")
        if case["causal"]:
            seen &= token <= place
        if case["window"]:
            seen &= token > place - case["window"]
        out, lse = [], []
        for h in range(case["kv"]):
            w = torch.einsum("nhd,td->nht", q[:, h], keys[h]) / math.sqrt(case["dim"])
            w = w.masked_fill(~seen, -math.inf)
            lse.append(torch.logsumexp(w, dim=2))
            out.append(torch.einsum("nht,td->nhd", torch.exp(w - lse[-1][:, :, None]), values[h]))
        parts.append(torch.cat(out, dim=1))
        sums.append(torch.cat(lse, dim=1))
    if case["op"] == "attend":
        return (torch.cat(parts), torch.cat(sums)) if case["lse"] else torch.cat(parts)
    return torch.cat(parts), torch.cat(sums)

"""The 8-bit key and value cache without a GPU: what its entry points refuse, and the definitions the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest
import torch

import fp8_cache_reference as ref
from paper_2410_16926_b200 import pvq

INVALID, UNSUPPORTED, ALIGN, SMALL = 1, 2, 3, 4
P = 1 << 20  # an aligned address; the checks come before anything is read


def cache(**change):
    d = dict(k=P, v=P, ks=P, vs=P, pages=8, heads=2, page=64, dim=128, page_step=16384, head_step=8192, token_step=128, scale_step=2)
    d.update(change)
    return C.byref(pvq.Fp8CacheDesc(*d.values()))


def step(**change):
    d = dict(table=P, lengths=P, starts=P, seqs=3, rows=10, width=4, ld=4)
    d.update(change)
    return C.byref(pvq.Fp8StepDesc(*d.values()))


def calls(c, p):
    L = pvq.lib()
    yield L.pvq_fp8_cache_write(c, p, P, 512, 128, P, 512, 128, 1, None, None)
    yield L.pvq_fp8_cache_read(c, p, P, 512, 128, P, 512, 128, 0, None, None)
    yield L.pvq_fp8_attention(c, p, P, 4, 512, 128, 1, 0, 0.1, P, 512, 128, None, P, 1 << 30, None, None)


BAD_CACHES = [(dict(k=None), INVALID), (dict(v=None), INVALID), (dict(ks=None), INVALID), (dict(vs=None), INVALID), (dict(pages=0), INVALID),
              (dict(heads=0), INVALID), (dict(dim=0), INVALID), (dict(page=0), INVALID), (dict(page_step=96), INVALID), (dict(head_step=96), INVALID),
              (dict(token_step=112), INVALID), (dict(scale_step=1), INVALID), (dict(page=48), UNSUPPORTED), (dict(page=8), UNSUPPORTED),
              (dict(page=256), UNSUPPORTED), (dict(dim=120), UNSUPPORTED), (dict(dim=144, token_step=144), UNSUPPORTED), (dict(pages=1 << 31), UNSUPPORTED),
              (dict(page_step=1 << 40), UNSUPPORTED), (dict(scale_step=1 << 40), UNSUPPORTED), (dict(k=P + 8), ALIGN), (dict(v=P + 4), ALIGN),
              (dict(page_step=16392), ALIGN), (dict(head_step=8200), ALIGN), (dict(token_step=136), ALIGN)]
BAD_STEPS = [(dict(table=None), INVALID), (dict(lengths=None), INVALID), (dict(seqs=0), INVALID), (dict(rows=0), INVALID), (dict(width=0), INVALID),
             (dict(ld=3), INVALID), (dict(starts=None), INVALID), (dict(rows=1 << 28), UNSUPPORTED), (dict(seqs=1 << 24), UNSUPPORTED),
             (dict(width=1 << 25, ld=1 << 25), UNSUPPORTED), (dict(width=1 << 60, ld=1 << 60), UNSUPPORTED), (dict(ld=1 << 31), UNSUPPORTED),
             (dict(table=P + 2), ALIGN), (dict(lengths=P + 1), ALIGN), (dict(starts=P + 3), ALIGN)]


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_caches_are_checked(bad, status):
    assert list(calls(cache(**bad), step())) == [status] * 3


@pytest.mark.parametrize("bad,status", BAD_STEPS)
def test_steps_are_checked(bad, status):
    assert list(calls(cache(), step(**bad))) == [status] * 3


def test_missing_descriptions():
    assert list(calls(None, step())) == [INVALID] * 3 and list(calls(cache(), None)) == [INVALID] * 3


@pytest.mark.parametrize("p,row,head,status", [(None, 512, 128, INVALID), (P, 112, 128, INVALID), (P, 512, 112, INVALID), (P + 8, 512, 128, ALIGN),
                                               (P, 516, 128, ALIGN), (P, 512, 132, ALIGN), (P, 1 << 35, 128, UNSUPPORTED), (P, 512, 1 << 35, UNSUPPORTED)])
def test_rows_are_checked(p, row, head, status):
    L, c, s = pvq.lib(), cache(), step()
    assert L.pvq_fp8_cache_write(c, s, p, row, head, P, 512, 128, 1, None, None) == status
    assert L.pvq_fp8_cache_write(c, s, P, 512, 128, p, row, head, 1, None, None) == status
    assert L.pvq_fp8_cache_read(c, s, p, row, head, P, 512, 128, 1, None, None) == status
    assert L.pvq_fp8_cache_read(c, s, P, 512, 128, p, row, head, 1, None, None) == status
    assert L.pvq_fp8_attention(c, s, p, 4, row, head, 1, 0, 0.1, P, 512, 128, None, P, 1 << 30, None, None) == status
    assert L.pvq_fp8_attention(c, s, P, 4, 512, 128, 1, 0, 0.1, p, row, head, None, P, 1 << 30, None, None) == status


def test_other_arguments_are_checked():
    L = pvq.lib()
    for dtype in (-1, 2):
        assert L.pvq_fp8_cache_write(cache(), step(), P, 512, 128, P, 512, 128, dtype, None, None) == INVALID
        assert L.pvq_fp8_cache_read(cache(), step(), P, 512, 128, P, 512, 128, dtype, None, None) == INVALID

    def attention(heads=4, causal=1, window=0, scale=0.1, lse=None, workspace=P, size=1 << 30, **rows):
        return L.pvq_fp8_attention(cache(), step(**rows), P, heads, 512, 128, causal, window, scale, P, 512, 128, lse, workspace, size, None, None)

    for heads in (0, -2, 3, 5):
        assert attention(heads=heads) == INVALID
    assert attention(heads=2 * 129) == UNSUPPORTED
    assert attention(heads=256, rows=(1 << 28) - 1) == UNSUPPORTED
    assert attention(causal=2) == INVALID and attention(window=-1) == INVALID and attention(causal=0, window=5) == INVALID
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert attention(scale=scale) == INVALID
    assert attention(lse=P + 2) == ALIGN and attention(workspace=P + 8) == ALIGN and attention(workspace=None) == INVALID
    need = L.pvq_fp8_attention_workspace(cache(), step(), 4)
    assert need > 0 and attention(size=need - 1) == SMALL
    for heads in (0, 5, 258, -4):
        assert L.pvq_fp8_attention_workspace(cache(), step(), heads) == 0
    assert [L.pvq_fp8_attention_workspace(cache(**bad), step(), 4) for bad, _ in BAD_CACHES] == [0] * len(BAD_CACHES)
    assert [L.pvq_fp8_attention_workspace(cache(), step(**bad), 4) for bad, _ in BAD_STEPS] == [0] * len(BAD_STEPS)
    # single tokens of few short sequences need none; longer tables, more sequences and more rows do
    one = dict(starts=None, seqs=2, rows=2)
    assert L.pvq_fp8_attention_workspace(cache(), step(**one), 4) == 0
    for more in (dict(width=4000, ld=4000), dict(seqs=200, rows=200), dict(starts=P)):
        assert L.pvq_fp8_attention_workspace(cache(), step(**{**one, **more}), 4) > 0


def test_the_binding_refuses_what_is_not_on_the_gpu_or_of_another_type():
    c = pvq.alloc_fp8_cache(4, 2, 16, 32, device="cpu")
    assert c.k.shape == (4, 2, 16, 32) and c.v_scales.shape == (4, 2)
    x, table, lengths = torch.zeros(3, 2, 32), torch.zeros(3, 1, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: pvq.fp8_cache_write(x, x, c, table, lengths), lambda: pvq.fp8_cache_read(c, table, lengths),
                 lambda: pvq.fp8_attention(x.bfloat16(), c, table, lengths)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        pvq.fp8_cache_write(x.double(), x, c, table, lengths)
    with pytest.raises(TypeError):
        pvq.fp8_cache_read(c, table, lengths, dtype=torch.float16)


def test_the_reference_says_what_the_header_does():
    """Scales from their definition, a page written at once or token by token, and attention against differences of its lse: the
    gradient of log sum exp(scale q k_j) by q is scale times the attention to the keys themselves."""
    assert [ref.page_scale(a) for a in (0.0, 448.0, 449.0, 1e-300, 3e38, 1.75, 1.7500001)] == [-40, 0, 1, -40, 40, -8, -7]
    rng = np.random.default_rng(3)
    x = rng.standard_normal((20, 2, 16)) * 10.0 ** rng.integers(-2, 3, (20, 1, 1))
    table = np.array([[1, 0]])
    once, e_once = np.zeros((2, 2, 16, 16)), np.full((2, 2), 5)
    ref.write(once, e_once, x, table, [20], [0, 20], 16)
    by_token, e_by = np.zeros((2, 2, 16, 16)), np.full((2, 2), 5)
    for i in range(20):
        ref.write(by_token, e_by, x[i:i + 1], table, [i + 1], [0, 1], 16)
    assert np.array_equal(e_once, e_by)
    # each change of the scale may round again, by half a step of the last scale
    got, want = (ref.sequence(c, e_once, table[0], 20, 16) for c, e in ((by_token, e_by), (once, e_once)))
    top = 2.0 ** np.repeat(e_once[table[0]].T, 16, axis=1)[:, :20, None]
    assert (np.abs(got - want) <= 8 * 2.0 ** -4 * np.maximum(np.abs(want), 2.0 ** -6 * top)).all()
    q = rng.standard_normal((3, 4, 16))
    held = [once, once], [e_once, e_once]
    out, lse, _, _ = ref.attention(q, *held, table, [20], [0, 3], 16, scale=0.01)
    for d in range(16):
        up, down = q.copy(), q.copy()
        up[:, :, d] += 1e-5
        down[:, :, d] -= 1e-5
        slope = (ref.attention(up, *held, table, [20], [0, 3], 16, scale=0.01)[1] - ref.attention(down, *held, table, [20], [0, 3], 16, scale=0.01)[1]) / 2e-5
        assert np.allclose(slope, 0.01 * out[:, :, d], rtol=1e-6, atol=1e-8)

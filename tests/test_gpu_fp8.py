"""The 8-bit floating-point operators on the GPU against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import fp8_reference as ref
from paper_2410_16926_b200 import pvq

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def normal(rows, cols, dtype, seed, pad=0, scale=1.0):
    """A seeded matrix; with `pad` its rows lie further apart than they are long (a multiple of 16 values)."""
    ld = -(-cols // 16) * 16 + pad
    x = torch.from_numpy(np.random.default_rng(seed).standard_normal((rows, ld)).astype(np.float32) * scale).to(dtype).cuda()
    return x[:, :cols]


def held(x64, tile, pad=0, fill=0x55):
    """An Fp8Matrix made on the host; the bytes between its rows hold anything."""
    q, b = ref.quantize(x64, tile)
    rows, cols = x64.shape
    codes = torch.full((rows, -(-cols // 16) * 16 + pad), fill, dtype=torch.uint8)
    codes[:, :cols] = torch.from_numpy(q.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8)
    scales = torch.full((b.shape[0], -(-b.shape[1] // 4) * 4 + pad // 4), 0xff, dtype=torch.uint8)
    scales[:, :b.shape[1]] = torch.from_numpy(b.astype(np.uint8))
    return pvq.Fp8Matrix(codes.cuda()[:, :cols].view(torch.float8_e4m3fn), scales.cuda()[:, :b.shape[1]].view(torch.float8_e8m0fnu), tile)


def random_held(rows, cols, tile, seed, pad=0, scale=1.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * scale * np.exp2(rng.integers(-3, 4, size=(rows, 1)))
    if rows > 4:
        x[rows // 2] = 0.0
    return held(x, tile, pad)


def guarded(rows, cols, dtype, unit, pad=16):
    """An output inside a larger buffer, and a check that nothing around it was written."""
    ld = -(-cols // unit) * unit + pad
    raw = torch.full((rows + 2, ld * torch.empty(0, dtype=dtype).element_size()), 0xa5, dtype=torch.uint8, device="cuda")
    whole = raw.view(dtype) if dtype.itemsize > 1 else raw
    out = whole[1:rows + 1, :cols]

    def check():
        torch.cuda.synchronize()
        keep = raw.clone()
        keep.view(dtype)[1:rows + 1, :cols] = torch.full((1,), 0, dtype=dtype, device="cuda") if dtype.itemsize > 1 else 0
        size = dtype.itemsize
        assert bool((keep[0] == 0xa5).all()) and bool((keep[-1] == 0xa5).all()) and bool((keep[1:-1, cols * size:] == 0xa5).all())
    return out, check


def same(q, x64, tile):
    codes, b = ref.quantize(x64, tile)
    assert np.array_equal(q.scales.view(torch.uint8).cpu().numpy(), b)
    got = ref.to64(q.codes)
    assert np.array_equal(got, codes, equal_nan=True)
    assert np.array_equal(np.signbit(got[np.isfinite(got)]), np.signbit(codes[np.isfinite(codes)]))


# ---- quantize, dequantize -------------------------------------------------------------

@pytest.mark.parametrize("tile", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 128, 0), (3, 7, 16), (2, 129, 0), (129, 250, 32), (300, 1000, 0), (5, 4096, 16), (128, 128, 0), (37, 388, 0)])
def test_quantize(rows, cols, pad, dtype, tile):
    x = normal(rows, cols, dtype, rows * 1000 + cols, pad)
    if rows > 2:
        x[1] = 0.0
        x[2] *= 2.0 ** -120
    same(pvq.fp8_quantize(x, tile=tile), ref.to64(x), tile)


@pytest.mark.parametrize("tile", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_quantize_of_special_values(dtype, tile):
    x = torch.zeros((40, 504), dtype=torch.float32)
    x[0, 3], x[0, 130] = float("nan"), float("inf")
    x[1, 0], x[1, 1] = -float("inf"), 5.0
    x[2, :128] = float("nan")
    x[3, :4] = torch.tensor([448.0, 449.0, -448.0, 1.0])
    x[4, :4] = torch.tensor([3.0e38, -3.0e38, 1.0, 1e-30])
    x[5, 503] = 1e-38
    x[6, 256:258] = torch.tensor([450.0, -0.0])
    x[7, 0:2] = torch.tensor([-0.0, 0.0])
    x[8, :3] = torch.tensor([2.0 ** -126, 2.0 ** -140, -2.0 ** -133])
    x[9, :128] = torch.linspace(-448, 448, 128)
    x[10, :128] = torch.arange(128) / 8 + 1 / 16 - 8
    x = x.to(dtype).cuda()
    same(pvq.fp8_quantize(x, tile=tile), ref.to64(x), tile)


@pytest.mark.parametrize("tile", [False, True])
@pytest.mark.parametrize("rows,cols", [(3, 7), (130, 250)])
def test_quantize_writes_its_matrix_alone(rows, cols, tile):
    x = normal(rows, cols, BF16, 5)
    codes, check_codes = guarded(rows, cols, torch.uint8, 16)
    scales, check_scales = guarded(-(-rows // 128) if tile else rows, -(-cols // 128), torch.uint8, 4)
    out = pvq.Fp8Matrix(codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu), tile)
    got = pvq.fp8_quantize(x, tile=tile, out=out)
    assert got.codes.data_ptr() == codes.data_ptr()
    same(got, ref.to64(x), tile)
    check_codes()
    check_scales()


@pytest.mark.parametrize("tile", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 7, 16), (129, 250, 32), (5, 4096, 0)])
def test_dequantize(rows, cols, pad, dtype, tile):
    q = random_held(rows, cols, tile, rows + cols, pad)
    out, check = guarded(rows, cols, dtype, 8)
    pvq.fp8_dequantize(q, dtype=dtype, out=out)
    check()
    assert np.array_equal(ref.to64(out), ref.values(q))
    assert torch.equal(pvq.fp8_dequantize(q, dtype=dtype), out)


def test_new_matrices_are_ordinary_tensors():
    """Codes and scales that share an allocation: shapes, strides, copies, views, and each outliving the other."""
    x = normal(130, 250, BF16, 3)
    q = pvq.fp8_quantize(x)
    assert q.codes.shape == (130, 250) and q.codes.stride() == (256, 1) and q.scales.shape == (130, 2) and q.scales.stride() == (4, 1)
    assert q.codes.dtype == torch.float8_e4m3fn and q.scales.dtype == torch.float8_e8m0fnu and q.codes.device == x.device
    want = ref.values(q)
    codes, scales = q.codes.clone(), q.scales.clone()
    assert np.array_equal(ref.to64(codes.float()) * ref.spread(ref.to64(scales.float()), 130, 250, False), want)
    kept = q.scales
    del q, codes
    assert torch.equal(kept.view(torch.uint8), scales.view(torch.uint8)) and not kept.requires_grad
    out = pvq.fp8_dequantize(pvq.fp8_quantize(x))
    assert out.shape == (130, 250) and out.stride() == (256, 1) and torch.equal(out.contiguous(), out)


def test_dequantize_into_rows_on_16_byte_boundaries_alone():
    q = random_held(40, 4096, False, 1)
    for ld in (4096, 4100, 4104):
        whole = torch.full((40, ld + 8), 7.0, device="cuda")
        for first in (0, 4):
            out = whole[:, first:first + 4096]
            pvq.fp8_dequantize(q, dtype=F32, out=out)
            assert np.array_equal(ref.to64(out), ref.values(q))
        assert bool((whole[:, 4100:] == 7.0).all())


def test_dequantize_of_every_code_and_scale():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).repeat(256, 1).cuda()
    scales = torch.arange(256, dtype=torch.int32).to(torch.uint8)[:, None].repeat(1, 4).cuda()[:, :2]
    q = pvq.Fp8Matrix(codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu), False)
    want = ref.values(q)
    with np.errstate(over="ignore"):
        want32 = want.astype(np.float32)
    assert np.array_equal(pvq.fp8_dequantize(q, dtype=F32).cpu().numpy(), want32, equal_nan=True)
    assert torch.equal(pvq.fp8_dequantize(q).float().nan_to_num(7.0), torch.from_numpy(want32).cuda().to(BF16).float().nan_to_num(7.0))


# ---- products -------------------------------------------------------------------------

def check_matmul(a, b, transposed, dtype, out=None):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = pvq.fp8_matmul(a, b, transposed=transposed, dtype=dtype, out=out, status=status)
    va, vb = ref.values(a), ref.values(b)
    vb = vb if transposed else vb.T
    want = va @ vb
    slack = ref.HALF_STEP[dtype] * np.abs(want) + 1.01 * ref.matmul_slack(va, vb, va.shape[1] / 32)
    err = np.abs(ref.to64(got) - want)
    assert int(status.item()) == 0
    assert got.shape == want.shape and np.all(err <= slack), float(np.max(err - slack))
    return got


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,inner,outer", [(1, 1, 1), (1, 128, 128), (2, 130, 7), (1, 4096, 1024), (5, 1000, 333), (8, 512, 4096), (16, 300, 136),
                                              (17, 257, 129), (33, 2048, 512), (64, 640, 200), (65, 127, 640), (128, 1024, 384), (129, 4096, 257),
                                              (300, 513, 1000), (513, 900, 770), (1024, 256, 2048), (1281, 1400, 2100), (2100, 260, 2600),
                                              (385, 300, 4700), (130, 520, 9480), (1025, 260, 2100)])
def test_matmul(rows, inner, outer, dtype, transposed):
    a = random_held(rows, inner, False, rows + inner, pad=16)
    shape = (inner, outer) if transposed else (outer, inner)
    b = random_held(*shape, True, outer, pad=16 * (outer % 3), scale=0.02)
    out, check = guarded(rows, outer, dtype, 8)
    check_matmul(a, b, transposed, dtype, out)
    check()


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows,inner,outer", [(3, 9000, 200), (1300, 8200, 2100), (2100, 16600, 2400)])
def test_matmul_of_long_sums(rows, inner, outer, transposed):
    """fp32 results over more than 8192 values are within 1e-6 of themselves (2-norm): sums that the tensor cores cut off alone
    would not be (8e-8 of a sum for every 1024 values)."""
    rng = np.random.default_rng(inner)
    make = lambda r, c: torch.from_numpy(rng.standard_normal((r, c)).astype(np.float32)).cuda()  # noqa: E731
    a = pvq.fp8_quantize(make(rows, -(-inner // 8) * 8)[:, :inner])
    shape = (inner, outer) if transposed else (outer, inner)
    b = pvq.fp8_quantize(make(shape[0], -(-shape[1] // 8) * 8)[:, :shape[1]], tile=True)
    va, vb = (pvq.fp8_dequantize(q, dtype=F32).double() for q in (a, b))
    want = va @ (vb if transposed else vb.t())
    got = pvq.fp8_matmul(a, b, transposed=transposed, dtype=F32).double()
    assert float((got - want).norm()) <= 1e-6 * float(want.norm())


@pytest.mark.parametrize("tiles", [(False, False), (True, True), (True, False)])
@pytest.mark.parametrize("rows,inner,outer", [(3, 300, 200), (200, 640, 300), (700, 384, 520), (1300, 700, 2050)])
def test_matmul_of_other_blocks(rows, inner, outer, tiles):
    a, b = random_held(rows, inner, tiles[0], 1), random_held(outer, inner, tiles[1], 2)
    check_matmul(a, b, False, BF16)


@pytest.mark.parametrize("rows,outer", [(2, 256), (300, 512), (600, 1024), (1700, 1800)])
def test_matmul_of_nan_and_of_scales_behind_the_end(rows, outer):
    """A NaN reaches its own row or column alone; what lies behind a row's end (scales of NaN, codes) reaches nothing."""
    inner = 300
    x = np.random.default_rng(3).standard_normal((rows, inner))
    w = np.random.default_rng(4).standard_normal((outer, inner))
    x[1, 17] = np.nan
    w[3, 299] = np.inf
    a, b = held(x, False, pad=16), held(w, True, pad=16)
    got = pvq.fp8_matmul(a, b, dtype=F32)
    nan = torch.isnan(got).cpu().numpy()
    want = np.zeros((rows, outer), dtype=bool)
    want[1] = True
    want[:, 3] = True
    assert np.array_equal(nan, want)


@pytest.mark.parametrize("rows,outer", [(2, 256), (300, 512), (1700, 1800)])
def test_matmul_of_a_scale_of_nan(rows, outer):
    a = random_held(rows, 500, False, 1)
    b = random_held(outer, 500, True, 2)
    a.scales.view(torch.uint8)[1, 2] = 255
    nan = torch.isnan(pvq.fp8_matmul(a, b, dtype=F32)).cpu().numpy()
    assert nan[1].all() and not np.delete(nan, 1, axis=0).any()
    assert torch.isnan(pvq.fp8_dequantize(a)[1, 256:384]).all() and not torch.isnan(pvq.fp8_dequantize(a)[1, :256]).any()
    dy = normal(rows, outer, BF16, 3)
    grad = torch.isnan(pvq.fp8_weight_grad(dy, a)).cpu().numpy()
    assert grad[:, 256:384].all() and not grad[:, :256].any() and not grad[:, 384:].any()


@pytest.mark.parametrize("rows", [1, 40, 300, 12300])
def test_matmul_of_far_apart_scales(rows):
    """Blocks whose scales are at the ends of the range: products that cancel their scales, and ones that vanish."""
    rng = np.random.default_rng(8)
    x = rng.standard_normal((rows, 512)) * np.repeat([2.0 ** 90, 1.0, 2.0 ** -90, 2.0 ** -60], 128)
    w = rng.standard_normal((256, 512)) * np.repeat([2.0 ** -90, 1.0, 2.0 ** 90, 2.0 ** -60], 128)
    check_matmul(held(x, False), held(w, True), False, F32)


def check_weight_grad(dy, x, dtype, out=None):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = pvq.fp8_weight_grad(dy, x, dtype=dtype, out=out, status=status)
    vd, vx = ref.to64(dy).T, ref.values(x)
    want = vd @ vx
    slack = ref.HALF_STEP[dtype] * np.abs(want) + 1.01 * ref.matmul_slack(vd, vx, vd.shape[1] / 16)
    err = np.abs(ref.to64(got) - want)
    assert int(status.item()) == 0
    assert got.shape == want.shape and np.all(err <= slack), float(np.max(err - slack))
    return got


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,inner,outer,tile", [(1, 1, 1, False), (1, 300, 200, False), (7, 130, 7, False), (64, 128, 128, False),
                                                   (65, 256, 264, True), (1000, 513, 257, False), (1001, 1024, 520, True), (2500, 300, 1000, False),
                                                   (4096, 128, 64, False), (129, 2048, 1024, False),
                                                   (1500, 1500, 2100, False), (700, 2600, 2060, True), (3000, 250, 130, False),
                                                   (2049, 2300, 2000, False), (1100, 2500, 2100, False), (1700, 2500, 2100, True),
                                                   (600, 1300, 1800, False), (2900, 1536, 1800, True), (500, 4736, 500, False)])
def test_weight_grad(rows, inner, outer, tile, dtype):
    dy = normal(rows, outer, BF16, rows, pad=16)
    x = random_held(rows, inner, tile, rows + 1, pad=16)
    out, check = guarded(outer, inner, dtype, 8)
    check_weight_grad(dy, x, dtype, out)
    check()


@pytest.mark.parametrize("rows,inner,outer", [(1700, 2500, 2100), (2800, 1504, 2104)])
def test_weight_grad_without_a_workspace(rows, inner, outer):
    """The C call takes NULL: the same bits."""
    import ctypes as C
    L = pvq.lib()
    assert L.pvq_fp8_weight_grad_workspace(rows, inner, outer) > 0
    dy, x = normal(rows, outer, BF16, 1), random_held(rows, inner, False, 2)
    want = pvq.fp8_weight_grad(dy, x)
    out, check = guarded(outer, inner, F32, 4)
    desc = pvq.Fp8Desc(x.codes.data_ptr(), x.scales.data_ptr(), rows, inner, x.codes.stride(0), x.scales.stride(0), 0)
    stream = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert L.pvq_fp8_weight_grad(dy.data_ptr(), outer, dy.stride(0), C.byref(desc), out.data_ptr(), 0, out.stride(0), None, 0, None, stream) == 0
    check()
    assert torch.equal(out, want)


def test_weight_grad_of_nan():
    dy, x = np.random.default_rng(1).standard_normal((70, 300)), np.random.default_rng(2).standard_normal((70, 400))
    dy[69, 5], x[3, 399] = np.inf, np.nan
    got = pvq.fp8_weight_grad(torch.from_numpy(np.pad(dy, ((0, 0), (0, 4)))).to(BF16).cuda()[:, :300], held(x, False))
    want = np.zeros((300, 400), dtype=bool)
    want[5] = True
    want[:, 399] = True
    assert np.array_equal(~torch.isfinite(got).cpu().numpy(), want)


# ---- the gated activation ---------------------------------------------------------------

def check_h(h, gate64, up64, act):
    """Codes of act(gate) * up: within half a step, plus what fp32 loses, of the value; scales those of the exact values
    wherever their largest is not that near to a limit."""
    want = ref.activation(gate64, act) * up64
    slack = np.where(want == 0, 0.0, np.abs(want) * (ref.sigma_slack(gate64, act) + 2.0 ** -22) + 2.0 ** -120)
    b = h.scales.view(torch.uint8).cpu().numpy().astype(np.int64)
    low, high = ref.scale_bytes(ref.block_max(np.abs(want) - slack, False)), ref.scale_bytes(ref.block_max(np.abs(want) + slack, False))
    assert np.all((b >= low) & (b <= high))
    s = ref.spread(np.ldexp(1.0, b - 127), *want.shape, False)
    err = np.abs(ref.values(h) - want)
    limit = ref.half_step_e4m3((np.abs(want) + slack) / s) * s + slack
    assert np.all(err <= limit), float(np.max(err - limit))


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 128, 0), (3, 7, 16), (129, 250, 32), (65, 1000, 0), (2, 14336, 0)])
def test_gated(rows, cols, pad, dtype, act):
    gate, up = normal(rows, cols, dtype, 1, pad, 3.0), normal(rows, cols, dtype, 2, pad + 16)
    if rows > 2:
        gate[1] = 0.0
    h, gate8, up8 = pvq.fp8_gated(gate, up, act=act, checkpoint=True)
    check_h(h, ref.to64(gate), ref.to64(up), act)
    same(gate8, ref.to64(gate), False)
    same(up8, ref.to64(up), False)
    alone = pvq.fp8_gated(gate, up, act=act)
    assert torch.equal(alone.codes.view(torch.uint8), h.codes.view(torch.uint8))
    assert torch.equal(alone.scales.view(torch.uint8), h.scales.view(torch.uint8))


def test_gated_of_special_values():
    gate = torch.zeros((2, 512))
    up = torch.ones((2, 512))
    gate[0, :8] = torch.tensor([float("nan"), float("inf"), -1e30, 1e30, -200.0, 200.0, -88.0, -104.0])
    up[0, 130], gate[0, 130] = float("inf"), 1.0
    up[0, 260:262], gate[0, 260:262] = torch.tensor([3e38, 2.0]), torch.tensor([1e5, 2.0])
    for act in ("silu", "gelu"):
        h = pvq.fp8_gated(gate.cuda(), up.cuda(), act=act)
        v = ref.values(h)
        assert np.isnan(v[0, [0, 1, 130, 260]]).all()
        assert np.isfinite(v[1]).all() and np.isfinite(np.delete(v[0], [0, 1, 130, 260])).all()
        assert v[0, 2] == 0 and v[0, 4] == 0 and abs(v[0, 3] / 1e30 - 1) <= 2.0 ** -4
        assert v[0, 261] == pytest.approx(float(ref.activation(np.array(2.0), act)) * 2.0, rel=2.0 ** -4)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 7, 16), (129, 250, 32), (65, 1000, 0), (2, 14336, 0)])
def test_gated_backward(rows, cols, pad, dtype, act):
    dh = normal(rows, cols, dtype, 3, pad)
    gate, up = random_held(rows, cols, False, 4, pad, 2.0), random_held(rows, cols, False, 5, pad)
    outs = [guarded(rows, cols, dtype, 8) for _ in range(2)]
    pvq.fp8_gated_backward(dh, gate, up, act=act, out=[o for o, _ in outs])
    for _, check in outs:
        check()
    d, g, u = ref.to64(dh), ref.values(gate), ref.values(up)
    w, dw = ref.argument(g, act)
    s = ref.sigma(w)
    loss = ref.sigma_slack(g, act)
    # the slope's two terms each lose sigma's error and a few roundings; 1 - sigma loses 2^-23 of 1 beside that
    slope_slack = s * (loss + 2.0 ** -21) + np.abs(g) * s * np.abs(dw) * ((1 - s) * (2 * loss + 2.0 ** -21) + s * loss + 2.0 ** -22)
    want = d * u * ref.slope(g, act)
    err = np.abs(ref.to64(outs[0][0]) - want)
    limit = 1.01 * (np.abs(want) * ref.HALF_STEP[dtype] + np.abs(d * u) * slope_slack) + 2.0 ** -120
    assert np.all(err <= limit), float(np.max(err - limit))
    want = d * ref.activation(g, act)
    err = np.abs(ref.to64(outs[1][0]) - want)
    limit = 1.01 * np.abs(want) * (ref.HALF_STEP[dtype] + loss + 2.0 ** -22) + 2.0 ** -120
    assert np.all(err <= limit), float(np.max(err - limit))
    new = pvq.fp8_gated_backward(dh, gate, up, act=act)
    assert all(torch.equal(a, o) for a, (o, _) in zip(new, outs))


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_backward_against_differences(act):
    """dgate and dup are the slopes of sum(dh * act(gate) * up) at the values that were kept."""
    rng = np.random.default_rng(6)
    gate, up = held(rng.standard_normal((4, 256)) * 2, False), held(rng.standard_normal((4, 256)), False)
    dh = torch.from_numpy(rng.standard_normal((4, 256)).astype(np.float32)).cuda()
    dgate, dup = pvq.fp8_gated_backward(dh, gate, up, act=act)
    d, g, u, e = ref.to64(dh), ref.values(gate), ref.values(up), 1e-5
    diff = (ref.activation(g + e, act) - ref.activation(g - e, act)) / (2 * e) * d * u
    assert np.allclose(ref.to64(dgate), diff, rtol=2.0 ** -18, atol=2.0 ** -18 * np.abs(d * u).max())
    diff = d * (ref.activation(g, act) * (1 + e) - ref.activation(g, act) * (1 - e)) / (2 * e)
    assert np.allclose(ref.to64(dup), diff, rtol=2.0 ** -18, atol=2.0 ** -30)


# ---- together ---------------------------------------------------------------------------

def feed_forward(x, gate_up, down, dy):
    """A training step of a gated feed-forward block with its weights and activations in 8 bits: everything it gives."""
    inner = gate_up.codes.shape[0] // 2
    xq = pvq.fp8_quantize(x)
    both = pvq.fp8_matmul(xq, gate_up)
    h, gate8, up8 = pvq.fp8_gated(both[:, :inner], both[:, inner:], checkpoint=True)
    y = pvq.fp8_matmul(h, down)
    dyq = pvq.fp8_quantize(dy)
    dh = pvq.fp8_matmul(dyq, down, transposed=True)
    d_down = pvq.fp8_weight_grad(dy, h)
    d_both = torch.empty_like(both)
    pvq.fp8_gated_backward(dh, gate8, up8, out=(d_both[:, :inner], d_both[:, inner:]))
    dx = pvq.fp8_matmul(pvq.fp8_quantize(d_both), gate_up, transposed=True)
    d_gate_up = pvq.fp8_weight_grad(d_both, xq)
    return [xq, both, h, gate8, up8, y, dyq, dh, d_down, d_both, dx, d_gate_up]


def flat(step):
    return [t for r in step for t in ((r.codes, r.scales) if isinstance(r, pvq.Fp8Matrix) else (r,))]


def decoded_weight(rows, cols, seed):
    """A weight as this library holds it: encoded by pyramid vectors, decoded, quantised to 8-bit tiles."""
    N, b = 32, 8
    K = pvq.max_pulses(N, 96)
    table = pvq.build_count_table(N, K)
    edges, levels = pvq.build_scale_codebook(N, cols // N, b)
    w = normal(rows, cols, BF16, seed, scale=0.05)
    codes, sidx, rnorm = pvq.encode(w, N, K, b, table, edges)
    return pvq.fp8_quantize(pvq.decode(codes, sidx, rnorm, N, K, b, table, levels), tile=True)


@pytest.fixture(scope="module")
def step_inputs():
    tokens, features, inner = 333, 512, 640
    return normal(tokens, features, BF16, 31), decoded_weight(2 * inner, features, 32), decoded_weight(features, inner, 33), normal(tokens, features, BF16, 34)


def test_a_training_step(step_inputs):
    """Each result is within its own roundings of the exact result on the operands it was given."""
    x, gate_up, down, dy = step_inputs
    xq, both, h, gate8, up8, y, dyq, dh, d_down, d_both, dx, d_gate_up = feed_forward(*step_inputs)
    inner = down.codes.shape[1]
    same(xq, ref.to64(x), False)
    same(gate8, ref.to64(both[:, :inner]), False)
    same(up8, ref.to64(both[:, inner:]), False)
    same(dyq, ref.to64(dy), False)
    check_h(h, ref.to64(both[:, :inner]), ref.to64(both[:, inner:]), "silu")

    def near(got, va, vb, width):
        want = va @ vb
        slack = ref.HALF_STEP[got.dtype] * np.abs(want) + 1.01 * ref.matmul_slack(va, vb, va.shape[1] / width)
        assert np.all(np.abs(ref.to64(got) - want) <= slack)

    near(both, ref.values(xq), ref.values(gate_up).T, 32)
    near(y, ref.values(h), ref.values(down).T, 32)
    near(dh, ref.values(dyq), ref.values(down), 32)
    near(dx, ref.values(pvq.fp8_quantize(d_both)), ref.values(gate_up), 32)
    near(d_down, ref.to64(dy).T, ref.values(h), 16)
    near(d_gate_up, ref.to64(d_both).T, ref.values(xq), 16)
    # and the whole is what the step without 8 bits gives, as near as its 4-bit mantissas allow: relative errors of 2^-4 at
    # most, about 2^-5.6 of the mean square, from some six operands
    v = lambda q: ref.values(q)  # noqa: E731
    full = ref.to64(x) @ v(gate_up).T
    full_y = (ref.activation(full[:, :inner], "silu") * full[:, inner:]) @ v(down).T
    assert np.linalg.norm(ref.to64(y) - full_y) <= 6 * 2.0 ** -5 * np.linalg.norm(full_y)


def test_a_training_step_again_on_another_stream_and_captured(step_inputs):
    """The same bits every time: twice, on a side stream, and replayed from a graph on new inputs."""
    want = flat(feed_forward(*step_inputs))
    again = flat(feed_forward(*step_inputs))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = flat(feed_forward(*step_inputs))
    torch.cuda.current_stream().wait_stream(side)
    x, gate_up, down, dy = step_inputs
    gx, gdy = torch.zeros_like(x), torch.zeros_like(dy)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = flat(feed_forward(gx, gate_up, down, gdy))
    gx.copy_(x)
    gdy.copy_(dy)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for other in (again, there, captured):
        assert all(torch.equal(p.contiguous().view(torch.uint8), q.contiguous().view(torch.uint8)) for p, q in zip(want, other))


def test_tensors_of_different_devices_are_refused():
    x = normal(4, 128, BF16, 1)
    with pytest.raises(ValueError):
        pvq.fp8_quantize(x.cpu())
    q = pvq.fp8_quantize(x)
    with pytest.raises(ValueError):
        pvq.fp8_matmul(q, pvq.Fp8Matrix(q.codes.cpu(), q.scales, False))
    with pytest.raises(ValueError):
        pvq.fp8_matmul(q, pvq.fp8_quantize(normal(4, 256, BF16, 1)))
    with pytest.raises(ValueError):
        pvq.fp8_matmul(q, pvq.Fp8Matrix(q.codes, q.scales[:3], False))
    with pytest.raises(ValueError):
        pvq.fp8_quantize(x.t())
    with pytest.raises(pvq.PvqError):
        pvq.fp8_quantize(x[:, 1:])  # rows that do not start on 16-byte boundaries
    with pytest.raises(pvq.PvqError):
        pvq.fp8_quantize(x[:0])


@pytest.mark.parametrize("rows,inner,outer", [(130, 300, 200), (200, 2000, 1800)])
def test_weight_grad_of_every_code_at_the_ends_of_the_scales(rows, inner, outer):
    """All codes but NaN, subnormal ones among them, under scales from 2^-100 to 2^100; one row of x a row of dy, so that a
    sum has one product alone and is exact."""
    rng = np.random.default_rng(9)
    codes = rng.integers(0, 256, size=(rows, inner)).astype(np.uint8)
    codes[(codes & 0x7f) == 0x7f] = 0x80
    blocks = -(-inner // 128)
    scales = np.full((rows, -(-blocks // 4) * 4), 255, dtype=np.uint8)
    scales[:, :blocks] = rng.integers(27, 228, size=(rows, blocks))
    padded = np.zeros((rows, -(-inner // 16) * 16), dtype=np.uint8)
    padded[:, :inner] = codes
    x = pvq.Fp8Matrix(torch.from_numpy(padded).cuda()[:, :inner].view(torch.float8_e4m3fn),
                      torch.from_numpy(scales).cuda()[:, :blocks].view(torch.float8_e8m0fnu), False)
    dy = np.zeros((rows, outer), dtype=np.float32)
    where = rng.integers(0, rows, size=outer)
    dy[where, np.arange(outer)] = np.where(np.arange(outer) % 2 == 0, 1.0, -2.0)
    got = ref.to64(pvq.fp8_weight_grad(torch.from_numpy(dy).to(BF16).cuda(), x))
    assert np.array_equal(got, ref.values(x)[where] * np.where(np.arange(outer) % 2 == 0, 1.0, -2.0)[:, None])


def test_offsets_beyond_32_bits():
    """70000 x 32768 values: rows whose offsets pass 2^31, in every operator that takes such a matrix."""
    rows, cols, outs = 70000, 32768, 136
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((rows, cols), generator=g, device="cuda", dtype=BF16)
    some = torch.tensor([0, 1, 65535, 65536, 65537, rows - 2, rows - 1], device="cuda")

    def part(q):  # those rows
        return pvq.Fp8Matrix(q.codes.view(torch.uint8)[some].view(torch.float8_e4m3fn), q.scales.view(torch.uint8)[some].view(torch.float8_e8m0fnu), False)

    q = pvq.fp8_quantize(x)
    same(part(q), ref.to64(x[some]), False)
    v = pvq.fp8_dequantize(q)
    values = ref.values(part(q))
    assert np.array_equal(ref.to64(v[some]), values)
    h, gate8, up8 = pvq.fp8_gated(x, v, checkpoint=True)
    check_h(part(h), ref.to64(x[some]), ref.to64(v[some]), "silu")
    same(part(gate8), ref.to64(x[some]), False)
    same(part(up8), values, False)
    dgate, dup = pvq.fp8_gated_backward(x, h, gate8, out=(v, torch.empty_like(v)))
    want = pvq.fp8_gated_backward(x[some], part(h), part(gate8))
    assert torch.equal(dgate[some], want[0]) and torch.equal(dup[some], want[1])
    del h, gate8, up8, v, dgate, dup
    w = random_held(outs, cols, True, 7, scale=0.02)
    got = pvq.fp8_matmul(q, w, dtype=F32)
    exact = values @ ref.values(w).T
    assert np.all(np.abs(ref.to64(got[some]) - exact) <= 1.01 * ref.matmul_slack(values, ref.values(w).T, cols / 32))
    dy = torch.randn((rows, outs), generator=g, device="cuda", dtype=BF16)
    grad = pvq.fp8_weight_grad(dy, q)[:, cols - 128:]
    exponents = q.scales.view(torch.uint8)[:, cols // 128 - 1:].double() - 127
    exact = dy.double().t() @ (q.codes[:, cols - 128:].float().double() * torch.exp2(exponents))
    # 70000 / 16 steps in runs of 512: within 1e-6 of the norm, as by the sums' parts
    assert float((grad.double() - exact).norm()) <= 1e-6 * float(exact.norm())


@pytest.mark.parametrize("rows,inner,outer", [(1, 128, 200000), (2, 200000, 130), (100000, 40, 24)])
def test_matmul_of_long_sides(rows, inner, outer):
    a, b = random_held(rows, inner, False, 1), random_held(outer, inner, True, 2, scale=0.1)
    got = pvq.fp8_matmul(a, b, dtype=F32).double()
    va, vb = (pvq.fp8_dequantize(q, dtype=F32).double() for q in (a, b))
    want = va @ vb.t()
    # 1563 blocks of 128 in eight parts: 25000 values, 8e-8 of a sum for every 1024
    assert float((got - want).norm()) <= 3e-6 * float(want.norm())


@pytest.mark.parametrize("rows,inner,outer", [(70000, 130, 70), (300, 20000, 8), (300, 8, 20000)])
def test_weight_grad_of_long_sides(rows, inner, outer):
    dy, x = normal(rows, outer, BF16, 1), random_held(rows, inner, False, 2)
    got = pvq.fp8_weight_grad(dy, x).double()
    want = dy.double().t() @ pvq.fp8_dequantize(x, dtype=F32).double()
    assert float((got - want).norm()) <= 1e-6 * float(want.norm())


def test_rows_of_a_larger_matrix():
    """Views of some rows: other base addresses, the same values."""
    q, w = random_held(400, 500, False, 1), random_held(640, 500, True, 2)
    whole = pvq.fp8_matmul(q, w)
    some = pvq.Fp8Matrix(q.codes[37:301], q.scales[37:301], False)
    assert torch.equal(pvq.fp8_dequantize(some), pvq.fp8_dequantize(q)[37:301])
    assert torch.allclose(pvq.fp8_matmul(some, w).float(), whole[37:301].float(), rtol=2.0 ** -7, atol=1e-3)
    lower = pvq.Fp8Matrix(w.codes[128:], w.scales[1:], True)
    assert torch.allclose(pvq.fp8_matmul(q, lower).float(), whole[:, 128:].float(), rtol=2.0 ** -7, atol=1e-3)
    with pytest.raises(pvq.PvqError):  # scales that do not begin on a 4-byte boundary
        pvq.fp8_dequantize(pvq.Fp8Matrix(q.codes[:, 128:], q.scales[:, 1:], False))


def test_a_matrix_with_itself():
    q = random_held(300, 400, False, 1)
    got = pvq.fp8_matmul(q, q, dtype=F32)
    v = ref.values(q)
    assert np.all(np.abs(ref.to64(got) - v @ v.T) <= 2.0 ** -24 * np.abs(v @ v.T) + 1.01 * ref.matmul_slack(v, v.T, 400 / 32))
    h = pvq.fp8_gated(normal(5, 256, BF16, 1), normal(5, 256, BF16, 1))
    x = normal(5, 256, BF16, 1)
    one = pvq.fp8_gated(x, x)
    assert torch.equal(h.codes.view(torch.uint8), one.codes.view(torch.uint8))


def test_two_streams_at_once_and_graphs_with_workspaces():
    """Calls of every kernel on two streams, and two graphs replayed together, give what they give alone."""
    def calls(seed):
        x, dy = normal(2800, 1504, BF16, seed), normal(2800, 2104, BF16, seed + 1)
        w = pvq.fp8_quantize(normal(2104, 1504, BF16, seed + 2, scale=0.05), tile=True)
        few = normal(20, 1504, BF16, seed + 3)

        def run():
            q = pvq.fp8_quantize(x)
            y = pvq.fp8_matmul(q, w)
            return [y, pvq.fp8_matmul(pvq.fp8_quantize(few), w), pvq.fp8_matmul(pvq.fp8_quantize(y), w, transposed=True, dtype=F32),
                    pvq.fp8_weight_grad(dy, q), pvq.fp8_weight_grad(dy[:500], pvq.Fp8Matrix(q.codes[:500], q.scales[:500], False))]
        return run
    runs = [calls(10), calls(20)]
    want = [run() for run in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [None, None]
    for _ in range(3):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i] = runs[i]()
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(a, b) for a, b in zip(got[i], want[i]))
    graphs, outs = [], []
    for i in (0, 1):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            outs.append(runs[i]())
    for _ in range(3):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i]))

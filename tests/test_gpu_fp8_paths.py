"""The 8-bit products and weight gradients on every path that their sizes choose, the path itself asserted, so that a change of the rules
cannot take a path away from its tests: few rows with each height of a tile and each split of k, and longer than the rings of stages
and scales; weight gradients whose last round of tiles is shared."""
import pytest
import torch

import fp8_reference as ref
from fp8_launches import launches
from paper_2410_16926_b200 import pvq

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def held(rows, cols, tile, seed):
    """An Fp8Matrix of values whose rows are of different magnitudes; between its rows lie NaN, codes and scales."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, -(-cols // 4) * 4), generator=g, device="cuda") * torch.exp2(torch.randint(-3, 4, (rows, 1), generator=g, device="cuda").float())
    down, across = -(-rows // 128) if tile else rows, -(-cols // 128)
    codes = torch.full((rows, -(-cols // 16) * 16 + 16), 0x7f, dtype=torch.uint8, device="cuda")[:, :cols]
    scales = torch.full((down, -(-across // 4) * 4 + 4), 0xff, dtype=torch.uint8, device="cuda")[:, :across]
    return pvq.fp8_quantize(x[:, :cols], tile=tile, out=pvq.Fp8Matrix(codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu), tile))


def values(q):
    s = torch.exp2(q.scales.view(torch.uint8).double() - 127).repeat_interleave(128, dim=1)[:, :q.codes.shape[1]]
    if q.tile:
        s = s.repeat_interleave(128, dim=0)[:q.codes.shape[0]]
    return q.codes.double() * s


def check(got, va, vb, width, status):
    """Within a half step of the type, and what sums in fp32 may lose (`width` products a step of the tensor cores)."""
    want, magnitude = va @ vb, va.abs() @ vb.abs()
    slack = ref.HALF_STEP[got.dtype] * want.abs() + 1.01 * (va.shape[1] / width + 32) * 2.0 ** -23 * magnitude
    assert int(status.item()) == 0
    assert bool(((got.double() - want).abs() <= slack).all())


def guarded(rows, cols, dtype):
    whole = torch.full((rows + 2, -(-cols // 8) * 8 + 16), 77.0, dtype=dtype, device="cuda")
    out = whole[1:-1, :cols]

    def untouched():
        kept = out.clone()
        out.fill_(77.0)
        assert bool((whole == 77.0).all())
        out.copy_(kept)
    return out, untouched


# (How many clusters run at once differs between GPUs with the SMs that they have in a part: 33 to 37 of four, 15 to 18 of eight.  The numbers
# of tiles here keep away from those.)
# rows of a tile, split of k: outputs and k that lead there, with more than 16 blocks of 128 for each part (8 stages at most, 16 blocks of scales)
SHAPES = {(16, 8): (301, 20011), (16, 4): (5003, 9001), (16, 2): (12001, 5201), (16, 1): (13501, 2301),
          (32, 8): (301, 20011), (32, 4): (5003, 9001), (32, 2): (12001, 5201), (32, 1): (13501, 2301),
          (64, 8): (301, 20011), (64, 4): (2501, 9001), (64, 2): (8003, 4501), (64, 1): (12001, 2301),
          (128, 8): (301, 20011), (128, 4): (2501, 9001), (128, 2): (8003, 4501), (128, 1): (12001, 2301)}


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("high,split", list(SHAPES))
def test_products_of_few_rows(high, split, dtype, transposed):
    outer, inner = SHAPES[high, split]
    rows = {16: (3, 16), 32: (20, 32), 64: (33, 64), 128: (100, 128)}[high][dtype == BF16]
    a = held(rows, inner, transposed and dtype == F32, rows)  # (also in tiles)
    b = held(*((inner, outer) if transposed else (outer, inner)), True, outer)
    out, untouched = guarded(rows, outer, dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert launches(lambda: pvq.fp8_matmul(a, b, transposed=transposed, dtype=dtype)) == [
        ("matmul_few_kernel", (high, split, int(transposed), "bf16" if dtype == BF16 else "f32"), -(-outer // 128) * split, 1)]
    pvq.fp8_matmul(a, b, transposed=transposed, dtype=dtype, out=out, status=status)
    untouched()
    check(out, values(a), values(b) if transposed else values(b).t(), 32, status)


@pytest.mark.parametrize("tiles", [(False, True), (True, True), (True, False)])
@pytest.mark.parametrize("rows,inner,outer,split", [(300, 20011, 301, 8), (300, 9001, 1701, 2), (300, 2301, 5003, 1), (5000, 9001, 130, 1)])
def test_products_of_few_tiles(rows, inner, outer, split, tiles):
    """More rows than a tile has."""
    a, b = held(rows, inner, tiles[0], 1), held(outer, inner, tiles[1], 2)
    assert launches(lambda: pvq.fp8_matmul(a, b)) == [("matmul_few_kernel", (128, split, 0, "bf16"), -(-outer // 128) * split, -(-rows // 128))]
    for dtype in (BF16, F32):
        out, untouched = guarded(rows, outer, dtype)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        pvq.fp8_matmul(a, b, dtype=dtype, out=out, status=status)
        untouched()
        check(out, values(a), values(b).t(), 32, status)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,inner,outer,tile,last,split", [
    (2100, 2500, 2100, False, 16, 2), (2100, 2500, 2100, True, 16, 2),  # two rounds of tiles; a last column of tiles of 52 outputs: half of its quarters are empty
    (8200, 3700, 2660, False, 17, 2),                                   # three rounds; the last tiles are 100 by 116
    (8200, 3840, 1280, True, 1, 8), (4100, 3840, 1280, False, 1, 4), (8200, 3900, 1281, False, 22, 1)])
def test_weight_gradients_whose_last_round_is_shared(rows, inner, outer, tile, last, split, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows)
    dy = torch.randn((rows, -(-outer // 8) * 8 + 8), generator=g, device="cuda", dtype=BF16)[:, :outer]
    x = held(rows, inner, tile, inner)
    pairs = -(-outer // 256) * -(-inner // 256)
    t = "bf16" if dtype == BF16 else "f32"
    assert pairs % 74 == last
    for workspace in (True, False):
        ready = [("dequantize_kernel", ("bf16", 2))] if workspace else []
        if split > 1:
            want = ready + [("weight_grad_kernel", (0, 0, t), 4 * last * split), ("weight_grad_kernel", (1, int(workspace), t), 2 * min(74, pairs - last))]
        else:  # too many for clusters
            want = ready + [("weight_grad_kernel", (1, int(workspace), t), 2 * 74)]
        found = [k[:len(w)] for k, w in zip(launches(lambda: pvq.fp8_weight_grad(dy, x, dtype=dtype, workspace=workspace)), want, strict=True)]
        assert found == want
    out, untouched = guarded(outer, inner, dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    pvq.fp8_weight_grad(dy, x, dtype=dtype, out=out, status=status)
    untouched()
    check(out, dy.double().t(), values(x), 16, status)
    assert torch.equal(pvq.fp8_weight_grad(dy, x, dtype=dtype, workspace=False), out)

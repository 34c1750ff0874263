"""Where codes and scales of the groups that quantising can go wrong at lie, and when policies side
by side give the bits of one policy alone."""
import pytest

from test_gpu_fp4 import TYPES, U, check, weights

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("group", [32, 64, 128])
def test_codes_of_borders_ties_and_special_groups_lie_where_they_should(group):
    """The weights that malib_dequantize_fp4 gives and those that the header's places of codes and
    scales give are the same, at borders, ties, denormals, and in groups of NaN and infinities."""
    import paper_2106_07551_amd as M
    up = torch.nextafter(torch.tensor(2.5), torch.tensor(9.0)).item()
    down = torch.nextafter(torch.tensor(3.5), torch.tensor(0.0)).item()
    row = torch.tensor([6, .25, .2500001, .75, .7499999, 1.25, 1.2500001, 1.75, 1.7499999, 2.5, up,
                        3.5, down, 5, 5.000001, -0.25, -0.75, -6, -0.0, 1e-40, -1e-40])
    w = torch.zeros((21, 300), device="cuda")
    for r in range(21):   # every value in every place of a line
        w[r, r * 13:r * 13 + 21] = row.roll(r)
    w[3, 280], w[4, 140], w[5, 20] = float("nan"), float("inf"), -float("inf")
    w[6, :64] = 1e-45
    w[7, 64:128] = 3e38
    w[8, 128], w[8, 129] = 1e-38, -1e-38
    for dtype in TYPES:
        codes, scales = M.quantize_fp4(w.to(dtype), group)
        v = M.dequantize_fp4(codes, scales, 21, 300, dtype=torch.float32).double()
        at = weights(codes, scales, 21, 300)
        assert torch.equal(torch.isnan(v), torch.isnan(at))
        assert torch.equal(torch.nan_to_num(v, 7.0), torch.nan_to_num(at, 7.0))
        assert bool(torch.isnan(v).any()) and bool((v == 6).any())


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("groups, rows, n, k", [(16, 70, 250, 530), (24, 7, 600, 90), (5, 40, 18, 75),
                                                (16, 1, 64, 300), (24, 64, 333, 777),
                                                (40, 70, 500, 511), (200, 17, 100, 130),
                                                (12, 65, 512, 512)])
def test_policies_side_by_side_and_alone(dtype, groups, rows, n, k):
    """The order of a sum is that of the inputs' split, which goes by the type, the rows and the
    inputs alone up to 64 rows or 511 inputs, and in fp32: the same bits then.  Beyond, bf16
    rows may be split in two ways: each result is within its bound of the sum in 64 bits, so
    they are within twice that of each other."""
    import paper_2106_07551_amd as M
    g = torch.Generator(device="cuda").manual_seed(groups * n)
    w = torch.randn((groups, n, k), generator=g, device="cuda") * k ** -0.5
    codes, scales = M.quantize_fp4(w, 64)
    x = torch.randn((groups, rows, k), generator=g, device="cuda").to(dtype)
    b = torch.randn((groups, n), generator=g, device="cuda")
    y = check(x, codes, scales, n, b, M.ACT_RELU)
    for i in range(0, groups, max(1, groups // 8)):
        alone = check(x[i], codes[i], scales[i], n, b[i], M.ACT_RELU)
        if dtype is torch.float32 or rows <= 64 or k < 512:
            assert torch.equal(y[i], alone), i
            continue
        held = weights(codes[i], scales[i], n, k).abs().T.contiguous()
        size = x[i].double().abs() @ held + b[i].double().abs()
        # (the sum in 64 bits is alone's value to 2^-8 of it and a little more: 2^-16 of the rounding)
        bound = 2 * (1.13 * (k + 8) * U * size + 1.01 * 2.0 ** -8 * alone.double().abs()
                     + 2.0 ** -16 * size + 1e-36)
        assert bool(((y[i].double() - alone.double()).abs() <= bound).all()), i

"""Layers in 4 bits at the ends of fp32's range: results that fit fp32 come out finite, whatever
the way to them holds."""
import pytest

from test_gpu_fp4 import TYPES, check, weights

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# one block of inputs, few and many outputs; inputs split over wavefronts; rows through LDS
SIZES = [(1, 20, 100), (40, 9000, 100), (1, 40, 700), (33, 300, 777), (64, 4000, 1030),
         (70, 4161, 1027), (100, 4096, 600)]


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows, n, k", SIZES)
def test_sums_whose_products_with_scales_fit(dtype, group, rows, n, k):
    """Rows of 2^119 (32 terms of up to 6 leave fp32 before the scale, which is about 0.5 k^-0.5,
    brings them back), of one 2^126 among small ones (a term of its own does), and ordinary ones,
    whose bits do not depend on their neighbours.  A sum formed again takes one rounding more (its product
    with the scale: u of it), which the bound's (k + 8) u has room for."""
    import paper_2106_07551_amd as M
    g = torch.Generator(device="cuda").manual_seed(rows + n)
    w = torch.randn((n, k), generator=g, device="cuda") * k ** -0.5
    codes, scales = M.quantize_fp4(w, group)
    x = torch.randn((rows, k), generator=g, device="cuda")
    plain = x.to(dtype)
    x[::3] = x[::3].abs() * 2.0 ** 119
    x[1::9, k // 2] = 2.0 ** 126
    x = x.to(dtype)
    y = check(x, codes, scales, n, what="large")
    assert bool(torch.isfinite(y).all())
    big = (x != plain).any(1)
    alone = M.linear_fp4(plain, codes, scales, n)
    assert torch.equal(y[~big], alone[~big])
    # infinite and NaN inputs make what they make in 64 bits, in their own rows only
    bad = x.clone()
    bad[0, k - 1] = float("inf")
    bad[rows // 2, 0] = float("nan")
    z = bad.double() @ weights(codes, scales, n, k).T.contiguous()
    got = M.linear_fp4(bad, codes, scales, n)
    touched = ~torch.isfinite(bad).all(1)
    assert torch.equal(got[~touched], y[~touched])
    assert torch.equal(torch.isnan(got[touched]), torch.isnan(z[touched]))
    inf = torch.isinf(z)
    assert torch.equal(got.double()[inf], z[inf])


def test_sums_of_the_largest_inputs_exactly():
    """Whole numbers times 2^122: 128 terms of 6 are 768 x 2^122, beyond fp32, and with the scale 2^-8
    3 x 2^122, exactly."""
    import paper_2106_07551_amd as M
    for n, rows, k in ((16, 3, 128), (40, 1, 512), (4096, 70, 512)):
        w = torch.full((n, k), 6 * 2.0 ** -8, device="cuda")
        w[1::2] *= -1
        for dtype in TYPES:
            x = torch.full((rows, k), 2.0 ** 122, device="cuda").to(dtype)
            want = 6 * 2.0 ** -8 * k * 2.0 ** 122
            for group in (32, 64, 128):
                y = M.linear_fp4(x, *M.quantize_fp4(w, group), n)
                assert bool((y[:, ::2] == want).all()) and bool((y[:, 1::2] == -want).all())


@pytest.mark.parametrize("group", [32, 64, 128])
def test_the_largest_weights_come_back_finite(group):
    """Scales up to 85 x 2^119, six of which are bf16's largest number: larger weights take code 6 of
    it.  The others' scales as they always are, down to the last bit."""
    import paper_2106_07551_amd as M
    most = 85 * 2.0 ** 119
    limit = torch.tensor(1023 * 2.0 ** 118, device="cuda")
    far = torch.tensor(3e38, device="cuda")
    zero = torch.zeros((), device="cuda")
    tops = torch.stack([torch.tensor(torch.finfo(torch.float32).max, device="cuda"),
                        torch.tensor(torch.finfo(torch.bfloat16).max, device="cuda"),
                        torch.tensor(3.4e38, device="cuda"), torch.nextafter(limit, far),
                        torch.nextafter(limit, zero), limit, far, far / 3])
    w = torch.zeros((len(tops), 256), device="cuda")
    w[:, 5], w[:, 6], w[:, 7], w[:, 200] = tops, -tops, tops / 2, -tops / 4
    codes, scales = M.quantize_fp4(w, group)
    sixth = torch.tensor(1 / 6, dtype=torch.float32, device="cuda")
    want = (tops * sixth).bfloat16().double().clamp(max=most)
    assert torch.equal(scales[0, 0, :len(tops), 0].double(), want)
    assert float(want[0]) == most and 6 * most == torch.finfo(torch.bfloat16).max
    for dtype in TYPES:
        v = M.dequantize_fp4(codes, scales, len(tops), 256, dtype=dtype)
        assert bool(torch.isfinite(v).all())
        # (rounded to `dtype`: 6 s has up to 10 bits, bf16 holds 8)
        assert torch.equal(v[:, 5], (6 * want).to(dtype)) and torch.equal(v[:, 6], -v[:, 5])
        assert torch.equal(v[:, 7], (3 * want).to(dtype))
    assert torch.equal(weights(codes, scales, len(tops), 256), M.dequantize_fp4(
        codes, scales, len(tops), 256, dtype=torch.float32).double())
    x = torch.zeros((2, 256), device="cuda")
    x[0, 5], x[1, 6] = 1.0, 0.5
    y = M.linear_fp4(x, codes, scales, len(tops))
    assert torch.equal(y[0].double(), 6 * want) and torch.equal(y[1].double(), -3 * want)

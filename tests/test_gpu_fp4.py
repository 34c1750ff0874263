"""Layers in 4 bits on the GPU (malib_quantize_fp4, malib_dequantize_fp4, malib_linear_fp4)
against the definitions in 64 bits.

Codes, scales and the weights they stand for are exact.  A product's terms are exact; their
sum takes at most K additions in fp32: K u of the sum of the terms' magnitudes (u = 2^-24);
bias, activation and residual a few u of what they give (gelu: 2e-6), and slopes up to 1.13;
the output's rounding 2^-8 of it in bf16, u in fp32."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]
VALUES = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6],
                      dtype=torch.float64)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def padded(t, pad, shift=0):
    n, k = t.shape[-2:]
    wide = torch.full((t.numel() // k * (k + pad) + shift,), 3.0, dtype=t.dtype, device=t.device)
    v = wide[shift:].view(t.shape[:-1] + (k + pad,))[..., :k]
    v.copy_(t)
    return v


def weights(codes, scales, n, k):
    """Weight by weight, as the header says where code and scale lie."""
    if codes.dim() == 5:
        return torch.stack([weights(c, s, n, k) for c, s in zip(codes, scales)])
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(k, device="cuda")[None, :]
    byte = codes[i // 16, j // 128, j % 32 // 8 * 16 + i % 16, j % 128 // 32 * 4 + j % 8 // 2]
    code = (byte.long() >> (4 * (j % 2))) & 15
    group = 128 // scales.shape[-1]
    return VALUES.cuda()[code] * scales[i // 16, j // 128, i % 16, j % 128 // group].double()


def quantized64(w, group):
    """(scales [..][out][in / group], values) from the definition: every value's distance."""
    w = w.double()
    n, k = w.shape
    full = torch.nn.functional.pad(w, (0, -k % group)).reshape(n, -1, group)
    most = full.abs().amax(-1)
    sixth = torch.tensor(1 / 6, dtype=torch.float32, device=w.device)
    s = (most.float() * sixth).bfloat16().double()
    s = torch.where(torch.isfinite(full).all(-1), s, float("nan"))
    r = full.abs() / torch.where(s > 0, s, 1.0)[..., None]
    best = torch.zeros_like(r)
    for start in (1, 0):
        for v in VALUES[start:8:2].tolist():
            near, now = (r - v).abs(), (r - best).abs()
            best = torch.where((near < now) if start else (near <= now), v, best)
    best = torch.where(s[..., None] > 0, best, 0.0)
    val = torch.where(torch.isnan(s)[..., None], float("nan"), best * torch.sign(full) * s[..., None])
    return s, val.reshape(n, -1)[:, :k]


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n, k", [(1, 1), (3, 31), (16, 128), (17, 129), (40, 777), (333, 24),
                                  (250, 1000)])
def test_quantize(dtype, group, n, k):
    import paper_2106_07551_amd as M
    w = (torch.randn((n, k), device="cuda") * 0.1).to(dtype)
    w[0, 0] = 0.3
    for pad, shift in ((0, 0), (3, 1)):
        codes, scales = M.quantize_fp4(padded(w, pad, shift), group)
        s, val = quantized64(w, group)
        got = weights(codes, scales, n, k)
        assert torch.equal(got, val)
        i, j = torch.arange(n, device="cuda")[:, None], torch.arange(s.shape[1], device="cuda")
        per = 128 // group
        assert torch.equal(scales[i // 16, j // per, i % 16, j % per].double(), s)
        # padding: zeros
        nt, kb = codes.shape[:2]
        whole = weights(codes, scales, nt * 16, kb * 128)
        assert bool((whole[n:] == 0).all()) and bool((whole[:, k:] == 0).all())
        out = padded(torch.zeros((n, k), device="cuda"), 5)
        assert M.dequantize_fp4(codes, scales, n, k, out=out) is out
        assert torch.equal(out.double(), val)
        half = M.dequantize_fp4(codes, scales, n, k)
        assert half.dtype is torch.bfloat16 and torch.equal(half, val.float().bfloat16())


def test_borders_ties_and_special_groups():
    """A group's largest magnitude 6 makes its scale 1: borders are then at hand."""
    import paper_2106_07551_amd as M
    up = torch.nextafter(torch.tensor(2.5), torch.tensor(9.0)).item()
    down = torch.nextafter(torch.tensor(3.5), torch.tensor(0.0)).item()
    row = [6, .25, .2500001, .75, .7499999, 1.25, 1.2500001, 1.75, 1.7499999, 2.5, up, 3.5, down,
           5, 5.000001, -0.25, -0.75, -6, -0.0, 1e-40, -1e-40]
    want = [6, 0, .5, 1, .5, 1, 1.5, 2, 1.5, 2, 3, 4, 3, 4, 6, 0, -1, -6, 0, 0, 0]
    w = torch.zeros((4, 128), device="cuda")
    w[0, :len(row)] = torch.tensor(row)
    w[1, 0], w[1, 32], w[1, 64] = float("nan"), float("inf"), 2.0
    w[2, :32] = 1e-45          # the scale rounds to 0
    w[2, 32:64] = 3e38
    w[3, 0], w[3, 1] = 1e-38, -1e-38
    codes, scales = M.quantize_fp4(w, 32)
    v = M.dequantize_fp4(codes, scales, 4, 128, dtype=torch.float32)
    assert v[0, :len(row)].tolist() == want
    # 2 / 6 in bf16 is 0.333984375 (171 / 512)
    assert bool(torch.isnan(v[1, :64]).all())
    assert v[1, 64:].tolist() == [6 * 171 / 512] + [0.0] * 63
    assert bool((v[2, :32] == 0).all())
    assert bool(torch.isfinite(v[2, 32:64]).all())
    assert torch.equal(v.double(), weights(codes, scales, 4, 128)) or bool(torch.isnan(v).any())
    _, val = quantized64(w, 32)
    assert torch.equal(torch.nan_to_num(v.double(), 7.0), torch.nan_to_num(val, 7.0))


@pytest.mark.parametrize("exponent", [0, -118, -126, -131, 100, 119, 123])
def test_every_bf16_weight_of_some_scales(exponent):
    """All magnitudes of bf16 up to the largest of their group, ties among them, for every
    significand of the largest, and scales from denormal to near the top."""
    import paper_2106_07551_amd as M
    top = torch.arange(128, 256, device="cuda").float() * 2.0 ** (exponent - 7)
    low = torch.arange(128, 256, device="cuda").float() * 2.0 ** (exponent - 7)
    for down in range(7):
        w = torch.zeros((128, 1024), device="cuda")
        # 31 others and the largest in each group of 32: 128 significands in 5 groups
        part = torch.nn.functional.pad(low * 2.0 ** -down, (0, 27)).view(5, 31)
        w[:, :160].view(128, 5, 32)[:, :, :31] = part
        w[:, :160].view(128, 5, 32)[:, :, 31] = top[:, None]
        w = torch.where(w.abs() > torch.cat([top[:, None]], 1), -top[:, None], w)
        w[:, ::2] *= -1
        w = w.bfloat16()
        codes, scales = M.quantize_fp4(w, 32)
        _, val = quantized64(w, 32)
        assert torch.equal(M.dequantize_fp4(codes, scales, 128, 1024, dtype=torch.float32).double(),
                           val), down


def act64(act, z):
    import paper_2106_07551_amd as M
    if act == M.ACT_RELU:
        return torch.where(z > 0, z, 0.0 * z)
    if act == M.ACT_GELU:
        return z * torch.special.ndtr(z)
    return z * torch.sigmoid(z) if act == M.ACT_SILU else z


def check(x, codes, scales, n, bias=None, act=0, residual=None, what="", **kw):
    import paper_2106_07551_amd as M
    k = x.shape[-1]
    w = weights(codes, scales, n, k)
    y = M.linear_fp4(x, codes, scales, n, bias, act=act, residual=residual, **kw)
    z = x.double() @ w.transpose(-1, -2).contiguous()
    size = x.double().abs() @ w.abs().transpose(-1, -2).contiguous()
    if bias is not None:
        z = z + bias.double().unsqueeze(-2)
        size = size + bias.double().abs().unsqueeze(-2)
    a = act64(act, z)
    ref = a if residual is None else a + residual.double()
    eps = U if x.dtype is torch.float32 else 2.0 ** -8
    tol = 1.13 * (k + 8) * U * size + 3e-6 * a.abs() + 2 * U * ref.abs() + 1.01 * eps * ref.abs() \
        + 1e-36
    bad = ~((y.double() - ref).abs() <= tol)
    assert not bad.any(), (what, float(((y.double() - ref).abs() / tol).max()),
                           bad.nonzero()[:4].tolist())
    return y


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows", [1, 2, 7, 16, 17, 33, 64, 65, 150])
@pytest.mark.parametrize("n, k", [(5, 3), (16, 128), (50, 200), (333, 777), (64, 2048),
                                  (130, 4100)])
def test_linear(dtype, group, rows, n, k):
    import paper_2106_07551_amd as M
    codes, scales = M.quantize_fp4(torch.randn((n, k), device="cuda") * k ** -0.5, group)
    x = torch.randn((rows, k), device="cuda").to(dtype)
    bias = torch.randn(n, device="cuda")
    r = torch.randn((rows, n), device="cuda").to(dtype)
    y = check(x, codes, scales, n, what="plain")
    assert torch.equal(y, M.linear_fp4(x, codes, scales, n))
    check(padded(x, 3, 1), codes, scales, n, bias, M.ACT_GELU, padded(r, 1), "gelu")
    out = padded(torch.zeros_like(r), 5, 1)
    assert check(padded(x, 8), codes, scales, n, None, M.ACT_SILU, r, "silu", out=out) is out
    ri = r.clone()   # over the residual
    assert M.linear_fp4(x, codes, scales, n, bias, act=M.ACT_RELU, residual=ri, out=ri) is ri
    assert torch.equal(ri, check(x, codes, scales, n, bias, M.ACT_RELU, r, "relu"))


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows, n, k", [(65, 4200, 512), (100, 4090, 600), (129, 2563, 1111),
                                        (70, 4161, 1027), (97, 4096, 2560), (200, 1800, 5000),
                                        (40, 9000, 100), (3, 3001, 128), (64, 20000, 17)])
def test_enough_workgroups_for_the_card(dtype, group, rows, n, k):
    """Sizes that fill the CUs: rows through LDS, several tiles a wavefront, outputs of their own."""
    import paper_2106_07551_amd as M
    codes, scales = M.quantize_fp4(torch.randn((n, k), device="cuda") * k ** -0.5, group)
    x = torch.randn((rows, k), device="cuda").to(dtype)
    bias = torch.randn(n, device="cuda")
    r = torch.randn((rows, n), device="cuda").to(dtype)
    y = check(x, codes, scales, n, what="plain")
    assert torch.equal(y, M.linear_fp4(x, codes, scales, n))
    out = padded(torch.zeros_like(r), 3, 1)
    assert check(padded(x, 1, 1), codes, scales, n, bias, M.ACT_GELU, padded(r, 1), "gelu",
                 out=out) is out
    z = torch.zeros_like(x)
    z[rows - 1] = x[rows - 1]
    last = M.linear_fp4(z, codes, scales, n)
    assert bool((last[:-1] == 0).all()) and torch.equal(last[-1], y[-1])


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("groups, rows, n, k", [(16, 70, 250, 530), (24, 7, 600, 90), (1, 3, 20, 40), (3, 5, 33, 150), (5, 40, 18, 75),
                                                (16, 1, 64, 300)])
def test_policies_side_by_side(dtype, groups, rows, n, k):
    import paper_2106_07551_amd as M
    w = torch.randn((groups, n, k), device="cuda") * k ** -0.5
    codes, scales = M.quantize_fp4(w, 64)
    assert codes.shape[0] == groups
    x = torch.randn((groups, rows, k), device="cuda").to(dtype)
    b, r = torch.randn((groups, n), device="cuda"), torch.randn((groups, rows, n),
                                                                device="cuda").to(dtype)
    y = check(x, codes, scales, n, b, M.ACT_RELU, r)
    for g in range(groups):
        one = M.quantize_fp4(w[g], 64)
        assert torch.equal(one[0], codes[g]) and torch.equal(one[1], scales[g])
        alone = check(x[g], codes[g], scales[g], n, b[g], M.ACT_RELU, r[g])
        # (the order of sums goes by the sizes, of which the number of policies is one)
        assert torch.equal(y[g], alone) or groups * rows * n > 16384
    shared = M.linear_fp4(x[0], codes, scales, n)
    assert torch.equal(shared, M.linear_fp4(x[:1].expand(groups, -1, -1).contiguous(), codes,
                                            scales, n))
    half = M.dequantize_fp4(codes, scales, n, k, dtype=torch.float32)
    assert torch.equal(half.double(), weights(codes, scales, n, k))


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 16, 100])
def test_whole_numbers_are_exact(dtype, rows):
    """Whole numbers whose sums stay below 2^24: any order of additions gives them exactly."""
    import paper_2106_07551_amd as M
    n, k = 70, 1111
    for group in (32, 64, 128):
        w = torch.randint(-6, 7, (n, k), device="cuda").float()
        w[:, ::32] = 6.0     # scales are 1
        codes, scales = M.quantize_fp4(w, group)
        v = M.dequantize_fp4(codes, scales, n, k, dtype=torch.float32)
        x = torch.randint(-9, 10, (rows, k), device="cuda").to(dtype)
        ref = (x.double() @ v.double().T.contiguous())
        y = M.linear_fp4(x, codes, scales, n)
        assert torch.equal(y, ref.to(dtype))


def test_fp32_inputs_keep_their_bits():
    """One weight of 1 per output (and a 6 in every group, where x is 0, so that scales are 1): y is
    x itself, whatever its bits; infinities and NaN stay in their own rows."""
    import paper_2106_07551_amd as M
    k = 256
    w = torch.eye(k, device="cuda")
    w[:, ::32] = 6.0
    codes, scales = M.quantize_fp4(w, 32)
    x = torch.randn((3, k), device="cuda") * torch.logspace(-30, 30, k, device="cuda")
    x[0, 1:5] = torch.tensor([3.4028235e38, -3.4028235e38, 1.17549435e-38, 1 + 2 ** -23])
    x[:, ::32] = 0.0
    i = torch.arange(k, device="cuda") % 32 > 0
    assert torch.equal(M.linear_fp4(x, codes, scales, k)[:, i], x[:, i])
    x[1, 5] = float("inf")
    x[2, 6] = float("nan")
    y = M.linear_fp4(x, codes, scales, k)
    assert torch.equal(y[0, i], x[0, i]) and float(y[1, 5]) == float("inf")
    assert bool(torch.isnan(y[2]).all())


def test_padding_takes_no_part():
    """Codes and scales beyond the layer's sizes may hold anything."""
    import paper_2106_07551_amd as M
    for group in (32, 64):
        n, k = 20, 40
        codes, scales = M.quantize_fp4(torch.randn((n, k), device="cuda"), group)
        x = torch.randn((3, k), device="cuda")
        y = M.linear_fp4(x, codes, scales, n)
        i = torch.arange(32, device="cuda")[:, None]
        j = torch.arange(128 // group, device="cuda")[None, :]
        dirty = scales.clone()
        beyond = (i >= n) | (j * group >= k)
        dirty[i // 16, 0, i % 16, j] = torch.where(beyond, float("nan"),
                                                   dirty[i // 16, 0, i % 16, j])
        c = codes.clone()
        c[1, :, 4:16] = 0xFF           # outputs 20 to 31 of the lines 0 to 15
        c[:, :, :, 8:] = 0xFF           # inputs from 64 on
        assert torch.equal(M.linear_fp4(x, c, dirty, n), y)


def test_no_rows():
    import paper_2106_07551_amd as M
    codes, scales = M.quantize_fp4(torch.randn((20, 40), device="cuda"))
    assert M.linear_fp4(torch.empty((0, 40), device="cuda"), codes, scales, 20).shape == (0, 20)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("groups, rows, n, k", [(3, 17, 40, 200), (2, 70, 4000, 600)])
def test_rows_beyond_32_bits(dtype, groups, rows, n, k):
    """Rows of x, y and the residual and policies of x that are far apart (no difference to the
    result at all), and weights that are."""
    import paper_2106_07551_amd as M
    g = torch.Generator(device="cuda").manual_seed(rows)
    apart = ((1 << 32) // (rows * groups) + 1) | 1

    def far(t):
        lead, (r, c) = t.shape[0], t.shape[1:]
        wide = torch.empty((lead * r - 1) * apart + c, dtype=t.dtype, device="cuda")
        return wide.as_strided(t.shape, (r * apart, apart, 1)).copy_(t)

    w = torch.randn((groups, n, k), generator=g, device="cuda").to(dtype)
    x = torch.randn((groups, rows, k), generator=g, device="cuda").to(dtype)
    res = torch.randn((groups, rows, n), generator=g, device="cuda").to(dtype)
    codes, scales = M.quantize_fp4(w)
    y = check(x, codes, scales, n, residual=res)
    assert torch.equal(M.linear_fp4(far(x), codes, scales, n, residual=far(res),
                                    out=far(torch.zeros_like(res))), y)
    if n < 100:
        apart = (1 << 32) // (n * groups) + 1
        c, s = M.quantize_fp4(far(w))
        assert torch.equal(c, codes) and torch.equal(s.view(torch.int16), scales.view(torch.int16))
        plain = M.dequantize_fp4(codes, scales, n, k, dtype=dtype)
        assert torch.equal(M.dequantize_fp4(codes, scales, n, k, dtype=dtype,
                                            out=far(torch.zeros_like(plain))), plain)

"""The learner's linear layer on the GPU (malib_linear, malib_linear_backward)
against the formulas in 64 bits.

Tolerances.  Inputs are taken as they are (bf16 values are exact in 64 bits).
A sum of n fp32 products in any order is within (n + 2) 2^-24 sum |a b| of the
exact one, worst case; with signs at random the error is about sqrt(n) 2^-24 of
the root of the sum of squares, so 8 sqrt(n) 2^-24 sqrt(sum (a b)^2) bounds
every element with room to spare, plus the output's own rounding (2^-8 of it in
bf16, 2^-24 in fp32), plus a few 2^-24 of the terms of the epilogue.  The
backward pass rounds dz to bf16 where there is a smooth activation: 2^-8 of each
product's size, again as a root of squares (factor 4).  Activations are
Lipschitz (1.13 for GELU, 1.1 for SiLU) and evaluated to a few fp32 ulps."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ACTS = ["none", "relu", "gelu", "silu"]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _code(act):
    import paper_2106_07551_amd as MA
    return {"none": MA.ACT_NONE, "relu": MA.ACT_RELU, "gelu": MA.ACT_GELU,
            "silu": MA.ACT_SILU}[act]


def act64(name, z):
    if name == "relu":
        return torch.where(z > 0, z, 0 * z)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope64(name, z):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def view(t, pad, shift=0):
    """t as a view with `pad` spare elements behind each row, `shift` before the
    first, all NaN: whatever is read there shows."""
    lead = t.shape[:-1]
    n = t.shape[-1]
    wide = torch.full((math.prod(lead) * (n + pad) + shift,), float("nan"), dtype=t.dtype,
                      device=t.device)
    v = wide[shift:].view(*lead, n + pad)[..., :n]
    v.copy_(t)
    return v


def close(got, ref, bound, dtype, what):
    eps = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    err = (got.double() - ref).abs()
    tol = bound + 1.01 * eps * ref.abs() + 1e-30
    assert torch.isfinite(got).all(), what
    assert (err <= tol).all(), (what, float((err / tol).max()))


def sums(a, b):
    """(a b^T, root of the sums of squares) in 64 bits over the last index."""
    return a @ b.transpose(-1, -2).contiguous(), \
        torch.sqrt((a * a) @ (b * b).transpose(-1, -2).contiguous())


def inputs(dtype, G, M, K, N, seed, pad=0, shift=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    lead = () if G is None else (G,)

    def normal(*shape, t=dtype):
        return torch.randn(lead + shape, generator=g, device="cuda").to(t)

    x, w = normal(M, K), (normal(N, K, t=torch.float32) * K ** -0.5).to(dtype)
    b, r, dy = normal(N, t=torch.float32), normal(M, N), normal(M, N)
    return view(x, pad, shift), view(w, pad, shift), b, view(r, pad, shift), view(dy, pad, shift)


def check_layer(dtype, G, M, K, N, act, *, bias=True, residual=True, pad=0, shift=0, seed=1):
    import paper_2106_07551_amd as MA
    tag = f"{dtype} G={G} {M}x{K}->{N} {act} pad={pad} shift={shift}"
    print("[linear]", tag, flush=True)
    x, w, b, r, dy = inputs(dtype, G, M, K, N, seed, pad, shift)
    b, r = b if bias else None, r if residual else None
    pre = torch.empty(dy.shape, dtype=dtype, device="cuda")
    y = MA.linear(x, w, b, act=_code(act), residual=r, pre=pre)
    u = 2.0 ** -24
    xd, wd = x.double(), w.double()
    z, q = sums(xd, wd)
    mag = q * 8 * math.sqrt(K) * u
    if bias:
        z = z + b.double().unsqueeze(-2)
        mag = mag + 4 * u * z.abs()
    ref = act64(act, z)
    if residual:
        ref = ref + r.double()
        mag = mag + 4 * u * (ref.abs() + r.double().abs())
    close(pre, z, mag, dtype, tag + " pre")
    close(y, ref, 1.2 * mag + 8 * u * z.abs(), dtype, tag + " y")
    dx, dw, db = MA.linear_backward(dy, x, w, act=_code(act), pre=pre if act != "none" else None)
    s = slope64(act, pre.double())
    dz = dy.double() * s
    rough = 4 * 2.0 ** -8 if dtype == torch.bfloat16 and act in ("gelu", "silu") else 0.0
    fine = 8 * u    # the derivative itself
    ref, q = sums(dz, wd.transpose(-1, -2).contiguous())
    _, q1 = sums(dy.double(), wd.transpose(-1, -2).contiguous())
    close(dx, ref, q * (8 * math.sqrt(N) * u + rough) + 4 * q1 * fine, dtype, tag + " dx")
    ref, q = sums(dz.transpose(-1, -2).contiguous(), xd.transpose(-1, -2).contiguous())
    _, q1 = sums(dy.double().transpose(-1, -2).contiguous(), xd.transpose(-1, -2).contiguous())
    close(dw, ref, q * (8 * math.sqrt(M) * u + rough) + 4 * q1 * fine, dtype, tag + " dw")
    mag = torch.sqrt((dy.double() ** 2).sum(-2)) * 8 * (math.sqrt(M) * u + fine)
    close(db, dz.sum(-2), mag, torch.float32, tag + " db")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_activations(dtype, act):
    check_layer(dtype, None, 130, 96, 72, act)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_gelu_relative_to_itself(dtype):
    """GELU and its slope z by z, far into the tail, through every kernel that
    evaluates them.  Products of z with ones and zeros are exact, so each output is
    the function's, rounded once.  Roundings in fp32, u = 2^-24 each: of 1 / (1 + q |z|)
    3, which the fit in it magnifies by up to 2.5; of a sum of ten terms 3, the fit
    itself 0.5; of the exponential 2 and, from its exponent, 1.5 z^2; of the
    products 4: under (18 + 2 z^2) u of Phi and of z phi.  Then the output's rounding."""
    import paper_2106_07551_amd as MA
    u = 2.0 ** -24
    z = torch.linspace(-12.0, 8.0, 20001, device="cuda").to(dtype)
    zd = z.double()
    phi, cdf = torch.exp(-zd * zd / 2) / math.sqrt(2 * math.pi), \
        0.5 * torch.special.erfc(-zd / math.sqrt(2))
    half = 1.01 * (2.0 ** -8 if dtype == torch.bfloat16 else u)
    own = (18 + 2 * zd * zd) * u

    def check(got, ref, bound, what):
        err, tol = (got.double() - ref).abs(), bound + half * ref.abs()
        assert (err <= tol).all(), (what, float((err / tol).max()), float(zd[(err / tol).argmax()]))

    one = torch.ones((1, 1), dtype=dtype, device="cuda")
    value, slope = zd * cdf, cdf + zd * phi
    vb, sb = own * value.abs(), own * (cdf + (zd * phi).abs())
    col = z[:, None].contiguous()
    check(MA.linear(col, one, act=MA.ACT_GELU)[:, 0], value, vb, "tiles")
    check(MA.linear(one, col, act=MA.ACT_GELU)[0], value, vb, "few rows")
    dy = torch.ones_like(col)
    dx, _, _ = MA.linear_backward(dy, col, one, act=MA.ACT_GELU, pre=col)
    check(dx[:, 0], slope, sb, "slope, few values")
    n, m = 64, 312 * 64                       # more than 2^20 values, more than 128 inputs
    pre = col[:m].view(-1, n).repeat(64, 1)
    w = torch.zeros((n, 136), dtype=dtype, device="cuda")
    w[:, :n].fill_diagonal_(1.0)
    x = torch.zeros((pre.shape[0], 136), dtype=dtype, device="cuda")
    dx, _, _ = MA.linear_backward(torch.ones_like(pre), x, w, act=MA.ACT_GELU, pre=pre)
    got = dx[:, :n].reshape(64, m)
    assert (got == got[:1]).all()
    check(torch.cat([got[0], dx.new_zeros(zd.numel() - m)]), torch.cat([slope[:m], 0 * zd[m:]]),
          sb, "slope, many values")


# one row, one unit, one input; both sides of chunks, tiles and stages; the
# policies' own layers; long sums that are split over workgroups
SIZES = [(1, 1, 1), (1, 24, 64), (3, 5, 7), (2, 8, 3), (64, 64, 64), (65, 63, 66), (127, 129, 31),
         (128, 128, 128), (129, 200, 255), (256, 75, 256), (24, 256, 18), (192, 512, 18),
         (300, 24, 64), (5, 4096, 40), (2, 2048, 2056), (4100, 33, 17), (3000, 128, 96),
         (1000, 777, 333), (520, 264, 392), (1, 1024, 1024), (16, 513, 1024)]


@pytest.mark.parametrize("M, K, N", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_sizes(dtype, M, K, N):
    check_layer(dtype, None, M, K, N, "relu" if (M + K) % 2 else "silu", bias=N % 3 != 0,
                residual=K % 2 == 0, seed=M + K + N)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("M, K, N", [(2050, 1024, 1032), (4096, 2048, 512), (257, 4104, 520)])
def test_large_tiles(dtype, M, K, N):
    check_layer(dtype, None, M, K, N, "relu")


@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("M, K, N", [(2050, 1024, 1032), (4096, 520, 1304), (700, 2049, 3001)])
def test_large_sizes_unaligned(dtype, M, K, N, act):
    """Sizes that get the largest tiles, with rows that do not start on 16-byte
    boundaries."""
    check_layer(dtype, None, M, K, N, act, pad=1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("M", [1, 3, 7, 16, 17])
@pytest.mark.parametrize("K, N, G", [(8192, 136, None), (1024, 1000, 3), (130, 17, 2), (4100, 33, None),
                                     (96, 2000, None)])
def test_few_rows(dtype, M, K, N, G):
    check_layer(dtype, G, M, K, N, "silu")
    check_layer(dtype, G, M, K, N, "relu", pad=3, shift=1, bias=False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("G, M, K, N, act", [(1, 60001, 6, 24, "gelu"), (1, 40000, 40, 11, "relu"),
                                             (3, 30000, 16, 5, "silu"), (1, 50000, 200, 72, "silu"),
                                             (2, 9000, 320, 5, "gelu"), (1, 30000, 128, 64, "none")])
def test_many_rows_of_narrow_layers(dtype, G, M, K, N, act):
    """dW's sums in hundreds of parts, dbias from either kernel, dz's rows padded."""
    check_layer(dtype, G, M, K, N, act, residual=False)
    check_layer(dtype, G, M, K, N, act, residual=False, pad=3)


@pytest.mark.parametrize("rows", [(1 << 30) + 70, (1 << 31) - 1])
def test_most_rows(rows):
    """More tiles than one launch has threads for, and rows whose rounding up to
    tiles passes 31 bits.  Every number is exact: sums of
    ones stay below 2^24 in each part, and the parts' sum is rounded once at most."""
    import paper_2106_07551_amd as MA
    base = torch.randn((1 << 20) + 7, device="cuda").bfloat16()
    x = base.repeat(rows // base.numel() + 1)[:rows].view(rows, 1)
    w = torch.full((1, 1), 2.0, dtype=torch.bfloat16, device="cuda")
    print("[linear] most rows, forward", flush=True)
    y = MA.linear(x, w)
    assert torch.equal(y, x * 2)
    dy = torch.ones_like(x)
    print("[linear] most rows, backward", flush=True)
    dx, dw, db = MA.linear_backward(dy, dy, w)
    assert (dx == 2).all()
    assert float(dw) == float(torch.tensor(float(rows)).bfloat16())
    assert abs(float(db) - rows) <= 2.0 ** -23 * rows


@pytest.mark.parametrize("pad, shift", [(1, 0), (8, 0), (8, 1), (3, 5), (0, 2)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_strides_and_alignment(dtype, pad, shift):
    check_layer(dtype, None, 150, 88, 104, "gelu", pad=pad, shift=shift)
    check_layer(dtype, 3, 70, 40, 24, "relu", pad=pad, shift=shift)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("G, M, K, N", [(1, 40, 24, 64), (5, 200, 24, 64), (16, 33, 64, 3),
                                        (7, 1, 300, 20)])
def test_groups(dtype, G, M, K, N):
    check_layer(dtype, G, M, K, N, "relu")


def test_shared_input_and_strided_groups():
    """x shared by the groups; x, y and dx interleaved ([rows][groups][width])."""
    import paper_2106_07551_amd as MA
    G, M, K, N = 4, 50, 40, 24
    x, w, b, r, dy = inputs(torch.float32, G, M, K, N, 3)
    y = MA.linear(x[0].contiguous(), w, b, act=MA.ACT_RELU)
    one = MA.linear(x[:1].expand(G, M, K).contiguous(), w, b, act=MA.ACT_RELU)
    assert torch.equal(y, one)
    xs = x.transpose(0, 1).contiguous().transpose(0, 1)       # group stride K
    out = torch.empty((M, G, N), device="cuda").transpose(0, 1)
    MA.linear(xs, w, b, act=MA.ACT_RELU, out=out)
    assert torch.equal(out, MA.linear(x, w, b, act=MA.ACT_RELU))
    dx = torch.empty((M, G, K), device="cuda").transpose(0, 1)
    MA.linear_backward(dy, xs, w, dx=dx, want=(True, False, False))
    assert torch.equal(dx, MA.linear_backward(dy, x, w)[0])


def test_residual_in_place_and_outputs_left_out():
    import paper_2106_07551_amd as MA
    x, w, b, r, dy = inputs(torch.bfloat16, None, 200, 512, 136, 5)
    r = r.contiguous()
    ref = MA.linear(x, w, b, act=MA.ACT_GELU, residual=r)
    MA.linear(x, w, b, act=MA.ACT_GELU, residual=r, out=r)
    assert torch.equal(r, ref)
    pre = torch.randn((200, 136), device="cuda").bfloat16()
    whole = MA.linear_backward(dy, x, w, act=MA.ACT_GELU, pre=pre)
    for k in range(3):
        want = tuple(i == k for i in range(3))
        part = MA.linear_backward(dy, x, w, act=MA.ACT_GELU, pre=pre, want=want)
        assert [p is not None for p in part] == list(want)
        assert torch.equal(part[k], whole[k])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_no_rows(dtype):
    import paper_2106_07551_amd as MA
    x, w = torch.empty((0, 40), dtype=dtype, device="cuda"), torch.ones((24, 40), dtype=dtype,
                                                                        device="cuda")
    pre = torch.empty((0, 24), dtype=dtype, device="cuda")
    assert MA.linear(x, w, act=MA.ACT_SILU, pre=pre).shape == (0, 24)
    dx, dw, db = MA.linear_backward(pre, x, w, act=MA.ACT_SILU, pre=pre)
    assert dx.shape == (0, 40)
    assert dw.shape == (24, 40) and not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_infinities_and_nan_stay_in_their_rows(dtype):
    import paper_2106_07551_amd as MA
    x, w, b, r, dy = inputs(dtype, None, 140, 72, 40, 9)
    x[3, 5], x[70, 71], dy[9, 2] = float("nan"), float("inf"), float("nan")
    y = MA.linear(x, w, b, act=MA.ACT_RELU)
    bad = ~torch.isfinite(y)
    assert torch.isnan(y[3]).all() and bad[70].any()
    bad[[3, 70]] = False
    assert not bad.any()
    x, _, _, _, _ = inputs(dtype, None, 140, 72, 40, 9)
    dx, dw, db = MA.linear_backward(dy, x, w)
    assert torch.isnan(dx[9]).all() and torch.isfinite(dx[:9]).all() and \
        torch.isfinite(dx[10:]).all()
    assert torch.isnan(dw[2]).all() and torch.isfinite(dw[:2]).all()
    assert torch.isnan(db[2]) and int(torch.isnan(db).sum()) == 1


def test_gradient_against_differences():
    """Central differences of sum(y * c) in 64 bits along random directions."""
    import paper_2106_07551_amd as MA
    g = torch.Generator(device="cuda").manual_seed(4)
    x, w, b, _, c = inputs(torch.float32, None, 20, 30, 25, 11)
    for act in ("gelu", "silu"):
        pre = torch.empty((20, 25), device="cuda")
        MA.linear(x, w, b, act=_code(act), pre=pre)
        grads = MA.linear_backward(c, x, w, act=_code(act), pre=pre)
        d = [torch.randn(t.shape, generator=g, device="cuda").double() for t in (x, w, b)]
        h = 1e-5

        def f(s):
            z = (x.double() + s * d[0]) @ (w.double() + s * d[1]).T + b.double() + s * d[2]
            return float((act64(act, z) * c.double()).sum())

        num = (f(h) - f(-h)) / (2 * h)
        ana = sum(float((gr.double() * di).sum()) for gr, di in zip(grads, d))
        assert abs(num - ana) <= 1e-4 * max(1.0, abs(num)), (act, num, ana)


def test_own_stream_workspace_and_graph():
    """A split sum with the caller's workspace on another stream, and captured
    into a graph, replayed with other inputs."""
    import paper_2106_07551_amd as MA
    x, w, b, _, dy = inputs(torch.bfloat16, None, 4000, 64, 48, 13)
    x, dy = x.contiguous(), dy.contiguous()
    ref = MA.linear_backward(dy, x, w)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = MA.linear_backward(dy, x, w, stream=st)
    st.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ref, got))
    work = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(t) for t in ref]

    def call():
        MA.linear_backward(dy, x, w, dx=out[0], dw=out[1], dbias=out[2], work=work)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(4):
        x.normal_(generator=torch.Generator(device="cuda").manual_seed(k))
        ref = MA.linear_backward(dy, x, w)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(ref, out)), k

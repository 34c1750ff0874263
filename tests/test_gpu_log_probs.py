"""Log probabilities of given actions with entropy and top alternatives on the GPU
(malib_log_probs, malib_log_probs_backward) against the formulas in 64 bits.

Tolerances, with u = 2^-24, as for the losses: the exponent (x_j - m) / T of an entry is off by at
most 3 u of itself, at most 60 where it matters, so a row's sums are off by about 100 u
relative; log probabilities, entropies and ln s take one logarithm of such sums and differences
of numbers up to L = the largest |logit difference| / T (of entries whose p is not 0 in fp32: 110
at most) + ln n: 200 u (1 + L), and where l itself is larger, its own three roundings.  A
gradient entry is a sum of terms dl p_j + dH p_j (|log p_j| + H): 400 u (1 + L) times the sum of their
absolute values, plus the output's own rounding (2^-8 of it in bf16, u in fp32).  The largest
logit and the lists are exact."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def view(t, pad, shift=0):
    """t with `pad` spare elements (NaN, or 1 in masks) behind each row."""
    n, a = t.shape
    fill = float("nan") if t.is_floating_point() else 1
    wide = torch.full((n * (a + pad) + shift,), fill, dtype=t.dtype, device=t.device)
    v = wide[shift:].view(n, a + pad)[:, :a]
    v.copy_(t)
    return v


def close(got, ref, bound, what, eps=U):
    got = got.double()
    assert got.shape == ref.shape, what
    # (a finite l below -2^128, of an entry at the type's lowest value over T < 1, is -inf in fp32)
    same = (got == ref) | (torch.isnan(got) & torch.isnan(ref)) | \
        (torch.isinf(got) & (got == ref.float()))
    tol = bound + 1.01 * eps * ref.abs() + 1e-36
    ok = same | ((got - ref).abs() <= tol)
    assert ok.all(), (what, float(torch.nan_to_num(((got - ref).abs() / tol)[~ok]).max()))


def legal64(x, mask):
    x = x.double()
    return x if mask is None else x.masked_fill(mask == 0, -math.inf)


def reference(x, act, T=1.0, mask=None, top=0):
    """(stats, lists' indices, their log probabilities, L of each row) in 64 bits."""
    x = legal64(x, mask)
    n, a = x.shape
    at = torch.arange(n, device="cuda")
    special = torch.isnan(x).any(1) | (x == math.inf).any(1)
    empty = (x == -math.inf).all(1)
    m = torch.where(torch.isnan(x), -math.inf, x).amax(1)
    d = (x - torch.where(m > -math.inf, m, 0.0)[:, None]) / T
    lns = torch.where(empty, 0.0, torch.logsumexp(d, 1))
    logp = torch.where(empty[:, None], -math.inf, d - lns[:, None])
    p = logp.exp()
    H = -torch.special.xlogy(p, p).sum(1)
    act = act.long()
    ok = (act >= 0) & (act < a)
    act = act.clamp(0, a - 1)
    if mask is not None:
        ok &= mask[at, act] != 0
    lp = torch.where(ok & ~empty, logp[at, act], 0.0)
    lp[special & ok] = math.nan
    H[special] = lns[special] = math.nan
    # NaN first, whatever its sign (torch's sort goes by it on the device)
    val, idx = torch.sort(torch.where(torch.isnan(x), math.nan, x + 0.0), dim=1, descending=True,
                          stable=True)
    none = val[:, :top] == -math.inf
    best = logp.gather(1, idx)[:, :top]
    best = torch.where(special[:, None], math.nan, best).masked_fill(none, 0.0)
    idx = idx[:, :top].masked_fill(none, -1)
    pad = (0, max(0, top - a))
    idx = torch.nn.functional.pad(idx, pad, value=-1)
    best = torch.nn.functional.pad(best, pad)
    low = torch.where(x > -math.inf, x, math.inf).amin(1)
    L = torch.where(empty | special, 0.0, ((m - low) / T).clamp(max=110)) + math.log(a)
    return torch.stack([lp, H, m, lns]), idx.int(), best, L, special


def check(x, act, *, T=1.0, mask=None, top=0, what=""):
    import paper_2106_07551_amd as M
    stats, idx, val = M.log_probs(x, act, temperature=T, top=top, mask=mask)
    ref, ridx, rval, L, special = reference(x, act, T, mask, top)
    what = (what, tuple(x.shape), str(x.dtype), top, T, mask is not None)
    tol = 200 * U * (1 + L)
    for i, name in enumerate(("logp", "entropy", "max", "ln s")):
        if name == "max":
            assert torch.equal(stats[2][~special].double(), ref[2][~special]), (what, name)
        else:
            close(stats[i], ref[i], tol + 3 * U * ref[i].abs(), (what, name))
    if not top:
        assert idx is None and val is None
        return stats
    bad = (idx != ridx).any(1).nonzero()
    assert bad.numel() == 0, (what, "rows", bad[:4, 0].tolist(), idx[bad[0, 0]].tolist()[:40],
                              ridx[bad[0, 0]].tolist()[:40])
    close(val, rval, tol[:, None] + 3 * U * rval.abs(), (what, "lists"))
    return stats


KINDS = ("normal", "constant", "ties", "falling", "rising", "column", "sparse", "lowest", "zeros",
         "special", "empty", "peaked")


def row_of(kind, a, lane, dtype, g):
    """One row of logits of a kind that lists can go wrong at."""
    x = torch.randn(a, generator=g, device="cuda") * 2
    i = torch.arange(a, device="cuda")
    if kind == "constant":
        x = torch.full((a,), 0.25, device="cuda")
    elif kind == "ties":
        x = torch.randint(-2, 3, (a,), generator=g, device="cuda").float()
    elif kind == "falling":
        x = -i.float() / 64
    elif kind == "rising":
        x = i.float() / 64
    elif kind == "column":     # the large ones in few lanes
        x = torch.where(i // 8 % lane == 1, x + 40, x)
    elif kind == "sparse":
        x = torch.where(torch.rand(a, generator=g, device="cuda") < 20 / a, x, -math.inf)
    elif kind == "lowest":
        x = torch.where(torch.rand(a, generator=g, device="cuda") < 0.5, x,
                        torch.finfo(dtype).min)
    elif kind == "zeros":
        x = torch.where(i % 3 == 0, -0.0, torch.where(i % 3 == 1, 0.0, -1e-42))
    elif kind == "special":
        x[torch.randint(0, a, (3,), generator=g, device="cuda")] = math.nan
        x[torch.randint(0, a, (2,), generator=g, device="cuda")] = math.inf
        if g.initial_seed() % 2:
            x = -x
    elif kind == "empty":
        x = torch.full((a,), -math.inf, device="cuda")
    elif kind == "peaked":
        x[torch.randint(0, a, (1,), generator=g, device="cuda")] = 500.0
    return x.to(dtype)


SIZES = [(1, 5), (2, 70), (3, 300), (8, 65), (9, 33), (18, 257), (24, 64), (25, 40), (31, 129),
         (32, 70), (33, 40), (64, 130), (65, 67), (128, 40), (129, 40), (255, 37), (256, 30),
         (512, 26), (777, 26), (1024, 14), (1025, 14), (2048, 26), (2049, 13), (4097, 13),
         (8191, 12), (8193, 12), (20000, 140), (50001, 12), (65536, 130), (65537, 12),
         (131071, 3), (200003, 130), (1 << 20, 1)]


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("a, n", SIZES)
def test_lists_of_every_kind(dtype, a, n):
    g = torch.Generator(device="cuda").manual_seed(a * 7 + n)
    lane = next((t for t in (4, 8, 16, 32, 64, 128, 256, 512) if t * 32 >= a), 1024)
    x = torch.stack([row_of(KINDS[r % 12 if n < 100 or a < 4000 else 0], a, lane, dtype, g)
                     for r in range(n)])
    if a >= 4000 and n >= 100:
        for r, kind in enumerate(KINDS):
            x[r] = row_of(kind, a, lane, dtype, g)
    act = torch.randint(-1, a + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
    for top in (1, 6, 40, 256) if a < 4000 else (5, 64, 256):
        check(x, act, top=top, what="kinds")
    check(x, act, what="no lists")


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("a, n", [(1, 140000), (5, 140000), (18, 140000), (24, 70001), (31, 70001),
                                  (33, 33000), (100, 20000), (250, 9000), (500, 5000),
                                  (777, 4500), (1024, 4500), (1025, 2049), (2048, 2050),
                                  (3001, 2049), (8192, 2048)])
def test_many_rows_of_every_kind(dtype, a, n):
    """As above where there are rows for the whole card: 60 rows, each many times."""
    g = torch.Generator(device="cuda").manual_seed(a + n)
    lane = next((t for t in (4, 8, 16, 32) if t * 32 >= a), 64)
    some = torch.stack([row_of(KINDS[r % 12], a, lane, dtype, g) for r in range(60)])
    x = some[torch.randint(0, 60, (n,), generator=g, device="cuda")]
    act = torch.randint(-1, a + 1, (n,), generator=g, device="cuda", dtype=torch.int64)
    mask = torch.rand((n, a), generator=g, device="cuda") < 0.9
    for top in (1, 5, 64) if a < 9 else (0, 1, 6, 33, 64, 100):
        check(x, act, top=top, what="many")
    check(x, act, top=6, mask=mask, T=0.7, what="many, mask")
    check(view(x, 3, 1), act, top=6, mask=view(mask, 1), what="many, apart")


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("a, n", [(18, 200), (31, 67), (50, 66), (333, 33), (1500, 20),
                                  (5003, 9), (40001, 5), (70001, 200)])
@pytest.mark.parametrize("T", [1.0, 0.3, 2.5])
def test_masks_strides_and_temperatures(dtype, a, n, T):
    g = torch.Generator(device="cuda").manual_seed(a + n)
    x = (torch.randn((n, a), generator=g, device="cuda") * 3).to(dtype)
    mask = torch.rand((n, a), generator=g, device="cuda") < 0.7
    mask[1] = False
    mask[2] = False
    mask[2, a - 1] = True
    u = torch.rand((n, a), generator=g, device="cuda")
    for lo, v in ((0.0, math.nan), (0.2, math.inf), (0.4, -math.inf),
                  (0.6, torch.finfo(dtype).min)):
        x = torch.where(~mask & (u >= lo) & (u < lo + 0.2), v, x)
    x[3] = torch.where(mask[3], -math.inf, x[3])   # legal, but no entry above -inf
    act = torch.randint(0, a, (n,), generator=g, device="cuda")
    act[0] = 255 if a < 255 else -1
    for pad, shift, ids in ((0, 0, torch.int64), (3, 1, torch.int32), (8, 0, torch.uint8)):
        if ids is torch.uint8 and a > 255:
            ids = torch.int32
        ai = act.clamp(min=0).to(ids) if ids is torch.uint8 else act.to(ids)
        check(view(x, pad, shift), ai, T=T, mask=view(mask, pad), top=9, what=(pad, shift))
    check(x, act, T=T, mask=mask.to(torch.uint8) * 5, top=3, what="uint8 mask")


def test_long_lists_of_many_parts():
    """Lists whose bound lets more entries through than the merge sorts at once: every part of
    the row but one has 200 entries that could be listed."""
    import paper_2106_07551_amd as M
    a = 1 << 18
    g = torch.Generator(device="cuda").manual_seed(5)
    for dtype in TYPES:
        x = -500 + torch.rand((2, a), generator=g, device="cuda")
        i = torch.arange(a, device="cuda")
        x = torch.where(i % 4096 < 200, 10 + torch.rand((2, a), generator=g, device="cuda"), x)
        x[:, :8192] = -1000
        x = x.to(dtype)
        act = torch.tensor([7, a - 1], dtype=torch.int32, device="cuda")
        check(x, act, top=256, what="parts")
        x[1] = -math.inf
        x[1, 12345:12400] = 1.0
        check(x, act, top=200, what="parts, few entries")
    assert M.log_probs(x, act, top=1)[1].tolist()[1] == [12345]


def test_indices_beyond_24_bits_of_a_row():
    """The widest row: 2^24 entries, in parts."""
    a = 1 << 24
    x = torch.zeros((1, a), dtype=torch.bfloat16, device="cuda")
    x[0, a - 1] = 2.0
    x[0, a - 70000] = 3.0
    check(x, torch.tensor([a - 1], device="cuda"), top=4)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("a, n", [(9000, 2048), (40000, 260), (300000, 3)])
def test_equal_entries_and_a_few_others(dtype, a, n):
    """Equal entries with a few others anywhere: the exact search, part by part."""
    g = torch.Generator(device="cuda").manual_seed(a)
    x = torch.zeros((n, a), device="cuda")
    others = torch.tensor([1.0, -1.0, 0.0, 3e38, -math.inf, math.inf, math.nan, 2.0],
                          device="cuda")
    for r in range(0, n, max(1, n // 64)):
        at = torch.randint(0, a, (r % 7,), generator=g, device="cuda")
        x[r, at] = others[torch.randint(0, 3 + r % 6, (r % 7,), generator=g, device="cuda")]
    act = torch.randint(0, a, (n,), generator=g, device="cuda")
    for top in (1, 7, 64, 200):
        check(x.to(dtype), act, top=top, what="equal")


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("a, n, apart", [(18, 9, 1 << 28), (300, 5, 1 << 29), (5000, 5, 1 << 29),
                                         (70000, 17, (1 << 27) + 1)])
def test_rows_beyond_32_bits(dtype, a, n, apart):
    """Rows whose offsets in elements (of logits, mask and dlogits) do not fit 31 bits."""
    import paper_2106_07551_amd as M
    g = torch.Generator(device="cuda").manual_seed(a)
    wide = torch.empty((n - 1) * apart + a, dtype=dtype, device="cuda")
    x = wide.as_strided((n, a), (apart, 1))
    x.copy_(torch.randn((n, a), generator=g, device="cuda") * 3)
    mask = torch.empty((n - 1) * apart + a, dtype=torch.uint8, device="cuda") \
        .as_strided((n, a), (apart, 1))
    mask.copy_(torch.rand((n, a), generator=g, device="cuda") < 0.8)
    act = torch.randint(0, a, (n,), generator=g, device="cuda")
    stats = check(x, act, top=9, mask=mask, what="far apart")
    near, legal = x.contiguous(), mask.contiguous()
    assert torch.equal(M.log_probs(near, act, top=9, mask=legal)[0], stats)
    dl, dh = torch.randn((2, n), generator=g, device="cuda")
    ref = M.log_probs_backward(near, act, stats, dl, dh, mask=legal)
    assert M.log_probs_backward(x, act, stats, dl, dh, mask=mask, dlogits=x) is x
    assert torch.equal(x, ref)


@pytest.mark.parametrize("n, a", [(0, 5), (0, 5000), (1, 1)])
def test_no_rows_and_one_entry(n, a):
    import paper_2106_07551_amd as M
    x = torch.full((n, a), 3.0, device="cuda")
    act = torch.zeros(n, dtype=torch.int32, device="cuda")
    stats, idx, val = M.log_probs(x, act, top=2)
    assert stats.shape == (4, n) and idx.shape == (n, 2) and val.shape == (n, 2)
    if n:
        assert stats[:, 0].tolist() == [0, 0, 3, 0]
        assert idx.tolist() == [[0, -1]] and val.tolist() == [[0, 0]]
    dx = M.log_probs_backward(x, act, stats, torch.ones(n, device="cuda"))
    assert dx.shape == (n, a) and bool((dx == 0).all())


def test_without_actions():
    import paper_2106_07551_amd as M
    for n, a in ((9, 7), (4, 500), (2, 90000)):
        x = torch.randn((n, a), device="cuda")
        act = torch.zeros(n, dtype=torch.int32, device="cuda")
        s1, i1, v1 = M.log_probs(x, top=5)
        s2, i2, v2 = M.log_probs(x, act, top=5)
        assert bool((s1[0] == 0).all()) and torch.equal(s1[1:], s2[1:])
        assert torch.equal(i1, i2) and torch.equal(v1, v2)
        d = torch.randn(n, device="cuda")
        g = M.log_probs_backward(x, None, s1, None, d)
        assert torch.equal(g, M.log_probs_backward(x, act, s2, torch.zeros(n, device="cuda"), d))


# ------------------------------------------------------------------- gradient

def grad64(x, act, dl, dh, T, mask):
    x = legal64(x, mask)
    n, a = x.shape
    at = torch.arange(n, device="cuda")
    empty = (x == -math.inf).all(1)
    logp = torch.where(empty[:, None], -math.inf, torch.log_softmax(x / T, 1))
    p = logp.exp()
    lz = torch.where(p > 0, logp, 0.0)
    H = -(p * lz).sum(1, keepdim=True)
    act = act.long()
    ok = (act >= 0) & (act < a)
    act = act.clamp(0, a - 1)
    if mask is not None:
        ok &= mask[at, act] != 0
    dl = torch.where(ok, dl.double(), 0.0)
    dh = torch.zeros_like(dl) if dh is None else dh.double()
    g = -p * dl[:, None] - dh[:, None] * p * (lz + H)
    size = p * dl.abs()[:, None] + dh.abs()[:, None] * p * (lz.abs() + H)
    hot = torch.zeros_like(g)
    hot[at, act] = 1.0
    g, size = (g + hot * dl[:, None]) / T, (size + hot * dl.abs()[:, None]) / T
    gone = (x == -math.inf) | empty[:, None]
    low = torch.where(x > -math.inf, x, math.inf).amin(1)
    L = torch.where(empty, 0.0, (x.amax(1) - low) / T) + math.log(a)
    return g.masked_fill(gone, 0.0), size.masked_fill(gone, 0.0), L


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("a, n", [(1, 3), (2, 300), (18, 130), (31, 65), (32, 66), (45, 300),
                                  (129, 40), (500, 33), (1025, 20), (3001, 9), (9999, 300),
                                  (50001, 3), (140000, 2)])
def test_gradient(dtype, a, n):
    import paper_2106_07551_amd as M
    eps = 2.0 ** -8 if dtype is torch.bfloat16 else U
    g = torch.Generator(device="cuda").manual_seed(a * 3 + n)
    x = (torch.randn((n, a), generator=g, device="cuda") * 3).to(dtype)
    mask = torch.rand((n, a), generator=g, device="cuda") < 0.7
    mask[n - 1] = False
    x = torch.where(~mask & (torch.rand((n, a), generator=g, device="cuda") < 0.3), math.nan, x)
    act = torch.randint(-1, a, (n,), generator=g, device="cuda", dtype=torch.int32)
    dl, dh = (torch.randn(n, generator=g, device="cuda") for _ in range(2))
    clean = torch.where(torch.isnan(x), 0.5, x)
    for T, m, e, pad, shift in ((1.0, None, None, 0, 0), (1.0, mask, dh, 0, 0),
                                (0.6, mask, dh, 5, 1), (2.0, None, dh, 3, 0),
                                (1.0, mask, None, 8, 0)):
        xv = view(x if m is not None else clean, pad, shift)
        mv = None if m is None else view(m, pad)
        stats = M.log_probs(xv, act, temperature=T, mask=mv)[0]
        out = view(torch.full_like(xv, 7.0), pad, shift)
        got = M.log_probs_backward(xv, act, stats, dl, e, temperature=T, mask=mv, dlogits=out)
        assert got is out
        ref, size, L = grad64(xv, act, dl, e, T, mv)
        close(got, ref, 400 * U * (1 + L)[:, None] * size, (a, n, T, pad, e is None), eps)
        dense = M.log_probs_backward(xv, act, stats, dl, e, temperature=T, mask=mv)
        assert torch.equal(dense, got)
        again = xv.clone() if pad == 0 else view(xv, pad, shift)
        assert M.log_probs_backward(again, act, stats, dl, e, temperature=T, mask=mv,
                                    dlogits=again) is again
        assert torch.equal(again, got)   # in place


@pytest.mark.parametrize("a", [7, 60, 5000])
def test_gradient_against_differences(a):
    """Along random directions, central differences of the 64-bit function: off by h^2 / 6 times
    the third derivative (below 20 here for |direction| = 1) and rounding 1e-16 / h."""
    import paper_2106_07551_amd as M
    g = torch.Generator(device="cuda").manual_seed(a)
    n, T, h = 12, 1.3, 1e-4
    x = torch.randn((n, a), generator=g, device="cuda") * 2
    mask = torch.rand((n, a), generator=g, device="cuda") < 0.8
    mask[:, 3] = True
    act = torch.full((n,), 3, device="cuda")
    dl, dh = (torch.randn(n, generator=g, device="cuda") for _ in range(2))
    stats = M.log_probs(x, act, temperature=T, mask=mask)[0]
    dx = M.log_probs_backward(x, act, stats, dl, dh, temperature=T, mask=mask).double()

    def f(y):
        s = reference(y, act, T, mask)[0]
        return dl.double() * s[0] + dh.double() * s[1]

    _, size, L = grad64(x, act, dl, dh, T, mask)
    for _ in range(3):
        v = torch.randn((n, a), generator=g, device="cuda", dtype=torch.float64)
        v /= v.norm(dim=1, keepdim=True)
        num = (f(x.double() + h * v) - f(x.double() - h * v)) / (2 * h)
        tol = (400 * U * (1 + L)[:, None] * size * v.abs()).sum(1) + 20 * h * h / 6 + 1e-10
        assert bool(((num - (dx * v).sum(1)).abs() <= tol).all())


def test_gradient_of_special_rows():
    """A legal NaN or +inf makes its row's legal entries NaN, no other row's; gradients of inf or
    NaN leave illegal entries and rows of no action alone."""
    import paper_2106_07551_amd as M
    for a in (9, 300):
        x = torch.randn((6, a), device="cuda")
        mask = torch.ones((6, a), dtype=torch.bool, device="cuda")
        mask[:, 2] = False
        x[0, 1], x[1, 1], x[2, 2] = math.nan, math.inf, math.nan
        act = torch.tensor([0, 0, 0, -1, 2, 0], dtype=torch.int32, device="cuda")
        stats = M.log_probs(x, act, mask=mask)[0]
        dl = torch.tensor([1, 1, 1, math.nan, math.inf, math.nan], device="cuda")
        dx = M.log_probs_backward(x, act, stats, dl, mask=mask)
        assert bool(torch.isnan(dx[0][mask[0]]).all()) and bool(torch.isnan(dx[1][mask[1]]).all())
        assert bool(torch.isfinite(dx[2]).all())
        assert bool((dx[3:5] == 0).all())     # no action, an action that is not legal
        assert bool(torch.isnan(dx[5][mask[5]]).all()) and bool((dx[:, 2] == 0).all())


# ------------------------------------------------------------------- as used

def test_outputs_given_streams_and_repeats():
    import paper_2106_07551_amd as M
    x = torch.randn((40, 3000), device="cuda").bfloat16()
    act = torch.randint(0, 3000, (40,), device="cuda")
    out = M.log_probs(x, act, top=7)
    into = tuple(torch.full_like(t, 3) for t in out)
    got = M.log_probs(x, act, top=7, stats=into[0], top_idx=into[1], top_logp=into[2])
    assert all(a is b for a, b in zip(got, into)) and all(map(torch.equal, got, out))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    slow = M.log_probs(x, act, top=7, stream=side)
    dl = torch.randn(40, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    dslow = M.log_probs_backward(x, act, slow[0], dl, stream=side)
    side.synchronize()
    assert all(map(torch.equal, slow, out))
    assert torch.equal(dslow, M.log_probs_backward(x, act, out[0], dl))
    wide = torch.randn((3, 131071), device="cuda")
    first = M.log_probs(wide, top=256)
    for _ in range(3):
        assert all(map(torch.equal, M.log_probs(wide, top=256), first))
    w = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    assert all(map(torch.equal, M.log_probs(wide, top=256, work=w), first))


def test_feeds_the_losses():
    """Old log probabilities and teachers' lists as policy_loss and distill_loss take them: the
    policy that acted has ratio 1, a student that is its teacher (all entries listed) no loss."""
    import paper_2106_07551_amd as M
    n, a = 500, 18
    x = torch.randn((n, a), device="cuda")
    mask = torch.rand((n, a), device="cuda") < 0.8
    mask[:, 0] = True
    act = torch.zeros(n, dtype=torch.int32, device="cuda")
    adv = torch.randn(n, device="cuda")
    stats, idx, val = M.log_probs(x, act, top=a, mask=mask)
    _, own, dx = M.policy_loss(x, act, stats[0], adv, entropy_coef=0.0, mask=mask)
    close(own[1], stats[0].double(), 1e-6, "log probability")
    close(own[3], stats[1].double(), 2e-6, "entropy")
    close(own[0], -adv.double(), 1e-5, "loss")
    want = M.log_probs_backward(x, act, stats, -adv / n, mask=mask)
    close(dx, want.double(), 1e-8, "gradient")
    total, loss, grad = M.distill_loss(x, idx, val, mask=mask)
    assert float(loss.abs().max()) < 2e-6 and float(grad.abs().max()) < 1e-6 / n

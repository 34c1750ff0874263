"""The learner's losses on the GPU (malib_policy_loss, malib_distill_loss)
against the formulas in 64 bits.

Tolerances, with u = 2^-24.  The exponent of e_j is (x_j - m) c in fp32: its
absolute error is at most 2 u |d_j| + u |d_j|, |d_j| <= 60 where e_j matters, so
e_j, a part's sums and the row's sums are off by at most about 100 u relative
(rescaling to a common maximum adds a few u per level).  Log probabilities,
entropies and divergences take one logarithm of such sums and differences of
numbers up to L = the largest |logit difference| + ln n: 200 u (1 + L).  The
ratio multiplies the log probability's error by r; the loss adds A, the
coefficients: 400 u (1 + L) (1 + r |A| + kl + ...).  A gradient entry is a sum of
terms w (G p_j + kl p_j |log p_j - log q_j - KL| + ...): 400 u (1 + L) times the sum
of their absolute values, plus the output's own rounding (2^-8 of it in bf16, u
in fp32)."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24
LO, HI = 0.2, 0.3


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
    same = (got == ref) | (torch.isnan(got) & torch.isnan(ref))
    tol = bound + 1.01 * eps * ref.abs() + 1e-36
    ok = same | ((got - ref).abs() <= tol)
    assert ok.all(), (what, float(torch.nan_to_num(((got - ref).abs() / tol)[~ok]).max()))


def log_probs(x, mask):
    x = x.double()
    if mask is not None:
        x = x.masked_fill(mask == 0, -math.inf)
    return x - torch.logsumexp(x, 1, keepdim=True)


def policy64(x, act, old, adv, *, kl=0.0, ent=0.0, ref_logp=None, ref_logits=None, mask=None,
             weight=None):
    """(total, stats, gradient, scale of a row's loss, scale of the gradient, L)."""
    n, a = x.shape
    act = act.long()
    ok = (act >= 0) & (act < a)
    act = act.clamp(0, a - 1)
    at = torch.arange(n, device="cuda")
    legal = torch.ones((n, a), dtype=torch.bool, device="cuda") if mask is None else mask != 0
    ok &= legal[at, act]
    w = (torch.full((n,), 1.0 / n, device="cuda") if weight is None else weight).double()
    ok &= w != 0
    ok &= ~(x.double().masked_fill(~legal, -math.inf) == -math.inf).all(1)
    logp = log_probs(x, mask)
    p = torch.exp(logp)
    lz = torch.where(p > 0, logp, 0.0)
    lp = logp[at, act]
    r, A = torch.exp(lp - old.double()), adv.double()
    s1, s2 = r * A, r.clamp(1 - LO, 1 + HI) * A
    H = -(p * lz).sum(1)
    G = torch.where(s1 <= s2, -s1, 0.0)
    KL = torch.zeros_like(H)
    grad = ent * p * (lz + H[:, None])
    size = abs(ent) * p * (lz.abs() + H[:, None].abs())
    if ref_logp is not None:
        d = ref_logp.double() - lp
        KL = torch.expm1(d) - d
        G = G - kl * torch.expm1(d)
    if ref_logits is not None:
        gap = torch.where(p > 0, lz - log_probs(ref_logits, mask), 0.0)
        KL = (p * gap).sum(1)
        grad = grad + kl * p * (gap - KL[:, None])
        size = size + abs(kl) * p * (gap.abs() + KL[:, None].abs() + 1)
    loss = -torch.minimum(s1, s2) + kl * KL - ent * H
    grad = grad - G[:, None] * p
    gs = s1.abs() + abs(kl) * (1 + KL.abs())
    size = size + gs[:, None] * p
    grad[at, act] += G
    size[at, act] += gs
    grad, size = grad * w[:, None], size * w[:, None].abs()
    grad[~ok], size[~ok] = 0, 0
    stats = torch.stack([loss, lp, KL, H])
    stats[:, ~ok] = 0
    fin = torch.where(torch.isfinite(logp), logp, 0.0)
    L = (fin.max(1).values - fin.min(1).values + math.log(a) + 1)
    scale = 1 + s1.abs() + s2.abs() + abs(kl) * (1 + KL.abs()) + abs(ent) * (1 + H)
    return (w * stats[0]).sum(), stats, grad, scale, size, L, w, ok


def policy_inputs(dtype, n, a, *, seed=0, mask=False, weight=False, ids=torch.int32, pad=0,
                  shift=0, spread=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rnd(*s):
        return torch.randn(s, generator=g, device="cuda")

    x = (rnd(n, a) * spread).to(dtype)
    d = dict(mask=None, weight=None)
    if mask:
        u = torch.rand((n, a), generator=g, device="cuda")
        m = u < 0.7
        m[torch.rand(n, generator=g, device="cuda") < 0.1] = False     # nothing left
        x = torch.where(u > 0.9, torch.full_like(x, float("nan")), x)
        x = torch.where((u > 0.8) & (u <= 0.9), torch.full_like(x, float("inf")), x)
        d["mask"] = view(m, pad)
    if weight:
        d["weight"] = torch.rand(n, generator=g, device="cuda")
        d["weight"][::5] = 0.0
    act = torch.randint(0, a, (n,), generator=g, device="cuda")
    act[3::11] = 255 if ids == torch.uint8 else -1
    act[5::13] = a if a < 255 else -1
    d.update(logits=view(x, pad, shift), actions=act.to(ids))
    base = -math.log(a) - 0.5 * spread * spread
    d["old_logp"] = base + 0.5 * rnd(n)
    d["advantage"] = rnd(n)
    d["ref_logp"] = base + 0.5 * rnd(n)
    y = torch.where(torch.isfinite(x), x, torch.zeros_like(x)).float() + 0.3 * rnd(n, a)
    d["ref_logits"] = view(y.to(dtype), pad, shift)
    return d


def check_policy(d, *, how, kl=0.07, ent=0.02, tag=""):
    import paper_2106_07551_amd as MA
    print("[policy]", tag, how, flush=True)
    kw = dict(mask=d["mask"], weight=d["weight"])
    kl = 0.0 if how == "none" else kl
    ref = dict(ref_logp=d["ref_logp"] if how == "sampled" else None,
               ref_logits=d["ref_logits"] if how == "full" else None)
    total, stats, grad = MA.policy_loss(
        d["logits"], d["actions"], d["old_logp"], d["advantage"], clip_low=LO, clip_high=HI,
        kl_coef=kl, entropy_coef=ent, **ref, **kw)
    T, S, G, scale, size, L, w, ok = policy64(d["logits"], d["actions"], d["old_logp"],
                                              d["advantage"], kl=kl, ent=ent, **ref, **kw)
    bound = 400 * U * L * scale
    close(stats[1:], S[1:], 200 * U * (L * (1 + S[2].abs()))[None, :], tag + " stats")
    close(stats[0], S[0], bound, tag + " loss")
    close(total[0], T, (w.abs() * bound)[ok].sum(), tag + " total")
    eps = 2.0 ** -8 if d["logits"].dtype == torch.bfloat16 else U
    close(grad, G, 400 * U * L[:, None] * size, tag + " gradient", eps)
    # the forward alone gives the same
    t2, s2, none = MA.policy_loss(
        d["logits"], d["actions"], d["old_logp"], d["advantage"], clip_low=LO, clip_high=HI,
        kl_coef=kl, entropy_coef=ent, grad=False, **ref, **kw)
    assert none is None and torch.equal(t2, total) and torch.equal(s2, stats)


DTYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
# both sides of every variant's bounds, odd sizes, one row, one action
SHAPES = [(1, 1), (1, 2), (7, 3), (300, 18), (5000, 5), (64, 31), (65, 32), (257, 33), (100, 128),
          (33, 129), (70, 255), (40, 257), (19, 1023), (21, 1025), (9, 2049), (600, 2049),
          (5, 4097), (3, 8192), (200, 8193), (1, 8193), (130, 16385), (2, 32769), (150, 33000),
          (1, 131071), (520, 40001)]


@DTYPES
@pytest.mark.parametrize("n, a", SHAPES)
def test_policy_sizes(dtype, n, a):
    how = ("none", "sampled", "full")[(n + a) % 3]
    d = policy_inputs(dtype, n, a, seed=n + a, weight=n % 2 == 0,
                      ids=(torch.int32, torch.int64)[a % 2])
    check_policy(d, how=how, tag=f"{dtype} {n}x{a}")


@DTYPES
@pytest.mark.parametrize("how", ["none", "sampled", "full"])
@pytest.mark.parametrize("n, a", [(400, 6), (90, 100), (60, 700), (30, 5000), (140, 12000),
                                  (3, 70001)])
def test_policy_masks_and_strides(dtype, n, a, how):
    for pad, shift in ((0, 0), (3, 1), (8, 0)):
        d = policy_inputs(dtype, n, a, seed=n + a + pad, mask=True, weight=pad == 3,
                          ids=torch.uint8 if a < 200 else torch.int32, pad=pad, shift=shift)
        check_policy(d, how=how, tag=f"{dtype} {n}x{a} mask pad={pad}")


# rows of up to 8 chunks of 16 bytes per thread of a workgroup, whole rounds of chunks or
# not, and one entry more than registers take
LONG_ROWS = [(130, 16384), (129, 24577), (140, 32767), (131, 32768), (128, 49152), (133, 65535),
             (129, 65536), (128, 65537)]


@DTYPES
@pytest.mark.parametrize("n, a", LONG_ROWS)
def test_policy_long_rows(dtype, n, a):
    how = ("none", "sampled", "full")
    d = policy_inputs(dtype, n, a, seed=n + a, weight=True)
    check_policy(d, how=how[a % 3], tag=f"{dtype} {n}x{a}")
    d = policy_inputs(dtype, n, a, seed=n + a + 1, mask=True, pad=3, shift=1)
    check_policy(d, how=how[(a + 1) % 3], tag=f"{dtype} {n}x{a} mask")


@DTYPES
@pytest.mark.parametrize("a", [4, 40, 900, 6000, 20000, 70000])
def test_policy_infinite_logits(dtype, a):
    """-inf and the type's lowest number as masks in the logits themselves, in some
    rows everywhere; a NaN stays in its row; a reference that excludes what the
    policy allows gives an infinite divergence."""
    import paper_2106_07551_amd as MA
    n = 12
    d = policy_inputs(dtype, n, a, seed=a)
    x, y = d["logits"], d["ref_logits"]
    act = torch.zeros(n, dtype=torch.int32, device="cuda")
    low = torch.finfo(dtype).min
    x[0, 1:] = -math.inf                 # certain
    x[1, :] = -math.inf                  # nothing
    x[2, a // 2:] = -math.inf
    x[3, 1:] = low
    x[4, 0] = -math.inf                  # the action itself
    x[5, :] = low                        # uniform
    y[2, a // 2:] = -math.inf
    d["actions"], d["advantage"][4] = act, 1.0
    for how in ("none", "full"):
        kw = dict(ref_logits=y if how == "full" else None, kl_coef=0.07 if how == "full" else 0.0)
        total, stats, grad = MA.policy_loss(x, act, d["old_logp"], d["advantage"], clip_low=LO,
                                            clip_high=HI, entropy_coef=0.02, **kw)
        _, S, G, scale, size, L, _, _ = policy64(
            x, act, d["old_logp"], d["advantage"], kl=kw["kl_coef"], ent=0.02,
            ref_logits=kw["ref_logits"])
        # the lowest number is about 2^128: differences from it are exact enough only
        # as "never drawn", so row 3's log probabilities of the rest are not compared
        L = L.clamp(max=100 + math.log(a))
        assert not grad[1].any() and not stats[:, 1].any()
        eps = 2.0 ** -8 if dtype == torch.bfloat16 else U
        close(stats[:, [0, 2, 6, 7, 8, 9, 10, 11]], S[:, [0, 2, 6, 7, 8, 9, 10, 11]],
              (400 * U * L * scale)[[0, 2, 6, 7, 8, 9, 10, 11]], "stats")
        assert float(stats[1, 4]) == -math.inf and torch.isfinite(grad[4]).all()
        assert abs(float(stats[3, 5]) - math.log(a)) < 1e-4
        for r in (0, 2, 4, 6, 7):
            close(grad[r], G[r], 400 * U * 100 * size[r], f"gradient of row {r}", eps)
        assert torch.isfinite(grad[3]).all() and not grad[3, 1:].any()
    x[7, a - 1] = float("nan")
    total, stats, grad = MA.policy_loss(x, act, d["old_logp"], d["advantage"], entropy_coef=0.02)
    assert torch.isnan(total).all() and torch.isnan(grad[7]).all() and torch.isnan(stats[0, 7])
    keep = [r for r in range(n) if r != 7]
    assert torch.isfinite(grad[keep]).all()
    x[7, a - 1] = 0.0
    y[8, a - 1] = -math.inf
    _, stats, _ = MA.policy_loss(x, act, d["old_logp"], d["advantage"], ref_logits=y, kl_coef=0.1)
    assert float(stats[2, 8]) == math.inf


# rows by one lane, by lanes of a wavefront, by workgroups, read twice, in parts
@DTYPES
@pytest.mark.parametrize("n, a", [(70, 18), (40, 300), (20, 6000), (130, 12000), (520, 66000),
                                  (3, 131071)])
def test_policy_divergence_as_statistic(dtype, n, a):
    """With a coefficient of 0 a divergence is only reported: loss and gradient are
    those without a reference, where it is infinite or NaN too."""
    import paper_2106_07551_amd as MA
    d = policy_inputs(dtype, n, a, seed=n + a, weight=True)
    x, old, adv = d["logits"], d["old_logp"], d["advantage"]
    d["weight"][:2] = 0.5
    act = torch.zeros(n, dtype=torch.int32, device="cuda")
    y, ref_logp = d["ref_logits"], d["ref_logp"]
    y[0, a - 1] = -math.inf           # excluded by the reference, not by the policy
    y[1, :] = -math.inf
    y[2, a // 2] = float("nan")
    ref_logp[0], ref_logp[1], ref_logp[2] = 200.0, math.inf, float("nan")
    x[0, 0] = -math.inf               # the action itself
    T, S, G, scale, size, L, w, ok = policy64(x, act, old, adv, ent=0.02, weight=d["weight"])
    eps = 2.0 ** -8 if dtype == torch.bfloat16 else U
    for ref in (dict(ref_logits=y), dict(ref_logp=ref_logp)):
        print("[statistic]", dtype, n, a, list(ref), flush=True)
        total, stats, grad = MA.policy_loss(x, act, old, adv, clip_low=LO, clip_high=HI,
                                            entropy_coef=0.02, weight=d["weight"], **ref)
        assert not torch.isfinite(stats[2, :3][ok[:3]]).any()
        bound = 400 * U * L * scale
        close(stats[0], S[0], bound, "loss")
        close(total[0], T, (w.abs() * bound)[ok].sum(), "total")
        close(grad, G, 400 * U * L[:, None] * size, "gradient", eps)


def test_policy_no_rows_and_one_action():
    import paper_2106_07551_amd as MA
    e = torch.empty(0, device="cuda")
    total, stats, grad = MA.policy_loss(torch.empty((0, 7), device="cuda"), e.int(), e, e)
    assert float(total) == 0.0 and stats.shape == (4, 0) and grad.shape == (0, 7)
    x = torch.randn((5, 1), device="cuda")
    z = torch.zeros(5, device="cuda")
    _, stats, grad = MA.policy_loss(x, z.int(), z, z + 1.0)
    assert not grad.any() and not stats[1].any() and torch.equal(stats[0], z - 1.0)


def test_policy_clipping_sides():
    """r far above and below the range, either sign of the advantage: the
    gradient vanishes exactly on the clipped sides."""
    import paper_2106_07551_amd as MA
    x = torch.zeros((4, 2), device="cuda")
    old = torch.tensor([-3.0, -3.0, 0.0, 0.0], device="cuda")     # r = e^2.3.., e^-0.69..
    adv = torch.tensor([1.0, -1.0, 1.0, -1.0], device="cuda")
    act = torch.zeros(4, dtype=torch.int32, device="cuda")
    _, stats, grad = MA.policy_loss(x, act, old, adv)
    r = 0.5 / torch.exp(old.double())
    ref = torch.tensor([-1.2, float(r[1]), -float(r[2]), 0.8], device="cuda").double()
    close(stats[0], ref, 20 * U * ref.abs(), "loss")
    assert not grad[0].any() and not grad[3].any() and grad[1].any() and grad[2].any()
    _, stats, grad = MA.policy_loss(x, act, old, adv, clip_low=math.inf, clip_high=math.inf)
    close(stats[0], -r * adv.double(), 20 * U * r, "unclipped")
    assert grad[0].any() and grad[3].any()


def distill64(x, idx, val, T, mask=None, weight=None):
    n, a = x.shape
    i = idx.long()
    live = (i >= 0) & (i < a)
    i = i.clamp(0, a - 1)
    legal = torch.ones((n, a), dtype=torch.bool, device="cuda") if mask is None else mask != 0
    live &= legal.gather(1, i)
    w = (torch.full((n,), 1.0 / n, device="cuda") if weight is None else weight).double()
    v = torch.where(live, val.double() / T, -math.inf)
    ok = (v != -math.inf).any(1) & (w != 0)
    ok &= ~(x.double().masked_fill(~legal, -math.inf) == -math.inf).all(1)
    logt = v - torch.logsumexp(v, 1, keepdim=True)
    t = torch.where(live, torch.exp(logt), 0.0)
    t[~ok] = 0
    logq = log_probs(x.double() / T, mask)
    gap = torch.where(t > 0, logt - logq.gather(1, i), 0.0)
    loss = T * T * (t * gap).sum(1)
    mag = T * T * (t * (1 + gap.abs())).sum(1)
    q = torch.exp(logq)
    grad, size = T * q, T * q
    grad = grad.scatter_add(1, i, -T * t) * w[:, None]
    size = size.scatter_add(1, i, T * t) * w[:, None].abs()
    grad[~ok], size[~ok], loss[~ok] = 0, 0, 0
    fin = torch.where(torch.isfinite(logq), logq, 0.0)
    L = fin.max(1).values - fin.min(1).values + math.log(a) + 1 + \
        torch.where(live, val.double().abs(), 0.0).max(1).values * 2 / T
    return (w * loss).sum(), loss, grad, mag, size, L, w, ok


def check_distill(dtype, n, a, top, T, *, mask=False, weight=False, pad=0, shift=0, repeat=False,
                  seed=0):
    import paper_2106_07551_amd as MA
    tag = f"{dtype} {n}x{a} top={top} T={T} mask={mask} pad={pad}"
    print("[distill]", tag, flush=True)
    d = policy_inputs(dtype, n, a, seed=seed + n + a, mask=mask, weight=weight, pad=pad,
                      shift=shift)
    g = torch.Generator(device="cuda").manual_seed(seed + 5)
    if repeat:
        idx = torch.randint(0, max(1, a // 2), (n, top), generator=g, device="cuda")
    else:
        idx = torch.argsort(torch.rand((n, a), generator=g, device="cuda"), 1)[:, :top]
    idx = idx.int().contiguous()
    idx[torch.rand((n, top), generator=g, device="cuda") < 0.1] = -1
    idx[1::7] = -1                                   # rows with no list
    idx[2::9, 0] = a
    val = torch.randn((n, top), generator=g, device="cuda") * 2
    val[torch.rand((n, top), generator=g, device="cuda") < 0.05] = -math.inf
    total, loss, grad = MA.distill_loss(d["logits"], idx, val, temperature=T, mask=d["mask"],
                                        weight=d["weight"])
    R = distill64(d["logits"], idx, val, T, d["mask"], d["weight"])
    bound = 400 * U * R[5] * R[3]
    close(loss, R[1], bound, tag + " loss")
    close(total[0], R[0], (R[6].abs() * bound)[R[7]].sum(), tag + " total")
    eps = 2.0 ** -8 if dtype == torch.bfloat16 else U
    close(grad, R[2], 400 * U * R[5][:, None] * R[4], tag + " gradient", eps)
    t2, l2, none = MA.distill_loss(d["logits"], idx, val, temperature=T, mask=d["mask"],
                                   weight=d["weight"], grad=False)
    assert none is None and torch.equal(t2, total) and torch.equal(l2, loss)


@DTYPES
@pytest.mark.parametrize("n, a", SHAPES)
def test_distill_sizes(dtype, n, a):
    check_distill(dtype, n, a, min(a, (1, 6, 64, 256)[n % 4]), (1.0, 2.0, 0.7)[a % 3],
                  weight=n % 2 == 1)


@DTYPES
@pytest.mark.parametrize("n, a", LONG_ROWS)
def test_distill_long_rows(dtype, n, a):
    check_distill(dtype, n, a, 40, 2.0, weight=True)
    check_distill(dtype, n, a, 70, 1.0, mask=True, repeat=True, pad=3, shift=1)


@DTYPES
@pytest.mark.parametrize("n, a, top", [(300, 16, 15), (300, 16, 16), (257, 31, 1), (70, 20, 11)])
def test_distill_few_actions_long_lists(dtype, n, a, top):
    check_distill(dtype, n, a, top, 1.0, weight=True)


@DTYPES
@pytest.mark.parametrize("n, a", [(400, 6), (90, 100), (60, 700), (30, 5000), (140, 12000),
                                  (3, 70001)])
def test_distill_masks_repeats_and_strides(dtype, n, a):
    check_distill(dtype, n, a, 13, 1.5, mask=True, repeat=True, pad=5, shift=3)
    check_distill(dtype, n, a, min(a, 30), 1.0, mask=True, weight=True)


def test_policy_no_rows_with_a_reference():
    import paper_2106_07551_amd as MA
    none = torch.empty(0, device="cuda")
    for kw in (dict(ref_logp=none), dict(ref_logits=torch.empty((0, 7), device="cuda"))):
        total, stats, grad = MA.policy_loss(
            torch.empty((0, 7), device="cuda"), none.int(), none, none, kl_coef=0.5, **kw)
        assert float(total) == 0.0 and stats.shape == (4, 0) and grad.shape == (0, 7)


def test_distill_no_rows():
    import paper_2106_07551_amd as MA
    total, loss, grad = MA.distill_loss(
        torch.empty((0, 7), device="cuda"), torch.empty((0, 3), device="cuda", dtype=torch.int32),
        torch.empty((0, 3), device="cuda"))
    assert float(total) == 0.0 and loss.shape == (0,) and grad.shape == (0, 7)


def test_gradients_against_differences():
    """Central differences in 64 bits along random directions of the logits."""
    import paper_2106_07551_amd as MA
    g = torch.Generator(device="cuda").manual_seed(2)
    d = policy_inputs(torch.float32, 50, 20, seed=9)
    dirn = torch.randn((50, 20), generator=g, device="cuda").double()
    h = 1e-6
    for how in ("none", "sampled", "full"):
        kw = dict(ref_logp=d["ref_logp"] if how == "sampled" else None,
                  ref_logits=d["ref_logits"] if how == "full" else None)
        kl = 0.0 if how == "none" else 0.3

        def f(s):
            return float(policy64(d["logits"].double() + s * dirn, d["actions"], d["old_logp"],
                                  d["advantage"], kl=kl, ent=0.1, **kw)[0])

        grad = MA.policy_loss(d["logits"], d["actions"], d["old_logp"], d["advantage"],
                              clip_low=LO, clip_high=HI, kl_coef=kl, entropy_coef=0.1, **kw)[2]
        num, ana = (f(h) - f(-h)) / (2 * h), float((grad.double() * dirn).sum())
        assert abs(num - ana) <= 1e-4 * max(0.1, abs(num)), (how, num, ana)
    idx = torch.randint(0, 20, (50, 8), generator=g, device="cuda", dtype=torch.int32)
    val = torch.randn((50, 8), generator=g, device="cuda")
    grad = MA.distill_loss(d["logits"], idx, val, temperature=2.0)[2]
    num = (float(distill64(d["logits"].double() + h * dirn, idx, val, 2.0)[0]) -
           float(distill64(d["logits"].double() - h * dirn, idx, val, 2.0)[0])) / (2 * h)
    assert abs(num - float((grad.double() * dirn).sum())) <= 1e-4 * max(0.1, abs(num))


@pytest.mark.parametrize("n, a", [(3000, 18), (700, 300), (300, 9000), (3, 60000)])
def test_streams_and_graph_replays(n, a):
    """The same bits on another stream and from a captured graph that is replayed
    with other inputs between eager calls."""
    import paper_2106_07551_amd as MA
    d = policy_inputs(torch.bfloat16, n, a, seed=1)
    args = (d["logits"], d["actions"], d["old_logp"], d["advantage"])
    ref = MA.policy_loss(*args, ref_logits=d["ref_logits"], kl_coef=0.1)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = MA.policy_loss(*args, ref_logits=d["ref_logits"], kl_coef=0.1, stream=st)
    st.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ref, got))
    out = [torch.empty_like(t) for t in ref]
    work = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def call():
        MA.policy_loss(*args, ref_logits=d["ref_logits"], kl_coef=0.1, total=out[0],
                       stats=out[1], dlogits=out[2], work=work)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(4):
        d["logits"].normal_(generator=torch.Generator(device="cuda").manual_seed(k))
        ref = MA.policy_loss(*args, ref_logits=d["ref_logits"], kl_coef=0.1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(ref, out)), k

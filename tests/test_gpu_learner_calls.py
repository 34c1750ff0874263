"""The native calls of the learner operators (csrc/learner_calls.cpp): what they take
gives the same bits as the binding's own way to the library, and what they do not
take is refused, or answered, by the binding as before."""
import ctypes
import os
import subprocess

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def both_ways(fn, *a, **kw):
    """fn's outputs through the native call and through the binding alone."""
    import paper_2106_07551_amd as M
    native = fn(*a, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    slow = fn(*a, **kw, stream=side)
    side.synchronize()
    one = isinstance(native, torch.Tensor)
    for p, q in zip((native,) if one else native, (slow,) if one else slow):
        assert (p is None) == (q is None)
        if p is not None:
            assert p.shape == q.shape and p.dtype == q.dtype and p.stride() == q.stride()
            assert torch.equal(p, q)
    assert M.binding._calls is not None
    return native


def rnd(*s, dtype=torch.float32):
    return torch.randn(s, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lead", [(), (3,), (1,)])
@pytest.mark.parametrize("rows", [0, 1, 3, 70])
def test_linear(dtype, lead, rows):
    import paper_2106_07551_amd as M
    x, w = rnd(*lead, rows, 21, dtype=dtype), rnd(*lead, 13, 25, dtype=dtype)[..., :21]
    b, r = rnd(*lead, 13), rnd(*lead, rows, 13, dtype=dtype)
    pre = torch.empty_like(r)
    both_ways(M.linear, x, w)
    y = both_ways(M.linear, x, w, b, act=M.ACT_GELU, residual=r, pre=pre)
    out = torch.empty_like(y)
    assert M.linear(x, w, b, act=M.ACT_GELU, residual=r, out=out) is out and torch.equal(out, y)
    both_ways(M.linear_backward, r, x, w)
    dx, dw, db = both_ways(M.linear_backward, r, x, w, act=M.ACT_SILU, pre=pre)
    for want in ((True, False, False), (False, True, False), (False, False, True)):
        g = both_ways(M.linear_backward, r, x, w, act=M.ACT_SILU, pre=pre, want=want)
        assert [t is not None for t in g] == list(want)
    into = torch.empty_like(dw)
    g = M.linear_backward(r, x, w, act=M.ACT_SILU, pre=pre, dw=into)
    assert g[1] is into and torch.equal(into, dw)


def test_shared_input():
    """x without the group dimension is not the native call's: the binding takes it."""
    import paper_2106_07551_amd as M
    x, w = rnd(9, 8), rnd(3, 5, 8)
    assert M.binding._native().linear(x, w, None, 0, None, None, None, None,
                                      M.binding._current_stream()) is None
    both_ways(M.linear, x, w)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("ids", [torch.uint8, torch.int32, torch.int64])
@pytest.mark.parametrize("n, a", [(0, 4), (1, 1), (50, 9), (40, 300), (3, 40000)])
def test_losses(dtype, ids, n, a):
    import paper_2106_07551_amd as M
    x, ref = rnd(n, a + 3, dtype=dtype)[:, :a], rnd(n, a, dtype=dtype)
    act = (torch.arange(n, device="cuda") % min(a, 100)).to(ids)
    old, adv, w = rnd(n), rnd(n), torch.rand(n, device="cuda")
    mask = torch.rand((n, a), device="cuda") < 0.8
    both_ways(M.policy_loss, x, act, old, adv)
    both_ways(M.policy_loss, x, act, old, adv, kl_coef=0.1, ref_logp=old, weight=w, clip_low=1)
    out = both_ways(M.policy_loss, x, act, old, adv, kl_coef=0.1, ref_logits=ref,
                    mask=mask.to(torch.uint8), entropy_coef=0.01)
    assert both_ways(M.policy_loss, x, act, old, adv, grad=False)[2] is None
    total, stats, dx = (torch.full_like(t, 7) for t in out)
    got = M.policy_loss(x, act, old, adv, kl_coef=0.1, ref_logits=ref, mask=mask,
                        entropy_coef=0.01, total=total, stats=stats, dlogits=dx,
                        work=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    assert got[0] is total and got[1] is stats and got[2] is dx
    assert all(torch.equal(p, q) for p, q in zip(out, got))
    idx = torch.randint(0, a, (n, 4), device="cuda", dtype=torch.int32)
    both_ways(M.distill_loss, x, idx, rnd(n, 4), temperature=2)
    both_ways(M.distill_loss, x, idx, rnd(n, 4), mask=mask, weight=w)
    assert both_ways(M.distill_loss, x, idx, rnd(n, 4), grad=False)[2] is None


def test_refusals_name_the_argument():
    import paper_2106_07551_amd as M
    x, w = rnd(9, 8), rnd(5, 8)
    old = rnd(9)
    act = torch.zeros(9, dtype=torch.int32, device="cuda")
    idx = torch.zeros((9, 2), dtype=torch.int32, device="cuda")
    for fn, word in (
            (lambda: M.linear(x, w.double()), "w"),
            (lambda: M.linear(x, w[:, :7]), "x"),
            (lambda: M.linear(x, w.cpu()), "w"),
            (lambda: M.linear(x, w, act=9), "act"),
            (lambda: M.linear(x, w, rnd(4)), "bias"),
            (lambda: M.linear(x.t(), rnd(5, 9)), "x"),
            (lambda: M.linear(x, w, out=rnd(9, 6)), "out"),
            (lambda: M.linear_backward(rnd(9, 5), x, w, act=M.ACT_RELU), "pre"),
            (lambda: M.linear_backward(rnd(9, 5), x, w, dbias=rnd(6)), "dbias"),
            (lambda: M.policy_loss(x, act.float(), old, old), "actions"),
            (lambda: M.policy_loss(x, act[:8], old, old), "actions"),
            (lambda: M.policy_loss(x, act, old, old, kl_coef=1.0), "kl_coef"),
            (lambda: M.policy_loss(x, act, old, old, clip_low=-1.0), "clip_low"),
            (lambda: M.policy_loss(x, act, old, old, mask=x), "mask"),
            (lambda: M.policy_loss(x, act, old, old, stats=rnd(9)), "stats"),
            (lambda: M.distill_loss(x, idx.long(), rnd(9, 2)), "teacher_idx"),
            (lambda: M.distill_loss(x, idx, rnd(9, 3)), "teacher_logits"),
            (lambda: M.distill_loss(x, idx, rnd(9, 2), temperature=0.0), "temperature"),
            (lambda: M.distill_loss(x, idx, rnd(9, 2), weight=old.cpu()), "weight"),
            (lambda: M.linear(rnd(64, 65536), rnd(24, 65536),
                              work=torch.empty(16, device="cuda")), "work")):
        with pytest.raises(M.MalibError, match=word):
            fn()


STAND_IN = r"""
#include "malib.h"
int calls, status;
malib_status malib_linear_work(const malib_linear_desc* d, int32_t b, int64_t* n)
{ *n = 0; return MALIB_OK; }
malib_status malib_loss_work(int32_t t, int64_t r, int64_t a, int64_t* n) { *n = 0; return MALIB_OK; }
malib_status malib_linear(const malib_linear_desc* d, const malib_mat* x, const malib_mat* w,
    const float* bias, const malib_mat* residual, const malib_mat* pre, const malib_mat* y,
    void* work, int64_t work_bytes, void* stream) { ++calls; return (malib_status)status; }
malib_status malib_linear_backward(const malib_linear_desc* d, const malib_mat* dy,
    const malib_mat* x, const malib_mat* w, const malib_mat* pre, const malib_mat* dx,
    const malib_mat* dw, float* dbias, void* work, int64_t work_bytes, void* stream)
{ ++calls; return (malib_status)status; }
malib_status malib_policy_loss(const malib_policy_loss_desc* d, const void* logits,
    const void* actions, const float* old_logp, const float* advantage, const float* ref_logp,
    const void* ref_logits, const uint8_t* mask, const float* weight, float* total, float* stats,
    void* dlogits, void* work, int64_t work_bytes, void* stream)
{ ++calls; return (malib_status)status; }
malib_status malib_distill_loss(const malib_distill_desc* d, const void* logits,
    const int32_t* idx, const float* val, const uint8_t* mask, const float* weight, float* total,
    float* loss, void* dlogits, void* work, int64_t work_bytes, void* stream)
{ ++calls; return (malib_status)status; }
"""


def test_a_failed_launch_is_raised_once(tmp_path):
    """A status from behind the checks (a stand-in library returns it and launches
    nothing) is raised: the call is not made again, over a residual that is the output, say.
    What the checks refuse is still the binding's to name."""
    import paper_2106_07551_amd as M
    B = M.binding
    src, so = tmp_path / "stand_in.c", tmp_path / "stand_in.so"
    src.write_text(STAND_IN)
    include = os.path.join(os.path.dirname(os.path.dirname(B.LIB_PATH)), "include")
    subprocess.run(["gcc", "-shared", "-fPIC", "-I", include, str(src), "-o", str(so)], check=True)
    L = ctypes.CDLL(str(so))
    calls, status = ctypes.c_int.in_dll(L, "calls"), ctypes.c_int.in_dll(L, "status")
    x, w, y = rnd(9, 8), rnd(5, 8), rnd(9, 5)
    act = torch.zeros(9, dtype=torch.int32, device="cuda")
    old, before = rnd(9), y.clone()
    whole = M.linear(x, w, residual=before)
    fns = [lambda: M.linear(x, w, residual=y, out=y), lambda: M.linear_backward(y, x, w),
           lambda: M.policy_loss(x, act, old, old),
           lambda: M.distill_loss(x, act[:, None].contiguous(), old[:, None].contiguous())]
    B._native().load(str(so))
    try:
        for code in (B.E_HIP, B.E_NOMEM):
            status.value = code
            for n, fn in enumerate(fns):
                calls.value = 0
                with pytest.raises(M.MalibError) as e:
                    fn()
                assert e.value.status == code and calls.value == 1, n
                assert torch.equal(y, before)
        status.value, calls.value = B.E_INVAL, 0
        assert torch.equal(fns[0](), whole) and calls.value == 1
    finally:
        B._native().load(B.LIB_PATH)
    assert M.linear(x, w).shape == (9, 5)

"""What the learner operators refuse, on the host and before any device work:
the library's own checks (pointers are never dereferenced) and the binding's
checks of shapes, types, strides and devices."""
import ctypes as C

import pytest
import torch

import paper_2106_07551_amd as M
from paper_2106_07551_amd import binding as B

P = 4096          # an address that is never read


def _linear(L, *, dtype=B.DT_BF16, act=B.ACT_NONE, groups=1, rows=8, n_in=16, n_out=24, x=None,
            w=None, y=None, bias=None, residual=None, pre=None, work=None, nbytes=0):
    d = B.LinearDesc(dtype, act, groups, rows, n_in, n_out)
    x = B.Mat(P, n_in, rows * n_in) if x is None else x
    w = B.Mat(P, n_in, n_out * n_in) if w is None else w
    y = B.Mat(P, n_out, rows * n_out) if y is None else y
    ref = [None if m is None or m == 0 else C.byref(m) for m in (x, w, residual, pre, y)]
    return L.malib_linear(C.byref(d), ref[0], ref[1], bias, ref[2], ref[3], ref[4], work, nbytes,
                          None)


@pytest.mark.parametrize("kw, word", [
    (dict(dtype=7), b"dtype"), (dict(act=9), b"activation"), (dict(groups=0), b"groups"),
    (dict(groups=65536), b"groups"), (dict(rows=-1), b"rows"), (dict(rows=1 << 31), b"rows"),
    (dict(n_in=0), b"in and out"), (dict(n_out=(1 << 24) + 1), b"in and out"),
    (dict(x=0), b"x is NULL"), (dict(w=0), b"w is NULL"), (dict(y=0), b"y is NULL"),
    (dict(x=B.Mat(None, 16, 0)), b"x is NULL"), (dict(x=B.Mat(P + 1, 16, 0)), b"aligned"),
    (dict(y=B.Mat(P, 23, 0)), b"row stride"), (dict(x=B.Mat(P, -1, 0)), b"row stride"),
    (dict(x=B.Mat(P, 16, -4)), b"group stride"), (dict(x=B.Mat(P, 1 << 41, 0)), b"too large"),
    (dict(groups=2, y=B.Mat(P, 24, 0)), b"overlap"),
    (dict(groups=2, y=B.Mat(P, 24, 24)), b"overlap"),
    (dict(groups=2, pre=B.Mat(P, 24, 100)), b"overlap"),
    (dict(bias=P + 2), b"bias"), (dict(residual=B.Mat(P + 1, 24, 0)), b"residual"),
    (dict(rows=64, n_in=65536), b"workspace"),
    (dict(rows=64, n_in=65536, work=P, nbytes=16), b"workspace"),
    (dict(rows=64, n_in=65536, work=P + 8, nbytes=1 << 30), b"16 bytes"),
])
def test_linear_refuses(kw, word):
    L = M.lib()
    assert _linear(L, **kw) == B.E_INVAL
    assert word in L.malib_last_error()


@pytest.mark.parametrize("groups, rows, row, group, apart", [
    (2, 8, 8, 8, False),        # group 1's row r is group 0's row r + 1
    (3, 8, 12, 6, False), (2, 8, 8, 5, False), (2, 3, 8, 16, False),
    (2, 8, 8, 4, True), (3, 8, 12, 4, True), (2, 8, 9, 5, True), (2, 3, 8, 20, True),
    (3, 8, 12, 8, True), (4, 8, 12, 8, False), (3, 8, 13, 9, True), (3, 2, 12, 8, True),
    (2, 1, 8, 4, True), (2, 1, 8, 3, False), (2, 1 << 30, 1 << 40, 4, True),
    (2, 1 << 30, 1 << 40, 1 << 40, False)])
def test_linear_groups_of_outputs(groups, rows, row, group, apart):
    """Groups of an output share no element, whatever their order in memory: dx of 4
    columns, whose layer then lacks its workspace."""
    L = M.lib()
    if rows < 16:
        places = {g * group + r * row + c for g in range(groups) for r in range(rows)
                  for c in range(4)}
        assert apart == (len(places) == groups * rows * 4)
    d = B.LinearDesc(B.DT_F32, B.ACT_NONE, groups, rows, 4, 65536 if rows < 16 else 64)
    m = C.byref(B.Mat(P, 65536, 0))
    assert L.malib_linear_backward(C.byref(d), m, m, m, None, C.byref(B.Mat(P, row, group)), None,
                                   None, None, 0, None) == B.E_INVAL
    assert (b"workspace" if apart else b"dx: the groups overlap") in L.malib_last_error()


def test_linear_desc_and_work_refused():
    L = M.lib()
    n = C.c_int64()
    assert L.malib_linear_work(None, 0, C.byref(n)) == B.E_INVAL
    d = B.LinearDesc(B.DT_F32, B.ACT_RELU, 1, 100000, 16, 24)
    assert L.malib_linear_work(C.byref(d), 0, None) == B.E_INVAL
    # (dW sums over 100000 rows: split over workgroups)
    assert L.malib_linear_work(C.byref(d), 1, C.byref(n)) == B.MALIB_OK and n.value > 0
    # more tiles than one launch takes
    d = B.LinearDesc(B.DT_F32, B.ACT_NONE, 65535, (1 << 31) - 1, 8, 1 << 24)
    m = B.Mat(P, 1 << 24, 1 << 45)
    assert L.malib_linear(C.byref(d), C.byref(m), C.byref(m), None, None, None,
                          C.byref(B.Mat(P, 1 << 40, 1 << 24)), P, 1 << 62,
                          None) in (B.E_UNSUPPORTED, B.E_INVAL)
    assert L.malib_linear_backward(None, None, None, None, None, None, None, None, None, 0,
                                   None) == B.E_INVAL


@pytest.mark.parametrize("act, groups, rows, n_in, n_out", [
    (B.ACT_GELU, 65535, (1 << 31) - 1, 1 << 24, 1 << 24), (B.ACT_RELU, 1024, (1 << 31) - 1, 1, 1 << 24),
    (B.ACT_GELU, 1, (1 << 31) - 1, 8, 1 << 16), (B.ACT_NONE, 65535, 1 << 31 >> 1, 8, 2)])
def test_linear_sizes_beyond_64_bits(act, groups, rows, n_in, n_out):
    """Bytes of matrices that no machine holds would not fit 64 bits: refused before
    any size is computed from them."""
    L = M.lib()
    n = C.c_int64(-5)
    for dtype in (B.DT_F32, B.DT_BF16):
        d = B.LinearDesc(dtype, act, groups, rows, n_in, n_out)
        for backward in (0, 1):
            assert L.malib_linear_work(C.byref(d), backward, C.byref(n)) == B.E_UNSUPPORTED
            assert b"2^46" in L.malib_last_error() and n.value == -5
    m = B.Mat(P, 1 << 24, 0)
    assert L.malib_linear(C.byref(d), C.byref(m), C.byref(m), None, None, None, C.byref(m), None,
                          0, None) == B.E_UNSUPPORTED
    assert L.malib_linear_backward(C.byref(d), C.byref(m), C.byref(m), C.byref(m), C.byref(m),
                                   None, None, None, None, 0, None) == B.E_UNSUPPORTED
    # the largest layer that is taken
    d = B.LinearDesc(B.DT_BF16, B.ACT_GELU, 1 << 15, 1 << 30, 1 << 24, 2)
    assert L.malib_linear_work(C.byref(d), 1, C.byref(n)) == B.MALIB_OK
    assert n.value >= 2 << 45


def test_linear_without_rows_does_nothing():
    L = M.lib()
    d = B.LinearDesc(B.DT_F32, B.ACT_NONE, 1, 0, 16, 24)
    assert L.malib_linear(C.byref(d), None, None, None, None, None, None, None, 0,
                          None) == B.MALIB_OK


@pytest.mark.parametrize("kw, word", [
    (dict(dy=None), b"dy is NULL"), (dict(x=None), b"x is NULL"), (dict(w=None), b"w is NULL"),
    (dict(act=B.ACT_GELU), b"pre is NULL"), (dict(dw=B.Mat(P, 15, 0)), b"dw"),
    (dict(dx=B.Mat(P, 15, 0)), b"dx"), (dict(dbias=P + 1), b"dbias"),
    (dict(rows=100000, nbytes=0), b"workspace"), (dict(rows=100000, work=None), b"workspace"),
])
def test_linear_backward_refuses(kw, word):
    L = M.lib()
    a = dict(rows=8, act=B.ACT_NONE, dy=B.Mat(P, 24, 0), x=B.Mat(P, 16, 0), w=B.Mat(P, 16, 0), pre=None,
             dx=B.Mat(P, 16, 0), dw=B.Mat(P, 16, 0), dbias=P, work=P, nbytes=1 << 30)
    a.update(kw)
    d = B.LinearDesc(B.DT_F32, a["act"], 1, a["rows"], 16, 24)
    ref = [None if a[k] is None else C.byref(a[k]) for k in ("dy", "x", "w", "pre", "dx", "dw")]
    assert L.malib_linear_backward(C.byref(d), *ref, a["dbias"], a["work"], a["nbytes"],
                                   None) == B.E_INVAL
    assert word in L.malib_last_error()


def test_linear_binding_checks():
    x, w = torch.zeros(4, 8), torch.zeros(6, 8)
    with pytest.raises(M.ArgumentError, match="device tensor"):
        M.linear(x, w)
    for bad, match in ((dict(x=x.half()), "dtype"), (dict(w=w.bfloat16()), "w: expected dtype"),
                       (dict(w=torch.zeros(6, 9)), "x: expected shape"),
                       (dict(w=torch.zeros(6)), "w: expected"),
                       (dict(x=torch.zeros(2, 4, 8)), "x: expected"),
                       (dict(x=torch.zeros(8, 4).t()), "contiguous rows"),
                       (dict(bias=torch.zeros(5)), "bias"),
                       (dict(bias=torch.zeros(6).double()), "bias"),
                       (dict(residual=torch.zeros(4, 5)), "residual"),
                       (dict(pre=torch.zeros(3, 6)), "pre"), (dict(act=5), "act")):
        kw = dict(x=x, w=w)
        kw.update(bad)
        with pytest.raises(M.ArgumentError, match=match):
            M.linear(**kw)
    dy = torch.zeros(4, 6)
    with pytest.raises(M.ArgumentError, match="pre"):
        M.linear_backward(dy, x, w, act=M.ACT_RELU)
    with pytest.raises(M.ArgumentError, match="dy: expected shape"):
        M.linear_backward(torch.zeros(4, 5), x, w)
    with pytest.raises(M.ArgumentError, match="x: expected shape"):
        M.linear_backward(dy, torch.zeros(5, 8), w)


def _policy(L, *, ptrs=(), work=P, nbytes=1 << 20, **kw):
    f = dict(dtype=B.DT_F32, action_bytes=4, rows=600, n_actions=5, logits_stride=5,
             ref_stride=5, dlogits_stride=5, mask_stride=5, clip_low=0.2, clip_high=0.2,
             kl_coef=0.0, entropy_coef=0.0)
    f.update(kw)
    a = dict(logits=P, actions=P, old=P, adv=P, ref_logp=None, ref_logits=None, mask=None,
             weight=None, total=P, stats=P, dlogits=P)
    a.update(ptrs)
    return L.malib_policy_loss(C.byref(B.PolicyLossDesc(*f.values())), *a.values(), work, nbytes,
                               None)


@pytest.mark.parametrize("kw, word", [
    (dict(dtype=3), b"dtype"), (dict(action_bytes=2), b"action_bytes"), (dict(rows=-1), b"rows"),
    (dict(rows=1 << 31), b"rows"), (dict(n_actions=0), b"n_actions"),
    (dict(n_actions=(1 << 24) + 1), b"n_actions"), (dict(clip_low=-0.1), b"clip"),
    (dict(clip_high=float("nan")), b"clip"), (dict(kl_coef=float("inf")), b"finite"),
    (dict(entropy_coef=float("nan")), b"finite"), (dict(kl_coef=0.1), b"kl_coef needs"),
    (dict(ptrs=dict(ref_logp=P, ref_logits=P)), b"exclude"),
    (dict(ptrs=dict(logits=None)), b"NULL"), (dict(ptrs=dict(actions=None)), b"NULL"),
    (dict(ptrs=dict(old=None)), b"NULL"), (dict(ptrs=dict(adv=None)), b"NULL"),
    (dict(ptrs=dict(logits=P + 2)), b"logits"), (dict(ptrs=dict(actions=P + 2)), b"actions"),
    (dict(logits_stride=-5), b"logits"), (dict(dlogits_stride=4), b"dlogits"),
    (dict(ref_stride=1 << 41, ptrs=dict(ref_logits=P)), b"ref_logits"),
    (dict(mask_stride=-1, ptrs=dict(mask=P)), b"mask"), (dict(work=None), b"workspace"),
    (dict(nbytes=4), b"workspace"), (dict(work=P + 4), b"16 bytes"),
])
def test_policy_loss_refuses(kw, word):
    L = M.lib()
    assert _policy(L, **kw) == B.E_INVAL
    assert word in L.malib_last_error()


def _distill(L, *, ptrs=(), work=P, nbytes=1 << 20, **kw):
    f = dict(dtype=B.DT_F32, top=3, rows=600, n_actions=5, logits_stride=5, dlogits_stride=5,
             mask_stride=5, temperature=1.0)
    f.update(kw)
    a = dict(logits=P, idx=P, val=P, mask=None, weight=None, total=P, loss=P, dlogits=P)
    a.update(ptrs)
    return L.malib_distill_loss(C.byref(B.DistillDesc(*f.values())), *a.values(), work, nbytes,
                                None)


@pytest.mark.parametrize("kw, word", [
    (dict(dtype=3), b"dtype"), (dict(top=0), b"top"), (dict(top=257), b"top"),
    (dict(temperature=0.0), b"temperature"), (dict(temperature=float("inf")), b"temperature"),
    (dict(temperature=float("nan")), b"temperature"), (dict(rows=-1), b"rows"),
    (dict(n_actions=0), b"n_actions"), (dict(ptrs=dict(logits=None)), b"NULL"),
    (dict(ptrs=dict(idx=None)), b"NULL"), (dict(ptrs=dict(val=None)), b"NULL"),
    (dict(dlogits_stride=4), b"dlogits"), (dict(work=None), b"workspace"),
])
def test_distill_loss_refuses(kw, word):
    L = M.lib()
    assert _distill(L, **kw) == B.E_INVAL
    assert word in L.malib_last_error()


def test_loss_work_and_null_descriptions():
    L = M.lib()
    n = C.c_int64(-1)
    assert L.malib_loss_work(B.DT_F32, 100, 5, None) == B.E_INVAL
    assert L.malib_loss_work(9, 100, 5, C.byref(n)) == B.E_INVAL
    assert L.malib_loss_work(B.DT_F32, 100, 5, C.byref(n)) == B.MALIB_OK and n.value >= 0
    assert L.malib_policy_loss(None, *[None] * 12, 0, None) == B.E_INVAL
    assert L.malib_distill_loss(None, *[None] * 9, 0, None) == B.E_INVAL


def test_loss_binding_checks():
    n, a = 6, 9
    ok = dict(logits=torch.zeros(n, a), actions=torch.zeros(n, dtype=torch.int32),
              old_logp=torch.zeros(n), advantage=torch.zeros(n))
    with pytest.raises(M.ArgumentError, match="device tensor"):
        M.policy_loss(**ok)
    for bad, match in ((dict(logits=torch.zeros(n, a).half()), "dtype"),
                       (dict(logits=torch.zeros(n)), "logits: expected"),
                       (dict(logits=torch.zeros(a, n).t()), "contiguous rows"),
                       (dict(actions=torch.zeros(n, dtype=torch.int16)), "actions"),
                       (dict(actions=torch.zeros(n - 1, dtype=torch.int32)), "actions"),
                       (dict(old_logp=torch.zeros(n).double()), "old_logp"),
                       (dict(advantage=torch.zeros(n + 1)), "advantage"),
                       (dict(ref_logp=torch.zeros(n - 1)), "ref_logp"),
                       (dict(ref_logits=torch.zeros(n, a).bfloat16()), "ref_logits"),
                       (dict(mask=torch.zeros(n, a)), "mask"),
                       (dict(mask=torch.zeros((n, a + 1), dtype=torch.bool)), "mask"),
                       (dict(weight=torch.zeros(1)), "weight"),
                       (dict(stats=torch.zeros(n)), "stats"),
                       (dict(dlogits=torch.zeros(n, a + 1)), "dlogits")):
        with pytest.raises(M.ArgumentError, match=match):
            M.policy_loss(**{**ok, **bad})
    ok = dict(logits=torch.zeros(n, a), teacher_idx=torch.zeros((n, 2), dtype=torch.int32),
              teacher_logits=torch.zeros(n, 2))
    with pytest.raises(M.ArgumentError, match="device tensor"):
        M.distill_loss(**ok)
    for bad, match in ((dict(teacher_idx=torch.zeros((n, 2), dtype=torch.int64)), "teacher_idx"),
                       (dict(teacher_idx=torch.zeros(n, dtype=torch.int32)), "teacher_idx"),
                       (dict(teacher_logits=torch.zeros(n, 3)), "teacher_logits"),
                       (dict(loss=torch.zeros(2)), "loss"), (dict(total=torch.zeros(2)), "total")):
        with pytest.raises(M.ArgumentError, match=match):
            M.distill_loss(**{**ok, **bad})

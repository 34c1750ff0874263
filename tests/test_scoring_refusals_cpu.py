"""What log probabilities, dropout and the layers in 4 bits refuse, on the host and before any
device work: the library's own checks (pointers are never dereferenced) and the binding's checks
of shapes, types, strides and devices."""
import ctypes as C

import pytest
import torch

import paper_2106_07551_amd as M
from paper_2106_07551_amd import binding as B

P = 4096          # an address that is never read


def refused(status, word):
    assert status == B.E_INVAL or status == B.E_UNSUPPORTED
    assert word in B.lib().malib_last_error(), B.lib().malib_last_error()


def _log_probs(*, dtype=B.DT_BF16, size=4, rows=3, n=50, stride=None, mask_stride=0, top=2, T=1.0,
               logits=P, actions=P, mask=None, stats=P, idx=P, val=P, work=None, nbytes=0):
    d = B.LogProbsDesc(dtype, size, rows, n, n if stride is None else stride, 0, mask_stride, top,
                       T)
    return M.lib().malib_log_probs(C.byref(d), logits, actions, mask, stats, idx, val, work,
                                   nbytes, None)


@pytest.mark.parametrize("kw, word", [
    (dict(dtype=7), b"dtype"), (dict(rows=-1), b"rows"), (dict(rows=1 << 31), b"rows"),
    (dict(n=0), b"n_actions"), (dict(n=(1 << 24) + 1), b"n_actions"), (dict(T=0.0), b"temperature"),
    (dict(T=float("nan")), b"temperature"), (dict(T=float("inf")), b"temperature"),
    (dict(T=-1.0), b"temperature"), (dict(top=-1), b"top"), (dict(top=257), b"top"),
    (dict(logits=None), b"logits"), (dict(logits=P + 1), b"logits"), (dict(stride=-1), b"logits"),
    (dict(stride=1 << 41), b"logits"), (dict(size=2), b"action_bytes"),
    (dict(actions=P + 2), b"actions"), (dict(mask=P, mask_stride=-3), b"mask"),
    (dict(stats=None), b"stats"), (dict(stats=P + 2), b"stats"), (dict(idx=None), b"top_idx"),
    (dict(val=None), b"top_idx"), (dict(idx=P + 2), b"top_idx"), (dict(val=P + 1), b"top_logp"),
    (dict(n=1 << 20), b"workspace"), (dict(n=1 << 20, work=P, nbytes=16), b"workspace"),
    (dict(n=1 << 20, work=P + 8, nbytes=1 << 30), b"16 bytes"),
])
def test_log_probs_refuses(kw, word):
    refused(_log_probs(**kw), word)


def test_log_probs_sizes_of_products():
    need = C.c_int64()
    L = M.lib()
    refused(L.malib_log_probs_work(B.DT_F32, 1 << 31, 5, 1, C.byref(need)), b"rows")
    refused(L.malib_log_probs_work(B.DT_F32, 5, 5, 257, C.byref(need)), b"top")
    refused(L.malib_log_probs_work(B.DT_F32, 5, 5, 7, None), b"work_bytes")
    assert L.malib_log_probs_work(B.DT_F32, (1 << 31) - 1, 18, 256, C.byref(need)) == B.MALIB_OK
    assert need.value == 0
    for rows, n, top in ((3, 131071, 8), (1, 1 << 24, 256), (700, 1 << 24, 256), (200, 70001, 1)):
        assert L.malib_log_probs_work(B.DT_F32, rows, n, top, C.byref(need)) == B.MALIB_OK
        assert need.value > 0


def _backward(*, rows=3, n=50, stride=None, T=1.0, logits=P, actions=P, stats=P, dlogp=P, dent=P,
              dlogits=P):
    d = B.LogProbsDesc(B.DT_F32, 4, rows, n, n, n if stride is None else stride, 0, 0, T)
    return M.lib().malib_log_probs_backward(C.byref(d), logits, actions, None, stats, dlogp, dent,
                                            dlogits, None)


@pytest.mark.parametrize("kw, word", [
    (dict(T=0.0), b"temperature"), (dict(stats=None), b"stats"), (dict(dlogits=None), b"dlogits"),
    (dict(actions=None), b"actions"), (dict(dlogp=P + 1), b"dlogp"), (dict(dent=P + 2), b"dentropy"),
    (dict(stride=49), b"dlogits"), (dict(dlogits=P + 2), b"dlogits"), (dict(logits=None), b"logits"),
])
def test_log_probs_backward_refuses(kw, word):
    refused(_backward(**kw), word)


def _dropout(*, dtype=B.DT_F32, rows=4, cols=8, xs=8, rs=8, ys=8, p=0.5, x=P, r=None, step=None,
             y=P):
    d = B.DropoutDesc(dtype, 0, rows, cols, xs, rs, ys, 1, 2, p)
    return M.lib().malib_dropout(C.byref(d), x, r, step, y, None)


@pytest.mark.parametrize("kw, word", [
    (dict(dtype=3), b"dtype"), (dict(rows=-1), b"rows"), (dict(rows=1 << 31), b"rows"),
    (dict(cols=0), b"cols"), (dict(cols=(1 << 24) + 1), b"cols"), (dict(p=-0.1), b"p must"),
    (dict(p=1.1), b"p must"), (dict(p=float("nan")), b"p must"), (dict(x=None), b"x and y"),
    (dict(y=None), b"x and y"), (dict(ys=7), b"y: bad"), (dict(xs=-1), b"x: bad"),
    (dict(x=P + 2), b"x is not"), (dict(r=P + 1), b"residual"), (dict(step=P + 4), b"device_step"),
])
def test_dropout_refuses(kw, word):
    refused(_dropout(**kw), word)


def _fp4(call, *, dtype=B.DT_F32, act=0, groups=1, rows=2, n_in=40, n_out=20, group=32, reserved=0,
         m=P, ld=None, gs=0, codes=P, scales=P, bias=None, y=P, yld=None):
    d = B.Fp4Desc(dtype, act, groups, rows, n_in, n_out, group, reserved)
    L = M.lib()
    w = None if m is None else C.byref(B.Mat(m, n_in if ld is None else ld, gs))
    if call == "quantize":
        return L.malib_quantize_fp4(C.byref(d), w, codes, scales, None)
    if call == "dequantize":
        return L.malib_dequantize_fp4(C.byref(d), codes, scales, w, None)
    out = None if y is None else C.byref(B.Mat(y, n_out if yld is None else yld, gs))
    return L.malib_linear_fp4(C.byref(d), w, codes, scales, bias, None, out, None)


@pytest.mark.parametrize("call", ["quantize", "dequantize", "linear"])
@pytest.mark.parametrize("kw, word", [
    (dict(dtype=9), b"dtype"), (dict(act=9), b"activation"), (dict(groups=0), b"groups"),
    (dict(n_in=0), b"in and out"), (dict(n_out=1 << 25), b"in and out"),
    (dict(group=16), b"scale_group"), (dict(group=256), b"scale_group"),
    (dict(reserved=1), b"reserved"), (dict(m=None), b"is NULL"), (dict(m=P + 1), b"aligned"),
    (dict(codes=None), b"codes"), (dict(scales=None), b"codes"), (dict(codes=P + 8), b"codes"),
    (dict(scales=P + 4), b"scales"), (dict(ld=-1), b"row stride"),
    (dict(groups=65535, n_in=1 << 24, n_out=1 << 24), b"2^46"),
])
def test_fp4_refuses(call, kw, word):
    refused(_fp4(call, **kw), word)


@pytest.mark.parametrize("kw, word", [
    (dict(y=None), b"y is NULL"), (dict(yld=19), b"row stride"), (dict(bias=P + 2), b"bias"),
    (dict(rows=-1), b"rows"), (dict(groups=2, gs=4), b"overlap"),
])
def test_linear_fp4_refuses(kw, word):
    refused(_fp4("linear", **kw), word)


X, F = torch.ones(3, 8), torch.zeros(3)
A = torch.zeros(3, dtype=torch.int32)
CODES, SCALES = torch.zeros((1, 1, 64, 16), dtype=torch.uint8), torch.zeros((1, 1, 16, 4),
                                                                           dtype=torch.bfloat16)


@pytest.mark.parametrize("call, word", [
    (lambda: M.log_probs(X, A), "logits: expected a device"),
    (lambda: M.log_probs(X.double(), A), "logits: expected dtype"),
    (lambda: M.log_probs(X[0], A), "logits: expected"),
    (lambda: M.log_probs(X.t(), A), "logits: expected contiguous"),
    (lambda: M.log_probs(X, A.float()), "actions: expected dtype"),
    (lambda: M.log_probs(X, A[:2]), "actions: expected 3"),
    (lambda: M.log_probs(X, A, top=257), "top"),
    (lambda: M.log_probs(X, A, top=-1), "top"),
    (lambda: M.log_probs(X, A, mask=X), "mask: expected dtype"),
    (lambda: M.log_probs(X, A, mask=X[:2].bool()), "mask: expected shape"),
    (lambda: M.log_probs(X, A, stats=F), "stats: expected 12"),
    (lambda: M.log_probs(X, A, top=2, top_idx=A), "top_idx: expected 6"),
    (lambda: M.log_probs(X, A, top=2, top_logp=A), "top_logp: expected dtype"),
    (lambda: M.log_probs_backward(X, A, F, F), "stats: expected 12"),
    (lambda: M.log_probs_backward(X, A, torch.zeros(4, 3), A), "dlogp: expected dtype"),
    (lambda: M.log_probs_backward(X, A, torch.zeros(4, 3), F, F[:1]), "dentropy: expected 3"),
    (lambda: M.log_probs_backward(X, A, torch.zeros(4, 3), F, dlogits=X[:2]), "dlogits"),
    (lambda: M.log_probs_backward(X, A, torch.zeros(4, 3), F), "expected a device"),
    (lambda: M.dropout(X, 0.5, 1), "x: expected a device"),
    (lambda: M.dropout(X.half(), 0.5, 1), "x: expected dtype"),
    (lambda: M.dropout(X, 1.5, 1), "p: expected"),
    (lambda: M.dropout(X, float("nan"), 1), "p: expected"),
    (lambda: M.dropout(X, 0.5, -1), "seed"),
    (lambda: M.dropout(X, 0.5, 1 << 64), "seed"),
    (lambda: M.dropout(X, 0.5, 1, -1), "step"),
    (lambda: M.dropout(X, 0.5, 1, layer=1 << 32), "layer"),
    (lambda: M.dropout(X, 0.5, 1, residual=X[:2]), "residual: expected shape"),
    (lambda: M.dropout(X, 0.5, 1, residual=X.double()), "residual: expected dtype"),
    (lambda: M.dropout(X.t(), 0.5, 1), "x: expected a contiguous"),
    (lambda: M.dropout(X, 0.5, 1, out=X.t().contiguous().t()), "out: expected a contiguous"),
    (lambda: M.dropout(X, 0.5, 1, device_step=A), "device_step: expected dtype"),
    (lambda: M.dropout_backward(X, 0.5, 1, dx=X[:1]), "out: expected shape"),
    (lambda: M.quantize_fp4(X), "w: expected a device"),
    (lambda: M.quantize_fp4(X[0]), "w: expected"),
    (lambda: M.quantize_fp4(X, 16), "group"),
    (lambda: M.dequantize_fp4(CODES, SCALES, 17, 8), "codes: expected shape"),
    (lambda: M.dequantize_fp4(CODES, SCALES, 5, 8, dtype=torch.float16), "dtype"),
    (lambda: M.dequantize_fp4(CODES, SCALES, 5, 8), "codes: expected a device"),
    (lambda: M.dequantize_fp4(CODES.float(), SCALES, 5, 8), "codes: expected dtype"),
    (lambda: M.dequantize_fp4(CODES, SCALES[..., :3], 5, 8), "scales: expected 1, 2 or 4"),
    (lambda: M.linear_fp4(X, CODES, SCALES, 5), "x: expected a device"),
    (lambda: M.linear_fp4(X, CODES, SCALES, 17), "codes: expected shape"),
    (lambda: M.linear_fp4(X[None], CODES, SCALES, 5), "x: expected"),
    (lambda: M.linear_fp4(X, CODES, SCALES, 5, act=9), "act"),
    (lambda: M.linear_fp4(X, CODES, SCALES, 5, F), "bias: expected 5"),
    (lambda: M.linear_fp4(X, CODES, SCALES, 5, residual=X), "residual: expected shape"),
])
def test_binding_refuses(call, word):
    with pytest.raises(M.ArgumentError, match=word):
        call()


@pytest.mark.parametrize("name, n", [("log_probs", 10), ("log_probs_backward", 9), ("dropout", 9),
                                     ("quantize_fp4", 5), ("dequantize_fp4", 7),
                                     ("linear_fp4", 9)])
def test_native_calls_leave_what_they_do_not_take(name, n):
    call = getattr(B._native(), name)
    with pytest.raises(TypeError):
        call(X)
    for args in ((None,) * n, ("x",) * n, (X,) * n, (X, A, 1.0, 2) + (None,) * (n - 4)):
        assert call(*args) is None

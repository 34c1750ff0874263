"""Log probabilities, dropout and the layers in 4 bits as a learner runs them: the native calls
against the binding's own way, together in one step, and captured into graphs."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def tensors(out):
    return (out,) if isinstance(out, torch.Tensor) else out


def both_ways(fn, *a, **kw):
    """fn's outputs through the native call and through the binding alone."""
    native = fn(*a, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    slow = fn(*a, **kw, stream=side)
    side.synchronize()
    for p, q in zip(tensors(native), tensors(slow)):
        assert (p is None) == (q is None)
        if p is not None:
            assert p.shape == q.shape and p.dtype == q.dtype and p.stride() == q.stride()
            assert torch.equal(torch.nan_to_num(p.float(), 7.0), torch.nan_to_num(q.float(), 7.0))
    return native


def rnd(*s, dtype=torch.float32):
    return torch.randn(s, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_both_ways(dtype):
    import paper_2106_07551_amd as M
    B = M.binding
    for n, a in ((0, 4), (1, 1), (50, 9), (40, 300), (3, 40000)):
        x = rnd(n, a + 3, dtype=dtype)[:, :a]
        mask = torch.rand((n, a), device="cuda") < 0.8
        d = rnd(n)
        for ids in (torch.uint8, torch.int32, torch.int64):
            act = (torch.arange(n, device="cuda") % min(a, 100)).to(ids)
            both_ways(M.log_probs, x, act)
            s, _, _ = both_ways(M.log_probs, x, act, top=5, mask=mask, temperature=2)
            both_ways(M.log_probs_backward, x, act, s, d, d, mask=mask.byte(), temperature=2)
        assert both_ways(M.log_probs, x, top=3)[1].shape == (n, 3)
    for shape in ((5, 7), (3, 4, 33), (40,)):
        x, r = rnd(*shape, dtype=dtype), rnd(*shape, dtype=dtype)
        both_ways(M.dropout, x, 0.3, 2 ** 64 - 1, 2 ** 64 - 1, layer=2 ** 32 - 1, residual=r)
        both_ways(M.dropout_backward, x, 0.3, 5)
    for lead in ((), (1,), (3,)):
        w, x = rnd(*lead, 20, 150, dtype=dtype), rnd(*lead, 5, 150, dtype=dtype)
        for group in (32, 64, 128):
            codes, scales = both_ways(M.quantize_fp4, w, group)
            both_ways(M.dequantize_fp4, codes, scales, 20, 150)
            both_ways(M.dequantize_fp4, codes, scales, 20, 150, dtype=torch.float32)
            y = both_ways(M.linear_fp4, x, codes, scales, 20, rnd(*lead, 20), act=M.ACT_GELU,
                          residual=rnd(*lead, 5, 20, dtype=dtype))
            into = M.dequantize_fp4(codes, scales, 20, 150, out=torch.empty_like(w))
            assert into.dtype is dtype
        assert y.shape == lead + (5, 20)
    assert B._calls is not None


def test_refusals_name_the_argument():
    import paper_2106_07551_amd as M
    x, act = rnd(9, 8), torch.zeros(9, dtype=torch.int32, device="cuda")
    codes, scales = M.quantize_fp4(rnd(5, 8))
    s = M.log_probs(x, act)[0]
    odd = torch.empty(codes.numel() + 8, dtype=torch.uint8, device="cuda")[8:].view(codes.shape)
    for fn, word in (
            (lambda: M.log_probs(x, act.cpu()), "actions"),
            (lambda: M.log_probs(x, act, temperature=0.0), "temperature"),
            (lambda: M.log_probs(x, act, mask=torch.ones(9, 8)), "mask"),
            (lambda: M.log_probs(rnd(2, 1 << 20), top=2,
                                 work=torch.empty(8, device="cuda")), "work"),
            (lambda: M.log_probs_backward(x, None, s, s[0]), "dlogp"),
            (lambda: M.log_probs_backward(x, act, s, s[0], dlogits=rnd(9, 7)), "dlogits"),
            (lambda: M.log_probs_backward(x, act, s.cpu(), s[0].contiguous()), "stats"),
            (lambda: M.dropout(x, 0.5, 1, residual=x.cpu()), "residual"),
            (lambda: M.dropout(x, 0.5, 1, device_step=torch.zeros(2, dtype=torch.int64,
                                                                  device="cuda")), "device_step"),
            (lambda: M.dropout(x, 0.5, 1, out=x[:1].expand(9, 8)), "y"),
            (lambda: M.quantize_fp4(x, 48), "group"),
            (lambda: M.dequantize_fp4(odd, scales, 5, 8), "codes"),
            (lambda: M.dequantize_fp4(codes, scales, 5, 8, out=rnd(5, 9)), "out"),
            (lambda: M.linear_fp4(x, codes, scales, 5, rnd(4)), "bias"),
            (lambda: M.linear_fp4(x, codes, scales.cpu(), 5), "scales"),
            (lambda: M.linear_fp4(rnd(9, 200), codes, scales, 5), "codes")):
        with pytest.raises(M.MalibError, match=word):
            fn()


class Step:
    """A distillation step: teachers in 4 bits, their lists, a student's layer with dropout, the
    loss and the layer's gradients; and the scores of the student's own actions."""

    def __init__(self, rows=40, width=96, actions=50, teachers=3, dtype=torch.bfloat16):
        import paper_2106_07551_amd as M
        self.M = M
        self.rows, self.actions = rows, actions
        self.held = M.quantize_fp4(rnd(teachers, actions, width) * width ** -0.5)
        self.w1, self.w2 = rnd(64, width, dtype=dtype), rnd(actions, 64, dtype=dtype)
        self.x = rnd(rows, width, dtype=dtype)
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.act = torch.randint(0, actions, (rows,), device="cuda")
        self.work = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def __call__(self):
        M = self.M
        teacher = M.linear_fp4(self.x, *self.held, self.actions).float().mean(0)
        _, idx, val = M.log_probs(teacher, top=7, work=self.work)
        pre = torch.empty((self.rows, 64), dtype=self.x.dtype, device="cuda")
        h = M.linear(self.x, self.w1, act=M.ACT_GELU, pre=pre)
        h = M.dropout(h, 0.2, 77, layer=1, device_step=self.step)
        logits = M.linear(h, self.w2)
        total, loss, dlogits = M.distill_loss(logits, idx, val)
        stats, _, _ = M.log_probs(logits, self.act, work=self.work)
        dscore = M.log_probs_backward(logits, self.act, stats, loss, loss)
        dh, dw2, _ = M.linear_backward(dlogits, h, self.w2)
        dh = M.dropout_backward(dh, 0.2, 77, layer=1, device_step=self.step)
        _, dw1, _ = M.linear_backward(dh, self.x, self.w1, act=M.ACT_GELU, pre=pre)
        self.step.add_(1)
        return teacher, idx, val, total, loss, stats, dscore, dw1, dw2


def test_a_step_against_plain_operations():
    """The whole step in 64 bits with the dropout's own mask: gradients of the student's
    layers by torch's autograd.  In fp32 the sums have up to 96 terms (96 u of the largest, u =
    2^-24), softmax and its logarithms 200 u (as in the losses), GELU and its slope 10 u, the
    other operations a few each: 500 u of the largest entry covers them."""
    s = Step(dtype=torch.float32)
    M = s.M
    teacher, idx, val, total, loss, stats, dscore, dw1, dw2 = s()
    keep = (M.dropout(torch.ones((s.rows, 64), device="cuda"), 0.2, 77, 0, layer=1) > 0).double()
    w1, w2 = (w.double().requires_grad_() for w in (s.w1, s.w2))
    q = 1 - round(0.2 * 65536) / 65536
    h = torch.nn.functional.gelu(s.x.double() @ w1.T) * keep / q
    logits = h @ w2.T
    logp = torch.log_softmax(logits, 1)
    t = torch.softmax(val.double(), 1)
    per_row = (t * (t.log() - logp.gather(1, idx.long()))).sum(1)
    per_row.mean().backward()
    for got, ref in ((dw1, w1.grad), (dw2, w2.grad), (loss, per_row.detach())):
        assert float((got.double() - ref).abs().max()) <= 500 * 2 ** -24 * float(ref.abs().max())
    ent = -(logp.exp() * logp).sum(1)
    lp = logp[torch.arange(s.rows, device="cuda"), s.act]
    z = logits.detach().requires_grad_()
    lz = torch.log_softmax(z, 1)
    (loss.double() * (lz[torch.arange(s.rows, device="cuda"), s.act] -
                      (lz.exp() * lz).sum(1))).sum().backward()
    for got, ref in ((stats[0], lp), (stats[1], ent), (dscore, z.grad)):
        ref = ref.detach()
        assert float((got.double() - ref).abs().max()) <= 500 * 2 ** -24 * float(ref.abs().max())


def captured(step):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    step.step.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    return g, out


@pytest.mark.parametrize("actions", [18, 50, 20000])
def test_captured_steps(actions):
    """Two graphs that share a workspace, replayed in turn, with new inputs and eager calls between
    the replays: every replay equals the eager call with its step's number."""
    a, b = Step(actions=actions), Step(rows=7, actions=actions)
    b.work = a.work
    (ga, oa), (gb, ob) = captured(a), captured(b)
    for replay in range(4):
        for s, g, out in ((a, ga, oa), (b, gb, ob)):
            s.x.copy_(rnd(*s.x.shape, dtype=s.x.dtype))
            s.step.fill_(replay)
            eager = s()
            s.step.fill_(replay)
            eager[0].sum()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for p, q in zip(out, eager):
                assert torch.equal(p, q), (actions, replay)
            assert int(s.step) == replay + 1


def test_two_streams_at_once():
    """Calls on two streams at the same time, each with workspaces of its own."""
    import paper_2106_07551_amd as M
    xs = [rnd(4, 200000), rnd(4, 200000)]
    want = [M.log_probs(x, top=64) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(5):
        for i, st in enumerate(streams):
            got[i].append(M.log_probs(xs[i], top=64, stream=st))
    torch.cuda.synchronize()
    for i in range(2):
        for out in got[i]:
            assert all(map(torch.equal, out, want[i]))


def test_example_with_dropout_and_teachers_in_4_bits():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import learner
    lines = []
    out = learner.run(n_envs=64, horizon=3, policies=4, steps=3, dropout=0.1, teacher_bits=4,
                      say=lines.append)
    assert len(lines) == 4 and all(x == x for x in out["losses"])
    assert torch.isfinite(out["stats"]).all() and torch.isfinite(out["sigma"]).all()
    w = [torch.randn((3, 40, 24), device="cuda"), torch.randn((3, 40, 40), device="cuda"),
         torch.randn((3, 18, 40), device="cuda")]
    b = [torch.randn(v.shape[:2], device="cuda") for v in w]
    held = learner.Teachers(w, b, 4)
    obs = torch.randn((learner.Teachers.FEW + 1, 24), device="cuda").bfloat16()
    few, many = held.logits(obs[:5]), held.logits(obs)[:, :5]
    # both ways' hidden values are bf16 roundings of the same sums: one of a value's last places
    # (2^-7) apart at most, twice
    assert float((few - many).abs().max()) <= 2 ** -6 * float(many.abs().max())

"""Timed cases of the learner's operators: the linear layer with its epilogue,
forward and backward, and the two losses over a policy's logits, each with its
gradient.

    listed()         the cases
    draw(rng)        another case of the same ranges
    prepare(case, s) the inputs a learner holds before the call
    run(state)       one pass: the library's operator where `own` is true, else
                     its plain form in elementary torch operations
    work(case)       bytes and operations one pass cannot do without
    exact(case, s)   the outputs in 64 bits, from the formulas

Formulas (all sums over the last index; a row is one decision of one seat):

  linear            z = x W^T + b,  y = act(z) + residual
  linear, backward  dz = dy act'(z);  dx = dz W,  dW = dz^T x,  db = sum_rows dz
  policy loss       p = softmax over the legal entries, l = log p[action],
                    r = exp(l - old), s = min(r A, clip(r, 1 - lo, 1 + hi) A),
                    KL = sum_j p_j (log p_j - log q_j) against reference logits,
                    or e^d - 1 - d with d = ref - l against a reference log
                    probability, H = -sum_j p_j log p_j,
                    loss = -s + kl KL - ent H, total = sum_rows w loss
  distillation      t = softmax of the teacher's listed logits / T, q = softmax
                    of the student's legal logits / T,
                    loss = T^2 sum_k t_k (log t_k - log q[idx_k])

A row of the policy loss counts if its action is a legal entry and its weight
is not 0; an entry of a teacher's list counts if its index is a legal entry,
and a row of the distillation if any entry does and its weight is not 0.  Rows
that do not count give zeros.
"""
import math

import torch

own = False

ACTS = ("none", "relu", "gelu", "silu")
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _linear(name, way, dtype, rows, n_in, n_out, act, *, groups=1, bias=True, residual=False,
            train=False, pad=0):
    """way "forward" (train: the values before the activation are kept for the
    backward pass) or "backward"; groups: policies with weights of their own;
    pad: elements between the end of a row of x or dy and the next row."""
    c = {"op": "linear", "way": way, "dtype": dtype, "rows": rows, "in": n_in, "out": n_out,
         "act": act, "groups": groups, "bias": bias, "residual": residual, "train": train,
         "pad": pad}
    if name:
        c["name"] = name
    return c


def _policy(name, dtype, rows, actions, *, kl="sampled", ids="int32", mask=False, weight=False,
            pad=0):
    """kl "none", "sampled" (against the reference's log probability of the
    action) or "full" (against the reference's logits); ids: type of the
    actions; pad: elements between a row's logits and the next row's."""
    c = {"op": "policy", "dtype": dtype, "rows": rows, "actions": actions, "kl": kl, "ids": ids,
         "mask": mask, "weight": weight, "pad": pad}
    if name:
        c["name"] = name
    return c


def _distill(name, dtype, rows, actions, top, *, temperature=1.0, mask=False, weight=False,
             pad=0):
    c = {"op": "distill", "dtype": dtype, "rows": rows, "actions": actions, "top": top,
         "temperature": temperature, "mask": mask, "weight": weight, "pad": pad}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the first layer of the 4v4 game's policies over one step of the whole
        # batch (16384 envs x 8 seats), kept for the backward pass
        _linear("linear_team_forward", "forward", "bf16", 131072, 256, 512, "relu", train=True),
        # the second layer's backward pass on the same rows: dW sums over 131072
        _linear("linear_team_backward", "backward", "bf16", 131072, 512, 512, "relu"),
        # a few decisions at a time through a wide layer: the weights are the work
        _linear("linear_few_rows_forward", "forward", "bf16", 3, 8192, 8192, "silu",
                residual=True),
        # a large network's layer: the matrix products are the work
        _linear("linear_large_backward", "backward", "bf16", 8192, 4096, 4096, "gelu"),
        # the iterated game's 16 fp32 policies trained side by side
        _linear("linear_population_forward", "forward", "f32", 8192, 24, 64, "relu", groups=16,
                train=True),
        # odd sizes: no row starts on a 16-byte boundary
        _linear("linear_odd_backward", "backward", "f32", 5003, 777, 333, "silu", pad=1),
        # 16 steps of 4v4 records: 18 actions, byte actions with 255 where an
        # env had finished
        _policy("policy_records", "f32", 2097152, 18, ids="uint8"),
        # a batch of 24 envs x 8 seats with legal-action masks: latency
        _policy("policy_small", "f32", 192, 18, kl="full", mask=True, weight=True),
        # a large action space (token-sized), against a reference policy's logits
        _policy("policy_wide", "bf16", 4096, 65536, kl="full"),
        # three decisions over an odd large space with masks
        _policy("policy_few_rows", "bf16", 3, 131071, mask=True),
        # one step of the 4v4 batch distilled from six listed actions of its teachers
        _distill("distill_actions", "f32", 131072, 18, 6, mask=True, weight=True),
        # a large odd action space, padded rows, the teacher's 64 best
        _distill("distill_wide", "bf16", 2047, 50001, 64, temperature=2.0, pad=7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: as it falls, or a multiple of 8 or 64 as networks have them."""
    n = _log(rng, lo, hi)
    m = rng.choice([1, 8, 64, 64])
    return n if n < m else n // m * m


def draw(rng):
    """Another case of the ranges above: every direction, type, activation and
    divergence, one row to as many as fit the largest case's work."""
    op = rng.choice(["linear", "linear", "linear", "policy", "policy", "distill"])
    dtype = rng.choice(["f32", "bf16"])
    pad = rng.choice([0, 0, 0, 1, 8, 13])
    if op == "linear":
        way = rng.choice(["forward", "backward"])
        groups = rng.choice([1, 1, 1, 1, rng.randint(2, 24)])
        while True:
            rows, n_in, n_out = _log(rng, 1, 131072), _width(rng, 3, 8192), _width(rng, 3, 8192)
            if groups * rows * n_in * n_out <= (1 << 36) >> (dtype == "f32") * 2 and \
                    groups * rows * max(n_in, n_out) <= 1 << 27 and \
                    groups * n_in * n_out <= 1 << 26:
                break
        return _linear("", way, dtype, rows, n_in, n_out, rng.choice(ACTS), groups=groups,
                       bias=rng.random() < 0.7, residual=rng.random() < 0.4,
                       train=rng.random() < 0.6, pad=pad)
    while True:
        rows, actions = _log(rng, 1, 2097152), _log(rng, 2, 131072)
        if rows * actions <= 1 << 27:
            break
    mask, weight = rng.random() < 0.4, rng.random() < 0.5
    if op == "policy":
        ids = rng.choice(["uint8", "int32", "int64"]) if actions < 256 else \
            rng.choice(["int32", "int64"])
        return _policy("", dtype, rows, actions, kl=rng.choice(["none", "sampled", "full"]),
                       ids=ids, mask=mask, weight=weight, pad=pad)
    top = min(actions, _log(rng, 1, 128))
    while rows * top > 1 << 25:
        top = (top + 1) // 2
    return _distill("", dtype, rows, actions, top,
                    temperature=rng.choice([1.0, 2.0, 0.7, 4.0]), mask=mask, weight=weight,
                    pad=pad)


# ------------------------------------------------------------------ inputs

CLIP_LOW, CLIP_HIGH, KL_COEF, ENTROPY_COEF = 0.2, 0.28, 0.05, 0.01


def _padded(x, pad):
    """x as a view with `pad` more elements (of other data) behind each row."""
    if not pad:
        return x.contiguous()
    wide = torch.full(x.shape[:-1] + (x.shape[-1] + pad,), 7.0, dtype=x.dtype, device=x.device)
    wide[..., :x.shape[-1]] = x
    return wide[..., :x.shape[-1]]


def _grouped(c, *shape):
    return (c["groups"],) + shape if c["groups"] > 1 else shape


def _prepare_linear(c, g):
    t, M, K, N = TYPES[c["dtype"]], c["rows"], c["in"], c["out"]

    def normal(scale, *shape, dtype=t):
        return (torch.randn(_grouped(c, *shape), generator=g, device="cuda") * scale).to(dtype)

    s = {"x": _padded(normal(1.0, M, K), c["pad"]), "w": normal(K ** -0.5, N, K)}
    if c["way"] == "forward":
        s["bias"] = normal(0.1, N, dtype=torch.float32) if c["bias"] else None
        s["residual"] = normal(1.0, M, N) if c["residual"] else None
    else:
        s["dy"] = _padded(normal(1.0, M, N), c["pad"])
        s["pre"] = normal(1.0, M, N) if c["act"] != "none" else None
    return s


def _prepare_loss(c, g):
    """Logits, the legal entries and the rows' weights of either loss.  Masked
    places hold what buffers hold there: numbers, the lowest number, infinities
    and NaN."""
    t, n, a = TYPES[c["dtype"]], c["rows"], c["actions"]
    logits = (torch.randn((n, a), generator=g, device="cuda") * 2.0).to(t)
    s = {"mask": None, "weight": None}
    if c["mask"]:
        u = torch.rand((n, a), generator=g, device="cuda")
        s["mask"] = u < 0.8
        s["mask"][torch.rand(n, generator=g, device="cuda") < 0.02] = False
        for lo, hi, v in ((0.8, 0.81, math.nan), (0.81, 0.82, math.inf), (0.82, 0.83, -math.inf),
                          (0.83, 0.84, torch.finfo(t).min)):
            logits = torch.where((u >= lo) & (u < hi), torch.full_like(logits, v), logits)
        del u
    if c["weight"]:
        w = torch.rand(n, generator=g, device="cuda") + 0.5
        s["weight"] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.1,
                                  torch.zeros_like(w), w) / n
    s["logits"] = _padded(logits, c["pad"])
    return s


def _legal_logits(s, logits):
    x = logits.float()
    return x if s["mask"] is None else torch.where(s["mask"], x, torch.full_like(x, -math.inf))


def _prepare_policy(c, g):
    n, a = c["rows"], c["actions"]
    s = _prepare_loss(c, g)
    x = _legal_logits(s, s["logits"])
    # actions drawn from the policy (the largest logit plus Gumbel noise)
    noise = torch.empty((n, a), device="cuda").exponential_(generator=g)
    act = torch.argmax(x - torch.log(noise), dim=1)
    del noise
    lse = torch.logsumexp(x, dim=1)
    logp = torch.gather(x, 1, act[:, None])[:, 0] - lse
    logp = torch.where(torch.isfinite(logp), logp, torch.zeros_like(logp))

    def near(scale):
        return logp + scale * torch.randn(n, generator=g, device="cuda")

    s["old_logp"], s["ref_logp"], s["ref_logits"] = near(0.15), None, None
    if c["kl"] == "sampled":
        s["ref_logp"] = near(0.2)
    if c["kl"] == "full":
        y = s["logits"].float()
        y = y + 0.3 * torch.randn((n, a), generator=g, device="cuda")
        s["ref_logits"] = _padded(y.to(TYPES[c["dtype"]]), c["pad"])
    s["advantage"] = torch.randn(n, generator=g, device="cuda")
    # finished envs: no action
    none = 255 if c["ids"] == "uint8" else -1
    act = torch.where(torch.rand(n, generator=g, device="cuda") < 0.03,
                      torch.full_like(act, none), act)
    s["actions"] = act.to(getattr(torch, c["ids"]))
    return s


def _prepare_distill(c, g):
    n, a, k = c["rows"], c["actions"], c["top"]
    s = _prepare_loss(c, g)
    # the teacher's k best of its own logits, best first, some rows with fewer
    idx = torch.empty((n, k), dtype=torch.int32, device="cuda")
    val = torch.empty((n, k), device="cuda")
    step = max(1, (1 << 27) // a)
    for r in range(0, n, step):
        m = min(step, n - r)
        v, i = torch.topk(torch.randn((m, a), generator=g, device="cuda") * 2.0, k, dim=1)
        idx[r:r + m], val[r:r + m] = i.int(), v
    have = torch.where(torch.rand(n, generator=g, device="cuda") < 0.9, 1.0,
                       torch.rand(n, generator=g, device="cuda")) * k
    gone = torch.arange(k, device="cuda")[None, :] >= have[:, None]
    s["idx"], s["val"] = torch.where(gone, torch.full_like(idx, -1), idx), val
    return s


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(0x0BE8A70 + 7919 * seed)
    s = {"linear": _prepare_linear, "policy": _prepare_policy,
         "distill": _prepare_distill}[c["op"]](c, g)
    s["case"] = c
    return s


# ------------------------------------------------------- the library's calls

def _run_own(s):
    import paper_2106_07551_amd as M
    c = s["case"]
    if c["op"] == "linear":
        act = {"none": M.ACT_NONE, "relu": M.ACT_RELU, "gelu": M.ACT_GELU,
               "silu": M.ACT_SILU}[c["act"]]
        if c["way"] == "backward":
            return M.linear_backward(s["dy"], s["x"], s["w"], act=act, pre=s["pre"])
        if not c["train"]:
            return M.linear(s["x"], s["w"], s["bias"], act=act, residual=s["residual"])
        pre = torch.empty(_grouped(c, c["rows"], c["out"]), dtype=s["x"].dtype, device="cuda")
        y = M.linear(s["x"], s["w"], s["bias"], act=act, residual=s["residual"], pre=pre)
        return y, pre
    if c["op"] == "policy":
        return M.policy_loss(s["logits"], s["actions"], s["old_logp"], s["advantage"],
                             clip_low=CLIP_LOW, clip_high=CLIP_HIGH,
                             kl_coef=0.0 if c["kl"] == "none" else KL_COEF,
                             entropy_coef=ENTROPY_COEF, ref_logp=s["ref_logp"],
                             ref_logits=s["ref_logits"], mask=s["mask"], weight=s["weight"])
    return M.distill_loss(s["logits"], s["idx"], s["val"], temperature=c["temperature"],
                          mask=s["mask"], weight=s["weight"])


# ------------------------------------------------------------- plain forms

def _act(name, z):
    if name == "relu":
        return torch.clamp(z, min=0.0)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(name, z):
    if name == "relu":
        return (z > 0.0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + \
            z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    sig = 1.0 / (1.0 + torch.exp(-z))
    return sig * (1.0 + z * (1.0 - sig))


def _plain_linear(c, s):
    x, w, t = s["x"].float(), s["w"].float(), s["x"].dtype
    if c["way"] == "forward":
        z = torch.matmul(x, w.transpose(-1, -2))
        if s["bias"] is not None:
            z = z + s["bias"].unsqueeze(-2)
        y = _act(c["act"], z)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return (y.to(t), z.to(t)) if c["train"] else y.to(t)
    dz = s["dy"].float()
    if c["act"] != "none":
        dz = dz * _act_slope(c["act"], s["pre"].float())
    return (torch.matmul(dz, w).to(t), torch.matmul(dz.transpose(-1, -2), x).to(t),
            dz.sum(-2))


def _row_weights(s, n):
    return s["weight"] if s["weight"] is not None else \
        torch.full((n,), 1.0 / n, device="cuda")


def _softmax(x):
    """exp(x - max), its sum and the logarithms of the quotients of a row; a
    row that mask or data leave empty gets zeros."""
    m = torch.amax(x, dim=1, keepdim=True)
    m = torch.where(torch.isfinite(m), m, torch.zeros_like(m))
    e = torch.exp(x - m)
    z = e.sum(1, keepdim=True)
    z = torch.where(z > 0.0, z, torch.ones_like(z))
    return e / z, (x - m) - torch.log(z)


def _plain_policy(c, s):
    n, a = c["rows"], c["actions"]
    act = s["actions"].long()
    inside = (act >= 0) & (act < a)
    act = torch.where(inside, act, torch.zeros_like(act))
    if s["mask"] is not None:
        inside = inside & torch.gather(s["mask"], 1, act[:, None])[:, 0]
    w = _row_weights(s, n)
    counts = inside & (w != 0.0)
    p, logp = _softmax(_legal_logits(s, s["logits"]))
    lp = torch.gather(logp, 1, act[:, None])[:, 0]
    ratio = torch.exp(lp - s["old_logp"])
    adv = s["advantage"]
    s1, s2 = ratio * adv, torch.clamp(ratio, 1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * adv
    loss, slope = -torch.minimum(s1, s2), torch.where(s1 <= s2, -s1, torch.zeros_like(s1))
    some = p > 0.0
    zero = torch.zeros_like(p)
    ent = -torch.where(some, p * logp, zero).sum(1)
    loss = loss - ENTROPY_COEF * ent
    grad = torch.where(some, ENTROPY_COEF * p * (logp + ent[:, None]), zero)
    kl = torch.zeros_like(ent)
    if c["kl"] == "sampled":
        d = s["ref_logp"] - lp
        kl = torch.expm1(d) - d
        slope = slope - KL_COEF * torch.expm1(d)
    elif c["kl"] == "full":
        _, logq = _softmax(_legal_logits(s, s["ref_logits"]))
        gap = torch.where(some, logp - logq, zero)
        kl = (p * gap).sum(1)
        grad = grad + KL_COEF * p * (gap - kl[:, None])
    loss = loss + KL_COEF * kl
    grad = grad - slope[:, None] * p
    grad.scatter_add_(1, act[:, None], slope[:, None])
    grad = torch.where(counts[:, None], grad * w[:, None], zero)
    if s["mask"] is not None:
        grad = torch.where(s["mask"], grad, zero)
    stats = torch.stack([loss, lp, kl, ent])
    stats = torch.where(counts[None, :], stats, torch.zeros_like(stats))
    total = torch.where(counts, w * loss, torch.zeros_like(loss)).sum()
    return total.reshape(1), stats, grad.to(s["logits"].dtype)


def _plain_distill(c, s):
    n, a, T = c["rows"], c["actions"], c["temperature"]
    idx = s["idx"].long()
    live = (idx >= 0) & (idx < a)
    idx = torch.where(live, idx, torch.zeros_like(idx))
    if s["mask"] is not None:
        live = live & torch.gather(s["mask"], 1, idx)
    w = _row_weights(s, n)
    counts = live.any(1) & (w != 0.0)
    t, logt = _softmax(torch.where(live, s["val"] / T, torch.full_like(s["val"], -math.inf)))
    q, logq = _softmax(_legal_logits(s, s["logits"]) / T)
    zero = torch.zeros_like(t)
    loss = T * T * torch.where(t > 0.0, t * (logt - torch.gather(logq, 1, idx)), zero).sum(1)
    grad = T * q
    grad.scatter_add_(1, idx, torch.where(live, -T * t, zero))
    grad = torch.where(counts[:, None], grad * w[:, None], torch.zeros_like(grad))
    loss = torch.where(counts, loss, torch.zeros_like(loss))
    return (w * loss).sum().reshape(1), loss, grad.to(s["logits"].dtype)


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    return {"linear": _plain_linear, "policy": _plain_policy,
            "distill": _plain_distill}[c["op"]](c, state)


# ------------------------------------------------------------------- floors

def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "linear":
        g, m, k, n = c["groups"], c["rows"], c["in"], c["out"]
        if c["way"] == "forward":
            big = m * k + n * k + m * n * (1 + c["residual"] + c["train"])
            return {"bytes": g * (es * big + 4 * n * c["bias"]),
                    "flops": g * (2 * m * n * k + 4 * m * n)}
        big = 2 * m * k + 2 * n * k + m * n * (1 + (c["act"] != "none"))
        return {"bytes": g * (es * big + 4 * n), "flops": g * (4 * m * n * k + 4 * m * n)}
    n, a = c["rows"], c["actions"]
    size = 2 * es + c["mask"]
    if c["op"] == "policy":
        size += es * (c["kl"] == "full")
        row = {"uint8": 1, "int32": 4, "int64": 8}[c["ids"]] + 8 + 4 * (c["kl"] == "sampled") + \
            4 * c["weight"] + 16
        return {"bytes": n * (a * size + row) + 4, "flops": 20 * n * a}
    return {"bytes": n * (a * size + 8 * c["top"] + 4 * c["weight"] + 4) + 4,
            "flops": 8 * n * a}


# -------------------------------------------------- the definitions in 64 bits

def _exact_linear(c, s):
    x, w = s["x"].double(), s["w"].double()
    M, K, N, G = c["rows"], c["in"], c["out"], c["groups"]
    x, w = x.reshape(G, M, K), w.reshape(G, N, K)

    def phi(z):
        return torch.special.ndtr(z)

    out = []
    for i in range(G):
        if c["way"] == "forward":
            z = x[i] @ w[i].T.contiguous()
            if s["bias"] is not None:
                z += s["bias"].reshape(G, 1, N)[i].double()
            y = {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, 0.0 * z),
                 "gelu": lambda: z * phi(z), "silu": lambda: z * torch.sigmoid(z)}[c["act"]]()
            if s["residual"] is not None:
                y = y + s["residual"].reshape(G, M, N)[i].double()
            out.append((y, z) if c["train"] else (y,))
            continue
        dz = s["dy"].reshape(G, M, N)[i].double()
        if c["act"] != "none":
            z = s["pre"].reshape(G, M, N)[i].double()
            dz = dz * {"relu": lambda: torch.where(z > 0, 1.0, 0.0).double(),
                       "gelu": lambda: phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi),
                       "silu": lambda: torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))}[c["act"]]()
        out.append((dz @ w[i], dz.T.contiguous() @ x[i], dz.sum(0)))
    shaped = tuple(torch.stack(v) if G > 1 else v[0] for v in zip(*out))
    return shaped if len(shaped) > 1 else shaped[0]


def _log_probs(x, mask):
    """log softmax over the legal entries in 64 bits, -inf elsewhere."""
    x = x.double()
    if mask is not None:
        x = x.masked_fill(~mask, -math.inf)
    return x - torch.logsumexp(x, 1, keepdim=True)


def _exact_policy(c, s):
    n, a = c["rows"], c["actions"]
    act = s["actions"].long()
    ok = (act >= 0) & (act < a)
    act = act.clamp(0, a - 1)
    if s["mask"] is not None:
        ok &= s["mask"][torch.arange(n, device="cuda"), act]
    w = _row_weights(s, n).double()
    ok &= w != 0
    logp = _log_probs(s["logits"], s["mask"])
    p = torch.exp(logp)
    plain = torch.where(p > 0, logp, 0.0)
    lp = logp[torch.arange(n, device="cuda"), act]
    r, adv = torch.exp(lp - s["old_logp"].double()), s["advantage"].double()
    s1, s2 = r * adv, r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * adv
    ent = -(p * plain).sum(1)
    by_logp = torch.where(s1 <= s2, -s1, 0.0)         # d loss / d log p[action]
    kl = torch.zeros_like(ent)
    by_logit = ENTROPY_COEF * p * (plain + ent[:, None])
    if c["kl"] == "sampled":
        d = s["ref_logp"].double() - lp
        kl = torch.expm1(d) - d
        by_logp = by_logp - KL_COEF * torch.expm1(d)
    if c["kl"] == "full":
        gap = torch.where(p > 0, plain - _log_probs(s["ref_logits"], s["mask"]), 0.0)
        kl = (p * gap).sum(1)
        by_logit += KL_COEF * p * (gap - kl[:, None])
    loss = -torch.minimum(s1, s2) - ENTROPY_COEF * ent + KL_COEF * kl
    by_logit -= by_logp[:, None] * p
    by_logit[torch.arange(n, device="cuda"), act] += by_logp
    by_logit *= w[:, None]
    by_logit[~ok] = 0
    stats = torch.stack([loss, lp, kl, ent])
    stats[:, ~ok] = 0
    return (w * stats[0]).sum().reshape(1), stats, by_logit


def _exact_distill(c, s):
    n, a, T = c["rows"], c["actions"], c["temperature"]
    idx = s["idx"].long()
    live = (idx >= 0) & (idx < a)
    idx = idx.clamp(0, a - 1)
    if s["mask"] is not None:
        live &= s["mask"].gather(1, idx)
    w = _row_weights(s, n).double()
    ok = live.any(1) & (w != 0)
    logt = _log_probs(s["val"].double() / T, live)
    t = torch.where(live, torch.exp(logt), 0.0)
    t[~ok] = 0
    logq = _log_probs(s["logits"].double() / T, s["mask"])
    gap = torch.where(t > 0, logt - logq.gather(1, idx), 0.0)
    loss = T * T * (t * gap).sum(1)
    grad = T * torch.exp(logq)
    grad.scatter_add_(1, idx, -T * t)
    grad *= w[:, None]
    grad[~ok] = 0
    return (w * loss).sum().reshape(1), loss, grad


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "policy": _exact_policy,
            "distill": _exact_distill}[case["op"]](s["case"], s)

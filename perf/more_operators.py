"""Timed cases of what a learner runs around its losses: log probabilities of given
actions with entropy and top alternatives, and their gradient; dropout from the
library's random stream; layers of frozen policies held in 4 bits.

    listed()         the cases
    draw(rng)        another case of the same ranges
    prepare(case, s) the inputs a learner holds before the call
    run(state)       one pass: the library's operators where `own` is true, else
                     their plain form in elementary torch operations
    work(case)       bytes and operations one pass cannot do without
    exact(case, s)   the outputs in 64 bits, from the formulas

Formulas (sums over a row's legal entries):

  log probabilities  m = max x,  s = sum_j e^((x_j - m) / T),  p_j = e^((x_j - m) / T) / s,
                     l = (x_a - m) / T - ln s (0 where the action a is not a legal entry),
                     H = -sum_j p_j ln p_j,  stats = (l, H, m, ln s);
                     the `top` entries of largest x above -inf, ties to the lowest
                     index, and their ln p (-1 and 0 behind the last one);
                     a row without an entry above -inf: stats (0, 0, -inf, 0)
  backward           dx_j = (dl ([j = a] - p_j) - dH p_j (ln p_j + H)) / T
  dropout            y = x k / q + residual,  k = 1 where the value's 16 random bits are
                     at least t = rint(65536 p), q = 1 - t / 65536.  Value i of
                     the tensor takes bits 16 (i % 16) up of the Philox4x64-10 block with
                     counter (i / 16, step, 3 * 2^32 + layer, 0) and key (seed, 0)
  fp4                a weight is v s: v of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, s
                     the scale of `group` weights along the input,
                     s = bf16(max |w| / 6), v the nearest to w / s (ties to the even code)
  linear             y = act(x W^T + b) + residual, W in fp4

Codes and scales are laid out for 16x16x32 matrix products, outputs padded to 16 and
inputs to 128 with zeros: code (n, k) is a nibble (the lower one first) at
[n / 16][k / 128][(k % 32) / 8][n % 16][(k % 128) / 32][k % 8], scale (n, k / group) at
[n / 16][k / 128][n % 16][(k % 128) / group].
"""
import math

import torch

own = False

ACTS = ("none", "relu", "gelu", "silu")
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _named(name, c):
    return dict(c, name=name) if name else c


def _logp(name, way, dtype, rows, actions, *, top=0, temperature=1.0, ids="int32", mask=False,
          entropy=False, pad=0):
    """way "forward" or "backward" (entropy: with a gradient of the entropy too); top:
    listed alternatives; ids: type of the actions; pad: elements between a row's logits and
    the next row's."""
    return _named(name, {"op": "logp", "way": way, "dtype": dtype, "rows": rows,
                         "actions": actions, "top": top, "temperature": temperature, "ids": ids,
                         "mask": mask, "entropy": entropy, "pad": pad})


def _dropout(name, way, dtype, rows, cols, p, *, residual=False, pad=0):
    return _named(name, {"op": "dropout", "way": way, "dtype": dtype, "rows": rows, "cols": cols,
                         "p": p, "residual": residual, "pad": pad})


def _linear(name, dtype, rows, n_in, n_out, act, *, group=32, groups=1, bias=True, residual=False,
            pad=0):
    """group: weights that share a scale; groups: policies with weights of their own."""
    return _named(name, {"op": "linear", "dtype": dtype, "rows": rows, "in": n_in, "out": n_out,
                         "act": act, "group": group, "groups": groups, "bias": bias,
                         "residual": residual, "pad": pad})


def _pack(name, dtype, n_in, n_out, *, group=32, groups=1, pad=0):
    return _named(name, {"op": "pack", "dtype": dtype, "in": n_in, "out": n_out, "group": group,
                         "groups": groups, "pad": pad})


def listed():
    return [
        # a batch of 24 envs x 8 seats with legal-action masks, four alternatives: latency
        _logp("logp_small", "forward", "f32", 192, 18, top=4, mask=True),
        # one step of the 4v4 batch (16384 envs x 8 seats): the teachers' six best actions
        # for the distillation, and the log probability of the action taken
        _logp("logp_lists", "forward", "f32", 131072, 18, top=6, ids="uint8", mask=True),
        # a large action space (token-sized): a reference policy's log probabilities and
        # 64 best
        _logp("logp_wide", "forward", "bf16", 4096, 65536, top=64, ids="int64"),
        # three decisions over an odd large space with masks, eight alternatives
        _logp("logp_few_rows", "forward", "bf16", 3, 131071, top=8, mask=True),
        # gradient into a large odd action space, padded rows, entropy's too
        _logp("logp_wide_backward", "backward", "bf16", 2047, 50001, temperature=0.7,
              entropy=True, pad=7),
        # hidden values of the 4v4 game's policies over one step of the batch, residual added
        _dropout("dropout_team_residual", "forward", "bf16", 131072, 512, 0.1, residual=True),
        # odd sizes: rows that start at any element, gradient
        _dropout("dropout_odd_backward", "backward", "f32", 5003, 777, 0.25, pad=1),
        # one decision through a wide layer: the weights are the work
        _linear("fp4_one_row", "bf16", 1, 8192, 8192, "silu", residual=True),
        # a batch of decisions of a large network
        _linear("fp4_many_rows", "bf16", 192, 4096, 4096, "gelu", group=128),
        # five frozen fp32 policies with seven decisions each, odd sizes
        _linear("fp4_population", "f32", 7, 777, 333, "relu", groups=5, group=64, pad=1),
        # a large layer's weights into 4 bits and back, as a population takes them
        _pack("fp4_pack_large", "bf16", 4096, 8192),
        # 24 fp32 policies' first layers, odd sizes
        _pack("fp4_pack_population", "f32", 75, 250, group=64, groups=24, pad=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: as it falls, or a multiple of 8 or 64 as networks have them."""
    n = _log(rng, lo, hi)
    m = rng.choice([1, 8, 64, 64])
    return n if n < m else n // m * m


def draw(rng):
    """Another case of the ranges above: every direction, type, activation and scale
    group, one row to as many as fit the largest case's work."""
    op = rng.choice(["logp", "logp", "logp", "dropout", "dropout", "linear", "linear", "pack"])
    dtype = rng.choice(["f32", "bf16"])
    pad = rng.choice([0, 0, 0, 1, 8, 13])
    if op == "logp":
        while True:
            rows, actions = _log(rng, 1, 1048576), _log(rng, 2, 131072)
            if rows * actions <= 1 << 27:
                break
        ids = rng.choice(["uint8", "int32", "int64"]) if actions < 256 else \
            rng.choice(["int32", "int64"])
        mask, t = rng.random() < 0.4, rng.choice([1.0, 1.0, 0.7, 2.0])
        if rng.random() < 0.3:
            return _logp("", "backward", dtype, rows, actions, temperature=t, ids=ids, mask=mask,
                         entropy=rng.random() < 0.6, pad=pad)
        top = rng.choice([0, 1, 1]) * _log(rng, 1, 256)
        while rows * top > 1 << 24:
            top //= 2
        return _logp("", "forward", dtype, rows, actions, top=top, temperature=t, ids=ids,
                     mask=mask, pad=pad)
    if op == "dropout":
        while True:
            rows, cols = _log(rng, 1, 131072), _width(rng, 1, 16384)
            if rows * cols <= 1 << 26:
                break
        way = rng.choice(["forward", "backward"])
        return _dropout("", way, dtype, rows, cols, rng.choice([0.05, 0.1, 0.25, 0.5]),
                        residual=way == "forward" and rng.random() < 0.5, pad=pad)
    group = rng.choice([32, 64, 128])
    groups = rng.choice([1, 1, 1, rng.randint(2, 24)])
    while True:
        n_in, n_out = _width(rng, 3, 16384), _width(rng, 3, 16384)
        if groups * n_in * n_out <= 1 << (26 if op == "linear" else 25):
            break
    if op == "pack":
        return _pack("", dtype, n_in, n_out, group=group, groups=groups, pad=pad)
    rows = _log(rng, 1, 256)
    while groups * rows * n_in * n_out > 1 << 32:
        rows = (rows + 1) // 2
    return _linear("", dtype, rows, n_in, n_out, rng.choice(ACTS), group=group, groups=groups,
                   bias=rng.random() < 0.7, residual=rng.random() < 0.4, pad=pad)


# ------------------------------------------------------------------ inputs

def _padded(x, pad):
    """x as a view with `pad` more elements (of other data) behind each row."""
    if not pad:
        return x.contiguous()
    wide = torch.full(x.shape[:-1] + (x.shape[-1] + pad,), 7.0, dtype=x.dtype, device=x.device)
    wide[..., :x.shape[-1]] = x
    return wide[..., :x.shape[-1]]


def _prepare_logp(c, g):
    """Masked places hold what buffers hold there: numbers, the lowest number,
    infinities and NaN."""
    t, n, a = TYPES[c["dtype"]], c["rows"], c["actions"]
    logits = (torch.randn((n, a), generator=g, device="cuda") * 2.0).to(t)
    s = {"mask": None}
    if c["mask"]:
        u = torch.rand((n, a), generator=g, device="cuda")
        s["mask"] = u < 0.8
        s["mask"][torch.rand(n, generator=g, device="cuda") < 0.02] = False
        for lo, hi, v in ((0.8, 0.81, math.nan), (0.81, 0.82, math.inf), (0.82, 0.83, -math.inf),
                          (0.83, 0.84, torch.finfo(t).min)):
            logits = torch.where((u >= lo) & (u < hi), torch.full_like(logits, v), logits)
        del u
    s["logits"] = _padded(logits, c["pad"])
    del logits
    # actions drawn from the policy (the largest logit plus Gumbel noise); finished envs have none
    noise = torch.empty((n, a), device="cuda").exponential_(generator=g)
    act = torch.argmax(_legal(s) - torch.log(noise), dim=1)
    del noise
    act = torch.where(torch.rand(n, generator=g, device="cuda") < 0.03,
                      torch.full_like(act, 255 if c["ids"] == "uint8" else -1), act)
    s["actions"] = act.to(getattr(torch, c["ids"]))
    if c["way"] == "backward":
        s["stats"] = _plain_stats(c, s)[0]
        s["dlogp"] = torch.randn(n, generator=g, device="cuda") / n
        s["dentropy"] = torch.randn(n, generator=g, device="cuda") * 0.01 / n \
            if c["entropy"] else None
    return s


def _prepare_dropout(c, g):
    t, shape = TYPES[c["dtype"]], (c["rows"], c["cols"])
    s = {"x": _padded(torch.randn(shape, generator=g, device="cuda").to(t), c["pad"]),
         "residual": None}
    if c["residual"]:
        s["residual"] = torch.randn(shape, generator=g, device="cuda").to(t)
    step, layer, lo, hi = torch.randint(0, 1 << 31, (4,), generator=g, device="cuda").tolist()
    s["step"], s["layer"], s["seed"] = step, layer % 64, lo << 33 | hi
    return s


def _grouped(c, *shape):
    return (c["groups"],) + shape if c["groups"] > 1 else shape


def _prepare_linear(c, g):
    t, n_in, n_out = TYPES[c["dtype"]], c["in"], c["out"]

    def normal(scale, *shape, dtype=t):
        return (torch.randn(_grouped(c, *shape), generator=g, device="cuda") * scale).to(dtype)

    w = normal(n_in ** -0.5, n_out, n_in, dtype=torch.float32)
    s = {"x": _padded(normal(1.0, c["rows"], n_in), c["pad"])}
    s["codes"], s["scales"] = _quantize(w, c["group"])
    s["bias"] = normal(0.1, n_out, dtype=torch.float32) if c["bias"] else None
    s["residual"] = normal(1.0, c["rows"], n_out) if c["residual"] else None
    return s


def _prepare_pack(c, g):
    shape = _grouped(c, c["out"], c["in"])
    w = torch.randn(shape, generator=g, device="cuda") * c["in"] ** -0.5
    return {"w": _padded(w.to(TYPES[c["dtype"]]), c["pad"])}


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(0x5C0FE + 7919 * seed)
    s = {"logp": _prepare_logp, "dropout": _prepare_dropout, "linear": _prepare_linear,
         "pack": _prepare_pack}[c["op"]](c, g)
    s["case"] = c
    return s


# ------------------------------------------------------- the library's calls

def _run_own(s):
    import paper_2106_07551_amd as M
    c = s["case"]
    if c["op"] == "logp" and c["way"] == "backward":
        return M.log_probs_backward(s["logits"], s["actions"], s["stats"], s["dlogp"],
                                    s["dentropy"], temperature=c["temperature"], mask=s["mask"])
    if c["op"] == "logp":
        out = M.log_probs(s["logits"], s["actions"], top=c["top"], temperature=c["temperature"],
                          mask=s["mask"])
        return out if c["top"] else out[0]
    if c["op"] == "dropout" and c["way"] == "backward":
        return M.dropout_backward(s["x"], c["p"], s["seed"], s["step"], layer=s["layer"])
    if c["op"] == "dropout":
        return M.dropout(s["x"], c["p"], s["seed"], s["step"], layer=s["layer"],
                         residual=s["residual"])
    if c["op"] == "linear":
        act = {"none": M.ACT_NONE, "relu": M.ACT_RELU, "gelu": M.ACT_GELU,
               "silu": M.ACT_SILU}[c["act"]]
        return M.linear_fp4(s["x"], s["codes"], s["scales"], c["out"], s["bias"], act=act,
                            residual=s["residual"])
    codes, scales = M.quantize_fp4(s["w"], c["group"])
    return scales, M.dequantize_fp4(codes, scales, c["out"], c["in"], dtype=s["w"].dtype)


# ------------------------------------------------------------- plain forms

def _legal(s):
    x = s["logits"].float()
    return x if s["mask"] is None else torch.where(s["mask"], x, torch.full_like(x, -math.inf))


def _legal_actions(c, s):
    """The actions, and whether each is a legal entry."""
    act = s["actions"].long()
    inside = (act >= 0) & (act < c["actions"])
    act = torch.where(inside, act, torch.zeros_like(act))
    if s["mask"] is not None:
        inside = inside & torch.gather(s["mask"], 1, act[:, None])[:, 0]
    return act, inside


def _plain_stats(c, s):
    """(stats, ln p of every entry)"""
    x = _legal(s)
    m = torch.amax(x, dim=1)
    some = m > -math.inf
    zero = torch.zeros_like(m)
    d = (x - torch.where(some, m, zero)[:, None]) / c["temperature"]
    e = torch.exp(d)
    z = e.sum(1)
    z = torch.where(some, z, torch.ones_like(z))
    lns = torch.log(z)
    logp = d - lns[:, None]
    p = e / z[:, None]
    ent = -torch.where(p > 0.0, p * logp, torch.zeros_like(p)).sum(1)
    act, inside = _legal_actions(c, s)
    lp = torch.where(inside & some, torch.gather(logp, 1, act[:, None])[:, 0], zero)
    return torch.stack([lp, torch.where(some, ent, zero), m, torch.where(some, lns, zero)]), logp


def _plain_logp(c, s):
    n, a = c["rows"], c["actions"]
    if c["way"] == "forward":
        stats, logp = _plain_stats(c, s)
        if not c["top"]:
            return stats
        # whole numbers in the order of the values, ties by the index
        x = _legal(s)
        bits = (x + 0.0).view(torch.int32)
        bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = bits * (1 << 32) + ((1 << 31) - torch.arange(a, device="cuda"))[None, :]
        key = torch.where(x > -math.inf, key, torch.full_like(key, -(1 << 63)))
        k = min(c["top"], a)
        best, idx = torch.topk(key, k, dim=1)
        live = best > -(1 << 63)
        top_logp = torch.where(live, torch.gather(logp, 1, idx), torch.zeros_like(logp[:, :k]))
        idx = torch.where(live, idx, torch.full_like(idx, -1)).int()
        if k < c["top"]:
            idx = torch.cat([idx, torch.full((n, c["top"] - k), -1, dtype=torch.int32,
                                             device="cuda")], 1)
            top_logp = torch.cat([top_logp, torch.zeros((n, c["top"] - k), device="cuda")], 1)
        return stats, idx, top_logp
    _, ent, m, lns = s["stats"]
    act, inside = _legal_actions(c, s)
    some = m > -math.inf
    zero = torch.zeros_like(m)
    x = _legal(s)
    logp = (x - torch.where(some, m, zero)[:, None]) / c["temperature"] - lns[:, None]
    p = torch.exp(logp)
    dl = torch.where(inside, s["dlogp"], zero)
    grad = -dl[:, None] * p
    if s["dentropy"] is not None:
        bend = torch.where(p > 0.0, p * (logp + ent[:, None]), torch.zeros_like(p))
        grad = grad - s["dentropy"][:, None] * bend
    grad.scatter_add_(1, act[:, None], dl[:, None])
    live = (x > -math.inf) & some[:, None]
    grad = torch.where(live, grad / c["temperature"], torch.zeros_like(grad))
    return grad.to(s["logits"].dtype)


_LOW = 0xFFFFFFFF


def _signed(v):
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


def _mul_hilo(a, b):
    """Low and high half of the 128-bit product of unsigned 64-bit a (a tensor) and b."""
    a0, a1, b0, b1 = a & _LOW, (a >> 32) & _LOW, b & _LOW, b >> 32
    p = a0 * b0
    t = a0 * b1 + ((p >> 32) & _LOW)
    u = a1 * b0 + (t & _LOW)
    return (u << 32) | (p & _LOW), a1 * b1 + ((t >> 32) & _LOW) + ((u >> 32) & _LOW)


def _philox(block, step, layer, seed):
    """Philox4x64-10 blocks of counters (block, step, 3 * 2^32 + layer, 0), key (seed, 0)."""
    c = [block] + [torch.full_like(block, _signed(v)) for v in (step, (3 << 32) + layer, 0)]
    for r in range(10):
        k0, k1 = seed + r * 0x9E3779B97F4A7C15, r * 0xBB67AE8584CAA73B
        lo0, hi0 = _mul_hilo(c[0], 0xD2E7470EE14C6C93)
        lo1, hi1 = _mul_hilo(c[2], 0xCA5A826395121157)
        c = [hi1 ^ c[1] ^ _signed(k0), lo1, hi0 ^ c[3] ^ _signed(k1), lo0]
    return torch.stack(c, 1)


def _plain_dropout(c, s):
    rows, cols, t = c["rows"], c["cols"], round(65536 * c["p"])
    blocks = torch.arange((rows * cols + 15) // 16, device="cuda")
    words = _philox(blocks, s["step"], s["layer"], s["seed"])
    bits = torch.stack([(words >> (16 * i)) & 0xFFFF for i in range(4)], 2).reshape(-1)
    keep = (bits[:rows * cols] >= t).reshape(rows, cols)
    x = s["x"].float()
    y = torch.where(keep, x * (65536.0 / (65536 - t)), torch.zeros_like(x))
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_BORDERS = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True),
            (5.0, False))   # (between two values, whether it belongs to the upper one)


def _quantize(w, group):
    """(codes, scales) of w [..][out][in] in the layout above."""
    lead, (n, k) = w.shape[:-2], w.shape[-2:]
    nt, ch = (n + 15) // 16, (k + 127) // 128
    full = torch.zeros(lead + (nt * 16, ch * 128), device=w.device)
    full[..., :n, :k] = w
    parts = full.reshape(lead + (nt * 16, ch * 128 // group, group))
    scale = (parts.abs().amax(-1) / 6.0).bfloat16()
    s, mag = scale.float()[..., None], parts.abs()
    code = torch.zeros_like(mag, dtype=torch.uint8)
    for border, up in _BORDERS:
        at = s * border
        code += (mag >= at) if up else (mag > at)
    code = torch.where(s > 0.0, code, torch.zeros_like(code))
    code += 8 * ((parts < 0.0) & (code > 0)).to(torch.uint8)
    code = code.reshape((-1, nt, 16, ch, 4, 4, 4, 2)).permute(0, 1, 3, 5, 2, 4, 6, 7)
    codes = (code[..., 0] | (code[..., 1] << 4)).reshape(lead + (nt, ch, 64, 16))
    scales = scale.reshape((-1, nt, 16, ch, 128 // group)).transpose(2, 3)
    return codes, scales.reshape(lead + (nt, ch, 16, 128 // group)).contiguous()


def _dequantize(codes, scales, n, k):
    """The weights that codes and scales stand for, fp32."""
    lead, (nt, ch) = codes.shape[:-4], codes.shape[-4:-2]
    code = torch.stack([codes & 15, codes >> 4], -1).reshape((-1, nt, ch, 4, 16, 4, 8))
    code = code.permute(0, 1, 4, 2, 5, 3, 6).reshape(lead + (nt * 16, ch * 128)).long()
    v = torch.tensor(_VALUES + tuple(-x for x in _VALUES), device=codes.device)[code]
    per = scales.shape[-1]
    s = scales.float().reshape((-1, nt, ch, 16, per)).transpose(2, 3)
    s = s.reshape(lead + (nt * 16, ch * per, 1))
    v = v.reshape(lead + (nt * 16, ch * per, 128 // per)) * s
    return v.reshape(lead + (nt * 16, ch * 128))[..., :n, :k]


def _act(name, z):
    if name == "relu":
        return torch.clamp(z, min=0.0)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _plain_linear(c, s):
    w = _dequantize(s["codes"], s["scales"], c["out"], c["in"])
    z = torch.matmul(s["x"].float(), w.transpose(-1, -2))
    if s["bias"] is not None:
        z = z + s["bias"].unsqueeze(-2)
    y = _act(c["act"], z)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _plain_pack(c, s):
    codes, scales = _quantize(s["w"].float(), c["group"])
    return scales, _dequantize(codes, scales, c["out"], c["in"]).to(s["w"].dtype)


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    return {"logp": _plain_logp, "dropout": _plain_dropout, "linear": _plain_linear,
            "pack": _plain_pack}[c["op"]](c, state)


# ------------------------------------------------------------------- floors

def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "logp":
        n, a = c["rows"], c["actions"]
        ids = {"uint8": 1, "int32": 4, "int64": 8}[c["ids"]]
        if c["way"] == "forward":
            return {"bytes": n * (a * (es + c["mask"]) + ids + 16 + 8 * c["top"]),
                    "flops": 5 * n * a}
        return {"bytes": n * (a * (2 * es + c["mask"]) + ids + 20 + 4 * c["entropy"]),
                "flops": 6 * n * a}
    if c["op"] == "dropout":
        n = c["rows"] * c["cols"]
        return {"bytes": es * n * (2 + c["residual"]), "flops": 3 * n}
    g, k, n = c["groups"], c["in"], c["out"]
    held = g * (n * k // 2 + 2 * n * ((k + c["group"] - 1) // c["group"]))
    if c["op"] == "pack":   # codes and scales written, and read again
        return {"bytes": 2 * g * es * n * k + 2 * held, "flops": 4 * g * n * k}
    m = c["rows"]
    return {"bytes": held + g * (es * (m * k + m * n * (1 + c["residual"])) + 4 * n * c["bias"]),
            "flops": g * (2 * m * n * k + 4 * m * n)}


# -------------------------------------------------- the definitions in 64 bits

def _exact_logp(c, s):
    n, a, T, k = c["rows"], c["actions"], c["temperature"], min(c["top"], c["actions"])
    out = []
    step = max(1, (1 << 26) // a)
    for r in range(0, n, step):   # rows apart: 64 bits of the largest case at once are 2 GiB
        x = s["logits"][r:r + step].double()
        legal = torch.ones_like(x, dtype=torch.bool) if s["mask"] is None else \
            s["mask"][r:r + step]
        x = x.masked_fill(~legal, -math.inf)
        act = s["actions"][r:r + step].long()
        ok = (act >= 0) & (act < a)
        rows = torch.arange(x.shape[0], device="cuda")
        act = act.clamp(0, a - 1)
        ok &= legal[rows, act]
        some = (x > -math.inf).any(1)
        logp = torch.where(some[:, None], torch.log_softmax(x / T, 1), -math.inf)
        p = logp.exp()
        ent = -(torch.special.xlogy(p, p)).sum(1)
        if c["way"] == "backward":
            dl = torch.where(ok, s["dlogp"][r:r + step].double(), 0.0)
            grad = -p * dl[:, None]
            grad[rows, act] += dl
            if s["dentropy"] is not None:
                grad -= s["dentropy"][r:r + step].double()[:, None] * (
                    torch.special.xlogy(p, p) + p * ent[:, None])
            grad[~some] = 0
            grad[x == -math.inf] = 0
            out.append((grad / T,))
            continue
        m = x.amax(1)
        lns = torch.where(some, torch.logsumexp(x / T, 1) - m / T, 0.0)
        lp = torch.where(ok & some, logp[rows, act], 0.0)
        stats = torch.stack([lp, torch.where(some, ent, 0.0), m, lns])
        if not k:
            out.append((stats.T,))
            continue
        val, idx = torch.sort(x, dim=1, descending=True, stable=True)
        val, idx = val[:, :k], idx[:, :k]
        none = val == -math.inf
        best = logp.gather(1, idx).masked_fill(none, 0.0)
        idx = idx.masked_fill(none, -1).int()
        more = c["top"] - k
        out.append((stats.T, torch.nn.functional.pad(idx, (0, more), value=-1),
                    torch.nn.functional.pad(best, (0, more))))
    got = [torch.cat(v) for v in zip(*out)]
    if c["way"] == "backward":
        return got[0]
    got[0] = got[0].T.contiguous()
    return tuple(got) if c["top"] else got[0]


def _exact_dropout(c, s):
    import numpy as np
    n, t = c["rows"] * c["cols"], round(65536 * c["p"])
    # numpy's generator steps its counter before each block
    at = (s["step"] << 64) + (((3 << 32) + s["layer"]) << 128) - 1
    words = np.random.Philox(counter=at, key=s["seed"]).random_raw((n + 15) // 16 * 4)
    bits = torch.from_numpy(words.astype("<u8").view("<u2")[:n].astype(np.int32)).cuda()
    keep = (bits >= t).reshape(c["rows"], c["cols"])
    y = torch.where(keep, s["x"].double() / (1.0 - t / 65536.0), 0.0)
    return y if s["residual"] is None else y + s["residual"].double()


def _exact_weights(codes, scales, n, k):
    """Weight by weight: where code and scale of (n, k) lie."""
    table = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float64, device="cuda") / 2
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(k, device="cuda")[None, :]
    byte = codes[i // 16, j // 128, j % 32 // 8 * 16 + i % 16, j % 128 // 32 * 4 + j % 8 // 2]
    nibble = (byte.long() >> (4 * (j % 2))) & 15
    group = 128 // scales.shape[-1]
    v = table[nibble & 7] * (1 - 2 * (nibble >> 3))
    return v * scales[i // 16, j // 128, i % 16, j % 128 // group].double()


def _exact_linear(c, s):
    G, out = c["groups"], []

    def of(name, i):
        t = s[name]
        return t if G == 1 or t is None else t[i]

    for i in range(G):
        w = _exact_weights(of("codes", i), of("scales", i), c["out"], c["in"])
        z = of("x", i).double() @ w.T.contiguous()
        if c["bias"]:
            z += of("bias", i).double()
        y = {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, 0.0 * z),
             "gelu": lambda: z * torch.special.ndtr(z), "silu": lambda: z * torch.sigmoid(z)
             }[c["act"]]()
        out.append(y + of("residual", i).double() if c["residual"] else y)
    return torch.stack(out) if G > 1 else out[0]


def _exact_pack(c, s):
    """Scales from the largest magnitudes, weights from the distances to every value."""
    G, n, k, group = c["groups"], c["out"], c["in"], c["group"]
    nt, ch, per = (n + 15) // 16, (k + 127) // 128, 128 // group
    w = s["w"].double().reshape(G, n, k)
    w = torch.nn.functional.pad(w, (0, ch * 128 - k, 0, nt * 16 - n))
    w = w.reshape(G, nt * 16, ch * per, group)
    scale = (w.abs().amax(-1) / 6).float().bfloat16().double()
    ratio = w.abs() / torch.where(scale > 0, scale, 1.0)[..., None]
    best = torch.zeros_like(ratio)
    for even in (1, 0):   # values of even codes last: they win ties
        for v in _VALUES[even::2]:
            near, now = (ratio - v).abs(), (ratio - best).abs()
            best = torch.where(near < now if even else near <= now, v, best)
    best = torch.where(scale[..., None] > 0, best, 0.0)
    val = (best * torch.sign(w) * scale[..., None]).reshape(G, nt * 16, ch * 128)[:, :n, :k]
    scale = scale.reshape(G, nt, 16, ch, per).transpose(2, 3)
    if G == 1:
        val, scale = val[0], scale[0]
    return scale.contiguous(), val


def exact(case, seed):
    s = prepare(case, seed)
    return {"logp": _exact_logp, "dropout": _exact_dropout, "linear": _exact_linear,
            "pack": _exact_pack}[case["op"]](s["case"], s)

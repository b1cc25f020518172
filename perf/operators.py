"""The operators around a trained network's layers, as cases that can be timed: layer norm, log probabilities of given
classes (tokens) with entropy and top alternatives, and the AdamW step.

A case names an operator and a direction, its sizes, layout and types:

  norm_fwd, norm_bwd   y = (x - mean) / sqrt(var + eps) * weight + bias over the C channels of every one of B x N positions;
                       gradients of x, weight and bias from the saved mean and 1 / sqrt(var + eps)
  logp_fwd, logp_bwd   over the C scores of a position: log softmax at its target, entropy, log of the sum of exponentials,
                       the `top` best log probabilities with their classes (ties: the lower class first); the gradient of the
                       scores from those of the log probability and the entropy.  A negative target: the position is ignored
  adamw                decoupled weight decay and Adam over a list of tensors, states in 32 bits, or in 8: e4m3 values under one
                       power of two for every 32, stored by stochastic rounding (the second moment by its square root)

Tensors are [B,N,C] ("bnc") or [B,C,N] ("bcn"), in fp32, bf16 or fp16; statistics and log probabilities are fp32.
`run` computes the plain form from elementary torch operations, in 32 bits, or, where `own` is set, calls this library.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
BETAS, ADAM_EPS, LR, DECAY, DONE = (0.9, 0.999), 1e-8, 1e-3, 0.1, 9
M32 = 0xFFFFFFFF


# ---- cases -------------------------------------------------------------------------------------------------------------

def _norm(op, layout, dtype, B, N, C, wtype="f32", name=None):
    c = dict(op=op, layout=layout, dtype=dtype, wtype=wtype, B=B, N=N, C=C)
    return dict(c, name=name) if name else c


def _logp(op, layout, dtype, B, N, C, top=0, row=0, ignored=0.0, entropy=True, name=None):
    c = dict(op=op, layout=layout, dtype=dtype, B=B, N=N, C=C, top=top, row=max(row, C), ignored=ignored, entropy=entropy)
    return dict(c, name=name) if name else c


def _adamw(kind, layers, width, ptype, gtype, bits, copy=False, name=None):
    c = dict(op="adamw", kind=kind, layers=layers, width=width, ptype=ptype, gtype=gtype, bits=bits, copy=copy)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of a serving step: nothing but latency
        _norm("norm_fwd", "bnc", "bf16", 1, 1, 4096, "bf16", name="norm_fwd_token_4096"),
        # every point of a scanned room, behind a 128-channel layer
        _norm("norm_fwd", "bnc", "f32", 1, 1_000_000, 128, name="norm_fwd_room1m_128"),
        # a batch of object scans in the paper's channel-major form, backward
        _norm("norm_bwd", "bcn", "f32", 8, 4096, 64, name="norm_bwd_8x4k_64_bcn"),
        # a training step's tokens at a wide layer, an odd number of them, backward
        _norm("norm_bwd", "bnc", "bf16", 4, 2047, 5120, "bf16", name="norm_bwd_8k_5120"),
        # one generated token over a large vocabulary, with the alternatives that a service shows
        _logp("logp_fwd", "bnc", "bf16", 1, 1, 131072, top=20, name="logp_fwd_token_131072"),
        # class scores of every point of a room: 13 classes, some points without a label
        _logp("logp_fwd", "bnc", "f32", 1, 1_000_000, 13, top=3, ignored=0.2, name="logp_fwd_room1m_13"),
        # a batch of sampled answers under the model: a vocabulary whose rows are padded, prompts ignored
        _logp("logp_fwd", "bnc", "bf16", 2, 1023, 129_280, top=8, row=129_536, ignored=0.1, name="logp_fwd_2k_129280"),
        # its gradient, with an entropy bonus
        _logp("logp_bwd", "bnc", "bf16", 2, 1023, 129_280, row=129_536, ignored=0.1, name="logp_bwd_2k_129280"),
        # the loss of a training batch of 16 chunks of 128 x 128 points, channel-major
        _logp("logp_bwd", "bcn", "f32", 16, 16_384, 13, ignored=0.2, entropy=False, name="logp_bwd_16x16k_13_bcn"),
        # the parameters of a six-stage point network: theta, bias and norms, many of them small
        _adamw("flexconv", 6, 20, "f32", "f32", 32, name="adamw_network_32bit"),
        # a language model's parameters with a master copy: fp32 weights, bf16 gradients, bf16 copy written along
        _adamw("dense", 16, 1152, "f32", "bf16", 32, copy=True, name="adamw_master_32bit"),
        # the same kind of model, larger, in bf16 throughout with 8-bit states
        _adamw("dense", 24, 1408, "bf16", "bf16", 8, name="adamw_8bit"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm_fwd", "norm_bwd", "logp_fwd", "logp_bwd", "adamw"))
    if op == "adamw":
        kind = rng.choice(("flexconv", "dense"))
        ptype = rng.choice(("f32", "bf16", "f16"))
        layers = rng.randint(1, 6) if kind == "flexconv" else rng.randint(1, 20)
        width = _log(rng, 3, 40) if kind == "flexconv" else _log(rng, 33, 1200)
        return _adamw(kind, layers, width, ptype, rng.choice(("f32", ptype)), rng.choice((32, 8)), ptype == "f32" and rng.random() < 0.3)
    layout = rng.choice(("bnc", "bnc", "bcn"))
    dtype = rng.choice(("f32", "bf16", "f16"))
    B = rng.choice((1, 1, 2, 3, 8))
    if op.startswith("norm"):
        C = _log(rng, 8, 512 if layout == "bcn" else 16_000)
        N = _log(rng, 1, max(2, min(1_000_000, 120_000_000 // C) // B))
        return _norm(op, layout, dtype, B, N, C, rng.choice(("f32", dtype)))
    C = _log(rng, 2, 64 if layout == "bcn" else 200_000)
    N = _log(rng, 1, max(2, min(1_000_000, 250_000_000 // C) // B))
    top = min(C, rng.choice((0, 1, 3, 8, 20))) if op == "logp_fwd" else 0
    row = C + rng.choice((0, 0, 3, 64)) if layout == "bnc" else C
    return _logp(op, layout, dtype, B, N, C, top, row, rng.choice((0.0, 0.1, 0.5)), rng.random() < 0.7)


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _shape(c):
    return (c["B"], c["C"], c["N"]) if c["layout"] == "bcn" else (c["B"], c["N"], c["C"])


def _dim(c):
    return 1 if c["layout"] == "bcn" else 2


def _pshape(c):
    """A vector over the channels, as it multiplies a tensor of the case."""
    return (1, c["C"], 1) if c["layout"] == "bcn" else (1, 1, c["C"])


def _sizes(c):
    """(element count, decayed) of every parameter tensor."""
    w, got = c["width"], []
    for i in range(c["layers"]):
        if c["kind"] == "flexconv":  # theta [3,d,d], bias [d,d], a norm's weight and bias; the width doubles from stage to stage
            d = w << i
            got += [(3 * d * d, True), (d * d, True), (d, False), (d, False)]
        else:
            got += [(w * w, True), (4 * w * w, True), (4 * w, False), (4 * w * w, True), (w, False), (w, False)]
    return got


def _places(c):
    """(begin, element count, decay) of every tensor in a flat buffer, each on a multiple of 64 elements, and the buffer's size."""
    at, got = 0, []
    for n, decayed in _sizes(c):
        got.append((at, n, DECAY if decayed else 0.0))
        at += -(-n // 64) * 64
    return got, at


def _adamw_state(c, g):
    places, total = _places(c)
    live = torch.zeros(total, dtype=torch.bool, device="cuda")
    for at, n, _ in places:
        live[at:at + n] = True
    s = {"case": c, "places": places, "t": DONE}

    def flat(scale, dtype):
        return (torch.randn(total, device="cuda", generator=g) * scale).mul_(live).to(dtype)

    s["p"] = flat(0.02, DTYPE[c["ptype"]])
    s["g"] = flat(1e-3, DTYPE[c["gtype"]])
    m, v = flat(3e-4, torch.float32), flat(1e-3, torch.float32).square_()
    if c["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        for name, x in (("m", m), ("v", v.sqrt_())):
            x = x.view(-1, 32)
            e = _exponent(x.abs().amax(1)).sub_(7).clamp_(-100, 120)  # the largest magnitude comes to [128, 256)
            s[name] = (x * _power(-e)[:, None]).to(torch.float8_e4m3fn).view(-1)
            s[name + "_scale"] = (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
    if c["copy"]:
        s["copy"] = s["p"].to(torch.bfloat16)
    for k in ("p", "g", "m", "v", "copy"):
        if k in s:
            s[k + "_list"] = [s[k][at:at + n] for at, n, _ in places]
    for k in ("m_scale", "v_scale"):
        if k in s:
            s[k + "_list"] = [s[k][at // 32:at // 32 + -(-n // 32)] for at, n, _ in places]
    s["decay"] = [d for _, _, d in places]
    s["lr"] = LR
    s["clip"] = torch.full((1,), 0.75, device="cuda")
    s["seed"] = 1234
    return s


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = DTYPE.get(c.get("dtype"))

    def normal(shape, scale=1.0, shift=0.0, dtype=torch.float32):
        return torch.randn(shape, device="cuda", generator=g).mul_(scale).add_(shift).to(dtype)

    if c["op"] == "adamw":
        s = _adamw_state(c, g)
        if own:
            import paper_1803_07289_amd as fx
            s["fx"] = fx
            s["plan"] = fx.flexadamw_plan_build(s["p_list"], s["m_list"], s["v_list"], s.get("m_scale_list"), s.get("v_scale_list"),
                                                s.get("copy_list"), weight_decay=s["decay"], betas=BETAS, eps=ADAM_EPS,
                                                steps=DONE, seed=s["seed"])
        return s
    s = {"case": c}
    if own:
        import paper_1803_07289_amd as fx
        s["fx"] = fx
    if c["op"].startswith("norm"):
        s["x"] = normal(_shape(c), 1.5, 0.5, dt)
        s["w"], s["b"] = normal(c["C"], 0.1, 1.0, DTYPE[c["wtype"]]), normal(c["C"], 0.1, 0.0, DTYPE[c["wtype"]])
        if c["op"] == "norm_bwd":
            x = s["x"].float()
            s["mean"] = x.mean(_dim(c))
            x = x.sub_(s["mean"].unsqueeze(_dim(c))).square_()
            s["rstd"] = torch.rsqrt(x.mean(_dim(c)) + EPS)
            s["gy"] = normal(_shape(c), 0.5, 0.0, dt)
        return s
    B, N, C = c["B"], c["N"], c["C"]
    if c["layout"] == "bcn":
        s["x"] = normal((B, C, N), 2.5, 0.0, dt)
    else:  # rows of c["row"] scores, of which the first C are classes
        s["x"] = normal((B, N, c["row"]), 2.5, 0.0, dt)[:, :, :C]
    t = torch.randint(0, C, (B, N), device="cuda", generator=g, dtype=torch.int32)
    off = torch.rand((B, N), device="cuda", generator=g) < c["ignored"]
    off[:, 0] = False
    s["t"] = torch.where(off, -1, t).to(torch.int32)
    if c["op"] == "logp_bwd":
        x = s["x"].float()
        s["lse"] = torch.logsumexp(x, _dim(c))
        x = x.sub_(s["lse"].unsqueeze(_dim(c)))
        s["h"] = -(x.exp().mul_(x)).sum(_dim(c))
        del x
        keep = (s["t"] >= 0).float()
        s["lse"], s["h"] = s["lse"] * keep, s["h"] * keep
        s["gl"] = normal((B, N), 1.0)
        s["gh"] = normal((B, N), 0.01) if c["entropy"] else None
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------------

def _norm_fwd(s, c):
    d, x = _dim(c), s["x"].float()
    mean = x.mean(d, keepdim=True)
    x = x - mean
    rstd = torch.rsqrt((x * x).mean(d, keepdim=True) + EPS)
    y = x * rstd * s["w"].float().view(_pshape(c)) + s["b"].float().view(_pshape(c))
    return y.to(s["x"].dtype), mean.squeeze(d), rstd.squeeze(d)


def _norm_bwd(s, c):
    d, rows = _dim(c), (0, 2) if c["layout"] == "bcn" else (0, 1)
    rstd, gy = s["rstd"].unsqueeze(d), s["gy"].float()
    xh = (s["x"].float() - s["mean"].unsqueeze(d)) * rstd
    wg = gy * s["w"].float().view(_pshape(c))
    gx = (wg - wg.mean(d, keepdim=True) - xh * (wg * xh).mean(d, keepdim=True)) * rstd
    wt = s["w"].dtype
    return gx.to(s["x"].dtype), (gy * xh).sum(rows).to(wt), gy.sum(rows).to(wt)


def _logp_fwd(s, c):
    d, x, t = _dim(c), s["x"].float(), s["t"]
    on = t >= 0
    m = x.amax(d, keepdim=True)
    z = x - m
    e = z.exp()
    total = e.sum(d, keepdim=True)
    log_total = total.log()
    h = log_total - (e * z).sum(d, keepdim=True) / total
    at = t.clamp(min=0).long().unsqueeze(d)
    logp = z.gather(d, at) - log_total
    zero = torch.zeros_like(m.squeeze(d))
    got = [torch.where(on, v.squeeze(d), zero) for v in (logp, h, m + log_total)]
    if not c["top"]:
        return got
    best, which = torch.sort(z, dim=d, descending=True, stable=True)
    best, which = best.narrow(d, 0, c["top"]) - log_total, which.narrow(d, 0, c["top"]).int()
    on = on.unsqueeze(d)
    return got + [torch.where(on, best, -math.inf), torch.where(on, which, -1)]


def _logp_bwd(s, c):
    d, t = _dim(c), s["t"]
    lp = s["x"].float() - s["lse"].unsqueeze(d)
    p = lp.exp()
    gl = s["gl"].unsqueeze(d)
    gx = -(p * gl)
    if s["gh"] is not None:
        gx = gx - p * (lp + s["h"].unsqueeze(d)) * s["gh"].unsqueeze(d)
    gx = gx.scatter_add(d, t.clamp(min=0).long().unsqueeze(d), gl)
    return torch.where((t >= 0).unsqueeze(d), gx, 0.0).to(s["x"].dtype)


def _mix(x):
    """32 well-mixed bits of a 32-bit number: two rounds of shift and multiplication (the fractions of sqrt 2 and sqrt 3)."""
    x = (x ^ (x >> 16)) * 0x6A09E667 & M32
    x = (x ^ (x >> 15)) * 0xBB67AE85 & M32
    return x ^ (x >> 16)


def _noise(n, key):
    """Two numbers in [0,1), in steps of 2^-16, for each of n elements of a tensor in a step."""
    x = _mix(torch.arange(key, key + n, dtype=torch.int64, device="cuda") & M32)
    return (x & 0xFFFF).float() * 2.0 ** -16, (x >> 16).float() * 2.0 ** -16


def _power(e):
    return (e + 127 << 23).view(torch.float32)


def _exponent(x):
    return (x.view(torch.int32) >> 23 & 0xFF) - 127


def _blocks(x):
    """x [n] as rows of 32, the last one filled up with zeros."""
    return torch.nn.functional.pad(x, (0, -x.numel() % 32)).view(-1, 32)


def _block_scale(x):
    """The exponent of each row's power of two: its largest magnitude comes to at most 448, the largest e4m3 value."""
    bits = x.amax(1).view(torch.int32)
    return ((bits >> 23) - 135 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(-100, 120)


def _store(codes, scale, steps, ey, e, negative, n):
    code = ((ey + 6 << 3) + steps.int()).clamp(max=126) | negative.int() << 7
    codes.copy_(code.view(-1)[:n].to(torch.uint8).view(torch.float8_e4m3fn))
    scale.copy_((e + 127).to(torch.uint8).view(torch.float8_e8m0fnu))


def _store_first(m, r, codes, scale):
    n, m, r = m.numel(), _blocks(m), _blocks(r)
    e = _block_scale(m.abs())
    y = m.abs() * _power(-e)[:, None]
    ey = _exponent(y).clamp(min=-6)
    _store(codes, scale, torch.floor(y * _power(3 - ey) + r), ey, e, m.view(torch.int32) < 0, n)


def _store_second(v, root, r, codes, scale):
    """The root's two nearest values, chosen between so that the square comes out as v in the mean; one above zero stays above zero."""
    n, v, root, r = v.numel(), _blocks(v), _blocks(root), _blocks(r)
    e = _block_scale(root)
    y = root * _power(-e)[:, None]
    ey = _exponent(y).clamp(min=-6)
    f = _power(3 - ey)
    steps = torch.floor(y * f)
    f = f * _power(-e)[:, None]
    w = v * f * f
    steps = steps + (r * (2 * steps + 1) < w - steps * steps).float()
    steps = torch.where(v > 0, steps.clamp(min=1), steps)
    _store(codes, scale, steps, ey, e, torch.zeros_like(v), n)


def _widen(codes, scale):
    return codes.float() * scale.float().repeat_interleave(32)[:codes.numel()]


def _adamw_32(s, c):
    t, (b1, b2) = s["t"], BETAS
    p, clip = [x.float() for x in s["p_list"]], s["clip"]
    g = [x.float() * clip for x in s["g_list"]]
    torch._foreach_mul_(s["m_list"], b1)
    torch._foreach_add_(s["m_list"], torch._foreach_mul(g, 1 - b1))
    torch._foreach_mul_(s["v_list"], b2)
    torch._foreach_add_(s["v_list"], torch._foreach_mul(torch._foreach_mul(g, g), 1 - b2))
    under = torch._foreach_sqrt(s["v_list"])
    torch._foreach_mul_(under, 1 / math.sqrt(1 - b2 ** t))
    torch._foreach_add_(under, ADAM_EPS)
    by = torch._foreach_div(s["m_list"], under)
    p = torch._foreach_mul(p, [1 - s["lr"] * d for d in s["decay"]])
    torch._foreach_sub_(p, torch._foreach_mul(by, s["lr"] / (1 - b1 ** t)))
    torch._foreach_copy_(s["p_list"], p)
    if c["copy"]:
        torch._foreach_copy_(s["copy_list"], p)


def _adamw_8(s, k):
    t, (b1, b2) = s["t"], BETAS
    p, codes, codes2, scale, scale2 = (s[x + "_list"][k] for x in ("p", "m", "v", "m_scale", "v_scale"))
    g = s["g_list"][k].float() * s["clip"]
    m = _widen(codes, scale) * b1 + g * (1 - b1)
    root = _widen(codes2, scale2)
    v = root * root * b2 + g * g * (1 - b2)
    root = v.sqrt()
    under = root * (1 / math.sqrt(1 - b2 ** t)) + ADAM_EPS
    new = p.float() * (1 - s["lr"] * s["decay"][k]) - m / under * (s["lr"] / (1 - b1 ** t))
    p.copy_(new)
    if "copy" in s:
        s["copy_list"][k].copy_(new)
    r, r2 = _noise(p.numel(), _mix(_mix(s["seed"] + t & M32) + k & M32))
    _store_first(m, r, codes, scale)
    _store_second(v, root, r2, codes2, scale2)


def _adamw_run(s, c):
    s["t"] += 1
    if c["bits"] == 32:
        _adamw_32(s, c)
    else:
        [_adamw_8(s, k) for k in range(len(s["places"]))]


def _adamw_outputs(s):
    return {k: s[k] for k in ("p", "m", "v", "m_scale", "v_scale", "copy") if k in s}


def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if not own:
        if op == "adamw":
            _adamw_run(s, c)
            return _adamw_outputs(s)
        return {"norm_fwd": _norm_fwd, "norm_bwd": _norm_bwd, "logp_fwd": _logp_fwd, "logp_bwd": _logp_bwd}[op](s, c)
    fx = s["fx"]
    if op == "adamw":
        fx.flexadamw_step(s["plan"], s["g_list"], s["lr"], grad_scale=s["clip"])
        return _adamw_outputs(s)
    if op == "norm_fwd":
        return fx.flexnorm_fwd(s["x"], s["w"], s["b"], eps=EPS, layout=c["layout"])
    if op == "norm_bwd":
        return fx.flexnorm_bwd(s["x"], s["w"], s["gy"], s["mean"], s["rstd"], layout=c["layout"])
    if op == "logp_fwd":
        return [v for v in fx.flexlogp_fwd(s["x"], s["t"], top=c["top"], layout=c["layout"]) if v is not None]
    return fx.flexlogp_bwd(s["x"], s["t"], s["lse"], s["h"], s["gl"], s["gh"], layout=c["layout"])


# ---- work and exact values ---------------------------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "adamw":
        n = sum(k for k, _ in _sizes(c))
        state = 16 if c["bits"] == 32 else 4 + 4 / 32
        return {"bytes": n * (2 * BYTES[c["ptype"]] + BYTES[c["gtype"]] + state + (2 if c["copy"] else 0)), "flops": 16 * n}
    rows, n = c["B"] * c["N"], c["B"] * c["N"] * c["C"]
    e = BYTES[c["dtype"]]
    if c["op"] == "norm_fwd":
        return {"bytes": 2 * n * e + 8 * rows + 2 * c["C"] * BYTES[c["wtype"]], "flops": 8 * n}
    if c["op"] == "norm_bwd":
        return {"bytes": 3 * n * e + 8 * rows + 3 * c["C"] * BYTES[c["wtype"]], "flops": 14 * n}
    live = 1 - c["ignored"]  # an ignored position's scores need not be read
    if c["op"] == "logp_fwd":
        return {"bytes": n * e * live + (16 + 8 * c["top"]) * rows, "flops": 6 * n * live}
    return {"bytes": n * e * (1 + live) + (20 if c["entropy"] else 12) * rows, "flops": 7 * n * live}


def _exact_norm(s, c):
    x = s["x"].double()
    x = x.transpose(1, 2) if c["layout"] == "bcn" else x
    w, b = s["w"].double(), s["b"].double()
    back = (lambda v: v.transpose(1, 2).contiguous()) if c["layout"] == "bcn" else (lambda v: v)
    if c["op"] == "norm_fwd":
        mean = x.sum(-1) / c["C"]
        var = ((x - mean[..., None]) ** 2).sum(-1) / c["C"]
        return back((x - mean[..., None]) / torch.sqrt(var + EPS)[..., None] * w + b), mean, 1 / torch.sqrt(var + EPS)
    gy = s["gy"].double()
    gy = gy.transpose(1, 2) if c["layout"] == "bcn" else gy
    xh = (x - s["mean"].double()[..., None]) * s["rstd"].double()[..., None]
    gw, gb = (gy * xh).sum((0, 1)), gy.sum((0, 1))
    wg = gy * w
    off = (wg.sum(-1)[..., None] + xh * (wg * xh).sum(-1)[..., None]) / c["C"]
    return back((wg - off) * s["rstd"].double()[..., None]), gw, gb


def _exact_logp(s, c):
    bcn, C, top = c["layout"] == "bcn", c["C"], c["top"]
    x = (s["x"].transpose(1, 2) if bcn else s["x"]).reshape(-1, C)
    t = s["t"].reshape(-1).long()
    rows, got = t.numel(), []
    for at in range(0, rows, max(1, (1 << 27) // C)):
        part = slice(at, min(rows, at + max(1, (1 << 27) // C)))
        z, tt = x[part].double(), t[part]
        on, k = tt >= 0, tt.clamp(min=0)[:, None]
        if c["op"] == "logp_fwd":
            lse = torch.logsumexp(z, 1)
            lp = z - lse[:, None]
            h = -(lp.exp() * lp).sum(1)
            one = [torch.where(on, v, 0.0) for v in (lp.gather(1, k)[:, 0], h, lse)]
            if top:
                one.append(torch.where(on[:, None], lp.topk(top, 1).values, -math.inf))
            got.append(one)
        else:
            gl = s["gl"].reshape(-1)[part].double()[:, None]
            lp = z - s["lse"].reshape(-1)[part].double()[:, None]
            p = lp.exp()
            gx = torch.zeros_like(z).scatter_(1, k, gl) - gl * p
            if s["gh"] is not None:
                gx -= s["gh"].reshape(-1)[part].double()[:, None] * p * (lp + s["h"].reshape(-1)[part].double()[:, None])
            got.append([torch.where(on[:, None], gx, 0.0)])
    outs = [torch.cat(v).view(c["B"], c["N"], -1) for v in zip(*got)]
    wide = (lambda v: v.transpose(1, 2).contiguous()) if bcn else (lambda v: v)
    if c["op"] == "logp_bwd":
        return wide(outs[0])
    return [v.squeeze(-1) for v in outs[:3]] + ([wide(outs[3]), None] if top else [])


def _power_64(e):
    return (e.long() + 1023 << 52).view(torch.float64)


def _exact_codes(x, square, r):
    """8-bit values of a row of up to 32 numbers each (square: numbers whose root is stored), as values and powers of two."""
    root = x.sqrt() if square else x.abs()
    fraction, e = torch.frexp(root.amax(1))
    e = (e - 9 + (fraction > 0.875).int()).clamp(-100, 120)  # the largest comes to (224, 448]
    scaled = root * _power_64(-e)[:, None]
    unit = _power_64((torch.frexp(scaled).exponent - 1).clamp(min=-6) - 3 + e[:, None])
    low = torch.floor(root / unit)
    if square:
        up = r * (2 * low + 1) < x / unit / unit - low * low
        low = torch.where(x > 0, (low + up).clamp(min=1), low)
    else:
        low = torch.floor(root / unit + r)
    value = (low * unit * _power_64(-e)[:, None]).clamp(max=448.0)
    return (value if square else torch.where(x < 0, -value, value)), _power_64(e)


def _exact_adamw(s, c):
    t, (b1, b2) = s["t"] + 1, BETAS
    out = {k: s[k].double() for k in ("p", "m", "v", "m_scale", "v_scale", "copy") if k in s}
    for k, (at, n, decay) in enumerate(s["places"]):
        here = slice(at, at + n)
        g = s["g"][here].double() * s["clip"].double()
        m, v = s["m"][here].double(), s["v"][here].double()
        if c["bits"] == 8:
            part = slice(at // 32, at // 32 + -(-n // 32))
            m = m * s["m_scale"][part].double().repeat_interleave(32)[:n]
            v = (v * s["v_scale"][part].double().repeat_interleave(32)[:n]) ** 2
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        p = s["p"][here].double()
        p = p - LR * decay * p - LR * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + ADAM_EPS)
        out["p"][here] = p
        if "copy" in s:
            out["copy"][here] = p
        if c["bits"] == 32:
            out["m"][here], out["v"][here] = m, v
            continue
        key = _mix(_mix(s["seed"] + t & M32) + k & M32)
        for name, x, r in (("m", m, 0), ("v", v, 1)):
            values, powers = _exact_codes(_blocks(x), name == "v", _blocks(_noise(n, key)[r].double()))
            out[name][here] = values.view(-1)[:n]
            out[name + "_scale"][part] = powers
    return out


def exact(case, seed):
    s, c = prepare(case, seed), dict(case)
    if c["op"] == "adamw":
        return _exact_adamw(s, c)
    return _exact_norm(s, c) if c["op"].startswith("norm") else _exact_logp(s, c)

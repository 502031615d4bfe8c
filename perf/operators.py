"""Layers and first-order steps as cases that can be timed and compared.

Three operators: `forward` is out = residual + scale * act(x w^T + bias), `backward` its gradient, `adamw` a step over many
tensors with the moments in 32 or in 8 bits.  Where `own` is false they are computed in their plain form, from elementary torch
operations in 32 bits; where it is true, by the package.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
ACTS = ("identity", "relu", "sigmoid", "gelu", "gelu_tanh", "silu")
BLOCK = 256                      # elements that share a scale, moments in 8 bits


def _forward(name, dtype, n, k, m, act="identity", bias=False, residual=False, scale=1.0, x_cols=False, w_cols=False, preact=False):
    c = dict(op="forward", dtype=dtype, n=n, k=k, m=m, act=act, bias=bias, residual=residual, scale=scale, x_cols=x_cols,
             w_cols=w_cols, preact=preact)
    return dict(c, name=name) if name else c


def _backward(name, dtype, n, k, m, act="identity", scale=1.0, x_cols=False, w_cols=False, gx=True, gw=True, gbias=True):
    c = dict(op="backward", dtype=dtype, n=n, k=k, m=m, act=act, scale=scale, x_cols=x_cols, w_cols=w_cols, gx=gx, gw=gw,
             gbias=gbias)
    return dict(c, name=name) if name else c


def _adamw(name, params, grads, bits, masters, count, smallest, largest, step, weight_decay=0.01, l1=0.0, grad_scale=1.0,
           align=64):
    c = dict(op="adamw", align=align, params=params, grads=grads, bits=bits, masters=masters, count=count, smallest=smallest, largest=largest,
             step=step, weight_decay=weight_decay, l1=l1, grad_scale=grad_scale)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the working residual y - sigma(X beta) of a logistic fit on the smallest dense configuration: a column-major design, one response
        _forward("residual_logistic_small", "f32", 1_000, 10_000, 1, act="sigmoid", residual=True, scale=-1.0, x_cols=True),
        # the residuals of a path of 20 fits on the middle dense configuration
        _forward("residuals_of_a_path", "f32", 10_000, 100_000, 20, residual=True, scale=-1.0, x_cols=True),
        # one token through a layer: latency counts
        _forward("forward_one_row", "bf16", 1, 4_096, 4_096, act="silu", bias=True),
        # a few sequences' tokens through a wide layer
        _forward("forward_few_rows", "bf16", 24, 4_096, 16_384, act="relu", bias=True, residual=True),
        # sizes that divide by nothing, in half precision
        _forward("forward_ragged", "f16", 777, 1_001, 2_053, act="gelu", bias=True, residual=True, preact=True),
        # a training batch through a large layer
        _forward("forward_large", "bf16", 8_192, 8_192, 8_192, act="gelu_tanh", bias=True, residual=True),
        # minus the gradient of a squared loss: X^T resid on the smallest dense configuration
        _backward("gradient_small", "f32", 1_000, 10_000, 1, scale=-1.0, x_cols=True, gx=False, gbias=False),
        # sizes that divide by nothing
        _backward("backward_ragged", "f16", 333, 1_001, 517, act="silu"),
        # a training batch back through a layer
        _backward("backward_large", "bf16", 4_096, 4_096, 8_192, act="gelu"),
        # the coefficients and intercepts of a few small models, with the L1 threshold
        _adamw("adamw_small", "f32", "f32", 32, False, 12, 1, 10_000, 100, weight_decay=0.0, l1=0.05),
        # a network of some 150 tensors: parameters, gradients and moments in 32 bits
        _adamw("adamw_large", "f32", "f32", 32, False, 150, 64, 8_000_000, 1_000),
        # the same in 16 bits with masters, moments in 8 bits
        _adamw("adamw_8bit_large", "bf16", "bf16", 8, True, 150, 64, 8_000_000, 1_000, grad_scale=0.125),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("forward", "forward", "backward", "adamw"))
    if op == "adamw":
        count = _log(rng, 1, 600)
        largest = _log(rng, 40, min(8_000_000, max(41, 600_000_000 // count)))
        params = rng.choice(("f32", "f32", "bf16", "f16"))
        return _adamw(None, params, rng.choice(("f32", params)), rng.choice((32, 8)), params != "f32" and rng.random() < 0.7, count,
                      _log(rng, 1, 40), largest, _log(rng, 1, 100_000), weight_decay=rng.choice((0.0, 0.01, 0.1)),
                      l1=rng.choice((0.0, 0.0, 0.01)), grad_scale=rng.choice((1.0, 0.125)), align=rng.choice((64, 64, 1)))
    dtype = rng.choice(("f32", "bf16", "f16"))
    top = (2 ** 36 if dtype == "f32" else 2 ** 38) // (1 if op == "forward" else 2)
    while True:
        n, k, m = _log(rng, 1, 8_192), _log(rng, 1, 16_384), _log(rng, 1, 16_384)
        if 2 ** 12 <= n * k * m <= top:
            break
    shape = dict(act=rng.choice(ACTS), scale=rng.choice((1.0, -1.0, 0.5)), x_cols=rng.random() < 0.3, w_cols=rng.random() < 0.3)
    if op == "forward":
        return _forward(None, dtype, n, k, m, bias=rng.random() < 0.7, residual=rng.random() < 0.5, preact=rng.random() < 0.3, **shape)
    return _backward(None, dtype, n, k, m, gx=rng.random() < 0.8, gbias=rng.random() < 0.7, **shape)


# ---- inputs ----

def _matrix(rows, cols, by_columns, dtype, gen, factor):
    t = torch.randn((cols, rows) if by_columns else (rows, cols), generator=gen, device="cuda", dtype=torch.float32)
    t = t.mul_(factor).to(dtype)
    return t.t() if by_columns else t


def _layer_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, n, k, m = DTYPES[case["dtype"]], case["n"], case["k"], case["m"]
    # a design has standardised columns of unit length and sparse coefficients of order one; a layer inputs of order one and weights ~ 1 / sqrt(k)
    design = case["dtype"] == "f32"
    d = dict(x=_matrix(n, k, case["x_cols"], dt, gen, 1.0 / math.sqrt(n) if design else 1.0))
    w = _matrix(m, k, case["w_cols"], dt, gen, 1.0 if design else 1.0 / math.sqrt(k))
    if design:
        w.mul_(torch.rand((m, k), generator=gen, device="cuda") < max(0.01, 4.0 / k))
    d["w"] = w
    if case["op"] == "forward":
        d["bias"] = torch.randn(m, generator=gen, device="cuda").mul_(0.5).to(dt) if case["bias"] else None
        d["residual"] = torch.randn((n, m), generator=gen, device="cuda").to(dt) if case["residual"] else None
    else:
        d["gout"] = torch.randn((n, m), generator=gen, device="cuda").to(dt)
        # what the forward pass kept of z: its rounding
        d["preact"] = (d["x"].float() @ d["w"].float().t()).to(dt) if case["act"] != "identity" else None
    return d


def _sizes(case):
    """The tensors' lengths, the same for every seed: spread over their logarithm, the largest among them."""
    lo, hi, c = math.log(case["smallest"]), math.log(case["largest"]), case["count"]
    return [int(round(math.exp(hi - (hi - lo) * ((i * 7) % c) / max(1, c)))) for i in range(c)]


def _starts(case):
    """Where each tensor starts in the flat buffer that a program keeps its parameters, gradients and moments in; the buffer's length."""
    starts, at = [], 0
    for n in _sizes(case):
        starts.append(at)
        at += -(-n // case["align"]) * case["align"]
    return starts, at


def _cut(case, flat):
    return [flat[a:a + n] for a, n in zip(_starts(case)[0], _sizes(case))]


def _blocks(case):
    """Where the elements of each block of 256 lie in the flat buffer, [blocks, 256], and which of them there are: a tensor's
    last block may be shorter, and no block spans two tensors.  Also the number of blocks of each tensor."""
    length = torch.tensor(_sizes(case), device="cuda")
    count = (length + BLOCK - 1) // BLOCK
    tensor = torch.arange(len(length), device="cuda").repeat_interleave(count)
    inside = torch.arange(len(tensor), device="cuda") - (count.cumsum(0) - count)[tensor]
    at = inside[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
    there = at < length[tensor][:, None]
    return torch.where(there, at + torch.tensor(_starts(case)[0], device="cuda")[tensor][:, None], 0), there, count.tolist()


def _encode_m(m):
    """Codes and scales of first moments in blocks [blocks, 256]: m = s q |q|, q = -128 where it is not finite."""
    mag = m.abs()
    top = torch.where(torch.isfinite(mag), mag, 0.0).amax(1)
    s = torch.where(top >= 2.0 ** -100, top * (1.0 / 16129.0), 0.0)
    r = torch.where(s > 0, 1.0 / s, 0.0)
    q = torch.round(torch.sqrt(mag * r[:, None]))
    return torch.where(torch.isfinite(mag), torch.where(m < 0, -q, q), -128.0).to(torch.int8), s


def _encode_root(root):
    """Codes and scales of the roots of second moments: sqrt(v) = s q^2, q = 255 where it is not finite, at least 1 where it is not 0."""
    top = torch.where(torch.isfinite(root), root, 0.0).amax(1)
    s = torch.where(top >= 2.0 ** -100, top * (1.0 / 64516.0), 0.0)
    r = torch.where(s > 0, 1.0 / s, 0.0)
    q = torch.round(torch.sqrt(root * r[:, None]))
    q = torch.where(root > 0, q.clamp(min=1.0), q)
    return torch.where(torch.isfinite(root), q, 255.0).to(torch.uint8), s


def _decode_m(q, s):
    v = q.float()
    return torch.where(q == -128, float("nan"), (v * v.abs()) * s[:, None])


def _decode_root(q, s):
    v = q.float()
    return torch.where(q == 255, float("nan"), (v * v) * s[:, None])


def _adamw_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    starts, total = _starts(case)
    normal = lambda: torch.randn(total, generator=gen, device="cuda")
    # every tensor has gradients of a size of its own
    size = torch.exp(torch.rand(len(starts), generator=gen, device="cuda") * -6.0)
    length = torch.tensor(starts[1:] + [total], device="cuda") - torch.tensor(starts, device="cuda")
    size = size.repeat_interleave(length, output_size=total)
    p = normal().mul_(0.05)
    g = normal().mul_(size).div_(case["grad_scale"])
    m = normal().mul_(size).mul_(0.3)
    v = torch.rand(total, generator=gen, device="cuda").add_(0.05).mul_(size).mul_(size)
    d = dict(params=p.to(DTYPES[case["params"]]), grads=g.to(DTYPES[case["grads"]]))
    if case["masters"]:
        d["masters"] = p
    d["first"], d["second"] = m, v
    if case["bits"] == 8:
        at, there, _ = _blocks(case)
        rows = lambda t: torch.where(there, t[at], 0.0)
        (q1, d["scale1"]), (q2, d["scale2"]) = _encode_m(rows(m)), _encode_root(rows(v).sqrt())
        d["code1"] = torch.zeros(total, dtype=torch.int8, device="cuda").index_put_((at[there],), q1[there])
        d["code2"] = torch.zeros(total, dtype=torch.uint8, device="cuda").index_put_((at[there],), q2[there])
        d["first"], d["second"] = torch.zeros_like(m), torch.zeros_like(v)      # where the values go that the codes stand for
    return d


LR, BETA1, BETA2, EPS = 1e-3, 0.9, 0.999, 1e-8


def prepare(case, seed):
    if case["op"] != "adamw":
        return dict(case=case, **_layer_inputs(case, seed))
    state = dict(case=case, step=case["step"], **_adamw_inputs(case, seed))
    # the tensors of the network: views of the flat buffers
    lists = {key: _cut(case, t) for key, t in state.items() if isinstance(t, torch.Tensor) and not key.startswith("scale")}
    if case["bits"] == 8:
        state["at"], state["there"], count = _blocks(case)
        moments = (lists["code1"], state["scale1"].split(count), lists["code2"], state["scale2"].split(count))
    else:
        inside = torch.zeros(state["params"].numel(), dtype=torch.bool, device="cuda")
        for t in _cut(case, inside):
            t.fill_(True)
        state["inside"] = inside
        moments = (lists["first"], lists["second"])
    state["lists"] = lists
    if own:
        from paper_1312_5766_b200 import binding
        state["opt"] = binding.AdamW(lists["params"], bits=case["bits"], masters=lists.get("masters"), moments=moments,
                                     betas=(BETA1, BETA2), eps=EPS, weight_decay=case["weight_decay"], l1=case["l1"])
    return state


# ---- the plain forms ----

def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "sigmoid":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 - s)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * z * z)
    s = 1.0 / (1.0 + torch.exp(-z))
    return s + z * s * (1.0 - s)


def _plain_forward(st):
    c = st["case"]
    dt = st["x"].dtype
    z = st["x"].float() @ st["w"].float().t()
    if st["bias"] is not None:
        z = z + st["bias"].float()
    out = c["scale"] * _act(z, c["act"])
    if st["residual"] is not None:
        out = st["residual"].float() + out
    out = out.to(dt)
    return [out, z.to(dt)] if c["preact"] else [out]


def _plain_backward(st):
    c = st["case"]
    dt = st["x"].dtype
    gz = c["scale"] * st["gout"].float()
    if c["act"] != "identity":
        gz = gz * _act_slope(st["preact"].float(), c["act"])
    out = []
    if c["gx"]:
        out.append((gz @ st["w"].float()).to(dt))
    if c["gw"]:
        out.append((gz.t() @ st["x"].float()).to(dt))
    if c["gbias"]:
        out.append(gz.sum(0).to(dt))
    return out


def _plain_adamw(st):
    c, t = st["case"], st["step"]
    f32 = lambda x: torch.tensor(x, dtype=torch.float32).item()      # the scalars are formed in 64 bits and rounded once
    b1, ob1, b2, ob2 = f32(BETA1), f32(1.0 - BETA1), f32(BETA2), f32(1.0 - BETA2)
    move, unbias, keep = f32(LR / (1.0 - BETA1 ** t)), f32(1.0 / math.sqrt(1.0 - BETA2 ** t)), f32(1.0 - LR * c["weight_decay"])
    threshold = f32(LR * c["l1"])
    at = st["masters"] if c["masters"] else st["params"].float()
    g = st["grads"].float() * c["grad_scale"]
    if c["bits"] == 32:
        m, v = st["first"], st["second"]
    else:
        where, there = st["at"], st["there"]
        rows = lambda t: torch.where(there, t[where], 0)
        at, g = rows(at), rows(g)
        m = _decode_m(rows(st["code1"]), st["scale1"])
        root = _decode_root(rows(st["code2"]), st["scale2"])
        v = root * root
    m = m * b1 + g * ob1
    v = v * b2 + (g * g) * ob2
    root = torch.sqrt(v)
    inv = 1.0 / (root * unbias + EPS)
    at = at * keep - (m * move) * inv
    if c["l1"] > 0:
        size = (at.abs() - threshold * inv).clamp(min=0.0)
        at = torch.where(at < 0, -size, size)
    if c["bits"] == 32:
        put = lambda flat, t: flat.copy_(torch.where(st["inside"], t.to(flat.dtype), flat))
    else:
        where = where[there]
        put = lambda flat, t: flat.index_put_((where,), t[there].to(flat.dtype))
        (q1, s1), (q2, s2) = _encode_m(m), _encode_root(root)
        st["scale1"].copy_(s1)
        st["scale2"].copy_(s2)
        put(st["code1"], q1)
        put(st["code2"], q2)
        m, root = _decode_m(q1, s1), _decode_root(q2, s2)
        v = root * root
    put(st["params"], at)
    if c["masters"]:
        put(st["masters"], at)
    put(st["first"], m)
    put(st["second"], v)
    return _adamw_outputs(st)


def _adamw_outputs(st):
    return [st["params"], st["first"], st["second"]] + ([st["masters"]] if st["case"]["masters"] else [])


def run(state):
    c = state["case"]
    if c["op"] == "forward":
        if not own:
            return _plain_forward(state)
        from paper_1312_5766_b200 import binding
        out = binding.linear_forward(state["x"], state["w"], bias=state["bias"], residual=state["residual"], activation=c["act"],
                                     scale=c["scale"], want_preact=c["preact"])
        return list(out) if c["preact"] else [out]
    if c["op"] == "backward":
        if not own:
            return _plain_backward(state)
        from paper_1312_5766_b200 import binding
        grads = binding.linear_backward(state["gout"], state["x"], state["w"], preact=state["preact"], activation=c["act"],
                                        scale=c["scale"], want_x=c["gx"], want_w=c["gw"], want_bias=c["gbias"])
        return [g for g in grads if g is not None]
    if not own:
        out = _plain_adamw(state)
    else:
        opt, lists = state["opt"], state["lists"]
        opt.step(lists["grads"], lr=LR, step=state["step"], grad_scale=c["grad_scale"])
        if c["bits"] == 8:
            opt.moments(out=(lists["first"], lists["second"]))
        out = _adamw_outputs(state)
    state["step"] += 1
    return out


def work(case):
    if case["op"] == "adamw":
        n = sum(_sizes(case))
        p, g = SIZE[case["params"]], SIZE[case["grads"]]
        moments = 16 if case["bits"] == 32 else 4 + 16 / BLOCK + 8        # 8 bits: read, written, and read back as 32-bit values
        return {"bytes": int(n * (2 * p + g + moments - (p if case["masters"] else 0) + (8 if case["masters"] else 0))), "flops": 14 * n}
    n, k, m, s = case["n"], case["k"], case["m"], SIZE[case["dtype"]]
    if case["op"] == "forward":
        out = n * m * s
        return {"bytes": s * (n * k + m * k + (m if case["bias"] else 0)) + out * (1 + case["residual"] + case["preact"]), "flops": 2 * n * k * m}
    b = s * n * m * (2 if case["act"] != "identity" else 1)
    b += (s * (m * k + n * k) if case["gx"] else 0) + (s * (n * k + m * k) if case["gw"] else 0) + (s * m if case["gbias"] else 0)
    return {"bytes": b, "flops": 2 * n * k * m * (case["gx"] + case["gw"])}


# ---- the operators by their definition, in 64 bits ----

def exact(case, seed):
    if case["op"] == "adamw":
        return _exact_adamw(case, seed)
    d = _layer_inputs(case, seed)
    x, w = d["x"].double(), d["w"].double()
    act, scale = case["act"], case["scale"]
    if case["op"] == "forward":
        z = torch.mm(x, w.t())
        if d["bias"] is not None:
            z += d["bias"].double()[None, :]
        a = {"identity": lambda: z, "relu": lambda: z.clamp(min=0), "sigmoid": lambda: torch.special.expit(z),
             "gelu": lambda: z * torch.special.ndtr(z), "silu": lambda: z * torch.special.expit(z),
             "gelu_tanh": lambda: z * torch.special.expit(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))}[act]()
        out = a * scale
        if d["residual"] is not None:
            out = out + d["residual"].double()
        return [out, z] if case["preact"] else [out]
    gz = d["gout"].double() * scale
    if act != "identity":
        z = d["preact"].double()
        s = torch.special.expit(z)
        if act == "relu":
            slope = torch.heaviside(z, torch.zeros((), dtype=torch.float64, device="cuda"))
        elif act == "sigmoid":
            slope = s * torch.special.expit(-z)
        elif act == "silu":
            slope = s * (1 + z * torch.special.expit(-z))
        elif act == "gelu":
            slope = torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        else:
            c = 2.0 * math.sqrt(2.0 / math.pi)
            e = torch.special.expit(c * (z + 0.044715 * z ** 3))
            slope = e + z * e * (1 - e) * c * (1 + 3 * 0.044715 * z ** 2)
        gz = gz * slope
    out = []
    if case["gx"]:
        out.append(torch.mm(gz, w))
    if case["gw"]:
        out.append(torch.mm(gz.t(), x))
    if case["gbias"]:
        out.append(gz.sum(0))
    return out


def _exact_adamw(case, seed):
    d = _adamw_inputs(case, seed)
    t, at, there = case["step"], *_blocks(case)[:2]
    at = at[there]                                                # (what lies between two tensors stays as it is)
    if case["bits"] == 32:
        m, v = d["first"].double()[at], d["second"].double()[at]
    else:
        q = d["code1"][at].double()
        m = q.sign() * q ** 2 * d["scale1"].double()[:, None].expand(there.shape)[there]
        v = (d["code2"][at].double() ** 2 * d["scale2"].double()[:, None].expand(there.shape)[there]) ** 2
    g = d["grads"].double()[at] * case["grad_scale"]
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g ** 2
    metric = (v / (1 - BETA2 ** t)).sqrt() + EPS
    p = d["masters" if case["masters"] else "params"].double()[at]
    p = p * (1 - LR * case["weight_decay"]) - LR * m / (1 - BETA1 ** t) / metric
    if case["l1"] > 0:
        p = torch.sgn(p) * (p.abs() - LR * case["l1"] / metric).clamp(min=0)
    put = lambda key, new: d[key].double().index_put_((at,), new)
    # a moment held in 8 bits is the nearest code of its block, not the number itself
    moments = [put("first", m), put("second", v)] if case["bits"] == 32 else [None, None]
    return [put("params", p)] + moments + ([put("masters", p)] if case["masters"] else [])

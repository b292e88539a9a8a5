"""Performance cases of the full step's operators and of the 8-bit history.

Operators (field ``op``)
  norm     h = x + gate * branch; RMS norm of h with weight, scale and shift; the new hidden state and
           the normalised rows in 8 bits (e4m3, one scale a row) or 16
  linear   act(x w^T + bias) as the branch output and/or added, gated, to the hidden state; x and w in
           bf16, or in e4m3 with a scale per row of x and of w
  write    a full step's branch outputs into an int8 history (blocks of 64 elements, a scale each), and
           the entry read back as predictions at its own time
  read     a skipped step's predictions and/or hidden states from the int8 history
"""
import math

import torch

own = False

DEV = "cuda"
TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "fp32": 4, "e4m3": 1}
BLOCK = 64             # elements of the history that share a scale
TINY = 2.0 ** -126     # the smallest scale
EPS = 1e-6
T_MIN, T_MAX, T_STEP = 0.0, 999.0, 80.0


def _norm(name, **kw):
    c = dict(name=name, op="norm", batch=1, tokens=256, hidden=1152, x="bf16", branch="bf16", out="e4m3", gated=True,
             modulated=True, weight=False)
    c.update(kw)
    return c


def _linear(name, **kw):
    c = dict(name=name, op="linear", batch=1, tokens=256, k=1152, n=4608, type="bf16", act="none", out="bf16", resid="",
             gated=False)
    c.update(kw)
    return c


def _history(name, op, **kw):
    c = dict(name=name, op=op, blocks=1, branches=2, batch=1, tokens=256, hidden=1152, K=4, feat="bf16", io="bf16",
             preds=True, hidden_states=False, gate="")
    c.update(kw)
    return c


def listed():
    return [
        # the 77 text tokens of one prompt: a call that is all latency
        _norm("norm_text", tokens=77, hidden=768, gated=False, modulated=False, weight=True),
        # odd sizes: rows off the 16-byte grid, 16-bit output for a layer that is kept in 16 bits
        _norm("norm_odd", batch=3, tokens=333, hidden=577, out="bf16"),
        # PixArt-Sigma 1024^2 with the residual stream in fp32
        _norm("norm_pixart_fp32", batch=2, tokens=4096, x="fp32"),
        # the modulation of one DiT-XL/2 block from the conditioning vectors of 8 samples: weights are all the traffic
        _linear("linear_modulation", batch=8, tokens=1, n=6912),
        # odd sizes in every direction
        _linear("linear_odd", batch=3, tokens=333, k=577, n=1155, act="silu", resid="fp32"),
        # DiT-XL/2 512^2, first MLP product from the norm's 8-bit rows
        _linear("linear_mlp_in_e4m3", batch=4, tokens=1024, type="e4m3", act="gelu"),
        # PixArt-Sigma 1024^2, second MLP product: the feature for the history and the gated hidden state
        _linear("linear_mlp_out", batch=2, tokens=4096, k=4608, n=1152, resid="bf16", gated=True),
        # FLUX.1-dev 1024^2, the output product of a single-stream block, the largest
        _linear("linear_flux_single", tokens=4608, k=15360, n=3072, out="", resid="bf16", gated=True),
        # a program that hooks single blocks reads the history once per block: all latency
        _history("read_one_block", "read", K=3),
        # DiT-XL/2 512^2, hidden states only, three branches of odd sizes under per-channel gates
        _history("read_odd_gated", "read", blocks=8, branches=3, batch=3, tokens=333, hidden=577, K=5, preds=False,
                 hidden_states=True, gate="bf16"),
        # the 38 single-stream blocks of FLUX.1-dev 1024^2
        _history("read_flux_single", "read", blocks=38, branches=1, tokens=4608, hidden=3072, K=5),
        # DiT-XL/2 256^2, a full step of all blocks
        _history("write_dit256", "write", blocks=28, batch=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Spread over the logarithm; three in four are multiples of 8."""
    v = _log(rng, lo, hi)
    return v if rng.random() < 0.25 else max(8, v // 8 * 8)


def draw(rng):
    op = rng.choice(["norm", "linear", "linear", "read", "write"])
    batch = rng.randint(1, 8)
    if op == "norm":
        c = _norm("", batch=batch, tokens=max(1, _log(rng, 8, 32768) // batch), hidden=_size(rng, 64, 8192),
                  x=rng.choice(["bf16", "fp32"]), branch=rng.choice(["bf16", "bf16", "fp32", ""]),
                  out=rng.choice(["e4m3", "e4m3", "bf16", "fp32"]), gated=rng.random() < 0.6,
                  modulated=rng.random() < 0.6, weight=rng.random() < 0.5)
        c["gated"] = c["gated"] and c["branch"] != ""
    elif op == "linear":
        c = _linear("", batch=batch, tokens=max(1, _log(rng, 1, 16384) // batch), k=_size(rng, 64, 16384),
                    n=_size(rng, 64, 16384), type=rng.choice(["bf16", "bf16", "e4m3"]),
                    act=rng.choice(["none", "none", "gelu", "silu"]), out=rng.choice(["bf16", "bf16", "fp32", ""]),
                    resid=rng.choice(["", "bf16", "fp32"]))
        if not c["out"] and not c["resid"]:
            c["out"] = "bf16"
        c["gated"] = c["resid"] != "" and rng.random() < 0.5
    else:
        c = _history("", op, blocks=rng.randint(1, 38), branches=rng.randint(1, 4), batch=batch,
                     hidden=_size(rng, 256, 4096), K=rng.randint(1, 8), feat=rng.choice(["bf16", "bf16", "fp32"]),
                     io=rng.choice(["bf16", "bf16", "fp32"]))
        rows = _log(rng, 3e5, 3e8) // (c["blocks"] * c["branches"] * batch * c["hidden"])
        c["tokens"] = max(1, min(8192, rows))
        if op == "read":
            c["preds"] = rng.random() < 0.7
            c["hidden_states"] = not c["preds"] or rng.random() < 0.5
            if c["hidden_states"] and rng.random() < 0.5:
                c["gate"] = rng.choice(["bf16", "fp32"])
    while work(c)["bytes"] > 3.5e9 or work(c)["flops"] > 4.2e11:
        c["tokens"] = -(-c["tokens"] // 2)
    del c["name"]
    return c


# ---- inputs

def _generator(seed, *at):
    g = torch.Generator(device=DEV)
    h = int(seed) + 1
    for p in at:
        h = (h * 1000003 + p + 7) % (1 << 62)
    g.manual_seed(h)
    return g


def _randn(shape, g, std=1.0):
    return torch.randn(shape, generator=g, device=DEV).mul_(std)


def _e4m3_rows(y):
    """Rows in e4m3, each with the scale that takes its largest value to 448."""
    s = (y.abs().amax(-1, keepdim=True) * (1.0 / 448.0)).clamp_min(TINY)
    return (y * torch.reciprocal(s)).to(torch.float8_e4m3fn), s.squeeze(-1)


def _norm_inputs(c, seed):
    g = _generator(seed, 1)
    b, t, h = c["batch"], c["tokens"], c["hidden"]
    channels = torch.exp(_randn((h,), g, 0.7))  # some channels of a hidden state are far larger than others
    s = {"x": (_randn((b, t, h), g) * channels).to(TORCH[c["x"]])}
    if c["branch"]:
        s["branch"] = _randn((b, t, h), g, 0.5).to(TORCH[c["branch"]])
    if c["gated"]:
        s["gate"] = _randn((b, h), g, 0.5).to(torch.bfloat16)
    if c["weight"]:
        s["weight"] = (1.0 + _randn((h,), g, 0.2)).to(torch.bfloat16)
    if c["modulated"]:
        s["scale"] = _randn((b, h), g, 0.3).to(torch.bfloat16)
        s["shift"] = _randn((b, h), g, 0.3).to(torch.bfloat16)
    return s


def _linear_inputs(c, seed):
    g = _generator(seed, 2)
    m, k, n = c["batch"] * c["tokens"], c["k"], c["n"]
    x, w = _randn((m, k), g), _randn((n, k), g, 1.0 / math.sqrt(k))
    s = {"bias": _randn((n,), g, 0.2).to(torch.bfloat16)}
    if c["type"] == "e4m3":
        (s["x"], s["x_scale"]), (s["w"], s["w_scale"]) = _e4m3_rows(x), _e4m3_rows(w)
    else:
        s["x"], s["w"] = x.to(torch.bfloat16), w.to(torch.bfloat16)
    if c["resid"]:
        s["resid"] = _randn((m, n), g).to(TORCH[c["resid"]])
    if c["gated"]:
        s["gate"] = _randn((c["batch"], n), g, 0.5).to(torch.bfloat16)
    return s


def _shape(c):
    """All branch outputs of the case: [tensors, batch, tokens, hidden]."""
    return c["blocks"] * c["branches"], c["batch"], c["tokens"], c["hidden"]


def _nodes(c):
    """Times of the K full steps, oldest first, and of the skipped step behind them."""
    nodes = [T_MAX - T_STEP * j for j in range(c["K"])]
    return nodes, nodes[-1] - T_STEP / 2


def _features(c, seed, j):
    """All branch outputs at the full step j: a smooth trajectory in time with noise."""
    x = 2.0 * (_nodes(c)[0][j] - T_MIN) / (T_MAX - T_MIN) - 1.0
    f = _randn(_shape(c), _generator(seed, 3, 10 + j), 0.1)
    for d, a in enumerate((1.0, x / 4, (2 * x * x - 1) / 9)):
        f.add_(_randn(_shape(c), _generator(seed, 3, d)), alpha=a)
    return f.to(TORCH[c["feat"]])


def _hidden_states(c, seed):
    return _randn((c["blocks"],) + _shape(c)[1:], _generator(seed, 4)).to(TORCH[c["io"]])


def _gates(c, seed):
    n, b, _, h = _shape(c)
    return _randn((n, b, h), _generator(seed, 5), 0.5).to(TORCH[c["gate"]])


def _to_blocks(f):
    """[tensors, blocks of 64], each tensor's tail filled up with zeros."""
    f = f.reshape(f.shape[0], -1)
    pad = -f.shape[1] % BLOCK
    return torch.nn.functional.pad(f, (0, pad)).view(f.shape[0], -1, BLOCK)


def _quantise(f):
    """Codes and scales of every block: the scale is a bf16, rounded up, codes are rounded to nearest even."""
    v = _to_blocks(f).float()
    s = v.abs().amax(-1, keepdim=True) * (1.0 / 127.0)
    s = ((s.view(torch.int32) + 0xFFFF) & -0x10000).view(torch.float32).clamp_min(TINY)
    return torch.round(v * torch.reciprocal(s)).to(torch.int8), s


def prepare(case, seed):
    c = dict(case)
    if c["op"] == "norm":
        s = {"c": c, **_norm_inputs(c, seed)}
        return _own_norm(s) if own else s
    if c["op"] == "linear":
        s = {"c": c, **_linear_inputs(c, seed)}
        return _own_linear(s) if own else s
    s = {"c": c}
    if c["hidden_states"]:
        s["x"] = _hidden_states(c, seed)
    if c["gate"]:
        s["gates"] = _gates(c, seed)
    if c["op"] == "write":
        s["feats"] = _features(c, seed, 0)
    if own:
        return _own_history(s, seed)
    if c["op"] == "read":  # the history as the full steps left it
        s["history"] = [_quantise(_features(c, seed, j)) for j in range(c["K"])]
    return s


# ---- the framework's operators

def _own_norm(s):
    from paper_2608_23429_gb300 import block, chebboost as cb
    c, code = s["c"], {"bf16": cb.CB_BF16, "fp32": cb.CB_FP32, "e4m3": cb.CB_E4M3}
    rows = c["batch"] * c["tokens"]
    s["call"] = block.cb_norm_residual
    s["desc"] = block.cb_norm_desc(rows=rows, hidden=c["hidden"], tokens=c["tokens"], x_dtype=code[c["x"]],
                                   branch_dtype=code[c["branch"] or "bf16"], param_dtype=cb.CB_BF16,
                                   out_dtype=code[c["out"]], eps=EPS)
    s["y"] = {"out": torch.empty(s["x"].shape, dtype=TORCH[c["out"]], device=DEV)}
    if c["branch"]:
        s["y"]["x"] = torch.empty_like(s["x"])
    if c["out"] == "e4m3":
        s["y"]["scale"] = torch.empty(s["x"].shape[:2], device=DEV)
    return s


def _own_linear(s):
    from paper_2608_23429_gb300 import block, chebboost as cb
    c, code = s["c"], {"": cb.CB_BF16, "bf16": cb.CB_BF16, "fp32": cb.CB_FP32, "e4m3": cb.CB_E4M3}
    rows = c["batch"] * c["tokens"]
    s["call"] = block.cb_linear_run
    s["layer"] = block.cb_linear_create(s["w"], c["n"], c["k"], code[c["type"]], w_scale=s.get("w_scale"), bias=s["bias"],
                                        bias_dtype=cb.CB_BF16, activation=getattr(block, "CB_ACT_" + c["act"].upper()))
    s["desc"] = block.cb_linear_io(rows=rows, tokens=c["tokens"], out_dtype=code[c["out"]], resid_dtype=code[c["resid"]],
                                   gate_dtype=cb.CB_BF16)
    s["y"] = {}
    if c["out"]:
        s["y"]["out"] = torch.empty((rows, c["n"]), dtype=TORCH[c["out"]], device=DEV)
    if c["resid"]:
        s["y"]["x"] = torch.empty_like(s["resid"])
    return s


def _own_history(s, seed):
    from paper_2608_23429_gb300 import chebboost as cb
    c, code = s["c"], {"": cb.CB_BF16, "bf16": cb.CB_BF16, "fp32": cb.CB_FP32}
    shape = _shape(c)
    nodes, target = _nodes(c)
    plan = cb.cb_plan_create(nodes, c["K"], [(i // c["branches"], i % c["branches"], math.prod(shape[1:]), i // c["branches"])
                                             for i in range(shape[0])], cb.CB_INT8, T_MIN, T_MAX)
    cb.cb_plan_set_shapes(plan, [shape[1:]] * shape[0])
    s["arena"] = torch.zeros(cb.cb_plan_cache_bytes(plan), dtype=torch.uint8, device=DEV)
    cb.cb_plan_bind_cache(plan, s["arena"], s["arena"].numel())
    cb.cb_plan_set_option(plan, cb.CB_OPT_PARTIAL_HISTORY, 1)
    if c["op"] == "read":
        for j, t in enumerate(nodes):
            f = _features(c, seed, j)
            cb.cb_cache_push(plan, list(f), code[c["feat"]], t)
    else:
        s["feats_at"] = cb.ptr_array(list(s["feats"]))
    if c["preds"]:
        s["preds"] = torch.empty(shape, dtype=TORCH[c["io"]], device=DEV)
    s.update(cb=cb, plan=plan, feat=code[c["feat"]], io=code[c["io"]], gate=code[c["gate"]], node=nodes[0], target=target,
             preds_at=cb.ptr_array(list(s["preds"])) if c["preds"] else None,
             x_at=cb.ptr_array(list(s["x"])) if c["hidden_states"] else None,
             gates_at=cb.ptr_array(list(s["gates"])) if c["gate"] else None)
    return s


def _run_own(s):
    op = s["c"]["op"]
    if op == "norm":
        y = s["y"]
        s["call"](s["desc"], s["x"], s.get("branch"), s.get("gate"), s.get("weight"), s.get("scale"), s.get("shift"),
                  y.get("x"), y["out"], y.get("scale"))
        return y
    if op == "linear":
        y = s["y"]
        s["call"](s["layer"], s["desc"], s["x"], s.get("x_scale"), s.get("resid"), s.get("gate"), y.get("out"), y.get("x"))
        return y
    cb, plan = s["cb"], s["plan"]
    if op == "write":
        cb.cb_plan_reset(plan)
        cb.cb_cache_push(plan, s["feats_at"], s["feat"], s["node"])
        cb.cb_extrapolate(plan, s["node"], s["preds_at"], s["io"])
    elif s["gates_at"] is not None:
        cb.cb_extrapolate_gated(plan, s["target"], s["preds_at"], s["io"], s["x_at"], s["io"], s["gates_at"], s["gate"])
    else:
        cb.cb_extrapolate(plan, s["target"], s["preds_at"], s["io"], s["x_at"], s["io"])
    return {k: s[k] for k in ("preds", "x") if k in s}


# ---- the plain forms

def _activate(v, act):
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    return v / (1.0 + torch.exp(-v)) if act == "silu" else v


def _run_norm(s):
    c, y = s["c"], {}
    h = s["x"].float()
    if c["branch"]:
        r = s["branch"].float()
        h = h + (r * s["gate"].float()[:, None, :] if c["gated"] else r)
        y["x"] = h.to(s["x"].dtype)
    n = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)
    if c["weight"]:
        n = n * s["weight"].float()
    if c["modulated"]:
        n = n * (1.0 + s["scale"].float()[:, None, :]) + s["shift"].float()[:, None, :]
    if c["out"] == "e4m3":
        y["out"], y["scale"] = _e4m3_rows(n)
    else:
        y["out"] = n.to(TORCH[c["out"]])
    return y


def _run_linear(s):
    c, y = s["c"], {}
    v = s["x"].float() @ s["w"].float().t()
    if c["type"] == "e4m3":
        v = v * s["x_scale"][:, None] * s["w_scale"]
    v = _activate(v + s["bias"].float(), c["act"])
    if c["out"]:
        y["out"] = v.to(TORCH[c["out"]])
    if c["resid"]:
        if c["gated"]:
            v = (v.view(c["batch"], c["tokens"], -1) * s["gate"].float()[:, None, :]).view(v.shape)
        y["x"] = (s["resid"].float() + v).to(s["resid"].dtype)
    return y


def _weights(nodes, t):
    return [math.prod((t - b) / (a - b) for b in nodes if b != a) for a in nodes]


def _from_blocks(p, c):
    shape = _shape(c)
    return p.view(shape[0], -1)[:, : math.prod(shape[1:])].reshape(shape)


def _run_history(s):
    c, y = s["c"], {}
    if c["op"] == "write":
        q, scale = _quantise(s["feats"])
        return {"preds": _from_blocks(q.float() * scale, c).to(TORCH[c["io"]])}
    p = None
    for w, (q, scale) in zip(_weights(*_nodes(c)), s["history"]):
        f = q.float() * (scale * w)
        p = f if p is None else p.add_(f)
    p = _from_blocks(p, c)
    if c["preds"]:
        y["preds"] = p.to(TORCH[c["io"]])
    if c["hidden_states"]:
        if c["gate"]:
            p = p * s["gates"].float()[:, :, None, :]
        add = p.view((c["blocks"], c["branches"]) + p.shape[1:]).sum(1)
        s["x"].copy_(s["x"].float() + add)
        y["x"] = s["x"]
    return y


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _run_norm, "linear": _run_linear}.get(state["c"]["op"], _run_history)(state)


def work(case):
    c = case
    if c["op"] == "norm":
        b, h = c["batch"], c["hidden"]
        n = b * c["tokens"] * h
        lines = b * h * (c["gated"] + 2 * c["modulated"]) + (h if c["weight"] else 0)
        per = SIZE[c["x"]] * (2 if c["branch"] else 1) + (SIZE[c["branch"]] if c["branch"] else 0) + SIZE[c["out"]]
        return {"bytes": n * per + 2 * lines + (4 * b * c["tokens"] if c["out"] == "e4m3" else 0), "flops": 10 * n}
    if c["op"] == "linear":
        m, k, n = c["batch"] * c["tokens"], c["k"], c["n"]
        per = (SIZE[c["out"]] if c["out"] else 0) + (2 * SIZE[c["resid"]] if c["resid"] else 0)
        lines = 2 * n + (2 * c["batch"] * n if c["gated"] else 0) + (4 * (m + n) if c["type"] == "e4m3" else 0)
        return {"bytes": SIZE[c["type"]] * k * (m + n) + m * n * per + lines, "flops": 2 * m * n * k}
    n = math.prod(_shape(c))
    held, io = n * (1 + 2 / BLOCK), SIZE[c["io"]]
    if c["op"] == "write":
        return {"bytes": n * (SIZE[c["feat"]] + io) + 2 * held, "flops": 3 * n}
    x = 2 * io * n // c["branches"] if c["hidden_states"] else 0
    gates = SIZE[c["gate"]] * n // c["tokens"] if c["gate"] else 0
    return {"bytes": c["K"] * held + (io * n if c["preds"] else 0) + x + gates, "flops": 2 * c["K"] * n}


# ---- the same in 64 bits

def _e4m3_grid(v):
    """v in [-448, 448] on the grid of e4m3: three bits behind the leading one, multiples of 2^-9 at least."""
    e = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(v / step) * step


def _exact_norm(c, seed):
    s = {k: v.double() for k, v in _norm_inputs(c, seed).items()}
    y, h = {}, s["x"]
    if c["branch"]:
        h = h + s["branch"] * (s["gate"].unsqueeze(1) if c["gated"] else 1.0)
        y["x"] = h
    n = h / torch.sqrt(h.square().mean(dim=2, keepdim=True) + EPS)
    if c["weight"]:
        n = n * s["weight"]
    if c["modulated"]:
        n = n + n * s["scale"].unsqueeze(1) + s["shift"].unsqueeze(1)
    y["out"] = n
    if c["out"] == "e4m3":
        y["scale"] = (n.abs().amax(dim=2) / 448.0).clamp_min(TINY)
        y["out"] = _e4m3_grid(n / y["scale"].unsqueeze(2))
    return y


def _exact_linear(c, seed):
    s = {k: v.double() for k, v in _linear_inputs(c, seed).items()}
    if c["type"] == "e4m3":
        s["x"], s["w"] = s["x"] * s["x_scale"].unsqueeze(1), s["w"] * s["w_scale"].unsqueeze(1)
    v = torch.addmm(s["bias"].unsqueeze(0), s["x"], s["w"].transpose(0, 1))
    if c["act"] == "gelu":  # 1/2 (1 + tanh u) = 1 / (1 + exp(-2u))
        v = v / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
    elif c["act"] == "silu":
        v = v * torch.sigmoid(v)
    y = {"out": v} if c["out"] else {}
    if c["resid"]:
        gate = s["gate"].repeat_interleave(c["tokens"], dim=0) if c["gated"] else 1.0
        y["x"] = torch.addcmul(s["resid"], v, gate) if c["gated"] else s["resid"] + v
    return y


def _exact_history(c, seed):
    n, b, t, h = _shape(c)
    gates = _gates(c, seed).double() if c["gate"] else None
    y = {"preds": torch.empty((n, b, t, h), dtype=torch.float64, device=DEV)} if c["preds"] else {}
    if c["hidden_states"]:
        y["x"] = _hidden_states(c, seed).double()
    if c["op"] == "write":
        v = _to_blocks(_features(c, seed, 0)).double()
        top = v.abs().amax(dim=2, keepdim=True) / 127.0
        unit = torch.exp2(torch.floor(torch.log2(top.clamp_min(TINY))) - 7)  # a bf16 has eight bits
        scale = (torch.ceil(top / unit) * unit).clamp_min(TINY)
        y["preds"] = (torch.round(v / scale) * scale).view(n, -1)[:, : b * t * h].reshape(n, b, t, h)
        return y
    nodes, at = _nodes(c)
    held = [_quantise(_features(c, seed, j)) for j in range(c["K"])]
    for i in range(n):
        p = torch.zeros(held[0][0].shape[1:], dtype=torch.float64, device=DEV)
        for j, (q, scale) in enumerate(held):
            w = 1.0
            for other in nodes[:j] + nodes[j + 1:]:
                w *= (at - other) / (nodes[j] - other)
            p.addcmul_(q[i].double(), scale[i].double(), value=w)
        p = p.reshape(-1)[: b * t * h].view(b, t, h)
        if c["preds"]:
            y["preds"][i] = p
        if c["hidden_states"]:
            y["x"][i // c["branches"]] += p * gates[i].unsqueeze(1) if c["gate"] else p
    return y


def exact(case, seed):
    c = dict(case)
    if c["op"] == "norm":
        return _exact_norm(c, seed)
    return _exact_linear(c, seed) if c["op"] == "linear" else _exact_history(c, seed)

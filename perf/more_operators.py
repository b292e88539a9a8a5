"""Performance cases of the norms around a block and of products in 4 bits.

Operators (field ``op``)
  norms    the norm after a branch, its addition to the hidden state under a gate and two scales, and the norm before the
           next branch (each none, root mean square, or layer norm), the rows in 16, 32, 8 (e4m3) or 4 bits; rows in 4 bits are
           read back as the values they stand for
  mx       rows quantised to 4 bits (MXFP4: e2m1 with a power of two for 32 consecutive elements) and read back
  linear   act(x w^T + bias) with x and w in MXFP4, as the branch output and/or added, gated, to the hidden state
  mlp      an MLP branch in 4 bits: norms, product with GELU to rows in 4 bits, product with the gated hidden state
"""
import math

import torch

own = False

DEV = "cuda"
TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "fp32": 4, "e4m3": 1}
BLOCK = 32             # elements that share a power of two
TINY = 2.0 ** -126     # the smallest scale of a row in e4m3
EPS, EPS_AFTER = 1e-6, 1e-5


def _norms(name, **kw):
    c = dict(name=name, op="norms", batch=1, tokens=256, hidden=1152, x="bf16", branch="bf16", after="none", before="layer",
             gated=True, modulated=True, affine=False, keep=1.0, add=1.0, out="bf16")
    c.update(kw)
    return c


def _mx(name, **kw):
    c = dict(name=name, op="mx", rows=256, k=1152, x="bf16")
    c.update(kw)
    return c


def _linear(name, **kw):
    c = dict(name=name, op="linear", batch=1, tokens=256, k=1152, n=4608, act="none", out="bf16", resid="", gated=False)
    c.update(kw)
    return c


def _mlp(name, **kw):
    c = dict(name=name, op="mlp", batch=1, tokens=256, hidden=1152, wide=4608)
    c.update(kw)
    return c


def listed():
    return [
        # the 77 text tokens of one prompt in a block with norms on both sides: a call that is all latency
        _norms("norms_text", tokens=77, hidden=768, after="rms", before="rms", gated=False, modulated=False, affine=True),
        # odd sizes: rows off the 16-byte grid, a scaled branch, 16-bit output for a layer that is kept in 16 bits
        _norms("norms_odd", batch=3, tokens=333, hidden=577, after="layer", before="rms", affine=True, add=0.25),
        # DiT-XL/2 512^2: the adaptive layer norm in front of a product in 4 bits
        _norms("norms_dit512", batch=4, tokens=1024, out="mxfp4"),
        # PixArt-Sigma 1024^2 with the residual stream in fp32, the branch normalised before it is added
        _norms("norms_pixart_fp32", batch=2, tokens=4096, x="fp32", after="rms", affine=True, out="e4m3"),
        # odd activations: the last block of a row is not whole
        _mx("mx_odd", rows=999, k=577),
        # the first MLP weights of DiT-XL/2's 28 blocks, from the checkpoint's fp32
        _mx("mx_weights", rows=28 * 4608, x="fp32"),
        # the modulation of one DiT-XL/2 block from the conditioning vectors of 8 samples: weights are all the traffic
        _linear("linear_modulation", batch=8, tokens=1, n=6912),
        # odd sizes in every direction
        _linear("linear_odd", batch=3, tokens=333, k=577, n=1155, act="silu", resid="fp32"),
        # PixArt-Sigma 1024^2, second MLP product: the feature for the history and the gated hidden state
        _linear("linear_mlp_out", batch=2, tokens=4096, k=4608, n=1152, resid="bf16", gated=True),
        # a large square product, the largest: the tensor cores' rate
        _linear("linear_large", tokens=8192, k=8192, n=8192),
        # one image of DiT-XL/2 256^2, its MLP branch: latency
        _mlp("mlp_dit256"),
        # two of PixArt-Sigma 1024^2
        _mlp("mlp_pixart", batch=2, tokens=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Spread over the logarithm; three in four are multiples of 8."""
    v = _log(rng, lo, hi)
    return v if rng.random() < 0.25 else max(8, v // 8 * 8)


def draw(rng):
    op = rng.choice(["norms", "norms", "mx", "linear", "linear", "mlp"])
    batch = rng.randint(1, 8)
    if op == "norms":
        c = _norms("", batch=batch, tokens=max(1, _log(rng, 8, 32768) // batch), hidden=_size(rng, 64, 8192),
                   x=rng.choice(["bf16", "fp32"]), branch=rng.choice(["bf16", "bf16", "fp32", ""]),
                   after=rng.choice(["none", "rms", "layer"]), before=rng.choice(["rms", "layer"]),
                   gated=rng.random() < 0.6, modulated=rng.random() < 0.6, affine=rng.random() < 0.5,
                   keep=rng.choice([1.0, 1.0, 1.5]), add=rng.choice([1.0, 1.0, 0.25]),
                   out=rng.choice(["mxfp4", "e4m3", "bf16", "fp32"]))
        if not c["branch"]:
            c.update(after="none", gated=False, add=1.0)
    elif op == "mx":
        c = _mx("", rows=_log(rng, 1, 131072), k=_size(rng, 32, 16384), x=rng.choice(["bf16", "fp32"]))
    elif op == "linear":
        c = _linear("", batch=batch, tokens=max(1, _log(rng, 1, 16384) // batch), k=_size(rng, 64, 16384),
                    n=_size(rng, 64, 16384), act=rng.choice(["none", "none", "gelu", "silu"]),
                    out=rng.choice(["bf16", "bf16", "fp32", ""]), resid=rng.choice(["", "bf16", "fp32"]))
        if not c["out"] and not c["resid"]:
            c["out"] = "bf16"
        c["gated"] = c["resid"] != "" and rng.random() < 0.5
    else:
        c = _mlp("", batch=batch, tokens=max(1, _log(rng, 8, 16384) // batch), hidden=_size(rng, 64, 4096))
        c["wide"] = 4 * c["hidden"] if rng.random() < 0.7 else _size(rng, 64, 16384)
    while work(c)["bytes"] > 1.2e9 or work(c)["flops"] > 1.0e12:
        at = "rows" if op == "mx" else "tokens"
        c[at] = -(-c[at] // 2)
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


def _channels(h, g):
    """Some channels of a hidden state are far larger than others."""
    return torch.exp(_randn((h,), g, 0.7))


def _tiles(e):
    """Scales [rows, blocks] in tiles of 128 rows by 4 blocks: 512 bytes, those of rows r, r + 32, r + 64 and r + 96 in 16."""
    r, b = e.shape
    e = torch.nn.functional.pad(e, (0, -b % 4, 0, -r % 128))
    return e.view(-(-r // 128), 4, 32, -(-b // 4), 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _from_tiles(t, r, b):
    rt, bt = -(-r // 128), -(-b // 4)
    return t.view(rt, bt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rt * 128, bt * 4)[:r, :b]


def _to_blocks(v):
    v = torch.nn.functional.pad(v, (0, -v.shape[-1] % BLOCK))
    return v.view(v.shape[0], -1, BLOCK)


def _block_scales(v):
    """Exponents (the power of two that takes the block's largest magnitude below 7), and the power's reciprocal and itself."""
    e = ((v.abs().amax(-1).view(torch.int32) + 0x200000) >> 23) - 2
    e = e.clamp(0, 254)
    low = torch.where(e == 0, 0x400000, e << 23)  # 2^-127 is a subnormal
    return e, ((254 - e) << 23).view(torch.float32).unsqueeze(-1), low.view(torch.float32).unsqueeze(-1)


def _e2m1(a):
    """a on the grid 0, 1/2, 1, 3/2, 2, 3, 4, 6, ties to even."""
    m = a.abs()
    step = torch.where(m < 2.0, 0.5, torch.where(m < 4.0, 1.0, 2.0))
    return torch.copysign((torch.round(m / step) * step).clamp_max(6.0), a)


def _mx_values(y):
    """fp32 rows as the values that MXFP4 holds."""
    v = _to_blocks(y)
    _, inverse, power = _block_scales(v)
    return (_e2m1(v * inverse) * power).view(y.shape[0], -1)[:, : y.shape[1]]


def _mx_rows(y):
    """fp32 rows in MXFP4: codes, two a byte with the even element in the low half, and scales in tiles."""
    v = _to_blocks(y)
    e, inverse, _ = _block_scales(v)
    a = _e2m1(v * inverse)
    m = a.abs()
    code = torch.where(m < 2.0, m * 2.0, torch.where(m < 4.0, m + 2.0, m / 2.0 + 4.0)).to(torch.uint8)
    code = (code | (torch.signbit(a).to(torch.uint8) << 3)).view(y.shape[0], -1)
    return code[:, 0::2] | (code[:, 1::2] << 4), _tiles(e.to(torch.uint8))


def _mx_read(codes, scales, k):
    """The values of rows in MXFP4 in fp32."""
    rows, blocks = codes.shape[0], codes.shape[1] // 16
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=DEV)
    grid = torch.cat([grid, -grid])
    v = grid[torch.stack([codes & 15, codes >> 4], -1).int()].view(rows, blocks, BLOCK)
    e = _from_tiles(scales, rows, blocks).int()
    power = torch.where(e == 0, 0x400000, e << 23).view(torch.float32)
    return (v * power.unsqueeze(-1)).view(rows, -1)[:, :k]


def _norms_inputs(c, seed):
    g = _generator(seed, 1)
    b, t, h = c["batch"], c["tokens"], c["hidden"]
    s = {"x": (_randn((b, t, h), g) * _channels(h, g) + _randn((h,), g, 0.2)).to(TORCH[c["x"]])}
    if c["branch"]:
        s["branch"] = (_randn((b, t, h), g, 0.5) + _randn((h,), g, 0.1)).to(TORCH[c["branch"]])
    if c["gated"]:
        s["gate"] = _randn((b, h), g, 0.5).to(torch.bfloat16)
    if c["affine"]:
        for n in ("after", "before"):
            if c[n] != "none":
                s[n + "_weight"] = (1.0 + _randn((h,), g, 0.2)).to(torch.bfloat16)
            if c[n] == "layer":
                s[n + "_bias"] = _randn((h,), g, 0.2).to(torch.bfloat16)
    if c["modulated"]:
        s["scale"] = _randn((b, h), g, 0.3).to(torch.bfloat16)
        s["shift"] = _randn((b, h), g, 0.3).to(torch.bfloat16)
    return s


def _mx_inputs(c, seed):
    g = _generator(seed, 2)
    return {"x": (_randn((c["rows"], c["k"]), g) * _channels(c["k"], g)).to(TORCH[c["x"]])}


def _layer_inputs(g, n, k):
    w, w_scale = _mx_rows(_randn((n, k), g, 1.0 / math.sqrt(k)))
    return {"w": w, "w_scale": w_scale, "bias": _randn((n,), g, 0.2).to(torch.bfloat16)}


def _linear_inputs(c, seed):
    g = _generator(seed, 3)
    m, k, n = c["batch"] * c["tokens"], c["k"], c["n"]
    s = _layer_inputs(g, n, k)
    s["x"], s["x_scale"] = _mx_rows(_randn((m, k), g))
    if c["resid"]:
        s["resid"] = _randn((m, n), g).to(TORCH[c["resid"]])
    if c["gated"]:
        s["gate"] = _randn((c["batch"], n), g, 0.5).to(torch.bfloat16)
    return s


def _mlp_inputs(c, seed):
    s = _norms_inputs(_as_norms(c), seed)
    g = _generator(seed, 4)
    s["first"], s["second"] = _layer_inputs(g, c["wide"], c["hidden"]), _layer_inputs(g, c["hidden"], c["wide"])
    s["gate2"] = _randn((c["batch"], c["hidden"]), g, 0.5).to(torch.bfloat16)
    return s


def _as_norms(c):
    return _norms("", batch=c["batch"], tokens=c["tokens"], hidden=c["hidden"], out="mxfp4")


INPUTS = {"norms": _norms_inputs, "mx": _mx_inputs, "linear": _linear_inputs, "mlp": _mlp_inputs}


def prepare(case, seed):
    c = dict(case)
    s = {"c": c, **INPUTS[c["op"]](c, seed)}
    if own:
        {"norms": _own_norms, "mx": _own_mx, "linear": _own_linear, "mlp": _own_mlp}[c["op"]](s)
    return s


# ---- the framework's operators

def _buffer(rows, k):
    """Codes and scales of rows in MXFP4."""
    from paper_2608_23429_gb300 import block
    return (torch.zeros((rows, -(-k // BLOCK) * 16), dtype=torch.uint8, device=DEV),
            torch.zeros(block.cb_mx_scale_bytes(rows, k), dtype=torch.uint8, device=DEV))


def _types():
    from paper_2608_23429_gb300 import chebboost as cb
    return {"": cb.CB_BF16, "bf16": cb.CB_BF16, "fp32": cb.CB_FP32, "e4m3": cb.CB_E4M3, "mxfp4": cb.CB_MXFP4}


def _norms_call(c):
    """Description of a call of the norms."""
    from paper_2608_23429_gb300 import block
    kind, code = {"none": block.CB_NORM_NONE, "rms": block.CB_NORM_RMS, "layer": block.CB_NORM_LAYER}, _types()
    return block.cb_norm_around_desc(
        rows=c["batch"] * c["tokens"], hidden=c["hidden"], tokens=c["tokens"], x_dtype=code[c["x"]],
        branch_dtype=code[c["branch"]], param_dtype=code["bf16"], out_dtype=code[c["out"]], after=kind[c["after"]],
        before=kind[c["before"]], after_eps=EPS_AFTER, before_eps=EPS, x_factor=c["keep"], branch_factor=c["add"])


def _own_norms(s):
    from paper_2608_23429_gb300 import block
    c = s["c"]
    s["norms"], s["desc"] = block.cb_norm_around, _norms_call(c)
    rows, h = c["batch"] * c["tokens"], c["hidden"]
    if c["out"] == "mxfp4":
        s["held"] = _buffer(rows, h)
        s["read"] = block.cb_mx_dequantize
        s["read_desc"] = block.cb_mx_desc(rows=rows, features=h, dtype=_types()["bf16"])
        s["y"] = {"out": torch.empty(s["x"].shape, dtype=torch.bfloat16, device=DEV)}
    else:
        s["y"] = {"out": torch.empty(s["x"].shape, dtype=TORCH[c["out"]], device=DEV)}
    s["y"]["x"] = torch.empty_like(s["x"])
    if c["out"] == "e4m3":
        s["y"]["scale"] = torch.empty(s["x"].shape[:2], device=DEV)


def _own_mx(s):
    from paper_2608_23429_gb300 import block
    c = s["c"]
    s["held"] = _buffer(c["rows"], c["k"])
    s["write"], s["read"] = block.cb_mx_quantize, block.cb_mx_dequantize
    s["desc"] = block.cb_mx_desc(rows=c["rows"], features=c["k"], dtype=_types()[c["x"]])
    s["y"] = {"out": torch.empty_like(s["x"])}


def _layer(p, n, k, act):
    from paper_2608_23429_gb300 import block
    code = _types()
    return block.cb_linear_create(p["w"], n, k, code["mxfp4"], w_scale=p["w_scale"], bias=p["bias"], bias_dtype=code["bf16"],
                                  activation=getattr(block, "CB_ACT_" + act.upper()))


def _own_linear(s):
    from paper_2608_23429_gb300 import block
    c, code = s["c"], _types()
    rows = c["batch"] * c["tokens"]
    s["call"], s["layer"] = block.cb_linear_run, _layer(s, c["n"], c["k"], c["act"])
    s["desc"] = block.cb_linear_io(rows=rows, tokens=c["tokens"], out_dtype=code[c["out"]], resid_dtype=code[c["resid"]],
                                   gate_dtype=code["bf16"])
    s["y"] = {}
    if c["out"]:
        s["y"]["out"] = torch.empty((rows, c["n"]), dtype=TORCH[c["out"]], device=DEV)
    if c["resid"]:
        s["y"]["x"] = torch.empty_like(s["resid"])


def _own_mlp(s):
    from paper_2608_23429_gb300 import block
    c, code = s["c"], _types()
    rows, h, wide = c["batch"] * c["tokens"], c["hidden"], c["wide"]
    s["norms"], s["call"], s["desc"] = block.cb_norm_around, block.cb_linear_run, _norms_call(_as_norms(c))
    s["held"], s["mid"] = _buffer(rows, h), _buffer(rows, wide)
    s["layers"] = _layer(s["first"], wide, h, "gelu"), _layer(s["second"], h, wide, "none")
    s["io"] = (block.cb_linear_io(rows=rows, out_dtype=code["mxfp4"], out_scale=s["mid"][1].data_ptr()),
               block.cb_linear_io(rows=rows, tokens=c["tokens"], out_dtype=code["bf16"], resid_dtype=code["bf16"],
                                  gate_dtype=code["bf16"]))
    s["y"] = {"out": torch.empty((rows, h), dtype=torch.bfloat16, device=DEV), "x": torch.empty_like(s["x"])}


def _run_own(s):
    op, y = s["c"]["op"], s["y"]
    if op == "linear":
        s["call"](s["layer"], s["desc"], s["x"], s["x_scale"], s.get("resid"), s.get("gate"), y.get("out"), y.get("x"))
    elif op == "mx":
        s["write"](s["desc"], s["x"], *s["held"])
        s["read"](s["desc"], *s["held"], y["out"])
    else:
        out, out_scale = s["held"] if "held" in s else (y["out"], y.get("scale"))
        s["norms"](s["desc"], s["x"], s.get("branch"), s.get("gate"), s.get("after_weight"), s.get("after_bias"),
                   s.get("before_weight"), s.get("before_bias"), s.get("scale"), s.get("shift"), y["x"], out, out_scale)
        if op == "mlp":
            s["call"](s["layers"][0], s["io"][0], *s["held"], None, None, s["mid"][0])
            s["call"](s["layers"][1], s["io"][1], *s["mid"], y["x"], s["gate2"], y["out"], y["x"])
        elif "held" in s:
            s["read"](s["read_desc"], *s["held"], y["out"])
    return y


# ---- the plain forms

def _activate(v, act):
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    return v / (1.0 + torch.exp(-v)) if act == "silu" else v


def _normed(v, kind, eps, weight, bias):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + eps)
    if weight is not None:
        v = v * weight.float()
    return v if bias is None else v + bias.float()


def _norms_plain(c, s):
    """The hidden state and the normalised rows, both in fp32."""
    h = s["x"].float() * c["keep"]
    if c["branch"]:
        r = _normed(s["branch"].float(), c["after"], EPS_AFTER, s.get("after_weight"), s.get("after_bias"))
        h = h + c["add"] * (r * s["gate"].float()[:, None, :] if c["gated"] else r)
    n = _normed(h, c["before"], EPS, s.get("before_weight"), s.get("before_bias"))
    if c["modulated"]:
        n = n * (1.0 + s["scale"].float()[:, None, :]) + s["shift"].float()[:, None, :]
    return h, n


def _run_norms(s):
    c = s["c"]
    h, n = _norms_plain(c, s)
    y = {"x": h.to(s["x"].dtype)}
    if c["out"] == "e4m3":
        a = (n.abs().amax(-1, keepdim=True) * (1.0 / 448.0)).clamp_min(TINY)
        y["out"], y["scale"] = (n * torch.reciprocal(a)).to(torch.float8_e4m3fn), a.squeeze(-1)
    elif c["out"] == "mxfp4":
        y["out"] = _mx_values(n.view(-1, c["hidden"])).reshape(n.shape).to(torch.bfloat16)
    else:
        y["out"] = n.to(TORCH[c["out"]])
    return y


def _product(x, p, act):
    """The layer p of rows in fp32."""
    return _activate(x @ _mx_read(p["w"], p["w_scale"], x.shape[1]).t() + p["bias"].float(), act)


def _gated(v, gate, c):
    return (v.view(c["batch"], c["tokens"], -1) * gate.float()[:, None, :]).view(v.shape)


def _run_linear(s):
    c, y = s["c"], {}
    v = _product(_mx_read(s["x"], s["x_scale"], c["k"]), s, c["act"])
    if c["out"]:
        y["out"] = v.to(TORCH[c["out"]])
    if c["resid"]:
        y["x"] = (s["resid"].float() + (_gated(v, s["gate"], c) if c["gated"] else v)).to(s["resid"].dtype)
    return y


def _run_mlp(s):
    c = s["c"]
    h, n = _norms_plain(_as_norms(c), s)
    mid = _product(_mx_values(n.view(-1, c["hidden"])), s["first"], "gelu")
    v = _product(_mx_values(mid), s["second"], "none")
    h = h.to(torch.bfloat16).float()  # as it is held between the calls
    return {"out": v.to(torch.bfloat16), "x": (h + _gated(v, s["gate2"], c).view(h.shape)).to(torch.bfloat16)}


def run(state):
    if own:
        return _run_own(state)
    op = state["c"]["op"]
    if op == "mx":
        x = state["x"]
        return {"out": _mx_values(x.float()).to(x.dtype)}
    return {"norms": _run_norms, "linear": _run_linear, "mlp": _run_mlp}[op](state)


def _held(rows, k):
    """Bytes of rows in MXFP4."""
    return rows * -(-k // BLOCK) * 17


def work(case):
    c = case
    if c["op"] == "norms":
        b, h = c["batch"], c["hidden"]
        rows = b * c["tokens"]
        n = rows * h
        lines = b * h * (c["gated"] + 2 * c["modulated"])
        if c["affine"]:
            lines += h * sum({"none": 0, "rms": 1, "layer": 2}[c[k]] for k in ("after", "before"))
        out = 2 * _held(rows, h) + 2 * n if c["out"] == "mxfp4" else n * SIZE[c["out"]] + (4 * rows if c["out"] == "e4m3" else 0)
        return {"bytes": n * (2 * SIZE[c["x"]] + (SIZE[c["branch"]] if c["branch"] else 0)) + out + 2 * lines, "flops": 16 * n}
    if c["op"] == "mx":
        n = c["rows"] * c["k"]
        return {"bytes": 2 * n * SIZE[c["x"]] + 2 * _held(c["rows"], c["k"]), "flops": 4 * n}
    rows = c["batch"] * c["tokens"]
    if c["op"] == "linear":
        k, n = c["k"], c["n"]
        per = (SIZE[c["out"]] if c["out"] else 0) + (2 * SIZE[c["resid"]] if c["resid"] else 0)
        lines = 2 * n + (2 * c["batch"] * n if c["gated"] else 0)
        return {"bytes": _held(rows, k) + _held(n, k) + rows * n * per + lines, "flops": 2 * rows * n * k}
    h, wide = c["hidden"], c["wide"]
    lines = 2 * (4 * c["batch"] * h + wide + h)
    return {"bytes": 8 * rows * h + _held(wide, h) + _held(h, wide) + lines, "flops": 4 * rows * h * wide}


# ---- the same in 64 bits

def _power(e):
    """2^e in 64 bits, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_block_scale(v):
    """The power of two of blocks in 64 bits: the largest magnitude is m 2^e with m in [1/2, 1); from 7/8 on it is the next."""
    m, e = torch.frexp(v.abs().amax(dim=-1, keepdim=True))
    e = torch.where(m >= 0.875, e + 1, e) - 3
    return _power(e.clamp(-127, 127))


def _exact_mx(y):
    k = y.shape[1]
    v = torch.nn.functional.pad(y, (0, (BLOCK - k % BLOCK) % BLOCK)).unflatten(1, (-1, BLOCK))
    s = _exact_block_scale(v)
    a = v / s
    m = a.abs()
    step = 0.5 + 0.5 * (m >= 2.0) + (m >= 4.0)
    return ((torch.round(a / step) * step).clamp(-6.0, 6.0) * s).flatten(1)[:, :k]


def _exact_mx_read(codes, scales, k):
    rows, blocks = codes.shape[0], codes.shape[1] // 16
    code = torch.stack((codes.remainder(16), codes.div(16, rounding_mode="floor")), dim=2).flatten(1).long()
    low, exponent = code & 1, (code >> 1) & 3
    a = torch.where(exponent == 0, 0.5 * low.double(), (1.0 + 0.5 * low.double()) * _power(exponent - 1))
    a = torch.where(code >= 8, -a, a)
    r = torch.arange(rows, device=DEV).unsqueeze(1)
    b = torch.arange(blocks, device=DEV).unsqueeze(0)
    at = ((r // 128) * ((blocks + 3) // 4) + b // 4) * 512 + (r % 32) * 16 + (r // 32 % 4) * 4 + b % 4
    s = _power(scales[at].long() - 127)
    return (a.view(rows, blocks, BLOCK) * s.unsqueeze(2)).flatten(1)[:, :k]


def _exact_normed(v, kind, eps, weight, bias):
    if kind == "none":
        return v
    mean = v.mean(dim=2, keepdim=True) if kind == "layer" else 0.0
    v = (v - mean) / torch.sqrt((v - mean).square().mean(dim=2, keepdim=True) + eps)
    v = v * weight if weight is not None else v
    return v + bias if bias is not None else v


def _exact_norms_rows(c, s):
    s = {k: v.double() for k, v in s.items() if torch.is_tensor(v)}
    h = c["keep"] * s["x"]
    if c["branch"]:
        r = _exact_normed(s["branch"], c["after"], EPS_AFTER, s.get("after_weight"), s.get("after_bias"))
        h = torch.addcmul(h, r, s["gate"].unsqueeze(1) * c["add"]) if c["gated"] else h + c["add"] * r
    n = _exact_normed(h, c["before"], EPS, s.get("before_weight"), s.get("before_bias"))
    if c["modulated"]:
        n = n + n * s["scale"].unsqueeze(1) + s["shift"].unsqueeze(1)
    return h, n


def _exact_norms(c, seed):
    h, n = _exact_norms_rows(c, _norms_inputs(c, seed))
    y = {"x": h, "out": n}
    if c["out"] == "e4m3":
        y["scale"] = (n.abs().amax(dim=2) / 448.0).clamp_min(TINY)
        v = n / y["scale"].unsqueeze(2)
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
        y["out"] = torch.round(v / step) * step
    elif c["out"] == "mxfp4":
        y["out"] = _exact_mx(n.flatten(0, 1)).view(n.shape)
    return y


def _exact_layer(x, p, act):
    v = torch.addmm(p["bias"].double().unsqueeze(0), x, _exact_mx_read(p["w"], p["w_scale"], x.shape[1]).transpose(0, 1))
    if act == "gelu":  # 1/2 (1 + tanh u) = 1 / (1 + exp(-2u))
        return v / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
    return v * torch.sigmoid(v) if act == "silu" else v


def _exact_linear(c, seed):
    s = _linear_inputs(c, seed)
    v = _exact_layer(_exact_mx_read(s["x"], s["x_scale"], c["k"]), s, c["act"])
    y = {"out": v} if c["out"] else {}
    if c["resid"]:
        gate = s["gate"].double().repeat_interleave(c["tokens"], dim=0) if c["gated"] else torch.ones_like(v)
        y["x"] = torch.addcmul(s["resid"].double(), v, gate)
    return y


def _exact_mlp(c, seed):
    s = _mlp_inputs(c, seed)
    h, n = _exact_norms_rows(_as_norms(c), s)
    mid = _exact_layer(_exact_mx(n.flatten(0, 1)), s["first"], "gelu")
    v = _exact_layer(_exact_mx(mid), s["second"], "none")
    held = h.to(torch.bfloat16).double()  # the hidden state is a bf16 between the calls
    return {"out": v, "x": torch.addcmul(held, v.view(h.shape), s["gate2"].double().unsqueeze(1))}


def exact(case, seed):
    c = dict(case)
    if c["op"] == "mx":
        return {"out": _exact_mx(_mx_inputs(c, seed)["x"].double())}
    return {"norms": _exact_norms, "linear": _exact_linear, "mlp": _exact_mlp}[c["op"]](c, seed)

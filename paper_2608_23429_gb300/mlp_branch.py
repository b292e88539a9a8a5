"""The MLP branches of a few blocks over a run with skipped steps, in 8 or 4 bits: an example of the block operators
(``chebboost_block.h``) with the int8 history.

The blocks are made up around the operators: norms with a modulation (root mean square in 8 bits, the adaptive layer norm in 4), at
a diffusion transformer's sizes.

Full step: each block's norm adds the previous branch to the hidden state and gives e4m3 rows; the first matrix product reads
them and applies GELU; the second gives the un-gated branch output, which the int8 history keeps; the last one also makes
the gated hidden state. In 4 bits the norm's rows, what GELU gives, and all weights are in MXFP4. Skipped step: one call predicts
all branches from the history and adds them, gated.

``python -m paper_2608_23429_gb300.mlp_branch`` runs it beside the same blocks in plain fp32 operations and prints how far
apart the hidden states are, and the time of a step of either kind.
"""
from __future__ import annotations

import math

import torch

from . import block, chebboost as cb

EPS = 1e-6


def mx_buffer(rows: int, features: int):
    """Codes and scales of rows in CB_MXFP4."""
    return (torch.empty(rows, -(-features // block.CB_MX_BLOCK) * block.CB_MX_BLOCK // 2, dtype=torch.uint8, device="cuda"),
            torch.zeros(block.cb_mx_scale_bytes(rows, features), dtype=torch.uint8, device="cuda"))


def quantised(w):
    """A weight in fp32 as codes and scales in CB_MXFP4."""
    buffer = mx_buffer(*w.shape)
    block.cb_mx_quantize(block.cb_mx_desc(rows=w.shape[0], features=w.shape[1], dtype=cb.CB_FP32), w, *buffer)
    return buffer


def values_of(buffer, rows: int, features: int):
    """What codes and scales in CB_MXFP4 stand for, in fp32."""
    w = torch.empty(rows, features, device="cuda")
    block.cb_mx_dequantize(block.cb_mx_desc(rows=rows, features=features, dtype=cb.CB_FP32), *buffer, w)
    return w


class MlpBranches:
    """Up to CB_MAX_BRANCHES MLP branches on one hidden state [batch, tokens, hidden] in bf16. ``bits``: 8 or 4."""

    def __init__(self, depth: int, batch: int, tokens: int, hidden: int, times, K: int = 3, seed: int = 0, bits: int = 8):
        if bits not in (4, 8):
            raise ValueError(f"bits = {bits}: 8 or 4")
        if not 1 <= depth <= cb.CB_MAX_BRANCHES:
            raise ValueError(f"depth = {depth}: one residual group holds 1 to {cb.CB_MAX_BRANCHES} branches")
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        rows, wide = batch * tokens, 4 * hidden
        self.depth, self.shape, self.bits = depth, (batch, tokens, hidden), bits
        self.params, self.layers = [], []
        for _ in range(depth):
            w1, w2 = r(wide, hidden) / math.sqrt(hidden), r(hidden, wide) / math.sqrt(wide)
            if bits == 4:
                p = {"b1": (0.1 * r(wide)).bfloat16(), "b2": (0.1 * r(hidden)).bfloat16(), "w1": quantised(w1), "w2": quantised(w2)}
                self.params.append(p)
                self.layers.append((
                    block.cb_linear_create(p["w1"][0], wide, hidden, cb.CB_MXFP4, p["w1"][1], p["b1"], activation=block.CB_ACT_GELU),
                    block.cb_linear_create(p["w2"][0], hidden, wide, cb.CB_MXFP4, p["w2"][1], p["b2"])))
                continue
            s1 = w1.abs().amax(1) / 448.0
            p = {"w1": (w1 / s1[:, None]).to(torch.float8_e4m3fn), "s1": s1, "b1": (0.1 * r(wide)).bfloat16(),
                 "w2": w2.bfloat16(), "b2": (0.1 * r(hidden)).bfloat16()}
            self.params.append(p)
            self.layers.append((
                block.cb_linear_create(p["w1"], wide, hidden, cb.CB_E4M3, p["s1"], p["b1"], activation=block.CB_ACT_GELU),
                block.cb_linear_create(p["w2"], hidden, wide, cb.CB_BF16, bias=p["b2"])))
        # per sample and block: shift and scale as they lie in one modulation tensor, and the gate
        self.lines = (0.3 * r(depth, batch, 2, hidden)).bfloat16()
        self.gates = (0.5 * r(depth, batch, hidden)).bfloat16()
        # a gate's lines follow each other, those of shift and scale lie two apart
        self.io1 = block.cb_linear_io(rows=rows, out_dtype=cb.CB_BF16)
        self.io2 = block.cb_linear_io(rows=rows, tokens=tokens, out_dtype=cb.CB_BF16, resid_dtype=cb.CB_BF16,
                                      gate_dtype=cb.CB_BF16)
        self.norm = block.cb_norm_desc(rows=rows, hidden=hidden, tokens=tokens, line_stride=2 * hidden, x_dtype=cb.CB_BF16,
                                       branch_dtype=cb.CB_BF16, out_dtype=cb.CB_E4M3, eps=EPS)
        self.gate_lines = torch.zeros(depth, batch, 2, hidden, dtype=torch.bfloat16, device="cuda")
        self.gate_lines[:, :, 0] = self.gates
        self.rows8 = torch.empty(rows, hidden, dtype=torch.float8_e4m3fn, device="cuda")
        self.row_scale = torch.empty(rows, device="cuda")
        self.mid = torch.empty(rows, wide, dtype=torch.bfloat16, device="cuda")
        if bits == 4:
            self.rows4, self.mid4 = mx_buffer(rows, hidden), mx_buffer(rows, wide)
            self.io1 = block.cb_linear_io(rows=rows, out_dtype=cb.CB_MXFP4, out_scale=self.mid4[1].data_ptr())
            self.around = block.cb_norm_around_desc(rows=rows, hidden=hidden, tokens=tokens, line_stride=2 * hidden, x_dtype=cb.CB_BF16,
                                                    branch_dtype=cb.CB_BF16, out_dtype=cb.CB_MXFP4, before=block.CB_NORM_LAYER,
                                                    before_eps=EPS)
        self.feats = torch.empty(depth, rows, hidden, dtype=torch.bfloat16, device="cuda")
        self.plan = cb.cb_plan_create(times, K, [(i, 0, rows * hidden, 0) for i in range(depth)], cb.CB_INT8,
                                      min(times) - 1.0, max(times) + 1.0)
        cb.cb_plan_set_shapes(self.plan, [self.shape] * depth)
        self.arena = torch.empty(cb.cb_plan_cache_bytes(self.plan), dtype=torch.uint8, device="cuda")
        cb.cb_plan_bind_cache(self.plan, self.arena, self.arena.numel())
        self.feats_at, self.gates_at = cb.ptr_array(list(self.feats)), cb.ptr_array(list(self.gates))

    def full_step(self, x, t: float, stream=None) -> None:
        """x (bf16, updated in place): every branch computed, the outputs into the history."""
        for i, (first, second) in enumerate(self.layers):
            before = (self.feats[i - 1], self.gate_lines[i - 1]) if i else (None, None)
            last = (x, self.gates[i]) if i + 1 == self.depth else (None, None)
            if self.bits == 4:
                block.cb_norm_around(self.around, x, *before, scale=self.lines[i, :, 1], shift=self.lines[i, :, 0],
                                     x_out=x if i else None, out=self.rows4[0], out_scale=self.rows4[1], stream=stream)
                block.cb_linear_run(first, self.io1, *self.rows4, out=self.mid4[0], stream=stream)
                block.cb_linear_run(second, self.io2, *self.mid4, *last, out=self.feats[i], resid_out=last[0], stream=stream)
                continue
            block.cb_norm_residual(self.norm, x, *before, scale=self.lines[i, :, 1], shift=self.lines[i, :, 0],
                                   x_out=x if i else None, out=self.rows8, out_scale=self.row_scale, stream=stream)
            block.cb_linear_run(first, self.io1, self.rows8, self.row_scale, out=self.mid, stream=stream)
            block.cb_linear_run(second, self.io2, self.mid, None, *last, out=self.feats[i], resid_out=last[0], stream=stream)
        cb.cb_cache_push(self.plan, self.feats_at, cb.CB_BF16, t, stream)

    def skipped_step(self, x, t: float, stream=None) -> None:
        """x (bf16, updated in place): every branch predicted from the history and added, gated."""
        cb.cb_extrapolate_gated(self.plan, t, None, cb.CB_BF16, [x], cb.CB_BF16, self.gates_at, cb.CB_BF16, stream)

    def close(self) -> None:
        cb.cb_plan_destroy(self.plan)
        for layers in self.layers:
            for layer in layers:
                block.cb_linear_destroy(layer)


class PlainBranches:
    """The same blocks in plain operations of ``dtype``, with an exact history."""

    def __init__(self, m: MlpBranches, dtype=torch.float32):
        f = lambda t: t.to(dtype) if t.dtype != torch.float8_e4m3fn else t.float().to(dtype)  # noqa: E731
        self.layer_norm, hidden = m.bits == 4, m.shape[2]
        if m.bits == 4:
            self.blocks = [(f(values_of(p["w1"], 4 * hidden, hidden)), f(p["b1"]), f(values_of(p["w2"], hidden, 4 * hidden)), f(p["b2"]))
                           for p in m.params]
        else:
            self.blocks = [(f(p["w1"]) * f(p["s1"])[:, None], f(p["b1"]), f(p["w2"]), f(p["b2"])) for p in m.params]
        self.lines, self.gates, self.shape, self.history = f(m.lines), f(m.gates), m.shape, []

    def _features(self, x):
        feats = []
        for i, (w1, b1, w2, b2) in enumerate(self.blocks):
            n = x - x.mean(-1, keepdim=True) if self.layer_norm else x
            n = n * torch.rsqrt((n * n).mean(-1, keepdim=True) + EPS)
            n = n * (1 + self.lines[i, :, None, 1]) + self.lines[i, :, None, 0]
            v = n @ w1.t() + b1
            v = v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
            feats.append(v @ w2.t() + b2)
            x = x + self.gates[i, :, None] * feats[-1]
        return feats, x

    def full_step(self, x, t: float):
        feats, x = self._features(x)
        self.history.append((t, feats))
        return x

    def skipped_step(self, x, t: float, K: int):
        held = self.history[-K:]
        for i in range(len(self.blocks)):
            p = sum(math.prod((t - b) / (a - b) for b, _ in held if b != a) * f[i] for a, f in held)
            x = x + self.gates[i, :, None] * p
        return x


def run(depth=4, batch=4, tokens=1024, hidden=1152, K=3, dtype=torch.float32, bits=8):
    """Three full steps and a skipped one on inputs that change smoothly with time: for every step the relative distance of the
    hidden state from the plain one's, and of the change that the step makes to it."""
    times, target = [9.0, 8.0, 7.0], 6.5
    m = MlpBranches(depth, batch, tokens, hidden, times, K, bits=bits)
    p = PlainBranches(m, dtype)
    g = torch.Generator(device="cuda").manual_seed(7)
    a, b = (torch.randn(batch, tokens, hidden, generator=g, device="cuda") for _ in range(2))
    off = []
    for t in times + [target]:
        x0 = (a + 0.05 * t * b).bfloat16()
        x, plain = x0.clone(), x0.to(dtype)
        if t == target:
            m.skipped_step(x, t)
            plain = p.skipped_step(plain, t, K)
        else:
            m.full_step(x, t)
            plain = p.full_step(plain, t)
        d = (x.to(dtype) - plain).norm()
        off.append((t, float(d / plain.norm()), float(d / (plain - x0.to(dtype)).norm())))
    torch.cuda.synchronize()
    assert cb.cb_plan_device_status(m.plan) == 0 and block.cb_linear_device_status() == 0
    return m, off


def main() -> None:
    for bits in (8, 4):
        m, off = run(bits=bits)
        for t, rel, change in off:
            print(f"{bits} bits, t = {t}: hidden state {rel:.1e} off the plain fp32 one, its change {change:.1e}")
        x = torch.randn(m.shape, device="cuda").bfloat16()
        for name, step in (("full", lambda i: m.full_step(x, 6.0 - i)), ("skipped", lambda i: m.skipped_step(x, -40.0))):
            for i in range(3):
                step(i / 100)
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            for i in range(20):
                step(1 + i / 10)
            end.record()
            torch.cuda.synchronize()
            print(f"{bits} bits, {name} step of {m.depth} branches on {tuple(m.shape)}: {begin.elapsed_time(end) / 20 * 1e3:.0f} us")
        m.close()


if __name__ == "__main__":
    main()

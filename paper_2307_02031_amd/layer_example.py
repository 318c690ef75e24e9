"""A transformer layer's training step on this device, measured, and planned with.

    python -m paper_2307_02031_amd.layer_example --model BERT-Huge-32 --batch 16 --devices 8 --mem-gb 16

Section 5's cost estimator takes a layer's time from running it on one device.  Here one layer of a row of the
paper's model table runs forward and backward with the library's operators (layer norm, attention, gradient
clipping; the matrix products are torch's), and the rate it reaches replaces the round figure of the analytic cost
model, whose tables the planner then searches (as in plan_example).

--norm rms and --rotary make it a present-day decoder's layer.  --states 32 or 8 adds the optimizer's step (AdamW) and
plans with the bytes that weights, gradients and its states take for each parameter.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

# weights of a layer, [out][in], and vectors; products in the activations' type, norms' parameters in float32
SHAPES = dict(qkv=lambda h: (3 * h, h), qkv_bias=lambda h: (3 * h,), proj=lambda h: (h, h), proj_bias=lambda h: (h,),
              up=lambda h: (4 * h, h), up_bias=lambda h: (4 * h,), down=lambda h: (h, 4 * h), down_bias=lambda h: (h,),
              norm1=lambda h: (h,), norm1_bias=lambda h: (h,), norm2=lambda h: (h,), norm2_bias=lambda h: (h,))


class Layer:
    """x + attention(norm(x)), then the same around a two-product network with GELU.  rms: norms by the root mean square,
    which take the addition before them; rotary: queries and keys turn by their positions."""

    def __init__(self, g, hidden: int, head: int, causal: bool, dtype=torch.bfloat16, seed: int = 0, rms: bool = False,
                 rotary: bool = False):
        self.g, self.hidden, self.head, self.causal, self.rms = g, hidden, head, causal, rms
        self.freq = g.gbmw_rotary_frequencies(head) if rotary else None
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.w, self.grad = {}, {}
        for name, shape in SHAPES.items():
            if rms and name in ("norm1_bias", "norm2_bias"):
                continue
            size, kind = shape(hidden), torch.float32 if name.startswith("norm") else dtype
            if len(size) == 2:
                w = torch.randn(size, generator=gen, device="cuda") * (size[1] ** -0.5)
            else:
                w = torch.ones(size, device="cuda") if name in ("norm1", "norm2") else torch.zeros(size, device="cuda")
            self.w[name] = w.to(kind)
            self.grad[name] = torch.zeros_like(self.w[name])
        # the gradients stay where they are, so the list is made once; the optimizer gets float32
        self.main = {n: torch.empty(t.shape, dtype=torch.float32, device="cuda") for n, t in self.grad.items()}
        self.list = g.gbmw_gradient_list_create(self.grad.values(), self.main.values())

    def norm(self, name, x, residual=None):
        """The sum, its norm, and what the backward pass wants of it."""
        g, w = self.g, self.w
        if self.rms:
            r = g.gbmw_rms_norm_forward(x, w[name], residual=residual)
            return r.h, r.y, (r.rstd,)
        if residual is not None:
            x = x.add_(residual)
        y, mean, rstd = g.gbmw_layer_norm_forward(x, w[name], w[name + "_bias"])
        return x, y, (mean, rstd)

    def norm_backward(self, name, dy, x, stats, dres):
        """The gradient of the sum, of which dres reached it past the norm."""
        g, w = self.g, self.w
        if self.rms:
            dx, dw = g.gbmw_rms_norm_backward(dy, x, w[name], *stats, dres=dres)
        else:
            dx, dw, db = g.gbmw_layer_norm_backward(dy, x, w[name], *stats)
            dx.add_(dres)
            self.grad[name + "_bias"].copy_(db)
        self.grad[name].copy_(dw)
        return dx

    def forward(self, x, len_x=None):
        """x [B][L][hidden]; len_x: int32 [B], the samples' lengths."""
        g, w, B, L, h = self.g, self.w, x.shape[0], x.shape[1], self.hidden
        _, n1, stats1 = self.norm("norm1", x)
        qkv = torch.addmm(w["qkv_bias"], n1.view(-1, h), w["qkv"].t()).view(B, L, 3, -1, self.head)
        q, k, v = qkv.unbind(2)
        if self.freq is not None:
            g.gbmw_rotary_forward(q, k, self.freq, len_x=len_x, q_out=q, k_out=k)     # where the product left them
        out, lse = g.gbmw_attention_forward(q, k, v, causal=self.causal, len_q=len_x, len_k=len_x)
        y = torch.addmm(w["proj_bias"], out.view(-1, h), w["proj"].t()).view(x.shape)
        y, n2, stats2 = self.norm("norm2", y, x)
        u = torch.addmm(w["up_bias"], n2.view(-1, h), w["up"].t())
        a = torch.nn.functional.gelu(u)
        z = torch.addmm(w["down_bias"], a, w["down"].t()).view(x.shape).add_(y)
        self.kept = (x, len_x, n1, stats1, q, k, v, out, lse, y, n2, stats2, u, a)
        return z

    def backward(self, dz):
        """dx; the weights' gradients are in self.grad."""
        g, w, h = self.g, self.w, self.hidden
        x, len_x, n1, stats1, q, k, v, out, lse, y, n2, stats2, u, a = self.kept

        def product(name, d, inp):     # of inp @ weight.t() + bias
            torch.mm(d.t(), inp, out=self.grad[name])
            torch.sum(d, 0, out=self.grad[name + "_bias"])
            return d @ w[name]

        dz2 = dz.view(-1, h)
        du = torch.ops.aten.gelu_backward(product("down", dz2, a), u)
        dn2 = product("up", du, n2.view(-1, h)).view(x.shape)
        dy = self.norm_backward("norm2", dn2, y, stats2, dz)
        dout = product("proj", dy.view(-1, h), out.view(-1, h)).view(out.shape)
        dqkv = torch.empty(*q.shape[:2], 3, *q.shape[2:], dtype=q.dtype, device="cuda")
        dq, dk, dv = dqkv.unbind(2)     # written where the product before them reads them
        g.gbmw_attention_backward(dout, q, k, v, out, lse, causal=self.causal, len_q=len_x, len_k=len_x, dq=dq, dk=dk,
                                  dv=dv)
        if self.freq is not None:     # rows beyond a sample's length have gradients of 0, turned or not
            g.gbmw_rotary_backward(dq, dk, self.freq, len_x=len_x, q_out=dq, k_out=dk)
        dn1 = product("qkv", dqkv.view(-1, 3 * h), n1.view(-1, h)).view(x.shape)
        return self.norm_backward("norm1", dn1, x, stats1, dy)

    def clip(self, max_norm: float):
        """The gradients, clipped, in self.main; their norm before."""
        return self.g.gbmw_clip_gradients(self.list, max_norm)

    def optimizer(self, state_bits: int, weight_decay: float = 0.1):
        """States of AdamW for self.step.  Products' weights get parameters in float32, of which they are copies; the
        step clips gradients as it reads them, so their list here is for the norm alone."""
        g, names = self.g, list(self.w)
        wide = {n: self.w[n].float() if self.w[n].dtype != torch.float32 else self.w[n] for n in names}
        kind = torch.float8_e4m3fn if state_bits == 8 else torch.float32
        # zeroed in float32, and then given the type
        zeros = lambda: {n: torch.zeros(self.w[n].shape, device="cuda").to(kind) for n in names}
        scales = lambda: {n: torch.zeros((self.w[n].numel() + 255) // 256, device="cuda") for n in names}
        self.param, self.m, self.v, self.steps = wide, zeros(), zeros(), 0
        self.m_scale, self.v_scale = (scales(), scales()) if state_bits == 8 else ({}, {})
        self.norm_list = g.gbmw_gradient_list_create(self.grad.values(), norm_only=True)
        self.adamw = g.gbmw_adamw_list_create(
            wide.values(), [self.grad[n] for n in names], self.m.values(), self.v.values(),
            m_scales=self.m_scale.values() if state_bits == 8 else None,
            v_scales=self.v_scale.values() if state_bits == 8 else None,
            copies=[None if wide[n] is self.w[n] else self.w[n] for n in names],
            weight_decay=[weight_decay if self.w[n].dim() == 2 else 0.0 for n in names])

    def step(self, lr: float, max_norm: float):
        """One step of the optimizer; the gradients' norm before clipping."""
        self.steps += 1
        norm = self.g.gbmw_clip_gradients(self.norm_list, float("inf"))
        self.g.gbmw_adamw_step(self.adamw, lr, self.steps, norm=norm, max_norm=max_norm, seed=1)
        return norm


def measured(f, steps: int) -> float:
    """Seconds of one call, on the device."""
    for _ in range(3):
        f()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    for _ in range(steps):
        f()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) * 1e-3 / steps


def main():
    import gbmw_inputs as gi
    import paper_2307_02031_amd as g
    from paper_2307_02031_amd.plan_example import plan

    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--model", default="BERT-Huge-32", choices=sorted(gi.TABLE1))
    ap.add_argument("--batch", type=int, default=16, help="samples of the measured layer")
    ap.add_argument("--head", type=int, default=64, help="head size")
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--norm", default="layer", choices=("layer", "rms"))
    ap.add_argument("--rotary", action="store_true", help="turn queries and keys by their positions")
    ap.add_argument("--states", type=int, default=0, choices=(0, 8, 32), help="run AdamW's step with states of so many bits")
    ap.add_argument("--devices", type=int, default=8)
    ap.add_argument("--mem-gb", type=float, default=16.0, help="memory budget per device of the plan")
    ap.add_argument("--unit-mb", type=float, default=8.0)
    args = ap.parse_args()

    _, hidden, _, _, tokens = gi.TABLE1[args.model]
    layers = gi.table1_layers(args.model)
    layer = Layer(g, hidden, args.head, causal=args.model.startswith("GPT"), rms=args.norm == "rms",
                  rotary=args.rotary)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(args.batch, tokens, hidden, generator=gen, device="cuda").bfloat16()
    dz = torch.randn(args.batch, tokens, hidden, generator=gen, device="cuda").bfloat16() * 0.01
    times = dict(forward=measured(lambda: layer.forward(x), args.steps),
                 backward=measured(lambda: layer.backward(dz), args.steps),
                 clip=measured(lambda: layer.clip(1.0), args.steps))
    if args.states:
        layer.optimizer(args.states)
        times["step"] = measured(lambda: layer.step(1e-4, 1.0), args.steps)
    print(f"{args.model}: one layer of {hidden} x {tokens} tokens x {args.batch} samples: " +
          ", ".join(f"{n} {t * 1e3:.3f} ms" for n, t in times.items()) + f", gradient norm {float(layer.clip(1.0)):.4g}")

    hw = gi.default_hardware(unit_mb=args.unit_mb)
    hw["island"] = min(hw["island"], args.devices)
    if args.states:     # weights and gradients in 16 bits, parameters in 32, two states
        hw["state_bytes"] = 2 + 2 + 4 + 2 * args.states / 8 + (2 * 4 / 256 if args.states == 8 else 0)
    # the model prices a step at three forward passes of `flops / rate`
    hw["rate"] = 3 * float(layers[0, 1]) * args.batch / (times["forward"] + times["backward"])
    print(f"rate of the layer: {hw['rate'] / 1e12:.1f} TFLOP/s (backward {times['backward'] / times['forward']:.2f} x forward; "
          "the model says 2)")
    best, _, _ = plan(g, gi, layers, args.devices, int(args.mem_gb * 1024 / args.unit_mb), hw, [8.0, 16.0, 32.0, 64.0], 8,
                      log=print)
    if best is None:
        print("no feasible plan")
    else:
        print(f"best: batch {int(best['B'])}, PP={best['P']}, partition {best['part']}, throughput {best['tpt']:.4g} samples/s")


if __name__ == "__main__":
    main()

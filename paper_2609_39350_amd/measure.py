"""Measured planner inputs of the GPU this runs on (Section 3.3, warm-up profiling: expert and
router times, router statistics, optimizer time).

One mixture-of-experts layer of a problem's model takes training steps on the operators of
``operators.py``: router, gated expert FFNs, the sum of each token's expert outputs, all of it
backward, and AdamW over the experts.  Its weights and inputs are random.  ``apply`` puts what
was measured in the place of one device type's entries, so that the planner weighs that type by
what its operators take:

    python -m paper_2609_39350_amd.measure --config 2 --type 2

prints the measurement and the plans before and after, both with the workload's router counts.
"""
from __future__ import annotations

import argparse
import copy
import math

import numpy as np
import torch

from . import binding, operators, workloads

STATE_BYTES = {32: 18, 8: 12}   # of an expert parameter on the GPU: copy, gradient, master and moments


def router_forward(x, router, top_k):
    logits = x @ router.T
    return logits, operators.route(logits, top_k)


def router_backward(x, router, logits, routing, d_weight):
    """The gradients of the router's matrix and, through it, of x in fp32."""
    d_logits = operators.route_backward(logits, routing, d_weight)
    return d_logits.T @ x, (d_logits @ router).float()


def layer_step(x, router, experts, d_out, top_k, mark=lambda name: None):
    """One layer forward and backward.  x [tokens, hidden], router [n_experts, hidden], experts: the gate, up
    and down matrices [n_experts, width, hidden], the same, [n_experts, hidden, width], d_out: the gradient of the
    output.  Returns the routing, the output and the gradients; calls mark(name) where a part of the layer ends."""
    gate, up, down = experts
    logits, r = router_forward(x, router, top_k)
    mark("route")
    g = operators.expert_matmul(x, gate, r.offset, slot=r.slot, top_k=top_k)
    u = operators.expert_matmul(x, up, r.offset, slot=r.slot, top_k=top_k)
    s = torch.sigmoid(g.float())
    a = g.float() * s                       # the gate's activation
    h = (a * u.float()).to(x.dtype)
    y = operators.expert_matmul(h, down, r.offset)
    mark("experts")
    out = operators.combine(y, r.place, r.weight)
    d_y, d_weight = operators.combine_backward(d_out, y, r.slot, r.place, r.weight)
    mark("combine")
    d_h = operators.expert_matmul_grad_x(d_y, down, r.offset).float()
    d_down = operators.expert_matmul_grad_w(d_y, h, r.offset)
    d_u = (d_h * a).to(x.dtype)
    d_g = (d_h * u.float() * (s + a * (1 - s))).to(x.dtype)
    d_gate = operators.expert_matmul_grad_w(d_g, x, r.offset, slot=r.slot, top_k=top_k)
    d_up = operators.expert_matmul_grad_w(d_u, x, r.offset, slot=r.slot, top_k=top_k)
    d_rows = operators.expert_matmul_grad_x(d_g, gate, r.offset), operators.expert_matmul_grad_x(d_u, up, r.offset)
    mark("experts")
    d_x = operators.combine(d_rows[0], r.place).float() + operators.combine(d_rows[1], r.place).float()
    mark("combine")
    d_router, d_rest = router_backward(x, router, logits, r, d_weight)
    d_x += d_rest
    mark("route")
    return {"routing": r, "out": out, "d_x": d_x.to(x.dtype), "d_router": d_router,
            "d_experts": (d_gate, d_up, d_down)}


class Layer:
    """The layer's weights, AdamW state and inputs on the current device, random."""

    def __init__(self, tokens, hidden, width, n_experts, top_k, state_bits=32, skew=1.1, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, scale=1.0, dtype=torch.bfloat16):
            out = torch.empty(shape, dtype=dtype, device="cuda")
            for part in out.view(-1).split(1 << 26):
                part.copy_(torch.randn(part.numel(), generator=gen, device="cuda") * scale)
            return out

        self.top_k = top_k
        shapes = [(n_experts, width, hidden)] * 2 + [(n_experts, hidden, width)]
        self.masters = [normal(*s, scale=s[2] ** -0.5, dtype=torch.float32) for s in shapes]
        self.experts = [m.bfloat16() for m in self.masters]
        self.router = normal(n_experts, hidden, scale=hidden ** -0.5)
        self.x, self.d_out = normal(tokens, hidden), normal(tokens, hidden, scale=1e-3)
        # experts taken unevenly: a direction that the tokens share carries a bias of each expert
        bias = torch.log(torch.arange(1, n_experts + 1, device="cuda").float()) * -skew
        bias = bias[torch.randperm(n_experts, generator=gen, device="cuda")]
        self.x[:, 0] = 1.0
        self.router[:, 0] = bias
        state = {"dtype": torch.float32 if state_bits == 32 else torch.uint8, "device": "cuda"}
        m, v = ([torch.zeros(s, **state) for s in shapes] for _ in range(2))
        small = {}
        if state_bits == 8:
            blocks = [-(-math.prod(s) // operators.BLOCK) for s in shapes]
            small = {k: [torch.zeros(b, dtype=torch.int8, device="cuda") for b in blocks] for k in ("m_exp", "v_exp")}
        self.optimizer = operators.AdamW(self.masters, m, v, copies=self.experts, weight_decay=0.1, **small)
        self.steps = 0

    def step(self, mark=lambda name: None):
        """A training step; the optimizer's part is marked "optimizer"."""
        got = layer_step(self.x, self.router, self.experts, self.d_out, self.top_k, mark)
        self.steps += 1
        self.optimizer.step(got["d_experts"], lr=1e-4, step=self.steps, seed=self.steps)
        mark("optimizer")
        return got


def _router_step(tokens, hidden, experts, top_k, seed):
    """The router of a layer of this size, forward and backward, by itself."""
    layer = Layer(tokens, hidden, 1, experts, top_k, seed=seed)
    d_weight = torch.ones((tokens, top_k), device="cuda")
    d_x = torch.zeros((tokens, hidden), device="cuda")

    def step(mark):
        logits, r = router_forward(layer.x, layer.router, top_k)
        _, d_rest = router_backward(layer.x, layer.router, logits, r, d_weight)
        d_x.add_(d_rest)
        mark("route")
    return step


def _times(step, warmup, steps):
    """What the last of warmup + steps calls of step(mark) returned, and the median ns of what it marks, without the
    first warmup."""
    spent, got = {}, None
    for i in range(warmup + steps):
        marks = [("start", torch.cuda.Event(enable_timing=True))]
        marks[0][1].record()

        def mark(name):
            marks.append((name, torch.cuda.Event(enable_timing=True)))
            marks[-1][1].record()

        got = step(mark)
        torch.cuda.synchronize()
        if i >= warmup:
            one = {}
            for (_, a), (name, b) in zip(marks, marks[1:]):
                one[name] = one.get(name, 0.0) + a.elapsed_time(b) * 1e6
            for name, t in one.items():
                spent.setdefault(name, []).append(t)
    return got, {name: sorted(v)[len(v) // 2] for name, v in spent.items()}


def measure(problem, layer=None, steps=5, warmup=2, state_bits=32, limit_bytes=100 * 10**9, seed=0):
    """Time the MoE layer ``layer`` (the first, if None) of a problem's model on the current device.

    Where all its experts do not fit ``limit_bytes``, an equal part of them takes an equal part of the tokens and
    the times of the experts and of the rows' sum count for the whole; the router, whose work is tokens times experts,
    then runs by itself at its whole size (by equal parts of its experts, where they are more than it takes).  Returns
    ns of the parts for one micro-batch, forward and backward, the optimizer's ns a parameter and the router's counts."""
    m = problem["model"]
    moe = [i for i in range(m["n_layers"]) if m["is_moe"][i]]
    if not moe:
        raise ValueError("the model has no mixture-of-experts layer")
    layer = moe[0] if layer is None else layer
    if layer not in moe:
        raise ValueError(f"layer {layer} has no experts")
    experts, hidden, top_k = int(m["n_experts"]), int(m["hidden"]), int(m["top_k"])
    tokens = int(m["seq_len"]) * int(m["micro_batch_size"])
    width = max(1, int(m["params_expert"][layer]) // (3 * experts * hidden))
    part = 1
    while experts // part * 3 * width * hidden * STATE_BYTES[state_bits] > limit_bytes and \
            experts % (2 * part) == 0 and experts // (2 * part) >= top_k and tokens % (2 * part) == 0:
        part *= 2
    run = Layer(tokens // part, hidden, width, experts // part, top_k, state_bits, seed=seed)
    got, ns = _times(run.step, warmup, steps)
    route_ns = ns["route"]
    if part > 1:
        cut = 1   # where the router cannot take all experts at once
        while experts // cut > operators.MAX_EXPERTS:
            cut *= 2
        route_ns = _times(_router_step(tokens, hidden, experts // cut, top_k, seed), warmup, steps)[1]["route"] * cut
    params = experts // part * 3 * width * hidden
    return {"layer": layer, "tokens": tokens, "hidden": hidden, "width": width, "experts": experts, "part": part,
            "route_ns": route_ns, "combine_ns": ns["combine"] * part, "experts_ns": ns["experts"] * part,
            "opt_ns_per_param": ns["optimizer"] / params,
            "expert_tokens": got["routing"].count.cpu().numpy().astype(np.int64)}


def apply(problem, device_type, measured, shared=None, counts=True):
    """A problem whose device type has what was measured: the expert FFN's time (with its share over TP and CP as
    it was), the router's (with the rows' sum), and for all types the optimizer's time a parameter.

    counts: the router's counts, if the whole layer ran, become those of the layer measured.  They are those of a
    random router, whose experts are taken as unevenly as ``Layer``'s skew says: False where the problem's come of a
    model's own router.

    What ran are a token's top_k routed experts.  shared: experts that every token takes beside them, each counted
    as long as a routed one; None: what moe_ffn_mult has above top_k, which holds where it counts experts and not
    an expert's size."""
    out = copy.deepcopy(problem)
    m, c, h = out["model"], out["cluster"], int(device_type)
    if not 0 <= h < int(c["n_types"]):
        raise ValueError(f"device type {h} of {c['n_types']}")
    c["eff"][h] = 1.0
    c["route_coef"][h] = (measured["route_ns"] + measured["combine_ns"]) / (measured["tokens"] * measured["hidden"])
    k, mult = int(m["top_k"]), float(m["moe_ffn_mult"])
    shared = max(0.0, mult - k) if shared is None else shared
    # Eq. 2 multiplies t_ffn by moe_ffn_mult, for the routed and the shared experts together
    one = measured["experts_ns"] * (k + shared) / k / (mult or k)
    moe = np.asarray(m["is_moe"]) == 1
    was = np.asarray(c["t_ffn"][h], dtype=np.float64)
    share = np.where(was[0, 0] > 0, was / np.maximum(was[0, 0], 1.0), 1.0)   # of a (TP, CP) of the whole
    ffn = np.where(moe, np.ceil(one * share), was).astype(np.int64)
    c["t_dense"][h] = c["t_dense"][h] - c["t_ffn"][h] + ffn
    c["t_ffn"][h] = ffn
    out["params"]["opt_coef"] = measured["opt_ns_per_param"]
    if counts and measured["part"] == 1:
        m["expert_tokens"][measured["layer"]] = measured["expert_tokens"]
    return out


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--config", type=int, default=2, help="workload (1..5)")
    p.add_argument("--type", type=int, default=0, help="device type that this GPU stands for")
    p.add_argument("--state-bits", type=int, default=32, choices=(8, 32))
    p.add_argument("--steps", type=int, default=5)
    a = p.parse_args(argv)
    problem = workloads.config(a.config)
    got = measure(problem, steps=a.steps, state_bits=a.state_bits)
    print(f"layer {got['layer']}: {got['tokens']} tokens, hidden {got['hidden']}, {got['experts']} experts of width "
          f"{got['width']}" + (f", one of {got['part']} parts run" if got["part"] > 1 else ""))
    flops = 3 * 6.0 * got["tokens"] * int(problem["model"]["top_k"]) * got["hidden"] * got["width"]
    print(f"experts {got['experts_ns'] / 1e3:.0f} us ({flops / got['experts_ns'] / 1e3:.0f} TFLOP/s), router "
          f"{got['route_ns'] / 1e3:.0f} us, rows' sum {got['combine_ns'] / 1e3:.0f} us, optimizer "
          f"{got['opt_ns_per_param'] * 1e3:.2f} ps a parameter")
    for name, q in (("as given", problem), ("measured", apply(problem, a.type, got, counts=False))):
        plan = binding.Planner(q, "cuda:0").run()
        print(f"{name}: (PP, TP, CP, DP, EP, TPE) {plan['config']}, B {plan['n_micro']}, {plan['objective']} ns, layers "
              f"{plan['layers']}")


if __name__ == "__main__":
    main()

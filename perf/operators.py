"""The operators of a mixture-of-experts training step whose measured times and counts the
planner takes as input, as timed and checked cases.

  route    a token's experts: the k largest logits, their softmax weights, the count of every
           expert and the order that puts each expert's tokens together; its gradient
  combine  the sum of a token's expert outputs under its weights; its gradient
  product  matrix products grouped by expert, a ragged number of rows each; both gradients
  adamw    one AdamW step over many tensors, moments in 32 bits or in 8

``listed()`` names the cases, ``draw(rng)`` draws more of the same ranges, ``prepare`` makes a
case's inputs, ``run`` passes once through the operator: in plain torch operations, or where
``own`` is set through the package's operators.  ``work`` is what a pass cannot do without and
``exact`` the outputs in 64 bits.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2}
_BLOCK = 256   # elements of a tensor that share a scale where its moments have 8 bits

_LISTED = [
    # one decoding step of a few sequences on the 32-layer model (64 experts, top 8): latency
    {"name": "route_decode", "op": "route", "form": "forward", "tokens": 4, "experts": 64, "top_k": 8,
     "type": "f32", "renormalize": True, "padded": False},
    # eight micro-batches of the 61-layer model (256 experts, top 8), some of the tokens padding
    {"name": "route_train", "op": "route", "form": "step", "tokens": 32768, "experts": 256, "top_k": 8,
     "type": "f32", "renormalize": False, "padded": True},
    # the expert outputs of a decoding step, at the hidden size of the 61-layer model
    {"name": "combine_decode", "op": "combine", "form": "forward", "tokens": 16, "experts": 256, "top_k": 8,
     "hidden": 7168, "type": "bf16", "padded": False},
    # a micro-batch of the 32-layer model, forward and backward
    {"name": "combine_train", "op": "combine", "form": "step", "tokens": 4096, "experts": 64, "top_k": 8,
     "hidden": 4096, "type": "bf16", "padded": False},
    # decoding on the 32-layer model: a row or two an expert, the weights have to be read
    {"name": "product_decode", "op": "product", "form": "forward", "tokens": 16, "experts": 64, "top_k": 8,
     "inputs": 4096, "outputs": 2048, "type": "bf16", "grad_type": "bf16", "skew": 0.0, "gather": True},
    # a short prompt on the 61-layer model: some 16 rows for each of 256 experts
    {"name": "product_prompt", "op": "product", "form": "forward", "tokens": 512, "experts": 256, "top_k": 8,
     "inputs": 7168, "outputs": 2048, "type": "bf16", "grad_type": "bf16", "skew": 1.1, "gather": True},
    # a micro-batch of the 32-layer model, forward
    {"name": "product_forward", "op": "product", "form": "forward", "tokens": 4096, "experts": 64, "top_k": 8,
     "inputs": 4096, "outputs": 2048, "type": "bf16", "grad_type": "bf16", "skew": 1.1, "gather": True},
    # an eighth of the experts of the 96-layer model with the rows that eight ranks send, forward and backward
    {"name": "product_shard_step", "op": "product", "form": "step", "tokens": 32768, "experts": 16, "top_k": 1,
     "inputs": 8192, "outputs": 4096, "type": "bf16", "grad_type": "f32", "skew": 1.1, "gather": False},
    # sizes that no tile or vector divides, in the other type, forward and backward
    {"name": "product_odd_step", "op": "product", "form": "step", "tokens": 777, "experts": 8, "top_k": 2,
     "inputs": 1023, "outputs": 681, "type": "f16", "grad_type": "f16", "skew": 2.0, "gather": True},
    # norms and routers of the 8-layer model, which every rank holds: many small tensors, latency
    {"name": "adamw_small", "op": "adamw", "bits": 32, "copy": "none", "grad_type": "f32", "tensors": 24,
     "elements": 3413, "step": 10},
    # the experts of a layer of the 96-layer model on one of eight ranks: fp32 master and moments, bf16 copy
    {"name": "adamw_experts", "op": "adamw", "bits": 32, "copy": "bf16", "grad_type": "f32", "tensors": 16,
     "elements": 33554432, "step": 1000},
    # a sixteenth of the experts of a layer of the 61-layer model, moments in 8 bits
    {"name": "adamw_8bit", "op": "adamw", "bits": 8, "copy": "bf16", "grad_type": "bf16", "tensors": 16,
     "elements": 14680064, "step": 1000},
]


def listed():
    return [dict(c) for c in _LISTED]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["route", "combine", "product", "product", "adamw"])
    kind = rng.choice(["bf16", "f16"])
    if op == "route":
        experts = rng.choice([8, 64, 128, 256, rng.randint(8, 256)])
        return {"op": op, "form": rng.choice(["forward", "step"]), "tokens": _spread(rng, 1, 32768),
                "experts": experts, "top_k": rng.choice([1, 2, 4, 8, rng.randint(1, 8)]),
                "type": rng.choice(["f32", kind]), "renormalize": rng.random() < 0.5, "padded": rng.random() < 0.5}
    if op == "combine":
        return {"op": op, "form": rng.choice(["forward", "step"]), "tokens": _spread(rng, 1, 4096),
                "experts": rng.choice([8, 64, 256]), "top_k": rng.randint(1, 8),
                "hidden": rng.choice([1024, 4096, 7168, _spread(rng, 64, 8192)]), "type": rng.choice(["f32", kind]),
                "padded": rng.random() < 0.5}
    if op == "product":
        top_k = rng.choice([1, 2, 4, 8])
        inputs, outputs = _spread(rng, 256, 8192), _spread(rng, 256, 4096)
        if rng.random() < 0.7:   # as models have them; the others are odd ones
            inputs, outputs = -(-inputs // 128) * 128, -(-outputs // 128) * 128
        experts = rng.choice([8, 16, 64, 256, rng.randint(8, 256)])
        while experts * inputs * outputs > 256 * 7168 * 2048 // 2:
            experts //= 2
        return {"op": op, "form": rng.choice(["forward", "forward", "step"]),
                "tokens": _spread(rng, 1, 32768 // top_k), "experts": max(experts, top_k), "top_k": top_k,
                "inputs": inputs, "outputs": outputs, "type": kind, "grad_type": rng.choice(["f32", kind]),
                "skew": rng.choice([0.0, 1.1, 2.0]), "gather": rng.random() < 0.7}
    tensors = _spread(rng, 1, 64)
    return {"op": op, "bits": rng.choice([8, 32]), "copy": rng.choice(["none", kind]),
            "grad_type": rng.choice(["f32", kind]), "tensors": tensors,
            "elements": _spread(rng, 1, 200_000_000 // tensors), "step": rng.choice([1, 1000])}


# ------------------------------------------------------------------ inputs
def _normal(gen, shape, kind, scale=1.0):
    """Normal values, drawn in pieces where they are many, so that only their own type is held whole."""
    out = torch.empty(shape, dtype=_TYPES[kind], device="cuda")
    flat = out.view(-1)
    for piece in flat.split(1 << 27):
        piece.copy_(torch.randn(piece.numel(), generator=gen, device="cuda").mul_(scale))
    return out


def _choices(gen, tokens, experts, top_k, skew):
    """Each token's experts [tokens, top_k], an expert's share falling with its (shuffled) rank to the power skew."""
    rank = torch.randperm(experts, generator=gen, device="cuda").double() + 1
    noise = torch.rand((tokens, experts), generator=gen, device="cuda", dtype=torch.float64).clamp_min(1e-300)
    return torch.topk(noise.log() * rank.pow(skew), top_k, dim=1).indices


def _dispatch(expert, experts):
    """Rows sorted by expert: offset [experts + 1], and of every row the flat (token, choice) it holds; place is the
    inverse.  An expert of -1 has no row: its place and the rows left over at the end are -1."""
    flat = expert.reshape(-1).long()
    key = torch.where(flat < 0, experts, flat)
    order = torch.sort(key, stable=True).indices
    count = torch.zeros(experts + 1, dtype=torch.int64, device=key.device).index_add_(0, key, torch.ones_like(key))
    count = count[:experts]
    offset = torch.cat([count.new_zeros(1), count.cumsum(0)])
    rows = torch.arange(flat.numel(), device=key.device)
    slot = torch.where(rows < offset[-1], order, -1)
    place = torch.empty_like(order).index_copy_(0, order, rows)
    place = torch.where(flat < 0, -1, place).view(expert.shape)
    return count.int(), offset.int(), slot.int(), place.int()


def _odd(sizes):
    """Every fourth tensor is shorter by one and by its number, as norms and biases beside matrices are."""
    return [max(1, n - i) if i % 4 == 3 else n for i, n in enumerate(sizes)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": case}
    if case["op"] == "route":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        logits = _normal(gen, (T, E), case["type"], 2.0)
        logits[torch.rand((T, E), generator=gen, device="cuda") < 0.01] = -math.inf   # experts closed to a token
        state["logits"] = logits
        state["keep"] = torch.rand(T, generator=gen, device="cuda") < 0.9 if case["padded"] else None
        state["d_weight"] = _normal(gen, (T, k), "f32")
        if own:
            from paper_2609_39350_amd import operators
            state["routing"] = operators.Routing(T, E, k, "cuda")   # the buffers that a serving loop keeps
    elif case["op"] == "combine":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        expert = _choices(gen, T, E, k, 1.1)
        if case["padded"]:
            expert = torch.where(torch.rand((T, 1), generator=gen, device="cuda") < 0.9, expert, -1)
        count, offset, slot, place = _dispatch(expert, E)
        weight = torch.rand((T, k), generator=gen, device="cuda")
        state.update(slot=slot, place=place, weight=torch.where(place < 0, 0.0, weight),
                     y=_normal(gen, (T * k, case["hidden"]), case["type"]),
                     d_out=_normal(gen, (T, case["hidden"]), case["type"]))
    elif case["op"] == "product":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        count, offset, slot, place = _dispatch(_choices(gen, T, E, k, case["skew"]), E)
        x_rows = T if case["gather"] else T * k
        state.update(offset=offset, slot=slot if case["gather"] else None,
                     x=_normal(gen, (x_rows, case["inputs"]), case["type"]),
                     w=_normal(gen, (E, case["outputs"], case["inputs"]), case["type"], case["inputs"] ** -0.5))
        if case["form"] == "step":
            state["d_y"] = _normal(gen, (T * k, case["outputs"]), case["type"])
    else:
        # every tensor starts on a multiple of 256 elements of one flat buffer
        sizes = _odd([case["elements"]] * case["tensors"])
        padded = [-(-n // _BLOCK) * _BLOCK for n in sizes]
        total = sum(padded)
        starts = [sum(padded[:i]) for i in range(len(padded))]
        real = torch.zeros(total, dtype=torch.bool, device="cuda")
        for n, at in zip(sizes, starts):
            real[at:at + n] = True
        param = _normal(gen, (total,), "f32", 0.02)
        m = _normal(gen, (total,), "f32", 1e-3)
        v = _normal(gen, (total,), "f32", 1e-3).square_()
        for x in (param, m, v):
            x.mul_(real)
        decay = [0.0 if i % 4 == 3 else 0.1 for i in range(len(sizes))]
        state.update(
            sizes=sizes, starts=starts, param=param,
            copy=None if case["copy"] == "none" else param.to(_TYPES[case["copy"]]),
            grads=[_normal(gen, (n,), case["grad_type"], 1e-3) for n in sizes],
            pads=[torch.zeros(p - n, device="cuda") for n, p in zip(sizes, padded)],
            decays=decay, decay=torch.repeat_interleave(torch.tensor(decay, device="cuda"),
                                                        torch.tensor(padded, device="cuda"), output_size=total),
            hyper={"lr": 3e-4, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "step": case["step"],
                   "grad_scale": 0.5, "seed": 12345 + seed})
        del real
        if case["bits"] == 32:
            state.update(m=m, v=v)
        else:
            half = torch.full((total,), 1 << 15, dtype=torch.int32, device="cuda")
            state["m"], state["m_exp"] = _encode_m(m, half)
            state["v"], state["v_exp"] = _encode_v(v, half)
            del half
        if own:
            from paper_2609_39350_amd import operators
            part = lambda t, unit=1: [t[at // unit:at // unit + -(-n // unit)] for n, at in zip(sizes, starts)]  # noqa: E731
            small = {} if case["bits"] == 32 else {"m_exp": part(state["m_exp"], _BLOCK),
                                                   "v_exp": part(state["v_exp"], _BLOCK)}
            state["optimizer"] = operators.AdamW(
                part(param), part(state["m"]), part(state["v"]),
                copies=None if state["copy"] is None else part(state["copy"]), weight_decay=decay, **small)
    return state


# ------------------------------------------------------- the operators' calls
def _run_own(state):
    from paper_2609_39350_amd import operators
    case = state["case"]
    if case["op"] == "route":
        r = operators.route(state["logits"], case["top_k"], keep=state["keep"], renormalize=case["renormalize"],
                            out=state["routing"])
        out = {"expert": r.expert, "weight": r.weight, "count": r.count, "offset": r.offset, "slot": r.slot,
               "place": r.place}
        if case["form"] == "step":
            out["d_logits"] = operators.route_backward(state["logits"], r, state["d_weight"],
                                                       renormalize=case["renormalize"])
        return out
    if case["op"] == "combine":
        out = {"out": operators.combine(state["y"], state["place"], state["weight"])}
        if case["form"] == "step":
            out["d_y"], out["d_weight"] = operators.combine_backward(state["d_out"], state["y"], state["slot"],
                                                                     state["place"], state["weight"])
        return out
    if case["op"] == "product":
        x, w, offset, slot, k = state["x"], state["w"], state["offset"], state["slot"], case["top_k"]
        out = {"y": operators.expert_matmul(x, w, offset, slot=slot, top_k=k)}
        if case["form"] == "step":
            out["d_x"] = operators.expert_matmul_grad_x(state["d_y"], w, offset)
            out["d_w"] = operators.expert_matmul_grad_w(state["d_y"], x, offset, slot=slot, top_k=k,
                                                        dtype=_TYPES[case["grad_type"]])
        return out
    state["optimizer"].step(state["grads"], **state["hyper"])
    out = {"param": state["param"]}
    if state["copy"] is not None:
        out["copy"] = state["copy"]
    if case["bits"] == 32:
        out["m"], out["v"] = state["m"], state["v"]
    else:
        m, v = state["optimizer"].moments(torch.bfloat16)
        out.update({"m%d" % i: x for i, x in enumerate(m)}, **{"v%d" % i: x for i, x in enumerate(v)})
        out = _few(out, m, v)
    return out


def _few(out, m, v):
    """The moments of up to 16 tensors each by itself; of more, in one piece."""
    if len(m) <= 16:
        return out
    out = {k: x for k, x in out.items() if k in ("param", "copy")}
    return dict(out, m=torch.cat(m), v=torch.cat(v))


# ----------------------------------------------------------- the plain forms
def _softmax(logits, keep):
    """e = exp(x - max) in fp32 and the clean logits; a masked or NaN logit counts as -inf, and where the largest is
    +inf the share is equal among those."""
    x = logits.float()
    x = torch.where(x.isnan(), -math.inf, x)
    if keep is not None:
        x = torch.where(keep[:, None], x, -math.inf)
    top = x.amax(1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    return x, torch.where(x == top, 1.0, (x - top).exp())


def _plain_route(state):
    case, E, k = state["case"], state["case"]["experts"], state["case"]["top_k"]
    x, e = _softmax(state["logits"], state["keep"])
    value, index = torch.sort(x, dim=1, descending=True, stable=True)
    value, index = value[:, :k], index[:, :k]
    ok = value > -math.inf
    chosen = e.gather(1, index)
    total = (torch.where(ok, chosen, 0.0) if case["renormalize"] else e).sum(1, keepdim=True).clamp_min(1e-30)
    weight = torch.where(ok, chosen / total, 0.0)
    expert = torch.where(ok, index, -1)
    count, offset, slot, place = _dispatch(expert, E)
    out = {"expert": expert.int(), "weight": weight, "count": count, "offset": offset, "slot": slot, "place": place}
    if case["form"] == "step":
        g = torch.where(ok, state["d_weight"], 0.0)
        mean = (g * weight).sum(1, keepdim=True)
        if case["renormalize"]:
            d = torch.zeros_like(e).scatter_(1, index, weight * (g - mean))
        else:
            d = (e / total * -mean).scatter_add_(1, index, weight * g)
        out["d_logits"] = d.to(state["logits"].dtype)
    return out


def _plain_combine(state):
    y, place, weight = state["y"], state["place"].long(), state["weight"]
    taken = torch.where((place < 0)[..., None], 0.0, y[place.clamp_min(0)].float())
    out = {"out": (taken * weight[..., None]).sum(1).to(y.dtype)}
    if state["case"]["form"] == "step":
        d_out = state["d_out"].float()
        out["d_weight"] = (taken * d_out[:, None]).sum(2)
        slot = state["slot"].long()
        at = slot.clamp_min(0)
        d_y = d_out[at // place.shape[1]] * weight.reshape(-1)[at][:, None]
        out["d_y"] = torch.where((slot < 0)[:, None], 0.0, d_y).to(y.dtype)
    return out


def _plain_product(state):
    case, x, w, d_y = state["case"], state["x"], state["w"], state.get("d_y")
    bounds = state["offset"].tolist()
    spans = [slice(a, b) for a, b in zip(bounds, bounds[1:])]
    if state["slot"] is not None:
        x = x[state["slot"].long() // case["top_k"]]
    out = {"y": torch.cat([(x[s].float() @ w[e].float().T).to(x.dtype) for e, s in enumerate(spans)])}
    if case["form"] == "step":
        out["d_x"] = torch.cat([(d_y[s].float() @ w[e].float()).to(x.dtype) for e, s in enumerate(spans)])
        out["d_w"] = torch.stack([(d_y[s].float().T @ x[s].float()).to(_TYPES[case["grad_type"]]) for s in spans])
    return out


# Moments in 8 bits.  A block of 256 elements shares a power of two.  m: sign, 4 exponent bits of bias 7, 3 of
# mantissa, the block's largest below 2^8 units; v: 5 exponent bits of bias 15, 3 of mantissa, the largest below 2^16.
# Both round up with the probability of what is cut off, by 16 random bits; a v above zero stays above zero.
def _block_exponent(x, least):
    field = (x.view(torch.int32) >> 23 & 255).view(-1, _BLOCK).amax(1).clamp(max=254)
    return (field - 127).clamp_min(least)


def _scaled(x, exponent):
    """x * 2^-exponent, exponent one for each block."""
    factor = (127 - exponent << 23).view(torch.float32)
    return (x.view(-1, _BLOCK) * factor[:, None]).view(-1)


def _round_code(a, random, bias):
    normal = (a.view(torch.int32) + (random << 4) >> 20) - (127 - bias << 3)
    small = (a * 2.0 ** (bias + 2 + 16)).clamp(max=2.0 ** 20).to(torch.int32) + random >> 16
    code = torch.where(a < 2.0 ** (1 - bias), small, normal)
    return torch.where(a.isfinite(), code, 127 if bias == 7 else 255)


def _encode_m(m, random):
    exponent = _block_exponent(m, -119) - 7
    code = _round_code(_scaled(m.abs(), exponent), random, 7)
    return (code | (m < 0).int() << 7).to(torch.uint8), exponent.to(torch.int8)


def _encode_v(v, random):
    exponent = _block_exponent(v, -111) - 15
    code = _round_code(_scaled(v, exponent), random, 15)
    return torch.where(v > 0, code.clamp_min(1), code).to(torch.uint8), exponent.to(torch.int8)


def _decode(code, exponent, bias, signed):
    code = code.int()
    mark = 127 if signed else 255
    size = code & mark
    field, frac = size >> 3, size & 7
    value = torch.where(field == 0, frac.float() * 2.0 ** (-bias - 2),
                        ((field + 127 - bias << 23) + (frac << 20)).view(torch.float32))
    value = torch.where(size == mark, math.nan, value)
    if signed:
        value = torch.where(code > 127, -value, value)
    return _scaled(value, -exponent.int())


def _random32(seed, n):
    """32 random bits for every element index, a mix of the index and the seed."""
    low = 0xFFFFFFFF
    i = torch.arange(n, device="cuda")
    h = i * 0x9E3779B1 + (seed & low) & low
    h = h ^ ((i >> 32) * 0xC8B3A5D7 + (seed >> 32 & low) & low)
    h = (h ^ h >> 16) * 0x6C5B7F4D & low
    h = (h ^ h >> 15) * 0xB1E5A92B & low
    return h ^ h >> 16


def _plain_adamw(state):
    case, hyper, param = state["case"], state["hyper"], state["param"]
    parts = [p for g, pad in zip(state["grads"], state["pads"]) for p in (g.float(), pad)]
    g = torch.cat(parts) * hyper["grad_scale"]
    if case["bits"] == 32:
        m, v = state["m"], state["v"]
    else:
        m = _decode(state["m"], state["m_exp"], 7, True)
        v = _decode(state["v"], state["v_exp"], 15, False)
    m.mul_(hyper["beta1"]).add_(g * (1 - hyper["beta1"]))
    v.mul_(hyper["beta2"]).add_(g * (1 - hyper["beta2"]) * g)
    size = hyper["lr"] / (1 - hyper["beta1"] ** hyper["step"])
    root = 1 / math.sqrt(1 - hyper["beta2"] ** hyper["step"])
    step = m * size / (v.sqrt() * root + hyper["eps"])
    param.sub_(step + state["decay"] * hyper["lr"] * param)
    out = {"param": param}
    if state["copy"] is not None:
        out["copy"] = state["copy"].copy_(param)
    if case["bits"] == 32:
        return dict(out, m=m, v=v)
    random = _random32(hyper["seed"], param.numel())
    code, exponent = _encode_m(m, (random & 0xFFFF).int())
    state["m"].copy_(code), state["m_exp"].copy_(exponent)
    code, exponent = _encode_v(v, (random >> 16).int())
    state["v"].copy_(code), state["v_exp"].copy_(exponent)
    m = _decode(state["m"], state["m_exp"], 7, True).bfloat16()
    v = _decode(state["v"], state["v_exp"], 15, False).bfloat16()
    m, v = ([x[at:at + n] for n, at in zip(state["sizes"], state["starts"])] for x in (m, v))
    return _few(dict(out, **{"m%d" % i: x for i, x in enumerate(m)}, **{"v%d" % i: x for i, x in enumerate(v)}), m, v)


def run(state):
    if own:
        return _run_own(state)
    return {"route": _plain_route, "combine": _plain_combine, "product": _plain_product,
            "adamw": _plain_adamw}[state["case"]["op"]](state)


# ------------------------------------------------------------- what it takes
def work(case):
    if case["op"] == "route":
        T, E, k, size = case["tokens"], case["experts"], case["top_k"], _SIZE[case["type"]]
        one = T * E * size + T * k * 16 + 4 * (2 * E + 1)
        if case["form"] == "forward":
            return {"bytes": one, "flops": 4 * T * E}
        return {"bytes": one + T * E * size + T * k * 4, "flops": 8 * T * E}
    if case["op"] == "combine":
        T, k, H, size = case["tokens"], case["top_k"], case["hidden"], _SIZE[case["type"]]
        if case["form"] == "forward":
            return {"bytes": (T * k + T) * H * size + T * k * 8, "flops": 2 * T * k * H}
        return {"bytes": (2 * T * k + 2 * T) * H * size + T * k * 16, "flops": 5 * T * k * H}
    if case["op"] == "product":
        T, E, k, K, N = (case[f] for f in ("tokens", "experts", "top_k", "inputs", "outputs"))
        size, R = _SIZE[case["type"]], T * k
        # experts that some token takes: at most one a row
        used = min(E, R)
        x = (T if case["gather"] else R) * K * size
        n = 1
        moved = x + used * K * N * size + R * N * size
        if case["form"] == "step":
            n = 3
            moved += R * N * size + R * K * size + E * K * N * _SIZE[case["grad_type"]]
        return {"bytes": moved, "flops": n * 2 * R * K * N}
    n = sum(_odd([case["elements"]] * case["tensors"]))
    state = 16 if case["bits"] == 32 else 4 + 2 * 2   # both moments read and written; in 8 bits also given as values
    copy = 0 if case["copy"] == "none" else 2
    return {"bytes": n * (_SIZE[case["grad_type"]] + 8 + state + copy), "flops": 14 * n}


# -------------------------------------------------------- the same in 64 bits
def _exact_route(case, state):
    E, k, keep = case["experts"], case["top_k"], state["keep"]
    x = state["logits"].double().nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    if keep is not None:
        x[~keep] = -math.inf
    value, index = x.sort(dim=1, descending=True, stable=True)
    live = value[:, :k].isneginf().logical_not()
    prob = torch.softmax(x, 1).nan_to_num(nan=0.0)
    weight = prob.gather(1, index[:, :k]) * live
    if case["renormalize"]:
        weight = weight / weight.sum(1, keepdim=True).clamp_min(1e-300)
    expert = index[:, :k].masked_fill(~live, -1)
    flat = expert.flatten()
    one_hot = flat[:, None] == torch.arange(E, device=flat.device)
    count = one_hot.sum(0)
    offset = torch.nn.functional.pad(count.cumsum(0), (1, 0))
    # a row's place: the rows of lower experts and its own expert's earlier rows
    mine = flat.clamp_min(0)
    before = one_hot.int().cumsum(0, dtype=torch.int32).gather(1, mine[:, None])[:, 0] - 1
    place = (offset[mine] + before).masked_fill(flat < 0, -1)
    slot = torch.full_like(flat, -1)
    slot[place[flat >= 0]] = torch.nonzero(flat >= 0)[:, 0]
    out = {"expert": expert.int(), "weight": weight, "count": count.int(), "offset": offset.int(),
           "slot": slot.int(), "place": place.view_as(expert).int()}
    if case["form"] == "step":
        g = state["d_weight"].double() * live
        if case["renormalize"]:
            d = torch.zeros_like(x)
            d.scatter_(1, index[:, :k], weight * (g - (g * weight).sum(1, keepdim=True)))
        else:
            full = torch.zeros_like(x).scatter_(1, index[:, :k], g)
            d = prob * (full - (full * prob).sum(1, keepdim=True))
        out["d_logits"] = d
    return out


def _exact_combine(case, state):
    place, weight, y = state["place"].long(), state["weight"].double(), state["y"].double()
    T, k, rows = case["tokens"], case["top_k"], y.shape[0]
    out = y.new_zeros((T, case["hidden"]))
    d_y, d_weight = torch.zeros_like(y), torch.zeros_like(weight)
    d_out = state["d_out"].double()
    for j in range(k):
        t = torch.nonzero(place[:, j] >= 0)[:, 0]
        p = place[t, j]
        out[t] += weight[t, j, None] * y[p]
        d_y[p] = weight[t, j, None] * d_out[t]
        d_weight[t, j] = torch.linalg.vecdot(d_out[t], y[p])
    return {"out": out} if case["form"] == "forward" else {"out": out, "d_y": d_y, "d_weight": d_weight}


def _exact_product(case, state):
    x, w, offset = state["x"], state["w"], state["offset"].tolist()
    R, (E, N, K) = case["tokens"] * case["top_k"], w.shape
    row = torch.arange(R, device=x.device) if state["slot"] is None else state["slot"].long() // case["top_k"]
    step = case["form"] == "step"
    f64 = {"dtype": torch.float64, "device": x.device}
    out = {"y": torch.zeros((R, N), **f64)}
    if step:
        out.update(d_x=torch.zeros((R, K), **f64), d_w=torch.zeros((E, N, K), **f64))
    for e in range(E):
        a, b = offset[e], offset[e + 1]
        if a == b:
            continue
        xe, we = x[row[a:b]].double(), w[e].double()
        torch.mm(xe, we.mT.contiguous(), out=out["y"][a:b])
        if step:
            de = state["d_y"][a:b].double()
            torch.mm(de, we, out=out["d_x"][a:b])
            torch.mm(de.mT.contiguous(), xe, out=out["d_w"][e])
    return out


def _exact_moment(code, exponent, signed):
    """The values of 8-bit moments in 64 bits."""
    table = torch.arange(256, dtype=torch.float64, device=code.device)
    field, frac = (table % 128 if signed else table).div(8, rounding_mode="floor"), table % 8
    bias = 7 if signed else 15
    table = torch.where(field > 0, (8 + frac) * 2.0 ** (field - 3 - bias), frac * 2.0 ** (-2 - bias)) \
        * torch.where(table >= 128, -1.0, 1.0) ** int(signed)
    return (table[code.long()].view(-1, _BLOCK) * 2.0 ** exponent.double()[:, None]).view(-1)


def _exact_stored(x, random, top, least, keep):
    """What a moment is after rounding to 4 significant bits, or to the least unit, up with the chance of the rest."""
    big = x.abs().view(-1, _BLOCK).amax(1)
    exponent = torch.frexp(big).exponent - 1
    exponent = torch.where(big > 0, exponent, -127).clamp_min(-119 if top == 7 else -111) - top
    a = x.abs().view(-1, _BLOCK) * 2.0 ** -exponent.double()[:, None]
    unit = 2.0 ** ((torch.frexp(a).exponent - 1).clamp_min(least).double() - 3)
    unit = torch.where(a > 0, unit, 2.0 ** (least - 3))
    level = (a / unit + random.double().view(-1, _BLOCK) / 65536).floor()
    if keep:
        level = torch.where(a > 0, level.clamp_min(1), level)
    return (level * unit * 2.0 ** exponent.double()[:, None]).view(-1) * x.sign()


def _exact_adamw(case, state):
    h = state["hyper"]
    n = state["param"].numel()
    f64 = {"dtype": torch.float64, "device": "cuda"}
    grad = torch.zeros(n, **f64)
    decay = torch.zeros(n, **f64)
    for g, at, d in zip(state["grads"], state["starts"], state["decays"]):
        grad[at:at + g.numel()] = g.double() * h["grad_scale"]
        decay[at:at + g.numel()] = d
    if case["bits"] == 32:
        m, v = state["m"].double(), state["v"].double()
    else:
        m = _exact_moment(state["m"], state["m_exp"], True)
        v = _exact_moment(state["v"], state["v_exp"], False)
    m = h["beta1"] * m + (1 - h["beta1"]) * grad
    v = h["beta2"] * v + (1 - h["beta2"]) * grad ** 2
    m_hat, v_hat = m / (1 - h["beta1"] ** h["step"]), v / (1 - h["beta2"] ** h["step"])
    p = state["param"].double()
    p = p * (1 - h["lr"] * decay) - h["lr"] * m_hat / (v_hat.sqrt() + h["eps"])
    out = {"param": p}
    if state["copy"] is not None:
        out["copy"] = p
    if case["bits"] == 32:
        return dict(out, m=m, v=v)
    del grad, decay, m_hat, v_hat
    bits = _random32(h["seed"], n)
    m = _exact_stored(m, bits % 65536, 7, -6, False)
    v = _exact_stored(v, bits // 65536, 15, -14, True)
    m, v = ([x[at:at + n] for n, at in zip(state["sizes"], state["starts"])] for x in (m, v))
    return _few(dict(out, **{"m%d" % i: x for i, x in enumerate(m)}, **{"v%d" % i: x for i, x in enumerate(v)}), m, v)


def exact(case, seed):
    global own
    kept, own = own, False   # the inputs alone
    try:
        state = prepare(case, seed)
    finally:
        own = kept
    return {"route": _exact_route, "combine": _exact_combine, "product": _exact_product,
            "adamw": _exact_adamw}[case["op"]](case, state)

"""More operators of a transformer layer's training whose speed counts: RMS norm, rotary positions, AdamW.

Beside attention, layer norm and clipping, a layer of a present-day decoder and the step that ends its training take

  rms      h = x + residual in x's type, the norm of h by its root mean square, times weights, as y in x's type and/or as
           codes of 8 bits with a scale for each row, or for each group of columns; and dx, dweight (backward)
  rotary   pairs of each head's first `rot` values turned by position times frequency, for queries and keys together
           (forward), and the same backwards for their gradients
  adamw    one step over all tensors of a model's part: parameters in 32 bits, a copy of them in the type that products
           read, first and second moments in 32 bits, or in 8 with a scale for each 256 values

Layouts: x [rows][cols]; q [B][L][Hq][D], k [B][L][Hk][D].  A pair is (i, i + rot / 2), or (2 i, 2 i + 1) where
interleaved.  8 bits are e4m3: a value x of a group is held as round(x / scale), scale = max(largest |x| / 448, 2^-126).
AdamW holds the square root of the second moment, and rounds both up or down at random, in proportion (to the nearest,
moments that change by less than half a step a time would never change); a root that is not 0 is never held as 0.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
F8, TOP, LEAST, LEAST_SCALE = torch.float8_e4m3fn, 448.0, 2.0 ** -9, 2.0 ** -126
EPS = 1e-5
ADAM = dict(lr=1e-4, beta1=0.9, beta2=0.999, eps=1e-8)
DECAY, MAX_NORM, FIRST_STEP = 0.1, 1.0, 100
BLOCK = 256      # values that share a scale in AdamW's states; the flat buffers' tensors start at multiples of it
SEED = 20231        # of the random numbers that AdamW rounds by: a hash of seed, step and the value's place
THETA, ORIGINAL, BY = 10000.0, 4096.0, 8.0     # frequencies of positions up to 4096, scaled for 8 times as many


def listed():
    rms = dict(op="rms", train=False, dtype="bf16", wdtype="f32", rows=8192, cols=5120, residual=True, out="y", group=0)
    rotary = dict(op="rotary", train=False, dtype="bf16", B=4, L=2048, Hq=40, Hk=40, D=128, rot=128, interleaved=False,
                  scaling="none", far=0, ragged=False)
    adamw = dict(op="adamw", dtype="bf16", copy="bf16", bits=32, hidden=1280, layers=1, clip=True)
    return [
        # Four tokens of a decoder that answers (hidden 5120), the product behind the norm in 8 bits: latency.
        dict(rms, name="rms_token_8", rows=4, out="q"),
        # A prompt's 8192 tokens, 8 bits alone, a scale for each 128 columns.
        dict(rms, name="rms_prompt_8", out="q", group=128),
        # Training of an encoder's layer in 32 bits, no residual, a row length off every tile edge.
        dict(rms, name="rms_train_odd", train=True, dtype="f32", rows=6304, cols=1283, residual=False),
        # Training of a decoder's layer: 16384 tokens of 5120 values.
        dict(rms, name="rms_train_5120", train=True, rows=16384),
        # One new token for each of 64 sequences at far positions, eight key heads, frequencies scaled.
        dict(rotary, name="rotary_token", B=64, L=1, Hq=32, Hk=8, scaling="ramp", far=131072),
        # A part of heads of 80, pairs next to each other, short samples padded to the longest, forward and backward.
        dict(rotary, name="rotary_train_part", train=True, dtype="f16", B=32, L=197, Hq=16, Hk=16, D=80, rot=40,
             interleaved=True, ragged=True),
        # One long prompt behind a longer one, key heads shared by four.
        dict(rotary, name="rotary_prompt", B=1, L=16384, Hq=32, Hk=8, scaling="base", far=65536),
        # Training of a decoder's layer: 4 x 2048 tokens, 40 heads of 128.
        dict(rotary, name="rotary_train_2048", train=True),
        # The step of a small part (hidden 128, one layer), states in 8 bits: latency.
        dict(adamw, name="adamw_small_8", hidden=128, bits=8),
        # The step of one encoder layer (hidden 1280), everything in 32 bits, gradients as they are.
        dict(adamw, name="adamw_layer", dtype="f32", copy="", clip=False),
        # A pipeline stage of twelve such layers, states in 8 bits.
        dict(adamw, name="adamw_stage_8", layers=12, bits=8),
        # The same with states in 32 bits: the largest.
        dict(adamw, name="adamw_stage", layers=12),
    ]


MOST_NORM = 16384.0 * 5120
MOST_ROTARY = 4.0 * 2048 * 80 * 128
MOST_LAYERS = 12


def draw(rng):
    def log(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    op = rng.choice(["rms", "rotary", "adamw"])
    if op == "rms":
        while True:
            c = dict(op=op, train=rng.random() < 0.5, dtype=rng.choice(["f32", "f16", "bf16", "bf16"]), wdtype="f32",
                     rows=log(1, 65536), cols=log(64, 10240), residual=rng.random() < 0.6,
                     out=rng.choice(["y", "y", "q", "both"]), group=rng.choice([0, 0, 32, 64, 128]))
            if rng.random() < 0.3:
                c["wdtype"] = c["dtype"]
            if c["out"] == "y":
                c["group"] = 0
            if c["rows"] * c["cols"] <= MOST_NORM:
                return c
    if op == "adamw":
        return dict(op=op, dtype=rng.choice(["f32", "f16", "bf16", "bf16"]), copy=rng.choice(["", "f16", "bf16"]),
                    bits=rng.choice([8, 32]), hidden=log(100, 1280), layers=log(1, MOST_LAYERS), clip=rng.random() < 0.6)
    while True:
        Hk, D = log(1, 40), rng.choice([40, 64, 64, 80, 96, 128, 128])
        c = dict(op=op, train=rng.random() < 0.5, dtype=rng.choice(["f32", "f16", "bf16", "bf16"]), B=log(1, 64),
                 L=log(1, 16384), Hq=Hk * rng.choice([1, 1, 2, 4, 8]), Hk=Hk, D=D,
                 rot=rng.choice([D, D, D, D // 2, 2 * rng.randint(2, D // 2)]), interleaved=rng.random() < 0.4,
                 scaling=rng.choice(["none", "linear", "base", "ramp"]), far=rng.choice([0, 0, 4096, 131072, 1 << 20]),
                 ragged=rng.random() < 0.4)
        if 1e3 <= c["B"] * c["L"] * float(c["Hq"] + Hk) * D <= MOST_ROTARY and c["Hq"] <= 64:
            return c


def lengths(case):
    """The samples' lengths: from full ones down to half, the same multiset for every seed."""
    part = [1.0 - 0.5 * b / case["B"] if case["ragged"] else 1.0 for b in range(case["B"])]
    return [max(1, round(case["L"] * p)) for p in part]


def tensor_sizes(case):
    """The parameter tensors of a layer, and whether they decay: products into q, k, v, out of the heads, into two gates,
    down again, their biases and two norms' weights."""
    h = case["hidden"]
    f = 2 * h
    return case["layers"] * [(3 * h * h, 1), (3 * h, 0), (h * h, 1), (h, 0), (2 * f * h, 1), (2 * f, 0), (f * h, 1),
                             (h, 0), (h, 0), (h, 0)]


def padded(n):
    return -(-n // BLOCK) * BLOCK


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.float32, spread=1.0, middle=0.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * spread + middle).to(dtype)

    st = dict(case=case)
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "rms":
        rows, cols, wdtype = case["rows"], case["cols"], DTYPES[case["wdtype"]]
        st["x"] = normal(rows, cols, dtype=dtype)
        st["residual"] = normal(rows, cols, dtype=dtype, spread=2.0) if case["residual"] else None
        st["weight"] = normal(cols, dtype=wdtype, spread=0.2, middle=1.0)
        if case["train"]:
            st["dy"] = normal(rows, cols, dtype=dtype, spread=0.1)
            # the gradient that reaches h past this norm
            st["dres"] = normal(rows, cols, dtype=dtype, spread=0.1) if case["residual"] else None
    elif case["op"] == "rotary":
        B, L, Hq, Hk, D = (case[n] for n in ("B", "L", "Hq", "Hk", "D"))
        # q and k are what a layer's one product into q, k and v leaves
        qkv = normal(B, L, (Hq + 2 * Hk) * D, dtype=dtype)
        st["q"], st["k"], _ = (t.unflatten(2, (-1, D)) for t in qkv.split([Hq * D, Hk * D, Hk * D], 2))
        if case["train"]:
            st["dq"], st["dk"] = normal(B, L, Hq, D, dtype=dtype, spread=0.1), normal(B, L, Hk, D, dtype=dtype, spread=0.1)
        st["positions"] = st["len"] = None
        if case["far"]:
            start = torch.randint(0, case["far"], (B, 1), generator=gen, device="cuda")
            st["positions"] = (start + torch.arange(L, device="cuda")).to(torch.int32)
        st["factor"] = 0.1 * math.log(BY) + 1.0 if case["scaling"] == "ramp" else 1.0
        names = [("q_out", Hq), ("k_out", Hk)] + ([("dq_out", Hq), ("dk_out", Hk)] if case["train"] else [])
        st.update((n, None) for n, _ in names)
        if case["ragged"]:
            turn, n = seed % B, lengths(case)
            st["len"] = torch.tensor(n[turn:] + n[:turn], dtype=torch.int32, device="cuda")
            # the program's own buffers: what is behind a sample's length stays as it is
            st.update((name, torch.zeros(B, L, H, D, dtype=dtype, device="cuda")) for name, H in names)
        if own:
            import paper_2307_02031_amd as g
            how = dict(none={}, linear=dict(by=BY), base=dict(by=BY), ramp=dict(by=BY, original=ORIGINAL))
            st["freq"] = g.gbmw_rotary_frequencies(case["rot"], THETA, case["scaling"], **how[case["scaling"]])
    else:
        sizes = [n for n, _ in tensor_sizes(case)]
        room = [padded(n) for n in sizes]
        there = torch.zeros(sum(room), dtype=torch.bool, device="cuda")
        for t, n in zip(there.split(room), sizes):
            t[:n] = True

        def flat(spread, kind=torch.float32):     # zeros between the tensors
            return torch.where(there, normal(sum(room), spread=spread), 0.0).to(kind)

        # gradients of one tensor after the other in one buffer, as a bucket for their sum over devices has them
        spread = torch.tensor([10.0 ** -(2 + i % 3) for i in range(len(room))], device="cuda")
        spread = torch.repeat_interleave(spread, torch.tensor(room, device="cuda"))
        st["grad"] = flat(spread, dtype)
        st["param"] = flat(0.03)
        st["copy"] = torch.zeros(sum(room), dtype=DTYPES[case["copy"]], device="cuda") if case["copy"] else None
        st["m"] = flat(spread * 0.3)
        st["v"] = torch.where(there, flat(spread).abs() + 0.5 * spread, 0.0).square_()
        st["m_scale"] = st["v_scale"] = None
        if case["bits"] == 8:
            st["m"], st["m_scale"] = codes(st["m"], BLOCK, F8)
            st["v"], st["v_scale"] = codes(st["v"].sqrt(), BLOCK, F8, least=LEAST)
        st["norm"] = torch.rand(1, generator=gen, device="cuda") * 3.0 + 0.5 if case["clip"] else None
        st["step"] = FIRST_STEP
        st["decay"] = torch.tensor([DECAY * d for _, d in tensor_sizes(case)], device="cuda")
        st["blocks"] = torch.tensor([r // BLOCK for r in room], device="cuda")
        if own:
            import paper_2307_02031_amd as g
            parts = lambda t: None if t is None else [p[:n] for p, n in zip(t.split(room), sizes)]
            scales = lambda t: None if t is None else list(t.split([r // BLOCK for r in room]))
            st["list"] = g.gbmw_adamw_list_create(
                parts(st["param"]), parts(st["grad"]), parts(st["m"]), parts(st["v"]), m_scales=scales(st["m_scale"]),
                v_scales=scales(st["v_scale"]), copies=parts(st["copy"]),
                weight_decay=[DECAY * d for _, d in tensor_sizes(case)])
    return st


def run(state):
    return (run_own if own else run_plain)(state)


def run_own(st):
    import paper_2307_02031_amd as g
    case = st["case"]
    if case["op"] == "rms":
        r = g.gbmw_rms_norm_forward(st["x"], st["weight"], EPS, residual=st["residual"],
                                    qtype=None if case["out"] == "y" else F8, group=case["group"],
                                    want_y=case["out"] != "q")
        res = dict(y=r.y, h=r.h if case["residual"] else None, rstd=r.rstd, q=r.q, scale=r.scale)
        if case["train"]:
            res["dx"], res["dweight"] = g.gbmw_rms_norm_backward(st["dy"], r.h, st["weight"], r.rstd, dres=st["dres"])
        return res
    if case["op"] == "rotary":
        how = dict(positions=st["positions"], len_x=st["len"], interleaved=case["interleaved"], factor=st["factor"])
        q, k = g.gbmw_rotary_forward(st["q"], st["k"], st["freq"], q_out=st["q_out"], k_out=st["k_out"], **how)
        res = dict(q=q, k=k)
        if case["train"]:
            res["dq"], res["dk"] = g.gbmw_rotary_backward(st["dq"], st["dk"], st["freq"], q_out=st["dq_out"],
                                                          k_out=st["dk_out"], **how)
        return res
    st["step"] += 1
    g.gbmw_adamw_step(st["list"], ADAM["lr"], st["step"], ADAM["beta1"], ADAM["beta2"], ADAM["eps"], norm=st["norm"],
                      max_norm=MAX_NORM, seed=SEED)
    return {n: st[n] for n in ("param", "copy", "m", "v", "m_scale", "v_scale")}


# ---- the plain forms: 32 bits, rounded once at the end --------------------------------------------------------------

def run_plain(st):
    return dict(rms=plain_rms, rotary=plain_rotary, adamw=plain_adamw)[st["case"]["op"]](st)


def codes(x, group, kind, least=0.0, random=None):
    """Codes of 8 bits like x, whose last axis is cut into groups, and a scale for each; nothing that is not 0 is held
    as less than `least` times the scale.  random: numbers of [0, 1), one for each value; rounded up where the part
    that is cut off is more than 1 less the number."""
    cols = x.shape[-1]
    g = torch.nn.functional.pad(x, (0, -cols % group)).unflatten(-1, (-1, group))
    scale = (g.abs().amax(-1) / TOP).clamp_min(LEAST_SCALE)
    c = g / scale.unsqueeze(-1)
    if least:
        c = torch.where(g > 0, c.clamp_min(least), c)
    if random is not None:
        step = torch.ldexp(torch.ones_like(c), (torch.frexp(c).exponent - 1).clamp_min(-6) - 3)
        c = torch.copysign(torch.floor(c.abs().clamp_max(TOP) / step + random.view_as(c)) * step, c)
    return c.flatten(-2)[..., :cols].contiguous().to(kind), scale


def plain_rms(st):
    case, dtype = st["case"], st["x"].dtype
    h = st["x"] if st["residual"] is None else (st["x"].float() + st["residual"].float()).to(dtype)
    s, w = h.float(), st["weight"].float()
    rstd = 1.0 / torch.sqrt((s * s).mean(1, keepdim=True) + EPS)
    y = s * rstd * w
    res = dict(y=y.to(dtype) if case["out"] != "q" else None, h=h if case["residual"] else None, rstd=rstd.squeeze(1),
               q=None, scale=None)
    if case["out"] != "y":
        res["q"], res["scale"] = codes(y, case["group"] or case["cols"], F8)
    if case["train"]:
        dy, xhat = st["dy"].float(), s * rstd
        g = dy * w
        dx = (g - xhat * (g * xhat).mean(1, keepdim=True)) * rstd
        if st["dres"] is not None:
            dx = dx + st["dres"].float()
        res.update(dx=dx.to(dtype), dweight=(dy * xhat).sum(0).to(st["weight"].dtype))
    return res


def plain_frequencies(case):
    i = torch.arange(case["rot"] // 2, dtype=torch.float64, device="cuda")
    theta = THETA * BY ** (case["rot"] / (case["rot"] - 2)) if case["scaling"] == "base" else THETA
    freq = theta ** (-2.0 * i / case["rot"])
    if case["scaling"] == "linear":
        return freq / BY
    if case["scaling"] == "ramp":     # all of it where it turns 32 times in the original length, scaled where once
        part = ((ORIGINAL * freq / (2.0 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
        return part * freq + (1.0 - part) * freq / BY
    return freq


def plain_rotary(st):
    case = st["case"]
    B, L, rot = case["B"], case["L"], case["rot"]
    pos = torch.arange(L, device="cuda").unsqueeze(0) if st["positions"] is None else st["positions"]
    angle = (pos.double().unsqueeze(2) * plain_frequencies(case)).unsqueeze(2)
    cos, sin = torch.cos(angle).float() * st["factor"], torch.sin(angle).float() * st["factor"]
    first = slice(0, rot, 2) if case["interleaved"] else slice(0, rot // 2)
    second = slice(1, rot, 2) if case["interleaved"] else slice(rot // 2, rot)

    def turned(x, out, sin):
        a, b = x[..., first].float(), x[..., second].float()
        y = x.clone(memory_format=torch.contiguous_format)
        y[..., first] = (a * cos - b * sin).to(x.dtype)
        y[..., second] = (a * sin + b * cos).to(x.dtype)
        if st["len"] is None:
            return y
        there = torch.arange(L, device="cuda").view(1, L, 1, 1) < st["len"].view(B, 1, 1, 1)
        return out.copy_(torch.where(there, y, out))

    res = dict(q=turned(st["q"], st["q_out"], sin), k=turned(st["k"], st["k_out"], sin))
    if case["train"]:
        res.update(dq=turned(st["dq"], st["dq_out"], -sin), dk=turned(st["dk"], st["dk_out"], -sin))
    return res


def bits(x):      # a hash of 32 bits
    x = (x * 0x9E3779B1) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x85EBCA77) & 0xFFFFFFFF
    return x ^ (x >> 13)


def plain_adamw(st):
    case, a = st["case"], ADAM
    st["step"] += 1
    grad = st["grad"].float()
    if st["norm"] is not None:
        grad = grad * torch.where(st["norm"] > MAX_NORM, MAX_NORM / st["norm"], 1.0)
    held = lambda c, scale: (c.float().view(-1, BLOCK) * scale.unsqueeze(1)).view(-1)
    if case["bits"] == 8:
        m, v = held(st["m"], st["m_scale"]), held(st["v"], st["v_scale"]).square()
    else:
        m, v = st["m"], st["v"]
    m = m * a["beta1"] + grad * (1.0 - a["beta1"])
    v = v * a["beta2"] + grad * grad * (1.0 - a["beta2"])
    root = torch.sqrt(v)
    c1, c2 = 1.0 - a["beta1"] ** st["step"], 1.0 - a["beta2"] ** st["step"]
    keep = (1.0 - a["lr"] * torch.repeat_interleave(st["decay"], st["blocks"])).unsqueeze(1)
    step = m / (root * (1.0 / math.sqrt(c2)) + a["eps"]) * (a["lr"] / c1)
    st["param"].copy_((st["param"].view(-1, BLOCK) * keep).view(-1) - step)
    if st["copy"] is not None:
        st["copy"].copy_(st["param"])
    if case["bits"] == 8:
        key = bits((SEED + st["step"] * 0x9E3779B9) & 0xFFFFFFFF)
        word = bits(torch.arange(m.numel(), device="cuda") ^ key)
        high, low = ((w.float() + 0.5) / 65536.0 for w in (word >> 16, word & 65535))
        c, scale = codes(m, BLOCK, F8, random=high)
        st["m"].copy_(c), st["m_scale"].copy_(scale)
        c, scale = codes(root, BLOCK, F8, least=LEAST, random=low)
        st["v"].copy_(c), st["v_scale"].copy_(scale)
    else:
        st["m"].copy_(m), st["v"].copy_(v)
    return {n: st[n] for n in ("param", "copy", "m", "v", "m_scale", "v_scale")}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    size = {"f32": 4, "f16": 2, "bf16": 2, "": 0}
    s = size[case["dtype"]]
    if case["op"] == "rms":
        n, w, some = case["rows"] * case["cols"], case["cols"] * size[case["wdtype"]], int(case["residual"])
        parts = -(-case["cols"] // case["group"]) if case["group"] else 1
        moved = n * s * (1 + 2 * some) + w + 4 * case["rows"]
        if case["out"] != "q":
            moved += n * s
        if case["out"] != "y":
            moved += n + 4 * case["rows"] * parts
        if not case["train"]:
            return dict(bytes=moved, flops=(5.0 + some) * n)
        return dict(bytes=moved + n * s * (2 + some) + w, flops=(14.0 + 2 * some) * n)
    if case["op"] == "rotary":
        heads, passes = sum(lengths(case)) * (case["Hq"] + case["Hk"]), 2 if case["train"] else 1
        turns = 0 if not case["far"] else 4 * sum(lengths(case))
        return dict(bytes=2.0 * heads * case["D"] * s * passes + turns, flops=3.0 * heads * case["rot"] * passes)
    n = sum(k for k, _ in tensor_sizes(case))
    states = 2 * 8 if case["bits"] == 32 else 2 * 2
    scales = 0 if case["bits"] == 32 else 16 * sum(padded(k) // BLOCK for k, _ in tensor_sizes(case))
    return dict(bytes=n * (s + 8 + states + size[case["copy"]]) + scales, flops=(15.0 if case["bits"] == 32 else 24.0) * n)


# ---- the definition in 64 bits --------------------------------------------------------------------------------------

def exact(case, seed):
    return dict(rms=exact_rms, rotary=exact_rotary, adamw=exact_adamw)[case["op"]](prepare(case, seed), case)


def exact_scale(y, group):
    """The scale of each of y's groups of columns, and each column's."""
    cols = y.shape[1]
    scale = torch.stack([c.abs().amax(1) for c in y.split(group, 1)], 1).div(448).clamp(min=2.0 ** -126)
    return scale, scale.repeat_interleave(group, 1)[:, :cols]


def exact_rms(st, case):
    h = st["x"].double()
    if case["residual"]:
        h = h.add(st["residual"].double()).to(st["x"].dtype).double()     # h is what is normed
    n, w = case["cols"], st["weight"].double()
    rstd = torch.rsqrt(torch.linalg.vector_norm(h, dim=1).square() / n + EPS)
    xhat = h * rstd[:, None]
    y = torch.mul(xhat, w)
    res = dict(y=y if case["out"] != "q" else None, h=h if case["residual"] else None, rstd=rstd, q=None, scale=None)
    if case["out"] != "y":
        res["scale"], each = exact_scale(y, case["group"] or n)
        res["q"] = y / each
    if case["train"]:
        dy = st["dy"].double()
        along = torch.linalg.vecdot(dy * w, xhat) / n
        dx = torch.addcmul(dy * w, xhat, along[:, None], value=-1) * rstd[:, None]
        res["dx"] = dx if st["dres"] is None else st["dres"].double().add(dx)
        res["dweight"] = torch.linalg.vecdot(dy, xhat, dim=0)
    return res


def exact_rotary(st, case):
    B, L, D, rot = case["B"], case["L"], case["D"], case["rot"]
    freq = []
    for i in range(rot // 2):
        f = math.exp(-2 * i * math.log(THETA) / rot)
        if case["scaling"] == "base":
            f *= BY ** (-2 * i / (rot - 2))
        elif case["scaling"] == "linear":
            f /= BY
        elif case["scaling"] == "ramp":
            turns = ORIGINAL * f / (2 * math.pi)
            share = min(1.0, max(0.0, (turns - 1) / (32 - 1)))
            f = f / BY + share * (f - f / BY)
        freq.append(f)
    freq = torch.tensor(freq, dtype=torch.float64, device="cuda")
    pos = torch.arange(L, device="cuda").expand(B, L) if st["positions"] is None else st["positions"]
    turn = torch.polar(torch.full((), st["factor"], dtype=torch.float64, device="cuda"), pos.double()[..., None] * freq)[:, :, None]
    n = [L] * B if st["len"] is None else st["len"].tolist()

    def turned(x, turn):
        x = x.double()
        head = x[..., :rot]
        pairs = head.unflatten(3, (-1, 2)) if case["interleaved"] else head.unflatten(3, (2, -1)).transpose(3, 4)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        out = torch.cat([(z if case["interleaved"] else z.transpose(3, 4)).flatten(3), x[..., rot:]], 3)
        for b in range(B):
            out[b, n[b]:] = 0
        return out

    res = dict(q=turned(st["q"], turn), k=turned(st["k"], turn))
    if case["train"]:
        res.update(dq=turned(st["dq"], turn.conj()), dk=turned(st["dk"], turn.conj()))
    return res


def exact_adamw(st, case):
    t, b1, b2 = FIRST_STEP + 1, ADAM["beta1"], ADAM["beta2"]
    g = st["grad"].double()
    if case["clip"]:
        norm = float(st["norm"])
        g *= min(1.0, MAX_NORM / norm)
    if case["bits"] == 8:
        m = st["m"].double() * st["m_scale"].double().repeat_interleave(BLOCK)
        v = (st["v"].double() * st["v_scale"].double().repeat_interleave(BLOCK)) ** 2
    else:
        m, v = st["m"].double(), st["v"].double()
    m = torch.lerp(g, m, b1)
    v = torch.lerp(g ** 2, v, b2)
    change = (m / -math.expm1(t * math.log(b1))) / ((v / -math.expm1(t * math.log(b2))).sqrt() + ADAM["eps"])
    decay = torch.cat([torch.full((padded(n),), DECAY * d, dtype=torch.float64, device="cuda") for n, d in tensor_sizes(case)])
    p = st["param"].double()
    p -= ADAM["lr"] * (change + decay * p)
    res = dict(param=p, copy=p if case["copy"] else None, m=m, v=v, m_scale=None, v_scale=None)
    if case["bits"] == 8:
        for name, x in (("m", m.view(-1, BLOCK)), ("v", v.sqrt().view(-1, BLOCK))):
            scale, each = exact_scale(x, BLOCK)
            res[name], res[name + "_scale"] = (x / each).view(-1), scale.view(-1)
    return res

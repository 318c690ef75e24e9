"""The operators of a transformer layer's training whose speed counts: attention, layer norm, gradient clipping.

A planner's cost model needs the time of one layer on one device (forward, backward and the optimizer step's share of
it).  Beside the matrix products a layer spends it in the operators here:

  attention   out and the rows' log-sum-exp from q, k, v (forward), and dq, dk, dv from those (backward)
  norm        layer norm over the last axis (forward), and dx, dweight, dbias (backward)
  clip        the norm of all gradients of a model's part, and the gradients scaled to at most that norm, written in
              the type that the optimizer reads

Layouts: q [B][Lq][Hq][D], k and v [B][Lk][Hk][D] (Hq a multiple of Hk: query head h reads key head h / (Hq / Hk)).
Sample b has len_q[b] queries and len_k[b] keys; query i sees key j < len_k[b], with a causal mask
j <= i + len_k[b] - len_q[b].  A row that sees no key, or is beyond len_q[b], has output 0 and log-sum-exp -inf, and
passes no gradient on.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
NORM_EPS = 1e-5
MAX_NORM = 1.0


def listed():
    attn = dict(op="attention", train=False, dtype="bf16", B=1, Hq=16, Hk=16, Lq=512, Lk=512, D=64, causal=False,
                ragged=False)
    norm = dict(op="norm", train=False, dtype="bf16", wdtype="f32", rows=512, cols=1280)
    clip = dict(op="clip", dtype="bf16", out="f32", hidden=1280, layers=1)
    return [
        # A decoder of four targets that attends to the 512 encoder outputs of eight sources: a call's latency.
        dict(attn, name="attn_short", B=8, Lq=4, Lk=512, ragged=True),
        # One new token for each of four sequences, over thousands of keys that eight heads share: the serving form.
        dict(attn, name="attn_token", B=4, Hq=32, Hk=8, Lq=1, Lk=6000, D=128, causal=True, ragged=True),
        # Inference of a decoder layer (hidden 5120, 2048 tokens: a row of the planner's model table).
        dict(attn, name="attn_causal", B=4, Hq=40, Hk=40, Lq=2048, Lk=2048, D=128, causal=True),
        # Training of an image encoder's layer (hidden 1280, 197 patches): odd lengths, heads of 80.
        dict(attn, name="attn_train_197", train=True, dtype="f16", B=32, Lq=197, Lk=197, D=80),
        # Training of a text encoder's layer (hidden 1280, 512 tokens), sentences padded to the longest.
        dict(attn, name="attn_train_512", train=True, B=16, Hq=20, Hk=20, ragged=True),
        # Training of a decoder's layer (hidden 5120, 2048 tokens), two samples.
        dict(attn, name="attn_train_2048", train=True, B=2, Hq=40, Hk=40, Lq=2048, Lk=2048, D=128, causal=True),
        # Training on one long document, key heads shared by four query heads: the largest.
        dict(attn, name="attn_train_8192", train=True, Hq=32, Hk=8, Lq=8192, Lk=8192, D=128, causal=True),
        # The norm of one sample's 512 tokens: latency.
        dict(norm, name="norm_512"),
        # Training, 32 samples of 197 patches, in 32 bits throughout, a row length off every tile edge.
        dict(norm, name="norm_train_odd", train=True, dtype="f32", rows=6304, cols=1283),
        # Training of a decoder's layer: 16384 tokens of 5120 values.
        dict(norm, name="norm_train_5120", train=True, rows=16384, cols=5120),
        # The gradients of one encoder layer (hidden 1280) in 32 bits.
        dict(clip, name="clip_layer", dtype="f32"),
        # The gradients of a pipeline stage of twelve such layers, bf16 in, 32 bits for the optimizer.
        dict(clip, name="clip_stage", layers=12),
    ]


MOST_PAIRS = 32.0 * 8192 * 8192 * 128     # B Hq Lq Lk D of the largest listed attention
MOST_NORM = 16384.0 * 5120
MOST_CLIP = 12


def draw(rng):
    def log(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    op = rng.choice(["attention", "attention", "attention", "norm", "clip"])
    if op == "norm":
        while True:
            c = dict(op=op, train=rng.random() < 0.7, dtype=rng.choice(["f32", "f16", "bf16", "bf16"]), wdtype="f32",
                     rows=log(1, 65536), cols=log(64, 10240))
            if rng.random() < 0.3:
                c["wdtype"] = c["dtype"]
            if c["rows"] * c["cols"] <= MOST_NORM:
                return c
    if op == "clip":
        dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
        return dict(op=op, dtype=dtype, out=rng.choice([dtype, "f32"]), hidden=log(100, 1280), layers=log(1, MOST_CLIP))
    while True:
        Hk, Lk = log(1, 40), log(1, 8192)
        c = dict(op=op, train=rng.random() < 0.6, dtype=rng.choice(["f16", "bf16", "bf16"]), B=log(1, 64),
                 Hq=Hk * rng.choice([1, 1, 2, 4, 8]), Hk=Hk, Lq=rng.choice([Lk, Lk, log(1, Lk)]), Lk=Lk,
                 D=rng.choice([40, 64, 64, 80, 96, 128, 128]), causal=rng.random() < 0.5, ragged=rng.random() < 0.5)
        if 1e4 <= c["B"] * c["Hq"] * float(c["Lq"]) * Lk * c["D"] <= MOST_PAIRS and c["Hq"] <= 64 \
                and c["B"] * c["Hq"] * max(c["Lq"], Lk) * c["D"] <= 2.5e8:
            return c


def lengths(case):
    """The samples' lengths (queries, keys): from full ones down to half, the same multiset for every seed."""
    B = case["B"]
    part = [1.0 - 0.5 * b / B if case["ragged"] else 1.0 for b in range(B)]
    return [max(1, round(case["Lq"] * p)) if case["Lq"] > 4 else case["Lq"] for p in part], \
           [max(1, round(case["Lk"] * p)) for p in part]


def tensor_sizes(case):
    """The parameter tensors of a layer: products into q, k, v, out of the heads, up by four and down, their biases
    and two norms."""
    h = case["hidden"]
    return case["layers"] * [3 * h * h, 3 * h, h * h, h, 4 * h * h, 4 * h, 4 * h * h, h, h, h, h, h]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype, spread=1.0, middle=0.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * spread + middle).to(dtype)

    st = dict(case=case)
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "attention":
        B, Lq, Lk, Hq, Hk, D = (case[n] for n in ("B", "Lq", "Lk", "Hq", "Hk", "D"))
        # q, k and v are what a layer's one product into 3 * hidden leaves, where the lengths let them be
        if Lq == Lk:
            qkv = normal(B, Lq, (Hq + 2 * Hk) * D, dtype=dtype)
            st["q"], st["k"], st["v"] = (t.unflatten(2, (-1, D)) for t in qkv.split([Hq * D, Hk * D, Hk * D], 2))
        else:
            st["q"] = normal(B, Lq, Hq, D, dtype=dtype)
            st["k"], st["v"] = normal(B, Lk, 2 * Hk, D, dtype=dtype).split(Hk, 2)
        if case["train"]:
            st["dout"] = normal(B, Lq, Hq, D, dtype=dtype, spread=0.1)
        st["len_q"] = st["len_k"] = None
        if case["ragged"]:
            nq, nk = lengths(case)
            turn = seed % B
            st["len_q"] = torch.tensor(nq[turn:] + nq[:turn], dtype=torch.int32, device="cuda")
            st["len_k"] = torch.tensor(nk[turn:] + nk[:turn], dtype=torch.int32, device="cuda")
    elif case["op"] == "norm":
        rows, cols, wdtype = case["rows"], case["cols"], DTYPES[case["wdtype"]]
        st["x"] = normal(rows, cols, dtype=dtype, spread=2.0, middle=0.5)
        st["weight"] = normal(cols, dtype=wdtype, spread=0.2, middle=1.0)
        st["bias"] = normal(cols, dtype=wdtype, spread=0.2)
        if case["train"]:
            st["dy"] = normal(rows, cols, dtype=dtype, spread=0.1)
    else:
        out = DTYPES[case["out"]]
        st["grads"] = [normal(n, dtype=dtype, spread=10.0 ** -(1 + i % 3)) for i, n in enumerate(tensor_sizes(case))]
        # the optimizer's buffer: the tensors end to end, wherever that puts them
        st["flat"] = torch.empty(sum(tensor_sizes(case)), dtype=out, device="cuda")
        st["outs"] = list(st["flat"].split(tensor_sizes(case)))
        if own:
            import paper_2307_02031_amd as g
            st["list"] = g.gbmw_gradient_list_create(st["grads"], st["outs"])
    return st


def run(state):
    return (run_own if own else run_plain)(state)


def run_own(st):
    import paper_2307_02031_amd as g
    case = st["case"]
    if case["op"] == "attention":
        mask = dict(causal=case["causal"], len_q=st["len_q"], len_k=st["len_k"])
        out, lse = g.gbmw_attention_forward(st["q"], st["k"], st["v"], **mask)
        if not case["train"]:
            return dict(out=out, lse=lse)
        dq, dk, dv = g.gbmw_attention_backward(st["dout"], st["q"], st["k"], st["v"], out, lse, **mask)
        return dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv)
    if case["op"] == "norm":
        y, mean, rstd = g.gbmw_layer_norm_forward(st["x"], st["weight"], st["bias"], NORM_EPS)
        if not case["train"]:
            return dict(y=y, mean=mean, rstd=rstd)
        dx, dweight, dbias = g.gbmw_layer_norm_backward(st["dy"], st["x"], st["weight"], mean, rstd)
        return dict(y=y, mean=mean, rstd=rstd, dx=dx, dweight=dweight, dbias=dbias)
    norm = g.gbmw_clip_gradients(st["list"], MAX_NORM)
    return dict(norm=norm, flat=st["flat"])


# ---- the plain forms: 32 bits, rounded once at the end --------------------------------------------------------------

def run_plain(st):
    return dict(attention=plain_attention, norm=plain_norm, clip=plain_clip)[st["case"]["op"]](st)


def plain_attention(st):
    case, q, k, v = st["case"], st["q"], st["k"], st["v"]
    B, Lq, Hq, D = q.shape
    Lk, Hk = k.shape[1], k.shape[2]
    share, scale = Hq // Hk, 1.0 / math.sqrt(D)
    res = dict(out=torch.empty(q.shape, dtype=q.dtype, device="cuda"),
               lse=torch.empty(B, Hq, Lq, device="cuda"))
    if case["train"]:
        res.update(dq=torch.empty(q.shape, dtype=q.dtype, device="cuda"),
                   dk=torch.empty(k.shape, dtype=q.dtype, device="cuda"),
                   dv=torch.empty(k.shape, dtype=q.dtype, device="cuda"))
    i = torch.arange(Lq, device="cuda").view(1, 1, 1, Lq, 1)
    j = torch.arange(Lk, device="cuda").view(1, 1, 1, 1, Lk)
    # as many samples and key heads at a time as give 2^28 probabilities
    heads = max(1, min(Hk, (1 << 28) // (share * Lq * Lk)))
    samples = max(1, min(B, (1 << 28) // (Hq * Lq * Lk)))

    def part(t, b, h, n):      # [samples, key heads, query heads of each, rows, D] in 32 bits
        t = t[b:b + samples, :, h * n:(h + heads) * n].float()
        return t.unflatten(2, (-1, n)).permute(0, 2, 3, 1, 4)

    def whole(t, dtype):       # and back
        return t.permute(0, 3, 1, 2, 4).flatten(2, 3).to(dtype)

    for b in range(0, B, samples):
        for h in range(0, Hk, heads):
            qs, ks, vs = part(q, b, h, share), part(k, b, h, 1), part(v, b, h, 1)
            x = torch.matmul(qs, ks.transpose(3, 4)) * scale
            nq = Lq if st["len_q"] is None else st["len_q"][b:b + samples].view(-1, 1, 1, 1, 1)
            nk = Lk if st["len_k"] is None else st["len_k"][b:b + samples].view(-1, 1, 1, 1, 1)
            sees = (j < nk) & (i < nq)
            if case["causal"]:
                sees = sees & (j <= i + nk - nq)
            x = torch.where(sees, x, -math.inf)
            top = x.amax(4, keepdim=True)
            p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
            total = p.sum(4, keepdim=True)
            p = p / torch.where(total == 0, 1.0, total)
            sb, sq, sk = slice(b, b + samples), slice(h * share, (h + heads) * share), slice(h, h + heads)
            out = torch.matmul(p, vs)
            res["out"][sb, :, sq] = whole(out, q.dtype)
            res["lse"][sb, sq] = (top + torch.log(total)).flatten(1, 2).squeeze(3)
            if case["train"]:
                do = part(st["dout"], b, h, share)
                dp = torch.matmul(do, vs.transpose(3, 4))
                ds = p * (dp - (do * out).sum(4, keepdim=True)) * scale
                res["dq"][sb, :, sq] = whole(torch.matmul(ds, ks), q.dtype)
                res["dk"][sb, :, sk] = whole(torch.matmul(ds.transpose(3, 4), qs).sum(2, keepdim=True), q.dtype)
                res["dv"][sb, :, sk] = whole(torch.matmul(p.transpose(3, 4), do).sum(2, keepdim=True), q.dtype)
    return res


def plain_norm(st):
    x, w = st["x"].float(), st["weight"].float()
    mean = x.mean(1, keepdim=True)
    off = x - mean
    rstd = 1.0 / torch.sqrt((off * off).mean(1, keepdim=True) + NORM_EPS)
    xhat = off * rstd
    res = dict(y=(xhat * w + st["bias"].float()).to(st["x"].dtype), mean=mean.squeeze(1), rstd=rstd.squeeze(1))
    if st["case"]["train"]:
        dy = st["dy"].float()
        g = dy * w
        dx = (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)) * rstd
        res.update(dx=dx.to(st["x"].dtype), dweight=(dy * xhat).sum(0).to(st["weight"].dtype),
                   dbias=dy.sum(0).to(st["weight"].dtype))
    return res


def plain_clip(st):
    squares = torch.stack([(g.float() * g.float()).sum() for g in st["grads"]])
    norm = torch.sqrt(squares.sum()).reshape(1)
    factor = torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0)
    for g, out in zip(st["grads"], st["outs"]):
        out.copy_(g.float() * factor)
    return dict(norm=norm, flat=st["flat"])


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    size = {n: torch.empty(0, dtype=t).element_size() for n, t in DTYPES.items()}
    s = size[case["dtype"]]
    if case["op"] == "attention":
        pairs = rows = keys = 0
        for nq, nk in zip(*lengths(case)):
            rows, keys = rows + nq, keys + nk
            # row i sees the first min(nk, i + nk - nq + 1) keys, none where that is negative
            first = max(0, nq - nk)
            n = nq - first
            pairs += n * (nk - nq + 1) + (first + nq - 1) * n // 2 if case["causal"] else nq * nk
        # forward: q, k, v in; out and log-sum-exp out; two products.  Backward: those and dout in; dq, dk, dv out;
        # five products, one of them the probabilities' once more
        qs, ks, lse = rows * case["Hq"] * case["D"] * s, keys * case["Hk"] * case["D"] * s, rows * case["Hq"] * 4
        full = case["B"] * case["Hq"] * case["Lq"]
        written = full * (case["D"] * s + 4)
        product = 2.0 * pairs * case["Hq"] * case["D"]
        if not case["train"]:
            return dict(bytes=qs + 2 * ks + written, flops=2 * product)
        kept = case["B"] * case["Hk"] * case["Lk"] * case["D"] * s
        return dict(bytes=2 * qs + 2 * ks + lse + written + full * case["D"] * s + 2 * kept, flops=7 * product)
    if case["op"] == "norm":
        n, w = case["rows"] * case["cols"], case["cols"] * size[case["wdtype"]]
        if not case["train"]:
            return dict(bytes=2 * n * s + 2 * w + 8 * case["rows"], flops=8.0 * n)
        return dict(bytes=4 * n * s + 4 * w + 8 * case["rows"], flops=22.0 * n)
    n = sum(tensor_sizes(case))
    return dict(bytes=n * (s + size[case["out"]]) + 4, flops=3.0 * n)


# ---- the definition in 64 bits --------------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm":
        x, w, b = (st[n].double() for n in ("x", "weight", "bias"))
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = torch.rsqrt(var + NORM_EPS)
        xhat = torch.addcmul(-(mean * rstd)[:, None], x, rstd[:, None])
        res = dict(y=torch.addcmul(b, xhat, w), mean=mean, rstd=rstd)
        if case["train"]:
            dy = st["dy"].double()
            c1, c2 = dy @ w / x.shape[1], torch.linalg.vecdot(dy * xhat, w.expand_as(dy)) / x.shape[1]
            res.update(dx=torch.addcmul(dy * w - c1[:, None], xhat, c2[:, None], value=-1) * rstd[:, None],
                       dweight=torch.linalg.vecdot(dy, xhat, dim=0), dbias=dy.sum(0))
        return res
    if case["op"] == "clip":
        norm = math.sqrt(math.fsum(float(torch.dot(g.double(), g.double())) for g in st["grads"]))
        by = MAX_NORM / norm if norm > MAX_NORM else 1.0
        return dict(norm=torch.tensor([norm], dtype=torch.float64, device="cuda"),
                    flat=torch.cat(st["grads"]).double() * by)
    B, Lq, Hq, D = st["q"].shape
    Lk, Hk = st["k"].shape[1:3]
    new = lambda t: torch.zeros(t.shape, dtype=torch.float64, device="cuda")
    res = dict(out=new(st["q"]), lse=torch.full((B, Hq, Lq), -math.inf, dtype=torch.float64, device="cuda"))
    if case["train"]:
        res.update(dq=new(st["q"]), dk=new(st["k"]), dv=new(st["k"]))
    nqs = [Lq] * B if st["len_q"] is None else st["len_q"].tolist()
    nks = [Lk] * B if st["len_k"] is None else st["len_k"].tolist()
    for b in range(B):
        nq, nk = nqs[b], nks[b]
        first = max(0, nq - nk) if case["causal"] else 0      # the rows before it see no key
        if nk == 0 or first >= nq:
            continue
        rows, keys = slice(first, nq), slice(0, nk)
        hidden = torch.ones(nq - first, nk, dtype=torch.bool, device="cuda").triu(first + nk - nq + 1)
        for h in range(Hq):
            g = h * Hk // Hq
            q, k, v = st["q"][b, rows, h].double(), st["k"][b, keys, g].double(), st["v"][b, keys, g].double()
            x = q @ k.T / math.sqrt(D)
            if case["causal"]:
                x.masked_fill_(hidden, -math.inf)
            lse = torch.logsumexp(x, 1)
            p = x.sub_(lse[:, None]).exp_()
            res["lse"][b, h, rows] = lse
            res["out"][b, rows, h] = o = p @ v
            if case["train"]:
                do = st["dout"][b, rows, h].double()
                res["dv"][b, keys, g] += p.T @ do
                p *= do @ v.T - torch.linalg.vecdot(do, o)[:, None]
                res["dq"][b, rows, h] = p @ k / math.sqrt(D)
                res["dk"][b, keys, g] += p.T @ q / math.sqrt(D)
    return res

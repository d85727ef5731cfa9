"""Performance cases of what a decoder's training step computes between its MXFP4
products and behind the last of them: the root-mean-square norm with the residual's
addition, causal attention over packed sequences, and the clipped policy loss with its
gradient.

A case is a dict of plain values:

  do       norm        h = x + residual, y = norm(h) * gain
           quantize    the same with y as MXFP4 operands, by rows and by columns
           norm_train  norm, then the gradients of x (and the residual) and of the gain
           attention   outputs and log-sum-exps of packed sequences
           attention_train   the same, then the gradients of q, k and v
           loss        the policy loss's sums, the tokens' log-probabilities and the
                       gradient of the logits
  t, n     tokens and width (norm); t, v  tokens and vocabulary (loss)
  type     "f32" or "bf16" of the activations or logits
  res      a residual is added
  lengths  of the packed sequences, "4096 1 300"
  heads, kv, dim    query heads, heads of k and v, entries of a head
  kl       factor of the loss's KL term

The plain forms compute in 32 bits from elementary operations (sums of squares, and
log-probabilities, whose ratio meets a border, in 64).  `own` selects the library's entry
points instead.
"""

import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
CLIP = 0.2, 0.28
MID = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]       # between neighbouring E2M1 magnitudes
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the last norm of a few tokens that are sampled together: all latency
        dict(name="norm_tokens", do="norm", t=16, n=4096, type="bf16", res=False),
        # a layer's first norm in front of its MXFP4 products, 4096 tokens of a 4096-wide
        # model: the operand of the forward product and that of the weight's gradient
        dict(name="norm_quantize", do="quantize", t=4096, n=4096, type="bf16", res=True),
        # an odd batch of an odd width in fp32, forward and backward
        dict(name="norm_train_odd", do="norm_train", t=509, n=1003, type="f32", res=True),
        # a batch of 16384 tokens, forward and backward
        dict(name="norm_train_batch", do="norm_train", t=16384, n=4096, type="bf16", res=True),
        # one sequence of 256 tokens through a 1024-wide layer's 16 heads
        dict(name="attention_short", do="attention", lengths="256", heads=16, kv=16, dim=64),
        # a prompt of 16384 tokens, 28 heads on 4 of k and v
        dict(name="attention_long", do="attention", lengths="16384", heads=28, kv=4, dim=128),
        # a small packed batch whose lengths no tile divides
        dict(name="attention_train_odd", do="attention_train", lengths="1 17 129 300 64 5 511 77", heads=16, kv=16, dim=64),
        # documents of very different lengths packed into 8192 tokens, grouped heads
        dict(name="attention_train_packed", do="attention_train", lengths="4096 2048 1023 700 300 25", heads=28, kv=4, dim=128),
        # a batch of four full sequences, 32 heads
        dict(name="attention_train_batch", do="attention_train", lengths="4096 4096 4096 4096", heads=32, kv=32, dim=128),
        # a short answer's tokens
        dict(name="loss_answer", do="loss", t=24, v=32000, type="bf16", kl=0.05),
        # fp32 logits of an odd vocabulary, no KL term
        dict(name="loss_odd", do="loss", t=701, v=50001, type="f32", kl=0.0),
        # a batch of 8192 tokens
        dict(name="loss_batch", do="loss", t=8192, v=32000, type="bf16", kl=0.05),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["norm", "quantize", "norm_train", "norm_train", "attention", "attention_train", "attention_train",
                     "loss", "loss"])
    if do == "loss":
        while True:
            t, v = _log(rng, 1, 8192), _log(rng, 2, 150000)
            if t * v <= 2.6e8 / 2:
                return dict(do=do, t=t, v=v, type=rng.choice(["f32", "bf16"]), kl=rng.choice([0.0, 0.05]))
    if do.startswith("attention"):
        dim, kv, group = rng.choice([64, 128]), rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 1, 2, 4, 7])
        lengths, left = [], 1.5e11 / (dim * kv * group)
        for _ in range(rng.randint(1, 10)):
            n = _log(rng, 1, 8192)
            if n * n <= left:
                lengths.append(n)
                left -= n * n
        # a query that sees one key has no gradient: not all of them
        lengths = lengths if max(lengths, default=0) > 8 else lengths + [rng.randint(9, 200)]
        return dict(do=do, lengths=" ".join(map(str, lengths)), heads=kv * group, kv=kv, dim=dim)
    while True:
        t, n = _log(rng, 1, 16384), _log(rng, 16, 18944)
        if t * n <= 6e7 / 2:
            return dict(do=do, t=t, n=n, type=rng.choice(["f32", "bf16"]), res=rng.random() < 0.7)


# ---------------------------------------------------------------- inputs

def _lengths(case):
    return [int(x) for x in case["lengths"].split()]


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)
    if own:
        s["layer"] = _library().LayerGroup()        # the context of a program's layers
    if case["do"].startswith("attention"):
        # q, k and v are slices of one fused projection; keys share a direction, as trained
        # ones do, so that some scores stand out
        t, h, kv, d = sum(_lengths(case)), case["heads"], case["kv"], case["dim"]
        s["qkv"] = (normal(t, h + 2 * kv, d) + 0.5 * normal(1, h + 2 * kv, d)).to(torch.bfloat16)
        s["q"], s["k"], s["v"] = s["qkv"][:, :h], s["qkv"][:, h:h + kv], s["qkv"][:, h + kv:]
        s["do"] = normal(t, h, d).to(torch.bfloat16)
        if own:
            s["seqs"] = s["layer"].sequences(_lengths(case))    # of every layer of a step
        return s
    t, kind = case["t"], DT[case["type"]]
    if case["do"] == "loss":
        v = case["v"]
        z = normal(t, v) * 2
        s["logits"] = z.to(kind)
        s["targets"] = torch.randint(0, v, (t,), generator=g, device=DEV)
        z.scatter_add_(1, s["targets"].view(-1, 1), normal(t, 1).abs() * 4)      # what was sampled is likely
        s["logits"].copy_(z)
        lp = torch.log_softmax(z, 1).gather(1, s["targets"].view(-1, 1)).view(-1)
        # the policy has moved from the one that sampled, and from the reference
        s["old"], s["ref"] = lp + 0.2 * normal(t), lp + 0.3 * normal(t)
        s["adv"] = normal(t)
        s["weight"] = (torch.rand(t, generator=g, device=DEV) < 0.9) / t        # a prompt's tokens do not count
        return s
    n = case["n"]
    outlier = torch.exp(0.5 * normal(1, n))                  # channels of differing scale
    s["x"] = (normal(t, n) * outlier).to(kind)
    s["res"] = (normal(t, n) * outlier * 2).to(kind) if case["res"] else None
    s["gain"] = 1 + 0.1 * normal(n)
    s["dy"] = (normal(t, n) * 1e-3).to(kind)
    s["dh"] = (normal(t, n) * 1e-3).to(kind)
    if own and case["do"] == "quantize":
        s["fp4"] = _library().Fp4Group()
    return s


# ---------------------------------------------------------------- plain forms

def _power(e):
    """2^e of whole numbers in -127 .. 127, exactly."""
    h = e // 2
    return ((h + 127) << 23).view(torch.float32) * ((e - h + 127) << 23).view(torch.float32)


def _rounded(x):
    """The MXFP4 values of x by rows, blocks of 32."""
    m, k = x.shape
    kb = -(-k // 32)
    x = torch.nn.functional.pad(x.contiguous(), (0, kb * 32 - k)).view(m, kb, 32)
    top = x.abs().amax(2, keepdim=True).view(torch.int32)
    e = (((top + 0x3FFFFF) >> 23) - 129).clamp(min=-127)
    y = x * _power(-e)
    a = y.abs()
    mag = torch.bucketize(a, torch.tensor(MID, device=DEV))             # MID[i-1] < |y| <= MID[i]
    mag = mag + (a == 0.75).int() + (a == 1.75).int() + (a == 3.5).int()    # ties to the even code
    v = torch.tensor(E2M1, device=DEV)[mag]
    return (torch.where(y < 0, -v, v) * _power(e)).view(m, -1)[:, :k]


def _norm(s):
    """h as it is stored, its fp32 values, 1 / rms and the unrounded y."""
    h = s["x"] if s["res"] is None else (s["x"].float() + s["res"].float()).to(s["x"].dtype)
    f = h.float()
    rstd = (f.double().square().mean(1, keepdim=True) + EPS).rsqrt().float()
    return h, f, rstd, f * rstd * s["gain"]


def _normed(s, h, y, rstd):
    out = {"y": y, "rstd": rstd.view(-1)}
    return out if s["res"] is None else dict(out, h=h)


def _attention(s, grad):
    """Sequence by sequence; heads of a group beside one another."""
    c = s["case"]
    h, kv, d = c["heads"], c["kv"], c["dim"]
    scale, at, parts = d ** -0.5, 0, []
    for n in _lengths(c):
        rows = slice(at, at + n)
        at += n
        q = s["q"][rows].float().transpose(0, 1).reshape(kv, h // kv * n, d)
        k, v = (s[x][rows].float().transpose(0, 1) for x in ("k", "v"))
        hidden = torch.ones(n, n, dtype=torch.bool, device=DEV).triu_(1)
        score = (q @ k.transpose(1, 2) * scale).view(h, n, n).masked_fill_(hidden, -math.inf)
        top = score.amax(2, keepdim=True)
        p = score.sub_(top).exp_()
        total = p.sum(2, keepdim=True)
        p = p.div_(total).view(kv, -1, n)
        lse = (top + total.log()).view(h, n)
        o = p @ v

        def back(x, heads):
            return x.view(heads, n, d).transpose(0, 1).to(torch.bfloat16)
        part = {"out": back(o, h), "lse": lse.t()}
        if grad:
            do = s["do"][rows].float().transpose(0, 1).reshape(kv, -1, d)
            part["dv"] = back(p.transpose(1, 2) @ do, kv)
            ds = (do @ v.transpose(1, 2)).sub_((do * o).sum(2, keepdim=True)).mul_(p)
            part["dq"] = back(ds @ k * scale, h)
            part["dk"] = back(ds.transpose(1, 2) @ q * scale, kv)
        parts.append(part)
    out = {x: torch.cat([p[x] for p in parts]) for x in parts[0]}
    out["lse"] = out["lse"].t().contiguous()
    return out


def _loss(s):
    z = s["logits"].float()
    at = s["targets"].view(-1, 1)
    top = z.amax(1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(1, keepdim=True)
    lp = ((z.gather(1, at) - top).double() - total.double().log()).view(-1)
    old, adv, w = s["old"].double(), s["adv"].double(), s["weight"].double()
    ratio = (lp - old).exp()
    bound = ratio.clamp(1 - CLIP[0], 1 + CLIP[1])
    clipped = bound * adv < ratio * adv
    kl, dkl = torch.zeros_like(lp), torch.zeros_like(lp)
    if s["case"]["kl"]:
        r = s["ref"].double() - lp
        kl, dkl = r.exp() - r - 1, 1 - r.exp()
    loss = s["case"]["kl"] * kl - torch.minimum(ratio * adv, bound * adv)
    g = (w * (s["case"]["kl"] * dkl - torch.where(clipped, 0.0, ratio * adv))).float().view(-1, 1)
    dz = e.mul_(-g / total).scatter_add_(1, at, g)
    sums = torch.stack([(w * loss).sum(), (w * kl).sum(), (w * clipped).sum()])
    return {"sums": sums.float(), "logp": lp.float(), "dlogits": dz.to(s["logits"].dtype)}


def _plain(s):
    do = s["case"]["do"]
    if do.startswith("attention"):
        return _attention(s, do == "attention_train")
    if do == "loss":
        return _loss(s)
    h, f, rstd, y = _norm(s)
    if do == "quantize":
        out = _normed(s, h, _rounded(y).to(torch.bfloat16), rstd)
        return dict(out, cols=_rounded(y.t()).to(torch.bfloat16))
    out = _normed(s, h, y.to(h.dtype), rstd)
    if do == "norm_train":
        dy = s["dy"].float()
        d, n = dy * s["gain"], f * rstd
        dx = rstd * (d - n * (d * n).mean(1, keepdim=True))
        dx = dx if s["res"] is None else dx + s["dh"].float()
        out.update(dx=dx.to(h.dtype), dgain=(dy * n).double().sum(0).float())
    return out


# ---------------------------------------------------------------- the library's calls

def _library():
    import paper_2609_15037_gb300
    return paper_2609_15037_gb300


def _own(s):
    c, layer = s["case"], s["layer"]
    do = c["do"]
    if do.startswith("attention"):
        if do == "attention":
            out, lse = layer.attention(s["q"], s["k"], s["v"], s["seqs"])
            return {"out": out, "lse": lse}
        # rest: what the outputs' rounding dropped, kept for the gradients
        out, lse, rest = layer.attention(s["q"], s["k"], s["v"], s["seqs"], train=True)
        dq, dk, dv = layer.attention_backward(s["do"], s["q"], s["k"], s["v"], out, lse, s["seqs"], rest=rest)
        return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    if do == "loss":
        ref = s["ref"] if c["kl"] else None
        sums, logp, dz = layer.policy_loss(s["logits"], s["targets"], s["old"], s["adv"], weights=s["weight"], ref=ref,
                                           clip=CLIP, kl=c["kl"])
        return {"sums": sums, "logp": logp, "dlogits": dz}
    if do == "quantize":
        h, (a, b), rstd = layer.norm_quantize(s["x"], s["gain"], residual=s["res"], eps=EPS, rows=True, cols=True)
        return dict(_normed(s, h, s["fp4"].dequantize(a), rstd), cols=s["fp4"].dequantize(b))
    h, y, rstd = layer.norm(s["x"], s["gain"], residual=s["res"], eps=EPS, dtype=s["x"].dtype)
    out = _normed(s, h, y, rstd)
    if do == "norm_train":
        dh = None if s["res"] is None else s["dh"]
        out["dx"], out["dgain"] = layer.norm_backward(s["dy"], h, s["gain"], rstd, dh=dh)
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- what a pass needs

def work(case):
    do, size = case["do"], {"f32": 4, "bf16": 2}
    if do.startswith("attention"):
        t, h, kv, d = sum(_lengths(case)), case["heads"], case["kv"], case["dim"]
        pairs = sum(n * (n + 1) // 2 for n in _lengths(case)) * h * d
        # q, k, v read, out and lse written; for the gradients do read, dq, dk, dv written
        fwd = 2 * t * d * (2 * h + 2 * kv) + 4 * t * h
        if do == "attention":
            return {"bytes": fwd, "flops": 4 * pairs}
        return {"bytes": fwd + 2 * t * d * (2 * h + 2 * kv), "flops": 14 * pairs}
    e = size[case["type"]]
    if do == "loss":
        return {"bytes": case["t"] * (2 * e * case["v"] + 32), "flops": 8 * case["t"] * case["v"]}
    t, n = case["t"], case["n"]
    b = t * n * e * (3 if case["res"] else 1)               # x; with a residual, it and h
    if do == "quantize":
        return {"bytes": b + 4 * t * n, "flops": 12 * t * n}        # the operands' values
    b += t * n * e
    if do == "norm_train":
        b += t * n * e * (3 if case["res"] else 2)          # dy (and dh) read, dx written
    return {"bytes": b, "flops": (15 if do == "norm_train" else 5) * t * n}


# ---------------------------------------------------------------- definitions in 64 bits

def _exact_fp4(x):
    """The nearest magnitudes on each block's power-of-two grid, ties to the even code."""
    m, k = x.shape
    kb = -(-k // 32)
    x = torch.nn.functional.pad(x.contiguous(), (0, kb * 32 - k)).view(m, kb, 32)
    top = x.abs().amax(2, keepdim=True)
    e = torch.floor(torch.log2(torch.clamp(top, min=2.0 ** -150))) - 2
    e = torch.clamp(e + (top > 6 * torch.exp2(e)).double(), min=-127)
    y = x / torch.exp2(e)
    a = y.abs()
    # spacing of the magnitudes: 1/2 below 2, 1 below 4, 2 up to 6
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return (torch.sign(y) * torch.round(a / step) * step * torch.exp2(e)).view(m, -1)[:, :k]


def _exact_head(q, k, v, do, scale):
    """One sequence and one head of k and v with the g heads of q that share it."""
    n = len(k)
    seen = torch.arange(n, device=DEV).view(1, -1) <= torch.arange(n, device=DEV).view(-1, 1)
    score = torch.einsum("igd,jd->gij", q, k) * scale
    score = torch.where(seen, score, -math.inf)
    lse = torch.logsumexp(score, 2)
    p = torch.exp(score - lse.unsqueeze(2))
    del score
    o = torch.einsum("gij,jd->igd", p, v)
    if do is None:
        return o, lse
    # the softmax's derivative: ds_ij = p_ij (dp_ij - sum_l p_il dp_il)
    dp = torch.einsum("igd,jd->gij", do, v)
    ds = p * (dp - torch.einsum("gij,gij->gi", p, dp).unsqueeze(2)) * scale
    return (o, lse, torch.einsum("gij,jd->igd", ds, k), torch.einsum("gij,igd->jd", ds, q),
            torch.einsum("gij,igd->jd", p, do))


def _exact_attention(case, s):
    h, kv, d = case["heads"], case["kv"], case["dim"]
    g, train = h // kv, case["do"] == "attention_train"
    t = len(s["q"])
    names = ["out", "lse", "dq", "dk", "dv"] if train else ["out", "lse"]
    shape = {"out": (t, h, d), "lse": (h, t), "dq": (t, h, d), "dk": (t, kv, d), "dv": (t, kv, d)}
    got = {x: torch.empty(shape[x], dtype=torch.float64, device=DEV) for x in names}
    at = 0
    for n in _lengths(case):
        for j in range(kv):
            many, one = slice(j * g, j * g + g), j
            row = slice(at, at + n)
            parts = _exact_head(s["q"][row, many].double(), s["k"][row, one].double(), s["v"][row, one].double(),
                                s["do"][row, many].double() if train else None, d ** -0.5)
            for x, y in zip(names, parts):
                if x == "lse":
                    got[x][many, row] = y
                else:
                    got[x][row, one if x in ("dk", "dv") else many] = y
        at += n
    return got


def _exact_loss(case, s):
    z = s["logits"].double()
    t = torch.arange(len(z), device=DEV)
    logp = z - torch.logsumexp(z, 1, keepdim=True)
    lp = logp[t, s["targets"]]
    w, a = s["weight"].double(), s["adv"].double()
    rho = torch.exp(lp - s["old"].double())
    low, high = 1 - CLIP[0], 1 + CLIP[1]
    # the smaller of the two surrogates: the bound one where the ratio has left the range on
    # the side that the advantage points to
    cut = ((a > 0) & (rho > high)) | ((a < 0) & (rho < low))
    surrogate = torch.where(cut, torch.where(a > 0, high, low) * a, rho * a)
    x = s["ref"].double() - lp if case["kl"] else torch.zeros_like(lp)
    kl = torch.exp(x) - x - 1
    dlp = w * (torch.where(cut, torch.zeros_like(a), -rho * a) + case["kl"] * (1 - torch.exp(x)))
    dz = -dlp.unsqueeze(1) * torch.exp(logp)
    dz[t, s["targets"]] += dlp
    sums = [(w * (case["kl"] * kl - surrogate)).sum(), (w * kl).sum(), (w * cut).sum()]
    return {"sums": torch.stack(sums), "logp": lp, "dlogits": dz}


def exact(case, seed):
    s = prepare(case, seed)
    do = case["do"]
    if do.startswith("attention"):
        return _exact_attention(case, s)
    if do == "loss":
        return _exact_loss(case, s)
    h = s["x"].double() if s["res"] is None else (s["x"].double() + s["res"].double()).to(s["x"].dtype).double()
    gain = s["gain"].double()
    ms = torch.mean(h * h, 1, keepdim=True) + EPS
    y = h / torch.sqrt(ms) * gain
    out = {"y": _exact_fp4(y) if do == "quantize" else y, "rstd": (1 / torch.sqrt(ms)).view(-1)}
    if s["res"] is not None:
        out["h"] = h
    if do == "quantize":
        out["cols"] = _exact_fp4(y.t())
    if do == "norm_train":
        dy = s["dy"].double()
        # of y_j = h_j g_j ms^(-1/2), ms = mean h^2
        dms = -0.5 * (dy * gain * h).sum(1, keepdim=True) * ms ** -1.5
        dx = dy * gain / torch.sqrt(ms) + dms * 2 * h / case["n"]
        out["dx"] = dx if s["res"] is None else dx + s["dh"].double()
        out["dgain"] = (dy * h / torch.sqrt(ms)).sum(0)
    return out

"""Performance cases of the operators beside the projected-Adam step: the AdamW
step of the parameters that step does not own, the gradient norm with its
clipping coefficient, and MXFP4 quantisation and products (the forward and
backward products of a weight that the step updates, whose last one is the
step's gradient).

A case is a dict of plain values:

  do       adamw     one AdamW step over many tensors; the new parameters, their
                     bf16 copies, and the moments (8-bit ones as their values)
           norm      sum of squares, norm and clipping coefficient of many gradients
           quantize  MXFP4 values of a matrix by rows, and by columns (transposed)
           product   D = A B^T of MXFP4 operands ("packed"), or of a bf16 A that is
                     quantised in the call ("bf16")
           linear    quantisation of x and dy both ways, y = x W^T, dx = dy W and
                     dW = dy^T x
  sizes    "count x entries ..." of the tensors: "65x4096 2x131072000"
  param, grad, state    types: "f32", "bf16"; state "f32" or "block8"
  copy     a bf16 copy of each fp32 parameter is written too
  m, n, k  rows of A (tokens), rows of B (outputs), entries per row

The plain forms compute in 32 bits from elementary operations.  `own` selects
the library's entry points instead.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
T = 101             # Adam step
LR = 1e-3
SEED = 77           # of the 8-bit states' rounding
DECAY = 0.1
MAX_NORM = 1.0
BLOCK = 256         # entries per scale of an 8-bit state
B1, B2, EPS = (float(np.float32(x)) for x in (0.9, 0.999, 1e-8))
MID = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]       # between neighbouring E2M1 magnitudes
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
DT = {"f32": torch.float32, "bf16": torch.bfloat16}

# every matrix of 24 decoder layers of the 1024/2816 model, its embedding and
# head (32000 tokens), and its norm gains
SMALL_MODEL = "96x1048576 72x2883584 2x32768000 49x1024"


def listed():
    return [
        # norm gains of a 4096-wide model with 32 layers: 65 short tensors, all
        # latency when each takes launches of its own
        dict(name="adamw_f32_gains", do="adamw", sizes="65x4096", param="f32", grad="f32", state="f32", copy=False),
        # embedding and head (32000 x 4096) with fp32 master weights, bf16
        # gradients and the bf16 copy that the next forward pass reads
        dict(name="adamw_f32_embeddings", do="adamw", sizes="2x131072000", param="f32", grad="bf16", state="f32", copy=True),
        # biases, a scalar gate and small odd matrices with 8-bit states
        dict(name="adamw_block8_odd", do="adamw", sizes="1x1 7x255 5x257 3x1003 1x38577 1x1026549", param="f32",
             grad="f32", state="block8", copy=False),
        # a whole small model (374 million entries) in bf16 with 8-bit states
        dict(name="adamw_block8_model", do="adamw", sizes=SMALL_MODEL, param="bf16", grad="bf16", state="block8", copy=False),
        # the norm gains' part of the clipping norm
        dict(name="norm_gains", do="norm", sizes="65x4096", grad="f32"),
        # the clipping norm of the small model's gradients
        dict(name="norm_model", do="norm", sizes=SMALL_MODEL, grad="bf16"),
        # activations of a short, odd batch
        dict(name="quantize_odd", do="quantize", m=509, k=2049, grad="f32"),
        # an fp32 weight after its step: by rows for the forward product, by
        # columns for the backward one
        dict(name="quantize_weight", do="quantize", m=11008, k=4096, grad="f32"),
        # one token through a 4096 x 4096 weight: latency and the weight's bytes
        dict(name="product_token", do="product", a="bf16", m=1, n=4096, k=4096, out="bf16"),
        # sizes that no tile divides
        dict(name="product_odd", do="product", a="packed", m=77, n=1003, k=2049, out="f32"),
        # a batch of 16384 tokens through the up-projection of a 4096/11008 model
        dict(name="product_batch", do="product", a="packed", m=16384, n=11008, k=4096, out="bf16"),
        # training step of one weight: forward and both backward products
        dict(name="linear_train", do="linear", m=4096, n=4096, k=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["adamw"] * 3 + ["norm"] + ["quantize"] * 2 + ["product"] * 3 + ["linear"])
    if do in ("adamw", "norm"):
        sizes, left = [], 2e8
        for _ in range(rng.randint(1, 5)):
            n = _log(rng, 1, 3e7)
            count = min(_log(rng, 1, 100), int(left // n))
            if count:
                sizes.append("%dx%d" % (count, n))
                left -= count * n
        c = dict(do=do, sizes=" ".join(sizes), grad=rng.choice(["f32", "bf16"]))
        if do == "adamw":
            c.update(param=rng.choice(["f32", "bf16"]), state=rng.choice(["f32", "block8"]))
            c["copy"] = c["param"] == "f32" and rng.random() < 0.5
        return c
    if do == "quantize":
        while True:
            m, k = _log(rng, 1, 18944), _log(rng, 1, 18944)
            if m * k <= 4.5e7:
                return dict(do=do, m=m, k=k, grad=rng.choice(["f32", "bf16"]))
    while True:
        m, n, k = _log(rng, 1, 16384), _log(rng, 16, 18944), _log(rng, 16, 18944)
        if m * n * k <= (7e11 if do == "product" else 6e10):
            break
    if do == "linear":
        return dict(do=do, m=m, n=n, k=k)
    return dict(do=do, a=rng.choice(["packed", "bf16"]), m=m, n=n, k=k, out=rng.choice(["bf16", "bf16", "f32"]))


# ---------------------------------------------------------------- inputs

def _tensors(case):
    """Entries of each tensor, and where it starts in the flat buffers."""
    ns = []
    for part in case["sizes"].split():
        count, n = part.split("x")
        ns += [int(n)] * int(count)
    starts = np.concatenate([[0], np.cumsum([-(-n // BLOCK) * BLOCK for n in ns])])
    return ns, starts


def _real(ns, starts):
    """Truth value of each flat place: an entry, or the padding behind a tensor."""
    at = torch.arange(int(starts[-1]), device=DEV).view(-1, BLOCK)
    ends = torch.tensor([int(s) + n for s, n in zip(starts, ns)], device=DEV)
    blocks = torch.tensor(np.diff(starts) // BLOCK, device=DEV)
    return (at < torch.repeat_interleave(ends, blocks).view(-1, 1)).view(-1)


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["do"] in ("adamw", "norm"):
        ns, starts = _tensors(case)
        real = _real(ns, starts)
        # gradients of tensors of differing scale, with heavy tails inside a tensor
        blocks = torch.tensor(np.diff(starts) // BLOCK, device=DEV)
        size = torch.exp(torch.randn(len(ns), generator=g, device=DEV) - 6.0)
        size = torch.repeat_interleave(size, blocks).view(-1, 1)
        row = torch.exp(0.5 * torch.randn(len(size), 1, generator=g, device=DEV))

        def noise():
            return torch.randn(len(size), BLOCK, generator=g, device=DEV)
        s["ns"], s["starts"] = ns, starts
        s["grad"] = ((noise() * size * row).view(-1) * real).to(DT[case["grad"]])
        s["extra"] = torch.rand(1, generator=g, device=DEV)
        if case["do"] == "adamw":
            s["param"] = ((noise() * 0.02).view(-1) * real).to(DT[case["param"]])
            m = (noise() * size * row * 0.3).view(-1) * real
            v = ((noise().square_() * 0.1 + 0.9) * (size * row).square_()).view(-1) * real
            s["coef"] = 0.5 + 0.5 * torch.rand(1, generator=g, device=DEV)
            if case["state"] == "block8":
                r = torch.full_like(m, 32768.0).int()
                s["m"], s["m_scale"] = _encode8(m, r, -112, True)
                s["v"], s["v_scale"] = _encode8(v, r, -96, False)
            else:
                s["m"], s["v"] = m, v
            s["copy"] = s["param"].to(torch.bfloat16) if case["copy"] else None
        s["grads"] = _parts(s, "grad")
        if own:
            s["opt"] = _optimizer(s)
        return s
    m, k = case["m"], case["k"]
    if case["do"] == "quantize":
        # a matrix in a wider buffer, as a slice of a fused projection is
        wide = torch.randn(m, k + 8, generator=g, device=DEV) * 0.02
        wide *= torch.exp(torch.randn(m, 1, generator=g, device=DEV))
        s["x"] = wide.to(DT[case["grad"]])[:, :k]
        if own:
            s["fp4"] = _library().Fp4Group()
        return s
    n = case["n"]
    x = torch.randn(m, k, generator=g, device=DEV)
    x *= torch.exp(torch.randn(1, k, generator=g, device=DEV))      # channels of differing scale
    w = torch.randn(n, k, generator=g, device=DEV) * 0.02
    s["w"] = _pack(w)
    if case["do"] == "linear":
        s["wt"] = _pack(w.t())
        s["x"] = x.to(torch.bfloat16)
        s["dy"] = (torch.randn(m, n, generator=g, device=DEV) * 1e-3).to(torch.bfloat16)
    elif case["a"] == "packed":
        s["a"] = _pack(x)
    else:
        s["x"] = x.to(torch.bfloat16)
    if own:
        # the context, and the packed operands as the library holds them
        s["fp4"] = _library().Fp4Group()
        for key in ("a", "w", "wt"):
            if key in s:
                p = s[key]
                s["fp4_" + key] = _library().Fp4Matrix(p["rows"], p["cols"], q=p["q"], sf=p["sf"])
    return s


# ---------------------------------------------------------------- 8-bit states

def _mix(x):
    """Xor-shift-multiply mixing of 32-bit numbers (int64 tensors or ints)."""
    x = x ^ (x >> 16)
    x = (x * 0x85EBCA6B) & 0xFFFFFFFF
    x = x ^ (x >> 13)
    x = (x * 0xC2B2AE35) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random(ns, starts):
    """32 random bits of each flat place (int64), from seed, tensor, step and entry."""
    key = _mix(_mix(SEED) ^ (SEED >> 32))
    ids = torch.arange(len(ns), device=DEV)
    key = _mix(_mix(ids ^ key) ^ T)             # of each tensor
    key = _mix(key)                             # of its first 2^32 entries
    blocks = torch.tensor(np.diff(starts) // BLOCK, device=DEV)
    first = torch.repeat_interleave(torch.tensor(starts[:-1], device=DEV), blocks).view(-1, 1)
    i = torch.arange(int(starts[-1]), device=DEV).view(-1, BLOCK) - first
    return _mix(i ^ torch.repeat_interleave(key, blocks).view(-1, 1)).view(-1)


def _bits(x):
    return x.view(torch.int32)


def _encode8(x, r16, shift, signed):
    """Codes and block scales of x, rounded up where the 16 random bits r16 say so."""
    x = x.view(-1, BLOCK)
    top = _bits(x.abs()).max(1, keepdim=True).values.view(torch.float32)
    fits = ~(top < 2.0 ** -100)
    inv = torch.where(fits, torch.full_like(top, 1.875) / top, torch.zeros_like(top))
    scale = torch.where(fits, top * float(np.float32(1 / 1.875)), torch.zeros_like(top))
    z = (x.abs() * inv) * 2.0 ** shift
    code = (_bits(z) + (r16.view(-1, BLOCK).int() << 4)) >> 20
    if signed:
        code = code.clamp(max=127) | (_bits(x) < 0).int() << 7
    else:
        code = torch.maximum(code.clamp(max=255), (x > 0).int())
    return code.to(torch.uint8).view(-1), scale.view(-1)


def _decode8(code, scale, shift, signed):
    code = code.view(-1, BLOCK).int()
    y = ((code & 127 if signed else code) << 20).view(torch.float32) * 2.0 ** -shift * scale.view(-1, 1)
    return (torch.where(code > 127, -y, y) if signed else y).view(-1)


def _adamw(s):
    c, b8 = s["case"], s["case"]["state"] == "block8"
    p, g = s["param"].float(), s["grad"].float() * s["coef"]
    m = _decode8(s["m"], s["m_scale"], -112, True) if b8 else s["m"]
    v = _decode8(s["v"], s["v_scale"], -96, False) if b8 else s["v"]
    m = m * B1 + g * (1.0 - B1)
    v = v * B2 + g * g * (1.0 - B2)
    p = p * (1.0 - LR * DECAY) - m * (LR / (1.0 - B1 ** T)) / (v.sqrt() * (1.0 - B2 ** T) ** -0.5 + EPS)
    s["param"].copy_(p)
    out = {"param": s["param"]}
    if c["copy"]:
        out["copy"] = s["copy"].copy_(p)
    if b8:
        r = _random(s["ns"], s["starts"])
        s["m"], s["m_scale"] = _encode8(m, r & 0xFFFF, -112, True)
        s["v"], s["v_scale"] = _encode8(v, r >> 16, -96, False)
        out["m"] = _decode8(s["m"], s["m_scale"], -112, True)
        out["v"] = _decode8(s["v"], s["v_scale"], -96, False)
    else:
        out["m"], out["v"] = s["m"].copy_(m), s["v"].copy_(v)
    return out


# ---------------------------------------------------------------- MXFP4

def _quantize(x):
    """E2M1 codes (with the sign in bit 3) and E8M0 scales of x by rows, blocks of 32."""
    m, k = x.shape
    kb = -(-k // 32)
    x = torch.nn.functional.pad(x.float().contiguous(), (0, kb * 32 - k)).view(m, kb, 32)
    top = _bits(x.abs().amax(2, keepdim=True))
    e = (((top + 0x3FFFFF) >> 23) - 129).clamp(min=-127)
    y = x * _power(-e)
    mag = torch.bucketize(y.abs(), torch.tensor(MID, device=DEV))       # MID[i-1] < |y| <= MID[i]
    a = y.abs()
    mag = mag + (a == 0.75).int() + (a == 1.75).int() + (a == 3.5).int()    # ties to the even code
    code = mag.int() | (_bits(y) < 0).int() << 3
    return code.view(m, kb * 32), (e + 127).view(m, kb)


def _power(e):
    """2^e of whole numbers in -127 .. 127, exactly."""
    h = e // 2
    return ((h + 127) << 23).view(torch.float32) * ((e - h + 127) << 23).view(torch.float32)


def _values(code, scale, k):
    """The fp32 values of codes and scales."""
    m = code.shape[0]
    v = torch.tensor(E2M1 + [-x for x in E2M1], device=DEV)[code.long()].view(m, -1, 32)
    return (v * _power(scale - 127).unsqueeze(2)).view(m, -1)[:, :k]


def _pack(x):
    """The packed operand of x: two codes a byte, the even column in the low
    half, and the scales in tiles of 128 rows x 4 blocks of 512 bytes, at
    (row % 32) * 16 + (row / 32) * 4 + block inside a tile; unused scales are 127."""
    m, k = x.shape
    code, scale = _quantize(x)
    q = (code[:, 0::2] | code[:, 1::2] << 4).to(torch.uint8)
    rt, ct = -(-m // 128), -(-scale.shape[1] // 4)
    full = torch.full((rt * 128, ct * 4), 127, dtype=torch.uint8, device=DEV)
    full[:m, :scale.shape[1]] = scale.to(torch.uint8)
    sf = full.view(rt, 4, 32, ct, 4).permute(0, 3, 2, 1, 4).contiguous()
    return {"q": q, "sf": sf.view(-1), "rows": m, "cols": k}


def _unpack(p):
    m, k = p["rows"], p["cols"]
    kb = -(-k // 32)
    rt, ct = -(-m // 128), -(-kb // 4)
    q = p["q"].int()
    code = torch.stack([q & 15, q >> 4], 2).view(m, -1)
    full = p["sf"].view(rt, ct, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rt * 128, ct * 4)
    return _values(code, full[:m, :kb].int(), k)


def _rounded(x):
    return _values(*_quantize(x), x.shape[1])


def _plain(s):
    c = s["case"]
    if c["do"] == "adamw":
        return _adamw(s)
    if c["do"] == "norm":
        total = s["grad"].float().square().sum()
        norm = (total + s["extra"]).sqrt()
        return torch.cat([total.view(1), norm, (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)])
    if c["do"] == "quantize":
        return {"rows": _rounded(s["x"]).to(torch.bfloat16), "cols": _rounded(s["x"].t()).to(torch.bfloat16)}
    if c["do"] == "product":
        a = _unpack(s["a"]) if c["a"] == "packed" else _rounded(s["x"])
        return (a @ _unpack(s["w"]).t()).to(DT[c["out"]])
    y = _rounded(s["x"]) @ _unpack(s["w"]).t()
    dx = _rounded(s["dy"]) @ _unpack(s["wt"]).t()
    dw = _rounded(s["dy"].t()) @ _rounded(s["x"].t()).t()
    return {"y": y.to(torch.bfloat16), "dx": dx.to(torch.bfloat16), "dw": dw.to(torch.bfloat16)}


# ---------------------------------------------------------------- the library's calls

def _library():
    import paper_2609_15037_gb300
    return paper_2609_15037_gb300


def _parts(s, key):
    return [s[key][int(a):int(a) + n] for a, n in zip(s["starts"], s["ns"])]


def _optimizer(s):
    """The AdamW group over the tensors of the flat buffers, with their states."""
    c = s["case"]
    opt = _library().AdamWGroup(beta1=0.9, beta2=0.999, eps=1e-8, seed=SEED)
    if c["do"] == "norm":
        return opt
    b8 = c["state"] == "block8"
    at = [slice(int(a) // BLOCK, int(b) // BLOCK) for a, b in zip(s["starts"], s["starts"][1:])]
    copies = _parts(s, "copy") if c["copy"] else [None] * len(at)
    for i, (p, q, m, v) in enumerate(zip(_parts(s, "param"), copies, _parts(s, "m"), _parts(s, "v"))):
        opt.add(p, copy=q, state=c["state"], weight_decay=DECAY, exp_avg=m, exp_avg_sq=v,
                exp_avg_scale=s["m_scale"][at[i]] if b8 else None,
                exp_avg_sq_scale=s["v_scale"][at[i]] if b8 else None)
    if b8:
        s["values"] = [torch.zeros(int(s["starts"][-1]), device=DEV) for _ in range(2)]
        s["into"] = [[f[int(a):int(a) + n] for a, n in zip(s["starts"], s["ns"])] for f in s["values"]]
    return opt


def _own(s):
    c = s["case"]
    if c["do"] == "adamw":
        opt = s["opt"]
        opt.step(s["grads"], T, LR, grad_scale=s["coef"])
        out = {"param": s["param"], "m": s["m"], "v": s["v"]}
        if c["state"] == "block8":
            opt.moments(*s["into"])
            out["m"], out["v"] = s["values"]
        if c["copy"]:
            out["copy"] = s["copy"]
        return out
    if c["do"] == "norm":
        return s["opt"].grad_norm(s["grads"], MAX_NORM, extra_sq=s["extra"])
    fp4 = s["fp4"]
    if c["do"] == "quantize":
        rows, cols = fp4.quantize(s["x"], rows=True, cols=True)
        return {"rows": fp4.dequantize(rows), "cols": fp4.dequantize(cols)}
    if c["do"] == "product":
        if c["a"] == "packed":
            return fp4.product(s["fp4_a"], s["fp4_w"], dtype=DT[c["out"]])
        return fp4.linear(s["x"], s["fp4_w"], dtype=DT[c["out"]])
    x, xt = fp4.quantize(s["x"], rows=True, cols=True)
    dy, dyt = fp4.quantize(s["dy"], rows=True, cols=True)
    return {"y": fp4.product(x, s["fp4_w"]), "dx": fp4.product(dy, s["fp4_wt"]), "dw": fp4.product(dyt, xt)}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- what a pass needs

def work(case):
    do = case["do"]
    size = {"f32": 4, "bf16": 2}
    if do in ("adamw", "norm"):
        n = sum(_tensors(case)[0])
        if do == "norm":
            return {"bytes": n * size[case["grad"]], "flops": 2 * n}
        # parameters and moments in and out, gradients in, copies out; 8-bit
        # moments in and out, and out once more as fp32 values
        state = 16 if case["state"] == "f32" else 4 + 8 + 16 / BLOCK
        return {"bytes": n * (2 * size[case["param"]] + size[case["grad"]] + state + (2 if case["copy"] else 0)), "flops": 15 * n}
    m, k = case["m"], case["k"]
    if do == "quantize":
        return {"bytes": m * k * (size[case["grad"]] + 4), "flops": 4 * m * k}
    n, packed = case["n"], 17 / 32
    if do == "product":
        a = packed if case["a"] == "packed" else 2
        return {"bytes": m * k * a + n * k * packed + m * n * size[case["out"]], "flops": 2 * m * n * k}
    return {"bytes": 2 * m * (k + n) + 2 * n * k * packed + 2 * (m * n + m * k + n * k), "flops": 6 * m * n * k}


# ---------------------------------------------------------------- definitions in 64 bits

def _exact_code(y, r16, bits):
    """Floating code with 3 mantissa bits of y in [0, 1.875] whose largest
    exponent is 0, rounded up with probability by r16; y as 64-bit reals."""
    emin = 2 - 2 ** bits                        # exponent of the smallest normal value
    e = torch.floor(torch.log2(torch.clamp(y, min=2.0 ** emin)))
    e = e - (torch.exp2(e) > y).double() * (e > emin)
    at = (e - emin) * 8 + y * torch.exp2(3 - e)     # the code as a real number
    return torch.floor(at + r16.double() / 65536).clamp(max=2 ** (bits + 3) - 1)


def _exact_value(code, bits):
    emin = 2 - 2 ** bits
    e = torch.clamp(torch.floor(code / 8), min=1)
    return (code - (e - 1) * 8) * torch.exp2(e - 1 + emin - 3)


def _exact_round(x, r16, bits):
    top = x.abs().amax(1, keepdim=True)
    unit = torch.where(top > 0, top / 1.875, torch.ones_like(top))
    code = _exact_code(x.abs() / unit, r16, bits)
    if bits == 5:
        code = torch.maximum(code, (x > 0).double())
    return torch.sign(x) * _exact_value(code, bits) * unit


def _exact_adamw(case, s):
    shape = (-1, BLOCK)
    g = (s["grad"].double() * s["coef"].double()).view(shape)
    p = s["param"].double().view(shape)
    if case["state"] == "block8":
        mc, vc = s["m"].view(shape).double(), s["v"].view(shape).double()
        sign = torch.where(mc >= 128, -1.0, 1.0)
        m = sign * _exact_value(torch.where(mc >= 128, mc - 128, mc), 4) * s["m_scale"].double().view(-1, 1)
        v = _exact_value(vc, 5) * s["v_scale"].double().view(-1, 1)
    else:
        m, v = s["m"].double().view(shape), s["v"].double().view(shape)
    m = B1 * m + (1 - B1) * g
    v = B2 * v + (1 - B2) * g ** 2
    p = p - LR * DECAY * p - LR * (m / (1 - B1 ** T)) / (torch.sqrt(v / (1 - B2 ** T)) + EPS)
    if case["state"] == "block8":
        r = _random(s["ns"], s["starts"]).view(shape)
        m, v = _exact_round(m, r % 65536, 4), _exact_round(v, torch.div(r, 65536, rounding_mode="floor"), 5)
    out = {"param": p.view(-1), "m": m.view(-1), "v": v.view(-1)}
    if case["copy"]:
        out["copy"] = out["param"]
    return out


def _exact_fp4(x):
    """The MXFP4 values of x by rows: the nearest magnitudes on each block's
    power-of-two grid, ties to the even code."""
    x = x.double().contiguous()
    m, k = x.shape
    kb = -(-k // 32)
    x = torch.nn.functional.pad(x, (0, kb * 32 - k)).view(m, kb, 32)
    top = x.abs().amax(2, keepdim=True)
    e = torch.floor(torch.log2(torch.clamp(top, min=2.0 ** -150))) - 2
    e = e + (top > 6 * torch.exp2(e)).double()
    e = torch.clamp(e, min=-127)
    y = x / torch.exp2(e)
    a = y.abs()
    # spacing of the magnitudes: 1/2 below 2, 1 below 4, 2 up to 6
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return (torch.sign(y) * torch.round(a / step) * step * torch.exp2(e)).view(m, -1)[:, :k]


def _exact_operand(p):
    m, k = p["rows"], p["cols"]
    kb = -(-k // 32)
    row = torch.arange(m, device=DEV).view(-1, 1)
    blk = torch.arange(kb, device=DEV).view(1, -1)
    at = ((row // 128) * -(-kb // 4) + blk // 4) * 512 + (row % 32) * 16 + (row % 128) // 32 * 4 + blk % 4
    scale = torch.exp2(p["sf"][at].double() - 127)
    col = torch.arange(k, device=DEV)
    code = (p["q"][:, col // 2].long() >> (4 * (col % 2))) % 16
    sign = 1.0 - 2.0 * (code // 8).double()
    e, f = (code % 8) // 2, (code % 2).double()
    mag = torch.where(e == 0, 0.5 * f, torch.exp2(e.double() - 1) * (1 + 0.5 * f))
    return sign * mag * scale.repeat_interleave(32, 1)[:, :k]


def exact(case, seed):
    s = prepare(case, seed)
    do = case["do"]
    if do == "adamw":
        return _exact_adamw(case, s)
    if do == "norm":
        total = (s["grad"].double() ** 2).sum()
        norm = torch.sqrt(total + s["extra"].double())
        return torch.cat([total.view(1), norm, torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)])
    if do == "quantize":
        return {"rows": _exact_fp4(s["x"]), "cols": _exact_fp4(s["x"].t())}
    if do == "product":
        a = _exact_operand(s["a"]) if case["a"] == "packed" else _exact_fp4(s["x"])
        return a @ _exact_operand(s["w"]).t()
    x, dy, xt, dyt = (_exact_fp4(t) for t in (s["x"], s["dy"], s["x"].t(), s["dy"].t()))
    return {"y": x @ _exact_operand(s["w"]).t(), "dx": dy @ _exact_operand(s["wt"]).t(), "dw": dyt @ xt.t()}

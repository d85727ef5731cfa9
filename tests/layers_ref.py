"""Float64 definitions of the operators of a decoder's layers, for their tests, with what
the library's roundings may add up to (elementwise bounds)."""

import torch

BF16, F32 = 2.0 ** -8, 2.0 ** -24          # half a step, relative to the value


def half_step(dtype):
    return BF16 if dtype == torch.bfloat16 else F32


# ------------------------------------------------------------------------- norm
def norm(x, res, gain, eps):
    """h (as stored), y, rstd."""
    h = x if res is None else (x.float() + res.float()).to(x.dtype)
    d = h.double()
    s = (d.square().mean(1) + eps).rsqrt()
    return h, d * s[:, None] * gain.double(), s


def norm_backward(dy, h, gain, s, dh):
    """dx, dgain and bounds of their errors before dx's last rounding.  d = dy g and n = h s take a
    rounding each (s another), their mean's terms two more and four fp32 additions each; the rest of
    the mean is summed in two numbers: 8 roundings of every term cover it.  dgain: a CTA adds up to
    rows / 150 + 8 terms in fp32 (at least 152 CTAs, or one row each), the CTAs' sums in two numbers."""
    u, f, g = dy.double(), h.double(), gain.double()
    d, n = u * g, f * s[:, None]
    dx = s[:, None] * (d - n * (d * n).mean(1, keepdim=True))
    slack = 8 * F32 * s[:, None] * (d.abs() + n.abs() * (d * n).abs().mean(1, keepdim=True))
    if dh is not None:
        dx = dx + dh.double()
        slack = slack + F32 * (dh.double().abs() + dx.abs())
    return dx, (u * n).sum(0), slack, (len(h) / 150 + 12) * F32 * (u * n).abs().sum(0)


# -------------------------------------------------------------------- attention
def attention(q, k, v, lengths, scale, do=None):
    """Outputs, log-sum-exps and (with do) gradients, each with a bound of its error.

    eS: error of S from its products of dim terms (fp32 accumulation: one rounding or cut per 16
    terms and 8 inside), relative error of exp and of the row's sum beside it.  P and dS take one bf16
    rounding each, and so does every output; delta takes the error of O from P's rounding."""
    T, H, D = q.shape
    Hk = k.shape[1]
    g = H // Hk
    eps = (D / 16 + 8) * 2.0 ** -23
    q, k, v = (x.double() for x in (q, k, v))
    do = None if do is None else do.double()
    got = {"out": torch.zeros_like(q), "lse": q.new_zeros(H, T)}
    if do is not None:
        got.update(dq=torch.zeros_like(q), dk=torch.zeros_like(k), dv=torch.zeros_like(v))
    tol = {x: torch.zeros_like(y) for x, y in got.items()}
    at = 0
    for n in lengths:
        rows = slice(at, at + n)
        at += n
        hide = torch.ones(n, n, dtype=torch.bool, device=q.device).triu_(1)
        for h in range(H if n else 0):
            j = h // g
            Q, K, V = q[rows, h], k[rows, j], v[rows, j]
            S = (Q @ K.t() * scale).masked_fill(hide, float("-inf"))
            eS = (Q.abs() @ K.abs().t()).amax(1, keepdim=True) * scale * eps + 2.0 ** -20
            lse = torch.logsumexp(S, 1, keepdim=True)
            P = (S - lse).exp()
            O = P @ V
            got["out"][rows, h], got["lse"][h, rows] = O, lse[:, 0]
            eP = 2 * eS + 2.0 ** -21 * lse.abs()
            eO = (BF16 + eP) * (P @ V.abs())
            tol["out"][rows, h] = eO + BF16 * O.abs()
            tol["lse"][h, rows] = (eS + 2.0 ** -22 * lse.abs())[:, 0]
            if do is None:
                continue
            dO = do[rows, h]
            dP = dO @ V.t()
            delta = (P * dP).sum(1, keepdim=True)
            dS = P * (dP - delta)
            eD = (dO.abs() * (eO + 2.0 ** -16 * O.abs())).sum(1, keepdim=True) + D * F32 * (dO.abs() * O.abs()).sum(1, keepdim=True)
            edP = eps * (dO.abs() @ V.abs().t())
            edS = (BF16 + eP) * dS.abs() + (1 + BF16) * P * (edP + eD)
            got["dq"][rows, h] = dS @ K * scale
            tol["dq"][rows, h] = edS @ K.abs() * scale * (1 + eps)
            got["dk"][rows, j] += dS.t() @ Q * scale
            tol["dk"][rows, j] += edS.t() @ Q.abs() * scale * (1 + eps)
            got["dv"][rows, j] += P.t() @ dO
            tol["dv"][rows, j] += (BF16 + eP).mul(P).t() @ dO.abs() * (1 + eps)
    for x in ("dq", "dk", "dv"):
        if x in got:
            tol[x] = tol[x] * (1 + BF16) + BF16 * got[x].abs() + 2.0 ** -60
    return got, tol


# ------------------------------------------------------------------ policy loss
def policy_loss(z, target, old, adv, weight, ref, low, high, kl):
    """sums, logp, dz with bounds: a row's exponentials are off by 2^-21 and 2^-23 of their
    argument, their sum by V / 64 additions in fp32 at most; what follows takes a few roundings."""
    dtype, z = z.dtype, z.double()
    t = torch.arange(len(z), device=z.device)
    counts = (target >= 0) & (target < z.shape[1])
    a = torch.where(counts, target, 0)
    lse = torch.logsumexp(z, 1)
    lp = z[t, a] - lse
    w = torch.where(counts, weight.double(), 0.0)
    A = adv.double()
    rho = (lp - old.double()).exp()
    bound = rho.clamp(low, high)
    cut = bound * A < rho * A
    x = torch.zeros_like(lp) if ref is None else ref.double() - lp
    k3 = x.exp() - x - 1
    loss = kl * k3 - torch.minimum(rho * A, bound * A)
    g = kl * (1 - x.exp()) - torch.where(cut, 0.0, rho * A)
    live = w != 0
    zero = torch.zeros_like(w)
    loss, k3, g = (torch.where(live, w * y, zero) for y in (loss, k3, g))
    p = (z - lse[:, None]).exp()
    dz = -g[:, None] * p
    dz[t, a] += g
    sums = torch.stack([loss.sum(), k3.sum(), torch.where(live & cut, w, zero).sum()])
    # bounds
    far = (z - z.amax(1, keepdim=True)).abs().clamp(max=150)
    ep = 2.0 ** -20 + 2.0 ** -22 * far + z.shape[1] / 64 * F32
    elp = 2.0 ** -20 + (p * ep).sum(1) + 2.0 ** -23 * lp.abs()
    aw = torch.where(live, w.abs(), zero)
    eg = aw * ((rho * A).abs() + kl * x.exp()) * (elp + 2.0 ** -20)
    edz = g.abs()[:, None] * p * (ep + elp[:, None]) + eg[:, None] * p
    edz[t, a] += eg + 2 * F32 * g.abs()
    edz = edz * 2 + half_step(dtype) * dz.abs() + 2.0 ** -126
    el = torch.where(live, eg + 2.0 ** -20 * loss.abs() + 2.0 ** -20 * k3.abs(), zero)
    # the KL term is quadratic in x
    ek = torch.where(live, w.abs() * ((1 - x.exp()).abs() * elp + elp * elp) + 2.0 ** -20 * k3.abs(), zero)
    esums = torch.stack([el.sum() + kl * ek.sum(), ek.sum(), 2.0 ** -23 * aw.sum()]) + 2.0 ** -100
    return (sums, torch.where(counts, lp, zero), dz), (esums, elp, edz)


def within(got, want, tol):
    """|got - want| <= tol everywhere, the error named where not."""
    e = (got.double() - want).abs()
    bad = ~(e <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {(e / tol)[bad].max().item():.3g} times its bound"

"""The operators of a decoder's layers together, as a training step uses them; offsets
beyond 32 bits; waits that run out."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import layers_ref as R  # noqa: E402

EPS = 1e-6


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_15037_gb300 as pkg
    return pkg


@pytest.fixture(scope="module")
def both(M):
    g, f = M.LayerGroup(), M.Fp4Group()
    yield g, f
    assert g.status() == 0 and f.status() == 0
    g.close()
    f.close()


def rand(gen, *shape, dtype=torch.bfloat16, scale=1.0):
    return (scale * torch.randn(*shape, generator=gen, device="cuda")).to(dtype)


@pytest.mark.parametrize("lengths,heads,kv,dim,hidden,vocab", [([300, 1, 129, 0, 70], 4, 2, 64, 256, 500), ([700], 6, 1, 128, 320, 1003),
                                                              ([5], 2, 2, 64, 128, 33), ([128] * 9, 8, 2, 64, 512, 2048)])
def test_a_step(both, lengths, heads, kv, dim, hidden, vocab):
    """Each operator is held to its definition on what the one before it gave, eagerly and replayed."""
    layer, fp4 = both
    gen = torch.Generator(device="cuda").manual_seed(hidden + vocab)
    t, wide = sum(lengths), (heads + 2 * kv) * dim
    x, res = rand(gen, t, hidden), rand(gen, t, hidden)
    gain, last = (1 + rand(gen, hidden, dtype=torch.float32, scale=0.1) for _ in range(2))
    w_qkv, w_out, w_head = (rand(gen, *s, scale=s[1] ** -0.5) for s in ((wide, hidden), (hidden, heads * dim), (vocab, hidden)))
    b_qkv, b_out = fp4.quantize(w_qkv), fp4.quantize(w_out)
    b_back, b_in = fp4.quantize(w_out, rows=False, cols=True), fp4.quantize(w_qkv, rows=False, cols=True)
    targets = torch.randint(0, vocab, (t,), generator=gen, device="cuda")
    old = -torch.rand(t, generator=gen, device="cuda") * 5
    adv, ref = rand(gen, t, dtype=torch.float32), -torch.rand(t, generator=gen, device="cuda") * 5
    seqs = layer.sequences(lengths)

    def step():
        h, (a, at), s = layer.norm_quantize(x, gain, residual=res, cols=True)
        qkv = fp4.product(a, b_qkv).view(t, heads + 2 * kv, dim)
        q, k, v = qkv.split([heads, kv, kv], 1)
        out, lse, rest = layer.attention(q, k, v, seqs, train=True)
        o = fp4.linear(out.view(t, -1), b_out)
        h2, y, s2 = layer.norm(o, last, residual=h)
        logits = y @ w_head.t()
        sums, logp, dz = layer.policy_loss(logits, targets, old, adv, ref=ref, kl=0.05)
        dy = dz @ w_head
        dh, dlast = layer.norm_backward(dy, h2, last, s2)
        dout = fp4.linear(dh, b_back).view(t, heads, dim)
        dq, dk, dv = layer.attention_backward(dout, q, k, v, out, lse, seqs, rest=rest)
        dn = fp4.linear(torch.cat([dq, dk, dv], 1).view(t, -1), b_in)
        dx, dgain = layer.norm_backward(dn, h, gain, s, dh=dh)
        return h, a, at, s, qkv, out, lse, o, h2, y, s2, logits, sums, logp, dz, dy, dh, dlast, dout, dq, dk, dv, dn, dx, dgain

    got = step()
    h, a, at, s, qkv, out, lse, o, h2, y, s2, logits, sums, logp, dz, dy, dh, dlast, dout, dq, dk, dv, dn, dx, dgain = got
    assert torch.equal(h, R.norm(x, res, gain, EPS)[0]) and torch.equal(h2, R.norm(o, h, last, EPS)[0])
    for op, w in zip((a, at), fp4.quantize(layer.norm(h, gain, dtype=torch.float32)[1], cols=True)):
        assert torch.equal(op.q, w.q) and torch.equal(op.sf, w.sf)
    q, k, v = qkv.split([heads, kv, kv], 1)
    want, tol = R.attention(q, k, v, lengths, dim ** -0.5, dout)
    for name, value in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        R.within(value, want[name], tol[name])
    weight = torch.full((t,), 1 / t, device="cuda")
    lp = torch.log_softmax(logits.double(), 1).gather(1, targets[:, None])[:, 0]
    assert ((lp - old.double()).exp()[:, None] - torch.tensor([0.8, 1.2], device="cuda")).abs().min() > 1e-5
    for value, w, e in zip((sums, logp, dz), *R.policy_loss(logits, targets, old, adv, weight, ref, 0.8, 1.2, 0.05)):
        R.within(value, w, e)
    for dd, hh, gg, ss, past, dxx, dgg in ((dy, h2, last, s2, None, dh, dlast), (dn, h, gain, s, dh, dx, dgain)):
        wx, wg, ex, eg = R.norm_backward(dd, hh, gg, ss, past)
        R.within(dxx, wx, ex * (1 + R.BF16) + R.BF16 * wx.abs() + 2.0 ** -126)
        R.within(dgg, wg, eg + 2.0 ** -126)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = step()
    for _ in range(2):
        for value in again:
            if torch.is_tensor(value):
                value.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for value, first in zip(again, got):
            if torch.is_tensor(value):
                assert torch.equal(value, first)


# ------------------------------------------------------------ offsets beyond 32 bits
def test_attention_beyond_32_bits(both):
    layer, _ = both
    heads, dim, n = 128, 128, 1040
    lengths = [128] * n + [77, 300]
    t = sum(lengths)
    assert t * heads * dim > 2 ** 31
    q = torch.zeros(t, heads, dim, dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros(t, 2, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    do = torch.zeros_like(q)
    gen = torch.Generator(device="cuda").manual_seed(5)
    tail = slice(t - 377, t)
    for x in (q, k, v, do):
        x[tail] = rand(gen, *x[tail].shape)
    seqs = layer.sequences(lengths)
    out, lse, rest = layer.attention(q, k, v, seqs, train=True)
    grads = layer.attention_backward(do, q, k, v, out, lse, seqs, rest=rest)
    want, tol = R.attention(q[tail], k[tail], v[tail], [77, 300], dim ** -0.5, do[tail])
    R.within(out[tail], want["out"], tol["out"])
    R.within(lse[:, tail], want["lse"], tol["lse"])
    for name, x in zip(("dq", "dk", "dv"), grads):
        R.within(x[tail], want[name], tol[name])
        assert (x[:tail.start] == 0).all()
    assert (out[:tail.start] == 0).all()
    del q, k, v, do, out, rest, grads, x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("cols", [8192, 8195])
def test_norm_beyond_32_bits(both, cols):
    layer, _ = both
    rows = 2 ** 31 // cols + 300
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-300:] = rand(gen, 300, cols)
    gain = 1 + rand(gen, cols, dtype=torch.float32, scale=0.1)
    _, y, s = layer.norm(x, gain)
    h, wy, ws = R.norm(x[-300:], None, gain, EPS)
    R.within(y[-300:], wy, (R.BF16 + 16 * R.F32) * wy.abs())
    R.within(s[-300:], ws, 16 * R.F32 * ws)
    assert (y[:1] == y[1]).all() and torch.equal(y[1], y[-301])
    dy = y.zero_()
    dy[-300:] = rand(gen, 300, cols)
    dx, dgain = layer.norm_backward(dy, x, gain, s, out=dy.clone())
    wx, wg, ex, eg = R.norm_backward(dy[-300:], x[-300:], gain, s[-300:], None)
    R.within(dx[-300:], wx, ex * (1 + R.BF16) + R.BF16 * wx.abs() + 2.0 ** -126)
    R.within(dgain, wg, 25 * eg + 2.0 ** -126)       # a CTA may add up all 300 rows
    assert (dx[:-300] == 0).all()
    del x, y, h, dy, dx
    torch.cuda.empty_cache()


@pytest.mark.parametrize("vocab", [32000, 32003])
def test_loss_beyond_32_bits(both, vocab):
    layer, _ = both
    rows = 2 ** 31 // vocab + 200
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    z[-200:] = rand(gen, 200, vocab)
    targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    adv, weights = rand(gen, rows, dtype=torch.float32), torch.zeros(rows, device="cuda")
    weights[-200:] = 0.005
    old = torch.full((rows,), -12.0, device="cuda")
    sums, lp, dz = layer.policy_loss(z, targets, old, adv, weights=weights, clip=(1.0, 1e9))
    tail = slice(rows - 200, rows)
    for value, w, e in zip((sums, lp[tail], dz[tail]),
                           *R.policy_loss(z[tail], targets[tail], old[tail], adv[tail], weights[tail], None, 0.0, 1 + 1e9, 0.0)):
        R.within(value, w, e)
    assert (dz[:tail.start] == 0).all()
    del z, dz
    torch.cuda.empty_cache()


# ----------------------------------------------------------------- waits that run out
LIMITS = [100, 100, 500, 1000, 2000, 4000, 8000, 16000, 100000]


def interrupted(M, call, surely=True):
    """call(group) -> tensors under every limit: the host reads the status, and the next call with
    the default bound gives what the first one gave.  surely: some limit has to run out (a wait for a
    row's copy alone may end within the time that the hardware suspends one try)."""
    g = M.LayerGroup()
    want = call(g)
    torch.cuda.synchronize()
    assert g.status() == 0
    seen = []
    for limit in LIMITS:
        M.moara_set_wait_limit(g.ctx, limit)
        got = call(g)
        torch.cuda.synchronize()
        seen.append(g.status())
        if seen[-1] == 0:
            assert all(torch.equal(x, y) for x, y in zip(got, want))
        M.moara_set_wait_limit(g.ctx, 0)
        got = call(g)
        torch.cuda.synchronize()
        assert g.status() == 0 and all(torch.equal(x, y) for x, y in zip(got, want))
    g.close()
    assert set(seen) <= {0, M.MOARA_ERR_DEVICE_TIMEOUT} and (not surely or M.MOARA_ERR_DEVICE_TIMEOUT in seen), seen


@pytest.mark.parametrize("lengths,h,hk,d", [([2000, 300], 8, 2, 128), ([1500], 4, 4, 64), ([4096], 1, 1, 128), ([300] * 20, 16, 4, 64),
                                              ([700, 1] * 10, 16, 4, 128)])
def test_attention_gives_up_and_recovers(M, lengths, h, hk, d):
    t = sum(lengths)
    gen = torch.Generator(device="cuda").manual_seed(t)
    q, k, v, do = rand(gen, t, h, d), rand(gen, t, hk, d), rand(gen, t, hk, d), rand(gen, t, h, d)
    g = M.LayerGroup()
    seqs = g.sequences(lengths)
    out, lse, rest = g.attention(q, k, v, seqs, train=True)
    torch.cuda.synchronize()
    interrupted(M, lambda g: g.attention(q, k, v, seqs, train=True))
    interrupted(M, lambda g: g.attention_backward(do, q, k, v, out, lse, seqs, rest=rest))
    g.close()


@pytest.mark.parametrize("t,vocab,dtype", [(600, 32000, torch.bfloat16), (200, 50001, torch.float32), (2, 32000, torch.bfloat16)])
def test_loss_gives_up_and_recovers(M, t, vocab, dtype):
    gen = torch.Generator(device="cuda").manual_seed(t)
    z = rand(gen, t, vocab, dtype=dtype)
    targets = torch.randint(0, vocab, (t,), generator=gen, device="cuda")
    old, adv = torch.full((t,), -11.0, device="cuda"), rand(gen, t, dtype=torch.float32)
    interrupted(M, lambda g: g.policy_loss(z, targets, old, adv), surely=False)

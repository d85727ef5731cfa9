"""AdamW over many tensors, its 8-bit moments and the gradient norm against the
float64 definitions.

Tolerances, from the number of roundings: a moment takes three to four fp32
roundings of its two terms; the update's square root, division and products
stay within 16 fp32 units; an fp32 parameter is rounded once more, a bf16 one to
half a bf16 unit.  An 8-bit code is exact where its position on the code axis
is not within 2^-12 of a rounding boundary (positions are below 256 and carry a
few fp32 roundings).
"""

import numpy as np
import pytest

from oracle import operators_ref as o

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

T, LR, WD, EPS, SEED = 7, 1e-2, 0.1, 1e-8, (5 << 32) + 9
B1, B2 = float(np.float32(0.9)), float(np.float32(0.999))
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_15037_gb300 as pkg
    return pkg


def f64(x):
    return x.detach().double().cpu().numpy()


def make(rng, n, dtype, scale, offset=0):
    """A device tensor of n entries, `offset` entries into its buffer."""
    x = torch.tensor(rng.standard_normal(n + offset) * scale, dtype=torch.float32).to(DT[dtype]).cuda()
    return x[offset:]


def check_moment8(codes, scales, ref, signed, bits):
    pos, scale = o.code_position(ref, signed)
    assert np.allclose(scales, scale, rtol=8 * U, atol=0)
    want = pos + bits / 65536.0
    code = codes.astype(np.int64)
    if signed:
        nz = (code & 127) != 0
        assert np.array_equal((code[nz] & 128) != 0, ref[nz] < 0)
        code = code & 127
        low = np.zeros_like(code)
    else:
        low = (ref > 2.0 ** -150).astype(np.int64)              # what rounds to an fp32 above zero
    floor = np.clip(np.floor(want).astype(np.int64), low, 127 if signed else 255)
    near = np.abs(want - np.round(want)) < 2.0 ** -12
    assert np.array_equal(code[~near], floor[~near])
    assert np.all(np.abs(code - floor) <= 1)
    assert near.mean() < 0.02 or len(ref) < 200 or np.all(ref == 0)


SIZES = [1, 2, 31, 255, 256, 257, 1003, 2047, 2048, 2049, 5 * 2048 + 77]


@pytest.mark.parametrize("param", ["f32", "bf16"])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("state", ["f32", "block8"])
@pytest.mark.parametrize("offset", [0, 1])
def test_step(M, param, grad, state, offset):
    """Every size, in one call; offset 1: pointers aligned to their type only."""
    rng = np.random.default_rng(1)
    opt = M.AdamWGroup(0.9, 0.999, EPS, SEED)
    coef = torch.tensor([0.625], device="cuda")
    ps, gs, copies, before = [], [], [], []
    for i, n in enumerate(SIZES):
        p, g = make(rng, n, param, 0.05, offset), make(rng, n, grad, 10.0 ** -rng.integers(0, 6), offset)
        copy = make(rng, n, "bf16", 1.0, offset) if param == "f32" and i % 2 == 0 else None
        if state == "f32":
            kw = dict(exp_avg=make(rng, n, "f32", 1e-3, offset), exp_avg_sq=make(rng, n, "f32", 1e-3, offset).abs())
        else:
            nb = -(-n // 256)
            kw = dict(exp_avg=torch.tensor(rng.integers(0, 256, n + offset), dtype=torch.uint8).cuda()[offset:],
                      exp_avg_sq=torch.tensor(rng.integers(0, 256, n + offset), dtype=torch.uint8).cuda()[offset:],
                      exp_avg_scale=torch.tensor(rng.random(nb) * 1e-3, dtype=torch.float32).cuda(),
                      exp_avg_sq_scale=torch.tensor(rng.random(nb) * 1e-6, dtype=torch.float32).cuda())
        opt.add(p, copy=copy, state=state, weight_decay=WD if i % 3 else 0.0, lr_scale=1.0 + i, id=100 + i, **kw)
        ps.append(p), gs.append(g), copies.append(copy)
        before.append({"p": f64(p), **{k: x.cpu().numpy().copy() for k, x in kw.items()}})
    m0, v0 = opt.moments()
    opt.step(gs, T, LR, grad_scale=coef)
    m1, v1 = opt.moments()
    torch.cuda.synchronize()
    for i, n in enumerate(SIZES):
        b, g = before[i], f64(gs[i]) * 0.625
        if state == "f32":
            m, v = b["exp_avg"].astype(np.float64), b["exp_avg_sq"].astype(np.float64)
        else:
            m = o.decode8(b["exp_avg"], b["exp_avg_scale"], True)
            v = o.decode8(b["exp_avg_sq"], b["exp_avg_sq_scale"], False)
        # the moments as values: exact, or one product's rounding
        assert np.allclose(f64(m0[i]), m, rtol=2 * U, atol=1e-38) and np.allclose(f64(v0[i]), v, rtol=2 * U, atol=1e-38)
        wd, lr = WD if i % 3 else 0.0, LR * (1.0 + i)
        rp, rm, rv = o.adamw(b["p"], g, m, v, T, lr, B1, B2, EPS, wd)
        st = opt.states[i]
        if state == "f32":
            assert np.all(np.abs(f64(st["exp_avg"]) - rm) <= 4 * U * (np.abs(B1 * m) + np.abs((1 - B1) * g)))
            assert np.all(np.abs(f64(st["exp_avg_sq"]) - rv) <= 5 * U * rv + 1e-42)
        else:
            bits = o.random_bits(n, SEED, 100 + i, T)
            check_moment8(st["exp_avg"].cpu().numpy(), f64(st["exp_avg_scale"]), rm, True, bits & 0xFFFF)
            check_moment8(st["exp_avg_sq"].cpu().numpy(), f64(st["exp_avg_sq_scale"]), rv, False, bits >> 16)
            back = o.decode8(st["exp_avg"].cpu().numpy(), f64(st["exp_avg_scale"]), True)
            assert np.allclose(f64(m1[i]), back, rtol=2 * U, atol=1e-38)
        # cancellation inside m: its error reaches the update unscaled
        den = np.sqrt(rv / (1 - B2 ** T)) + EPS
        slack = 4 * U * (np.abs(B1 * m) + np.abs((1 - B1) * g)) / (1 - B1 ** T) / den * lr
        upd = np.abs(rp - b["p"] * (1 - lr * wd))
        tol = 3 * U * np.abs(b["p"]) + 16 * U * upd + slack
        bf = 2.0 ** -8 * np.abs(rp)
        assert np.all(np.abs(f64(ps[i]) - rp) <= tol + (bf if param == "bf16" else 0))
        if copies[i] is not None:
            assert torch.equal(copies[i], ps[i].to(torch.bfloat16))
    opt.close()


def test_many_tensors_groups_and_subsets(M):
    """More tensors than one launch takes; the same result in another grouping,
    and the tensors left out of a call stay."""
    rng = np.random.default_rng(2)
    sizes = [int(x) for x in rng.integers(0, 700, 1300)]
    outs = []
    grads = [make(rng, n, "bf16", 1e-2) for n in sizes]
    for parts in (1, 3):
        opt = M.AdamWGroup(0.9, 0.999, EPS, SEED)
        ps = [torch.full((n,), 0.5, device="cuda") for n in sizes]
        for p in ps:
            opt.add(p, state="block8")
        ids = list(range(len(sizes)))
        for t in (1, 2):
            for k in range(parts):
                opt.step(grads[k::parts], t, LR, ids=ids[k::parts])
        before = ps[3].clone()
        opt.step(grads[10:12], 3, LR, ids=[10, 11])
        assert torch.equal(before, ps[3])
        outs.append(ps + [x for s in opt.states for x in s.values()])
        opt.close()
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_rounding_is_unbiased(M):
    """The mean of a block's decoded second moments over 400 seeds is the value
    (standard error of the mean: a code step, at most 1/8 of the value, over
    sqrt(12 * 400 * 4096))."""
    n = 4096
    g = torch.linspace(0.5, 1.5, n, device="cuda")
    total = torch.zeros(n, device="cuda", dtype=torch.float64)
    for seed in range(400):
        opt = M.AdamWGroup(0.9, 0.999, EPS, seed)
        opt.add(torch.zeros(n, device="cuda"), state="block8")
        opt.step([g], 1, LR)
        total += opt.moments()[1][0].double()
        opt.close()
    want = 0.001 * g.double() ** 2 * (float(np.float32(1) - np.float32(0.999)) / 0.001)
    ratio = total / 400 / want
    assert abs(ratio.mean().item() - 1) < 5 * 0.125 / np.sqrt(12 * 400 * n)
    assert (ratio - 1).abs().max().item() < 6 * 0.125 / np.sqrt(12 * 400) * 2


def test_special_values(M):
    """Zero gradients leave zero moments zero and only decay the parameter; NaN
    and infinity reach their entry (fp32) or their block of 256 (8 bits); blocks
    below 2^-100 are stored as zero; eps = 0 with zero moments gives NaN as the
    formula does."""
    for state in ("f32", "block8"):
        for bad in (float("nan"), float("inf")):
            opt = M.AdamWGroup(0.9, 0.999, EPS)
            p = torch.ones(600, device="cuda")
            opt.add(p, state=state, weight_decay=0.5)
            g = torch.zeros(600, device="cuda")
            g[300] = bad
            opt.step([g], 1, 0.1)
            m, v = opt.moments()
            hit = torch.zeros(600, dtype=torch.bool, device="cuda")
            hit[300] = True
            assert torch.equal(torch.isnan(p), hit) and torch.allclose(p[~hit], torch.full_like(p[~hit], 0.95))
            if state == "block8":
                hit[256:512] = True
            assert torch.equal(~torch.isfinite(m[0]), hit) and torch.equal(~torch.isfinite(v[0]), hit)
            assert not m[0][~hit].any() and not v[0][~hit].any()
            opt.close()
    opt = M.AdamWGroup(0.9, 0.999, 0.0)
    p, q = torch.ones(8, device="cuda"), torch.ones(8, device="cuda")
    opt.add(p), opt.add(q, state="block8")
    opt.step([torch.zeros(8, device="cuda"), torch.full((8,), 1e-30, device="cuda")], 1, 0.1)
    m, v = opt.moments(ids=[1])
    # 0 / 0; and a gradient of 1e-30 makes a first moment of 1e-31, which fp32
    # holds, beside a second one of 1e-63, which is below every fp32: m / 0.  Both
    # are below 2^-100 = 7.9e-31
    assert torch.isnan(p).all() and (q == float("-inf")).all()
    assert not m[0].any() and not v[0].any()
    opt.close()


def test_eight_bit_training_follows_fp32(M):
    """A least-squares fit for 300 steps: 8-bit moments end within 2% of the
    loss that fp32 moments reach from the same start."""
    rng = np.random.default_rng(4)
    A = torch.tensor(rng.standard_normal((4096, 512)), dtype=torch.float32).cuda()
    y = A @ torch.tensor(rng.standard_normal(512), dtype=torch.float32).cuda() + torch.tensor(
        rng.standard_normal(4096), dtype=torch.float32).cuda()
    losses = []
    for state in ("f32", "block8"):
        w = torch.zeros(512, device="cuda")
        opt = M.AdamWGroup(0.9, 0.999, EPS, 3)
        opt.add(w, state=state)
        gen = torch.Generator(device="cuda").manual_seed(1)
        for t in range(1, 301):
            i = torch.randint(0, 4096, (512,), device="cuda", generator=gen)
            r = A[i] @ w - y[i]
            opt.step([A[i].t() @ r / 512], t, 0.02 * (1 - t / 310))
        losses.append((A @ w - y).square().mean().item())
        opt.close()
    assert abs(losses[1] / losses[0] - 1) < 0.02, losses


@pytest.mark.parametrize("sizes", [[1], [8192], [8193, 5, 0, 77], [3_000_001], [100] * 2500])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm(M, sizes, dtype):
    """fp32 sums of at most 32 squares, then fp64: relative 32 units at most."""
    rng = np.random.default_rng(5)
    grads = [make(rng, n, dtype, 10.0 ** -rng.integers(0, 4), i % 2) for i, n in enumerate(sizes)]
    opt = M.AdamWGroup()
    extra = torch.tensor([2.5], device="cuda")
    want = sum((f64(g) ** 2).sum() for g in grads)
    for e, c in ((None, 0.0), (extra, 0.25), (extra, 1e9)):
        for _ in range(2):                                   # the workspace is reusable
            out = opt.grad_norm(grads, c, extra_sq=e)
        s, norm, coef = f64(out)
        root = np.sqrt(want + (2.5 if e is not None else 0.0))
        assert abs(s - want) <= 33 * U * want and abs(norm - root) <= 33 * U * root
        assert abs(coef - (min(1.0, c / (root + 1e-6)) if c > 0 else 1.0)) <= 34 * U
    a = opt.grad_norm(grads, 1.0)
    b = opt.grad_norm(grads, 1.0)
    assert torch.equal(a, b)
    opt.close()


def test_norm_special_values(M):
    opt = M.AdamWGroup()
    assert opt.grad_norm([], 1.0).tolist() == [0.0, 0.0, 1.0]
    g = torch.ones(100, device="cuda")
    g[7] = float("inf")
    assert opt.grad_norm([g], 1.0).tolist() == [float("inf"), float("inf"), 0.0]
    g[8] = float("nan")
    assert torch.isnan(opt.grad_norm([g], 1.0)).all()
    assert opt.grad_norm([g], 0.0)[2].item() == 1.0
    opt.close()


def test_norm_joins_the_grouped_step(M):
    """The clipping norm of a projected step and of the tensors beside it: one
    coefficient for both."""
    rng = np.random.default_rng(6)
    m, n, r = 192, 320, 24
    grp = M.MoaraGroup(block_size=64, clip_norm=0.5)
    grp.add(m, n, r, "bf16")
    grp.load_projector(grp.ids[0], np.linalg.qr(rng.standard_normal((m, r)))[0])
    G, e = make(rng, m * n, "bf16", 1.0).view(m, n), make(rng, 5000, "f32", 1.0)
    opt = M.AdamWGroup()
    p = torch.zeros(5000, device="cuda")
    opt.add(p)
    part = opt.grad_norm([e])
    grp.set_clip_extra(part[:1])
    grp.step([G], 1, 1e-3)
    state = grp.clip_state()
    opt.step([e], 1, 1e-3, grad_scale=state[1:])
    root = np.sqrt((f64(G) ** 2).sum() + (f64(e) ** 2).sum())
    assert abs(f64(state)[0] / root - 1) < 1e-5 and abs(f64(state)[1] / (0.5 / (root + 1e-6)) - 1) < 1e-5
    m1, _ = opt.moments()
    assert np.allclose(f64(m1[0]), 0.1 * f64(e) * f64(state)[1], rtol=1e-5, atol=1e-9)
    grp.close(), opt.close()


def test_other_stream_and_capture(M):
    rng = np.random.default_rng(7)
    g = make(rng, 10_000, "bf16", 1.0)
    outs = []
    for captured in (False, True):
        opt = M.AdamWGroup(seed=1)
        p = torch.zeros(10_000, device="cuda")
        opt.add(p, state="block8")
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        out = torch.zeros(3, device="cuda")

        def calls(t):
            opt.grad_norm([g], 1.0, out=out)
            opt.step([g], t, LR, grad_scale=out[2:])
        with torch.cuda.stream(s):
            calls(1)
        s.synchronize()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                calls(2)
            graph.replay()
        else:
            opt.grad_norm([g], 1.0, out=out, stream=s.cuda_stream)
            opt.step([g], 2, LR, grad_scale=out[2:], stream=s.cuda_stream)
        torch.cuda.synchronize()
        outs.append([p, out] + list(opt.states[0].values()))
        opt.close()
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_recorded_norm_keeps_its_workspace(M):
    """A graph recorded after a call on its stream, replayed after a call there that
    needs a larger workspace and after others have taken freed memory."""
    rng = np.random.default_rng(17)
    g = [make(rng, 5000, "f32", 1.0) for _ in range(3)]
    opt = M.AdamWGroup()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.zeros(3, device="cuda")
    with torch.cuda.stream(s):
        first = opt.grad_norm(iter(g[:1]), 1.0).clone()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            opt.grad_norm(g[:1], 1.0, out=out)
        many = opt.grad_norm(g * 700, 1.0)
        taken = [torch.full((512 << i,), 255, dtype=torch.uint8, device="cuda") for i in range(12)]
        for _ in range(2):
            out.zero_()
            graph.replay()
            s.synchronize()
            assert torch.equal(out, first)
        assert torch.equal(opt.grad_norm(g * 700, 1.0), many)
    assert all(bool((x == 255).all()) for x in taken)
    opt.close()


def test_state_dict_of_others_is_refused(M):
    a, b = M.AdamWGroup(), M.AdamWGroup()
    for opt, sizes, state in ((a, (300, 7), "block8"), (b, (300,), "block8")):
        for n in sizes:
            opt.add(torch.ones(n, device="cuda"), state=state)
    sd = a.state_dict()
    for bad in (sd[:1], sd + sd[:1], sd[::-1], [sd[0], {"exp_avg": sd[1]["exp_avg"]}],
                [sd[0], {k: v.float() for k, v in sd[1].items()}]):
        with pytest.raises(ValueError):
            a.load_state_dict(bad)
    with pytest.raises(ValueError):
        b.load_state_dict(sd)
    a.step([torch.ones(300, device="cuda"), torch.ones(7, device="cuda")], 1, LR)
    a.load_state_dict(sd)
    assert all(torch.equal(x, y) for s, new in zip(a.states, sd) for x, y in zip(s.values(), new.values()))
    a.close(), b.close()


def test_refusals(M):
    opt = M.AdamWGroup()
    p = torch.ones(100, device="cuda")
    opt.add(p)
    g = torch.ones(100, device="cuda")
    before = M.moara_launch_count(opt.ctx)

    def code(call):
        with pytest.raises(M.MoaraError) as ei:
            call()
        return ei.value.code
    for bad in (dict(grads=[g[:99]]), dict(grads=[g.half()]), dict(grads=[g, g]), dict(grads=[g.cpu()]),
                dict(grads=[torch.ones(200, device="cuda")[::2]]), dict(grads=[g], grad_scale=torch.ones(2, device="cuda"))):
        with pytest.raises(ValueError):
            opt.step(t=1, lr=0.1, **bad)
    for kw in (dict(state="f16"), dict(copy=torch.ones(99, device="cuda", dtype=torch.bfloat16)),
               dict(exp_avg=torch.zeros(99, device="cuda"))):
        with pytest.raises(ValueError):
            opt.add(p, **kw)
    assert code(lambda: opt.step([g], 0, 0.1)) == M.MOARA_ERR_INVALID_ARG
    assert code(lambda: opt.step([g], 1, float("nan"))) == M.MOARA_ERR_INVALID_ARG

    def edited(**kw):
        d = opt._chosen([0])[0]
        d["grad"], d["grad_dtype"] = g.data_ptr(), 0
        for k, v in kw.items():
            d[k] = v
        return code(lambda: M.moara_adamw_step(opt.ctx, 1, d.ctypes.data, opt.hp, 1, 0.1))
    for kw, want in ((dict(n=-1), M.MOARA_ERR_SHAPE), (dict(grad=0), M.MOARA_ERR_INVALID_ARG),
                     (dict(param=p.data_ptr() + 2), M.MOARA_ERR_ALIGN), (dict(grad_dtype=2), M.MOARA_ERR_INVALID_ARG),
                     (dict(state_dtype=1), M.MOARA_ERR_INVALID_ARG), (dict(state_dtype=2), M.MOARA_ERR_INVALID_ARG),
                     (dict(weight_decay=-1.0), M.MOARA_ERR_INVALID_ARG), (dict(lr_scale=np.inf), M.MOARA_ERR_INVALID_ARG),
                     (dict(param_dtype=1, param_bf16=p.data_ptr()), M.MOARA_ERR_INVALID_ARG),
                     (dict(exp_avg=0), M.MOARA_ERR_INVALID_ARG), (dict(n=1 << 50), M.MOARA_ERR_SHAPE)):
        assert edited(**kw) == want, kw
    hp = M.binding.moara_adamw_hparams(1.0, 0.9, 1e-8, 0)
    assert code(lambda: M.moara_adamw_step(opt.ctx, 0, 0, hp, 1, 0.1)) == M.MOARA_ERR_INVALID_ARG
    ws = torch.zeros(M.moara_grad_norm_workspace_bytes(1), dtype=torch.uint8, device="cuda")
    a = np.array([g.data_ptr(), 100], dtype=np.int64)
    ty = np.array([0], dtype=np.int32)

    def norm(size=ws.numel(), at=ws.data_ptr(), out=p.data_ptr(), dtype=ty):
        return code(lambda: M.moara_grad_norm(opt.ctx, 1, a.ctypes.data, a.ctypes.data + 8, dtype.ctypes.data, 1.0, 0,
                                              out, at, size))
    assert norm(size=16) == M.MOARA_ERR_WORKSPACE and norm(at=None) == M.MOARA_ERR_WORKSPACE
    assert norm(at=ws.data_ptr() + 4) == M.MOARA_ERR_ALIGN and norm(out=None) == M.MOARA_ERR_INVALID_ARG
    assert norm(dtype=np.array([7], dtype=np.int32)) == M.MOARA_ERR_INVALID_ARG
    assert M.moara_launch_count(opt.ctx) == before
    torch.cuda.synchronize()
    assert torch.equal(p, torch.ones(100, device="cuda"))
    opt.close()


def check_last(opt, i, p0, g, m0, v0, first, t, eps=EPS, wd=0.0, ident=None):
    """The entries from `first` (a multiple of 256) of tensor i on, from their values before the step."""
    st, n = opt.states[i], len(g)
    s = slice(first // 256, first // 256 + -(-n // 256))
    bits = o.random_bits(n, opt.hp.seed, i if ident is None else ident, t, first=first)
    rp, rm, rv = o.adamw(p0, g, m0, v0, t, LR, B1, B2, eps, wd)
    check_moment8(st["exp_avg"][first:first + n].cpu().numpy(), f64(st["exp_avg_scale"][s]), rm, True, bits & 0xFFFF)
    check_moment8(st["exp_avg_sq"][first:first + n].cpu().numpy(), f64(st["exp_avg_sq_scale"][s]), rv, False, bits >> 16)
    got = f64(opt.params[i][first:first + n])
    den = np.sqrt(rv / (1 - B2 ** t)) + eps
    slack = 4 * U * (np.abs(B1 * m0) + np.abs((1 - B1) * g)) / (1 - B1 ** t) / den * LR
    bf = 2.0 ** -8 if opt.params[i].dtype == torch.bfloat16 else 0.0
    assert np.all(np.abs(got - rp) <= 3 * U * np.abs(p0) + 16 * U * np.abs(rp - p0) + slack + bf * np.abs(rp))


@pytest.mark.parametrize("param,grad", [("bf16", "bf16"), ("f32", "f32")])
def test_long_calls(M, param, grad):
    """A call with so many entries that a CTA takes several pieces of a tensor: the
    ends of a long tensor that no block divides, and the short ones beside it."""
    rng = np.random.default_rng(8)
    sizes = [300, 152 * 8 * 16384 + 2048 * 7 + 1003, 5000, 256]
    opt = M.AdamWGroup(0.9, 0.999, EPS, SEED)
    ps = [torch.randn(n, device="cuda").to(DT[param]) for n in sizes]
    for p in ps:
        opt.add(p, state="block8")
    gs = [torch.randn(n, device="cuda").to(DT[grad]) for n in sizes]
    opt.step(gs, 1, LR)
    gs = [torch.randn(n, device="cuda").to(DT[grad]) for n in sizes]
    m, v = opt.moments()
    before = [p.clone() for p in ps]
    opt.step(gs, 2, LR)
    for i, n in enumerate(sizes):
        for first in {0, n // 2 // 256 * 256, max(0, (n - 700) // 256 * 256)}:
            part = slice(first, min(n, first + 3 * 256 + 19))
            if part.stop < n:
                part = slice(first, first + 3 * 256)
            check_last(opt, i, f64(before[i][part]), f64(gs[i][part]), f64(m[i][part]), f64(v[i][part]), first, 2)
    opt.close()


def test_offsets_behind_32_bits(M):
    """A tensor of more than 2^32 entries: its last ones, and the norm of its gradient."""
    n = (1 << 32) + 1000
    opt = M.AdamWGroup(0.9, 0.999, EPS, SEED)
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(1000, device="cuda").bfloat16()
    p[-1000:], g[-1000:] = 1.0, tail
    opt.add(p, state="block8", id=3)
    opt.step([g], 5, LR)
    zero = np.zeros(1000)
    check_last(opt, 0, zero + 1.0, f64(tail), zero, zero, 1 << 32, 5, ident=3)
    assert not p[:-1000].any() and not opt.states[0]["exp_avg"][:1 << 32].any()
    want = (f64(tail) ** 2).sum()
    assert abs(opt.grad_norm([g])[0].item() / want - 1) <= 33 * U
    m, _ = opt.moments()
    assert (m[0][-1000:] != 0).any() and not m[0][:-1000].any()
    opt.close()


@pytest.mark.parametrize("size", [1e-28, 1e-6, 3e4, 1e8, 1e16])
@pytest.mark.parametrize("eps", [1e-8, 1e-12])
def test_scales_of_moments(M, size, eps):
    """Gradients from those whose moments are stored as zero to those whose code factors
    leave fp32's normal numbers, with the exact and the quick form of the update."""
    rng = np.random.default_rng(9)
    opt = M.AdamWGroup(0.9, 0.999, eps, SEED)
    p, g = make(rng, 1500, "f32", 1.0), make(rng, 1500, "f32", size)
    before = f64(p)
    opt.add(p, state="block8")
    opt.step([g], 3, LR)
    zero = np.zeros(1500)
    check_last(opt, 0, before, f64(g), zero, zero, 0, 3, eps=eps)
    opt.close()


def test_moments_of_many_tensors(M):
    """More tensors than one launch takes, into given outputs and into new ones."""
    rng = np.random.default_rng(10)
    sizes = [int(x) for x in rng.integers(0, 600, 1100)]
    opt = M.AdamWGroup(seed=2)
    for i, n in enumerate(sizes):
        opt.add(torch.zeros(n, device="cuda"), state="block8" if i % 2 else "f32")
    opt.step([make(rng, n, "f32", 1.0) for n in sizes], 1, LR)
    m, v = opt.moments()
    out = [[torch.full((n,), 7.0, device="cuda") for n in sizes] for _ in range(2)]
    opt.moments(*out)
    for i, n in enumerate(sizes):
        st = opt.states[i]
        if i % 2:
            want = o.decode8(st["exp_avg"].cpu().numpy(), f64(st["exp_avg_scale"]), True)
            assert np.allclose(f64(m[i]), want, rtol=2 * U, atol=1e-38)
        else:
            assert torch.equal(m[i], st["exp_avg"]) and torch.equal(v[i], st["exp_avg_sq"])
        assert torch.equal(out[0][i], m[i]) and torch.equal(out[1][i], v[i])
    opt.close()

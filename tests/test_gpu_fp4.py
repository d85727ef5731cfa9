"""MXFP4 quantisation and products against the float64 definitions.

Codes, scales and values are exact.  A product's error: the products of codes
and scales are exact, the fp32 accumulator is rounded (or cut) once per 64
entries of K and inside an MMA its terms are aligned to the largest, so
|error| <= (K / 64 + 8) 2^-23 sum |a b|, and half a unit of a bf16 result.
"""

import numpy as np
import pytest

from oracle import operators_ref as o

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_15037_gb300 as pkg
    return pkg


@pytest.fixture(scope="module")
def fp4(M):
    f = M.Fp4Group()
    yield f
    assert f.status() == 0
    f.close()


def f64(x):
    return x.detach().double().cpu().numpy()


def matrix(rng, m, k, dtype, pitch=0, offset=0):
    """A device matrix with rows of differing scale, in rows `pitch` entries
    wider than k, `offset` entries into its buffer."""
    x = rng.standard_normal((m, k)) * np.exp(2 * rng.standard_normal((m, 1)))
    buf = torch.full((m * (k + pitch) + offset,), float("nan"), dtype=DT[dtype], device="cuda")
    view = buf[offset:].view(m, k + pitch)[:, :k]
    view.copy_(torch.tensor(x))
    return view


def same(a, ref):
    """Equal values and signs, NaN for NaN."""
    assert np.array_equal(a, ref, equal_nan=True) and np.array_equal(np.signbit(a[ref == 0]), np.signbit(ref[ref == 0]))


SHAPES = [(1, 1), (1, 32), (1, 33), (3, 31), (32, 1), (127, 129), (128, 128), (129, 257), (1, 4097), (300, 95), (513, 640)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("pitch,offset", [(0, 0), (8, 0), (3, 0), (8, 1)])
def test_quantize(M, fp4, dtype, shape, pitch, offset):
    rng = np.random.default_rng(1)
    x = matrix(rng, *shape, dtype, pitch, offset)
    ref = f64(x)
    for rows, cols in ((True, True), (True, False), (False, True)):
        got = fp4.quantize(x, rows=rows, cols=cols)
        got = got if rows and cols else (got, None) if rows else (None, got)
        for a, r in zip(got, (ref, ref.T)):
            if a is None:
                continue
            q, sf, val = o.operand(r)
            assert np.array_equal(a.sf.cpu().numpy(), sf)
            assert np.array_equal(a.q.cpu().numpy(), q)
            same(f64(fp4.dequantize(a)), val)
            out = torch.full((a.rows, a.cols + 5), 7.0, device="cuda")
            fp4.dequantize(a, out=out[:, 1:a.cols + 1])
            same(f64(out)[:, 1:a.cols + 1], val)
            assert (out[:, 0] == 7).all() and (out[:, a.cols + 1:] == 7).all()


def test_quantize_every_rounding(fp4):
    """Every bf16 value beside a 6 in its block (scale 1) and beside the extreme
    magnitudes of fp32; fp32 neighbours of every tie."""
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16)
    v = bits.view(torch.bfloat16)
    v = v[torch.isfinite(v)]
    for top in (6.0, 2.0 ** -126, 3e38):
        x = torch.zeros((len(v) + 30) // 31, 32, dtype=torch.bfloat16)
        x[:, 0] = top
        x[:, 1:].reshape(-1)
        flat = torch.zeros(x.shape[0] * 31, dtype=torch.bfloat16)
        flat[:len(v)] = v
        x[:, 1:] = flat.view(-1, 31)
        a = fp4.quantize(x.cuda())
        code, scale = o.quantize(f64(x))
        q, sf = o.pack(code, scale)
        assert np.array_equal(a.q.cpu().numpy(), q) and np.array_equal(a.sf.cpu().numpy(), sf)
    mid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], dtype=np.float32)
    pts = np.concatenate([mid, np.nextafter(mid, np.float32(9)), np.nextafter(mid, np.float32(0))])
    x = np.zeros((len(pts) * 4, 32), dtype=np.float32)
    for i, s in enumerate((1.0, -1.0, 2.0 ** -60, 2.0 ** 90)):
        x[i::4, 3] = pts * np.float32(s)
        x[i::4, 0] = np.float32(6 * abs(s))
    a = fp4.quantize(torch.tensor(x).cuda())
    q, sf, val = o.operand(x)
    assert np.array_equal(a.q.cpu().numpy(), q) and np.array_equal(a.sf.cpu().numpy(), sf)


def test_quantize_special_values(fp4):
    """Zeros keep a zero block; NaN and infinities make their block NaN and no other."""
    x = torch.zeros(70, 96, device="cuda")
    x[1, 40], x[2, 0], x[3, 95] = float("nan"), float("inf"), float("-inf")
    x[4, :] = 1.0
    rows, cols = fp4.quantize(x, rows=True, cols=True)
    for a, r in ((rows, f64(x)), (cols, f64(x).T)):
        q, sf, val = o.operand(r)
        assert np.array_equal(a.sf.cpu().numpy(), sf)
        got = f64(fp4.dequantize(a))
        assert np.array_equal(np.isnan(got), np.isnan(val)) and np.array_equal(got[~np.isnan(val)], val[~np.isnan(val)])


def check_product(got, a, b, dtype, k):
    ref = a @ b.T
    bound = (k / 64 + 8) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T) + 1e-42
    if dtype == "bf16":
        bound = bound * 1.01 + 2.0 ** -8 * np.abs(ref) + 1e-40
    err = np.abs(got - ref)
    assert np.all(err <= bound), (err - bound).max()


PRODUCTS = [(1, 16, 16), (1, 4096, 4096), (2, 1000, 513), (7, 130, 64), (16, 257, 1000), (31, 128, 128), (33, 96, 4097),
            (64, 2048, 96), (77, 1003, 2049), (128, 256, 256), (129, 257, 255), (200, 600, 33), (256, 512, 320),
            (300, 300, 1), (511, 1025, 640), (1000, 16, 3000), (2049, 384, 65), (1, 1, 1), (5, 20000, 40), (640, 5000, 384)]


@pytest.mark.parametrize("shape", PRODUCTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_product(M, fp4, shape, dtype):
    m, n, k = shape
    rng = np.random.default_rng(m + n + k)
    x, w = matrix(rng, m, k, "bf16"), matrix(rng, n, k, "f32")
    A, W = fp4.quantize(x), fp4.quantize(w)
    a, b = o.operand(f64(x))[2], o.operand(f64(w))[2]
    got = fp4.product(A, W, dtype=DT[dtype])
    check_product(f64(got), a, b, dtype, k)
    assert torch.equal(got, fp4.product(A, W, dtype=DT[dtype]))
    # into a strided output whose surroundings stay
    for pitch, offset in ((8, 0), (3, 0), (8, 1)):
        buf = torch.full((m * (n + pitch) + offset,), 7.0, dtype=DT[dtype], device="cuda")
        out = buf[offset:].view(m, n + pitch)
        fp4.product(A, W, out=out[:, :n])
        assert torch.equal(out[:, :n], got) and (out[:, n:] == 7).all() and (buf[:offset] == 7).all()
    # the same with the quantisation inside the call
    for src in (x, x.float()):
        assert torch.equal(fp4.linear(src, W, dtype=DT[dtype]), got)


@pytest.mark.parametrize("shape", [(12, 128, 64), (13, 131, 64), (25, 128, 600), (48, 2600, 2048), (100, 9001, 300),
                                   (128, 2060, 2300), (260, 40, 100), (385, 200, 600), (1025, 640, 2049), (1030, 640, 2048)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_product_at_the_ends_of_its_forms(M, fp4, shape, dtype):
    """Around the sizes where the tokens of a CTA are added up four at a time, K is shared
    by more CTAs, and pairs take over; last tiles of few tokens."""
    test_product(M, fp4, shape, dtype)


@pytest.mark.parametrize("shape", [(1, 300, 520), (40, 300, 520), (300, 300, 520)])
def test_scales_of_the_whole_range(M, fp4, shape):
    """Scales 2^-127 to 2^126 on both sides, block by block, whose products stay
    in fp32's range; and a NaN block reaches its row only."""
    m, n, k = shape
    rng = np.random.default_rng(3)
    kb = -(-k // 32)
    e = rng.integers(-60, 60, kb)
    e[:2] = (-125, 120)
    x = rng.choice([1.0, 1.5, -2.0, 3.0, 6.0, -6.0], (m, kb * 32)) * np.repeat(2.0 ** e, 32)
    w = rng.choice([1.0, 1.5, -2.0, 3.0, 6.0, -6.0], (n, kb * 32)) * np.repeat(2.0 ** -e, 32)
    x, w = torch.tensor(x[:, :k], dtype=torch.float32).cuda(), torch.tensor(w[:, :k], dtype=torch.float32).cuda()
    W = fp4.quantize(w)
    got = fp4.product(fp4.quantize(x), W, dtype=torch.float32)
    check_product(f64(got), o.operand(f64(x))[2], o.operand(f64(w))[2], "f32", k)
    x[m // 2, 70] = float("nan")
    bad = fp4.product(fp4.quantize(x), W, dtype=torch.float32)
    assert torch.isnan(bad[m // 2]).all()
    keep = torch.arange(m, device="cuda") != m // 2
    assert torch.equal(bad[keep], got[keep])


def test_gradients_of_a_linear_layer(M, fp4):
    """dx and dW against the formulas on the quantised operands, and against
    differences: moving one entry of an operand to another code moves
    <dy, x W^T> by that entry of the gradient times the move."""
    rng = np.random.default_rng(9)
    t, n, k = 96, 160, 224
    x, w, dy = (matrix(rng, *s, "bf16") for s in ((t, k), (n, k), (t, n)))
    xr, xc = fp4.quantize(x, rows=True, cols=True)
    wr, wc = fp4.quantize(w, rows=True, cols=True)
    gr, gc = fp4.quantize(dy, rows=True, cols=True)
    X, W, G = f64(x), f64(w), f64(dy)
    q = lambda v: o.operand(v)[2]  # noqa: E731
    dx, dw = fp4.product(gr, wc, dtype=torch.float32), fp4.product(gc, xc, dtype=torch.float32)
    check_product(f64(dx), q(G), q(W.T), "f32", n)
    check_product(f64(dw), q(G.T), q(X.T), "f32", t)
    # dW by differences of <dy, x W^T> in W, with dy and x as their column
    # operands hold them
    Gq, Xq = q(G.T).T, q(X.T).T
    W0 = q(W)
    for i, j in ((0, 0), (n - 1, k - 1), (37, 101)):
        h = 0.5
        W1 = W0.copy()
        W1[i, j] += h
        diff = ((Gq * (Xq @ W1.T)).sum() - (Gq * (Xq @ W0.T)).sum()) / h
        scale = np.abs(Gq[:, i]) @ np.abs(Xq[:, j])
        assert abs(f64(dw)[i, j] - diff) <= (t / 64 + 8) * 2.0 ** -23 * scale + 1e-9 * np.abs(Gq * (Xq @ W0.T)).sum()
    Wq = q(W.T).T
    Gr = q(G)
    for i, j in ((0, 0), (t - 1, k - 1), (50, 3)):
        h = 0.5
        X0 = q(X)
        X1 = X0.copy()
        X1[i, j] += h
        diff = ((Gr * (X1 @ Wq.T)).sum() - (Gr * (X0 @ Wq.T)).sum()) / h
        scale = np.abs(Gr[i]) @ np.abs(Wq[:, j])
        assert abs(f64(dx)[i, j] - diff) <= (n / 64 + 8) * 2.0 ** -23 * scale + 1e-9 * np.abs(Gr * (X0 @ Wq.T)).sum()


def test_gradient_feeds_the_grouped_step(M, fp4):
    """dW in bf16 is a gradient of the projected step, and the new W is
    quantised for the next product."""
    rng = np.random.default_rng(10)
    t, n, k, r = 128, 192, 320, 24
    x, dy = matrix(rng, t, k, "bf16"), matrix(rng, t, n, "bf16")
    grp = M.MoaraGroup(block_size=64)
    grp.add(n, k, r, "bf16", W0=rng.standard_normal((n, k)) * 0.02)
    grp.load_projector(grp.ids[0], np.linalg.qr(rng.standard_normal((n, r)))[0])
    W = grp.modules[0].W
    before = fp4.quantize(W).q.clone()
    dw = fp4.product(fp4.quantize(dy, rows=False, cols=True), fp4.quantize(x, rows=False, cols=True))
    grp.step([dw], 1, 1e-1)
    after = fp4.quantize(W)
    assert grp.status() == 0 and not torch.equal(before, after.q)
    assert np.array_equal(after.q.cpu().numpy(), o.operand(f64(W))[0])
    grp.close()


def test_other_stream_and_capture(M, fp4):
    rng = np.random.default_rng(11)
    for m in (1, 40, 300):
        x, w = matrix(rng, m, 1000, "bf16"), matrix(rng, 600, 1000, "f32")
        W = fp4.quantize(w)
        want = fp4.linear(x, W)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            a = fp4.linear(x, W)
        b = fp4.linear(x, W, stream=s.cuda_stream)
        s.synchronize()
        out = torch.zeros_like(want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            fp4.linear(x, W, out=out)
        graph.replay()
        torch.cuda.synchronize()
        for y in (a, b, out):
            assert torch.equal(y, want)


def test_offsets_behind_32_bits(M, fp4):
    """A matrix of 2^31 + entries: its last rows and columns."""
    rows, cols = 40_000, 65_600                           # 2.6e9 bf16 entries
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(200, cols, device="cuda").to(torch.bfloat16)
    x[-200:] = tail
    a, b = fp4.quantize(x, rows=True, cols=True)
    ref = fp4.quantize(tail)
    kb = -(-cols // 32)
    assert torch.equal(a.q.view(rows, -1)[-200:], ref.q.view(200, -1))
    part = fp4.quantize(x[-320:, -64:].contiguous(), rows=False, cols=True)
    assert torch.equal(b.q.view(cols, -1)[-64:, -160:], part.q.view(64, -1))
    vals = fp4.dequantize(a)
    assert torch.equal(vals[-200:], fp4.dequantize(ref)) and not vals[:-200].any() and kb == 2050
    y = fp4.product(fp4.quantize(torch.ones(3, cols, device="cuda")), a, dtype=torch.float32)
    want = fp4.product(fp4.quantize(torch.ones(3, cols, device="cuda")), ref, dtype=torch.float32)
    assert torch.equal(y[:, -200:], want) and not y[:, :-200].any()
    del x, vals, a, b
    # an output of more than 2^31 entries
    p, q = fp4.quantize(torch.ones(50_000, 32, device="cuda")), fp4.quantize(torch.ones(44_000, 32, device="cuda"))
    d = fp4.product(p, q)
    assert d.min().item() == d.max().item() == 32.0


def test_refusals(M, fp4):
    x = torch.ones(64, 96, device="cuda")
    A = fp4.quantize(x)
    for call in (lambda: fp4.quantize(x[0]), lambda: fp4.quantize(x.t()), lambda: fp4.quantize(x.half()),
                 lambda: fp4.quantize(x.cpu()), lambda: fp4.quantize(x, rows=False),
                 lambda: fp4.quantize(x, out=M.Fp4Matrix(64, 64)), lambda: fp4.product(A, fp4.quantize(x[:, :64])),
                 lambda: fp4.product(A, A, dtype=torch.float16), lambda: fp4.product(A, A, out=x),
                 lambda: fp4.linear(x[:, :32], A), lambda: M.Fp4Matrix(64, 96, q=A.q[:-1])):
        with pytest.raises(ValueError):
            call()
    before = M.moara_launch_count(fp4.ctx)

    def code(call):
        with pytest.raises(M.MoaraError) as ei:
            call()
        return ei.value.code
    q, sf, X = A.q.data_ptr(), A.sf.data_ptr(), x.data_ptr()
    Q = lambda *a: code(lambda: M.moara_fp4_quantize(fp4.ctx, *a))  # noqa: E731
    assert Q(X, 0, 0, 96, 96, q, sf) == M.MOARA_ERR_SHAPE and Q(X, 0, 64, 96, 95, q, sf) == M.MOARA_ERR_SHAPE
    assert Q(X, 2, 64, 96, 96, q, sf) == M.MOARA_ERR_INVALID_ARG and Q(None, 0, 64, 96, 96, q, sf) == M.MOARA_ERR_INVALID_ARG
    assert Q(X, 0, 64, 96, 96) == M.MOARA_ERR_INVALID_ARG and Q(X, 0, 64, 96, 96, q) == M.MOARA_ERR_INVALID_ARG
    assert Q(X + 2, 0, 64, 96, 96, q, sf) == M.MOARA_ERR_ALIGN and Q(X, 0, 64, 96, 96, q + 8, sf) == M.MOARA_ERR_ALIGN
    assert Q(X, 0, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31, q, sf) == M.MOARA_ERR_SHAPE
    assert Q(X, 0, 2 ** 31 - 100, 1, 1, q, sf) == M.MOARA_ERR_SHAPE
    P = lambda *a: code(lambda: M.moara_fp4_product(fp4.ctx, *a))  # noqa: E731
    D = torch.zeros(64, 64, device="cuda")
    d = D.data_ptr()
    big = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    ws = (big.data_ptr(), big.numel())
    assert P(64, 64, 0, q, sf, q, sf, d, 0, 64) == M.MOARA_ERR_SHAPE
    assert P(64, 64, 96, q, sf, q, sf, d, 0, 63) == M.MOARA_ERR_SHAPE
    assert P(64, 64, 96, q, sf, q, sf, d, 5, 64) == M.MOARA_ERR_INVALID_ARG
    assert P(64, 64, 96, None, sf, q, sf, d, 0, 64) == M.MOARA_ERR_INVALID_ARG
    assert P(64, 64, 96, q, sf, q + 1, sf, d, 0, 64) == M.MOARA_ERR_ALIGN
    assert P(64, 64, 96, q, sf, q, sf, d + 2, 0, 64) == M.MOARA_ERR_ALIGN
    L = lambda *a: code(lambda: M.moara_fp4_linear(fp4.ctx, *a))  # noqa: E731
    assert L(64, 64, 96, X, 0, 96, q, sf, d, 0, 64, ws[0], 64) == M.MOARA_ERR_WORKSPACE
    assert L(64, 64, 96, X, 0, 95, q, sf, d, 0, 64, *ws) == M.MOARA_ERR_SHAPE
    assert L(64, 64, 96, X, 0, 96, q, sf, d, 0, 64, ws[0] + 8, ws[1] - 8) == M.MOARA_ERR_ALIGN
    assert M.moara_launch_count(fp4.ctx) == before


PAIRS = [(1300, 2501, 200), (2047, 1281, 1), (2560, 1026, 4097), (300, 9732, 520), (8300, 300, 96), (257, 9729, 33),
         (2000, 5003, 31), (4000, 1540, 260)]


@pytest.mark.parametrize("shape", PAIRS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_product(M, fp4, shape, dtype):
    """Shapes of the 2-CTA pairs, with rows of the output on every alignment; the
    reference on the device, whose fp64 products and sums it takes."""
    m, n, k = shape
    rng = np.random.default_rng(m + n)
    x, w = matrix(rng, m, k, "bf16"), matrix(rng, n, k, "f32")
    A, W = fp4.quantize(x), fp4.quantize(w)
    a, b = (fp4.dequantize(y, dtype=torch.float32).double() for y in (A, W))
    ref, size = a @ b.t(), a.abs() @ b.abs().t()
    bound = (k / 64 + 8) * 2.0 ** -23 * size + 1e-42
    if dtype == "bf16":
        bound = bound * 1.01 + 2.0 ** -8 * ref.abs() + 1e-40
    got = fp4.product(A, W, dtype=DT[dtype])
    assert ((got.double() - ref).abs() <= bound).all()
    for pitch, offset in ((1, 0), (2, 0), (3, 1), (4, 2), (8, 0)):
        buf = torch.full((m * (n + pitch) + offset,), 7.0, dtype=DT[dtype], device="cuda")
        out = buf[offset:].view(m, n + pitch)
        fp4.product(A, W, out=out[:, :n])
        assert torch.equal(out[:, :n], got) and (out[:, n:] == 7).all() and (buf[:offset] == 7).all()
    assert torch.equal(fp4.linear(x, W, dtype=DT[dtype]), got)


@pytest.mark.parametrize("m", [1, 5, 8, 9, 16, 17])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pitch,offset", [(3, 0), (8, 1), (8, 0)])
def test_linear_reads_strided_rows(M, fp4, m, dtype, pitch, offset):
    """x as a slice of wider rows, whose surroundings are NaN."""
    rng = np.random.default_rng(m)
    n, k = 200, 1003
    x, W = matrix(rng, m, k, dtype, pitch, offset), fp4.quantize(matrix(rng, n, k, "f32"))
    assert torch.equal(fp4.linear(x, W), fp4.product(fp4.quantize(x), W))


@pytest.mark.parametrize("shape", [(33, 700), (1, 70), (130, 1025)])
def test_values_on_any_boundary(M, fp4, shape):
    """Values into rows of every alignment, in both types."""
    rng = np.random.default_rng(5)
    x = matrix(rng, *shape, "f32")
    A = fp4.quantize(x)
    want = o.operand(f64(x))[2]
    m, k = shape
    for dtype in ("f32", "bf16"):
        for pitch, offset in ((0, 0), (1, 0), (1, 1), (2, 1), (4, 0), (5, 3)):
            buf = torch.full((m * (k + pitch) + offset,), 7.0, dtype=DT[dtype], device="cuda")
            out = buf[offset:].view(m, k + pitch)
            fp4.dequantize(A, out=out[:, :k])
            same(f64(out)[:, :k], want)
            assert (out[:, k:] == 7).all() and (buf[:offset] == 7).all()


def placed(m, k, dtype, first, pitch):
    """An m x k matrix that begins `first` entries into its memory, whose surroundings are NaN."""
    whole = torch.full((first + m * pitch + 64,), float("nan"), device="cuda", dtype=dtype)
    return whole, whole[first:first + m * pitch].view(m, pitch)[:, :k]


def surroundings_kept(whole, x):
    kept = whole.clone()
    kept[x.storage_offset():].as_strided(x.shape, x.stride()).fill_(float("nan"))
    return bool(torch.isnan(kept).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("first,extra", [(0, 1), (1, 0), (2, 3), (3, 6), (4, 4), (5, 9), (6, 2), (7, 5)])
def test_boundaries_of_rows(M, fp4, dtype, first, extra):
    """Rows that begin on every byte of a line give the bits that aligned rows give, and
    nothing beside them is written or read into the result."""
    m, k, n = 301, 1091, 5003
    x = torch.randn(m, k, device="cuda").to(dtype)
    # the pitch 1104 is aligned
    a, at = fp4.quantize(placed_copy(x, 0, 1104), rows=True, cols=True)
    b, bt = fp4.quantize(placed_copy(x, first, k + extra), rows=True, cols=True)
    for y, z in ((a, b), (at, bt)):
        assert torch.equal(y.q, z.q) and torch.equal(y.sf, z.sf)
    for op in (a, at):
        want = torch.empty(op.rows, 1104 if op.cols == k else 304, device="cuda", dtype=dtype)[:, :op.cols]
        fp4.dequantize(op, out=want)
        whole, got = placed(op.rows, op.cols, dtype, first, op.cols + extra)
        fp4.dequantize(op, out=got)
        assert torch.equal(got, want) and surroundings_kept(whole, got)
    w = fp4.quantize(torch.randn(n, k, device="cuda"))               # 2 x 20 tiles: pairs
    want = torch.empty(m, 5008, device="cuda", dtype=dtype)[:, :n]
    fp4.product(a, w, out=want)
    whole, got = placed(m, n, dtype, first, n + extra)
    fp4.product(a, w, out=got)
    assert torch.equal(got, want) and surroundings_kept(whole, got)


def placed_copy(x, first, pitch):
    y = placed(*x.shape, x.dtype, first, pitch)[1]
    y.copy_(x)
    return y


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("last", range(1, 10))
def test_last_columns_of_pairs(M, fp4, dtype, last):
    """A last tile, or half of one, of a few columns on every boundary."""
    m, k = 2305, 64                                                  # 10 x 3 tiles
    a = fp4.quantize(torch.randn(m, k, device="cuda"))
    for n in (512 + last, 640 + last):
        w = fp4.quantize(torch.randn(n, k, device="cuda"))
        want = torch.empty(m, 784, device="cuda", dtype=dtype)[:, :n]
        fp4.product(a, w, out=want)
        whole, got = placed(m, n, dtype, last, n)
        fp4.product(a, w, out=got)
        assert torch.equal(got, want) and surroundings_kept(whole, got)

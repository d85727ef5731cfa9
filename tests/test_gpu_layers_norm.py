"""The norm with its residual and gradients against the float64 definitions."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import layers_ref as R  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_15037_gb300 as pkg
    return pkg


@pytest.fixture(scope="module")
def layer(M):
    g = M.LayerGroup()
    yield g
    assert g.status() == 0
    g.close()


def matrix(gen, t, n, dtype, pitch=0, offset=0, scale=1.0):
    """In rows `pitch` entries wider than n, `offset` entries into a buffer of NaN."""
    buf = torch.full((t * (n + pitch) + offset,), float("nan"), dtype=dtype, device="cuda")
    x = buf[offset:].view(t, n + pitch)[:, :n]
    x.copy_(torch.randn(t, n, generator=gen, device="cuda") * scale * torch.exp(torch.randn(1, n, generator=gen, device="cuda") / 2))
    return x


def gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def check(layer, t, n, dtype, ydtype, res, pitch=0, offset=0):
    g = gen(t * 7 + n)
    x = matrix(g, t, n, dtype, pitch, offset)
    r = matrix(g, t, n, dtype, pitch, offset, 2.0) if res else None
    gain = 1 + 0.1 * torch.randn(n, generator=g, device="cuda")
    h, y, s = layer.norm(x, gain, residual=r, eps=EPS, dtype=ydtype)
    hw, yw, sw = R.norm(x, r, gain, EPS)
    assert y.dtype == ydtype and torch.equal(h, hw) and (res or h is x)
    # the squares of an access add up with three roundings (and one of each fp32 square), which the
    # root halves, the rest of the sum in two numbers; then the root's own rounding.  y takes two more.
    es = (1 + (3 if dtype == torch.bfloat16 else 4) / 2) * R.F32 + 2.0 ** -30
    R.within(s, sw, sw * es)
    R.within(y, yw, yw.abs() * ((es + 2 * R.F32) * (1 + R.BF16) + R.half_step(ydtype)) + 2.0 ** -133)
    dy, dh = matrix(g, t, n, ydtype, pitch, offset, 1e-3), matrix(g, t, n, dtype, pitch, offset, 1e-3) if res else None
    dx, dg = layer.norm_backward(dy, h, gain, s, dh=dh)
    dxw, dgw, edx, edg = R.norm_backward(dy, hw, gain, sw, dh)
    assert dx.dtype == dtype
    R.within(dx, dxw, edx * (1 + R.BF16) + R.half_step(dtype) * dxw.abs() + 2.0 ** -133)
    R.within(dg, dgw, edg)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t,n", [(1, 1), (1, 16), (3, 31), (2, 33), (17, 255), (1, 257), (700, 64), (5, 1000), (64, 1003),
                                 (9, 2048), (1200, 1024), (4, 4095), (33, 4096), (2, 4104), (3, 8192), (2, 8193), (2, 16384),
                                 (3, 16385), (2, 18944), (1, 49152)])
def test_sizes(layer, dtype, t, n):
    for res in (False, True):
        check(layer, t, n, DT[dtype], DT[dtype], res)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t,n", [(10000, 250), (20001, 33), (10000, 256), (2500, 1003), (700, 4096), (700, 4099), (1300, 2056),
                                 (400, 9001), (400, 10000), (310, 16390), (310, 18944)])
def test_many_rows(layer, dtype, t, n):
    """Enough to fill the GPU, which other kernels take."""
    for res in (False, True):
        check(layer, t, n, DT[dtype], DT[dtype], res)
    check(layer, t, n, DT[dtype], DT["f32" if dtype == "bf16" else "bf16"], True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t,n", [(5, 8191), (3, 16001), (310, 17003), (160, 18943), (200, 27999), (3, 30001), (2, 48001), (1, 49151)])
def test_wide_rows_on_odd_places(layer, dtype, t, n):
    for res in (False, True):
        check(layer, t, n, DT[dtype], DT[dtype], res)
    check(layer, t, n, DT[dtype], DT[dtype], True, 2, 1)
    check(layer, t, n, DT[dtype], DT["f32" if dtype == "bf16" else "bf16"], True)


@pytest.mark.parametrize("n", [1000, 1003, 17003])
def test_many_rows_in_place(layer, n):
    g = gen(8)
    x, r, dy, dh = (matrix(g, 3000, n, torch.bfloat16) for _ in range(4))
    gain = torch.rand(n, generator=g, device="cuda")
    h, y, s = layer.norm(x, gain, residual=r)
    dx, dg = layer.norm_backward(dy, h, gain, s, dh=dh)
    x2, r2 = x.clone(), r.clone()
    h2, y2, _ = layer.norm(x2, gain, residual=r2, h=r2, out=x2)
    assert torch.equal(h2, h) and torch.equal(y2, y)
    for out in ("dy", "dh", "h"):
        c = {"dy": dy.clone(), "dh": dh.clone(), "h": h.clone()}
        dx2, dg2 = layer.norm_backward(c["dy"], c["h"], gain, s, dh=c["dh"], out=c[out])
        assert torch.equal(dx2, dx) and torch.equal(dg2, dg)


@pytest.mark.parametrize("dtype,ydtype", [("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("t,n", [(3, 40), (5, 1001), (7, 4096), (2, 9000), (2, 20000)])
def test_mixed_types(layer, dtype, ydtype, t, n):
    check(layer, t, n, DT[dtype], DT[ydtype], True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pitch,offset", [(8, 0), (3, 0), (8, 1), (0, 3), (5, 2)])
def test_pitches(layer, dtype, pitch, offset):
    for t, n in ((6, 24), (6, 1000), (6, 9001), (2600, 1000)):
        check(layer, t, n, DT[dtype], DT[dtype], True, pitch, offset)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t,n", [(1, 1), (1, 33), (129, 100), (130, 512), (256, 4096), (37, 1003)])
def test_quantize_is_that_of_y(M, layer, dtype, t, n):
    """Bit for bit: the operands of the fp32 y that norm gives."""
    fp4 = M.Fp4Group()
    g = gen(5)
    for res in (False, True):
        x = matrix(g, t, n, DT[dtype])
        r = matrix(g, t, n, DT[dtype]) if res else None
        gain = 1 + 0.1 * torch.randn(n, generator=g, device="cuda")
        h, y, s = layer.norm(x, gain, residual=r, dtype=torch.float32)
        want = fp4.quantize(y, rows=True, cols=True)
        for rows, cols in ((True, True), (True, False), (False, True)):
            h2, got, s2 = layer.norm_quantize(x, gain, residual=r, rows=rows, cols=cols)
            assert torch.equal(h, h2) and torch.equal(s, s2)
            pairs = zip(got, want) if rows and cols else [(got, want[0] if rows else want[1])]
            for a, b in pairs:
                assert (a.rows, a.cols) == (b.rows, b.cols) and torch.equal(a.q, b.q) and torch.equal(a.sf, b.sf)
    assert fp4.status() == 0
    fp4.close()


@pytest.mark.parametrize("n", [1000, 1003, 20000])
def test_in_place(layer, n):
    g = gen(1)
    x, r = matrix(g, 9, n, torch.bfloat16), matrix(g, 9, n, torch.bfloat16)
    gain = torch.rand(n, generator=g, device="cuda")
    h, y, s = layer.norm(x, gain, residual=r)
    dy, dh = matrix(g, 9, n, torch.bfloat16), matrix(g, 9, n, torch.bfloat16)
    dx, dg = layer.norm_backward(dy, h, gain, s, dh=dh)
    r2, x2 = r.clone(), x.clone()
    h2, y2, s2 = layer.norm(x2, gain, residual=r2, h=r2, out=x2)
    assert h2 is r2 and y2 is x2
    assert torch.equal(h2, h) and torch.equal(y2, y) and torch.equal(s2, s)
    for out in ("dy", "dh", "h"):
        c = {"dy": dy.clone(), "dh": dh.clone(), "h": h.clone()}
        dx2, dg2 = layer.norm_backward(c["dy"], c["h"], gain, s, dh=c["dh"], out=c[out])
        assert dx2 is c[out] and torch.equal(dx2, dx) and torch.equal(dg2, dg)


def test_rows_that_are_not_finite_stay_alone(layer):
    g = gen(2)
    x = matrix(g, 8, 500, torch.float32)
    want = layer.norm(x, torch.ones(500, device="cuda"), dtype=torch.float32)[1].clone()
    x[3, 7], x[5, 0] = float("nan"), float("inf")
    x[6] = 0
    h, y, s = layer.norm(x, torch.ones(500, device="cuda"), dtype=torch.float32)
    keep = [0, 1, 2, 4, 7]
    assert torch.equal(y[keep], want[keep]) and y[3].isnan().all() and s[5] == 0 and y[5, 0].isnan() and (y[5, 1:] == 0).all()
    assert (y[6] == 0).all() and abs(s[6].item() - 1e3) < 1e-3


@pytest.mark.parametrize("t,n", [(6, 300), (4000, 1024), (4000, 1003)])
def test_infinite_gradients_stay_in_their_row_and_column(layer, t, n):
    g = gen(12)
    h, dy = torch.randn(t, n, generator=g, device="cuda"), torch.randn(t, n, generator=g, device="cuda")
    gain = 1 + 0.1 * torch.randn(n, generator=g, device="cuda")
    s = R.norm(h, None, gain, EPS)[2].float()
    h[3, 5] = h[3, 5].abs() + 0.1
    want = layer.norm_backward(dy, h, gain, s)
    dy[3, 5] = float("inf")
    dx, dg = layer.norm_backward(dy, h, gain, s)
    keep, others = torch.arange(t, device="cuda") != 3, torch.arange(n, device="cuda") != 5
    assert torch.equal(dx[keep], want[0][keep]) and torch.equal(dg[others], want[1][others])
    assert dg[5] == float("inf")
    # the row's mean is infinite: what it is taken from is infinite of the other sign
    assert (dx[3, others] == -torch.sign(h[3, others]) * float("inf")).all() and dx[3, 5].isnan()


def test_gradient_by_differences(layer):
    """Central differences of sum(c y) + sum(e h) in the fp32 operator: second-order terms 1e-4,
    roundings 2^-24 |y| sqrt(n) / step."""
    g = gen(3)
    n, step = 40, 2.0 ** -6
    x, r = matrix(g, 3, n, torch.float32), matrix(g, 3, n, torch.float32)
    gain, c, e = (torch.randn(*s, generator=g, device="cuda") for s in ((n,), (3, n), (3, n)))

    def value(x, gain):
        h, y, _ = layer.norm(x, gain, residual=r, dtype=torch.float32)
        return (c.double() * y.double()).sum() + (e.double() * h.double()).sum()
    h, _, s = layer.norm(x, gain, residual=r, dtype=torch.float32)
    dx, dg = layer.norm_backward(c, h, gain, s, dh=e)
    for i, j in ((0, 0), (1, 7), (2, 39)):
        d = torch.zeros_like(x)
        d[i, j] = step
        num = (value(x + d, gain) - value(x - d, gain)) / (2 * step)
        assert abs(num - dx[i, j]) < 5e-3 * dx.abs().max()
        d = torch.zeros_like(gain)
        d[j] = step
        num = (value(x, gain + d) - value(x, gain - d)) / (2 * step)
        assert abs(num - dg[j]) < 1e-3 * dg.abs().max()


def test_stream_and_graphs(M, layer):
    """On a stream of its own, and two graphs that keep what they read and write apart."""
    g = gen(4)
    x, r = matrix(g, 50, 2000, torch.bfloat16), matrix(g, 50, 2000, torch.bfloat16)
    gain = torch.rand(2000, generator=g, device="cuda")

    def run(**kw):
        h, y, s = layer.norm(x, gain, residual=r, **kw)
        return (h, y, s, *layer.norm_backward(y, h, gain, s, dh=h, **kw))
    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run()
        graphs.append((graph, out))
    for graph, out in graphs:
        for o in out:
            o.zero_()
    for graph, _ in graphs + graphs:
        graph.replay()
    torch.cuda.synchronize()
    for _, out in graphs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals(M, layer):
    x = torch.zeros(4, 8, device="cuda")
    gain = torch.ones(8, device="cuda")
    for bad in (dict(gain=gain[:7]), dict(gain=gain.bfloat16()), dict(residual=x[:3]), dict(residual=x.bfloat16()), dict(h=x),
                dict(out=x[:, :7]), dict(dtype=torch.float16), dict(residual=x, h=x.bfloat16()), dict(x=x.half()), dict(x=x[0]),
                dict(x=x.t()), dict(x=x.cpu())):
        with pytest.raises(ValueError):
            layer.norm(**{"x": x, "gain": gain, **bad})
    for bad in (dict(eps=-1.0), dict(eps=float("nan")), dict(x=x[:0])):
        with pytest.raises(M.MoaraError):
            layer.norm(**{"x": x, "gain": gain, **bad})
    wide = torch.zeros(1, 49153, device="cuda")
    with pytest.raises(M.MoaraError) as e:
        layer.norm(wide, torch.ones(49153, device="cuda"))
    assert e.value.code == M.MOARA_ERR_UNSUPPORTED
    h, y, s = layer.norm(x, gain)
    for bad in (dict(dy=y[:3]), dict(rstd=s[:3]), dict(dh=x.bfloat16()), dict(out=x.bfloat16()), dict(gain=gain[:5])):
        with pytest.raises(ValueError):
            layer.norm_backward(**{"dy": y, "h": h, "gain": gain, "rstd": s, **bad})
    with pytest.raises(ValueError):
        layer.norm_quantize(x, gain, rows=False)

"""Calls of the layers' operators beside one another: two host threads, graphs beside other shapes,
lists of sequences that another stream reads when they are released; the norm's smallest rows and its
gain's gradient over many rows."""

import threading

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import layers_ref as R  # noqa: E402


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


def rand(gen, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=gen, device="cuda").to(dtype)


# rows of both shapes are taken by the same kernels, with shared memory of different sizes
SHAPES = [(8, 16384), (1300, 4096)]


def test_two_threads_of_different_shapes(M):
    """Each with a context and a stream of its own, through the C entries."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    failed, results, threads = [], [], []

    def run(rows, cols, start):
        try:
            layer, stream = M.LayerGroup(), torch.cuda.Stream()
            x, dy, gain = rand(gen, rows, cols), rand(gen, rows, cols), torch.ones(cols, device="cuda")
            y, dx, rstd, dgain = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda")
            size = M.moara_rms_norm_backward_workspace_bytes(rows, cols)
            ws = torch.empty(size, dtype=torch.uint8, device="cuda")
            bf16, s = M.MOARA_DTYPE_BF16, stream.cuda_stream
            torch.cuda.synchronize()
            start.wait()
            for i in range(6000):
                M.moara_rms_norm(layer.ctx, rows, cols, x.data_ptr(), cols, 0, 0, bf16, gain.data_ptr(), 1e-6, 0, 0, y.data_ptr(), bf16,
                                 cols, rstd.data_ptr(), s)
                M.moara_rms_norm_backward(layer.ctx, rows, cols, dy.data_ptr(), bf16, cols, x.data_ptr(), bf16, cols, gain.data_ptr(),
                                          rstd.data_ptr(), 0, 0, dx.data_ptr(), cols, dgain.data_ptr(), ws.data_ptr(), size, s)
                if i % 500 == 499:
                    stream.synchronize()
            stream.synchronize()
            wx, wg, ex, eg = R.norm_backward(dy, x, gain, R.norm(x, None, gain, 1e-6)[2], None)
            results.append((dx, wx, ex * (1 + R.BF16) + R.BF16 * wx.abs() + 2.0 ** -126))
            results.append((dgain, wg, eg))
            assert layer.status() == 0
            layer.close()
        except Exception as e:                               # noqa: BLE001
            failed.append((rows, cols, e))
    start = threading.Barrier(len(SHAPES))
    for shape in SHAPES:
        threads.append(threading.Thread(target=run, args=(*shape, start)))
        threads[-1].start()
    for t in threads:
        t.join()
    assert not failed, failed
    for x in results:
        R.within(*x)


def test_graphs_beside_other_shapes(layer):
    """A recorded call keeps its shared memory where a smaller one follows."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = [(rand(gen, *s), rand(gen, *s), torch.ones(s[1], device="cuda")) for s in SHAPES]

    def run(a):
        h, y, s = layer.norm(a[0], a[2])
        return (y, s) + layer.norm_backward(a[1], h, a[2], s)
    want = [run(a) for a in x]
    graphs = []
    for a in x:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            got = run(a)
        graphs[-1].got = got
    for first, second in ((0, 1), (1, 0)):
        run(x[second])
        graphs[first].replay()
        run(x[second])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(graphs[first].got, want[first]))


@pytest.mark.parametrize("handle", [False, True])
def test_recorded_sequences_outlive_their_release(M, handle):
    layer = M.LayerGroup()
    lengths, h, d = [300, 77, 1000, 5], 2, 64
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (rand(gen, sum(lengths), h, d) for _ in range(3))
    want = layer.attention(q, k, v, layer.sequences(lengths))
    torch.cuda.synchronize()
    seqs = layer.sequences(lengths)
    place, size = seqs._tiles.data_ptr(), seqs._tiles.numel()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)                       # some 50 ms
    seqs.record_stream(side.cuda_stream if handle else side)
    got = layer.attention(q, k, v, seqs, stream=side.cuda_stream)
    del seqs
    # what is allocated now lies elsewhere, while the call still waits for its turn
    others = [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert not side.query() and all(x.data_ptr() != place for x in others)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and layer.status() == 0
    layer.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,value", [(2, 49152, 3e-18), (3, 4096, 1.2e-19), (700, 4096, 1.2e-19), (5, 1003, 2e-19), (3, 8, 1e-15)])
def test_rows_of_next_to_nothing(layer, dtype, rows, cols, value):
    """No epsilon, and a mean square below fp32's normal numbers: the sum of the squares is inside them."""
    x = torch.zeros(rows, cols, dtype=dtype, device="cuda")
    x[:, 3] = value
    x[rows - 1, 5] = -value
    gain = torch.ones(cols, device="cuda")
    for eps in (0.0, 1e-38):
        _, y, s = layer.norm(x, gain, eps=eps, dtype=torch.float32)
        _, yw, sw = R.norm(x, None, gain, eps)
        # two squares and their sum, one fp32 rounding each, which the root halves; the root's own, and y's two.  A float's
        # eps is not the double's
        es = (3 / 2 + 1) * R.F32 + (0 if eps == 0 else abs(torch.tensor(eps).double().item() / eps - 1)) + 2.0 ** -30
        R.within(s, sw, es * sw)
        R.within(y, yw, (es + 2 * R.F32) * yw.abs())


@pytest.mark.parametrize("cols", [1024, 1027])
def test_gain_of_rows_far_apart(layer, cols):
    """Rows are taken a grid apart: of 300 beside one another no CTA adds up more than two, however many rows there are."""
    gen = torch.Generator(device="cuda").manual_seed(cols)
    rows = 200_000
    h, dy = rand(gen, rows, cols), torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    dy[-300:] = rand(gen, 300, cols)
    gain = 1 + 0.1 * torch.randn(cols, generator=gen, device="cuda")
    s = layer.norm(h, gain)[2]
    dx, dgain = layer.norm_backward(dy, h, gain, s)
    wx, wg, ex, eg = R.norm_backward(dy[-300:], h[-300:], gain, s[-300:].double(), None)
    R.within(dgain, wg, eg)
    R.within(dx[-300:], wx, ex * (1 + R.BF16) + R.BF16 * wx.abs() + 2.0 ** -126)
    assert (dx[:-300] == 0).all()

"""Causal attention over packed sequences and its gradients against the float64 definition."""

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


def inputs(t, h, hk, d, seed=0):
    """q, k, v slices of one projection, keys and values with a common direction."""
    g = torch.Generator(device="cuda").manual_seed(seed + t * 3 + h * 5 + d)
    x = torch.randn(t, h + 2 * hk, d, generator=g, device="cuda") + 0.5 * torch.randn(1, h + 2 * hk, d, generator=g, device="cuda")
    x = x.to(torch.bfloat16)
    do = torch.randn(t, h, d, generator=g, device="cuda").to(torch.bfloat16)
    return x[:, :h], x[:, h:h + hk], x[:, h + hk:], do


def check(layer, lengths, h, hk, d, scale=None, grad=True, x=None):
    """Elementwise bounds, and the whole: a rounding's error is 2^-8 / sqrt(3) of its value at
    most on average, three of them come together (P, dS or the output of either pass), twice that
    where sums cancel."""
    n = sum(lengths)
    q, k, v, do = inputs(n, h, hk, d) if x is None else x
    seqs = layer.sequences(lengths)
    out, lse, rest = layer.attention(q, k, v, seqs, scale=scale, train=True)
    plain = layer.attention(q, k, v, seqs, scale=scale)
    assert len(plain) == 2 and torch.equal(plain[0], out) and torch.equal(plain[1], lse)
    got = {"out": out, "lse": lse}
    if grad:
        got["dq"], got["dk"], got["dv"] = layer.attention_backward(do, q, k, v, out, lse, seqs, rest=rest, scale=scale)
    assert layer.status() == 0
    want, tol = R.attention(q[:n], k[:n], v[:n], lengths, d ** -0.5 if scale is None else scale, do[:n] if grad else None)
    for name, w in want.items():
        R.within(got[name], w, tol[name])
        if name != "lse" and w.norm() > 0 and max(lengths) > 1:
            assert (got[name].double() - w).norm() <= 2.0 ** -7 * w.norm(), name
    return got


LENGTHS = [[1], [2], [16], [17], [64], [127], [128], [129], [255], [256], [257], [300], [1, 1, 1], [5, 128, 3], [0, 7, 0, 130, 0],
           [1, 17, 129, 300, 64, 5, 511, 77], [700]]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda x: "-".join(map(str, x)))
def test_outputs(layer, lengths, d):
    check(layer, lengths, 2, 1, d, grad=False)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda x: "-".join(map(str, x)))
def test_gradients(layer, lengths, d):
    check(layer, lengths, 2, 1, d)


@pytest.mark.parametrize("h,hk", [(1, 1), (3, 3), (4, 2), (7, 1), (28, 4), (16, 16)])
def test_heads(layer, h, hk):
    check(layer, [130, 33, 400], h, hk, 64)
    check(layer, [140], h, hk, 128)


@pytest.mark.parametrize("d", [8, 16, 40, 56, 72, 80, 96, 120])
def test_other_widths(layer, d):
    check(layer, [150, 20], 4, 2, d)


@pytest.mark.parametrize("d", [64, 128])
def test_long(layer, d):
    check(layer, [2500, 1], 2, 1, d)


MANY = [300, 1, 129, 256, 700, 128, 257, 64] * 4


@pytest.mark.parametrize("h,hk,d", [(16, 4, 64), (8, 8, 128), (14, 2, 128), (40, 1, 40)])
def test_more_pairs_of_tiles_than_run_at_once(layer, h, hk, d):
    check(layer, MANY, h, hk, d)


def test_long_and_more_than_run_at_once(layer):
    check(layer, [4200], 9, 3, 128)


def test_many_pairs_on_two_streams_and_replayed(layer):
    """Kernels that take over the tiles of CTAs that have not begun, beside one another."""
    xs = [inputs(sum(MANY), 16, 4, d, seed=7) for d in (64, 128)]
    seqs = layer.sequences(MANY)

    def both(x):
        q, k, v, do = x
        out, lse, rest = layer.attention(q, k, v, seqs, train=True)
        return (out, lse, rest) + layer.attention_backward(do, q, k, v, out, lse, seqs, rest=rest)
    want = [both(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    graphs, made = [], []
    for x, s in zip(xs, streams):
        with torch.cuda.stream(s):
            both(x)
        s.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=s):
            made.append(both(x))
    torch.cuda.synchronize()
    for _ in range(10):
        got = []
        for x, s, g in zip(xs, streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
                got.append(both(x))
        torch.cuda.synchronize()
        for a in (got, made):
            for x, y in zip(a, want):
                assert all(torch.equal(m, n) for m, n in zip(x, y))


def test_scale(layer):
    """Large scores: rows that see one key with all their weight, references that rise again and
    again."""
    check(layer, [300], 2, 2, 64, scale=2.0)
    q, k, v, do = inputs(600, 1, 1, 128)
    k = k * torch.linspace(0.1, 6, 600, device="cuda").view(-1, 1, 1).to(torch.bfloat16)
    check(layer, [600], 1, 1, 128, x=(q, k, v, do))


def test_orders_of_memory(layer):
    """Heads outermost, and padded pitches."""
    q, k, v, do = inputs(200, 4, 2, 64)
    want = check(layer, [150, 50], 4, 2, 64)

    def other(x, how):
        if how == "heads":
            return x.transpose(0, 1).contiguous().transpose(0, 1)
        y = torch.full((x.shape[0], x.shape[1] + 1, 72), float("nan"), dtype=x.dtype, device="cuda")[:, :x.shape[1], :64]
        return y.copy_(x)
    seqs = layer.sequences([150, 50])
    for how in ("heads", "padded"):
        a, b, c, g = (other(x, how) for x in (q, k, v, do))
        out, lse, rest = layer.attention(a, b, c, seqs, train=True)
        assert torch.equal(out, want["out"]) and torch.equal(lse, want["lse"])
        got = layer.attention_backward(g, a, b, c, out, lse, seqs, rest=rest)
        assert all(torch.equal(x, want[n]) for x, n in zip(got, ("dq", "dk", "dv")))


@pytest.mark.parametrize("d", [64, 128])
def test_sequences_do_not_meet(layer, d):
    """A sequence of infinities and NaN, and rows behind the last one, leave the others as they
    are, bit for bit."""
    lengths = [100, 60, 131, 20, 0, 7]
    q, k, v, do = inputs(sum(lengths) + 50, 4, 2, d)
    q, k, v, do = (x.clone() for x in (q, k, v, do))
    seqs = layer.sequences(lengths)

    def run():
        out, lse, rest = layer.attention(q, k, v, seqs, train=True)
        return (out, lse.t(), rest, *layer.attention_backward(do, q, k, v, out, lse, seqs, rest=rest))
    want = run()
    n = sum(lengths)
    for x in want:
        assert (x[n:] == 0).all() and x.isfinite().all()
    bad = slice(100, 160)
    for x in (q, k, v, do):
        x[bad] = float("nan")
        x[n:] = float("inf")
        x[n + 3:] = float("nan")
    got = run()
    for x, y in zip(got, want):
        assert torch.equal(x[:100], y[:100]) and torch.equal(x[160:], y[160:])
    for x in got[:2]:
        assert x[bad].isnan().all()


def test_keys_without_probability(layer):
    """A first tile of keys whose scores are minus infinity, before scores far below zero."""
    q, k, v, _ = (x.clone() for x in inputs(600, 2, 1, 64))
    q[:, :, 0], k[:, :, 0] = 1.0, -2000.0
    k[:128, :, 0] = float("-inf")
    out, lse = layer.attention(q, k, v, layer.sequences([600]))
    want, tol = R.attention(q, k, v, [600], 0.125)
    eS = (q.double().abs().amax() * 64 * 8 + 2000) * 0.125 * 12 * 2.0 ** -23        # of the scores that count
    for n in range(2):
        vs = v[128:, 0].double()
        slack = (2.0 ** -8 + 2 * eS + 2.0 ** -20 * want["lse"][n, 128:].abs().amax()) * vs.abs().amax() * 2
        assert (out[128:, n].double() - want["out"][128:, n]).abs().amax() <= slack
        assert (lse[n, 128:].double() - want["lse"][n, 128:]).abs().amax() <= eS + 2.0 ** -22 * 300
    assert out[:128].isnan().all() and want["out"][:128].isnan().all()


def test_rest_is_what_the_rounding_dropped(layer):
    q, k, v, do = inputs(500, 2, 1, 128)
    seqs = layer.sequences([500])
    out, lse, rest = layer.attention(q, k, v, seqs, train=True)
    want, tol = R.attention(q, k, v, [500], 128 ** -0.5)
    # what is left is P's rounding: 2^-8 of sum p |v|, the output's own rounding squared
    R.within(out.double() + rest.double(), want["out"], tol["out"] - R.BF16 * want["out"].abs() * (1 - 2 * R.BF16))
    without = layer.attention_backward(do, q, k, v, out, lse, seqs)
    with_ = layer.attention_backward(do, q, k, v, out, lse, seqs, rest=rest)
    assert torch.equal(without[2], with_[2]) and not torch.equal(without[0], with_[0])


def test_same_results_again(layer):
    q, k, v, do = inputs(900, 8, 2, 128)
    seqs = layer.sequences([500, 400])
    out, lse, rest = layer.attention(q, k, v, seqs, train=True)
    first = layer.attention_backward(do, q, k, v, out, lse, seqs, rest=rest)
    for _ in range(3):
        o, l, r = layer.attention(q, k, v, seqs, train=True)
        again = layer.attention_backward(do, q, k, v, o, l, seqs, rest=r)
        assert all(torch.equal(a, b) for a, b in zip((out, lse, rest, *first), (o, l, r, *again)))


def test_gradient_by_differences(layer):
    """Along a random direction of each input: the loss c out in fp32 of bf16 outputs, whose
    roundings are 2^-9 of sum |c out| / sqrt(n) over the step."""
    q, k, v, do = (x.clone() for x in inputs(200, 2, 1, 64))
    seqs = layer.sequences([200])
    out, lse, rest = layer.attention(q, k, v, seqs, train=True)
    grads = layer.attention_backward(do, q, k, v, out, lse, seqs, rest=rest)

    def value(*x):
        out, _, rest = layer.attention(*x, seqs, train=True)
        return ((out.double() + rest.double()) * do.double()).sum()
    g = torch.Generator(device="cuda").manual_seed(1)
    for i in range(3):
        x = [q, k, v]
        step = torch.randn(x[i].shape, generator=g, device="cuda").sign() * 0.0625
        y, z = list(x), list(x)
        y[i], z[i] = (x[i] + step).to(torch.bfloat16), (x[i] - step).to(torch.bfloat16)
        num = value(*y) - value(*z)
        want = (grads[i].double() * (y[i].double() - z[i].double())).sum()
        # third-order terms and P's rounding: a twentieth of the gradient's norm along such a direction
        assert abs(num - want) < 0.05 * grads[i].double().norm() * 0.125, i


def test_streams_and_graphs(M, layer):
    q, k, v, do = inputs(400, 4, 2, 128)
    seqs = layer.sequences([100, 300])

    def run(**kw):
        out, lse, rest = layer.attention(q, k, v, seqs, train=True, **kw)
        return (out, lse, rest, *layer.attention_backward(do, q, k, v, out, lse, seqs, rest=rest, **kw))
    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(stream=side.cuda_stream)
    also = run()                                                    # two calls at once
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, got, also))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run()
        graphs.append((graph, out))
    for graph, _ in graphs + graphs:
        graph.replay()
    torch.cuda.synchronize()
    for _, out in graphs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    # two graphs at once, each with its own outputs and workspaces
    with torch.cuda.stream(side):
        graphs[0][0].replay()
    graphs[1][0].replay()
    torch.cuda.synchronize()
    for _, out in graphs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_no_tokens(layer):
    q, k, v, do = inputs(5, 2, 1, 64)
    for lengths in ([], [0], [0, 0]):
        seqs = layer.sequences(lengths)
        for n in (0, 5):
            a = [x[:n] for x in (q, k, v, do)]
            out, lse, rest = layer.attention(*a[:3], seqs, train=True)
            got = layer.attention_backward(a[3], *a[:3], out, lse, seqs, rest=rest)
            assert out.shape == (n, 2, 64) and lse.shape == (2, n) and (out == 0).all() and all((x == 0).all() for x in got)


def test_refusals(M, layer):
    q, k, v, do = inputs(10, 4, 2, 64)
    seqs = layer.sequences([4, 6])
    out, lse, rest = layer.attention(q, k, v, seqs, train=True)
    for bad in (dict(q=q.float()), dict(q=q[0]), dict(k=k[:9]), dict(v=v[:, :1]), dict(k=k[..., :32]), dict(q=q.transpose(1, 2)),
                dict(v=v.cpu())):
        with pytest.raises(ValueError):
            layer.attention(**{"q": q, "k": k, "v": v, "seqs": seqs, **bad})

    def code(call):
        with pytest.raises(M.MoaraError) as e:
            call()
        return e.value.code
    three = torch.zeros(10, 3, 64, dtype=torch.bfloat16, device="cuda")
    assert code(lambda: layer.attention(q, three, three, seqs)) == M.MOARA_ERR_SHAPE
    assert code(lambda: layer.attention(q[:9], k[:9], v[:9], seqs)) == M.MOARA_ERR_SHAPE
    assert code(lambda: layer.attention(*(x[..., :60] for x in (q, k, v)), seqs)) == M.MOARA_ERR_UNSUPPORTED
    wide = torch.zeros(10, 2, 136, dtype=torch.bfloat16, device="cuda")
    assert code(lambda: layer.attention(wide, wide, wide, seqs)) == M.MOARA_ERR_UNSUPPORTED
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert code(lambda: layer.attention(q, k, v, seqs, scale=scale)) == M.MOARA_ERR_INVALID_ARG
    odd = torch.zeros(10, 2, 68, dtype=torch.bfloat16, device="cuda")[..., :64]
    assert code(lambda: layer.attention(q, odd, v, seqs)) == M.MOARA_ERR_ALIGN
    shifted = torch.zeros(10 * 2 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(10, 2, 64)
    assert code(lambda: layer.attention(q, k, shifted, seqs)) == M.MOARA_ERR_ALIGN
    assert code(lambda: layer.attention(q, k[:, :1].expand(10, 2, 64), v, seqs)) == M.MOARA_ERR_ALIGN
    for bad in (dict(out=out[:9]), dict(lse=lse.t()), dict(rest=rest.float()), dict(dout=do[:, :2]), dict(out=out.transpose(0, 1))):
        with pytest.raises(ValueError):
            layer.attention_backward(**{"dout": do, "q": q, "k": k, "v": v, "out": out, "lse": lse, "seqs": seqs, "rest": rest, **bad})
    for lengths in ([-1], [3, -2]):
        with pytest.raises(M.MoaraError):
            layer.sequences(lengths)
    with pytest.raises(ValueError):
        layer.sequences([2 ** 31])

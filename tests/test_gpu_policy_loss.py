"""The policy loss and its gradient against the float64 definition."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import layers_ref as R  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
CLIP = 0.2, 0.28


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


def inputs(t, v, dtype, pitch=0, offset=0, seed=0):
    """Ratios lie 1e-3 and more off the clip's borders."""
    g = torch.Generator(device="cuda").manual_seed(seed + t * 31 + v)

    def normal(*s):
        return torch.randn(*s, generator=g, device="cuda")
    buf = torch.full((t * (v + pitch) + offset,), float("nan"), dtype=dtype, device="cuda")
    z = buf[offset:].view(t, v + pitch)[:, :v]
    z.copy_(normal(t, v) * 2)
    target = torch.randint(0, v, (t,), generator=g, device="cuda")
    lp = torch.log_softmax(z.double(), 1).gather(1, target[:, None])[:, 0]
    d = 0.3 * normal(t).double()
    for b in (1 - CLIP[0], 1 + CLIP[1]):
        d = torch.where((d.exp() - b).abs() < 2e-3, d + 0.02, d)
    w = (torch.rand(t, generator=g, device="cuda") < 0.8) * (0.5 + torch.rand(t, generator=g, device="cuda")) / t
    return dict(logits=z, targets=target, old=(lp - d).float(), adv=normal(t), weights=w, ref=(lp + 0.3 * normal(t)).float())


def check(layer, x, kl, **kw):
    sums, lp, dz = layer.policy_loss(**x, clip=CLIP, kl=kl, **kw)
    ref = x["ref"] if kl else None
    want, tol = R.policy_loss(x["logits"], x["targets"], x["old"], x["adv"], x["weights"], ref, 1 - CLIP[0], 1 + CLIP[1], kl)
    assert dz.dtype == x["logits"].dtype
    for a, b, c in zip((sums, lp, dz), want, tol):
        R.within(a, b, c)
    return sums, lp, dz


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t,v", [(1, 1), (1, 2), (3, 7), (2, 8), (5, 33), (17, 1000), (1, 4099), (24, 32000), (300, 500), (1200, 97),
                                 (7, 50001), (2, 150000), (400, 40000)])
def test_sizes(layer, dtype, t, v):
    for kl in (0.0, 0.05):
        check(layer, inputs(t, v, DT[dtype]), kl)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_vocabulary_beyond_shared_memory(layer, dtype):
    check(layer, inputs(2, 900001, DT[dtype]), 0.05)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pitch,offset", [(8, 0), (3, 0), (8, 1), (0, 3), (1, 2)])
def test_pitches(layer, dtype, pitch, offset):
    for t, v in ((5, 333), (3, 20003)):
        x = inputs(t, v, DT[dtype], pitch, offset)
        want = check(layer, x, 0.05)
        # into other lines, and over the logits
        out = torch.full((t, v + 5), 7.0, dtype=DT[dtype], device="cuda")
        got = layer.policy_loss(**x, clip=CLIP, kl=0.05, out=out[:, 2:v + 2])[2]
        assert torch.equal(got, want[2]) and (out[:, :2] == 7).all() and (out[:, v + 2:] == 7).all()
        got = layer.policy_loss(**x, clip=CLIP, kl=0.05, out=x["logits"])
        assert got[2] is x["logits"] and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tokens_that_do_not_count(layer, dtype):
    """Whatever their inputs hold, and without a trace in the others."""
    x = inputs(12, 3001, DT[dtype])
    x["weights"][:] = 0.25
    want = [y.clone() for y in check(layer, x, 0.05)]
    off = [2, 3, 7, 11]
    x["weights"][[2, 3]] = 0
    x["targets"][7], x["targets"][11] = -100, 3001
    x["logits"][2] = float("nan")
    x["logits"][11, 5] = float("inf")
    for name in ("old", "adv", "ref"):
        x[name][off] = float("nan")
    sums, lp, dz = layer.policy_loss(**x, clip=CLIP, kl=0.05)
    keep = [i for i in range(12) if i not in off]
    assert torch.equal(dz[keep], want[2][keep]) and torch.equal(lp[keep], want[1][keep])
    assert (dz[off] == 0).all() and (lp[[7, 11]] == 0).all() and sums.isfinite().all()
    x = {k: v[keep].contiguous() for k, v in x.items()}
    check(layer, x, 0.05)


def test_masked_entries_of_the_vocabulary(layer):
    """Logits of minus infinity have no probability and no gradient."""
    for dtype, v in ((torch.float32, 40), (torch.bfloat16, 33000)):
        x = inputs(4, v, dtype)
        hidden = torch.rand(4, v, device="cuda") < 0.5
        hidden[:, :v // 3] = True                           # whole parts of a row among them
        hidden.scatter_(1, x["targets"][:, None], False)
        full = layer.policy_loss(**x, clip=CLIP)
        x["logits"].masked_fill_(hidden, float("-inf"))
        sums, lp, dz = layer.policy_loss(**x, clip=CLIP)
        z = x["logits"].double()
        want = torch.log_softmax(z, 1).gather(1, x["targets"][:, None])[:, 0]
        assert (dz[hidden] == 0).all() and dz.isfinite().all() and sums.isfinite().all()
        R.within(lp, want, 2.0 ** -18 + 2.0 ** -23 * want.abs())
        assert (lp >= full[1]).all()


def test_rows_of_nothing_but_infinities_are_nan(layer):
    x = inputs(3, 100, torch.float32)
    x["weights"][:] = 1.0
    x["logits"][1] = float("-inf")
    sums, lp, dz = layer.policy_loss(**x, clip=CLIP)
    assert lp[1].isnan() and sums[0].isnan() and dz[[0, 2]].isfinite().all()


def test_defaults(layer):
    """No weights: the mean.  No gradient where none is asked for."""
    x = inputs(9, 500, torch.float32)
    w = x.pop("weights")
    got = layer.policy_loss(**x, clip=CLIP, kl=0.1)
    x["weights"] = torch.full_like(w, 1 / 9)
    want = layer.policy_loss(**x, clip=CLIP, kl=0.1)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    sums, lp, dz = layer.policy_loss(**x, clip=CLIP, kl=0.1, grad=False)
    assert dz is None and torch.equal(sums, want[0]) and torch.equal(lp, want[1])


def test_gradient_by_differences(layer):
    """Central differences of the loss (fp32: 2^-23 of it over the step) along the logits."""
    x = inputs(4, 30, torch.float32)
    x["weights"][:] = 1.0
    dz = layer.policy_loss(**x, clip=CLIP, kl=0.3)[2].clone()
    step = 2.0 ** -8
    for i in range(4):
        for j in {0, 11, int(x["targets"][i])}:
            val = []
            for s in (step, -step):
                y = {k: v.clone() for k, v in x.items()}
                y["logits"][i, j] += s
                val.append(layer.policy_loss(**y, clip=CLIP, kl=0.3)[0][0].item())
            assert abs((val[0] - val[1]) / (2 * step) - dz[i, j].item()) < 1e-3


def test_stream_and_graphs(layer):
    x = inputs(60, 3000, torch.bfloat16)
    want = layer.policy_loss(**x, clip=CLIP, kl=0.05)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = layer.policy_loss(**x, clip=CLIP, kl=0.05, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = layer.policy_loss(**x, clip=CLIP, kl=0.05)
        graphs.append((graph, out))
    for graph, _ in graphs + graphs:
        graph.replay()
    torch.cuda.synchronize()
    for _, out in graphs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals(M, layer):
    x = inputs(4, 50, torch.float32)
    for bad in (dict(targets=x["targets"].int()), dict(old=x["old"][:3]), dict(adv=x["adv"].double()), dict(logits=x["logits"].half()),
                dict(ref=None, kl=0.1), dict(weights=x["weights"].bfloat16()), dict(out=x["logits"].bfloat16()),
                dict(grad=False, out=x["logits"]), dict(logits=x["logits"].t())):
        with pytest.raises(ValueError):
            layer.policy_loss(**{**x, "kl": 0.05, **bad})
    for bad in (dict(clip=(1.5, 0.2)), dict(clip=(-0.1, 0.2)), dict(clip=(0.2, -0.1)), dict(clip=(float("nan"), 0.2)), dict(kl=-1.0),
                dict(kl=float("nan"))):
        with pytest.raises(M.MoaraError):
            layer.policy_loss(**{**x, **bad})
    y = {k: v[:0] for k, v in x.items()}
    with pytest.raises(M.MoaraError):
        layer.policy_loss(**y)

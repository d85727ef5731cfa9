"""The policy loss where its exponentials or its gradient leave fp32's range, and where a row's
logits are the type's lowest or largest."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import layers_ref as R  # noqa: E402

CLIP = 0.2, 0.28
TYPES = [torch.float32, torch.bfloat16]
SIZES = [(300, 1000), (5, 1003), (2, 32003), (2, 900001)]       # a CTA a row, and clusters; the last from L2


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


def inputs(t, v, dtype):
    """Of unit weight; ratios are 1, away from the clip's borders."""
    g = torch.Generator(device="cuda").manual_seed(t + v)
    z = (2 * torch.randn(t, v, generator=g, device="cuda")).to(dtype)
    target = torch.randint(0, v, (t,), generator=g, device="cuda")
    lp = torch.log_softmax(z.double(), 1).gather(1, target[:, None])[:, 0]
    return dict(logits=z, targets=target, old=lp.float(), adv=torch.randn(t, generator=g, device="cuda"),
                weights=torch.ones(t, device="cuda"), ref=lp.float() + 0.1)


def unlikely(x, row, far):
    """The target's logit so that its log-probability is some -far."""
    z, t = x["logits"], x["targets"][row]
    z[row, t] = float("-inf")
    z[row, t] = torch.logsumexp(z[row].double(), 0) - far


def logp(x, row):
    return torch.log_softmax(x["logits"][row].double(), 0)[x["targets"][row]]


def within(x, kl, got):
    """R.policy_loss of rows whose largest logit is zero (what 64 bits hold of a sum's logarithm beside logits of 1e38
    is nothing), and what the rounding of a difference of 177 at most adds to its exponential."""
    dtype, z = x["logits"].dtype, x["logits"].double()
    z = z - z.amax(1, keepdim=True)
    want, tol = R.policy_loss(z, x["targets"], x["old"], x["adv"], x["weights"], x["ref"] if kl else None, 1 - CLIP[0], 1 + CLIP[1], kl)
    add = 177 * R.F32 + 2.0 ** -20
    tol = tol[0] + add * want[0].abs(), tol[1], tol[2] + (add + R.half_step(dtype)) * want[2].abs()
    for a, b, c in zip(got, want, tol):
        R.within(a, b, c)
    return want


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,v", SIZES)
@pytest.mark.parametrize("how", ["kl", "hidden target", "advantage", "-advantage", "weight"])
def test_an_infinite_gradient_is_no_zero(layer, dtype, t, v, how):
    """In its own row alone."""
    x = inputs(t, v, dtype)
    first = layer.policy_loss(**x, clip=CLIP, kl=0.05)
    if how == "kl":
        unlikely(x, 1, 150)
        x["ref"][1], x["old"][1] = 0.0, logp(x, 1)
    elif how == "hidden target":
        x["logits"][1, x["targets"][1]] = float("-inf")
    elif how == "weight":
        unlikely(x, 1, 60)
        x["ref"][1], x["old"][1], x["weights"][1] = 0.0, logp(x, 1), 1e30
    else:
        x["adv"][1] = float("inf" if how == "advantage" else "-inf")
    sums, lp, dz = layer.policy_loss(**x, clip=CLIP, kl=0.05)
    assert not sums[0].isfinite() and not dz[1, x["targets"][1]].isfinite() and not dz[1].isfinite().all()
    keep = [i for i in range(t) if i != 1]
    assert torch.equal(dz[keep], first[2][keep]) and torch.equal(lp[keep], first[1][keep])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,v", SIZES)
def test_an_advantage_of_zero_has_no_part(layer, dtype, t, v):
    """However far the policy has moved: a group of equal rewards."""
    x = inputs(t, v, dtype)
    x["adv"][1] = 0.0
    for old in (-95.0, -3e3, -1e30):
        x["old"][1] = old
        sums, lp, dz = layer.policy_loss(**x, clip=CLIP)
        y = {k: a.clone() for k, a in x.items()}
        y["old"][1] = logp(x, 1)
        want = layer.policy_loss(**y, clip=CLIP)
        assert torch.equal(sums, want[0]) and torch.equal(lp, want[1]) and torch.equal(dz, want[2]) and (dz[1] == 0).all()
    x["old"][1] = float("nan")
    assert layer.policy_loss(**x, clip=CLIP)[0][0].isnan()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,v", SIZES)
def test_an_exponential_beyond_the_range_with_a_product_inside(layer, dtype, t, v):
    """exp(ref - lp) or the ratio alone is infinite in fp32, the gradient is not."""
    x = inputs(t, v, dtype)
    unlikely(x, 1, 95)
    x["weights"][1], x["ref"][1] = 2.0 ** -13, -0.5
    x["old"][1] = logp(x, 1)
    want = within(x, 0.05, layer.policy_loss(**x, clip=CLIP, kl=0.05))
    assert 1e35 < want[2][1].abs().max() < 1e37
    x = inputs(t, v, dtype)
    x["old"][0], x["adv"][0], x["weights"][0] = logp(x, 0) - 95, -1.0, 2.0 ** -13
    want = within(x, 0.05, layer.policy_loss(**x, clip=CLIP, kl=0.05))
    assert 1e35 < want[2][0].abs().max() < 1e38
    x["adv"][0] = 1.0                                           # clipped: the ratio itself does not matter
    within(x, 0.0, layer.policy_loss(**x, clip=CLIP))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,v", SIZES + [(3, 7), (1, 1)])
def test_logits_hidden_by_the_lowest_value(layer, dtype, t, v):
    """They have no probability beside others, and are equal among themselves."""
    low = torch.finfo(dtype).min
    x = inputs(t, v, dtype)
    hidden = torch.rand(t, v, device="cuda") < 0.5
    hidden[:, :v // 3] = True                               # whole parts of a row among them
    hidden.scatter_(1, x["targets"][:, None], False)
    y = {k: a.clone() for k, a in x.items()}
    x["logits"].masked_fill_(hidden, low)
    y["logits"].masked_fill_(hidden, float("-inf"))
    got, want = layer.policy_loss(**x, clip=CLIP, kl=0.05), layer.policy_loss(**y, clip=CLIP, kl=0.05)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and got[2].isfinite().all()
    x["logits"][0] = low                                    # nothing is left of the row
    x["old"] = torch.stack([logp(x, i) for i in range(t)]).float()
    x["ref"] = x["old"] + 0.1
    within(x, 0.05, layer.policy_loss(**x, clip=CLIP, kl=0.05))


@pytest.mark.parametrize("dtype", TYPES)
def test_logits_of_any_size(layer, dtype):
    """Differences count, however large the logits themselves are."""
    big = torch.finfo(dtype).max
    for at in (1e3, -1e3, 1e30, -1e30, 2.5e38, -2.5e38, big):
        x = inputs(6, 2003, dtype)
        x["logits"][2] = at
        x["logits"][4] = at
        x["logits"][4, 77] = x["logits"][4, 77] * (1 - 2.0 ** -7)
        x["targets"][4] = 77 if at < 0 else 78
        x["old"] = torch.stack([logp(x, i) for i in range(6)]).float()
        x["ref"] = x["old"] + 0.1
        within(x, 0.05, layer.policy_loss(**x, clip=CLIP, kl=0.05))

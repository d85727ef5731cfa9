"""Registered tensors whose storage is replaced after they were added: a step writes
where the tensor is now, and a tensor that no longer fits is refused.  The replaced storage
is held by the tests, so that every address in play stays valid."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

N = 1000


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_15037_gb300 as pkg
    return pkg


def tensors(state):
    gen = torch.Generator(device="cuda").manual_seed(1)
    p = torch.nn.Parameter(torch.randn(N, generator=gen, device="cuda"))
    s = {"copy": p.detach().bfloat16()}
    if state == "f32":
        s.update(exp_avg=torch.zeros(N, device="cuda"), exp_avg_sq=torch.zeros(N, device="cuda"))
    else:
        s.update({k: torch.zeros(N, dtype=torch.uint8, device="cuda") for k in ("exp_avg", "exp_avg_sq")})
        s.update({k: torch.zeros(4, device="cuda") for k in ("exp_avg_scale", "exp_avg_sq_scale")})
    return p, s, torch.randn(N, generator=gen, device="cuda")


@pytest.mark.parametrize("state", ["f32", "block8"])
@pytest.mark.parametrize("ids", [None, [1]])
def test_replaced_storage_is_followed(M, state, ids):
    results = []
    for replaced in (False, True):
        p, s, g = tensors(state)
        opt = M.AdamWGroup(seed=3)
        opt.add(torch.zeros(5, device="cuda")), opt.add(p, state=state, **s)
        grads = [g] if ids else [torch.zeros(5, device="cuda"), g]
        opt.step(grads, 1, 1e-2, ids=ids)
        if replaced:
            both = [p, s["copy"]]
            old = [x.data for x in both]
            before = [x.clone() for x in old]
            for x in both:
                x.data = x.data.clone()
        opt.step(grads, 2, 1e-2, ids=ids)
        m, v = opt.moments(ids=[1])
        if replaced:
            assert all(torch.equal(x, y) for x, y in zip(old, before))
        results.append([p.detach(), *s.values(), m[0], v[0]])
        opt.close()
    for x, y in zip(*results):
        assert torch.equal(x, y)


@pytest.mark.parametrize("state", ["f32", "block8"])
def test_the_moments_memory_is_the_groups(M, state):
    """Whatever happens to the tensors that it was given with."""
    results = []
    for replaced in (False, True):
        p, s, g = tensors(state)
        opt = M.AdamWGroup(seed=3)
        opt.add(p, state=state, **s)
        opt.step([g], 1, 1e-2)
        if replaced:
            others = [x for k, x in s.items() if k != "copy"]
            for x in others:
                x.data = torch.ones_like(x)
        opt.step([g], 2, 1e-2)
        if replaced:
            assert all((x == 1).all() for x in others)
            sd = opt.state_dict()
            opt.step([g], 3, 1e-2)
            opt.load_state_dict(sd)
            assert all((x == 1).all() for x in others)
        results.append([p.detach().clone(), *opt.state_dict()[0].values(), *(x[0] for x in opt.moments())])
        if replaced:
            results[1][0] = q
        q = results[-1][0]
        with pytest.raises(TypeError):
            opt.states[0]["exp_avg"] = s["exp_avg"]
        opt.close()
    for x, y in zip(*results):
        assert torch.equal(x, y)


def test_another_type_is_followed(M):
    p, _, g = tensors("f32")
    q = p.detach().bfloat16()
    opt = M.AdamWGroup()
    opt.add(p), opt.add(q)
    old = p.data
    before = old.clone()
    p.data = p.data.bfloat16()
    opt.step([g, g], 1, 1e-2)
    assert torch.equal(p.detach(), q) and torch.equal(old, before)
    opt.close()


def test_what_no_longer_fits_is_refused(M):
    p, s, g = tensors("block8")
    opt = M.AdamWGroup()
    opt.add(p, state="block8", **s)
    launches = M.moara_launch_count(opt.ctx)
    for x, bad in ((p, torch.zeros(N + 1, device="cuda")), (p, torch.zeros(N)), (p, torch.zeros(2 * N, device="cuda")[::2]),
                   (s["copy"], torch.zeros(N, device="cuda")), (s["copy"], p.data)):
        old = x.data
        x.data = bad
        with pytest.raises(ValueError):
            opt.step([g], 1, 1e-2)
        x.data = old
    # a copy beside a bf16 parameter
    old, p.data = p.data, p.data.bfloat16()
    with pytest.raises(M.MoaraError):
        opt.step([g], 1, 1e-2)
    p.data = old
    assert M.moara_launch_count(opt.ctx) == launches
    opt.step([g], 1, 1e-2)
    opt.close()


def test_memory_freed_in_place(M):
    """As wrappers do that shard parameters or move states to the host: refused while it is gone,
    followed when it is back."""
    for name in ("param", "exp_avg", "exp_avg_sq_scale"):
        p, s, g = tensors("block8")
        q, r, _ = tensors("block8")
        opt, ref = M.AdamWGroup(), M.AdamWGroup()
        opt.add(p, state="block8", **s), ref.add(q, state="block8", **r)
        x = p.detach() if name == "param" else s[name]
        kept, launches = x.clone(), M.moara_launch_count(opt.ctx)
        x.untyped_storage().resize_(0)
        with pytest.raises(ValueError):
            opt.step([g], 1, 1e-2)
        if name != "param":                                  # which the moments' values do not need
            with pytest.raises(ValueError):
                opt.moments()
        assert M.moara_launch_count(opt.ctx) == launches
        taken = torch.full((1 << 16,), 7.0, device="cuda")
        x.untyped_storage().resize_(kept.nbytes)
        x.copy_(kept)
        opt.step([g], 1, 1e-2), ref.step([g], 1, 1e-2)
        assert torch.equal(p, q) and all(torch.equal(a, b) for a, b in zip(s.values(), r.values()))
        assert (taken == 7).all()
        opt.close(), ref.close()

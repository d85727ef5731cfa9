"""Bounded waits of the policy loss that run out, in rows of one CTA and of clusters: the shortest bound
surely where a CTA's part of a row is 64 KB and more (a few KB may be there before they are waited for).  The host reads the status, and the next call with the default bound is as the first one."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("t,vocab,dtype,surely", [(600, 32000, torch.bfloat16, True), (200, 50001, torch.float32, True),
                                                  (2, 32000, torch.bfloat16, False), (3, 300001, torch.float32, True),
                                                  (400, 1003, torch.float32, False)])
def test_loss_gives_up_and_recovers(t, vocab, dtype, surely):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_15037_gb300 as M
    g = M.LayerGroup()
    gen = torch.Generator(device="cuda").manual_seed(t)
    z = torch.randn(t, vocab, generator=gen, device="cuda").to(dtype)
    targets = torch.randint(0, vocab, (t,), generator=gen, device="cuda")
    old, adv = torch.full((t,), -11.0, device="cuda"), torch.randn(t, generator=gen, device="cuda")
    want = g.policy_loss(z, targets, old, adv)
    torch.cuda.synchronize()
    assert g.status() == 0
    seen = []
    for limit in (1, 1, 100, 500, 2000, 8000, 100000):
        M.moara_set_wait_limit(g.ctx, limit)
        out = torch.full((t + 2, vocab), 7.0, dtype=dtype, device="cuda")
        got = g.policy_loss(z, targets, old, adv, out=out[1:-1])
        torch.cuda.synchronize()
        seen.append(g.status())
        assert (out[0] == 7).all() and (out[-1] == 7).all()
        if seen[-1] == 0:
            assert all(torch.equal(x, y) for x, y in zip(got, want))
        M.moara_set_wait_limit(g.ctx, 0)
        got = g.policy_loss(z, targets, old, adv)
        torch.cuda.synchronize()
        assert g.status() == 0 and all(torch.equal(x, y) for x, y in zip(got, want))
    g.close()
    assert set(seen) <= {0, M.MOARA_ERR_DEVICE_TIMEOUT}
    assert not surely or seen[:2] == [M.MOARA_ERR_DEVICE_TIMEOUT] * 2, seen

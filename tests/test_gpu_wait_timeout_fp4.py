"""Bounded waits that run out in the MXFP4 products, at limits from far below a copy's
latency (every wait gives up) to above a whole product's: a kernel gives up anywhere in
between.  Each time the host reads the status, no copy is left in flight, an entry of the
output is right or untouched, what is not the output stays, and the next product with the default
bound is the one before."""

import time

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

LIMITS = [100, 100, 500, 1000, 2000, 4000, 8000, 16000, 100000]
PAIRS = [(300, 9732, 520), (1300, 2501, 4096), (4000, 3000, 250), (2100, 2560, 8000), (1300, 5001, 16000), (512, 2560, 20000)]
LONG = 8000         # K from which some wait outlasts the time that the hardware suspends a try by itself


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_15037_gb300 as pkg
    return pkg


def interrupted(M, call, want, m, n, dtype, surely):
    """call(group, out) under every limit: the results, statuses, and the surroundings of D.
    surely: the shortest limits have to run out."""
    f = M.Fp4Group()
    seen = []
    for limit in LIMITS:
        buf = torch.full((m + 2, n + 8), 7.0, dtype=dtype, device="cuda")
        M.moara_set_wait_limit(f.ctx, limit)
        call(f, buf[1:-1, :n])
        torch.cuda.synchronize()
        seen.append(f.status())
        D = buf[1:-1, :n]
        assert ((D == want) | (D == 7)).all()
        M.moara_set_wait_limit(f.ctx, 0)
        assert (buf[0] == 7).all() and (buf[-1] == 7).all() and (buf[:, n:] == 7).all()
        if seen[-1] == 0:
            assert torch.equal(buf[1:-1, :n], want)
        call(f, buf[1:-1, :n])
        torch.cuda.synchronize()
        assert f.status() == 0 and torch.equal(buf[1:-1, :n], want)
    f.close()
    assert set(seen) <= {0, M.MOARA_ERR_DEVICE_TIMEOUT}
    assert not surely or seen[:2] == [M.MOARA_ERR_DEVICE_TIMEOUT] * 2, seen


@pytest.mark.parametrize("shape", PAIRS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_pairs_give_up_and_recover(M, shape, dtype):
    m, n, k = shape
    f = M.Fp4Group()
    gen = torch.Generator(device="cuda").manual_seed(m)
    a, b = (f.quantize(torch.randn(x, k, generator=gen, device="cuda")) for x in (m, n))
    want = f.product(a, b, dtype=dtype)
    interrupted(M, lambda g, out: g.product(a, b, out=out), want, m, n, dtype, k >= LONG)
    f.close()


# tokens, N, K; few tiles, so that clusters share K, and several tiles; up to 8 tokens are
# quantised inside the kernel by linear
FEW = [(1, 4096, 4096), (5, 300, 160000), (8, 2600, 40000), (12, 300, 160000), (40, 1003, 80000), (128, 300, 160000),
       (200, 129, 160000), (77, 1003, 2049)]


@pytest.mark.parametrize("shape", FEW)
@pytest.mark.parametrize("form", ["product", "linear"])
def test_few_tokens_give_up_and_recover(M, shape, form):
    m, n, k = shape
    f = M.Fp4Group()
    gen = torch.Generator(device="cuda").manual_seed(n)
    x, w = (torch.randn(r, k, generator=gen, device="cuda") for r in (m, n))
    a, b = f.quantize(x), f.quantize(w)
    want = f.product(a, b)
    torch.cuda.synchronize()
    begin = time.time()
    interrupted(M, lambda g, out: g.product(a, b, out=out) if form == "product" else g.linear(x, b, out=out),
                want, m, n, torch.bfloat16, k >= 80000)
    # no wait for a phase that never ends: those take the default bound, 2 s each
    assert time.time() - begin < 2
    f.close()

"""Operands that another stream reads when they are released."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("handle", [False, True])
def test_recorded_operands_outlive_their_release(given, handle):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_15037_gb300 as M
    f = M.Fp4Group()
    m = n = 640
    k = 2048
    x, w = torch.randn(m, k, device="cuda"), torch.randn(n, k, device="cuda")
    W = f.quantize(w)
    want = f.product(f.quantize(x), W)
    a = f.quantize(x)
    if given:
        a = M.Fp4Matrix(m, k, a.q.clone(), a.sf.clone())
    place = a.q.data_ptr()
    out = torch.zeros_like(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)                       # some 50 ms
    f.product(a, W, out=out, stream=side.cuda_stream)
    a.record_stream(side.cuda_stream if handle else side)
    del a
    # what is allocated now lies elsewhere, while the product still waits for its turn
    others = [f.quantize(torch.randn(m, k, device="cuda")) for _ in range(4)]
    assert not side.query() and all(b.q.data_ptr() != place for b in others)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and f.status() == 0
    f.close()

"""Gradients of the attention again and again: the warps of a CTA hand steps over by barriers, whose
order may differ from call to call where the results may not."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("lengths,h,hk,d", [([300, 1, 129, 256, 700, 128, 257, 64] * 4, 16, 4, 64), ([2000, 300], 8, 8, 64),
                                            ([129] * 60, 8, 1, 40), ([1500, 256], 8, 4, 128)])
def test_gradients_repeat(lengths, h, hk, d):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_15037_gb300 as M
    layer, t = M.LayerGroup(), sum(lengths)
    g = torch.Generator(device="cuda").manual_seed(t + d)
    q, k, v, do = (torch.randn(t, n, d, generator=g, device="cuda").to(torch.bfloat16) for n in (h, hk, hk, h))
    seqs = layer.sequences(lengths)
    out, lse, rest = layer.attention(q, k, v, seqs, train=True)
    want = layer.attention_backward(do, q, k, v, out, lse, seqs, rest=rest)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    differ = [torch.zeros((), dtype=torch.int64, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    for i in range(300):
        with torch.cuda.stream(streams[i & 1]):
            got = layer.attention_backward(do, q, k, v, out, lse, seqs, rest=rest)
            for x, y in zip(got, want):
                differ[i & 1] += (x.view(torch.int16) != y.view(torch.int16)).sum()
    torch.cuda.synchronize()
    assert layer.status() == 0 and not any(x.item() for x in differ)
    layer.close()

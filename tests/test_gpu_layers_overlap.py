"""Outputs that lie over inputs: the input itself, or columns beside it, are taken; all else is refused."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


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


ROWS, COLS = 40, 96


def views(dtype):
    """(x, a tensor over or beside it, whether it is taken)."""
    def buf(r=ROWS + 8, c=3 * COLS):
        return torch.randn(r, c, device="cuda").to(dtype)
    b = buf()
    x = b[:ROWS, :COLS]
    yield x, x, True
    yield x, b[:ROWS, :COLS], True
    yield x, b[:ROWS, COLS:2 * COLS], True                  # beside it
    yield x, b[:ROWS, 2 * COLS:], True
    yield b[:ROWS, COLS:2 * COLS], b[3:ROWS + 3, :COLS], True
    yield x, b[1:ROWS + 1, :COLS], False                    # rows further on
    yield x, b[:ROWS, 8:COLS + 8], False                    # columns further on
    yield b[:ROWS, COLS:2 * COLS], b[2:ROWS + 2, COLS - 1:2 * COLS - 1], False
    flat = b.view(-1)
    yield flat[:ROWS * COLS].view(ROWS, COLS), flat[ROWS * COLS:2 * ROWS * COLS].view(ROWS, COLS), True
    yield flat[:ROWS * COLS].view(ROWS, COLS), flat[COLS // 2:ROWS * COLS + COLS // 2].view(ROWS, COLS), False
    yield x, flat[:ROWS * COLS].view(ROWS, COLS), False     # the same place, another pitch
    yield x[:1], flat[:COLS].view(1, COLS), True            # but of a single row
    yield x[:1], flat[8:COLS + 8].view(1, COLS), False


def both(M, call, taken):
    if taken:
        call()
    else:
        with pytest.raises((M.MoaraError, ValueError)) as e:
            call()
        if isinstance(e.value, M.MoaraError):
            assert e.value.code == M.MOARA_ERR_INVALID_ARG or "pitch" in str(e.value)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_overlaps(M, layer, dtype):
    for x, y, taken in views(dtype):
        first = x.clone()
        gain, other = torch.ones(COLS, device="cuda"), torch.randn(len(x), COLS, device="cuda").to(dtype)
        targets = torch.zeros(len(x), dtype=torch.int64, device="cuda")
        old = torch.zeros(len(x), device="cuda")
        h, z, s = layer.norm(first, gain, residual=other, dtype=dtype)
        dx, dg = layer.norm_backward(other, first, gain, s, dh=other)
        dz = layer.policy_loss(first, targets, old, old + 1)[2]
        for call, want in ((lambda: layer.norm(x, gain, residual=other, h=y)[0], h),
                           (lambda: layer.norm(other, gain, residual=x, h=y)[0], h),
                           (lambda: layer.norm(x, gain, residual=other, out=y)[1], z),
                           (lambda: layer.norm(other, gain, residual=x, out=y)[1], z),
                           (lambda: layer.norm_backward(other, x, gain, s, dh=other, out=y)[0], dx),
                           (lambda: layer.policy_loss(x, targets, old, old + 1, out=y)[2], dz)):
            x.copy_(first)
            both(M, lambda: torch.testing.assert_close(call(), want, rtol=0, atol=0, equal_nan=True), taken)
        x.copy_(first)
        both(M, lambda: layer.norm_quantize(x, gain, residual=other, h=y), taken)


def test_outputs_of_another_type_over_the_input(M, layer):
    """fp32 over bf16, at the same place, is neither."""
    b = torch.randn(ROWS, COLS, device="cuda")
    x = b.view(torch.bfloat16)[:, :COLS]
    gain = torch.ones(COLS, device="cuda")
    with pytest.raises(M.MoaraError):
        layer.norm(x, gain, out=b)
    # in the other half of the rows it lies apart
    b = torch.randn(ROWS, 2 * COLS, device="cuda")
    x = b.view(torch.bfloat16)[:, :COLS]
    x.copy_(torch.randn(ROWS, COLS, device="cuda"))
    want = layer.norm(x.clone(), gain, dtype=torch.float32)[1]
    assert torch.equal(layer.norm(x, gain, out=b[:, COLS:])[1], want)

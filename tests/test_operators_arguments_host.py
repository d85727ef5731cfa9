"""CPU tests of what the Python side of the operators refuses before it reaches the
library: groups without a context, on tensors of the host, whose device is -1."""

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def M():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2609_15037_gb300 as pkg
    return pkg


def operand(M, rows, cols, device=-1):
    q, sf = M.moara_fp4_bytes(rows, cols)
    return M.Fp4Matrix(rows, cols, torch.zeros(q, dtype=torch.uint8), torch.zeros(sf, dtype=torch.uint8), device)


def fp4_group(M, device):
    f = M.Fp4Group.__new__(M.Fp4Group)
    f.device, f.ctx = device, None
    return f


@pytest.mark.parametrize("device", [0, 1])
def test_operands_of_another_device_are_refused(M, device, monkeypatch):
    f, a = fp4_group(M, device), operand(M, 4, 64)

    def reached(*_):
        raise AssertionError("the library was called")
    for name in ("fp4_product", "fp4_linear", "fp4_dequantize"):
        monkeypatch.setattr(M.fp4._host, name, reached)
    monkeypatch.setattr(M.fp4._host, "matrix", lambda x, device: (x.data_ptr(), 0, 4, 64, 64))
    monkeypatch.setattr(M.fp4.B, "moara_fp4_quantize", reached)
    x = torch.zeros(4, 64)
    for call in (lambda: f.product(a, a), lambda: f.linear(x, a), lambda: f.dequantize(a),
                 lambda: f.quantize(x, out=a), lambda: f.quantize(x, rows=False, cols=True, out_cols=operand(M, 64, 4)),
                 lambda: f.product(a, a, stream=1), lambda: f.quantize(x, out=a, stream=1)):
        with pytest.raises(ValueError):
            call()

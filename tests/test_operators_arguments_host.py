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


def adamw_group(M):
    opt = M.AdamWGroup.__new__(M.AdamWGroup)
    create, destroy = M.adamw.B.moara_create, M.adamw.B.moara_destroy
    M.adamw.B.moara_create, M.adamw.B.moara_destroy = lambda *_: None, lambda *_: None
    try:
        opt.__init__(device=0)
    finally:
        M.adamw.B.moara_create, M.adamw.B.moara_destroy = create, destroy
    opt.device, opt._dev = -1, torch.device("cpu")
    return opt


def test_overlapping_registrations_are_refused(M):
    opt = adamw_group(M)
    flat = torch.zeros(1000)
    p = flat[100:300]
    half = torch.zeros(200, dtype=torch.bfloat16)
    m, v = torch.zeros(200), torch.zeros(200)
    assert opt.add(p, copy=half, exp_avg=m, exp_avg_sq=v) == 0
    other = torch.zeros(200)
    for bad, kw in ((p, {}), (flat[299:400], {}), (flat[:101], {}), (flat, {}), (flat[150:160], {}), (m, {}),
                    (other, dict(copy=half)), (other, dict(exp_avg=v)), (other, dict(exp_avg_sq=other)),
                    (other, dict(exp_avg=torch.zeros(200), exp_avg_sq=p))):
        with pytest.raises(ValueError):
            opt.add(bad, **kw)
    # refused ones left nothing behind; neighbours and empty tensors are fine
    assert opt.add(other) == 1 and opt.add(flat[:100]) == 2 and opt.add(flat[300:]) == 3
    assert opt.add(flat[:0]) == 4 and opt.add(flat[150:150]) == 5
    assert len(opt.states) == len(opt.params) == 6


def test_eight_bit_scales_are_ranges_too(M):
    opt = adamw_group(M)
    scales = torch.zeros(4)
    kw = dict(state="block8", exp_avg_scale=scales[:2], exp_avg_sq_scale=scales[2:])
    opt.add(torch.zeros(300), **kw)
    with pytest.raises(ValueError):
        opt.add(torch.zeros(300), **kw)


def test_a_tensor_is_taken_once_per_call(M, monkeypatch):
    opt = adamw_group(M)
    for _ in range(3):
        opt.add(torch.zeros(8))
    calls = []
    monkeypatch.setattr(M.adamw._host, "adamw_step", lambda *a: calls.append(a[2]) or 0)
    g = torch.zeros(8)
    for ids in ([0, 0], [2, 1, 2], [0, -3]):
        with pytest.raises(ValueError):
            opt.step([g] * len(ids), 1, 0.1, ids=ids, stream=0)
    with pytest.raises(IndexError):
        opt.step([g], 1, 0.1, ids=[3], stream=0)
    opt.step([g, g], 1, 0.1, ids=iter((2, 0)), stream=0)
    opt.step([], 1, 0.1, ids=[], stream=0)
    assert calls == [2, 0]


def test_replaced_storage_may_not_overlap(M):
    opt = adamw_group(M)
    a, b = torch.zeros(100), torch.zeros(100)
    opt.add(a), opt.add(b)
    old = b.data
    b.data = a.data
    with pytest.raises(ValueError):
        opt._follow()
    b.data = old
    a.data = torch.zeros(100)
    opt._follow()
    assert opt._table["param"][:2].tolist() == [a.data_ptr(), b.data_ptr()]


def test_memory_of_a_replaced_storage_is_free_again(M):
    opt = adamw_group(M)
    a = torch.zeros(100)
    opt.add(a)
    old = a.data
    a.data = torch.zeros(100)
    assert opt.add(old) == 1
    with pytest.raises(ValueError):
        opt.add(a.data)


def test_an_operand_keeps_the_memory_it_was_made_of(M):
    nq, nsf = M.moara_fp4_bytes(4, 64)
    q, sf = torch.ones(nq, dtype=torch.uint8), torch.ones(nsf, dtype=torch.uint8)
    a = M.Fp4Matrix(4, 64, q, sf, device=-1)
    places = q.data_ptr(), sf.data_ptr()
    q.data, sf.data = torch.zeros(nq, dtype=torch.uint8), torch.zeros(nsf, dtype=torch.uint8)
    assert (a.q.data_ptr(), a.sf.data_ptr()) == places == a._ptrs
    assert a.q.all() and a.sf.all()


@pytest.mark.parametrize("big", [2 ** 31, 2 ** 32 + 1, -2 ** 32 + 1])
def test_sizes_beyond_32_bits_are_refused(M, big):
    """Not taken by their lower half."""
    for call in (lambda: M.moara_fp4_bytes(big, 32), lambda: M.moara_fp4_bytes(32, big), lambda: M.Fp4Matrix(big, 32),
                 lambda: M.moara_fp4_linear_workspace_bytes(big, 32, 32), lambda: M.moara_fp4_linear_workspace_bytes(16, 32, big),
                 lambda: M.moara_fp4_quantize(None, 0, 0, big, 1, 1), lambda: M.moara_fp4_dequantize(None, 0, 0, 1, big, 0, 0, big),
                 lambda: M.moara_fp4_product(None, 1, big, 1, 0, 0, 0, 0, 0, 0, big),
                 lambda: M.moara_fp4_linear(None, 1, 1, big, 0, 0, big, 0, 0, 0, 0, 1)):
        with pytest.raises(ValueError):
            call()


def test_moments_into_iterables(M, monkeypatch):
    """Outputs that are no lists come back as lists, not as what was read to its end."""
    opt = adamw_group(M)
    opt.add(torch.zeros(8)), opt.add(torch.zeros(3))
    monkeypatch.setattr(M.adamw._host, "adamw_moments", lambda *a: 0)
    m, v = ([torch.zeros(8), torch.zeros(3)] for _ in range(2))
    got = opt.moments(iter(m), (x for x in v), stream=0)
    assert all(x is y for a, b in zip(got, (m, v)) for x, y in zip(a, b)) and [len(list(x)) for x in got] == [2, 2]
    assert opt.moments(m, v, stream=0)[0] is m

"""The C entries of the operators as their bindings pass them: outputs that are left out, values
into a pitch of the caller's."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2609_15037_gb300 as pkg
    return pkg


@pytest.mark.parametrize("state", ["f32", "block8"])
def test_moments_leave_out_what_is_null(M, state):
    sizes = [5, 0, 700]
    opt = M.AdamWGroup(seed=4)
    for n in sizes:
        opt.add(torch.zeros(n, device="cuda"), state=state)
    opt.step([torch.randn(n, device="cuda") for n in sizes], 1, 1e-2)
    want = opt.moments()
    d = opt._chosen(None)[0]
    for wanted in ((True, False), (False, True), (False, False), (True, True)):
        for first in (True, False):              # of the last tensor, or of all
            out = [[torch.full((n,), 7.0, device="cuda") for n in sizes] for _ in range(2)]
            at = [np.array([x.data_ptr() if w or (first and i < 2) else 0 for i, x in enumerate(xs)], dtype=np.uint64)
                  for w, xs in zip(wanted, out)]
            M.moara_adamw_moments(opt.ctx, 3, d.ctypes.data, at[0].ctypes.data, at[1].ctypes.data)
            torch.cuda.synchronize()
            for k, w in enumerate(wanted):
                for i, x in enumerate(out[k]):
                    assert torch.equal(x, want[k][i]) if w or (first and i < 2) else bool((x == 7).all())
    opt.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_values_into_a_pitch(M, dtype):
    f = M.Fp4Group()
    a = f.quantize(torch.randn(33, 70, device="cuda"))
    out = torch.full((33, 80), 7.0, dtype=dtype, device="cuda")
    M.moara_fp4_dequantize(f.ctx, a.q.data_ptr(), a.sf.data_ptr(), 33, 70, out.data_ptr(), 1 if dtype == torch.bfloat16 else 0, 80)
    torch.cuda.synchronize()
    assert torch.equal(out[:, :70], f.dequantize(a, dtype=dtype)) and (out[:, 70:] == 7).all() and f.status() == 0
    f.close()

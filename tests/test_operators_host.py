"""CPU tests of the operators beside the projected step: the float64
definitions against hand-computed cells, and the host side of the C entries."""

import ctypes

import numpy as np
import pytest

from oracle import operators_ref as o


@pytest.fixture(scope="module")
def M():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2609_15037_gb300 as pkg
    return pkg


def test_structs_match_header(M):
    assert ctypes.sizeof(M.binding.moara_adamw_hparams) == 24
    assert ctypes.sizeof(M.binding.moara_adamw_tensor) == 88
    assert M.binding.moara_adamw_tensor.lr_scale.offset == 84


@pytest.mark.parametrize("rows,cols,q,sf", [(1, 1, 16, 512), (128, 128, 8192, 512), (129, 33, 129 * 32, 1024),
                                            (1, 4097, 129 * 16, 33 * 512), (70000, 70000, 70000 * 2188 * 16, 547 * 547 * 512)])
def test_fp4_bytes(M, rows, cols, q, sf):
    assert M.moara_fp4_bytes(rows, cols) == (q, sf)


def test_host_sizes_refuse(M):
    for call in (lambda: M.moara_fp4_bytes(0, 1), lambda: M.moara_fp4_linear_workspace_bytes(1, 0, 1),
                 lambda: M.moara_fp4_linear_workspace_bytes(1, 1, -1)):
        with pytest.raises(M.MoaraError) as ei:
            call()
        assert ei.value.code == M.MOARA_ERR_SHAPE
    with pytest.raises(M.MoaraError) as ei:
        M.moara_grad_norm_workspace_bytes(-1)
    assert ei.value.code == M.MOARA_ERR_INVALID_ARG
    assert M.moara_grad_norm_workspace_bytes(0) == M.moara_grad_norm_workspace_bytes(1) > 16


def test_null_context_is_refused(M):
    lib = M.binding.lib
    assert lib.moara_adamw_step(None, 0, None, None, 1, 0.0, None, None) == M.MOARA_ERR_INVALID_ARG
    assert lib.moara_adamw_moments(None, 0, None, None, None, None) == M.MOARA_ERR_INVALID_ARG
    assert lib.moara_grad_norm(None, 0, None, None, None, 0.0, None, None, None, 0, None) == M.MOARA_ERR_INVALID_ARG
    assert lib.moara_fp4_quantize(None, None, 0, 1, 1, 1, None, None, None, None, None) == M.MOARA_ERR_INVALID_ARG
    assert lib.moara_fp4_product(None, 1, 1, 1, None, None, None, None, None, 0, 1, None) == M.MOARA_ERR_INVALID_ARG


def test_e2m1_rounding_by_hand():
    # one block, scale 1 (largest 6): ties go to the even code, signs are kept
    x = np.zeros((1, 32))
    x[0, :13] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.01, -0.26, -0.2, 0.74, -4.9]
    code, scale = o.quantize(x)
    assert scale.tolist() == [[127]]
    assert code[0, :13].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 7, 9, 8, 1, 14]


@pytest.mark.parametrize("top,byte", [(6.0, 127), (np.nextafter(6.0, 7.0), 128), (3.0, 126), (4.0, 127), (0.0, 0),
                                      (2.0 ** -149, 0), (6 * 2.0 ** -127, 0), (6.1 * 2.0 ** -127, 1),
                                      (float(np.finfo(np.float32).max), 253), (np.inf, 255), (np.nan, 255)])
def test_scale_rule_by_hand(top, byte):
    x = np.zeros((1, 40))
    x[0, 35] = top
    code, scale = o.quantize(x)
    assert scale.tolist() == [[0, byte]]


def test_code_axis_and_values_agree():
    """Position c of the value of code c, for every code of both kinds."""
    for signed, count in ((True, 128), (False, 256)):
        codes = np.arange(count)
        scales = np.full(-(-count // o.BLOCK), 1.0)
        v = o.decode8(codes, scales, signed)
        assert v.max() == 1.875 and np.all(np.diff(v) > 0)
        full = np.zeros(o.BLOCK)
        full[:count] = v
        pos, scale = o.code_position(full, signed)
        assert np.array_equal(pos[:count], codes) and scale[0] == 1.0


def test_adamw_definition_by_differences():
    """The first step from zero moments moves every entry by lr sign(g) (up to
    eps); without gradient only the decay remains."""
    g = np.array([0.5, -2.0, 1e-3, 0.0])
    p = np.array([1.0, 1.0, -1.0, 2.0])
    q, m, v = o.adamw(p, g, np.zeros(4), np.zeros(4), 1, 0.1, 0.9, 0.999, 1e-12, 0.5)
    assert np.allclose(q, p * 0.95 - 0.1 * np.sign(g), atol=1e-9)
    assert np.allclose(m, 0.1 * g) and np.allclose(v, 0.001 * g * g)


def test_random_bits_are_uniform_and_distinct():
    r = o.random_bits(1 << 16, 77, 3, 5)
    assert abs((r & 0xFFFF).mean() / 65535 - 0.5) < 0.01 and abs((r >> 16).mean() / 65535 - 0.5) < 0.01
    others = [o.random_bits(1 << 16, 78, 3, 5), o.random_bits(1 << 16, 77, 4, 5), o.random_bits(1 << 16, 77, 3, 6),
              o.random_bits(1 << 16, 77 + (1 << 32), 3, 5), o.random_bits(1 << 16, 77, 3, 5, first=1 << 32)]
    for x in others:
        assert (x == r).mean() < 1e-3 and abs(np.corrcoef(x.astype(float), r.astype(float))[0, 1]) < 0.02

"""Products of the workers' matrices: what is refused without a context, and the structs' layouts."""
import ctypes

import pytest

import paper_2505_22549_b200 as d
from paper_2505_22549_b200 import binding as B


def test_structs_are_the_headers():
    assert ctypes.sizeof(B.DeslocFfn) == 80 and B.DeslocFfn.weights.offset == 40 and B.DeslocFfn.h.offset == 48
    assert ctypes.sizeof(B.DeslocOrthogonal) == 64 and B.DeslocOrthogonal.updates.offset == 48 and B.DeslocOrthogonal.coefficients.offset == 24


def test_calls_refuse_none():
    L = d.raw_lib()
    rows = B.rows(64, d.DESLOC_BF16, 8, 8)
    f, how = B.ffn(0, 1, 2, 8, 8, 1, None, rows), B.orthogonal([0], [8])
    assert L.desloc_gated_ffn(None, f, None, None, rows, None, 0, None) == d.DESLOC_E_NULL
    assert L.desloc_gated_ffn_bytes(None, f) == d.DESLOC_E_NULL
    assert L.desloc_gated_ffn_grad(None, f, None, None, rows, rows, 0, None, None, 0, None) == d.DESLOC_E_NULL
    assert L.desloc_gated_ffn_grad_bytes(None, f, rows) == d.DESLOC_E_NULL
    assert L.desloc_orthogonalize(None, how, 0, None, None, 0, None) == d.DESLOC_E_NULL
    assert L.desloc_orthogonal_step(None, how, 0.1, None, 0, None) == d.DESLOC_E_NULL
    assert L.desloc_orthogonal_bytes(None, how) == d.DESLOC_E_NULL


def test_orthogonal_wants_a_width_per_tensor_and_three_coefficients_per_step():
    with pytest.raises(ValueError):
        B.orthogonal([0, 1], [8])
    with pytest.raises(ValueError):
        B.orthogonal([0], [8], steps=2, coefficients=[1.0] * 5)

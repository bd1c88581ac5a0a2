"""The workspace of layers' gradients: what a call does not write is not asked for."""
from __future__ import annotations

import ctypes

import pytest

import paper_2605_15073_amd as cg

F32, BF16, NONE, SILU = cg.CGTP_F32, cg.CGTP_BF16, cg.CGTP_ACT_NONE, cg.CGTP_ACT_SILU


def need(dtype, n, G, n_in, n_out, per_row, act):
    out = ctypes.c_size_t()
    status = cg.load_library().cgtp_grouped_layer_grad_bytes(dtype, n, G, n_in, n_out, per_row, act, ctypes.byref(out))
    assert status == cg.CGTP_OK
    return out.value


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,G,n_in,n_out", [(525308, 10, 64, 64), (525308, 55, 8, 60), (20000, 10, 64, 64), (300, 2, 4, 4)])
def test_narrow_layers_have_no_dz(dtype, n, G, n_in, n_out):
    """One pass forms dz and uses it: all that is kept are sums of chunks, 256 rows or more each."""
    got = need(dtype, n, G, n_in, n_out, 1, SILU)
    assert got == need(dtype, n, G, n_in, n_out, 1, NONE)
    assert got <= (2 * (n // 256) + 2) * (n_in + 1) * n_out * 4


def test_wide_layers_in_bf16_form_dz_in_the_products():
    """Up to 128 inputs: sums of chunks are all that is kept then."""
    dz = lambda n, n_out: n * n_out * 4
    assert need(BF16, 261764, 32, 128, 448, 1, SILU) < dz(261764, 448) / 4
    slots = (2 * (60000 // 256) + 2) * (1344 + 1) * 448 * 4      # of chunks of 256 rows, the shortest
    assert dz(60000, 448) <= need(BF16, 60000, 32, 1344, 448, 1, SILU) <= dz(60000, 448) + slots
    assert dz(60000, 448) <= need(F32, 60000, 32, 128, 448, 1, SILU) <= dz(60000, 448) + slots


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n_in", [64, 1344])
def test_rows_that_share_an_input_are_summed_in_fp32(dtype, n_in):
    assert need(dtype, 40000, 8, n_in, 128, 4, SILU) == need(dtype, 40000, 8, n_in, 128, 1, SILU) + 40000 * n_in * 4

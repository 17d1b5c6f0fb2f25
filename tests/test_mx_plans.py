"""CPU tests of which rows the microscaled product quantizes itself, seen in the workspace that
it asks for (none: nothing is quantized in a launch before it)."""

import pytest

from tests._util import ensure_built
from paper_2607_14107_amd import polestar as ps


@pytest.fixture(scope="module", autouse=True)
def built():
    ensure_built()


def _need(dtype, rows, n_in, n_out, fmt=ps.MXFP8):
    return ps.mx_quantize_linear_workspace_size(fmt, dtype, 1, rows, n_out, n_in)


@pytest.mark.parametrize("fmt", [ps.MXFP4, ps.MXFP8])
@pytest.mark.parametrize("dtype,most", [(ps.BF16, 16), (ps.FP32, 4)])
def test_few_rows_of_one_chunk_per_wave_on_one_round_of_workgroups(fmt, dtype, most):
    for n_in in (128, 2048, 4096):
        for n_out in (16, 1024, 4096):
            assert _need(dtype, 1, n_in, n_out, fmt) == _need(dtype, most, n_in, n_out, fmt) == 0
            assert _need(dtype, most + 1, n_in, n_out, fmt) > 0


@pytest.mark.parametrize("fmt", [ps.MXFP4, ps.MXFP8])
@pytest.mark.parametrize("dtype", [ps.BF16, ps.FP32])
@pytest.mark.parametrize("n_in,n_out", [(4224, 16), (8192, 2048), (65536, 256), (512, 4112), (1024, 8192), (256, 24576)])
def test_long_rows_and_many_outputs_are_quantized_before(fmt, dtype, n_in, n_out):
    """(Quantized by every workgroup, 8192 channels took a third longer than two launches and 65536 twice as long;
    on more than one workgroup per compute unit, 512 x 8192 two fifths longer.)"""
    for rows in (1, 2, 4):
        assert _need(dtype, rows, n_in, n_out, fmt) > 0

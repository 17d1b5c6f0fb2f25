"""CPU tests of the microscaled calls' plans, seen in the workspaces that they ask for."""

import pytest

from tests._util import ensure_built
from paper_2607_14107_amd import polestar as ps


@pytest.fixture(scope="module", autouse=True)
def built():
    ensure_built()


def _need(dtype, rows, n_in, n_out, fmt=ps.MXFP8):
    return ps.mx_quantize_linear_workspace_size(fmt, dtype, 1, rows, n_out, n_in)


# Rows that the product quantizes itself need no workspace.
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


BIG = 2 ** 31 - 1
# batch seq heads kv_heads head_dim rows: more than a launch holds, in each number and in products that pass 32 or 64 bits
REFUSED = [(1, 4096, 2 ** 18, 1, 128, 2 ** 19), (1, 4096, BIG, 1, 128, BIG), (65536, 64, 4, 4, 128, 1),
           (1, 64, 65536, 65536, 128, 1), (1, 2 ** 24 + 1, 4, 4, 128, 1), (65535, 64, 65535, 65535, 128, BIG),
           (BIG, BIG, BIG, BIG, 64, BIG), (1, 64, 1, 1, 64, 2 ** 28)]


@pytest.mark.parametrize("b,seq,heads,kvh,hd,rows", REFUSED)
def test_attention_sizes_of_refused_shapes(b, seq, heads, kvh, hd, rows):
    """A size query answers 0 for what the call refuses, however large the numbers."""
    assert ps.mx_attend_workspace_size(ps.BF16, b, seq, heads, kvh, hd, rows) == 0
    fake = 0x10000                                       # 16-byte aligned, never dereferenced
    assert ps.lib().polestar_mx_attend(ps.BF16, b, seq, heads, kvh, hd, rows, fake, heads * hd, fake, fake, fake, fake,
                                       None, 0.0, fake, None, None, 0, None) == 2


@pytest.mark.parametrize("kvh", [65536, 2 ** 25, 2 ** 31 - 1])
def test_store_refuses_more_heads_than_the_attention_takes(kvh):
    """2^26 heads of 128 are 2^31 groups of channels in a row's keys and values together."""
    fake = 0x10000
    assert ps.lib().polestar_mx_store_kv(ps.BF16, 1, 4, kvh, 128, 1, fake, fake, kvh * 128, None, None, 0, fake, fake,
                                         fake, fake, None) == 2

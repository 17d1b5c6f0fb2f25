"""GPU parity of the microscaled products where few rows meet long ones, where scales lie
far apart, and of the codes that the self-quantizing kernel makes; rows without channels
(oracle: oracle/mx_ref.py; bounds: tests/test_gpu_mx.py)."""

import numpy as np
import pytest

from oracle import mx_ref as mx
from tests._util import ensure_built, to_dev
from tests.test_gpu_mx import _bits, _dev, _guarded, _guards_hold, _held, _linear_bound, _vals

pytestmark = pytest.mark.gpu

BOTH = pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
DTYPES = pytest.mark.parametrize("dtype", ["bf16", "fp32"])


@pytest.fixture(scope="module")
def P():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    ensure_built()
    from paper_2607_14107_amd import polestar
    return polestar


def _type(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _check(y, want, tol):
    got = y.double().cpu().numpy().reshape(want.shape)
    err = np.abs(got - want)
    assert err.size and np.isfinite(want).all()
    assert (err <= tol).all(), (np.argwhere(~(err <= tol))[:4].tolist(), float(np.nanmax(err / tol)))


def _linear(P, g, fmt, dtype, rows, n_in, n_out, spread):
    import torch
    xc, xs, x = _held(g, (rows, n_in), fmt, spread)
    wc, ws, w = _held(g, (n_out, n_in), "mxfp4", spread)
    dt = _type(dtype)
    buf, raw = _guarded((rows * n_out * dt.itemsize,))
    y = raw.view(dt).view(rows, n_out)
    P.mx_linear(P.CODECS[fmt], _dev(xc), _dev(xs), _dev(wc), _dev(ws), y)
    want = x @ w.T
    _check(y, want, _linear_bound(x, w, want, fmt, dtype))
    _guards_hold(buf)
    assert torch.isfinite(y).all()


# More than 4096 channels: a wave of the few-rows kernel takes a second chunk of 512, whole or with 1 to 3 of
# its 4 steps past the end.
LONG = [(1, 4224, 144), (1, 12288, 528), (4, 8192, 80), (4, 8576, 272), (12, 4480, 48), (12, 12288, 16),
        (24, 4352, 64), (30, 8576, 32), (60, 4224, 32), (1, 8320, 8208), (2, 4608, 8224)]


@DTYPES
@BOTH
@pytest.mark.parametrize("rows,n_in,n_out", LONG)
def test_linear_of_few_long_rows(P, fmt, dtype, rows, n_in, n_out):
    _linear(P, np.random.default_rng(rows + n_in), fmt, dtype, rows, n_in, n_out, 2)


# The rows quantized by the product's own kernel (up to 16 rows of bf16, 4 of fp32, 4096 channels, 4096 outputs)
# and by a launch before it.
ROWS = [(1, 9, 8, 1, 4096, 256), (1, 1, 0, 1, 128, 16), (1, 3, 1, 1, 4224, 144), (2, 4, 2, 2, 8192, 80),
        (1, 20, 4, 16, 8576, 272), (4, 5, 1, 4, 4480, 64), (1, 7, 3, 4, 12288, 528), (1, 2, 1, 1, 65536, 256),
        (1, 64, 3, 1, 4096, 4096), (1, 3, 0, 3, 4096, 8208)]


@DTYPES
@BOTH
@pytest.mark.parametrize("b,seq,start,rows,n_in,n_out", ROWS)
def test_quantize_linear_values(P, fmt, dtype, b, seq, start, rows, n_in, n_out):
    import torch
    g = np.random.default_rng(n_in + n_out)
    x = g.standard_normal((b, seq, n_in)).astype(np.float32)
    x[..., ::50] *= 30
    x[:, :start] = x[:, start + rows:] = np.nan            # rows that are not asked for
    x = _bits(x, dtype)
    wc, ws, w = _held(g, (n_out, n_in), "mxfp4")
    wc, ws, xt, dt = _dev(wc), _dev(ws), to_dev(x, dtype), _type(dtype)
    f = P.CODECS[fmt]
    v = mx.values(*mx.quantize(_vals(x[:, start:start + rows], dtype), fmt), fmt).reshape(-1, n_in)
    want = v @ w.T
    tol = _linear_bound(v, w, want, fmt, dtype)
    buf, raw = _guarded((b * rows * n_out * dt.itemsize,))
    y = raw.view(dt).view(b, rows, n_out)
    P.mx_quantize_linear(f, xt, start, rows, wc, ws, y)
    _check(y, want, tol)
    _guards_hold(buf)
    z = torch.empty_like(y)
    P.mx_linear(f, *P.mx_quantize(f, xt, start, rows), wc, ws, z)
    _check(z, want, tol)


@DTYPES
@BOTH
@pytest.mark.parametrize("rows,n_in", [(1, 512), (3, 1152), (16, 640), (1, 4224), (4, 4096)])
def test_quantize_linear_reads_the_oracles_codes(P, fmt, dtype, rows, n_in):
    """Weights with a single 1 per output: the outputs are the rows' decoded channels, bit for bit (ties, values that
    saturate, zero blocks and blocks 2^60 apart among them)."""
    import torch
    if dtype == "fp32":
        rows = min(rows, 4)                                # the kernel that quantizes takes so many
    g = np.random.default_rng(rows + n_in)
    x = g.standard_normal((1, rows, n_in)) * 2.0 ** g.integers(-30, 31, (1, rows, n_in // 32)).repeat(32, axis=-1)
    blocks = x.reshape(-1, 32)
    ties = np.array([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -5, 7.5, -7.9, 448, 17, 19, -21, 2 ** -10, 3 * 2 ** -10])
    blocks[1::5] = np.resize(ties, 32) * 2.0 ** g.integers(-9, 10, (len(blocks[1::5]), 1))
    blocks[2::5] = np.resize(ties[:12], 32) * 2.0 ** g.integers(-9, 10, (len(blocks[2::5]), 1))
    blocks[3::11] = 0
    x = _bits(x.astype(np.float32), dtype)
    w = np.zeros((n_in, n_in))
    at = g.permutation(n_in)
    w[np.arange(n_in), at] = 1
    n_out = n_in if n_in < 2048 else 256                   # (few enough workgroups for that kernel)
    wc, ws = mx.quantize(w[:n_out], "mxfp4")
    y = torch.empty((1, rows, n_out), dtype=_type(dtype), device="cuda")
    P.mx_quantize_linear(P.CODECS[fmt], to_dev(x, dtype), 0, rows, _dev(mx.pack(wc, "mxfp4")), _dev(ws.astype(np.uint8)), y)
    want = mx.values(*mx.quantize(_vals(x, dtype), fmt), fmt)[..., at[:n_out]]
    assert np.array_equal(y.double().cpu().numpy(), want)


# Scales of rows and weights up to 2^40 and 2^20 apart, on the few-rows kernel, the tiles and a split product: what
# is added first must not cost more than the sum of the magnitudes allows.
@DTYPES
@BOTH
@pytest.mark.parametrize("spread", [10, 20])
@pytest.mark.parametrize("rows,n_in,n_out", [(3, 896, 144), (40, 640, 272), (97, 3584, 400), (513, 384, 784),
                                             (1000, 1152, 2064)])
def test_linear_of_scales_far_apart(P, fmt, dtype, rows, n_in, n_out, spread):
    _linear(P, np.random.default_rng(rows + spread), fmt, dtype, rows, n_in, n_out, spread)


def test_rows_without_channels_are_refused(P):
    import torch
    u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    x = torch.empty((4, 0), device="cuda")
    for call in (lambda: P.residual_rmsnorm_mx(P.MXFP8, x, None, None, u8(4, 0), u8(4, 0)),
                 lambda: P.mx_dequantize(P.MXFP4, u8(4, 0), u8(4, 0), x),
                 lambda: P.mx_quantize(P.MXFP4, x),
                 lambda: P.mx_linear(P.MXFP8, u8(0, 0), u8(0, 0), u8(16, 0), u8(16, 0), torch.empty((0, 16), device="cuda"))):
        with pytest.raises(P.PolestarError) as e:
            call()
        assert e.value.status == 1

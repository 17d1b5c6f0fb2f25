"""CPU tests of the microscaled forward's boundary and oracle: the header's
symbols are exported, bad arguments are refused on the host before anything is
enqueued (fake pointers below never reach a kernel), the Python entry points
refuse what does not fit, and the oracle's codes are the codec oracle's."""

import os
import re

import numpy as np
import pytest

from oracle import codec_ref as cr
from oracle import mx_ref as mx
from tests._util import ROOT, ensure_built
from paper_2607_14107_amd import polestar as ps

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 4
FAKE = 0x10000          # 16-byte aligned, never dereferenced
OFF4, OFF1 = 0x10004, 0x10001


@pytest.fixture(scope="module")
def L():
    return ensure_built()


def _refused(f, args, changes):
    for at, value, status in changes:
        a = list(args)
        a[at] = value
        assert f(*a) == status, (at, value)


def test_every_declared_symbol_is_exported(L):
    with open(os.path.join(ROOT, "include", "polestar_mx.h")) as f:
        names = set(re.findall(r"^(?:polestar_status|size_t) (polestar_[a-z_]+)\(", f.read(), re.M))
    assert len(names) == 10, names
    for n in names:
        assert hasattr(L, n), n


def test_quantize_refusals(L):
    # fmt dtype batch seq n row_start n_rows x codes scales stream
    a = [1, 1, 2, 8, 64, 2, 4, FAKE, FAKE, FAKE, None]
    _refused(L.polestar_mx_quantize, a, [
        (0, 2, INVALID), (0, -1, INVALID), (1, 2, INVALID), (2, 0, INVALID), (3, 0, INVALID), (4, 0, INVALID),
        (5, -1, INVALID), (5, 5, INVALID), (6, 0, INVALID), (6, 7, INVALID), (7, None, INVALID), (8, None, INVALID),
        (9, None, INVALID), (4, 48, UNSUPPORTED), (4, 4, UNSUPPORTED), (7, OFF4, UNSUPPORTED), (8, OFF4, UNSUPPORTED),
        (2, 65536, UNSUPPORTED)])


def test_dequantize_refusals(L):
    # fmt dtype rows n codes scales y stream
    a = [0, 1, 4, 64, FAKE, FAKE, FAKE, None]
    _refused(L.polestar_mx_dequantize, a, [
        (0, 2, INVALID), (1, 3, INVALID), (2, -1, INVALID), (3, 0, INVALID), (4, None, INVALID), (5, None, INVALID),
        (6, None, INVALID), (3, 4, UNSUPPORTED), (3, 40, UNSUPPORTED), (4, OFF4, UNSUPPORTED), (6, OFF4, UNSUPPORTED),
        (2, 1 << 40, UNSUPPORTED), (2, 0, 0)])


def test_linear_refusals(L):
    # x_fmt dtype rows n_in n_out xc xs wc ws y workspace bytes stream
    need = ps.mx_linear_workspace_size(1, 1, 96, 512, 4096)
    a = [1, 1, 96, 4096, 512, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, need, None]
    changes = [(0, 5, INVALID), (1, 2, INVALID), (2, -1, INVALID), (3, 0, INVALID), (4, 0, INVALID)]
    changes += [(i, None, INVALID) for i in range(5, 10)]
    changes += [(3, 4096 + 64, UNSUPPORTED), (4, 520, UNSUPPORTED), (5, OFF4, UNSUPPORTED), (7, OFF4, UNSUPPORTED),
                (9, OFF4, UNSUPPORTED), (10, OFF4, UNSUPPORTED), (6, OFF1, UNSUPPORTED), (8, OFF1, UNSUPPORTED),
                (2, 1 << 30, UNSUPPORTED), (2, 0, 0)]
    if need:
        changes += [(11, need - 1, WORKSPACE), (10, None, WORKSPACE)]
    _refused(L.polestar_mx_linear, a, changes)


def test_quantize_linear_refusals(L):
    # x_fmt dtype batch seq n_in n_out row_start n_rows x wc ws y workspace bytes stream
    need = ps.mx_quantize_linear_workspace_size(1, 1, 2, 48, 512, 4096)
    a = [1, 1, 2, 64, 4096, 512, 8, 48, FAKE, FAKE, FAKE, FAKE, FAKE, need, None]
    changes = [(0, 5, INVALID), (1, 2, INVALID), (2, 0, INVALID), (3, 0, INVALID), (4, 0, INVALID), (5, 0, INVALID),
               (6, -1, INVALID), (6, 17, INVALID), (7, 0, INVALID), (7, 57, INVALID)]
    changes += [(i, None, INVALID) for i in range(8, 12)]
    changes += [(4, 4096 + 32, UNSUPPORTED), (5, 8, UNSUPPORTED), (8, OFF4, UNSUPPORTED), (9, OFF4, UNSUPPORTED),
                (10, OFF1, UNSUPPORTED), (11, OFF4, UNSUPPORTED), (12, OFF4, UNSUPPORTED), (13, need - 1, WORKSPACE),
                (12, None, WORKSPACE), (2, 65536, UNSUPPORTED)]
    _refused(L.polestar_mx_quantize_linear, a, changes)


def test_norm_refusals(L):
    # fmt dtype rows d x y gain eps x_out codes scales stream
    a = [1, 1, 4, 4096, FAKE, FAKE, FAKE, 1e-5, FAKE, FAKE, FAKE, None]
    _refused(L.polestar_residual_rmsnorm_mx, a, [
        (0, 3, INVALID), (1, 2, INVALID), (2, -1, INVALID), (3, 0, INVALID), (4, None, INVALID), (7, -1.0, INVALID),
        (7, float("nan"), INVALID), (8, None, INVALID), (9, None, INVALID), (10, None, INVALID), (3, 48, UNSUPPORTED),
        (3, 16384 + 32, UNSUPPORTED), (4, OFF4, UNSUPPORTED), (5, OFF4, UNSUPPORTED), (6, OFF4, UNSUPPORTED),
        (8, OFF4, UNSUPPORTED), (9, OFF4, UNSUPPORTED), (2, 1 << 33, UNSUPPORTED), (2, 0, 0)])


def test_store_refusals(L):
    # dtype batch seq kvh hd n_rows k v stride idx count row_start kc ks vc vs stream
    a = [1, 2, 64, 4, 128, 16, FAKE, FAKE, 512, None, None, 8, FAKE, FAKE, FAKE, FAKE, None]
    changes = [(0, 2, INVALID), (1, 0, INVALID), (2, 0, INVALID), (3, 0, INVALID), (4, 0, INVALID), (5, -1, INVALID),
               (5, 57, INVALID), (8, 504, INVALID), (11, -1, INVALID), (11, 49, INVALID)]
    changes += [(i, None, INVALID) for i in (6, 7, 12, 13, 14, 15)]
    changes += [(4, 96, UNSUPPORTED), (8, 516, UNSUPPORTED), (6, OFF4, UNSUPPORTED), (7, OFF4, UNSUPPORTED),
                (12, OFF4, UNSUPPORTED), (14, OFF4, UNSUPPORTED), (13, OFF1, UNSUPPORTED), (15, OFF1, UNSUPPORTED),
                (1, 65536, UNSUPPORTED), (5, 0, 0)]
    _refused(L.polestar_mx_store_kv, a, changes)


def test_attend_refusals(L):
    # dtype batch seq heads kvh hd n_rows q stride kc ks vc vs kv_len scale out lse ws bytes stream
    need = ps.mx_attend_workspace_size(1, 2, 4096, 8, 2, 128, 32)
    a = [1, 2, 4096, 8, 2, 128, 32, FAKE, 1024, FAKE, FAKE, FAKE, FAKE, FAKE, 0.0, FAKE, FAKE, FAKE, need, None]
    changes = [(0, 2, INVALID), (1, 0, INVALID), (2, 0, INVALID), (3, 0, INVALID), (3, 7, INVALID), (4, 0, INVALID),
               (5, 0, INVALID), (6, 0, INVALID), (8, 1016, INVALID)]
    changes += [(i, None, INVALID) for i in (7, 9, 10, 11, 12, 15)]
    changes += [(5, 96, UNSUPPORTED), (8, 1028, UNSUPPORTED), (7, OFF4, UNSUPPORTED), (9, OFF4, UNSUPPORTED),
                (11, OFF4, UNSUPPORTED), (10, OFF1, UNSUPPORTED), (12, OFF1, UNSUPPORTED), (15, OFF4, UNSUPPORTED),
                (17, OFF4, UNSUPPORTED), (1, 65536, UNSUPPORTED)]
    if need:
        changes += [(18, need - 1, WORKSPACE), (17, None, WORKSPACE)]
    _refused(L.polestar_mx_attend, a, changes)


def test_workspace_sizes_of_bad_shapes_are_zero(L):
    assert ps.mx_linear_workspace_size(1, 1, 0, 512, 4096) == 0
    assert ps.mx_linear_workspace_size(7, 1, 4, 512, 4096) == 0
    assert ps.mx_linear_workspace_size(1, 1, 4, 512, 100) == 0
    assert ps.mx_quantize_linear_workspace_size(1, 1, 0, 4, 512, 4096) == 0
    assert ps.mx_quantize_linear_workspace_size(1, 3, 1, 4, 512, 4096) == 0
    assert ps.mx_attend_workspace_size(1, 0, 64, 4, 2, 128, 1) == 0
    assert ps.mx_attend_workspace_size(1, 1, 64, 4, 3, 128, 1) == 0
    assert ps.mx_attend_workspace_size(1, 1, 64, 4, 2, 96, 1) == 0


def test_store_refuses_a_single_row_with_heads_out_of_order():
    """One row has no row stride, but its heads still have to lie one after another, in v as in k."""
    torch = pytest.importorskip("torch")
    caches = [torch.zeros((1, 2, 9, n), dtype=torch.uint8) for n in (32, 2, 32, 2)]
    good = torch.zeros(1, 1, 2, 64)
    bad = torch.zeros(1, 1, 64, 2).transpose(2, 3)
    for k, v in ((good, bad), (bad, good)):
        with pytest.raises(ValueError, match="equally spaced"):
            ps.mx_store_kv(k, v, *caches)


def test_python_entry_points_refuse_cpu_tensors_and_shapes():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 4, 64)
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    with pytest.raises(ValueError):
        ps.mx_quantize(ps.MXFP8, x)                                              # not on the GPU
    with pytest.raises(ValueError):
        ps.mx_quantize(ps.MXFP8, x[0], row_start=1)
    with pytest.raises(ValueError):
        ps.mx_dequantize(ps.MXFP4, u8(4, 64), u8(4, 2), torch.zeros(4, 64))      # 64 bytes are 128 channels
    with pytest.raises(ValueError):
        ps.mx_linear(ps.MXFP8, u8(4, 128), u8(4, 4), u8(16, 32), u8(16, 2), torch.zeros(4, 16))
    with pytest.raises(ValueError):
        ps.mx_quantize_linear(ps.MXFP8, torch.zeros(1, 4, 128), 0, 4, u8(16, 64), u8(16, 4), torch.zeros(1, 3, 16))
    with pytest.raises(ValueError):
        ps.residual_rmsnorm_mx(ps.MXFP8, x, x, None, u8(2, 4, 64), u8(2, 4, 2))  # a sum needs x_out
    caches = [u8(2, 2, 9, 32), u8(2, 2, 9, 2)] * 2
    kv = torch.zeros(2, 3, 2, 64)
    with pytest.raises(ValueError):
        ps.mx_store_kv(kv[:, :, :, :32], kv[:, :, :, :32], *caches)
    with pytest.raises(ValueError):
        ps.mx_store_kv(kv.transpose(0, 1).contiguous().transpose(0, 1), kv, *caches)   # rows not equally spaced
    with pytest.raises(ValueError):
        ps.mx_store_kv(kv, kv, *caches, count=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        ps.mx_attend(torch.zeros(2, 3, 4, 128), *caches)
    with pytest.raises(ValueError):
        ps.mx_attend(torch.zeros(2, 3, 4, 64), *caches, kv_len=torch.zeros(3, dtype=torch.int32))


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
def test_oracle_codes_are_the_codec_oracles(fmt):
    g = np.random.default_rng(5)
    x = (g.standard_normal((6, 128)) * 10.0 ** g.uniform(-30, 30, (6, 4)).repeat(32, axis=1)).astype(np.float32)
    x[1, :32] = 0
    x[2, 32:64] = 1e-44                                    # subnormal: the scale's lower clamp
    vals, _ = cr._grid(fmt)
    mid = (vals[1:] + vals[:-1]) / 2
    x[3, :32] = np.resize(np.concatenate([mid, -mid]), 32) # ties
    x[3, 0] = vals[-1]
    codes, scales = mx.quantize(x, fmt)
    want, exps = cr.encode(x, np.zeros_like(x), fmt)
    assert np.array_equal(codes, want) and np.array_equal(scales, exps + 127)
    assert np.array_equal(mx.pack(codes, fmt), cr.pack(want, exps, fmt)[0])
    assert np.array_equal(mx.held(mx.pack(codes, fmt), scales, fmt), cr.decode(want, exps, np.zeros_like(x), fmt))


def test_oracle_marks_blocks_that_are_not_finite():
    x = np.ones((1, 96))
    x[0, 3], x[0, 40] = np.nan, -np.inf
    codes, scales = mx.quantize(x, "mxfp4")
    assert scales.tolist() == [[255, 255, 125]] and not codes[0, :64].any()
    v = mx.values(codes, scales, "mxfp4")
    assert np.isnan(v[0, :64]).all() and (v[0, 64:] == 1).all()

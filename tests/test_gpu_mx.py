"""GPU parity of the microscaled forward against the float64 oracle
(oracle/mx_ref.py): codes, scales and decoded values bit for bit; products,
attention and a layer's chain within bounds derived from the roundings.

Bounds.  A rounding to bf16 is off by at most 2^-8 relative (half a step), to fp32
by 2^-24.  A product of MXFP8 rows for bf16 outputs adds eight neighbours with a
unit of 2^-13 of the largest of them, seven of which can lose one unit: 7 * 2^-13
of the sum of the products' magnitudes.  Every other sum is n additions of fp32
numbers, each off by at most 2^-23 of the magnitudes' sum (a matrix instruction may
truncate)."""

import numpy as np
import pytest

from oracle import mx_ref as mx
from tests._util import ensure_built, from_dev, to_dev

pytestmark = pytest.mark.gpu

BF16, F32 = 2.0 ** -8, 2.0 ** -23
GUARD = 0xA5


@pytest.fixture(scope="module")
def P():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    ensure_built()
    from paper_2607_14107_amd import polestar
    return polestar


def _torch():
    import torch
    return torch


def _bits(x, dtype):
    """float32 values as stored: bf16 bits (nearest even) or float32."""
    if dtype == "fp32":
        return np.asarray(x, np.float32)
    torch = _torch()
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


def _vals(bits, dtype):
    """Stored array -> float64."""
    if dtype == "fp32":
        return bits.astype(np.float64)
    return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def _dev(x):
    return _torch().from_numpy(np.ascontiguousarray(x)).cuda()


def _guarded(shape):
    """A uint8 tensor of this shape inside a longer buffer of guard bytes."""
    torch = _torch()
    n = int(np.prod(shape))
    buf = torch.full((n + 512,), GUARD, dtype=torch.uint8, device="cuda")
    return buf, buf[256:256 + n].view(shape)


def _guards_hold(buf):
    assert (buf[:256] == GUARD).all() and (buf[-256:] == GUARD).all()


def _rows(g, *shape):
    """Blocks of magnitudes from 1e-30 to 1e30, zeros, subnormals, ties, one NaN and one infinity block."""
    n = shape[-1]
    x = g.standard_normal(shape) * 10.0 ** g.uniform(-30, 30, (*shape[:-1], n // 32)).repeat(32, axis=-1)
    flat = x.reshape(-1, 32)
    flat[::7] = 0
    flat[1::11] = 1e-41
    ties = np.array([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -5, 448, 17, 19, -21, 2 ** -10, 3 * 2 ** -10])
    flat[2::13] = np.resize(ties, 32) * 2.0 ** g.integers(-60, 60, (len(flat[2::13]), 1))
    flat[3::17] = np.abs(flat[3::17])
    if len(flat) > 5:
        flat[4, 9], flat[5, 31] = np.nan, np.inf
    return x.astype(np.float32)


SHAPES = [(1, 1, 32, 0, 1), (2, 7, 96, 3, 3), (3, 70, 4096, 0, 70), (1, 33, 3584, 1, 31), (2, 130, 160, 129, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
@pytest.mark.parametrize("b,seq,n,start,rows", SHAPES)
def test_quantize_is_the_oracles_bits_and_reads_back(P, fmt, dtype, b, seq, n, start, rows):
    torch = _torch()
    x = _bits(_rows(np.random.default_rng(n + seq), b, seq, n), dtype)
    f = P.CODECS[fmt]
    cb, codes = _guarded((b, rows, P.codec_row_bytes(f, n)))
    sb, scales = _guarded((b, rows, n // 32))
    P.mx_quantize(f, to_dev(x, dtype), start, rows, codes, scales)
    want, ws = mx.quantize(_vals(x[:, start:start + rows], dtype), fmt)
    assert np.array_equal(from_dev(scales), ws)
    assert np.array_equal(from_dev(codes), mx.pack(want, fmt))
    _guards_hold(cb)
    _guards_hold(sb)
    for out in (torch.float32, torch.bfloat16):
        y = torch.empty((b, rows, n), dtype=out, device="cuda")
        P.mx_dequantize(f, codes, scales, y)
        v = mx.values(want, ws, fmt)
        v[np.abs(v) < 2.0 ** -120] = 0                     # bf16 has fewer subnormals
        got = y.double().cpu().numpy()
        got[np.abs(got) < 2.0 ** -120] = 0
        assert np.array_equal(got, v, equal_nan=True)


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
def test_dequantize_every_code_at_every_scale(P, fmt):
    torch = _torch()
    f = P.CODECS[fmt]
    n = 32 if fmt == "mxfp4" else 256
    codes = np.tile(np.arange(n) % 16 if fmt == "mxfp4" else np.arange(n), (256, 1))
    if fmt == "mxfp8":
        codes[(codes & 127) == 127] = 0                    # the NaN pattern is no code of the format
    scales = np.repeat(np.arange(256)[:, None], n // 32, axis=1)
    y = torch.empty((256, n), device="cuda")
    P.mx_dequantize(f, _dev(mx.pack(codes, fmt)), _dev(scales.astype(np.uint8)), y)
    with np.errstate(over="ignore"):
        want = mx.values(codes, scales, fmt).astype(np.float32)
    assert np.array_equal(y.cpu().numpy(), want, equal_nan=True)
    z = torch.empty((256, n), dtype=torch.bfloat16, device="cuda")
    P.mx_dequantize(f, _dev(mx.pack(codes, fmt)), _dev(scales.astype(np.uint8)), z)
    normal = np.isnan(want) | (np.abs(want) >= 2.0 ** -126) | (want == 0)
    assert np.array_equal(z.float().cpu().numpy()[normal], want[normal], equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
@pytest.mark.parametrize("rows,d,gain,add,inplace", [(1, 32, False, True, False), (7, 96, True, True, True),
                                                     (130, 4096, False, True, True), (33, 3584, True, True, False),
                                                     (3, 16384, True, True, False), (5, 4128, True, False, False),
                                                     (2, 8192, False, False, True)])
def test_norm_is_the_oracles_bits(P, fmt, dtype, rows, d, gain, add, inplace):
    torch = _torch()
    g = np.random.default_rng(rows + d)
    f = P.CODECS[fmt]
    x = (g.standard_normal((rows, d)) * 3).astype(np.float32)
    x[:, ::37] *= 40
    if rows > 2:
        x[1] = 0                                           # eps alone keeps the row finite
        x[2, 5] = np.inf
    y = _bits(g.standard_normal((rows, d)), dtype)
    if rows > 2:
        y[1] = 0
    gn = (1 + 0.3 * g.standard_normal(d)).astype(np.float32) if gain else None
    xt = _dev(x)
    yt = to_dev(y, dtype) if add else None
    out = xt if inplace else (torch.empty_like(xt) if add else None)
    cb, codes = _guarded((rows, P.codec_row_bytes(f, d)))
    sb, scales = _guarded((rows, d // 32))
    P.residual_rmsnorm_mx(f, xt, yt, out, codes, scales, gain=None if gn is None else _dev(gn))
    s = x + _vals(y, dtype).astype(np.float32) if add else x
    with np.errstate(invalid="ignore"):
        want, ws = mx.quantize(mx.rmsnorm(s, gn, 1e-5), fmt)
    assert np.array_equal(from_dev(scales), ws)
    assert np.array_equal(from_dev(codes), mx.pack(want, fmt))
    if out is not None:
        assert np.array_equal(from_dev(out), s)
    _guards_hold(cb)
    _guards_hold(sb)


def _held(g, shape, fmt, spread=2):
    """Random codes and scale bytes around 1, and their values."""
    c = g.integers(0, 16 if fmt == "mxfp4" else 256, shape)
    if fmt == "mxfp8":
        c[(c & 127) == 127] = 1
    s = g.integers(127 - spread, 128 + spread, (*shape[:-1], shape[-1] // 32))
    return mx.pack(c, fmt), s.astype(np.uint8), mx.values(c, s, fmt)


def _linear_bound(x, w, want, fmt, dtype):
    mag = np.abs(x) @ np.abs(w).T
    tol = x.shape[1] * F32 * mag
    if dtype == "bf16":
        tol = tol + BF16 * np.abs(want) + (7 * 2.0 ** -13 * mag if fmt == "mxfp8" else 0)
    return tol


LINEAR = [(1, 128, 16), (1, 4096, 4096), (2, 256, 48), (5, 384, 272), (16, 1152, 64), (17, 640, 80), (32, 4096, 512),
          (33, 512, 144), (48, 896, 1040), (64, 384, 256), (65, 256, 272), (97, 3584, 1168), (130, 1024, 400),
          (256, 512, 528), (300, 2176, 256), (513, 384, 784), (64, 128, 8336), (3, 896, 8208), (40, 640, 8224)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
@pytest.mark.parametrize("rows,n_in,n_out", LINEAR)
def test_linear_matches_the_oracle(P, fmt, dtype, rows, n_in, n_out):
    torch = _torch()
    g = np.random.default_rng(rows * n_out + n_in)
    xc, xs, x = _held(g, (rows, n_in), fmt)
    wc, wsc, w = _held(g, (n_out, n_in), "mxfp4")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    buf, raw = _guarded((rows * n_out * dt.itemsize,))
    y = raw.view(dt).view(rows, n_out)
    P.mx_linear(P.CODECS[fmt], _dev(xc), _dev(xs), _dev(wc), _dev(wsc), y)
    want = x @ w.T
    err = np.abs(y.double().cpu().numpy() - want)
    tol = _linear_bound(x, w, want, fmt, dtype)
    assert (err <= tol).all(), (np.argwhere(err > tol)[:4].tolist(), (err / tol).max())
    _guards_hold(buf)


LARGE = [(4096, 384, 4096), (4000, 128, 4112), (2048, 896, 4096), (1000, 1152, 4096), (8192, 640, 2064), (1500, 2176, 4608),
         (512, 4224, 4096), (500, 2688, 2064)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
@pytest.mark.parametrize("rows,n_in,n_out", LARGE)
def test_linear_of_many_tiles_matches_the_oracle(P, fmt, dtype, rows, n_in, n_out):
    """Products that fill the GPU, on the larger tiles: 64 rows and 64 outputs of them are checked."""
    torch = _torch()
    g = np.random.default_rng(rows + n_in)
    xc, xs, x = _held(g, (rows, n_in), fmt)
    wc, wsc, w = _held(g, (n_out, n_in), "mxfp4")
    y = torch.empty((rows, n_out), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    P.mx_linear(P.CODECS[fmt], _dev(xc), _dev(xs), _dev(wc), _dev(wsc), y)
    r = np.unique(np.concatenate((g.integers(0, rows, 62), [0, rows - 1])))
    c = np.unique(np.concatenate((g.integers(0, n_out, 62), [0, n_out - 1])))
    got = y.double().cpu().numpy()
    for rr, cc in ((r, slice(None)), (slice(None), c)):
        want = x[rr] @ w[cc].T
        err = np.abs(got[rr][:, cc] - want)
        tol = _linear_bound(x[rr], w[cc], want, fmt, dtype)
        assert (err <= tol).all(), (err / tol).max()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
@pytest.mark.parametrize("rows", [3, 40, 200])
def test_linear_nan_blocks_reach_their_outputs_only(P, fmt, dtype, rows):
    torch = _torch()
    g = np.random.default_rng(rows)
    xc, xs, x = _held(g, (rows, 512), fmt)
    wc, wsc, w = _held(g, (96, 512), "mxfp4")
    xs[1, 7] = wsc[50, 3] = 255
    y = torch.empty((rows, 96), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    P.mx_linear(P.CODECS[fmt], _dev(xc), _dev(xs), _dev(wc), _dev(wsc), y)
    nan = torch.isnan(y).cpu().numpy()
    assert nan[1].all() and nan[:, 50].all()
    nan[1], nan[:, 50] = False, False
    assert not nan.any()


@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
def test_linear_extreme_scales(P, fmt):
    """Operands near the ends of the scales' range: 2^-90 times 2^90 is as 1 times 1."""
    torch = _torch()
    g = np.random.default_rng(1)
    xc, xs, x = _held(g, (70, 256), fmt, 1)
    wc, wsc, w = _held(g, (48, 256), "mxfp4", 1)
    xs, wsc = xs - 90, wsc + 90
    for dt in (torch.bfloat16, torch.float32):
        y = torch.empty((70, 48), dtype=dt, device="cuda")
        P.mx_linear(P.CODECS[fmt], _dev(xc), _dev(xs), _dev(wc), _dev(wsc), y)
        want = x @ w.T
        tol = _linear_bound(x, w, want, fmt, "bf16" if dt == torch.bfloat16 else "fp32")
        assert (np.abs(y.double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fmt", ["mxfp4", "mxfp8"])
@pytest.mark.parametrize("b,seq,start,rows,n_in,n_out", [(1, 9, 8, 1, 4096, 256), (1, 40, 3, 4, 640, 80),
                                                         (2, 20, 5, 8, 1152, 272), (3, 50, 1, 11, 384, 144),
                                                         (2, 96, 10, 65, 512, 400), (4, 130, 0, 130, 256, 272)])
def test_quantize_linear_is_the_two_calls(P, fmt, dtype, b, seq, start, rows, n_in, n_out):
    torch = _torch()
    f = P.CODECS[fmt]
    g = np.random.default_rng(seq + n_out)
    x = g.standard_normal((b, seq, n_in)).astype(np.float32)
    x[..., ::50] *= 30
    x[0, start, 40] = np.nan
    x = _bits(x, dtype)
    wc, wsc, w = _held(g, (n_out, n_in), "mxfp4")
    wc, wsc, xt = _dev(wc), _dev(wsc), to_dev(x, dtype)
    y = torch.empty((b, rows, n_out), dtype=xt.dtype, device="cuda")
    z = torch.empty_like(y)
    P.mx_quantize_linear(f, xt, start, rows, wc, wsc, y)
    P.mx_linear(f, *P.mx_quantize(f, xt, start, rows), wc, wsc, z)
    assert torch.isnan(y[0, 0]).all()
    v = mx.values(*mx.quantize(_vals(x[:, start:start + rows], dtype), fmt), fmt).reshape(-1, n_in)
    v[0] = 0
    want = v @ w.T
    for t in (y, z):
        err = np.abs(t.double().cpu().numpy().reshape(-1, n_out) - want)[1:]
        assert (err <= _linear_bound(v, w, want, fmt, dtype)[1:]).all()


# ---------------------------------------------------------------------------
# caches in MXFP4
# ---------------------------------------------------------------------------

def _packed(g, b, n, heads, hd, dtype, packed, extra=2):
    """[b][n][heads][hd] stored values, inside wider rows or rows of their own."""
    wide = heads + (extra if packed else 0)
    bits = _bits(g.standard_normal((b, n, wide, hd)).astype(np.float32) * 1.5, dtype)
    t = to_dev(bits, dtype)
    return bits[:, :, :heads], t[:, :, :heads]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("b,seq,kvh,n,listed,counted", [(1, 1, 1, 1, False, False), (2, 50, 3, 17, False, False),
                                                        (2, 50, 4, 23, True, True), (3, 400, 2, 300, True, False)])
def test_store_kv(P, dtype, hd, b, seq, kvh, n, listed, counted):
    torch = _torch()
    g = np.random.default_rng(seq + n)
    kb, k = _packed(g, b, n, kvh, hd, dtype, True)
    vb, v = _packed(g, b, n, kvh, hd, dtype, True)
    start = 0 if listed else seq - n
    pos = np.tile(np.arange(start, start + n), (b, 1))
    count = np.full(b, n)
    idx = cnt = None
    if listed:
        pos = g.integers(-2, seq + 2, (b, n))              # entries outside, and equal ones
        if counted:
            count = np.array([n + 5, 6, 0][:b])            # clamped to n
            cnt = _dev(count.astype(np.int32))
        idx = _dev(pos.astype(np.int32))
    caches, want = [], []
    for bits in (kb, vb):
        cb, codes = _guarded((b, kvh, seq, hd // 2))
        sb, scales = _guarded((b, kvh, seq, hd // 32))
        codes[:], scales[:] = GUARD, GUARD
        wc, wsc = np.full((b, kvh, seq, hd // 2), GUARD, np.uint8), np.full((b, kvh, seq, hd // 32), GUARD, np.uint8)
        q, s = mx.quantize(_vals(bits, dtype), "mxfp4")
        q = mx.pack(q, "mxfp4")
        for i in range(b):
            for r in range(min(n, count[i])):              # a later entry overwrites
                if 0 <= pos[i, r] < seq:
                    wc[i, :, pos[i, r]], wsc[i, :, pos[i, r]] = q[i, r], s[i, r]
        caches += [(codes, cb), (scales, sb)]
        want += [wc, wsc]
    P.mx_store_kv(k, v, *(t for t, _ in caches), row_start=start, idx=idx, count=cnt)
    for (t, buf), w in zip(caches, want):
        assert np.array_equal(from_dev(t), w)
        _guards_hold(buf)
    P.mx_store_kv(k[:, :0], v[:, :0], *(t for t, _ in caches))              # no rows: nothing happens


def _attend_case(P, g, dtype, b, seq, n, heads, kvh, hd, lens, packed, scale, want_lse=True):
    torch = _torch()
    kc, ks, kv = _held(g, (b, kvh, seq, hd), "mxfp4", 1)
    vc, vs, vv = _held(g, (b, kvh, seq, hd), "mxfp4", 2)
    qb, q = _packed(g, b, n, heads, hd, dtype, packed, 3)
    if lens is not None:
        for i, m in enumerate(lens):                       # anything may stand past the end
            ks[i, :, max(m, 0):] = vs[i, :, max(m, 0):] = 255
    buf, raw = _guarded((b * n * heads * hd * q.element_size(),))
    out = raw.view(q.dtype).view(b, n, heads, hd)
    lse = torch.full((b, heads, n), 7.0, device="cuda") if want_lse else None
    P.mx_attend(q, _dev(kc), _dev(ks), _dev(vc), _dev(vs), scale=scale, out=out, lse=lse,
                kv_len=None if lens is None else _dev(np.array(lens, np.int32)))
    _guards_hold(buf)
    got, gl = out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
    sc = scale if scale > 0 else 1 / np.sqrt(hd)
    qv = _vals(qb, dtype)
    for i in range(b):
        m = seq if lens is None else min(max(lens[i], 0), seq)
        for h in range(heads):
            kk, vx = np.nan_to_num(kv[i, h // (heads // kvh)]), np.nan_to_num(vv[i, h // (heads // kvh)])
            o, l, pv, qk = mx.attend(qv[i, :, h], kk, vx, m, sc)
            if m == 0:                                     # exactly zeros, and no weight at all
                assert not got[i, :, h].any() and (gl is None or np.isneginf(gl[i, h]).all())
                continue
            # a score: hd products, fp32 sums; a probability: its exponent's error twice, exp2's last bits
            ds = hd * F32 * qk + 4 * F32 * np.maximum(np.abs(l), 1) + 2.0 ** -21
            tol = (2 * ds + m * F32)[:, None] * pv
            if dtype == "bf16":
                tol = tol + BF16 * pv + BF16 * np.abs(o)
            err = np.abs(got[i, :, h] - o)
            assert (err <= tol).all(), (i, h, m, (err / np.maximum(tol, 1e-300)).max())
            if gl is not None:
                assert (np.abs(gl[i, h] - l) <= 2 * ds + m * F32).all()


ATTEND = [  # b, seq, rows, heads, kv_heads, lens, packed, scale
    (1, 1, 1, 1, 1, None, False, 0.0),
    (2, 33, 1, 4, 4, None, True, 0.0),
    (3, 97, 5, 4, 2, (97, 0, 13), False, 0.2),
    (2, 200, 32, 2, 2, (1, 200), False, 0.0),
    (1, 130, 33, 3, 3, None, False, 0.0),
    (2, 520, 1, 28, 4, (519, 64), True, 0.0),
    (1, 1025, 64, 14, 2, None, True, 0.0),
    (4, 65, 17, 6, 1, (65, 32, 31, 1000), True, 0.0),
    (1, 4100, 3, 8, 8, (4097,), False, 0.0),
    (5, 12, 2, 2, 1, (0, 0, -3, 12, 1), False, 0.0),
    (1, 9000, 1, 7, 1, (8999,), True, 0.0),
    (8, 530, 2, 20, 20, (530, 0, 1, 511, 513, 32, 31, 600), False, 0.0),      # 160 workgroups: no split
    (9, 513, 1, 30, 30, (513, 512, 17, 0, 480, 5, 513, 513, 100), True, 0.0),  # 270 workgroups
    (1, 33000, 1, 4, 1, (32999,), False, 0.0),                                # the most splits
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("b,seq,n,heads,kvh,lens,packed,scale", ATTEND)
def test_attend_matches_the_oracle(P, dtype, hd, b, seq, n, heads, kvh, lens, packed, scale):
    _attend_case(P, np.random.default_rng(seq + n), dtype, b, seq, n, heads, kvh, hd, lens, packed, scale)


def test_attend_without_lse(P):
    _attend_case(P, np.random.default_rng(3), "bf16", 2, 70, 3, 4, 2, 128, (70, 9), False, 0.0, want_lse=False)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attend_peaked_and_far_scores(P, dtype):
    """Scores hundreds apart, the largest first, last and in the middle: no overflow, the others vanish."""
    torch = _torch()
    b, seq, hd = 1, 700, 128
    for at in (0, 350, 699):
        kc, ks, kv = _held(np.random.default_rng(at), (b, 1, seq, hd), "mxfp4", 0)
        vc, vs, vv = _held(np.random.default_rng(at + 1), (b, 1, seq, hd), "mxfp4", 0)
        q = 40 * kv[0, 0, at]
        qt = _dev(q.astype(np.float32).reshape(1, 1, 1, hd)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
        out = P.mx_attend(qt, _dev(kc), _dev(ks), _dev(vc), _dev(vs))
        o, l, pv, qk = mx.attend(qt.double().cpu().numpy()[0, :, 0], kv[0, 0], vv[0, 0], seq, hd ** -0.5)
        tol = (2 * hd * F32 * qk[0] + 8 * F32 * abs(l[0]) + seq * F32) * pv + (2 * BF16 * pv if dtype == "bf16" else 0)
        assert (np.abs(out.double().cpu().numpy()[0, :, 0] - o) <= tol).all()


def test_attend_nan_key_reaches_its_head_only(P):
    torch = _torch()
    g = np.random.default_rng(9)
    kc, ks, _ = _held(g, (2, 2, 80, 64), "mxfp4", 1)
    vc, vs, _ = _held(g, (2, 2, 80, 64), "mxfp4", 1)
    ks[1, 0, 41, 1] = 255
    q = _dev(g.standard_normal((2, 3, 4, 64)).astype(np.float32)).bfloat16()
    out = torch.isnan(P.mx_attend(q, _dev(kc), _dev(ks), _dev(vc), _dev(vs)))
    assert out[1, :, :2].all() and not out[0].any() and not out[1, :, 2:].any()


def test_attend_offsets_past_32_bits(P):
    """The second sequence's caches start 2 GiB and its last heads' keys lie more than 4 GiB behind the pointers."""
    torch = _torch()
    b, kvh, seq, hd = 2, 32, 1_100_000, 128
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    codes = [torch.zeros((b, kvh, seq, hd // 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((b, kvh, seq, hd // 32), 127, dtype=torch.uint8, device="cuda") for _ in range(2)]
    g = np.random.default_rng(2)
    n = 40
    k, v = (_dev(g.standard_normal((b, n, kvh, hd)).astype(np.float32)).bfloat16() for _ in range(2))
    idx = _dev(np.tile(np.arange(n)[::-1], (b, 1)).astype(np.int32))
    P.mx_store_kv(k, v, codes[0], scales[0], codes[1], scales[1], idx=idx)
    q = _dev(g.standard_normal((b, 2, kvh, hd)).astype(np.float32)).bfloat16()
    out = P.mx_attend(q, codes[0], scales[0], codes[1], scales[1], kv_len=_dev(np.array([3, n], np.int32)))
    small = [t[:, :, :n].contiguous() for t in (codes[0], scales[0], codes[1], scales[1])]
    kk, vv = mx.held(from_dev(small[0]), from_dev(small[1]), "mxfp4"), mx.held(from_dev(small[2]), from_dev(small[3]), "mxfp4")
    wk = mx.values(*mx.quantize(k.double().cpu().numpy(), "mxfp4"), "mxfp4")
    assert np.array_equal(kk[1], wk[1, ::-1].transpose(1, 0, 2))
    for i, m in ((0, 3), (1, n)):
        for h in (0, 31):
            o, l, pv, qk = mx.attend(q.double().cpu().numpy()[i, :, h], kk[i, h], vv[i, h], m, hd ** -0.5)
            err = np.abs(out.double().cpu().numpy()[i, :, h] - o)
            assert (err <= (2 * hd * F32 * qk[:, None] + 2.0 ** -18) * pv + BF16 * (pv + np.abs(o))).all()


# ---------------------------------------------------------------------------
# together, on other streams, in graphs
# ---------------------------------------------------------------------------

class _Layer:
    """One layer's forward of a block in the microscaling formats, as a decoding loop would run it."""

    def __init__(self, P, b=2, seq=160, start=64, n=32, d=512, heads=8, kvh=2, hd=64):
        torch = _torch()
        self.P, self.dims = P, (b, seq, start, n, d, heads, kvh, hd)
        g = np.random.default_rng(11)
        f = lambda *s, std=1.0: _dev((g.standard_normal(s) * std).astype(np.float32))  # noqa: E731
        self.w_qkv = P.mx_quantize(P.MXFP4, f((heads + 2 * kvh) * hd, d, std=0.05).bfloat16())
        self.w_o = P.mx_quantize(P.MXFP4, f(d, heads * hd, std=0.05).bfloat16())
        self.x0, self.y0 = f(b, n, d, std=2), f(b, n, d, std=0.3).bfloat16()
        self.x = self.x0.clone()
        self.cache0 = (*P.mx_quantize(P.MXFP4, f(b, kvh * seq, hd)), *P.mx_quantize(P.MXFP4, f(b, kvh * seq, hd)))
        self.cache0 = [t.view(b, kvh, seq, -1) for t in self.cache0]
        self.cache = [t.clone() for t in self.cache0]
        self.len = _dev(np.array([start + n, seq][:b], np.int32))
        u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")  # noqa: E731
        bf = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.h = (u8(b, n, d), u8(b, n, d // 32))
        self.qkv, self.att, self.o = bf(b, n, (heads + 2 * kvh) * hd), bf(b, n, heads, hd), bf(b, n, d)
        self.lse = torch.empty((b, heads, n), device="cuda")
        self.ws1 = u8(max(16, P.mx_linear_workspace_size(P.MXFP8, P.BF16, b * n, (heads + 2 * kvh) * hd, d)))
        self.ws2 = u8(max(16, P.mx_attend_workspace_size(P.BF16, b, seq, heads, kvh, hd, n)))
        self.ws3 = u8(max(16, P.mx_quantize_linear_workspace_size(P.MXFP8, P.BF16, b, n, d, heads * hd)))

    def run(self, stream=None):
        P, (b, seq, start, n, d, heads, kvh, hd) = self.P, self.dims
        P.residual_rmsnorm_mx(P.MXFP8, self.x, self.y0, self.x, *self.h, stream=stream)
        P.mx_linear(P.MXFP8, *self.h, *self.w_qkv, self.qkv, workspace=self.ws1, stream=stream)
        rows = self.qkv.view(b, n, heads + 2 * kvh, hd)
        P.mx_store_kv(rows[:, :, heads:heads + kvh], rows[:, :, heads + kvh:], *self.cache, row_start=start, stream=stream)
        P.mx_attend(rows[:, :, :heads], *self.cache, kv_len=self.len, out=self.att, lse=self.lse, workspace=self.ws2,
                    stream=stream)
        P.mx_quantize_linear(P.MXFP8, self.att.view(b, n, heads * hd), 0, n, *self.w_o, self.o, workspace=self.ws3,
                             stream=stream)

    def reset(self):
        self.x.copy_(self.x0)
        for t, s in zip(self.cache, self.cache0):
            t.copy_(s)
        for t in (*self.h, self.qkv, self.att, self.o, self.lse):
            t.zero_()

    def results(self):
        return [t.clone() for t in (self.x, *self.h, self.qkv, *self.cache, self.att, self.lse, self.o)]


def test_layer_forward_stage_by_stage(P):
    """Every stage against the oracle on what the stage before it left."""
    a = _Layer(P)
    a.run()
    b, seq, start, n, d, heads, kvh, hd = a.dims
    wq, wo = (mx.held(from_dev(w[0]), from_dev(w[1]), "mxfp4") for w in (a.w_qkv, a.w_o))
    x = from_dev(a.x0) + _vals(from_dev(a.y0), "bf16").astype(np.float32)
    assert np.array_equal(from_dev(a.x), x)
    c, s = mx.quantize(mx.rmsnorm(x, None, 1e-5), "mxfp8")
    assert np.array_equal(from_dev(a.h[0]), c) and np.array_equal(from_dev(a.h[1]), s)
    h = mx.values(c, s, "mxfp8").reshape(-1, d)
    qkv = _vals(from_dev(a.qkv), "bf16")
    want = h @ wq.T
    assert (np.abs(qkv.reshape(want.shape) - want) <= _linear_bound(h, wq, want, "mxfp8", "bf16")).all()
    qkv = qkv.reshape(b, n, -1, hd)
    kv = []
    for i, at in ((0, heads), (2, heads + kvh)):
        got = mx.held(from_dev(a.cache[i]), from_dev(a.cache[i + 1]), "mxfp4")
        old = mx.held(from_dev(a.cache0[i]), from_dev(a.cache0[i + 1]), "mxfp4")
        old[:, :, start:start + n] = mx.values(*mx.quantize(qkv[:, :, at:at + kvh], "mxfp4"), "mxfp4").transpose(0, 2, 1, 3)
        assert np.array_equal(got, old)
        kv.append(got)
    att = _vals(from_dev(a.att), "bf16")
    lens = from_dev(a.len)
    for i in range(b):
        for j in range(heads):
            o, l, pv, qk = mx.attend(qkv[i, :, j], kv[0][i, j // (heads // kvh)], kv[1][i, j // (heads // kvh)], lens[i], hd ** -0.5)
            tol = (2 * hd * F32 * qk + 2.0 ** -18 + seq * F32)[:, None] * pv + BF16 * (pv + np.abs(o))
            assert (np.abs(att[i, :, j] - o) <= tol).all()
    v = mx.values(*mx.quantize(att.reshape(b * n, -1), "mxfp8"), "mxfp8")
    want = v @ wo.T
    assert (np.abs(_vals(from_dev(a.o), "bf16").reshape(want.shape) - want) <= _linear_bound(v, wo, want, "mxfp8", "bf16")).all()


def test_layer_forward_on_another_stream_and_twice_at_once(P):
    torch = _torch()
    a, c = _Layer(P), _Layer(P)
    a.run()
    want = a.results()
    a.reset()
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        a.reset(), c.reset()
        torch.cuda.synchronize()
        a.run(stream=s1)
        c.run(stream=s2)
        torch.cuda.synchronize()
        for t in (a, c):
            assert all(torch.equal(x, y) for x, y in zip(t.results(), want))


def test_layer_forward_in_a_graph(P):
    """Captured, then replayed with eager work between: every replay gives the eager bits."""
    torch = _torch()
    a = _Layer(P)
    a.run()
    want = a.results()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    for _ in range(4):
        a.reset()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a.results(), want))
        a.reset()
        a.run()
        assert all(torch.equal(x, y) for x, y in zip(a.results(), want))


def test_workspaces_that_are_missing_or_too_small(P):
    """Split products and attention on a side stream, their scratch and outputs made by the call: the same bits."""
    torch = _torch()
    g = np.random.default_rng(4)
    x = _dev(g.standard_normal((1, 80, 4096)).astype(np.float32)).bfloat16()
    w = P.mx_quantize(P.MXFP4, _dev(g.standard_normal((512, 4096)).astype(np.float32)))
    h = P.mx_quantize(P.MXFP8, x)
    caches = [t.view(2, 1, 4096, -1) for _ in range(2)
              for t in P.mx_quantize(P.MXFP4, _dev(g.standard_normal((8192, 128)).astype(np.float32)))]
    q = _dev(g.standard_normal((2, 3, 5, 128)).astype(np.float32)).bfloat16()
    sizes = [P.mx_linear_workspace_size(P.MXFP8, P.BF16, 80, 512, 4096),
             P.mx_quantize_linear_workspace_size(P.MXFP8, P.BF16, 1, 80, 512, 4096),
             P.mx_attend_workspace_size(P.BF16, 2, 4096, 5, 1, 128, 3)]
    assert all(sizes)
    y = lambda: torch.zeros((1, 80, 512), dtype=torch.bfloat16, device="cuda")  # noqa: E731

    def run(ws, **kw):
        return [P.mx_linear(P.MXFP8, *h, *w, y(), workspace=ws[0], **kw),
                P.mx_quantize_linear(P.MXFP8, x, 0, 80, *w, y(), workspace=ws[1], **kw),
                P.mx_attend(q, *caches, workspace=ws[2], **kw)]
    want = run([torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes])
    small = run([torch.empty(16, dtype=torch.uint8, device="cuda")] * 3)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        current = run([None] * 3)
    side.synchronize()
    for got in (small, current):
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    out = P.mx_attend(q, *caches, stream=side)              # a stream that is not the current one
    side.synchronize()
    assert torch.equal(out, want[2])


def test_no_rows_is_no_work(P):
    torch = _torch()
    u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    y = torch.empty((0, 16), device="cuda")
    assert P.mx_linear(P.MXFP8, u8(0, 128), u8(0, 4), u8(16, 64), u8(16, 4), y).shape == (0, 16)
    P.residual_rmsnorm_mx(P.MXFP4, torch.empty((0, 64), device="cuda"), None, None, u8(0, 32), u8(0, 2))
    P.mx_dequantize(P.MXFP4, u8(0, 32), u8(0, 2), torch.empty((0, 64), device="cuda"))

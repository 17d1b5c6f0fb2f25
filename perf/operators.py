"""The microscaled forward's operators: what one pass of each computes, over
which sizes, in plain torch operations and through the library.

A case is a dict of plain values.  Its "op" says which operator:

  linear   rows of a [batch][seq][n_in] array quantized to MXFP8 or MXFP4 and
           multiplied by weights held in MXFP4 (polestar_mx_quantize_linear)
  norm     residual add, RMSNorm, rows out in MXFP8 or MXFP4
           (polestar_residual_rmsnorm_mx; the rows are read back as values)
  store    new K/V rows quantized into caches held in MXFP4
           (polestar_mx_store_kv; the caches are read back as values)
  attend   attention of some query rows over caches held in MXFP4
           (polestar_mx_attend)

MXFP4 and MXFP8: 32 channels share a power of two 2^e, e = floor(log2 amax) -
emax (emax 2 and 8, e >= -127); values are rounded to nearest even on the
element's grid (E2M1 up to 6, E4M3 up to 448) and saturated.
"""

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp32": 4}
BITS = {"mxfp4": 4, "mxfp8": 8}
EPS = 1e-5


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def _linear(batch, seq, start, rows, n_in, n_out, fmt, dtype="bf16", **more):
    return dict(op="linear", batch=batch, seq=seq, start=start, rows=rows, n_in=n_in, n_out=n_out, fmt=fmt,
                dtype=dtype, **more)


def _norm(batch, rows, d, fmt, dtype="bf16", gain=False, **more):
    return dict(op="norm", batch=batch, rows=rows, d=d, fmt=fmt, dtype=dtype, gain=gain, **more)


def _store(batch, seq, rows, heads, kv_heads, hd, listed_rows, dtype="bf16", **more):
    return dict(op="store", batch=batch, seq=seq, rows=rows, heads=heads, kv_heads=kv_heads, hd=hd,
                listed_rows=listed_rows, dtype=dtype, **more)


def _attend(batch, seq, rows, heads, kv_heads, hd, ragged, packed, dtype="bf16", **more):
    return dict(op="attend", batch=batch, seq=seq, rows=rows, heads=heads, kv_heads=kv_heads, hd=hd, ragged=ragged,
                packed=packed, dtype=dtype, **more)


def listed():
    return [
        # one row through a square projection: the weights' stream and the launches
        _linear(1, 64, 63, 1, 4096, 4096, "mxfp8", name="linear_token"),
        # Dream-7B-shaped Q, K and V of a ragged set of rows, both operands in 4 bits, 32-bit outputs
        _linear(3, 160, 40, 97, 3584, 4608, "mxfp4", dtype="fp32", name="linear_ragged_fp32"),
        # LLaDA-8B-shaped down projection of the active blocks of 16 sequences (a plain decoding forward)
        _linear(16, 32, 0, 32, 12288, 4096, "mxfp8", name="linear_blocks_down"),
        # gate and up projections of whole sequences at a block entry: a large matrix product
        _linear(16, 768, 0, 768, 4096, 24576, "mxfp8", name="linear_entry_gate_up"),
        # one block's rows between two products
        _norm(1, 32, 4096, "mxfp8", name="norm_block"),
        # every row of 16 sequences
        _norm(16, 768, 4096, "mxfp8", name="norm_entry"),
        # stale rows and the block of one LLaDA-8B-shaped layer step, listed by position
        _store(1, 768, 138, 32, 32, 128, True, name="store_refresh"),
        # a block entry: every row of eight sequences, cut from the Q, K, V product
        _store(8, 1536, 1536, 28, 4, 128, False, name="store_entry"),
        # a tiny model's rows in 32 bits, head size 64, sequences of several lengths, one of them empty
        _attend(3, 97, 5, 4, 2, 64, True, False, dtype="fp32", name="attend_tiny_fp32"),
        # one token of two sequences over long caches
        _attend(2, 32768, 1, 28, 4, 128, True, True, name="attend_token_long"),
        # the active blocks of eight LLaDA-8B-shaped sequences
        _attend(8, 1536, 32, 32, 32, 128, False, False, name="attend_blocks"),
        # Dream-7B-shaped grouped heads, blocks of 64 rows, ragged lengths
        _attend(4, 2048, 64, 28, 4, 128, True, True, name="attend_grouped"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["linear", "linear", "linear", "norm", "store", "attend", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    fmt = rng.choice(["mxfp8", "mxfp4"])
    if op == "linear":
        n_in = 128 * _log_int(rng, 2, 96)
        n_out = 16 * _log_int(rng, 8, 1536)
        batch = _log_int(rng, 1, 16)
        rows = max(1, _log_int(rng, 1, 12288) // batch)
        while batch * rows * n_in * n_out > 12288 * 4096 * 24576:
            rows = (rows + 1) // 2
        seq = rows + rng.randrange(0, 64)
        return _linear(batch, seq, rng.randrange(0, seq - rows + 1), rows, n_in, n_out, fmt, dtype)
    if op == "norm":
        d = 32 * _log_int(rng, 2, 256)
        batch = _log_int(rng, 1, 16)
        rows = max(1, min(_log_int(rng, 1, 12288), 12288 * 4096 // d) // batch)
        return _norm(batch, rows, d, fmt, dtype, rng.random() < 0.5)
    hd = rng.choice([128, 128, 64])
    kv_heads = rng.choice([1, 2, 4, 8, 32])
    if op == "store":
        batch = _log_int(rng, 1, 8)
        seq = max(1, min(_log_int(rng, 1, 8192), 8 * 1536 * 4 // (batch * kv_heads)))
        heads = kv_heads * rng.choice([1, 4, 7])
        return _store(batch, seq, _log_int(rng, 1, seq), heads, kv_heads, hd, rng.random() < 0.5, dtype)
    heads = kv_heads * rng.choice([1, 4, 7] if kv_heads <= 8 else [1])
    batch = _log_int(rng, 1, 8)
    rows = rng.choice([1, 1, _log_int(rng, 2, 96), 32])
    seq = max(1, min(_log_int(rng, 1, 32768), 8 * 1536 * 32 * 32 // (batch * heads * rows),
                     8 * 1536 * 32 // (batch * kv_heads)))
    return _attend(batch, seq, rows, heads, kv_heads, hd, rng.random() < 0.5, rng.random() < 0.5, dtype)


# ---------------------------------------------------------------------------
# the microscaling formats in elementary operations
# ---------------------------------------------------------------------------

_GRID = {"mxfp4": (1, 0, 2, 6.0), "mxfp8": (3, -6, 8, 448.0)}   # mantissa bits, smallest exponent, emax, largest value


def _split(v, fmt):
    """v [..., n] -> whole grid steps' values [..., n/32, 32] and block exponents [..., n/32, 1] (v's precision)."""
    mant, emin, emax, top = _GRID[fmt]
    blocks = v.reshape(*v.shape[:-1], v.shape[-1] // 32, 32)
    amax = blocks.abs().amax(dim=-1, keepdim=True)
    e = torch.where(amax > 0, torch.frexp(amax).exponent - 1 - emax, -127).clamp(min=-127)
    scaled = _times_power(blocks, -e)
    step = (torch.frexp(scaled).exponent - 1).clamp(min=emin) - mant
    return _times_power(torch.round(_times_power(scaled, -step)), step).clamp(-top, top), e


def _times_power(v, e):
    """v * 2^e, in two factors so that neither leaves the type's range."""
    h = torch.div(e, 2, rounding_mode="floor")
    one = torch.ones((), dtype=v.dtype, device=v.device)
    return v * torch.ldexp(one, h) * torch.ldexp(one, e - h)


def _values(v, fmt):
    """What v's rows read as once they are held in the format."""
    q, e = _split(v, fmt)
    return _times_power(q, e).reshape(v.shape)


def _hold4(v):
    """MXFP4 codes [..., n/2] (lower channel in the low nibble) and scale bytes [..., n/32] of v [..., n]."""
    q, e = _split(v, "mxfp4")
    a = q.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code = (code | torch.where((q < 0), 8, 0).to(torch.uint8)).reshape(*v.shape[:-1], v.shape[-1] // 2, 2)
    return (code[..., 0] | (code[..., 1] << 4)).contiguous(), (e[..., 0] + 127).to(torch.uint8).contiguous()


def _read4(codes, scales, dtype=torch.float32):
    """The values of MXFP4 codes and scale bytes."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=dtype,
                         device=codes.device)
    nib = torch.stack((codes & 15, codes >> 4), dim=-1).reshape(*codes.shape[:-1], scales.shape[-1], 32)
    return _times_power(table[nib.int()], scales.int().unsqueeze(-1) - 127).reshape(*codes.shape[:-1],
                                                                                     2 * codes.shape[-1])


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV).manual_seed(1_000_003 * (seed + 1))
    dt = DTYPES[c["dtype"]]

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=g).to(dtype)

    if c["op"] == "linear":
        # normalised hidden states with a few strong channels, weights as a layer's, laid out in MXFP4 once
        x = normal(c["batch"], c["seq"], c["n_in"])
        x[..., ::97] *= 16
        w = _hold4(normal(c["n_out"], c["n_in"], std=0.02))
        y = torch.empty((c["batch"], c["rows"], c["n_out"]), dtype=dt, device=DEV)
        return {"case": c, "x": x.to(dt), "w": w, "y": y, "ws": {}}
    if c["op"] == "norm":
        shape = (c["batch"], c["rows"], c["d"])
        x = normal(*shape, std=3.0)
        x[..., ::61] *= 10
        gain = 1 + normal(c["d"], std=0.2) if c["gain"] else None
        rows = c["batch"] * c["rows"]
        return {"case": c, "x": x, "y": normal(*shape, std=0.5, dtype=dt), "gain": gain,
                "x_out": torch.empty_like(x),
                "codes": torch.empty((c["batch"], c["rows"], c["d"] * BITS[c["fmt"]] // 8), dtype=torch.uint8,
                                     device=DEV),
                "scales": torch.empty((c["batch"], c["rows"], c["d"] // 32), dtype=torch.uint8, device=DEV),
                "h": torch.empty(shape, dtype=torch.bfloat16, device=DEV), "rows": rows}
    b, n, H, G, hd, S = (c[k] for k in ("batch", "rows", "heads", "kv_heads", "hd", "seq"))
    k_codes, k_scales = _hold4(normal(b, G, S, hd))
    v_codes, v_scales = _hold4(normal(b, G, S, hd))
    st = {"case": c, "k_codes": k_codes, "k_scales": k_scales, "v_codes": v_codes, "v_scales": v_scales}
    if c["op"] == "store":
        qkv = normal(b, n, (H + 2 * G) * hd, dtype=dt)
        st["k"] = qkv[..., H * hd:(H + G) * hd].unflatten(-1, (G, hd))
        st["v"] = qkv[..., (H + G) * hd:].unflatten(-1, (G, hd))
        if c["listed_rows"]:
            at = torch.rand((b, S), generator=g, device=DEV).argsort(dim=1)[:, :n].sort(dim=1).values
            st["idx"] = at.to(torch.int32).contiguous()
            st["count"] = torch.randint((n + 1) // 2, n + 1, (b,), generator=g, device=DEV, dtype=torch.int32)
        st["k_out"] = torch.empty((b, G, S, hd), dtype=torch.bfloat16, device=DEV)
        st["v_out"] = torch.empty((b, G, S, hd), dtype=torch.bfloat16, device=DEV)
        return st
    # queries whose scores spread as a trained layer's do; cut from a Q, K, V product, or rows of their own
    if c["packed"]:
        st["q"] = normal(b, n, (H + 2 * G) * hd, std=1.5, dtype=dt)[..., :H * hd].unflatten(-1, (H, hd))
    else:
        st["q"] = normal(b, n, H, hd, std=1.5, dtype=dt)
    if c["ragged"]:
        st["kv_len"] = torch.randint((S + 1) // 2, S + 1, (b,), generator=g, device=DEV, dtype=torch.int32)
        if b > 2:
            st["kv_len"][1] = 0
    st["out"] = torch.empty((b, n, H, hd), dtype=dt, device=DEV)
    st["lse"] = torch.empty((b, H, n), dtype=torch.float32, device=DEV)
    st["ws"] = {}
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    return {"linear": _run_linear, "norm": _run_norm, "store": _run_store, "attend": _run_attend}[
        state["case"]["op"]](state)


def _workspace(P, state, nbytes):
    """The workspace that a serving loop keeps beside its buffers."""
    if "t" not in state["ws"]:
        state["ws"]["t"] = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=DEV)
    return state["ws"]["t"]


def _run_linear(s):
    c = s["case"]
    if own:
        from paper_2607_14107_amd import polestar as P
        fmt, dt = P.CODECS[c["fmt"]], P.BF16 if c["dtype"] == "bf16" else P.FP32
        ws = _workspace(P, s, P.mx_quantize_linear_workspace_size(fmt, dt, c["batch"], c["rows"], c["n_out"], c["n_in"]))
        P.mx_quantize_linear(fmt, s["x"], c["start"], c["rows"], *s["w"], s["y"], workspace=ws)
        return s["y"]
    x = _values(s["x"][:, c["start"]:c["start"] + c["rows"]].float(), c["fmt"])
    w = _read4(*s["w"])
    return (x.reshape(-1, c["n_in"]) @ w.t()).reshape(c["batch"], c["rows"], c["n_out"]).to(s["y"].dtype)


def _run_norm(s):
    c = s["case"]
    if own:
        from paper_2607_14107_amd import polestar as P
        fmt = P.CODECS[c["fmt"]]
        P.residual_rmsnorm_mx(fmt, s["x"], s["y"], s["x_out"], s["codes"], s["scales"], gain=s["gain"], eps=EPS)
        P.mx_dequantize(fmt, s["codes"], s["scales"], s["h"])
        return {"x": s["x_out"], "h": s["h"]}
    x = s["x"] + s["y"].float()
    # 64 bits: a value next to a border between two codes falls on the side the definition puts it
    z = x.double()
    h = z / torch.sqrt((z * z).mean(dim=-1, keepdim=True) + float(torch.tensor(EPS, dtype=torch.float32)))
    if s["gain"] is not None:
        h = h * s["gain"].double()
    return {"x": x, "h": _values(h, c["fmt"]).to(torch.bfloat16)}


def _run_store(s):
    c = s["case"]
    if own:
        from paper_2607_14107_amd import polestar as P
        P.mx_store_kv(s["k"], s["v"], s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], row_start=0,
                      idx=s.get("idx"), count=s.get("count"))
        P.mx_dequantize(P.MXFP4, s["k_codes"], s["k_scales"], s["k_out"])
        P.mx_dequantize(P.MXFP4, s["v_codes"], s["v_scales"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    got = {}
    b, n, G, hd, S = c["batch"], c["rows"], c["kv_heads"], c["hd"], c["seq"]
    if "idx" in s:
        used = torch.arange(n, device=DEV) < s["count"][:, None]
        at = torch.where(used, s["idx"].long(), S)                   # unused entries: a row past the end
    else:
        at = torch.arange(n, device=DEV).expand(b, n)
    for name in ("k", "v"):
        old = _read4(s[name + "_codes"], s[name + "_scales"])
        full = torch.cat((old, old.new_zeros((b, G, 1, hd))), dim=2)
        new = _values(s[name].float(), "mxfp4").permute(0, 2, 1, 3)
        full.scatter_(2, at[:, None, :, None].expand(b, G, n, hd), new)
        got[name] = full[:, :, :S].to(torch.bfloat16)
    return got


def _run_attend(s):
    c = s["case"]
    if own:
        from paper_2607_14107_amd import polestar as P
        dt = P.BF16 if c["dtype"] == "bf16" else P.FP32
        ws = _workspace(P, s, P.mx_attend_workspace_size(dt, c["batch"], c["seq"], c["heads"], c["kv_heads"], c["hd"],
                                                         c["rows"]))
        P.mx_attend(s["q"], s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], kv_len=s.get("kv_len"),
                    out=s["out"], lse=s["lse"], workspace=ws)
        return {"out": s["out"], "lse": s["lse"]}
    b, n, H, G, hd, S = (c[k] for k in ("batch", "rows", "heads", "kv_heads", "hd", "seq"))
    k, v = _read4(s["k_codes"], s["k_scales"]), _read4(s["v_codes"], s["v_scales"])
    q = s["q"].float().permute(0, 2, 1, 3).reshape(b, G, (H // G) * n, hd)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(hd)
    if "kv_len" in s:
        score = score.masked_fill(torch.arange(S, device=DEV) >= s["kv_len"][:, None, None, None], -math.inf)
    top = score.amax(dim=-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - top)
    z = p.sum(dim=-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(z > 0, z, 1.0)
    return {"out": out.reshape(b, H, n, hd).permute(0, 2, 1, 3).to(s["out"].dtype),
            "lse": (top + torch.log(z)).reshape(b, H, n)}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    c = case
    es = SIZE[c["dtype"]]
    if c["op"] == "linear":
        rows = c["batch"] * c["rows"]
        return {"bytes": rows * c["n_in"] * es + c["n_out"] * c["n_in"] * 17 / 32 + rows * c["n_out"] * es,
                "flops": 2.0 * rows * c["n_in"] * c["n_out"]}
    if c["op"] == "norm":
        n = c["batch"] * c["rows"] * c["d"]
        return {"bytes": n * (4 + es + 4 + BITS[c["fmt"]] / 8 + 1 / 32), "flops": 6.0 * n}
    kvd = c["kv_heads"] * c["hd"]
    if c["op"] == "store":
        rows = c["batch"] * c["rows"] * (0.75 if c["listed_rows"] else 1.0)
        return {"bytes": 2 * rows * kvd * (es + 17 / 32), "flops": 8.0 * rows * kvd}
    keys = c["batch"] * c["seq"] * (0.75 if c["ragged"] else 1.0)
    rows = c["batch"] * c["rows"] * c["heads"]
    return {"bytes": 2 * keys * kvd * 17 / 32 + rows * (2 * c["hd"] * es + 4),
            "flops": 4.0 * keys * c["rows"] * c["heads"] * c["hd"]}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _nearest(v, fmt):
    """v [..., n] (64 bits) on the format's grid: the nearest of its listed magnitudes, ties to the even one."""
    if fmt == "mxfp4":
        mags, emax = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], 2
    else:
        mags = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)]
        mags, emax = mags[:-1], 8                                    # the last pattern is NaN
    mags = torch.tensor(mags, dtype=torch.float64, device=v.device)
    mid = (mags[1:] + mags[:-1]) / 2
    out = []
    for rows in v.reshape(-1, v.shape[-1]).split(max(1, (1 << 25) // v.shape[-1])):
        blk = rows.reshape(rows.shape[0], -1, 32)
        amax = blk.abs().amax(dim=-1, keepdim=True)
        e = torch.floor(torch.log2(torch.where(amax > 0, amax, 1.0)))
        e = torch.where(torch.exp2(e) > amax, e - 1, torch.where(torch.exp2(e + 1) <= amax, e + 1, e)) - emax
        scale = torch.exp2(torch.where(amax > 0, e, -127.0).clamp(min=-127.0))
        a = (blk / scale).abs()
        lo = torch.bucketize(a, mid)                                 # a at a middle stays with the lower one
        tie = (lo < len(mid)) & (a == mid[lo.clamp(max=len(mid) - 1)]) & (lo % 2 == 1)
        out.append((torch.sign(blk) * mags[lo + tie.long()] * scale).reshape(rows.shape))
    return torch.cat(out).reshape(v.shape)


def _held(codes, scales):
    """Values of MXFP4 codes and scale bytes, from the bits."""
    nib = torch.stack((codes.long() % 16, codes.long() // 16), dim=-1).flatten(-2)
    ex, m = (nib // 2) % 4, (nib % 2).double()
    mag = torch.where(ex == 0, m / 2, (1 + m / 2) * torch.exp2(ex.double() - 1))
    return torch.where(nib >= 8, -mag, mag) * torch.exp2(scales.double() - 127).repeat_interleave(32, dim=-1)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] == "linear":
        x = _nearest(s["x"][:, c["start"]:c["start"] + c["rows"]].double(), c["fmt"]).reshape(-1, c["n_in"])
        y = torch.cat([x @ _held(cd, sc).t().contiguous()
                       for cd, sc in zip(s["w"][0].split(4096), s["w"][1].split(4096))], dim=1)
        return y.reshape(c["batch"], c["rows"], c["n_out"])
    if c["op"] == "norm":
        x = (s["x"] + s["y"].float()).double()                       # the stored sum, which the norm is taken of
        h = []
        for r in x.reshape(-1, c["d"]).split(2048):
            v = r * torch.rsqrt(r.square().sum(dim=-1, keepdim=True) / c["d"] + float(torch.tensor(EPS)))
            h.append(_nearest(v if s["gain"] is None else v * s["gain"].double(), c["fmt"]))
        return {"x": x, "h": torch.cat(h).reshape(x.shape)}
    if c["op"] == "store":
        got = {}
        for name in ("k", "v"):
            full = _held(s[name + "_codes"], s[name + "_scales"])
            new = _nearest(s[name].double(), "mxfp4")
            for b in range(c["batch"]):
                if "idx" in s:
                    m = int(s["count"][b])
                    full[b][:, s["idx"][b, :m].long()] = new[b, :m].transpose(0, 1)
                else:
                    full[b][:, :c["rows"]] = new[b].transpose(0, 1)
            got[name] = full
        return got
    H, G, hd = c["heads"], c["kv_heads"], c["hd"]
    out = torch.zeros((c["batch"], c["rows"], H, hd), dtype=torch.float64, device=DEV)
    lse = torch.full((c["batch"], H, c["rows"]), -math.inf, dtype=torch.float64, device=DEV)
    for b in range(c["batch"]):
        m = int(s["kv_len"][b]) if "kv_len" in s else c["seq"]
        if m == 0:
            continue
        k = _held(s["k_codes"][b, :, :m], s["k_scales"][b, :, :m])
        v = _held(s["v_codes"][b, :, :m], s["v_scales"][b, :, :m])
        for h in range(H):
            l = s["q"][b, :, h].double() @ k[h // (H // G)].t().contiguous() * hd ** -0.5
            lse[b, h] = torch.logsumexp(l, dim=-1)
            out[b, :, h] = torch.softmax(l, dim=-1) @ v[h // (H // G)]
    return {"out": out, "lse": lse}

// Products of microscaled operands (polestar_mx_linear and, after a quantization
// of the rows, polestar_mx_quantize_linear): y[r][o] = sum_i x[r][i] w[o][i].
//
// The scaled matrix instructions take 32 channels per lane and one scale for
// them, so a lane's share of a 64-channel step is one block of one row.  Operand A
// is the weights, operand B the rows, so that a lane's results are four
// neighbouring outputs of one row.
//
// fp32 outputs of MXFP8 rows are computed on bf16 instructions from the decoded
// values: the scaled instruction adds eight neighbouring products at a time with
// about 14 bits below the largest one (measured: 256 * 256 + 2^2 loses the 2^2),
// 1.5e-5 of the result's norm on normal data, which fp32 would show.  With MXFP4
// rows the products of a block span less than those bits and the sums are exact
// to fp32.
#include "host_common.hpp"
#include "mx_dev.hpp"

namespace ps {
namespace {

struct MxGemmArgs {
    const uint8_t *x, *xs, *w, *ws;
    char* y;
    long rows;
    int n_out, n_in;
};

// Operand fragments of a 64-channel step: lane l holds row l % 32, and of its
// channels the block l / 32 (h).
template <int FMT, bool DEC> struct Frag;
template <bool DEC> struct Frag<POLESTAR_MXFP4, DEC> {
    uint4 c;
    __device__ __forceinline__ void load(const uint8_t* row, int step, int h) { c = ld16(row + 32 * step + 16 * h); }
    __device__ __forceinline__ intx8 codes() const {
        return intx8{static_cast<int>(c.x), static_cast<int>(c.y), static_cast<int>(c.z), static_cast<int>(c.w), 0, 0, 0, 0};
    }
    __device__ __forceinline__ void decode(uint4* o, float sc) const {
        o[0] = mx_fp4_bf16(c.x, sc); o[1] = mx_fp4_bf16(c.y, sc);
        o[2] = mx_fp4_bf16(c.z, sc); o[3] = mx_fp4_bf16(c.w, sc);
    }
};
// 8-bit operands: the instruction's lane holds channels 16 h .. and 32 + 16 h ..
// of the step (its scale is still that of block h).
template <bool DEC> struct Frag<POLESTAR_MXFP8, DEC> {
    uint4 c[2];
    __device__ __forceinline__ void load(const uint8_t* row, int step, int h) {
        const uint8_t* p = row + 64 * step;
        c[0] = ld16(p + (DEC ? 32 * h : 16 * h));
        c[1] = ld16(p + (DEC ? 32 * h + 16 : 32 + 16 * h));
    }
    __device__ __forceinline__ intx8 codes() const {
        return intx8{static_cast<int>(c[0].x), static_cast<int>(c[0].y), static_cast<int>(c[0].z), static_cast<int>(c[0].w),
                     static_cast<int>(c[1].x), static_cast<int>(c[1].y), static_cast<int>(c[1].z), static_cast<int>(c[1].w)};
    }
    __device__ __forceinline__ void decode(uint4* o, float sc) const {
        o[0] = mx_fp8_bf16(c[0].x, c[0].y, sc); o[1] = mx_fp8_bf16(c[0].z, c[0].w, sc);
        o[2] = mx_fp8_bf16(c[1].x, c[1].y, sc); o[3] = mx_fp8_bf16(c[1].z, c[1].w, sc);
    }
};

// A wave per 32 x 32 outputs, operands straight from memory.  grid (rows / 64, n_out / 64)
template <int FMT, bool BF16>
__global__ __launch_bounds__(256) void mx_gemm_kernel(MxGemmArgs g) {
    constexpr bool DEC = FMT == POLESTAR_MXFP8 && !BF16;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int i = lane & 31, h = lane >> 5;
    const long m = static_cast<long>(blockIdx.x) * 64 + 32 * (w & 1) + i;
    const int n0 = blockIdx.y * 64 + 32 * (w >> 1);
    const long mr = min(m, g.rows - 1);                  // rows and columns past the end: the last one, not stored
    const int nr = min(n0 + i, g.n_out - 1);
    const uint8_t* xr = g.x + static_cast<size_t>(mr) * (g.n_in / 8) * Mx<FMT>::kBits;
    const uint8_t* xsr = g.xs + static_cast<size_t>(mr) * (g.n_in / 32);
    const uint8_t* wr = g.w + static_cast<size_t>(nr) * (g.n_in / 2);
    const uint8_t* wsr = g.ws + static_cast<size_t>(nr) * (g.n_in / 32);
    floatx16 acc;
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[j] = 0.f;
    for (int s = 0; s < g.n_in / 64; ++s) {
        Frag<FMT, DEC> fx;
        Frag<POLESTAR_MXFP4, DEC> fw;
        fx.load(xr, s, h);
        fw.load(wr, s, h);
        const uint32_t sx = xsr[2 * s + h], sw = wsr[2 * s + h];
        if constexpr (DEC) {
            uint4 ax[4], aw[4];
            fx.decode(ax, mx_scale(sx));
            fw.decode(aw, mx_scale(sw));
#pragma unroll
            for (int j = 0; j < 4; ++j) acc = Mma32<true>::step(aw[j], ax[j], acc);
        } else {
            acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fw.codes(), fx.codes(), acc, Mx<POLESTAR_MXFP4>::kMfma,
                                                                  Mx<FMT>::kMfma, 0, sw, 0, sx);
        }
    }
    if (m >= g.rows) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + 8 * j + 4 * h;
        if (n >= g.n_out) break;
        const size_t at = static_cast<size_t>(m) * g.n_out + n;
        if constexpr (BF16)
            *reinterpret_cast<uint2*>(g.y + 2 * at) =
                make_uint2(pack_bf16x2(acc[4 * j], acc[4 * j + 1]), pack_bf16x2(acc[4 * j + 2], acc[4 * j + 3]));
        else
            *reinterpret_cast<float4*>(g.y + 4 * at) = make_float4(acc[4 * j], acc[4 * j + 1], acc[4 * j + 2], acc[4 * j + 3]);
    }
}

bool mx_fmt_ok(int fmt) { return fmt == POLESTAR_MXFP4 || fmt == POLESTAR_MXFP8; }

size_t mx_linear_ws(int x_fmt, polestar_dtype dtype, long rows, int n_out, int n_in) { return 0; }

polestar_status mx_gemm_run(int x_fmt, polestar_dtype dtype, const MxGemmArgs& g, hipStream_t stream) {
    const dim3 grid(static_cast<unsigned>((g.rows + 63) / 64), ceil_div(g.n_out, 64));
    const bool bf16 = dtype == POLESTAR_BF16;
#define PS_GEMM(F, BF) hipLaunchKernelGGL((mx_gemm_kernel<F, BF>), grid, dim3(256), 0, stream, g)
    if (x_fmt == POLESTAR_MXFP4) { if (bf16) PS_GEMM(POLESTAR_MXFP4, true); else PS_GEMM(POLESTAR_MXFP4, false); }
    else { if (bf16) PS_GEMM(POLESTAR_MXFP8, true); else PS_GEMM(POLESTAR_MXFP8, false); }
#undef PS_GEMM
    return launch_status();
}

// Rows and outputs that the kernels' indices hold.
bool mx_shape_ok(long rows, int n_out, int n_in) {
    return n_in % 128 == 0 && n_out % 16 == 0 && rows <= (1L << 24) && n_out <= (1 << 22);
}

// Workspace of the quantized rows: codes, then scales.
size_t mx_rows_codes(int fmt, long rows, int n) { return align_up(rows * polestar_codec_row_bytes(fmt, n), 256); }
size_t mx_rows_ws(int fmt, long rows, int n) {
    return mx_rows_codes(fmt, rows, n) + align_up(static_cast<size_t>(rows) * (n / kMxBlock), 256);
}

}  // namespace
}  // namespace ps

extern "C" size_t polestar_mx_linear_workspace_size(int x_fmt, polestar_dtype dtype, long rows, int n_out, int n_in) {
    using namespace ps;
    if (!mx_fmt_ok(x_fmt) || !dtype_ok(dtype) || rows <= 0 || n_out <= 0 || n_in <= 0 || !mx_shape_ok(rows, n_out, n_in))
        return 0;
    return mx_linear_ws(x_fmt, dtype, rows, n_out, n_in);
}

extern "C" polestar_status polestar_mx_linear(int x_fmt, polestar_dtype dtype, long rows, int n_in, int n_out,
                                              const uint8_t* x_codes, const uint8_t* x_scales, const uint8_t* w_codes,
                                              const uint8_t* w_scales, void* y, void* workspace,
                                              size_t workspace_bytes, hipStream_t stream) {
    using namespace ps;
    if (!mx_fmt_ok(x_fmt) || !dtype_ok(dtype) || rows < 0 || n_in <= 0 || n_out <= 0 ||
        (rows > 0 && (!x_codes || !x_scales || !w_codes || !w_scales || !y)))
        return POLESTAR_ERR_INVALID_ARGUMENT;
    if (!mx_shape_ok(rows, n_out, n_in) || !aligned16(x_codes) || !aligned16(w_codes) || !aligned_to(x_scales, 4) ||
        !aligned_to(w_scales, 4) || !aligned16(y) || !aligned16(workspace))
        return POLESTAR_ERR_UNSUPPORTED;
    if (rows == 0) return POLESTAR_OK;
    const size_t need = mx_linear_ws(x_fmt, dtype, rows, n_out, n_in);
    if (workspace_bytes < need || (need > 0 && !workspace)) return POLESTAR_ERR_WORKSPACE;
    const MxGemmArgs g{x_codes, x_scales, w_codes, w_scales, static_cast<char*>(y), rows, n_out, n_in};
    return mx_gemm_run(x_fmt, dtype, g, stream);
}

extern "C" size_t polestar_mx_quantize_linear_workspace_size(int x_fmt, polestar_dtype dtype, int batch, int n_rows,
                                                             int n_out, int n_in) {
    using namespace ps;
    if (!mx_fmt_ok(x_fmt) || !dtype_ok(dtype) || batch <= 0 || n_rows <= 0 || n_out <= 0 || n_in <= 0) return 0;
    const long rows = static_cast<long>(batch) * n_rows;
    if (!mx_shape_ok(rows, n_out, n_in)) return 0;
    return mx_rows_ws(x_fmt, rows, n_in) + mx_linear_ws(x_fmt, dtype, rows, n_out, n_in);
}

extern "C" polestar_status polestar_mx_quantize_linear(int x_fmt, polestar_dtype dtype, int batch, int seq, int n_in,
                                                       int n_out, int row_start, int n_rows, const void* x,
                                                       const uint8_t* w_codes, const uint8_t* w_scales, void* y,
                                                       void* workspace, size_t workspace_bytes, hipStream_t stream) {
    using namespace ps;
    if (!mx_fmt_ok(x_fmt) || !dtype_ok(dtype) || batch <= 0 || seq <= 0 || n_in <= 0 || n_out <= 0 || n_rows <= 0 ||
        row_start < 0 || row_start > seq - n_rows || !x || !w_codes || !w_scales || !y)
        return POLESTAR_ERR_INVALID_ARGUMENT;
    const long rows = static_cast<long>(batch) * n_rows;
    if (!mx_shape_ok(rows, n_out, n_in) || !aligned16(x) || !aligned16(w_codes) || !aligned_to(w_scales, 4) ||
        !aligned16(y) || !aligned16(workspace) || batch > 65535)
        return POLESTAR_ERR_UNSUPPORTED;
    const size_t need = polestar_mx_quantize_linear_workspace_size(x_fmt, dtype, batch, n_rows, n_out, n_in);
    if (workspace_bytes < need || !workspace) return POLESTAR_ERR_WORKSPACE;
    uint8_t* codes = static_cast<uint8_t*>(workspace);
    uint8_t* scales = codes + mx_rows_codes(x_fmt, rows, n_in);
    const polestar_status st =
        polestar_mx_quantize(x_fmt, dtype, batch, seq, n_in, row_start, n_rows, x, codes, scales, stream);
    if (st != POLESTAR_OK) return st;
    const size_t used = mx_rows_ws(x_fmt, rows, n_in);
    return polestar_mx_linear(x_fmt, dtype, rows, n_in, n_out, codes, scales, w_codes, w_scales, y,
                              codes + used, workspace_bytes - used, stream);
}

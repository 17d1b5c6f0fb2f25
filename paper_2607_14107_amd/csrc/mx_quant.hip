// Rows into and out of the microscaling formats:
//
//   polestar_mx_quantize          rows of dtype -> codes and scales
//   polestar_mx_dequantize        codes and scales -> values
//   polestar_residual_rmsnorm_mx  residual add, RMSNorm, codes and scales
//   polestar_mx_store_kv          K/V rows -> caches held in MXFP4
//
// All are bound by the bytes they move: 12288 rows of 4096, the norm and then the
// dequantization of its MXFP8 codes, take 132 us (707 MB at 5.3 TB/s, a large copy's
// rate); 49152 rows of 128 are quantized in 4.1 to 6.0 us, about 2.5 of them the
// launch.  Eight channels per lane where a row is read once: a block is four
// neighbouring lanes, its maximum two shuffles.
#include <algorithm>

#include "host_common.hpp"
#include "mx_dev.hpp"

namespace ps {
namespace {

constexpr int kMxThreads = 256;

// One sequence's rows are one run of n8 groups of eight channels.  grid (.., batch)
template <int FMT, bool BF16>
__global__ __launch_bounds__(kMxThreads) void mx_quantize_kernel(const char* __restrict__ x, size_t seq_bytes,
                                                                 long n8, uint8_t* __restrict__ codes,
                                                                 uint8_t* __restrict__ scales) {
    constexpr int ES = Elem<BF16>::kBytes;
    const long i = static_cast<long>(blockIdx.x) * kMxThreads + threadIdx.x;
    if (i >= n8) return;                                 // whole blocks: n8 is a multiple of four
    float v[8];
    ld8<BF16>(x + blockIdx.y * seq_bytes + static_cast<size_t>(i) * 8 * ES, v);
    const uint32_t byte = mx_block_byte<FMT>(v);
    const size_t o = static_cast<size_t>(blockIdx.y) * n8 + i;
    mx_store8<FMT>(codes + o * Mx<FMT>::kBits, v, byte);
    if ((i & 3) == 0) scales[o >> 2] = static_cast<uint8_t>(byte);
}

template <int FMT, bool BF16>
__global__ __launch_bounds__(kMxThreads) void mx_dequantize_kernel(const uint8_t* __restrict__ codes,
                                                                   const uint8_t* __restrict__ scales, long n8,
                                                                   char* __restrict__ y) {
    const long i = static_cast<long>(blockIdx.x) * kMxThreads + threadIdx.x;
    if (i >= n8) return;
    const float sc = mx_scale(scales[i >> 2]);
    if constexpr (BF16) {
        uint4 o;
        if constexpr (FMT == POLESTAR_MXFP4) {
            o = mx_fp4_bf16(reinterpret_cast<const uint32_t*>(codes)[i], sc);
        } else {
            const uint2 w = reinterpret_cast<const uint2*>(codes)[i];
            o = mx_fp8_bf16(w.x, w.y, sc);
        }
        st16(y + 16 * i, o);
    } else {
        float2_hw o[4];
        if constexpr (FMT == POLESTAR_MXFP4) {
            const uint32_t w = reinterpret_cast<const uint32_t*>(codes)[i];
            o[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 0);
            o[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 1);
            o[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 2);
            o[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 3);
        } else {
            const uint2 w = reinterpret_cast<const uint2*>(codes)[i];
            o[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, sc, false);
            o[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, sc, true);
            o[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.y, sc, false);
            o[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.y, sc, true);
        }
        float4* d = reinterpret_cast<float4*>(y) + 2 * i;
        d[0] = make_float4(o[0].x, o[0].y, o[1].x, o[1].y);
        d[1] = make_float4(o[2].x, o[2].y, o[3].x, o[3].y);
    }
}

__device__ __forceinline__ double pow2(int e) { return __hiloint2double((1023 + e) << 20, 0); }
__device__ __forceinline__ int exponent_field(double v) { return (__double2hiint(v) >> 20) & 0x7ff; }

// x_out = x + y (fp32), then codes of x_out / sqrt(mean + eps) * gain.  The sum
// of squares, the norm and the rounding to the element's grid are in 64 bits: in
// 32 the last bit of the sum, which depends on its order, decides the code of
// about one channel in a million, one whole step of the grid.  A workgroup per
// row, four channels per thread and pass (eight lanes make a block).  The row is
// read once; the 64-bit work (about ten instructions a channel, at half the fp32
// rate) stays below the row's bytes.  grid rows
template <int FMT, bool BF16, int PER>
__global__ __launch_bounds__(kMxThreads) void residual_rmsnorm_mx_kernel(const float* x,
                                                                         const char* __restrict__ y,
                                                                         const float* __restrict__ gain, int d,
                                                                         float eps, float* x_out,
                                                                         uint8_t* __restrict__ codes,
                                                                         uint8_t* __restrict__ scales) {
    using F = Mx<FMT>;
    constexpr int ES = Elem<BF16>::kBytes;
    __shared__ double red[kMxThreads / kWave];
    const size_t row = static_cast<size_t>(blockIdx.x) * d;
    const float* xr = x + row;
    const char* yr = y ? y + row * ES : nullptr;
    float4 v[PER];
    double s = 0.0;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int c = 4 * (threadIdx.x + u * kMxThreads);
        v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < d) {
            v[u] = *reinterpret_cast<const float4*>(xr + c);
            if (yr) {
                float4 e;
                if constexpr (BF16) {
                    const uint2 w = *reinterpret_cast<const uint2*>(yr + 2 * c);
                    e = make_float4(bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y));
                } else {
                    e = *reinterpret_cast<const float4*>(yr + 4 * c);
                }
                v[u] = make_float4(v[u].x + e.x, v[u].y + e.y, v[u].z + e.z, v[u].w + e.w);
            }
            if (x_out) *reinterpret_cast<float4*>(x_out + row + c) = v[u];
        }
        const double a = v[u].x, b = v[u].y, e = v[u].z, f = v[u].w;
        s = fma(a, a, fma(b, b, fma(e, e, fma(f, f, s))));
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    double tot = 0.0;
#pragma unroll
    for (int w = 0; w < kMxThreads / kWave; ++w) tot += red[w];
    const double inv = 1.0 / sqrt(tot / d + static_cast<double>(eps));
    uint8_t* cr = codes + row * F::kBits / 8;
    uint8_t* sr = scales + row / kMxBlock;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int c = 4 * (threadIdx.x + u * kMxThreads);
        double z[4] = {v[u].x * inv, v[u].y * inv, v[u].z * inv, v[u].w * inv};
        if (gain && c < d) {
            const float4 g = *reinterpret_cast<const float4*>(gain + c);
            z[0] *= g.x; z[1] *= g.y; z[2] *= g.z; z[3] *= g.w;
        }
        int m = max(max(exponent_field(z[0]), exponent_field(z[1])), max(exponent_field(z[2]), exponent_field(z[3])));
#pragma unroll
        for (int o = 1; o < kMxBlock / 4; o <<= 1) m = max(m, __shfl_xor(m, o));
        if (c >= d) continue;                            // whole blocks: their eight lanes together
        const int e = min(max(m - 1023 - F::kEmax, -127), 127);
        const uint32_t byte = m == 0x7ff ? kMxNanScale : static_cast<uint32_t>(e + 127);
        const double scale = pow2(-e);
        float q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double t = z[i] * scale;
            const int step = max(exponent_field(t) - 1023, F::kEmin) - F::kMant;
            q[i] = static_cast<float>(rint(t * pow2(-step)) * pow2(step));   // exact from here on
        }
        if constexpr (FMT == POLESTAR_MXFP4) {
            const float q8[8] = {q[0], q[1], q[2], q[3], 0.f, 0.f, 0.f, 0.f};
            *reinterpret_cast<uint16_t*>(cr + c / 2) =
                byte == kMxNanScale ? 0 : static_cast<uint16_t>(mx_pack_fp4(q8, 1.f));
        } else {
            *reinterpret_cast<uint32_t*>(cr + c) = byte == kMxNanScale ? 0u : mx_pack_fp8(q, 1.f);
        }
        if ((c & (kMxBlock - 1)) == 0) sr[c / kMxBlock] = static_cast<uint8_t>(byte);
    }
}

constexpr int kMxStoreThreads = 512;                    // at most

struct StoreArgs {
    const char *k, *v;
    long row_stride;                                     // elements
    const int32_t *idx, *count;
    int row_start, n_rows, seq, heads;
    uint8_t *kc, *ks, *vc, *vs;
};

// A workgroup per row: K's channels, then V's, eight per thread and pass.  A
// listed row first looks whether a later entry names its position, so that two
// rows never mix in one.  As many threads as groups up to 512: 8 x 1536 rows of 4
// heads 7.7 us (8.4 with 256 threads, half of them idle), of 32 heads 45 (48 with 256,
// 51 with 1024), 138 listed rows of 32 heads 3.6 (4.0).  grid (n_rows, batch)
template <bool BF16, int HD>
__global__ __launch_bounds__(kMxStoreThreads) void mx_store_kv_kernel(StoreArgs a) {
    constexpr int ES = Elem<BF16>::kBytes;
    constexpr int G = HD / 8;                            // groups of eight channels in a head
    const int r = blockIdx.x, b = blockIdx.y;
    int p = a.row_start + r;
    if (a.idx) {
        const int cnt = a.count ? min(max(a.count[b], 0), a.n_rows) : a.n_rows;
        if (r >= cnt) return;
        const int32_t* list = a.idx + static_cast<size_t>(b) * a.n_rows;
        p = list[r];
        if (p < 0 || p >= a.seq) return;
        bool later = false;
        for (int i = r + 1 + threadIdx.x; i < cnt; i += blockDim.x) later |= list[i] == p;
        if (__syncthreads_or(later)) return;
    }
    const size_t row = (static_cast<size_t>(b) * a.n_rows + r) * a.row_stride * ES;
    const int n8 = a.heads * G;
    for (int i = threadIdx.x; i < 2 * n8; i += blockDim.x) {
        const bool is_v = i >= n8;
        const int j = is_v ? i - n8 : i;
        float f[8];
        ld8<BF16>((is_v ? a.v : a.k) + row + static_cast<size_t>(j) * 8 * ES, f);
        const uint32_t byte = mx_block_byte<POLESTAR_MXFP4>(f);
        const int h = j / G, g = j % G;
        const size_t at = (static_cast<size_t>(b) * a.heads + h) * a.seq + p;
        mx_store8<POLESTAR_MXFP4>((is_v ? a.vc : a.kc) + at * (HD / 2) + 4 * g, f, byte);
        if ((g & 3) == 0) (is_v ? a.vs : a.ks)[at * (HD / kMxBlock) + (g >> 2)] = static_cast<uint8_t>(byte);
    }
}

// Workgroups for n8 groups of eight channels; 0: more than a grid holds.
unsigned groups_grid(long n8) {
    const long g = (n8 + kMxThreads - 1) / kMxThreads;   // a launch has less than 2^32 threads
    return g > 0xffffffL ? 0u : static_cast<unsigned>(g);
}

}  // namespace
}  // namespace ps

extern "C" polestar_status polestar_mx_quantize(int fmt, polestar_dtype dtype, int batch, int seq, int n,
                                                int row_start, int n_rows, const void* x, uint8_t* codes,
                                                uint8_t* scales, hipStream_t stream) {
    using namespace ps;
    if (!mx_fmt_ok(fmt) || !dtype_ok(dtype) || batch <= 0 || seq <= 0 || n <= 0 || n_rows <= 0 || row_start < 0 ||
        row_start > seq - n_rows || !x || !codes || !scales)
        return POLESTAR_ERR_INVALID_ARGUMENT;
    const long n8 = static_cast<long>(n_rows) * (n / 8);
    if (n % kMxBlock || !aligned16(x) || !aligned16(codes) || batch > 65535 || groups_grid(n8) == 0)
        return POLESTAR_ERR_UNSUPPORTED;
    const size_t es = elem_bytes(dtype);
    const char* src = static_cast<const char*>(x) + static_cast<size_t>(row_start) * n * es;
    const size_t seq_bytes = static_cast<size_t>(seq) * n * es;
    const dim3 grid(groups_grid(n8), batch);
#define PS_QUANT(F, BF) \
    hipLaunchKernelGGL((mx_quantize_kernel<F, BF>), grid, dim3(kMxThreads), 0, stream, src, seq_bytes, n8, codes, scales)
    const bool bf16 = dtype == POLESTAR_BF16;
    if (fmt == POLESTAR_MXFP4) { if (bf16) PS_QUANT(POLESTAR_MXFP4, true); else PS_QUANT(POLESTAR_MXFP4, false); }
    else { if (bf16) PS_QUANT(POLESTAR_MXFP8, true); else PS_QUANT(POLESTAR_MXFP8, false); }
#undef PS_QUANT
    return launch_status();
}

extern "C" polestar_status polestar_mx_dequantize(int fmt, polestar_dtype dtype, long rows, int n,
                                                  const uint8_t* codes, const uint8_t* scales, void* y,
                                                  hipStream_t stream) {
    using namespace ps;
    if (!mx_fmt_ok(fmt) || !dtype_ok(dtype) || rows < 0 || n <= 0 || (rows > 0 && (!codes || !scales || !y)))
        return POLESTAR_ERR_INVALID_ARGUMENT;
    if (n % kMxBlock || !aligned16(codes) || !aligned16(y) || rows > 0xffffffL * kMxThreads / (n / 8))
        return POLESTAR_ERR_UNSUPPORTED;
    if (rows == 0) return POLESTAR_OK;
    const long n8 = rows * (n / 8);
    const dim3 grid(groups_grid(n8));
    char* out = static_cast<char*>(y);
#define PS_DEQUANT(F, BF) \
    hipLaunchKernelGGL((mx_dequantize_kernel<F, BF>), grid, dim3(kMxThreads), 0, stream, codes, scales, n8, out)
    const bool bf16 = dtype == POLESTAR_BF16;
    if (fmt == POLESTAR_MXFP4) { if (bf16) PS_DEQUANT(POLESTAR_MXFP4, true); else PS_DEQUANT(POLESTAR_MXFP4, false); }
    else { if (bf16) PS_DEQUANT(POLESTAR_MXFP8, true); else PS_DEQUANT(POLESTAR_MXFP8, false); }
#undef PS_DEQUANT
    return launch_status();
}

extern "C" polestar_status polestar_residual_rmsnorm_mx(int fmt, polestar_dtype dtype, long rows, int d,
                                                        const float* x, const void* y, const float* gain, float eps,
                                                        float* x_out, uint8_t* codes, uint8_t* scales,
                                                        hipStream_t stream) {
    using namespace ps;
    if (!mx_fmt_ok(fmt) || !dtype_ok(dtype) || rows < 0 || d <= 0 || !(eps >= 0.f) ||
        (rows > 0 && (!x || !codes || !scales || (y && !x_out))))
        return POLESTAR_ERR_INVALID_ARGUMENT;
    if (d % kMxBlock || d > 4 * kMxThreads * 16 || !aligned16(x) || !aligned16(y) || !aligned16(gain) ||
        !aligned16(x_out) || !aligned16(codes) || rows > 0xffffffL)
        return POLESTAR_ERR_UNSUPPORTED;
    if (rows == 0) return POLESTAR_OK;
    const dim3 grid(static_cast<unsigned>(rows));
    const int per = ceil_div(d, 4 * kMxThreads);
    const char* yc = static_cast<const char*>(y);
#define PS_NORM(F, BF, P)                                                                                        \
    hipLaunchKernelGGL((residual_rmsnorm_mx_kernel<F, BF, P>), grid, dim3(kMxThreads), 0, stream, x, yc, gain, d, \
                       eps, x_out, codes, scales)
#define PS_NORM_P(F, BF) if (per <= 4) PS_NORM(F, BF, 4); else if (per <= 8) PS_NORM(F, BF, 8); else PS_NORM(F, BF, 16)
    const bool bf16 = dtype == POLESTAR_BF16;
    if (fmt == POLESTAR_MXFP4) { if (bf16) { PS_NORM_P(POLESTAR_MXFP4, true); } else { PS_NORM_P(POLESTAR_MXFP4, false); } }
    else { if (bf16) { PS_NORM_P(POLESTAR_MXFP8, true); } else { PS_NORM_P(POLESTAR_MXFP8, false); } }
#undef PS_NORM_P
#undef PS_NORM
    return launch_status();
}

extern "C" polestar_status polestar_mx_store_kv(polestar_dtype dtype, int batch, int seq, int n_kv_heads,
                                                int head_dim, int n_rows, const void* k, const void* v,
                                                long row_stride, const int32_t* idx, const int32_t* count,
                                                int row_start, uint8_t* k_codes, uint8_t* k_scales,
                                                uint8_t* v_codes, uint8_t* v_scales, hipStream_t stream) {
    using namespace ps;
    if (!dtype_ok(dtype) || batch <= 0 || seq <= 0 || n_kv_heads <= 0 || head_dim <= 0 || n_rows < 0 ||
        row_stride < static_cast<long>(n_kv_heads) * head_dim ||
        (!idx && (row_start < 0 || row_start > seq - n_rows)) ||
        (n_rows > 0 && (!k || !v || !k_codes || !k_scales || !v_codes || !v_scales)))
        return POLESTAR_ERR_INVALID_ARGUMENT;
    if ((head_dim != 64 && head_dim != 128) || !row_ok(dtype, row_stride) || !aligned16(k) || !aligned16(v) ||
        !aligned16(k_codes) || !aligned16(v_codes) || !aligned_to(k_scales, head_dim / kMxBlock) ||
        !aligned_to(v_scales, head_dim / kMxBlock) || batch > 65535 || n_kv_heads > 65535 || n_rows > 0x7fffff)
        return POLESTAR_ERR_UNSUPPORTED;
    if (n_rows == 0) return POLESTAR_OK;
    const StoreArgs a{static_cast<const char*>(k), static_cast<const char*>(v), row_stride, idx, count, row_start,
                      n_rows, seq, n_kv_heads, k_codes, k_scales, v_codes, v_scales};
    const dim3 grid(n_rows, batch), block(std::min(kMxStoreThreads, ceil_div(n_kv_heads * (head_dim / 4), kWave) * kWave));
#define PS_STORE(BF, HD) hipLaunchKernelGGL((mx_store_kv_kernel<BF, HD>), grid, block, 0, stream, a)
    if (dtype == POLESTAR_BF16) { if (head_dim == 128) PS_STORE(true, 128); else PS_STORE(true, 64); }
    else { if (head_dim == 128) PS_STORE(false, 128); else PS_STORE(false, 64); }
#undef PS_STORE
    return launch_status();
}

// Attention over K/V caches held in MXFP4 (polestar_mx_attend).
//
// A wave takes 32 query vectors of one KV head (every query head that shares it,
// every row) and 32 keys at a time: S^T = K Q^T on v_mfma_f32_32x32x16_bf16, the
// keys' codes decoded to bf16 in registers (exact: three significant bits times a
// power of two), an online softmax in base 2 per query (a lane pair), and O^T +=
// V^T P^T, where S^T's result registers are P^T's operand registers.  V's codes
// are decoded on their way into LDS and read back transposed
// (ds_read_b64_tr_b16: four keys of one channel per lane).
//
// fp32 queries: q and p are taken as three bf16 terms each, so that the products
// with the exact keys and values keep 24 bits.
#include "host_common.hpp"
#include "mx_dev.hpp"

namespace ps {
namespace {

constexpr int kMxAttWaves = 4;
constexpr int kMxAttThreads = kMxAttWaves * kWave;
constexpr int kMxKeys = 32;                              // keys of a wave's step
constexpr int kMxQ = 32;                                 // query vectors of a workgroup

typedef short shortx4 __attribute__((ext_vector_type(4)));

struct MxAttArgs {
    const char* q;
    long q_stride;                                       // elements
    const uint8_t *kc, *ks, *vc, *vs;
    const int32_t* kv_len;
    char* out;
    float* lse;
    float scale2;                                        // scale * log2(e)
    int seq, n_rows, heads, kv_heads, tiles;             // tiles: query tiles of a KV head
};

// Four keys of one channel: lane i of 16 gives the address of four channels of
// key i / 4 and gets channel i of the four keys.
__device__ __forceinline__ uint2 lds_read_tr(const char* p) {
    auto q = (__attribute__((address_space(3))) shortx4*)(p);
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(q));
}

// v as NT bf16 terms whose sum has 8 NT bits of it.
template <int NT>
__device__ __forceinline__ void split_bf16(const float* v, uint4* o) {
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = v[i];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        o[t] = make_uint4(cvt_pk_bf16(r[0], r[1]), cvt_pk_bf16(r[2], r[3]), cvt_pk_bf16(r[4], r[5]),
                          cvt_pk_bf16(r[6], r[7]));
        if (t + 1 < NT) {
            float h[8];
            Elem<true>::unpack(o[t], h);
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] -= h[i];
        }
    }
}

// grid (tiles * kv_heads, batch)
template <bool BF16, int HD>
__global__ __launch_bounds__(kMxAttThreads) void mx_attend_kernel(MxAttArgs a) {
    constexpr int NT = BF16 ? 1 : 3;
    constexpr int ES = Elem<BF16>::kBytes;
    constexpr int NC = HD / 64;                          // 16-byte chunks of a key per lane
    constexpr int CT = HD / 32;                          // channel tiles
    constexpr int kPitch = 2 * HD + 64;                  // bytes of a key's row in LDS
    __shared__ __align__(16) char vbuf[kMxAttWaves][kMxKeys * kPitch];
    __shared__ float sm[kMxAttWaves][kMxQ], sl[kMxAttWaves][kMxQ];
    __shared__ __align__(16) float so[kMxQ][HD + 4];

    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int i = lane & 31, h = lane >> 5;
    const int b = blockIdx.y, g = blockIdx.x / a.tiles, qt = blockIdx.x % a.tiles;
    const int group = a.heads / a.kv_heads;
    const int len = a.kv_len ? min(max(a.kv_len[b], 0), a.seq) : a.seq;
    const int nq = group * a.n_rows;
    const int qv = qt * kMxQ + i;
    const int qc = min(qv, nq - 1);                      // past the end: the last one, not stored
    const int head = g * group + qc / a.n_rows, row = qc % a.n_rows;

    uint4 q[NC][4][NT];
    {
        const char* p = a.q + ((static_cast<size_t>(b) * a.n_rows + row) * a.q_stride + static_cast<size_t>(head) * HD) * ES;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const char* s = p + (32 * (2 * c + h) + 8 * t) * ES;
                if constexpr (BF16) {
                    q[c][t][0] = ld16(s);
                } else {
                    float v[8];
                    ld8<false>(s, v);
                    split_bf16<NT>(v, q[c][t]);
                }
            }
    }
    const size_t first = (static_cast<size_t>(b) * a.kv_heads + g) * a.seq;   // the head's first key
    const uint8_t* kc = a.kc + first * (HD / 2);
    const uint8_t* ks = a.ks + first * (HD / kMxBlock);
    const uint8_t* vc = a.vc + first * (HD / 2);
    const uint8_t* vs = a.vs + first * (HD / kMxBlock);

    floatx16 o[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[c][j] = 0.f;
    float m = -INFINITY, l = 0.f;
    char* vb = vbuf[w];
    for (int k0 = w * kMxKeys; k0 < len; k0 += kMxAttWaves * kMxKeys) {
        // V: lane (key, chunk) decodes 32 channels into LDS
#pragma unroll
        for (int u = 0; u < kMxKeys * CT / kWave; ++u) {
            const int at = u * kWave + lane, key = at / CT, c = at % CT;
            const bool in = k0 + key < len;
            const size_t kr = min(k0 + key, len - 1);
            const uint4 code = ld16(vc + kr * (HD / 2) + 16 * c);
            const float sc = in ? mx_scale(vs[kr * (HD / kMxBlock) + c]) : 1.f;
            const uint32_t keep = in ? ~0u : 0u;         // keys past the end hold anything, also NaN
            char* d = vb + key * kPitch + 64 * c;
            st16(d, mx_fp4_bf16(code.x & keep, sc));
            st16(d + 16, mx_fp4_bf16(code.y & keep, sc));
            st16(d + 32, mx_fp4_bf16(code.z & keep, sc));
            st16(d + 48, mx_fp4_bf16(code.w & keep, sc));
        }
        floatx16 s;
#pragma unroll
        for (int j = 0; j < 16; ++j) s[j] = 0.f;
        const size_t kr = min(k0 + i, len - 1);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const uint4 code = ld16(kc + kr * (HD / 2) + 16 * (2 * c + h));
            const float sc = mx_scale(ks[kr * (HD / kMxBlock) + 2 * c + h]);
            const uint32_t cw[4] = {code.x, code.y, code.z, code.w};
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint4 kf = mx_fp4_bf16(cw[t], sc);
#pragma unroll
                for (int n = 0; n < NT; ++n) s = Mma32<true>::step(kf, q[c][t][n], s);
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const bool in = k0 + 8 * (j >> 2) + 4 * h + (j & 3) < len;
            s[j] = in ? s[j] * a.scale2 : -INFINITY;
            top = fmaxf(top, s[j]);
        }
        top = fmaxf(top, __shfl_xor(top, 32));
        const float mn = fmaxf(m, top);
        const float ref = mn == -INFINITY ? 0.f : mn;
        const float f = fast_exp2(m - ref);
        m = mn;
        float sum = 0.f;
        float p[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            p[j] = fast_exp2(s[j] - ref);
            sum += p[j];
        }
        l = l * f + sum;                                 // of this lane's keys
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[c][j] *= f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uint4 pt[NT];
            split_bf16<NT>(p + 8 * u, pt);
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                // channel 32 c + i; keys 16 u + 4 h + 0..3 and 8 further on, as p's registers
                const char* s0 = vb + (16 * u + 4 * h + ((lane & 15) >> 2)) * kPitch + 64 * c +
                                 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
                const uint2 v0 = lds_read_tr(s0), v1 = lds_read_tr(s0 + 8 * kPitch);
                const uint4 vf = make_uint4(v0.x, v0.y, v1.x, v1.y);
#pragma unroll
                for (int n = 0; n < NT; ++n) o[c] = Mma32<true>::step(vf, pt[n], o[c]);
            }
        }
    }
    l += __shfl_xor(l, 32);
    if (h == 0) {
        sm[w][i] = m;
        sl[w][i] = l;
    }
    __syncthreads();
    float mt = -INFINITY, lt = 0.f;
#pragma unroll
    for (int x = 0; x < kMxAttWaves; ++x) mt = fmaxf(mt, sm[x][i]);
    const float ref = mt == -INFINITY ? 0.f : mt;
#pragma unroll
    for (int x = 0; x < kMxAttWaves; ++x) lt += sl[x][i] * fast_exp2(sm[x][i] - ref);
    const float f = fast_exp2(m - ref);
    // the waves' O, one after another
    for (int x = 0; x < kMxAttWaves; ++x) {
        if (x == w) {
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float4* d = reinterpret_cast<float4*>(&so[i][32 * c + 8 * j + 4 * h]);
                    float4 v = make_float4(o[c][4 * j] * f, o[c][4 * j + 1] * f, o[c][4 * j + 2] * f, o[c][4 * j + 3] * f);
                    if (x > 0) {
                        const float4 e = *d;
                        v = make_float4(v.x + e.x, v.y + e.y, v.z + e.z, v.w + e.w);
                    }
                    *d = v;
                }
        }
        __syncthreads();
    }
    // an empty sequence: zeros
    if (threadIdx.x < kMxQ && qv < nq && a.lse)
        a.lse[(static_cast<size_t>(b) * a.heads + head) * a.n_rows + row] = (mt + __log2f(lt)) * kLn2;
    for (int x = threadIdx.x; x < kMxQ * HD / 8; x += kMxAttThreads) {
        const int r = x / (HD / 8), c = (x % (HD / 8)) * 8;
        const int qx = qt * kMxQ + r;
        if (qx >= nq) continue;
        float lq = 0.f, mq = -INFINITY;
        for (int y = 0; y < kMxAttWaves; ++y) mq = fmaxf(mq, sm[y][r]);
        const float rq = mq == -INFINITY ? 0.f : mq;
        for (int y = 0; y < kMxAttWaves; ++y) lq += sl[y][r] * fast_exp2(sm[y][r] - rq);
        const float inv = len > 0 ? 1.f / lq : 0.f;
        const size_t at = ((static_cast<size_t>(b) * a.n_rows + qx % a.n_rows) * a.heads + g * group + qx / a.n_rows) * HD + c;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = len > 0 ? so[r][c + e] * inv : 0.f;
        if constexpr (BF16) {
            st16(a.out + 2 * at, make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                                            pack_bf16x2(v[6], v[7])));
        } else {
            *reinterpret_cast<float4*>(a.out + 4 * at) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(a.out + 4 * at + 16) = make_float4(v[4], v[5], v[6], v[7]);
        }
    }
}

}  // namespace
}  // namespace ps

extern "C" size_t polestar_mx_attend_workspace_size(polestar_dtype dtype, int batch, int seq, int n_heads,
                                                    int n_kv_heads, int head_dim, int n_rows) {
    using namespace ps;
    return 0;
}

extern "C" polestar_status polestar_mx_attend(polestar_dtype dtype, int batch, int seq, int n_heads, int n_kv_heads,
                                              int head_dim, int n_rows, const void* q, long q_stride,
                                              const uint8_t* k_codes, const uint8_t* k_scales, const uint8_t* v_codes,
                                              const uint8_t* v_scales, const int32_t* kv_len, float scale, void* out,
                                              float* lse, void* workspace, size_t workspace_bytes,
                                              hipStream_t stream) {
    using namespace ps;
    if (!dtype_ok(dtype) || batch <= 0 || seq <= 0 || n_heads <= 0 || n_kv_heads <= 0 || head_dim <= 0 || n_rows <= 0 ||
        n_heads % n_kv_heads != 0 || q_stride < static_cast<long>(n_heads) * head_dim || !q || !k_codes || !k_scales ||
        !v_codes || !v_scales || !out)
        return POLESTAR_ERR_INVALID_ARGUMENT;
    const long nq = static_cast<long>(n_heads / n_kv_heads) * n_rows;
    const long tiles = (nq + kMxQ - 1) / kMxQ;
    if ((head_dim != 64 && head_dim != 128) || !row_ok(dtype, q_stride) || !aligned16(q) || !aligned16(k_codes) ||
        !aligned16(v_codes) || !aligned_to(k_scales, head_dim / kMxBlock) || !aligned_to(v_scales, head_dim / kMxBlock) ||
        !aligned16(out) || !aligned16(workspace) || batch > 65535 || tiles * n_kv_heads > 0xffffff)
        return POLESTAR_ERR_UNSUPPORTED;
    const size_t need = polestar_mx_attend_workspace_size(dtype, batch, seq, n_heads, n_kv_heads, head_dim, n_rows);
    if (workspace_bytes < need || (need > 0 && !workspace)) return POLESTAR_ERR_WORKSPACE;
    if (!(scale > 0.f)) scale = 1.f / sqrtf(static_cast<float>(head_dim));
    const MxAttArgs a{static_cast<const char*>(q), q_stride, k_codes, k_scales, v_codes, v_scales, kv_len,
                      static_cast<char*>(out), lse, scale * kLog2e, seq, n_rows, n_heads, n_kv_heads,
                      static_cast<int>(tiles)};
    const dim3 grid(static_cast<unsigned>(tiles * n_kv_heads), batch);
#define PS_ATT(BF, HD) hipLaunchKernelGGL((mx_attend_kernel<BF, HD>), grid, dim3(kMxAttThreads), 0, stream, a)
    if (dtype == POLESTAR_BF16) { if (head_dim == 128) PS_ATT(true, 128); else PS_ATT(true, 64); }
    else { if (head_dim == 128) PS_ATT(false, 128); else PS_ATT(false, 64); }
#undef PS_ATT
    return launch_status();
}

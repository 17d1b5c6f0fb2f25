// Attention over K/V caches held in MXFP4 (polestar_mx_attend).
//
// A wave takes 32 query vectors of one KV head (every query head that shares it,
// every row) and 32 keys at a time: S^T = K Q^T on v_mfma_f32_32x32x16_bf16, the
// keys' codes decoded to bf16 in registers (exact: three significant bits times a
// power of two), an online softmax in base 2 per query (a lane pair), and O^T +=
// V^T P^T, where S^T's result registers are P^T's operand registers.  V's codes
// are decoded on their way into LDS and read back transposed
// (ds_read_b64_tr_b16: four keys of one channel per lane).  The next step's codes
// are loaded before this step's work.
//
// The waves of a workgroup take the steps in turn, and where the workgroups do not
// fill the GPU the keys are split over several; each part's (reference, sum, O) are
// joined at the end, in LDS and by a second kernel.  In LDS every wave puts its part
// down at once and every thread sums its share of the queries' channels behind one
// barrier: added in pairs with a barrier each, the join took 0.5 to 1.5 us more.
//
// Measured inside a graph, head_dim 128, bf16: 8 x 32 heads, 1 query: 256 keys 5.6
// us, 2048 keys 15.3, 8192 keys 54 to 65 (its 285 MB at 4.4 to 5.3 TB/s); 4 x 4 KV
// heads, 448 queries each: 1024 keys 11.3 us, 8192 keys 47.  Long caches of few queries
// are bound by memory.  Many queries saturate no unit: of a compute unit's time with
// two waves per SIMD the vector units are active in 46% (187 instructions for the 16
// matrix instructions of a step, 64 of them the codes' decoding, which every tile of
// 32 queries repeats), the matrix units in 21%, and waves wait in 41% of theirs.
// Computing the next step's scores beside this step's softmax was 5% slower, twelve
// waves or two steps of prefetch no faster, nor was an order that keeps a head's query
// tiles on one XCD.
//
// bf16 queries: the probabilities are rounded to bf16 for the second product, as in
// polestar_attend, and their sum is taken before.  The rounding is at most 2^-8 of a
// probability; outputs of 64 to 32768 keys were 0.0021 to 0.0023 of their norm off the
// 64-bit result, 0.0017 of that their own rounding.  A second term would double the
// second product and add 16 vector instructions to a step.
//
// fp32 queries: q and p are taken as three bf16 terms each, so that the products
// with the exact keys and values keep 24 bits.
#include <algorithm>

#include "host_common.hpp"
#include "mx_dev.hpp"

namespace ps {
namespace {

constexpr int kMxKeys = 32;                              // keys of a wave's step
constexpr int kMxQ = 32;                                 // query vectors of a workgroup
constexpr int kMxMaxSplits = 64;                         // a lane each in the merge
constexpr int kMxMaxSeq = 1 << 24;                       // a head's codes: offsets of 32 bits
constexpr float kMxSlack = 8.f;                          // see the softmax

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
    int splits;
    float* part;                                         // [batch][kv head][split][query][HD] O, then
    float2* ml;                                          // [batch][kv head][split][query] (reference, sum)
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

// V's rows in LDS: 2 HD bytes of a key and 64 more, and within each 64 bytes (the
// 32 channels that a lane decodes) the 16-byte chunks XORed by v_swizzle(key), so
// that the lanes whose stores run together, and the eight rows of a transposed
// read, lie in different banks.  (Conflicts are 31% of the LDS cycles with it and half
// without.)
template <int HD> __device__ __forceinline__ int v_swizzle(int key) { return (HD == 128 ? key : key ^ (key >> 2)) & 3; }

// A head's keys or values: buffers that end with the sequence's last key, so that
// what lies behind it (which may hold anything) reads as 0.
typedef __amdgpu_buffer_rsrc_t KvBuffer;
__device__ __forceinline__ KvBuffer kv_buffer(const uint8_t* base, size_t off, uint32_t bytes) {
    const uint64_t p = reinterpret_cast<uint64_t>(base) + off;
    const uint64_t u = static_cast<uint64_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p >> 32))) << 32 |
                       static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p)));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(u), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00027000);
}

// The codes of a step's 32 keys: lane (key i, half h) holds half of key i's, and of
// V's rows the chunks that it will decode.
template <int HD> struct KvStep {
    static constexpr int CT = HD / 32, NC = HD / 64, VU = HD / 64;
    uint4 k[NC], v[VU];
    uint32_t ks, vs[VU];
    __device__ __forceinline__ void load(KvBuffer kc, KvBuffer kss, KvBuffer vc, KvBuffer vss, int k0, int lane) {
        const int i = lane & 31, h = lane >> 5;
#pragma unroll
        for (int c = 0; c < NC; ++c)
            k[c] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(kc, i * (HD / 2) + 16 * h, k0 * (HD / 2) + 32 * c, 0));
        if constexpr (HD == 128) ks = __builtin_amdgcn_raw_buffer_load_b32(kss, i * CT, k0 * CT, 0);
        else ks = __builtin_amdgcn_raw_buffer_load_b16(kss, i * CT, k0 * CT, 0);
#pragma unroll
        for (int u = 0; u < VU; ++u) {
            v[u] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(vc, 16 * lane, k0 * (HD / 2) + 16 * kWave * u, 0));
            vs[u] = __builtin_amdgcn_raw_buffer_load_b8(vss, lane, k0 * CT + kWave * u, 0);
        }
    }
};

// The larger of a lane's value and that of the lane 32 away.
__device__ __forceinline__ float max_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// grid (tiles * kv_heads, splits, batch), NW waves
template <bool BF16, int HD, int NW>
__global__ __launch_bounds__(NW * kWave) void mx_attend_kernel(MxAttArgs a) {
    constexpr int NT = BF16 ? 1 : 3;
    constexpr int ES = Elem<BF16>::kBytes;
    constexpr int NC = HD / 64;                          // 16-byte chunks of a key per lane
    constexpr int CT = HD / 32;                          // channel tiles
    constexpr int kPitch = 2 * HD + 64;                  // bytes of a key's row in LDS
    constexpr int kOPitch = 4 * HD + 16;                 // of a query's O
    constexpr int kV = kMxKeys * kPitch, kO = kMxQ * kOPitch, kPart = kV > kO ? kV : kO;   // of a wave: V's rows, then O
    __shared__ __align__(16) char lds[NW * kPart];
    __shared__ float sm[NW][kMxQ], sl[NW][kMxQ];

    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 31, h = lane >> 5;
    const int b = blockIdx.z, g = blockIdx.x / a.tiles, qt = blockIdx.x % a.tiles, split = blockIdx.y;
    const int group = a.heads / a.kv_heads;
    const int len = a.kv_len ? min(max(a.kv_len[b], 0), a.seq) : a.seq;
    const int nq = group * a.n_rows;
    const int qv = qt * kMxQ + i;
    const int qc = min(qv, nq - 1);                      // past the end: the last one, not stored
    const int head = g * group + qc / a.n_rows, row = qc % a.n_rows;
    // this split's steps, of the sequence's own length
    const int steps = (len + kMxKeys - 1) / kMxKeys, per = (steps + a.splits - 1) / a.splits;
    const int s0 = min(split * per, steps), s1 = min(s0 + per, steps);

    const size_t first = (static_cast<size_t>(b) * a.kv_heads + g) * a.seq;   // the head's first key
    const KvBuffer kc = kv_buffer(a.kc, first * (HD / 2), len * (HD / 2)), ks = kv_buffer(a.ks, first * CT, len * CT);
    const KvBuffer vc = kv_buffer(a.vc, first * (HD / 2), len * (HD / 2)), vs = kv_buffer(a.vs, first * CT, len * CT);
    KvStep<HD> even, odd;                                // this step's codes and the next one's, in turn
    even.load(kc, ks, vc, vs, (s0 + w) * kMxKeys, lane);

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
    floatx16 o[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[c][j] = 0.f;
    float m = -INFINITY, l = 0.f;                        // the exponents' reference; l of this lane's keys
    char* vb = lds + w * kPart;
    // transposed reads: keys 4 h + 0..3 and 8 further on
    const int tk = 4 * h + ((lane & 15) >> 2), tq = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    const int tr0 = tk * kPitch + 16 * (tq ^ v_swizzle<HD>(tk)) + 8 * (lane & 1);
    const int tr1 = (tk + 8) * kPitch + 16 * (tq ^ v_swizzle<HD>(tk + 8)) + 8 * (lane & 1);
    auto step = [&](int st, const KvStep<HD>& cur) {
        const int k0 = st * kMxKeys;
        // V: lane (key, chunk) decodes 32 channels into LDS
#pragma unroll
        for (int u = 0; u < KvStep<HD>::VU; ++u) {
            const int at = u * kWave + lane, key = at / CT, c = at % CT;
            const uint4 code = cur.v[u];
            const float sc = mx_scale(cur.vs[u]);
            char* d = vb + key * kPitch + 64 * c;
            const int z = 16 * v_swizzle<HD>(key);
            st16(d + z, mx_fp4_bf16(code.x, sc));
            st16(d + (z ^ 16), mx_fp4_bf16(code.y, sc));
            st16(d + (z ^ 32), mx_fp4_bf16(code.z, sc));
            st16(d + (z ^ 48), mx_fp4_bf16(code.w, sc));
        }
        floatx16 s;
#pragma unroll
        for (int j = 0; j < 16; ++j) s[j] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const float sc = mx_scale((cur.ks >> (8 * (2 * c + h))) & 255u);
            const uint32_t cw[4] = {cur.k[c].x, cur.k[c].y, cur.k[c].z, cur.k[c].w};
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint4 kf = mx_fp4_bf16(cw[t], sc);
#pragma unroll
                for (int n = 0; n < NT; ++n) s = Mma32<true>::step(kf, q[c][t][n], s);
            }
        }
        if (k0 + kMxKeys > len) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (k0 + mfma32_row(lane, j) >= len) s[j] = -INFINITY;
        }
        // The reference moves only when a query's largest score passes it by more than
        // kMxSlack (exponents stay below 2^8, and (m, l, O) are exact for any
        // reference), so that O is rarely rescaled.
        float top = s[0];
#pragma unroll
        for (int j = 1; j < 16; ++j) top = fmaxf(top, s[j]);
        top = max_halves(top) * a.scale2;
        if (__builtin_amdgcn_ballot_w64(top > m + kMxSlack || m == -INFINITY) != 0) {
            const float mn = fmaxf(m, top);
            const float f = fast_exp2(m - (mn == -INFINITY ? 0.f : mn));
            m = mn;
            l *= f;
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[c][j] *= f;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        float p[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) p[j] = fast_exp2(fmaf(s[j], a.scale2, -ref));
#pragma unroll
        for (int j = 0; j < 16; j += 4) l += (p[j] + p[j + 1]) + (p[j + 2] + p[j + 3]);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uint4 pt[NT];
            split_bf16<NT>(p + 8 * u, pt);
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                // channel 32 c + i; keys 16 u + 4 h + 0..3 and 8 further on, as p's registers
                const uint2 x = lds_read_tr(vb + tr0 + 16 * u * kPitch + 64 * c);
                const uint2 y = lds_read_tr(vb + tr1 + 16 * u * kPitch + 64 * c);
                const uint4 vf = make_uint4(x.x, x.y, y.x, y.y);
#pragma unroll
                for (int n = 0; n < NT; ++n) o[c] = Mma32<true>::step(vf, pt[n], o[c]);
            }
        }
    };
    // (the queries' loads end here: inside the loop the wait for them would be one
    // for the next step's codes)
    __builtin_amdgcn_s_waitcnt(0);
    for (int st = s0 + w; st < s1; st += 2 * NW) {
        odd.load(kc, ks, vc, vs, (st + NW) * kMxKeys, lane);
        step(st, even);
        if (st + NW >= s1) break;
        even.load(kc, ks, vc, vs, (st + 2 * NW) * kMxKeys, lane);
        step(st + NW, odd);
    }
    // the waves' parts, (reference, sum, O) each, joined by every thread for its share
    l += __shfl_xor(l, 32);
    if (h == 0) {
        sm[w][i] = m;
        sl[w][i] = l;
    }
    // (V's rows lie in the wave's own part, so no barrier is needed before)
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            *reinterpret_cast<float4*>(lds + w * kPart + i * kOPitch + (32 * c + 8 * j + 4 * h) * 4) =
                make_float4(o[c][4 * j], o[c][4 * j + 1], o[c][4 * j + 2], o[c][4 * j + 3]);
    __syncthreads();
    const size_t slot = ((static_cast<size_t>(b) * a.kv_heads + g) * a.splits + split) * nq;
    for (int x = threadIdx.x; x < kMxQ * HD / 8; x += NW * kWave) {
        const int rq = x / (HD / 8), c = (x % (HD / 8)) * 8;
        const int qx = qt * kMxQ + rq;
        if (qx >= nq) continue;
        float mt = -INFINITY, lt = 0.f, f[NW];
#pragma unroll
        for (int y = 0; y < NW; ++y) mt = fmaxf(mt, sm[y][rq]);
        const float ref = mt == -INFINITY ? 0.f : mt;
#pragma unroll
        for (int y = 0; y < NW; ++y) {
            f[y] = fast_exp2(sm[y][rq] - ref);
            lt += sl[y][rq] * f[y];
        }
        float v[8] = {};
#pragma unroll
        for (int y = 0; y < NW; ++y) {
            const float4* src = reinterpret_cast<const float4*>(lds + y * kPart + rq * kOPitch + 4 * c);
            const float4 d = src[0], e = src[1];
            v[0] = fmaf(d.x, f[y], v[0]); v[1] = fmaf(d.y, f[y], v[1]); v[2] = fmaf(d.z, f[y], v[2]); v[3] = fmaf(d.w, f[y], v[3]);
            v[4] = fmaf(e.x, f[y], v[4]); v[5] = fmaf(e.y, f[y], v[5]); v[6] = fmaf(e.z, f[y], v[6]); v[7] = fmaf(e.w, f[y], v[7]);
        }
        const int hx = g * group + qx / a.n_rows, rx = qx % a.n_rows;
        if (a.splits > 1) {
            float4* d = reinterpret_cast<float4*>(a.part + (slot + qx) * HD + c);
            d[0] = make_float4(v[0], v[1], v[2], v[3]);
            d[1] = make_float4(v[4], v[5], v[6], v[7]);
            if (c == 0) a.ml[slot + qx] = make_float2(mt, lt);
            continue;
        }
        // an empty sequence: zeros; no finite score: NaN, as the quotient
        const float inv = len > 0 ? 1.f / lt : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= inv;
        const size_t at = ((static_cast<size_t>(b) * a.n_rows + rx) * a.heads + hx) * HD + c;
        if constexpr (BF16) {
            st16(a.out + 2 * at, make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                                            pack_bf16x2(v[6], v[7])));
        } else {
            *reinterpret_cast<float4*>(a.out + 4 * at) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(a.out + 4 * at + 16) = make_float4(v[4], v[5], v[6], v[7]);
        }
        if (a.lse && c == 0) a.lse[(static_cast<size_t>(b) * a.heads + hx) * a.n_rows + rx] = (mt + __log2f(lt)) * kLn2;
    }
}

// The splits' parts of a query vector: lane s weighs split s, then every wave adds
// its share of the splits, all of its loads in flight (one after another, they took
// 10 us for 32 splits).  grid (queries, kv_heads, batch), NW waves
template <bool BF16, int HD, int NW>
__global__ __launch_bounds__(NW * kWave) void mx_attend_merge_kernel(MxAttArgs a) {
    constexpr int ES = Elem<BF16>::kBytes, CH = HD / kWave;
    constexpr int U = kMxMaxSplits / 4 / (NW == 1 ? 2 : 1);   // splits of a wave: NW = 1 takes up to 8
    __shared__ float red[NW][HD];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int group = a.heads / a.kv_heads, nq = group * a.n_rows;
    const int qv = blockIdx.x, g = blockIdx.y, b = blockIdx.z;
    const size_t slot = (static_cast<size_t>(b) * a.kv_heads + g) * a.splits * nq + qv;
    float2 e = make_float2(-INFINITY, 0.f);
    if (lane < a.splits) e = a.ml[slot + static_cast<size_t>(lane) * nq];
    float p[U][CH];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int s = w + u * NW;
        const float* src = a.part + (slot + static_cast<size_t>(s) * nq) * HD + lane * CH;
#pragma unroll
        for (int c = 0; c < CH; ++c) p[u][c] = s < a.splits ? src[c] : 0.f;
    }
    const float m = wave_max(e.x);
    const float wgt = fast_exp2(e.x - (m == -INFINITY ? 0.f : m));
    const float l = wave_sum(e.y * wgt);
    float v[CH] = {};
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const float ws = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(wgt), w + u * NW));
#pragma unroll
        for (int c = 0; c < CH; ++c) v[c] = fmaf(p[u][c], ws, v[c]);
    }
    if constexpr (NW > 1) {
#pragma unroll
        for (int c = 0; c < CH; ++c) red[w][lane * CH + c] = v[c];
        __syncthreads();
        if (w > 0) return;
#pragma unroll
        for (int x = 1; x < NW; ++x)
#pragma unroll
            for (int c = 0; c < CH; ++c) v[c] += red[x][lane * CH + c];
    }
    const bool any = a.kv_len == nullptr || a.kv_len[b] > 0;
    const int head = g * group + qv / a.n_rows, row = qv % a.n_rows;
    char* d = a.out + (((static_cast<size_t>(b) * a.n_rows + row) * a.heads + head) * HD + lane * CH) * ES;
#pragma unroll
    for (int c = 0; c < CH; ++c) v[c] = any ? v[c] / l : 0.f;
    if constexpr (BF16 && CH == 2) *reinterpret_cast<uint32_t*>(d) = pack_bf16x2(v[0], v[1]);
    else if constexpr (BF16) *reinterpret_cast<uint16_t*>(d) = static_cast<uint16_t>(f32_to_bf16_bits(v[0]));
    else
#pragma unroll
        for (int c = 0; c < CH; ++c) reinterpret_cast<float*>(d)[c] = v[c];
    if (a.lse && lane == 0) a.lse[(static_cast<size_t>(b) * a.heads + head) * a.n_rows + row] = (m + __log2f(l)) * kLn2;
}

// Waves per workgroup and key splits: eight waves where the workgroups are at most the
// compute units and each wave has two steps (the registers allow two waves on each
// SIMD), and then as many splits as fill the units in one round, while a wave keeps two
// steps.  In a graph, us: one token of two sequences over 32768 keys, 4 KV heads (8
// workgroups): 131 unsplit, 24 with 8 splits, 17.4 with 16, 16.4 with 32 (chosen), 19.0
// with 64.  More splits than one round holds do not pay: 160 workgroups of 4096 keys 22
// to 24 unsplit (chosen), 34 with 2, 31 with 3; 240 of 4096 keys 28, 36, 40; 256 of 8192
// keys 54, 61.  What the rule leaves: 160 workgroups of 16384 keys 78 to 89 unsplit, 70
// with 3 splits (132: 73 to 75, 67), and, since the host does not know the lengths, one
// sequence of 8192 keys among 512s, 256 workgroups: 37.5 unsplit, 26.6 with 4 splits.
struct MxAttPlan {
    int tiles, waves, splits;
    size_t part, total;                                  // bytes: O parts, with the sums
};
MxAttPlan mx_att_plan(int batch, int seq, int heads, int kv_heads, int hd, int n_rows) {
    MxAttPlan p{};
    const long nq = static_cast<long>(heads / kv_heads) * n_rows;
    p.tiles = ceil_div(nq, kMxQ);
    const long wgs = static_cast<long>(batch) * kv_heads * p.tiles;
    const int steps = ceil_div(seq, kMxKeys);
    p.waves = steps >= 16 && wgs <= 256 ? 8 : 4;
    p.splits = p.waves == 8 ? static_cast<int>(std::min({256 / wgs, steps / 16L, static_cast<long>(kMxMaxSplits)})) : 1;
    if (p.splits > 1) {
        const size_t rows = static_cast<size_t>(batch) * kv_heads * p.splits * nq;
        p.part = align_up(rows * hd * sizeof(float), 256);
        p.total = p.part + rows * sizeof(float2);
    }
    return p;
}

// Sizes that the kernels' indices, and the plan's numbers, hold (all positive).
bool mx_att_shape_ok(int batch, int seq, int heads, int kv_heads, int hd, int n_rows) {
    const long nq = static_cast<long>(heads / kv_heads) * n_rows;
    return (hd == 64 || hd == 128) && batch <= 65535 && kv_heads <= 65535 && seq <= kMxMaxSeq &&
           nq <= (0x7fffffL << 5) && (nq + kMxQ) / kMxQ * kv_heads <= 0x7fffff;
}

template <bool BF16, int HD>
void mx_att_launch(const MxAttPlan& p, const MxAttArgs& a, int batch, hipStream_t stream) {
    const dim3 grid(p.tiles * a.kv_heads, p.splits, batch);
    if (p.waves == 8)
        hipLaunchKernelGGL((mx_attend_kernel<BF16, HD, 8>), grid, dim3(8 * kWave), 0, stream, a);
    else
        hipLaunchKernelGGL((mx_attend_kernel<BF16, HD, 4>), grid, dim3(4 * kWave), 0, stream, a);
    if (p.splits > 1) {
        const dim3 merge((a.heads / a.kv_heads) * a.n_rows, a.kv_heads, batch);
        if (p.splits <= 8) hipLaunchKernelGGL((mx_attend_merge_kernel<BF16, HD, 1>), merge, dim3(kWave), 0, stream, a);
        else hipLaunchKernelGGL((mx_attend_merge_kernel<BF16, HD, 4>), merge, dim3(4 * kWave), 0, stream, a);
    }
}

}  // namespace
}  // namespace ps

extern "C" size_t polestar_mx_attend_workspace_size(polestar_dtype dtype, int batch, int seq, int n_heads,
                                                    int n_kv_heads, int head_dim, int n_rows) {
    using namespace ps;
    if (!dtype_ok(dtype) || batch <= 0 || seq <= 0 || n_heads <= 0 || n_kv_heads <= 0 || n_rows <= 0 ||
        n_heads % n_kv_heads != 0 || !mx_att_shape_ok(batch, seq, n_heads, n_kv_heads, head_dim, n_rows))
        return 0;
    return mx_att_plan(batch, seq, n_heads, n_kv_heads, head_dim, n_rows).total;
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
    if (!mx_att_shape_ok(batch, seq, n_heads, n_kv_heads, head_dim, n_rows) || !row_ok(dtype, q_stride) ||
        !aligned16(q) || !aligned16(k_codes) || !aligned16(v_codes) || !aligned_to(k_scales, head_dim / kMxBlock) ||
        !aligned_to(v_scales, head_dim / kMxBlock) || !aligned16(out) || !aligned16(workspace))
        return POLESTAR_ERR_UNSUPPORTED;
    const MxAttPlan p = mx_att_plan(batch, seq, n_heads, n_kv_heads, head_dim, n_rows);
    if (workspace_bytes < p.total || (p.total > 0 && !workspace)) return POLESTAR_ERR_WORKSPACE;
    if (!(scale > 0.f)) scale = 1.f / sqrtf(static_cast<float>(head_dim));
    const MxAttArgs a{static_cast<const char*>(q), q_stride, k_codes, k_scales, v_codes, v_scales, kv_len,
                      static_cast<char*>(out), lse, scale * kLog2e, seq, n_rows, n_heads, n_kv_heads, p.tiles, p.splits,
                      static_cast<float*>(workspace),
                      reinterpret_cast<float2*>(static_cast<char*>(workspace) + p.part)};
    if (dtype == POLESTAR_BF16) {
        if (head_dim == 128) mx_att_launch<true, 128>(p, a, batch, stream);
        else mx_att_launch<true, 64>(p, a, batch, stream);
    } else {
        if (head_dim == 128) mx_att_launch<false, 128>(p, a, batch, stream);
        else mx_att_launch<false, 64>(p, a, batch, stream);
    }
    return launch_status();
}

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
// 1.5e-5 of the result's norm on normal data, which fp32 would show.  (Decoded channels
// are exact down to bf16's subnormals: those of blocks with scale bytes 0 to 2 are
// rounded to multiples of 2^-133.)  With MXFP4 rows the products of a block span less
// than those bits, and sums are as good as fp32 additions: measured over 1024 channels,
// exact where the rows' and the weights' scales span a factor of 16 each, and within 2.7
// 2^-24 of the magnitudes' sum where they span 2^40.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "host_common.hpp"
#include "mx_dev.hpp"

namespace ps {
namespace {

struct MxGemmArgs {
    const uint8_t *x, *xs, *w, *ws;
    char* y;
    float* part;                                         // split K: partials [split][rows][n_out]
    long rows;
    int n_out, n_in;
    int ksplit, steps;                                   // 128-channel steps of a split, an even number
    int row_tiles, col_tiles;
};

// Operand fragments of a step, 128 channels of the 16x16x128 instruction: lane l
// holds row l % 16 and the scale of block g = l / 16.  DEC: decoded to bf16 for four
// 16x16x32 instructions.
template <int FMT, bool DEC> struct Frag;
template <bool DEC> struct Frag<POLESTAR_MXFP4, DEC> {
    uint4 c;                                             // channels 32 g ..
    __device__ __forceinline__ intx8 codes() const {
        return intx8{static_cast<int>(c.x), static_cast<int>(c.y), static_cast<int>(c.z), static_cast<int>(c.w), 0, 0, 0, 0};
    }
    __device__ __forceinline__ void decode(uint4* o, float sc) const {
        o[0] = mx_fp4_bf16(c.x, sc); o[1] = mx_fp4_bf16(c.y, sc);
        o[2] = mx_fp4_bf16(c.z, sc); o[3] = mx_fp4_bf16(c.w, sc);
    }
};
// 8-bit operands: the instruction's lane holds channels 16 g .. and 64 + 16 g ..
// (its scale is still that of block g); decoded, 32 g .. as with 4 bits.
template <bool DEC> struct Frag<POLESTAR_MXFP8, DEC> {
    uint4 c[2];
    __device__ __forceinline__ intx8 codes() const {
        return intx8{static_cast<int>(c[0].x), static_cast<int>(c[0].y), static_cast<int>(c[0].z), static_cast<int>(c[0].w),
                     static_cast<int>(c[1].x), static_cast<int>(c[1].y), static_cast<int>(c[1].z), static_cast<int>(c[1].w)};
    }
    __device__ __forceinline__ void decode(uint4* o, float sc) const {
        o[0] = mx_fp8_bf16(c[0].x, c[0].y, sc); o[1] = mx_fp8_bf16(c[0].z, c[0].w, sc);
        o[2] = mx_fp8_bf16(c[1].x, c[1].y, sc); o[3] = mx_fp8_bf16(c[1].z, c[1].w, sc);
    }
};

// A K tile's rows in LDS (KS steps): 64 or 128 bytes, their 16-byte chunks
// XOR-swizzled so that the lanes whose reads run together (0-3, 12-15, 20-27 of each
// 32, and the others) lie in different banks.  With rows of 64 bytes swizzled by row
// / 4 half the LDS cycles of an MXFP4 product were conflicts.
template <int FMT, int KS> struct LdsRow {
    static constexpr int kBytes = KS * 16 * Mx<FMT>::kBits;
    static_assert(kBytes == 64 || kBytes == 128, "");
    __device__ __forceinline__ static int chunk(int row, int c) {
        return (c ^ (kBytes == 64 ? -(row >> 2) & 3 : (row >> 1) & 7)) << 4;
    }
    template <bool DEC> __device__ __forceinline__ static void load(Frag<FMT, DEC>& f, const char* tile, int r, int step, int g) {
        const char* p = tile + r * kBytes;
        if constexpr (FMT == POLESTAR_MXFP4) {
            f.c = ld16(p + chunk(r, 4 * step + g));
        } else {
            f.c[0] = ld16(p + chunk(r, DEC ? 2 * g : g));
            f.c[1] = ld16(p + chunk(r, DEC ? 2 * g + 1 : 4 + g));
        }
    }
};

constexpr int kMxTileThreads = 512;                      // eight waves, two per SIMD
constexpr int kMxBand = 4;                               // row tiles per band of the launch order
constexpr int kMxCus = 256;

// Transfers into LDS, 16 bytes per lane, from a buffer of `bytes` bytes at base: a
// lane's offset is one register, the K tile's a scalar; the lanes land one after
// another from lds on.  Written out, because the compiler waits for every transfer
// that it knows of before it reads LDS; the waits are the kernel's own (mx_wait_vm
// before the barrier that hands a slot over).  m0 is a register that the compiler
// reserves, hence its warning, but values of its own in m0 have to end here.
typedef uint32_t MxBuffer __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ MxBuffer mx_buffer(const void* base, uint32_t bytes) {
    const uint64_t p = reinterpret_cast<uint64_t>(base);
    return MxBuffer{uniform(static_cast<uint32_t>(p)), uniform(static_cast<uint32_t>(p >> 32)), uniform(bytes), 0x00027000u};
}
__device__ __forceinline__ uint32_t lds_offset(const char* p) {
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)p));
}
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void mx_dma16(MxBuffer b, uint32_t lane_off, uint32_t off, const char* lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :: "s"(uniform(lds_offset(lds))), "v"(lane_off), "s"(b), "s"(uniform(off)) : "memory", "m0");
}
#pragma clang diagnostic pop
// s_waitcnt immediates: at most n vector-memory operations outstanding / LDS reads done
constexpr int mx_wait_vm(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4) | (15 << 8); }
constexpr int kMxWaitLgkm0 = 15 | (3 << 14) | (7 << 4);

// A tile shape: BM = 16 MI WM rows x BN = 16 NJ (8 / WM) outputs per workgroup, its
// eight waves in a WM x (8 / WM) grid of MI x NJ tiles; K tiles of KS steps, NS of them
// in LDS; scales for R steps at a time, in two buffers.
template <int FMT_, int WM_, int MI_, int NJ_, int KS_, int NS_, int R_> struct MxShape {
    static constexpr int FMT = FMT_, WM = WM_, WN = 8 / WM_, MI = MI_, NJ = NJ_, KS = KS_, NS = NS_, R = R_;
    static constexpr int BM = 16 * MI * WM, BN = 16 * NJ * WN;
    // (the rows' steps one after another where two are more than an LDS row)
    static constexpr int kPlanes = FMT == POLESTAR_MXFP8 ? KS : 1;
    using X = LdsRow<FMT, KS / kPlanes>;
    using W = LdsRow<POLESTAR_MXFP4, KS>;
    static constexpr int kPlane = BM * X::kBytes, kX = kPlanes * kPlane, kSlot = kX + BN * W::kBytes;
    // a row's scales of R steps: chunks of 16 bytes, a lane each, swizzled like the
    // codes' (16 rows' reads in different banks)
    static constexpr int kChunks = (R + 3) / 4, kRow = 16 * kChunks, kScales = kRow * (BM + BN);
    static constexpr int kSRows = 64 / kChunks;          // rows of a transfer
    __device__ __forceinline__ static int scale_chunk(int row, int c) { return (c ^ row / (16 / kChunks) % kChunks) << 4; }
    static constexpr int kUnroll = R / KS;               // K tiles
    static_assert(NS * kSlot + 2 * kScales <= 160 * 1024 && kUnroll % NS == 0 && R % KS == 0, "");
};

// The scales of step `step` of the round in the buffer at byte buf.
struct Scales {
    int buf, step;
};

template <class F, int... U> __device__ __forceinline__ void mx_unrolled(F f, std::integer_sequence<int, U...>) {
    (f(std::integral_constant<int, U>{}), ...);
}

// Workgroup blk -> (split, row tile, column tile): consecutive workgroups go to
// different XCDs, so the ids are first regrouped per XCD, and each XCD walks
// bands of row tiles column by column, which keeps the rows and weights that its
// compute units share in its own L2.
__device__ __forceinline__ void mx_tile_coords(const MxGemmArgs& g, int blk, int& split, int& rt, int& ct) {
    const int ntiles = g.row_tiles * g.col_tiles, nb = ntiles * g.ksplit;
    const int xcd = blk & 7;
    const int bid = xcd * (nb >> 3) + min(xcd, nb & 7) + (blk >> 3);
    split = bid / ntiles;
    const int tl = bid - split * ntiles;
    const int band = tl / (kMxBand * g.col_tiles);
    const int rows_here = min(kMxBand, g.row_tiles - band * kMxBand);
    const int in = tl - band * kMxBand * g.col_tiles;
    ct = in / rows_here;
    rt = band * kMxBand + (in - ct * rows_here);
}

// A workgroup's tile: codes and scales by DMA into LDS slots, one barrier per K tile,
// a wave's blocks on the 16x16x128 scaled instruction (DEC: four 16x16x32 bf16 ones).
//
// What bounds it.  512 x 12288 x 4096 takes 28.3 us (MXFP8, 1.8 PFLOP/s) and 21.3
// (MXFP4, 2.4); the MXFP8 one's transfers alone take 23, its fragment reads and products
// alone 24.  The transfers' time goes by the cache lines they touch more than by bytes
// (3.64e6 requests to L2, about four clocks of a compute unit each): with K tiles of half
// lines and scales of one K tile at a time, 5.30e6 requests, it was 36.3 and 33.1 us.
// More slots (8 K tiles in flight) gained nothing, nor did two groups of waves with a
// step each (a third fewer LDS reads).  12288 x 4096 x 24576 takes 0.89 to 0.95 ms
// (MXFP8, 2.6 to 2.8 PFLOP/s) and 0.59 to 0.61 (MXFP4, 4.1 to 4.2).  There the clock
// falls under the load, three calls in a row from 2.3 GHz to 1.75 and 1.6 while the time
// grows by a fifth and the cycles shrink; of the cycles the matrix units are busy in two
// thirds (MXFP8) and half (MXFP4), and waves wait in 28% of theirs.
template <class T, bool BF16>
__global__ __launch_bounds__(kMxTileThreads) void mx_tile_kernel(MxGemmArgs g) {
    constexpr int FMT = T::FMT, MI = T::MI, NJ = T::NJ, KS = T::KS, BM = T::BM, BN = T::BN, NS = T::NS;
    constexpr bool DEC = FMT == POLESTAR_MXFP8 && !BF16;
    constexpr int XB = T::X::kBytes, WB = T::W::kBytes;
    constexpr int XG = BM * XB / 1024, WG = BN * WB / 1024;   // DMA groups of a K tile
    constexpr int XI = (XG * T::kPlanes + 7) / 8, WI = (WG + 7) / 8;   // instructions per wave
    static_assert(T::kPlanes == 1 || XG % 8 == 0, "");
    constexpr int ND = XI + WI;
    constexpr int SXG = BM / T::kSRows, SG = SXG + BN / T::kSRows, SI = (SG + 7) / 8;   // of R steps' scales
    __shared__ __align__(16) char lds[NS * T::kSlot + 2 * T::kScales];
    char* const sc = lds + NS * T::kSlot;

    int split, rt, ct;
    mx_tile_coords(g, blockIdx.x, split, rt, ct);
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = w % T::WM, wn = w / T::WM;
    const int r = lane & 15, grp = lane >> 4;
    const long m0 = static_cast<long>(rt) * BM;
    const int n0 = ct * BN;
    const int q0 = split * g.steps;                      // this split's steps
    const int nst = min(g.steps, g.n_in / 128 - q0), nkt = (nst + KS - 1) / KS;

    // DMA sources.  The buffers end with the tile's last row: what lies behind it
    // (rows and columns past the end, scales behind the last step) reads as 0.  A
    // group past the last (few rows): the last group again, the same bytes.
    const uint32_t xrow = static_cast<uint32_t>(g.n_in / 8) * Mx<FMT>::kBits, wrow = g.n_in / 2, srow = g.n_in / 32;
    const uint32_t mrows = static_cast<uint32_t>(min(g.rows - m0, static_cast<long>(BM))), nrows = min(g.n_out - n0, BN);
    const MxBuffer xbuf = mx_buffer(g.x + static_cast<size_t>(m0) * xrow, mrows * xrow);
    const MxBuffer wbuf = mx_buffer(g.w + static_cast<size_t>(n0) * wrow, nrows * wrow);
    constexpr int XR = 1024 / XB, WR = 1024 / WB;        // rows of a group
    const int xg = min(w, XG - 1), wg = min(w, WG - 1), xr = xg * XR + lane / (XB / 16), wr = wg * WR + lane / (WB / 16);
    const uint32_t xsrc = xr * xrow + T::X::chunk(xr, lane % (XB / 16));   // (the swizzle repeats with the groups)
    const uint32_t wsrc = wr * wrow + T::W::chunk(wr, lane % (WB / 16));
    // Scales, R steps at a time: a row's are one cache line for 32 steps.
    const MxBuffer xsbuf = mx_buffer(g.xs + static_cast<size_t>(m0) * srow, mrows * srow);
    const MxBuffer wsbuf = mx_buffer(g.ws + static_cast<size_t>(n0) * srow, nrows * srow);
    auto issue_scales = [&](int t, int buf) {
#pragma unroll
        for (int d = 0; d < SI; ++d) {
            const int gr = min(w + 8 * d, SG - 1), row = (gr < SXG ? gr : gr - SXG) * T::kSRows + lane / T::kChunks;
            mx_dma16(gr < SXG ? xsbuf : wsbuf, row * srow + T::scale_chunk(row, lane % T::kChunks), 4 * (q0 + t * KS),
                     sc + buf + gr * T::kSRows * T::kRow);
        }
    };
    // DMA instructions d0 .. d0 + n - 1 of K tile t (past the split: its last one again)
    auto issue = [&](int d0, int n, int t, const char* slot) {
        const uint32_t k = q0 + min(t, nkt - 1) * KS, kx = k * (16 * Mx<FMT>::kBits), kw = k * 64;
#pragma unroll
        for (int d = d0; d < d0 + n; ++d) {
            if (d < XI) mx_dma16(xbuf, xsrc, kx + 8 * d % max(XG, 8) * XR * xrow + 8 * d / max(XG, 8) * XB, slot + (xg + 8 * d) * 1024);
            else if (d < ND)
                mx_dma16(wbuf, wsrc, kw + 8 * (d - XI) * WR * wrow, slot + T::kX + (wg + 8 * (d - XI)) * 1024);
        }
    };

    // A wave's fragments.  The two largest shapes have 8 row (or output) tiles: they
    // hold the other operand's four and a ring of four of the eight, each replaced right
    // after its use by the one four on, of this step or the next (two steps' fragments
    // would not fit the registers); the smaller shapes hold two steps' in turn.
    constexpr bool kRing = MI * NJ == 32, kRingX = kRing && MI == 8;
    constexpr int NX = kRingX ? 4 : MI, NW = kRing && !kRingX ? 4 : NJ, SETS = 2;
    Frag<FMT, DEC> fx[SETS][NX];
    Frag<POLESTAR_MXFP4, DEC> fw[SETS][NW];
    uint32_t sx[SETS][NX], sw[SETS][NW];                 // scale bytes
    // a step's scales in the buffers: of row `row`, which is r behind a tile's first
    auto scales_at = [&](int row, int step) { return row * T::kRow + T::scale_chunk(r, step / 4) + 4 * (step % 4) + grp; };
    // fragment j of step s of a slot, its scales those of step `q` of a round
    auto read_x = [&](int set, int j, const char* slot, int s, Scales q) {
        const int plane = T::kPlanes > 1 ? s * T::kPlane : 0;
        T::X::load(fx[set][j % NX], slot + plane + 16 * (MI * wm + j) * XB, r, s, grp);
        sx[set][j % NX] = *reinterpret_cast<const uint8_t*>(sc + q.buf + scales_at(16 * MI * wm + r, q.step) + 16 * T::kRow * j);
    };
    auto read_w = [&](int set, int j, const char* slot, int s, Scales q) {
        T::W::load(fw[set][j % NW], slot + T::kX + 16 * (NJ * wn + j) * WB, r, s, grp);
        sw[set][j % NW] = *reinterpret_cast<const uint8_t*>(sc + q.buf + scales_at(BM + 16 * NJ * wn + r, q.step) + 16 * T::kRow * j);
    };
    floatx4 acc[MI][NJ];
#pragma unroll
    for (int a = 0; a < MI; ++a)
#pragma unroll
        for (int b = 0; b < NJ; ++b) acc[a][b] = floatx4{0.f, 0.f, 0.f, 0.f};
    auto mma = [&](int xset, int wset, int a, int b) {
        const auto& x = fx[xset][a % NX];
        const auto& v = fw[wset][b % NW];
        if constexpr (DEC) {
            uint4 dx[4], dw[4];
            x.decode(dx, mx_scale(sx[xset][a % NX]));
            v.decode(dw, mx_scale(sw[wset][b % NW]));
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[a][b] = mfma_bf16(dw[t], dx[t], acc[a][b]);
        } else {
            acc[a][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(v.codes(), x.codes(), acc[a][b],
                                                                         Mx<POLESTAR_MXFP4>::kMfma, Mx<FMT>::kMfma, 0,
                                                                         sw[wset][b % NW], 0, sx[xset][a % NX]);
        }
    };
    auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
    // The barrier of K tile t, for this wave's reads of its slot and its DMA of t + 1:
    // behind it t + 1 may be read and the slot takes t + NS.
    auto sync = [&] {
        fence();
        __builtin_amdgcn_s_waitcnt(mx_wait_vm((NS - 2) * ND) & kMxWaitLgkm0);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        fence();
    };
    issue_scales(0, 0);
#pragma unroll
    for (int t = 0; t < NS; ++t) issue(0, ND, t, lds + t * T::kSlot);
    __builtin_amdgcn_s_waitcnt(mx_wait_vm((NS - 1) * ND));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    // K tile t, in slot U, whose scales are in buffer `buf`.  (The slots are
    // constants: with a slot that moves, each read's address is computed behind the
    // barrier, 8% slower.)
    auto slot_of = [&](int u) { return lds + u % NS * T::kSlot; };
    auto scales_of = [&](int step, int buf) {            // of a step of the buffer's R, or the first of the next R
        return step < T::R ? Scales{buf, step} : Scales{buf ^ T::kScales, 0};
    };
    int buf = 0, t = 0;
    auto rounds = [&](int whole, auto ktile) {           // K tiles 0 .. whole - 1
        constexpr int kUnroll = T::kUnroll;
        for (; t + kUnroll <= whole; t += kUnroll, buf ^= T::kScales)
            mx_unrolled([&](auto u) {
                ktile(t + u, u);
                if (u == 0) issue_scales(t + kUnroll, buf ^ T::kScales);   // landed by the last sync before they are read
            }, std::make_integer_sequence<int, kUnroll>{});
        mx_unrolled([&](auto u) {
            if (t + u < whole) ktile(t + u, u);
        }, std::make_integer_sequence<int, kUnroll - 1>{});
    };
    if constexpr (kRing) {
        constexpr int NI = 4;                            // tiles of the operand that is held
        auto read_ring = [&](int j, const char* slot, int s, Scales q) {
            if constexpr (kRingX) read_x(0, j, slot, s, q);
            else read_w(0, j, slot, s, q);
        };
        auto read_held = [&](int set, const char* slot, int s, Scales q) {
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                if constexpr (kRingX) read_w(set, j, slot, s, q);
                else read_x(set, j, slot, s, q);
            }
        };
        auto row = [&](int j) {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                if constexpr (kRingX) mma(0, 0, j, i);
                else mma(0, 0, i, j);
            }
        };
        read_held(0, lds, 0, Scales{0, 0});
#pragma unroll
        for (int j = 0; j < 4; ++j) read_ring(j, lds, 0, Scales{0, 0});
        constexpr int DPR = (ND + 2) / 3;                // DMA instructions behind each of the last three
        auto ktile = [&](int kt, auto which) {
            constexpr int U = decltype(which)::value;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const bool last = s == KS - 1;
                const Scales q = scales_of(U * KS + s, buf), qn = scales_of(U * KS + s + 1, buf);
                const char* next = last ? slot_of(U + 1) : slot_of(U);
                const int sn = last ? 0 : s + 1;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    row(j);
                    if (j == 4) {
                        if (last) sync();
                        read_held(1, next, sn, qn);
                    }
                    fence();
                    if (j < 4) read_ring(j + 4, slot_of(U), s, q);
                    else read_ring(j - 4, next, sn, qn);
                    if (last && j > 4) issue((j - 5) * DPR, DPR, kt + NS, slot_of(U));
                    fence();
                }
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    if constexpr (kRingX) {
                        fw[0][i] = fw[1][i];
                        sw[0][i] = sw[1][i];
                    } else {
                        fx[0][i] = fx[1][i];
                        sx[0][i] = sx[1][i];
                    }
                }
            }
        };
        const int whole = nst / KS;
        rounds(whole, ktile);
        if (KS > 1 && whole < nkt) {                     // one step is left
            const int u = whole - t;                     // its slot
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                row(j);
                if (j < 4) read_ring(j + 4, slot_of(u), 0, scales_of(u * KS, buf));
            }
        }
    } else {
        static_assert(T::R % 2 == 0, "two register sets, in turn");
        constexpr int DPR = (ND + MI - 1) / MI;
        auto read = [&](int set, const char* slot, int s, Scales q) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) read_w(set, j, slot, s, q);
#pragma unroll
            for (int j = 0; j < MI; ++j) read_x(set, j, slot, s, q);
        };
        read(0, lds, 0, Scales{0, 0});
        const int whole = nst / KS;
        rounds(whole, [&](int kt, auto which) {
            constexpr int U = decltype(which)::value;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const bool last = s == KS - 1;
                const int set = (U * KS + s) % 2;
                if (last) sync();
                read(1 - set, last ? slot_of(U + 1) : slot_of(U), last ? 0 : s + 1, scales_of(U * KS + s + 1, buf));
                fence();
#pragma unroll
                for (int a = 0; a < MI; ++a) {
#pragma unroll
                    for (int b = 0; b < NJ; ++b) mma(set, set, a, b);
                    if (last) issue(a * DPR, DPR, kt + NS, slot_of(U));
                    fence();
                }
            }
        });
        if (KS > 1 && whole < nkt) {                     // one step is left
#pragma unroll
            for (int a = 0; a < MI; ++a)
#pragma unroll
                for (int b = 0; b < NJ; ++b) mma(0, 0, a, b);
        }
    }
    __builtin_amdgcn_s_waitcnt(0);                       // every DMA (the re-read tail too) has landed
    __syncthreads();                                     // and every wave is done with the slots

    // lane: row r of its tile, outputs 4 grp .. + 3
    const int nw = n0 + 16 * NJ * wn;
    if (g.ksplit > 1) {
#pragma unroll
        for (int a = 0; a < MI; ++a) {
            const long m = m0 + 16 * (MI * wm + a) + r;
            if (m >= g.rows) continue;
            float* p = g.part + (static_cast<size_t>(split) * g.rows + m) * g.n_out;
#pragma unroll
            for (int b = 0; b < NJ; ++b) {
                const int n = nw + 16 * b + 4 * grp;
                if (n < g.n_out) *reinterpret_cast<floatx4*>(p + n) = acc[a][b];
            }
        }
        return;
    }
    // through LDS, 16 rows of the wave at a time in a region of its own, then 16
    // bytes of a row per lane
    constexpr int ES = BF16 ? 2 : 4;
    constexpr int EP = 16 * NJ * ES + 16;                // bytes of a staged row
    constexpr int CPR = NJ * ES;                         // 16-byte chunks of a row
    static_assert(8 * 16 * EP <= sizeof(lds), "every wave's rows");
    char* ep = lds + w * 16 * EP;
#pragma unroll
    for (int a = 0; a < MI; ++a) {
#pragma unroll
        for (int b = 0; b < NJ; ++b) {
            char* d = ep + r * EP + (16 * b + 4 * grp) * ES;
            const floatx4& v = acc[a][b];
            if constexpr (BF16)
                *reinterpret_cast<uint2*>(d) = make_uint2(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]));
            else
                *reinterpret_cast<floatx4*>(d) = v;
        }
        __builtin_amdgcn_s_waitcnt(kMxWaitLgkm0);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int q = 0; q < (16 * CPR + 63) / 64; ++q) {
            const int at = 64 * q + lane, c = at % CPR;
            const long m = m0 + 16 * (MI * wm + a) + at / CPR;
            const int n = nw + c * (16 / ES);
            if (at < 16 * CPR && m < g.rows && n < g.n_out)
                st16(g.y + (static_cast<size_t>(m) * g.n_out + n) * ES, ld16(ep + at / CPR * EP + 16 * c));
        }
        __builtin_amdgcn_s_waitcnt(kMxWaitLgkm0);
        __builtin_amdgcn_wave_barrier();
    }
}

// ---------------------------------------------------------------------------
// Few rows: bound by the weights' stream and, below a few MB, by latency.  16 MT
// rows x 16 NT outputs per workgroup; its waves take chunks of 512 channels in turn
// (256 bytes of a weight row, 16 of its scales), every load of a chunk issued before
// its first product, and their sums are added in LDS: no split and no second launch.
// One row of 4096 x 4096 takes 3.5 us in a graph (8.9 MB at 2.5 TB/s), of 4096 x 24576
// 11.3 (53 MB at 4.7).
//
// RAW: the rows come as dtype and are quantized here, a lane the block that it holds
// (32 channels: no exchange for the maximum), so that one launch does both; every
// workgroup repeats that work, which is why only 16 rows are taken this way.
// ---------------------------------------------------------------------------

constexpr int kFewWaves = 8, kFewThreads = kFewWaves * kWave;
constexpr int kFewRows = 64;                             // most rows of these kernels
constexpr int kFewSteps = 4;                             // steps of a chunk, of 128 channels

struct MxFewArgs : MxGemmArgs {
    const char* raw;                                     // [batch][seq][n_in] dtype
    int seq, row_start, n_rows;
};

// Buffers whose end is checked, for loads into registers.
typedef __amdgpu_buffer_rsrc_t MxRows;
__device__ __forceinline__ MxRows mx_rows(const uint8_t* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, bytes, 0x00027000);
}
__device__ __forceinline__ uint4 mx_load16(MxRows b, uint32_t lane_off, uint32_t off) {
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(b, lane_off, off, 0));
}

// The operand of a step, 128 channels from LDS-free loads.  MXFP8 codes: as
// Frag<MXFP8>'s loads, from memory.
constexpr uint32_t kMxPastEnd = 0x40000000u;             // an offset behind every such buffer: reads as 0
template <int FMT, bool DEC>
__device__ __forceinline__ void frag_load(Frag<FMT, DEC>& f, MxRows b, uint32_t row, uint32_t step, bool in, int g) {
    if constexpr (FMT == POLESTAR_MXFP4) {
        f.c = mx_load16(b, row + 16 * g, in ? 64 * step : kMxPastEnd);
    } else {
        f.c[0] = mx_load16(b, row + (DEC ? 32 * g : 16 * g), in ? 128 * step : kMxPastEnd);
        f.c[1] = mx_load16(b, row + (DEC ? 32 * g + 16 : 64 + 16 * g), in ? 128 * step : kMxPastEnd);
    }
}

__device__ __forceinline__ void swap_rows16(uint32_t& a, uint32_t& b) {   // a's odd 16 lanes with b's even ones
    const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}

// 32 channels of block g quantized to the lane's operand; returns the scale byte of
// the block that the instruction expects it for.  MXFP8 (not decoded): lanes 0-15 and
// 16-31 hold the halves of two blocks each, so they exchange them, and the blocks in
// the instruction's order are 0, 2, 1, 3: the weights' lanes load them in that order.
template <int FMT, bool DEC>
__device__ __forceinline__ uint32_t frag_quantize(Frag<FMT, DEC>& f, const float* v) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    uint32_t byte = mx_scale_byte<FMT>(m);
    const float sc = mx_scale(byte);
    const uint32_t keep = byte == kMxNanScale ? 0u : ~0u;
    if constexpr (FMT == POLESTAR_MXFP4) {
        f.c = make_uint4(mx_pack_fp4(v, sc) & keep, mx_pack_fp4(v + 8, sc) & keep, mx_pack_fp4(v + 16, sc) & keep,
                         mx_pack_fp4(v + 24, sc) & keep);
    } else {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = mx_pack_fp8(v + 4 * i, sc) & keep;
        if constexpr (!DEC) {
#pragma unroll
            for (int i = 0; i < 4; ++i) swap_rows16(w[i], w[4 + i]);
            const int lane = threadIdx.x & 63, g = lane >> 4;
            byte = __shfl(static_cast<int>(byte), (lane & 15) + 16 * (g == 1 ? 2 : g == 2 ? 1 : g));
        }
        f.c[0] = make_uint4(w[0], w[1], w[2], w[3]);
        f.c[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
    return byte;
}

template <int FMT, bool BF16, bool RAW, int MT, int NT>
__global__ __launch_bounds__(kFewThreads) void mx_few_kernel(MxFewArgs g) {
    constexpr bool DEC = FMT == POLESTAR_MXFP8 && !BF16;
    constexpr bool kSwap = RAW && FMT == POLESTAR_MXFP8 && !DEC;   // blocks in the order 0, 2, 1, 3
    constexpr int ES = BF16 ? 2 : 4;
    constexpr int S = kFewSteps;
    static_assert(!RAW || (MT == 1 && NT == 1), "rows quantized here: one tile");
    __shared__ floatx4 red[kFewWaves][MT * NT][kWave];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, grp = lane >> 4;
    const int wgrp = kSwap ? (grp == 1 ? 2 : grp == 2 ? 1 : grp) : grp;
    const int n0 = blockIdx.x * 16 * NT, rows = static_cast<int>(g.rows);
    const uint32_t xrow = static_cast<uint32_t>(g.n_in / 8) * Mx<FMT>::kBits, wrow = g.n_in / 2, srow = g.n_in / 32;
    const uint32_t nrows = min(g.n_out - n0, 16 * NT);
    const MxRows wbuf = mx_rows(g.w + static_cast<size_t>(n0) * wrow, nrows * wrow);
    const MxRows wsbuf = mx_rows(g.ws + static_cast<size_t>(n0) * srow, nrows * srow);
    const MxRows xbuf = mx_rows(g.x, rows * xrow), xsbuf = mx_rows(g.xs, rows * srow);
    const char* raw = nullptr;
    if constexpr (RAW) {
        const int m = min(r, rows - 1);                  // past the end: the last one, not stored
        raw = g.raw + (static_cast<size_t>(m / g.n_rows) * g.seq + g.row_start + m % g.n_rows) * g.n_in * ES + 32 * grp * ES;
    }
    const int nsteps = g.n_in / 128;
    floatx4 acc[MT][NT];
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b) acc[a][b] = floatx4{0.f, 0.f, 0.f, 0.f};
    // TAIL: steps past the end multiply zeros by finite numbers
    auto chunk = [&](int c0, auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        auto in = [&](int s) { return !TAIL || c0 + s < nsteps; };
        Frag<POLESTAR_MXFP4, DEC> fw[S][NT];
        uint4 sw[NT], sx[MT];
        Frag<FMT, DEC> fx[S][MT];
        uint4 rv[RAW ? S : 1][RAW ? 2 * ES : 1];
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int b = 0; b < NT; ++b) frag_load(fw[s][b], wbuf, (16 * b + r) * wrow, c0 + s, in(s), wgrp);
#pragma unroll
        for (int b = 0; b < NT; ++b) sw[b] = mx_load16(wsbuf, (16 * b + r) * srow, 4 * c0);
        if constexpr (RAW) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const char* p = raw + static_cast<size_t>(min(c0 + s, nsteps - 1)) * 128 * ES;
#pragma unroll
                for (int i = 0; i < 2 * ES; ++i) rv[s][i] = ld16(p + 16 * i);
            }
        } else {
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int a = 0; a < MT; ++a) frag_load(fx[s][a], xbuf, (16 * a + r) * xrow, c0 + s, in(s), grp);
#pragma unroll
            for (int a = 0; a < MT; ++a) sx[a] = mx_load16(xsbuf, (16 * a + r) * srow, 4 * c0);
        }
        __builtin_amdgcn_sched_barrier(0);               // every load first
#pragma unroll
        for (int s = 0; s < S; ++s) {
            auto byte_of = [&](const uint4& v, int q) {
                const uint32_t d = s == 0 ? v.x : s == 1 ? v.y : s == 2 ? v.z : v.w;
                return in(s) ? (d >> (8 * q)) & 255u : 127u;
            };
            uint32_t bx[MT];
            if constexpr (RAW) {
                float v[32];
#pragma unroll
                for (int i = 0; i < 2 * ES; ++i) Elem<BF16>::unpack(rv[s][i], v + i * Elem<BF16>::E);
                if constexpr (TAIL) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = in(s) ? v[i] : 0.f;
                }
                bx[0] = frag_quantize<FMT, DEC>(fx[s][0], v);
            } else {
#pragma unroll
                for (int a = 0; a < MT; ++a) bx[a] = byte_of(sx[a], grp);
            }
#pragma unroll
            for (int b = 0; b < NT; ++b) {
                const uint32_t bw = byte_of(sw[b], wgrp);
                uint4 dw[4];
                if constexpr (DEC) fw[s][b].decode(dw, mx_scale(bw));
#pragma unroll
                for (int a = 0; a < MT; ++a) {
                    if constexpr (DEC) {
                        uint4 dx[4];
                        fx[s][a].decode(dx, mx_scale(bx[a]));
#pragma unroll
                        for (int t = 0; t < 4; ++t) acc[a][b] = mfma_bf16(dw[t], dx[t], acc[a][b]);
                    } else {
                        acc[a][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                            fw[s][b].codes(), fx[s][a].codes(), acc[a][b], Mx<POLESTAR_MXFP4>::kMfma, Mx<FMT>::kMfma, 0, bw,
                            0, bx[a]);
                    }
                }
            }
        }
    };
    int c0 = w * S;
    for (; c0 + S <= nsteps; c0 += kFewWaves * S) chunk(c0, std::false_type{});
    if (c0 < nsteps) chunk(c0, std::true_type{});
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b) red[w][a * NT + b][lane] = acc[a][b];
    __syncthreads();
    for (int t = threadIdx.x; t < MT * NT * kWave; t += kFewThreads) {
        const int tile = t / kWave, l = t % kWave;
        floatx4 v = red[0][tile][l];
#pragma unroll
        for (int x = 1; x < kFewWaves; ++x) v += red[x][tile][l];
        const int m = 16 * (tile / NT) + (l & 15), n = n0 + 16 * (tile % NT) + 4 * (l >> 4);
        if (m >= rows || n >= g.n_out) continue;
        const size_t at = static_cast<size_t>(m) * g.n_out + n;
        if constexpr (BF16) *reinterpret_cast<uint2*>(g.y + 2 * at) = make_uint2(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]));
        else *reinterpret_cast<floatx4*>(g.y + 4 * at) = v;
    }
}

// The splits' partials, added in order; four outputs per thread.
template <bool BF16>
__global__ __launch_bounds__(256) void mx_reduce_kernel(const float* __restrict__ part, int ksplit, long n4,
                                                        char* __restrict__ y) {
    const long i = static_cast<long>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= n4) return;
    const float4* p = reinterpret_cast<const float4*>(part) + i;
    float4 v = p[0];
    for (int s = 1; s < ksplit; ++s) {
        const float4 e = p[s * n4];
        v = make_float4(v.x + e.x, v.y + e.y, v.z + e.z, v.w + e.w);
    }
    if constexpr (BF16) reinterpret_cast<uint2*>(y)[i] = make_uint2(cvt_pk_bf16(v.x, v.y), cvt_pk_bf16(v.z, v.w));
    else reinterpret_cast<float4*>(y)[i] = v;
}

// The tile shapes by rows and outputs.  A wave's block has four of its 16 x 16 tiles on
// one side at least, rows or outputs by which fragments are fewer bytes, and K tiles of
// 256 channels (whole cache lines of the weights) where LDS holds enough of them:
// MXFP8, 64 x 128: 36.3 -> 31.2 us for 512 x 12288 x 4096; 128 x 128 and 128 x 256 with
// two of 256 instead of four of 128 channels were 0 to 16% slower.
template <int FMT, int BM, int BN> struct ShapeOf;
template <> struct ShapeOf<POLESTAR_MXFP8, 256, 256> { using T = MxShape<POLESTAR_MXFP8, 2, 8, 4, 1, 3, 3>; };
template <> struct ShapeOf<POLESTAR_MXFP4, 256, 256> { using T = MxShape<POLESTAR_MXFP4, 2, 8, 4, 2, 2, 4>; };
template <> struct ShapeOf<POLESTAR_MXFP8, 128, 256> { using T = MxShape<POLESTAR_MXFP8, 2, 4, 4, 1, 4, 8>; };
template <> struct ShapeOf<POLESTAR_MXFP4, 128, 256> { using T = MxShape<POLESTAR_MXFP4, 2, 4, 4, 2, 2, 16>; };
template <> struct ShapeOf<POLESTAR_MXFP8, 128, 128> { using T = MxShape<POLESTAR_MXFP8, 4, 2, 4, 1, 4, 16>; };
template <> struct ShapeOf<POLESTAR_MXFP4, 128, 128> { using T = MxShape<POLESTAR_MXFP4, 2, 4, 2, 2, 4, 16>; };
template <> struct ShapeOf<POLESTAR_MXFP8, 64, 256> { using T = MxShape<POLESTAR_MXFP8, 2, 2, 4, 1, 4, 16>; };
template <int FMT> struct ShapeOf<FMT, 64, 128> { using T = MxShape<FMT, 2, 2, 2, 2, 4, 16>; };
#define PS_MX_SHAPES(X) X(256, 256) X(128, 256) X(128, 128) X(64, 256) X(64, 128)

// A shape's time per step (us) for MXFP8 rows, MXFP4 rows and the decoded form; 0: not
// used there.  (The decoded form has no registers for the two largest; 64 x 256 in the
// others and 128 x 128 in the decoded form gained 0.1% in the mean.)
constexpr struct MxStep {
    int bm, bn;
    double us[3];
} kMxSteps[] = {{256, 256, {1.57, 1.26, 0}}, {128, 256, {0.82, 0.63, 0}}, {128, 128, {0.50, 0.41, 0}},
                {64, 256, {0, 0, 0.69}}, {64, 128, {0.29, 0.23, 0.40}}};
constexpr int mx_class(int x_fmt, bool bf16) { return x_fmt == POLESTAR_MXFP4 ? 1 : bf16 ? 0 : 2; }
constexpr bool mx_has_tile(int x_fmt, bool bf16, int bm, int bn) {
    for (const auto& s : kMxSteps)
        if (s.bm == bm && s.bn == bn) return s.us[mx_class(x_fmt, bf16)] > 0;
    return false;
}

struct MxPlan {
    int bm, bn, ksplit, steps;
    size_t ws_bytes;
};

// Tile shape and K split with the least estimated time (us): rounds of one workgroup
// per CU, each its steps and a fixed cost, and for a split the reduction's launch and
// the partials' way through memory (per MB).  The constants are fitted to half of 8197
// random shapes of 17 to 8192 rows, 128 to 24576 outputs and 256 to 12288 channels,
// each with every tile shape and split: on the other half the chosen plan is 1.0%
// (MXFP8), 1.3% (MXFP4) and 0.6% (decoded) slower than the fastest in the geometric
// mean, 7, 9 and 6% at the 95th percentile, 30% at most.
MxPlan mx_plan(int x_fmt, bool bf16, long rows, int n_out, int n_in) {
    static constexpr struct { double fixed, launch, per_mb; } costs[] = {{3.2, 2.9, 1.2}, {2.5, 3.75, 1.0}, {3.5, 1.5, 0.47}};
    const int cls = mx_class(x_fmt, bf16);
    const auto& c = costs[cls];
    const int nst = n_in / 128;
    MxPlan p{};
    double best = 1e30;
    for (const auto& s : kMxSteps) {
        if (s.us[cls] == 0) continue;
        const long tiles = (rows + s.bm - 1) / s.bm * ceil_div(n_out, s.bn);
        for (int ks = 1; ks <= 16 && ks <= nst; ++ks) {
            const int steps = ceil_div(ceil_div(nst, ks), 2) * 2;   // whole K tiles
            if (ceil_div(nst, steps) != ks) continue;
            if (ks > 1 && (tiles * (ks - 1) >= kMxCus || steps < 4)) break;
            const double rounds = static_cast<double>((tiles * ks + kMxCus - 1) / kMxCus);
            const double cost = rounds * (std::min(steps, nst) * s.us[cls] + c.fixed) +
                                (ks > 1 ? c.launch + 4.0 * ks * rows * n_out * 1e-6 * c.per_mb : 0.0);
            if (cost < best) {
                best = cost;
                p = MxPlan{s.bm, s.bn, ks, steps, ks > 1 ? 4 * static_cast<size_t>(ks) * rows * n_out : 0};
            }
        }
    }
    return p;
}

// (MT, NT) of the few-rows kernels; nt as mx_few_nt gives it.
template <int FMT, bool BF16>
void mx_launch_few(const MxFewArgs& g, int nt, hipStream_t stream) {
    constexpr bool kDec = FMT == POLESTAR_MXFP8 && !BF16;   // no registers for (4, 2)
    if (kDec && g.rows > 32) nt = 1;
    const dim3 grid(ceil_div(g.n_out, 16 * nt)), block(kFewThreads);
#define PS_FEW(RAW, MT, NT) hipLaunchKernelGGL((mx_few_kernel<FMT, BF16, RAW, MT, NT>), grid, block, 0, stream, g)
    if (g.raw) PS_FEW(true, 1, 1);                       // (mx_few_raw: as many workgroups as compute units at most)
    else if (g.rows <= 16) { if (nt == 1) PS_FEW(false, 1, 1); else PS_FEW(false, 1, 2); }
    else if (g.rows <= 32) { if (nt == 1) PS_FEW(false, 2, 1); else PS_FEW(false, 2, 2); }
    else if constexpr (!kDec) { if (nt == 1) PS_FEW(false, 4, 1); else PS_FEW(false, 4, 2); }
    else PS_FEW(false, 4, 1);
#undef PS_FEW
}

// Output tiles of a few-rows workgroup: two where one would make more than two
// workgroups per compute unit.
int mx_few_nt(int n_out) { return ceil_div(n_out, 16) > 2 * kMxCus ? 2 : 1; }

// Whether the few-rows kernels take a product: where the rows' codes that a compute
// unit reads, once per workgroup, are at most 160 KB, or 32 KB where the weights' stream
// fills every compute unit anyway.  Over 51920 random shapes of 1 to 64 rows, 128 to
// 28800 outputs and 256 to 14336 channels the kernel that this chooses is 1.1% slower
// than the faster of the two in the geometric mean, 4% at the 95th percentile.  Against
// the tile kernel's best plan, us: 4096 x 4096, MXFP8, 8 rows 4.6 (8.1), 32 rows 7.4
// (8.5), 64 rows 11.5 (10.0); 12288 x 4096, 8 rows 9.4 (10.6), 24 rows 15.3 (11.3);
// 4096 x 24576, 1 row 11.3 (11.4), 8 rows 13.0 (11.5).
bool mx_few(int x_fmt, long rows, int n_out, int n_in) {
    if (rows > kFewRows) return false;
    const int nt = mx_few_nt(n_out);
    const long per_cu = rows * polestar_codec_row_bytes(x_fmt, n_in) * ceil_div(ceil_div(n_out, 16 * nt), kMxCus);
    return per_cu <= (nt == 1 ? 160 : 32) * 1024;
}

template <int FMT, bool BF16>
void mx_launch(const MxPlan& p, const MxGemmArgs& g, hipStream_t stream) {
    const dim3 grid(g.row_tiles * g.col_tiles * g.ksplit), block(kMxTileThreads);
    switch (1000 * p.bm + p.bn) {
#define PS_CASE(BM, BN)                                                                                                   \
        case 1000 * BM + BN:                                                                                              \
            if constexpr (mx_has_tile(FMT, BF16, BM, BN))                                                                 \
                hipLaunchKernelGGL((mx_tile_kernel<typename ShapeOf<FMT, BM, BN>::T, BF16>), grid, block, 0, stream, g);  \
            break;
        PS_MX_SHAPES(PS_CASE)
#undef PS_CASE
    }
    if (g.ksplit > 1) {
        const long n4 = g.rows * (g.n_out / 4);
        hipLaunchKernelGGL((mx_reduce_kernel<BF16>), dim3(ceil_div(n4, 256)), dim3(256), 0, stream, g.part, g.ksplit, n4, g.y);
    }
}

size_t mx_linear_ws(int x_fmt, polestar_dtype dtype, long rows, int n_out, int n_in) {
    return mx_few(x_fmt, rows, n_out, n_in) ? 0 : mx_plan(x_fmt, dtype == POLESTAR_BF16, rows, n_out, n_in).ws_bytes;
}

polestar_status mx_few_run(int x_fmt, bool bf16, const MxFewArgs& g, hipStream_t stream) {
    const int nt = mx_few_nt(g.n_out);
    if (x_fmt == POLESTAR_MXFP4) {
        if (bf16) mx_launch_few<POLESTAR_MXFP4, true>(g, nt, stream);
        else mx_launch_few<POLESTAR_MXFP4, false>(g, nt, stream);
    } else {
        if (bf16) mx_launch_few<POLESTAR_MXFP8, true>(g, nt, stream);
        else mx_launch_few<POLESTAR_MXFP8, false>(g, nt, stream);
    }
    return launch_status();
}

polestar_status mx_gemm_run(int x_fmt, polestar_dtype dtype, MxGemmArgs g, void* workspace, hipStream_t stream) {
    const bool bf16 = dtype == POLESTAR_BF16;
    if (mx_few(x_fmt, g.rows, g.n_out, g.n_in)) {
        MxFewArgs f{};
        static_cast<MxGemmArgs&>(f) = g;
        return mx_few_run(x_fmt, bf16, f, stream);
    }
    const MxPlan p = mx_plan(x_fmt, bf16, g.rows, g.n_out, g.n_in);
    g.part = static_cast<float*>(workspace);
    g.ksplit = p.ksplit;
    g.steps = p.steps;
    g.row_tiles = ceil_div(g.rows, p.bm);
    g.col_tiles = ceil_div(g.n_out, p.bn);
    if (x_fmt == POLESTAR_MXFP4) {
        if (bf16) mx_launch<POLESTAR_MXFP4, true>(p, g, stream);
        else mx_launch<POLESTAR_MXFP4, false>(p, g, stream);
    } else {
        if (bf16) mx_launch<POLESTAR_MXFP8, true>(p, g, stream);
        else mx_launch<POLESTAR_MXFP8, false>(p, g, stream);
    }
    return launch_status();
}

// Rows and outputs that the kernels' indices hold.
bool mx_shape_ok(long rows, int n_out, int n_in) {
    return n_in % 128 == 0 && n_out % 16 == 0 && rows <= (1L << 24) && n_out <= (1 << 22) && n_in <= (1 << 22);
}

// Rows that the product's kernel quantizes itself: up to 16 (fp32 4), where a wave has
// one chunk of the rows and a compute unit one workgroup.  One launch less is 2.7 us
// less on the host (6.9 instead of 9.6 us a call, queued one after another).  In a
// graph, against two launches, us: 1024 x 1024, 1 to 16 rows 3.2 to 4.1 (3.7 to 4.4);
// 2048 channels up to a tenth less; 4096 channels mostly more, bf16 by up to a fifth,
// fp32 a quarter: 4096 x 4096, MXFP8, bf16, 1 row 6.6 (6.3), 16 rows 8.2 (7.7), fp32, 4
// rows 7.8 (6.9); 16 of fp32, which are not taken, 11.9 (8.1).  Past the limits every
// workgroup quantizes chunk after chunk of the same rows: 4224 x 256 6.7 (4.9), 8192 x
// 2048 10.1 (7.5), 65536 x 256 53 (29); and 512 x 8192 takes 6.5 (4.5), 4096 x 12288
// 14.1 (11.7).
bool mx_few_raw(bool bf16, long rows, int n_out, int n_in) {
    return rows <= (bf16 ? 16 : 4) && n_in <= 128 * kFewSteps * kFewWaves && ceil_div(n_out, 16) <= kMxCus;
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
    MxGemmArgs g{};
    g.x = x_codes;
    g.xs = x_scales;
    g.w = w_codes;
    g.ws = w_scales;
    g.y = static_cast<char*>(y);
    g.rows = rows;
    g.n_out = n_out;
    g.n_in = n_in;
    return mx_gemm_run(x_fmt, dtype, g, workspace, stream);
}

extern "C" size_t polestar_mx_quantize_linear_workspace_size(int x_fmt, polestar_dtype dtype, int batch, int n_rows,
                                                             int n_out, int n_in) {
    using namespace ps;
    if (!mx_fmt_ok(x_fmt) || !dtype_ok(dtype) || batch <= 0 || n_rows <= 0 || n_out <= 0 || n_in <= 0) return 0;
    const long rows = static_cast<long>(batch) * n_rows;
    if (!mx_shape_ok(rows, n_out, n_in) || mx_few_raw(dtype == POLESTAR_BF16, rows, n_out, n_in)) return 0;
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
    if (workspace_bytes < need || (need > 0 && !workspace)) return POLESTAR_ERR_WORKSPACE;
    if (mx_few_raw(dtype == POLESTAR_BF16, rows, n_out, n_in)) {
        MxFewArgs f{};
        f.w = w_codes;
        f.ws = w_scales;
        f.y = static_cast<char*>(y);
        f.rows = rows;
        f.n_out = n_out;
        f.n_in = n_in;
        f.raw = static_cast<const char*>(x);
        f.seq = seq;
        f.row_start = row_start;
        f.n_rows = n_rows;
        return mx_few_run(x_fmt, dtype == POLESTAR_BF16, f, stream);
    }
    uint8_t* codes = static_cast<uint8_t*>(workspace);
    uint8_t* scales = codes + mx_rows_codes(x_fmt, rows, n_in);
    const polestar_status st =
        polestar_mx_quantize(x_fmt, dtype, batch, seq, n_in, row_start, n_rows, x, codes, scales, stream);
    if (st != POLESTAR_OK) return st;
    const size_t used = mx_rows_ws(x_fmt, rows, n_in);
    return polestar_mx_linear(x_fmt, dtype, rows, n_in, n_out, codes, scales, w_codes, w_scales, y,
                              codes + used, workspace_bytes - used, stream);
}

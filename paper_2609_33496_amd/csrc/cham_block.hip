// Block-scaled product Y = (xc xs) (wc ws)^T on the 8-bit matrix cores.
//
//   Y[m][n] = sum_b xs[b][m] ws[n/128][b] sum_{k in b} xc[m][k] wc[n][k]
//
// v_mfma_f32_16x16x128_f8f6f4 contracts one block of 128 at once.  The weights are its first
// operand and the activations its second, so a lane's four results lie in one row of Y (one
// activation scale) and four channels of one weight block (one weight scale): the factor of a
// block is one number per lane and 16 rows.  With binary32 scales each block's product starts
// from zero and is added as acc += factor * product (one v_fma per result, 16 cycles beside the
// 32 of the matrix instruction); with powers of two the instruction applies the scale bytes
// itself and accumulates in place.
#include <algorithm>
#include <type_traits>

#include "cham_block_load.h"
#include "cham_device.h"

namespace cham {
namespace {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef int int4v __attribute__((ext_vector_type(4)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));

constexpr int kBufferFlags = 0x00020000;  // buffer descriptor word 3: 32-bit data, raw

struct BlockArgs {
    const uint8_t* xc;
    const void* xs;
    const uint8_t* wc;
    const void* ws;
    void* Y;
    int64_t ldy;
    int M, N, K, nkb;
    int tm, tn;    // tiles
    int vec;       // rows of Y start at multiples of 16 bytes: 2, of 8 bytes: 1, else 0
};

// How the products of a block are formed.  The 8-bit matrix instructions add groups of 8
// neighbouring k on a grid of 2^(e - 13), e the exponent of the group's largest product, and cut off
// (towards zero) what lies below it; the groups' sums and the blocks' are added in binary32, rounded
// to nearest, with scales that are powers of two as well (all measured).  A group so loses up to 7
// 2^-13 of its largest product: little beside the rounding of a 16-bit result on ordinary data (root
// mean square 3e-5 to 4e-5 of the result), everything beside products that cancel.  Binary32 results, and
// 16-bit ones on request, take the exact route: the codes as half precision (exact) through the f16
// instructions, whose sums lose no more than binary32 does, at half the rate.
enum { kCodes, kCodesPow2, kHalf, kHalfPow2 };
constexpr bool byte_scales(int mode) { return mode == kCodesPow2 || mode == kHalfPow2; }
constexpr bool exact(int mode) { return mode == kHalf || mode == kHalfPow2; }
template <bool BYTES>
struct ScaleOf {
    using type = float;
};
template <>
struct ScaleOf<true> {
    using type = uint8_t;
};
CHAM_DEV float factor(float s) { return s; }
CHAM_DEV float factor(uint8_t e) {  // 2^(e - 127); 255 is NaN
    return __uint_as_float(e == 0 ? 0x400000u : e == 255 ? 0x7fc00000u : (uint32_t)e << 23);
}

// One operand of a lane: 32 codes of a row, in any order of k that both operands share
union Codes {
    int8v v;
    int4v q[2];
    uint32_t u[8];
};
// The same as half precision, 8 codes for each of four f16 instructions
union Halves {
    half8v h[4];
    uint32_t u[16];
};
CHAM_DEV Halves to_half(const Codes& c) {
    Halves r;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        r.u[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c.u[i], 1.0f, false));
        r.u[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c.u[i], 1.0f, true));
    }
    return r;
}
CHAM_DEV const Codes& operand_as(const Codes& c, const Codes*) { return c; }
CHAM_DEV Halves operand_as(const Codes& c, const Halves*) { return to_half(c); }
template <int MODE>
using Operand = typename std::conditional<exact(MODE), Halves, Codes>::type;

CHAM_DEV float4v mfma(const Codes& a, const Codes& b, float4v c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, c, 0, 0, 0, 0, 0, 0);
}
CHAM_DEV float4v mfma_pow2(const Codes& a, const Codes& b, float4v c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, c, 0, 0, 0, sa, 0, sb);
}
CHAM_DEV float4v mfma_half(half8v a, half8v b, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

template <int YT>
CHAM_DEV void store1(void* Y, int64_t i, float v) {
    if constexpr (YT == CHAM_T_F32) ((float*)Y)[i] = v;
    else if constexpr (YT == CHAM_T_F16) ((_Float16*)Y)[i] = (_Float16)v;
    else ((__bf16*)Y)[i] = (__bf16)v;
}

// 4 and 8 consecutive channels of one row of Y
template <int YT>
CHAM_DEV void store4(const BlockArgs& a, int64_t m, int64_t n, float4v p) {
    if (m >= a.M) return;
    const int64_t i = m * a.ldy + n;
    if (a.vec >= (YT == CHAM_T_F32 ? 2 : 1) && n + 4 <= a.N) {
        if constexpr (YT == CHAM_T_F32) *(float4v*)((float*)a.Y + i) = p;
        else *(uint2*)((uint16_t*)a.Y + i) = make_uint2(narrow<YT>(p[0], p[1]), narrow<YT>(p[2], p[3]));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n + j < a.N) store1<YT>(a.Y, i + j, p[j]);
    }
}
template <int YT>
CHAM_DEV void store8(const BlockArgs& a, int64_t m, int64_t n, float4v p, float4v q) {
    const int64_t i = m * a.ldy + n;
    if (a.vec == 1 && YT != CHAM_T_F32 && n + 8 <= a.N) {
        if constexpr (YT != CHAM_T_F32) {
            *(uint2*)((uint16_t*)a.Y + i) = make_uint2(narrow<YT>(p[0], p[1]), narrow<YT>(p[2], p[3]));
            *(uint2*)((uint16_t*)a.Y + i + 4) = make_uint2(narrow<YT>(q[0], q[1]), narrow<YT>(q[2], q[3]));
        }
    } else if (a.vec == 2 && n + 8 <= a.N) {
        if constexpr (YT == CHAM_T_F32) {
            *(float4v*)((float*)a.Y + i) = p;
            *(float4v*)((float*)a.Y + i + 4) = q;
        } else {
            *(uint4*)((uint16_t*)a.Y + i) = make_uint4(narrow<YT>(p[0], p[1]), narrow<YT>(p[2], p[3]), narrow<YT>(q[0], q[1]),
                                                       narrow<YT>(q[2], q[3]));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (n + j < a.N) store1<YT>(a.Y, i + j, j < 4 ? p[j] : q[j - 4]);
    }
}

// ------------------------------------------------------------------------------------
// tiles through LDS
// ------------------------------------------------------------------------------------
// WM x WN wavefronts of (16 TM rows) x (16 TN channels).  A k-step's rows (128 bytes each) go
// from memory to LDS directly (16 bytes a lane), two steps ahead: activations in two buffers (a
// step's operands are in registers before its products begin, so its buffer takes the step after
// next then), weights in three.  The 16-byte chunk c of LDS row r lies at c ^ key(r): the lanes
// that read one chunk of 16 rows in one operand load then spread over all banks (no conflicts
// counted).  The channel order inside a wavefront's block is chosen so that a lane's results of
// two neighbouring operand blocks are 8 consecutive channels of Y.
//
// What bounds it, in tiles of 256 x 256: a step's products hold the matrix cores for 2048 cycles,
// and its LDS traffic (192 KB read, 64 KB written, 128 bytes a cycle) takes as many; the reads of
// the activations at a step's start overlap with no product.  8192 x 8192 x 8192: 437 us with
// binary32 scales (2.51 PFLOP/s, matrix cores busy 64 %), 394 with powers of two (2.79); the
// library's 8-bit product with one scale per tensor 333 (3.30).  Smaller tiles read more LDS per
// product (128 x 128: 64 KB for 512 cycles, 0.49 us a step beside others, 2.3 times its products; 2048
// x 10240 x 1280 33.4 us, 1.61 PFLOP/s); the smallest are bound by the loads into one CU's LDS (about
// 85 bytes a ns).  f16 route, tiles of 64 x 128: a wavefront's step is 32 products, 96 conversions (each
// code is converted in two wavefronts) and 32 scaled additions, so vector work takes as long as the
// products: 8192 x 8192 x 8192 1129 us (0.97 PFLOP/s; the library's bfloat16 product 664), 2048 x 10240 x
// 1280 67.3.  240 x 1152 x 4096 there 11.3 us (144 workgroups on 256 CUs, conversions and LDS latency in
// turn at 0.5 us a step).
//
// bytes of LDS; the address space is part of the type, so that reads of it cannot become others
typedef __attribute__((address_space(3))) uint8_t Lds;

CHAM_DEV int key_x(int r) { return (r >> 1) & 7; }
CHAM_DEV int key_w(int r) { return ((r >> 1) & 1) | ((r >> 3) & 3) << 1; }

// channel (within a run of 32) of operand row rr of the run's first block; 4 more in its second
CHAM_DEV int chan(int rr) { return (rr >> 2) * 8 + (rr & 3); }

// KS groups of WM x WN wavefronts: group q takes the k-steps q, q + KS, ... through buffers of its
// own, and the groups' sums are added in their order at the end.
template <int WM_, int WN_, int TM_, int TN_, int KS_>
struct Tile {
    static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, KS = KS_;
    static constexpr int BM = 16 * TM * WM, BN = 16 * TN * WN, kWaves = WM * WN;
    static constexpr int kLoadsX = BM / 8 / kWaves, kLoadsW = BN / 8 / kWaves;  // 1 KB each
    static constexpr int kLoads = kLoadsX + kLoadsW;
    static constexpr bool kSpread = TM * TN >= 16;  // loads of a step spread over its products
    static constexpr bool kFence = TM * TN >= 8;
    // A wavefront's channels are TN / 2 runs of 32, kRun apart, the first wavefront's from 0, the
    // next one's from kNext.  They are one piece where that lies in one 128-block of the weights'
    // scales; else the wavefronts take the runs in turn, so that each run of all wavefronts together
    // (64 channels) lies in one block, and every run has a scale of its own.
    static constexpr bool kOneBlock = 128 % (16 * TN) == 0;
    static constexpr int kRun = kOneBlock ? 32 : 32 * WN, kNext = kOneBlock ? 16 * TN : 32;
    static constexpr int kSlots = kOneBlock ? 1 : TN / 2;
    static constexpr int chan(int i) { return (i >> 1) * kRun + (i & 1) * 4; }  // of operand block i
    static_assert(kWaves % 4 == 0 && TN % 2 == 0 && BN <= 256 && (kOneBlock || 128 % kRun == 0), "layout");
    static_assert(KS == 1 || BM <= 64, "a group's sums fit its slices of two weight buffers");
};


// Workgroup -> tile.  Workgroups go round the 8 XCDs; each XCD takes a contiguous run of an
// order that walks kGroup tile rows down before it steps to the next tile column, so that the
// tiles an XCD works on at one time share their activation and weight rows in its L2.
constexpr int kGroup = 8;
CHAM_DEV void tile_of(const BlockArgs& a, int& bm, int& bn) {
    const int n = a.tm * a.tn, b = blockIdx.x;
    const int q = n >> 3, r = n & 7, x = b & 7;
    const int i = x * q + min(x, r) + (b >> 3);
    const int gsize = kGroup * a.tn, gi = i / gsize, rows = min(kGroup, a.tm - gi * kGroup), j = i - gi * gsize;
    bn = j / rows;
    bm = gi * kGroup + (j - bn * rows);
}

// The value is used no earlier than here (products of values still in flight would be formed, and
// waited for, where they are loaded).
CHAM_DEV void keep(float& v) { asm volatile("" : "+v"(v)); }
CHAM_DEV void keep(uint8_t& v) {
    uint32_t u = v;
    asm volatile("" : "+v"(u));
    v = (uint8_t)u;
}

// No memory operation moves across it, in the compiler's passes or its scheduler.
CHAM_DEV void order_loads() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Waits until at most N of this wavefront's memory loads (LDS writes among them) are in flight,
// then for the other wavefronts; loads stay in flight across it.
template <int N>
CHAM_DEV void landed_barrier() {
    order_loads();
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4 | 15 << 8);  // vmcnt(N)
    __builtin_amdgcn_s_barrier();
    order_loads();
}
// Waits until this wavefront's LDS reads are in registers, then for the other wavefronts.
CHAM_DEV void read_barrier() {
    order_loads();
    __builtin_amdgcn_s_waitcnt(15 | 3 << 14 | 7 << 4);  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    order_loads();
}

// A wavefront's part of the tile where rows of Y are not aligned: 16 rows at a time pass through
// LDS (16-byte chunks swizzled by the row), so that neighbouring lanes store neighbouring elements
// of a row: 4 bytes each, and where a row starts between two such words its first and last element
// alone.  Each lane storing its own 8 elements one by one took 45.7 us for bfloat16 3001 x 4001 x
// 1280, now 32.9; binary32 67.0, now 45.7.
template <class T, int YT>
CHAM_DEV void store_through_lds(const BlockArgs& a, const float4v (&acc)[T::TN][T::TM], Lds* buf, int64_t m0, int64_t n0,
                                int lane) {
    typedef __attribute__((address_space(3))) int4v Lds16;
    typedef __attribute__((address_space(3))) uint32_t Lds4;
    typedef __attribute__((address_space(3))) uint16_t Lds2;
    constexpr bool kWide = YT == CHAM_T_F32;
    constexpr int kSize = kWide ? 4 : 2, W = 16 * T::TN, kRow = W * kSize;
    constexpr int kMask = kRow / 16 % 8 == 0 ? 7 : 3;
    constexpr int kSeg = T::kOneBlock ? W : 32;          // consecutive channels
    constexpr int P = kWide ? kSeg : kSeg / 2, R = 64 / P;  // lanes a row, rows an instruction
    static_assert(16 * kRow * T::kWaves <= T::BN * BK && 64 % P == 0 && kRow / 16 % (kMask + 1) == 0, "layout");
    const int rr = lane & 15, g = lane >> 4;
    auto at = [&](int row, int e) { return buf + row * kRow + (((e * kSize >> 4) ^ (row & kMask)) << 4) + (e * kSize & 15); };
#pragma unroll
    for (int t = 0; t < T::TM; ++t) {
        order_loads();  // the rows before are in registers
#pragma unroll
        for (int i = 0; i < T::TN; i += 2) {
            const float4v p = acc[i][t], q = acc[i + 1][t];
            const int e = i * 16 + g * 8;
            if constexpr (kWide) {
                *(Lds16*)at(rr, e) = __builtin_bit_cast(int4v, p);
                *(Lds16*)at(rr, e + 4) = __builtin_bit_cast(int4v, q);
            } else {
                *(Lds16*)at(rr, e) = int4v{(int)narrow<YT>(p[0], p[1]), (int)narrow<YT>(p[2], p[3]), (int)narrow<YT>(q[0], q[1]),
                                           (int)narrow<YT>(q[2], q[3])};
            }
        }
        __builtin_amdgcn_wave_barrier();
        order_loads();  // one wavefront's LDS accesses are done in their order
#pragma unroll
        for (int sg = 0; sg < W / kSeg; ++sg) {
            const int64_t n = n0 + sg * T::kRun;
#pragma unroll
            for (int r = 0; r < 16; r += R) {
                const int row = r + lane / P, d = lane % P;
                const int64_t m = m0 + t * 16 + row, i = m * a.ldy + n;
                if constexpr (kWide) {
                    const uint32_t v = *(Lds4*)at(row, sg * kSeg + d);
                    if (m < a.M && n + d < a.N) ((uint32_t*)a.Y)[i + d] = v;
                } else {
                    const int odd = (int)(((uint64_t)(uintptr_t)a.Y / 2 + (uint64_t)i) & 1), e = 2 * d - odd;
                    const uint32_t lo = *(Lds2*)at(row, sg * kSeg + max(e, 0)), hi = *(Lds2*)at(row, sg * kSeg + e + 1);
                    uint16_t* const y = (uint16_t*)a.Y + i + e;
                    if (m < a.M) {
                        if (e >= 0 && n + e + 1 < a.N) *(uint32_t*)y = lo | hi << 16;
                        else if (e < 0 && n < a.N) y[1] = (uint16_t)hi;
                        else if (e >= 0 && n + e < a.N) y[0] = (uint16_t)lo;
                    }
                }
            }
            if constexpr (!kWide) {  // the last element of the rows that start between words
                const int64_t m = m0 + t * 16 + rr, i = m * a.ldy + n + kSeg - 1;
                const uint16_t v = *(Lds2*)at(rr, sg * kSeg + kSeg - 1);
                // its word's lower half: the row's start, an odd number of elements before, is an upper one
                if (g == 0 && (((uint64_t)(uintptr_t)a.Y / 2 + (uint64_t)i) & 1) == 0 && m < a.M && n + kSeg - 1 < a.N)
                    ((uint16_t*)a.Y)[i] = v;
            }
        }
    }
}

template <class T, int MODE, int YT>
__global__ __launch_bounds__(T::kWaves * T::KS * 64, 2) void tile_kernel(BlockArgs a) {
    constexpr int WM = T::WM, TM = T::TM, TN = T::TN, KS = T::KS;
    using Scale = typename ScaleOf<byte_scales(MODE)>::type;
    constexpr int kX = T::BM * BK, kW = T::BN * BK;  // bytes of a step
    __shared__ __align__(16) uint8_t X0[KS * kX], X1[KS * kX];
    __shared__ __align__(16) uint8_t W0[KS * kW], W1[KS * kW], W2[KS * kW];
    const int lane = threadIdx.x & 63, all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = KS > 1 ? all / T::kWaves : 0, wave = all - group * T::kWaves;
    const int wm = wave % WM, wn = wave / WM;
    int bm, bn;
    tile_of(a, bm, bn);
    const int64_t m0 = (int64_t)bm * T::BM, n0 = (int64_t)bn * T::BN;
    const int K = a.K, nkb = a.nkb;

    const int mrows = min((int64_t)T::BM, a.M - m0), nrows = min((int64_t)T::BN, a.N - n0);
    const __amdgpu_buffer_rsrc_t rx =
        __builtin_amdgcn_make_buffer_rsrc((void*)(a.xc + m0 * K), (short)0, mrows * K, kBufferFlags);
    const __amdgpu_buffer_rsrc_t rw =
        __builtin_amdgcn_make_buffer_rsrc((void*)(a.wc + n0 * K), (short)0, nrows * K, kBufferFlags);

    // Load i of a wavefront: rows (i kWaves + wave) 8 .. + 7, lane l the slot l % 8 of row l / 8.
    // The rows of two loads differ by a multiple of 32, so a lane's chunk is the same in all.
    // Rows past the tile's last and chunks past K are outside the buffer: zeros.
    const int r0 = wave * 8 + (lane >> 3);
    const int cx0 = (lane & 7) ^ key_x(r0), cw0 = (lane & 7) ^ key_w(r0);
    uint32_t offx = (uint32_t)r0 * K + cx0 * 16, offw = (uint32_t)r0 * K + cw0 * 16;
    const bool lastx = past_row(nkb, cx0, K), lastw = past_row(nkb, cw0, K);
    const uint32_t rstep = (uint32_t)T::kWaves * 8 * K;
    // load i of a step: its weights first, then its activations
    auto issue = [&](Lds* x, Lds* w, int i, int kb) {
        const bool isx = i >= T::kLoadsW;
        const int j = isx ? i - T::kLoadsW : i;
        const LoadAt at = load_at(isx ? offx : offw, isx ? lastx : lastw, kb, nkb);
        Lds* const to = (isx ? x + group * kX : w + group * kW) + (j * T::kWaves + wave) * 1024;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(isx ? rx : rw, (__attribute__((address_space(3))) void*)to, 16,
                                                 at.lane + j * rstep, at.wave, 0, 0);
    };
    auto issue_all = [&](Lds* x, Lds* w, int kb) {
#pragma unroll
        for (int i = 0; i < T::kLoads; ++i) issue(x, w, i, kb);
    };

    // scales of the lane's rows (one per 16-row block) and of the wavefront's channels
    const int rr = lane & 15, g = lane >> 4;
    constexpr int kSlots = T::kSlots;
    const Scale* wsp[kSlots];
#pragma unroll
    for (int u = 0; u < kSlots; ++u)
        wsp[u] = (const Scale*)a.ws + min((n0 + wn * T::kNext + u * T::kRun) / 128, ((int64_t)a.N - 1) / 128) * nkb;
    struct Factors {
        Scale x[TM], w[kSlots];
    };
    Factors s0, s1;
    auto scales = [&](Factors& s, int kb) {
        // one block's scales from the tile's first row on; zeros past the last row
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
            (void*)((const Scale*)a.xs + (int64_t)min(kb, nkb - 1) * a.M + m0), (short)0, mrows * (int)sizeof(Scale), kBufferFlags);
#pragma unroll
        for (int u = 0; u < kSlots; ++u) {
            const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(
                (void*)(wsp[u] + min(kb, nkb - 1)), (short)0, (int)sizeof(Scale), kBufferFlags);
            if constexpr (byte_scales(MODE)) s.w[u] = __builtin_amdgcn_raw_buffer_load_b8(rb, 0, 0, 0);
            else s.w[u] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rb, 0, 0, 0));
        }
#pragma unroll
        for (int t = 0; t < TM; ++t) {
            const int o = (int)((wm * TM * 16 + rr) * sizeof(Scale) + t * 16 * sizeof(Scale));
            if constexpr (byte_scales(MODE)) s.x[t] = __builtin_amdgcn_raw_buffer_load_b8(rs, o, 0, 0);
            else s.x[t] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rs, o, 0, 0));
        }
    };

    float4v acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = float4v{0.0f, 0.0f, 0.0f, 0.0f};

    // byte offsets of the lane's two chunks: its key is the same in every 16-row block
    const int x0 = group * kX + (wm * TM * 16 + rr) * BK, w0 = group * kW + (wn * T::kNext + chan(rr)) * BK;
    const int xlo = x0 + ((g ^ key_x(rr)) << 4), xhi = x0 + (((g + 4) ^ key_x(rr)) << 4);
    const int wlo = w0 + ((g ^ key_w(chan(rr))) << 4), whi = w0 + (((g + 4) ^ key_w(chan(rr))) << 4);
    auto operand = [&](const Lds* buf, int lo, int hi, int off) {
        Codes o;
        o.q[0] = *(const __attribute__((address_space(3))) int4v*)(buf + lo + off);
        o.q[1] = *(const __attribute__((address_space(3))) int4v*)(buf + hi + off);
        return o;
    };

    // The group's step j: X and W hold it, X and Wn take its step j + 2.
    auto step = [&](Lds* X, const Lds* W, Lds* Wn, Factors& s, int j) {
        const int next = __builtin_amdgcn_readfirstlane((j + 2) * KS + group);
        landed_barrier<T::kLoads + TM + kSlots>();  // step j is there; W of step j - 1 is free
        float f[kSlots][TM];
        Scale cx[TM], cw[kSlots];
#pragma unroll
        for (int u = 0; u < kSlots; ++u) {
            cw[u] = s.w[u];
            keep(cw[u]);
        }
#pragma unroll
        for (int t = 0; t < TM; ++t) {
            cx[t] = s.x[t];
            keep(cx[t]);
#pragma unroll
            for (int u = 0; u < kSlots; ++u)
                if constexpr (MODE != kCodesPow2) f[u][t] = factor(cx[t]) * factor(cw[u]);
        }
        Codes b[TM];
#pragma unroll
        for (int t = 0; t < TM; ++t) b[t] = operand(X, xlo, xhi, t * 16 * BK);
        Codes w[2];
        w[0] = operand(W, wlo, whi, 0);
        asm volatile("" : "+v"(offx), "+v"(offw));  // keeps the sums of issue() from living in registers
        scales(s, next);
        if constexpr (!T::kSpread) {
#pragma unroll
            for (int l = 0; l < T::kLoads; ++l) {
                if (l == T::kLoadsW) read_barrier();
                issue(X, Wn, l, next);
            }
        }
        // Operand block i + 1 is read from LDS while block i is multiplied, and 8-bit products are
        // scaled and added behind later ones, so that no instruction waits for the one before it.
        // The scheduling groups interleave matrix and vector instructions evenly (16 additions
        // behind 4 products left the matrix cores idle in between: 8192 x 8192 x 8192 in 256 x 256
        // tiles 476 us -> 455); the fences keep the compiler from gathering all reads in front (more
        // registers than there are).  Small tiles add in place: each exit of the loop took registers
        // of its own for the sums (64 x 64 with two k groups 145 registers, now 73; 2048 x 10240 x
        // 1280 in such tiles 73.4 us -> 56.6).
        auto add = [&](int i, int t, const float4v& p) {
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[i][t][q] = __builtin_fmaf(p[q], f[i * kSlots / TN][t], acc[i][t][q]);
            if constexpr (!T::kSpread) asm volatile("" : "+v"(acc[i][t]));
        };
        // The loads of step j + 2 go out between the products, a few at a time: all at once they
        // hold up the wavefront until the memory pipe has taken them (1 KB each, 16 cycles or
        // more; the same product 502 us -> 476).
        auto spread = [&](int i) {
            if constexpr (T::kSpread) {
#pragma unroll
                for (int l = i * T::kLoads / TN; l < (i + 1) * T::kLoads / TN; ++l) {
                    if (l == T::kLoadsW) read_barrier();  // X is in registers everywhere
                    issue(X, Wn, l, next);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        const float4v zero = {0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (exact(MODE)) {
            Halves hb[TM];
#pragma unroll
            for (int t = 0; t < TM; ++t) hb[t] = to_half(b[t]);
            float4v d[TM];
#pragma unroll
            for (int i = 0; i < TN; ++i) {
                if (i + 1 < TN) w[(i + 1) & 1] = operand(W, wlo, whi, T::chan(i + 1) * BK);
                const Halves hw = to_half(w[i & 1]);
#pragma unroll
                for (int h = 0; h < 4; ++h)
#pragma unroll
                    for (int t = 0; t < TM; ++t) d[t] = mfma_half(hw.h[h], hb[t].h[h], h == 0 ? zero : d[t]);
#pragma unroll
                for (int t = 0; t < TM; ++t) add(i, t, d[t]);
                if constexpr (T::kFence) __builtin_amdgcn_sched_barrier(0);
                spread(i);
            }
        } else {
            // products between one and its addition: the ring d holds them and the one being formed
            constexpr int kRing = 4, kLag = TN * TM < kRing ? TN * TM : kRing - 1;
            static_assert(kLag < kRing && TN * TM >= kLag, "every product is added once, from the first on");
            float4v d[kRing];
#pragma unroll
            for (int i = 0; i < TN; ++i) {
                if (i + 1 < TN) w[(i + 1) & 1] = operand(W, wlo, whi, T::chan(i + 1) * BK);
#pragma unroll
                for (int t = 0; t < TM; ++t) {
                    const int j = i * TM + t, k = j - kLag;
                    if constexpr (MODE == kCodesPow2) {
                        acc[i][t] = mfma_pow2(w[i & 1], b[t], acc[i][t], cw[i * kSlots / TN], cx[t]);
                    } else {
                        d[j % kRing] = mfma(w[i & 1], b[t], zero);
                        if (k >= 0) add(k / TM, k % TM, d[k % kRing]);
                    }
                }
                if constexpr (MODE == kCodes && T::kFence) {
#pragma unroll
                    for (int t = 0; t < TM; ++t) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
                    }
                }
                if constexpr (T::kFence) __builtin_amdgcn_sched_barrier(0);
                spread(i);
            }
            if constexpr (MODE == kCodes) {
#pragma unroll
                for (int k = TN * TM - kLag; k < TN * TM; ++k) add(k / TM, k % TM, d[k % kRing]);
            }
        }
    };

    Lds *const x_0 = (Lds*)X0, *const x_1 = (Lds*)X1;
    Lds *const w_0 = (Lds*)W0, *const w_1 = (Lds*)W1, *const w_2 = (Lds*)W2;
    // A step's barrier counts the loads of the step behind it, so none may move from one step's to
    // another's.
    scales(s0, group);
    issue_all(x_0, w_0, group);
    order_loads();
    scales(s1, KS + group);
    issue_all(x_1, w_1, KS + group);
    order_loads();
    const int steps = (nkb + KS - 1) / KS;  // the same for all groups: steps past the last block are zeros
    for (int j = 0;; j += 6) {
        step(x_0, w_0, w_2, s0, j);
        if (j + 1 >= steps) break;
        step(x_1, w_1, w_0, s1, j + 1);
        if (j + 2 >= steps) break;
        step(x_0, w_2, w_1, s0, j + 2);
        if (j + 3 >= steps) break;
        step(x_1, w_0, w_2, s1, j + 3);
        if (j + 4 >= steps) break;
        step(x_0, w_1, w_0, s0, j + 4);
        if (j + 5 >= steps) break;
        step(x_1, w_2, w_1, s1, j + 5);
        if (j + 6 >= steps) break;
    }
    landed_barrier<0>();  // no write to LDS outlives the workgroup or meets the sums below
    const int l = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0));  // the lane, in no register till here

    if constexpr (KS > 1) {
        auto part = [&](int q, int i, int t) {  // block (i, t) of this wavefront's counterpart in group q
            float4v* p = (float4v*)((i < TN / 2 ? W0 : W1) + q * kW);
            return p + ((wave * (TN / 2) + i % (TN / 2)) * TM + t) * 64 + l;
        };
        if (group > 0) {
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int t = 0; t < TM; ++t) *part(group, i, t) = acc[i][t];
        }
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int q = 1; q < KS; ++q)
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int t = 0; t < TM; ++t) acc[i][t] += *part(q, i, t);
    }

    // 16-bit rows that start at multiples of 8 bytes are stored directly too (8192 x 2300 x 1280
    // 35.3 us, through LDS 45.4)
    if (a.vec < (YT == CHAM_T_F32 ? 2 : 1)) {
        Lds* const buf = (Lds*)W0 + wave * (16 * 16 * TN * (YT == CHAM_T_F32 ? 4 : 2));
        store_through_lds<T, YT>(a, acc, buf, m0 + wm * TM * 16, n0 + wn * T::kNext, l);
        return;
    }
#pragma unroll
    for (int t = 0; t < TM; ++t) {
        const int64_t m = m0 + (wm * TM + t) * 16 + (l & 15);
        if (m < a.M) {
#pragma unroll
            for (int i = 0; i < TN; i += 2)
                store8<YT>(a, m, n0 + wn * T::kNext + (i >> 1) * T::kRun + (l >> 4) * 8, acc[i][t], acc[i + 1][t]);
        }
    }
}

// ------------------------------------------------------------------------------------
// few rows: operands straight from memory, k split over the workgroup's wavefronts
// ------------------------------------------------------------------------------------
// A workgroup makes 16 TM rows x 16 TN channels; wavefront v of NW takes the k-steps v, v + NW,
// ...  With few rows every weight is read by few workgroups, so LDS would only stand in the way:
// a lane loads its operands of the next step while it multiplies.  The partial sums meet in LDS
// and are added in the order of the wavefronts (no second launch, no atomics).  Bound by the
// weights' bytes and the launch: 1 x 10240 x 1280 4.5 us (13 MB, 2.9 TB/s; 5.3 in a kernel trace).  32
// x 1280 x 5120 6.8 us for 6.7 MB: 160 workgroups, whose eight wavefronts make five steps in turn, each
// a memory latency with one step in flight ahead.
template <int TM, int TN, int NW, int MODE, int YT>
__global__ __launch_bounds__(NW * 64) void few_rows_kernel(BlockArgs a) {
    using Scale = typename ScaleOf<byte_scales(MODE)>::type;
    __shared__ float4v part[NW][TN * TM][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rr = lane & 15, g = lane >> 4, K = a.K, nkb = a.nkb;
    const int64_t m0 = (int64_t)(blockIdx.x % a.tm) * 16 * TM, n0 = (int64_t)(blockIdx.x / a.tm) * 16 * TN;
    const uint8_t *px[TM], *pw[TN];
    const Scale* ps[TM];
#pragma unroll
    for (int t = 0; t < TM; ++t) {
        const int64_t m = min(m0 + t * 16 + rr, (int64_t)a.M - 1);  // past the last row: repeats of it, not written
        px[t] = a.xc + m * K;
        ps[t] = (const Scale*)a.xs + m;
    }
#pragma unroll
    for (int i = 0; i < TN; ++i) pw[i] = a.wc + min(n0 + i * 16 + rr, (int64_t)a.N - 1) * K;
    const Scale* const wsp = (const Scale*)a.ws + n0 / 128 * nkb;  // 16 TN divides 128

    struct Step {
        Codes x[TM], w[TN];
        Scale sx[TM], sw;
    };
    auto load = [&](Step& s, int kb) {
        const int k0 = kb * BK + g * 16, k1 = k0 + 64;  // the lane's two chunks
        const int c0 = min(k0, K - 16), c1 = min(k1, K - 16);
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            s.w[i].q[0] = *(const int4v*)(pw[i] + c0);
            s.w[i].q[1] = *(const int4v*)(pw[i] + c1);
        }
#pragma unroll
        for (int t = 0; t < TM; ++t) {
            s.x[t].q[0] = *(const int4v*)(px[t] + c0);
            s.x[t].q[1] = *(const int4v*)(px[t] + c1);
            s.sx[t] = ps[t][(int64_t)kb * a.M];
        }
        s.sw = wsp[kb];
    };
    float4v acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int t = 0; t < TM; ++t) acc[i][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    auto multiply = [&](Step& s, int kb) {
        if (kb == nkb - 1 && K % BK != 0) {  // chunks past K: zeros in both operands
            const int k0 = kb * BK + g * 16;
            const int4v z = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < TN; ++i) {
                if (k0 >= K) s.w[i].q[0] = z;
                if (k0 + 64 >= K) s.w[i].q[1] = z;
            }
#pragma unroll
            for (int t = 0; t < TM; ++t) {
                if (k0 >= K) s.x[t].q[0] = z;
                if (k0 + 64 >= K) s.x[t].q[1] = z;
            }
        }
        Operand<MODE> b[TM];
#pragma unroll
        for (int t = 0; t < TM; ++t) b[t] = operand_as(s.x[t], (const Operand<MODE>*)nullptr);
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            const Operand<MODE> w = operand_as(s.w[i], (const Operand<MODE>*)nullptr);
#pragma unroll
            for (int t = 0; t < TM; ++t) {
                if constexpr (MODE == kCodesPow2) {
                    acc[i][t] = mfma_pow2(w, b[t], acc[i][t], s.sw, s.sx[t]);
                } else {
                    float4v d = {0.0f, 0.0f, 0.0f, 0.0f};
                    if constexpr (exact(MODE)) {
#pragma unroll
                        for (int h = 0; h < 4; ++h) d = mfma_half(w.h[h], b[t].h[h], d);
                    } else {
                        d = mfma(w, b[t], d);
                    }
                    const float f = factor(s.sx[t]) * factor(s.sw);
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[i][t][q] = __builtin_fmaf(d[q], f, acc[i][t][q]);
                }
            }
        }
    };
    Step s0, s1;
    if (wave < nkb) load(s0, wave);
    for (int kb = wave; kb < nkb; kb += 2 * NW) {
        if (kb + NW < nkb) load(s1, kb + NW);
        multiply(s0, kb);
        if (kb + NW >= nkb) break;
        if (kb + 2 * NW < nkb) load(s0, kb + 2 * NW);
        multiply(s1, kb + NW);
    }
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int t = 0; t < TM; ++t) part[wave][i * TM + t][lane] = acc[i][t];
    __syncthreads();
    for (int e = threadIdx.x; e < TN * TM * 64; e += NW * 64) {
        const int j = e >> 6, l = e & 63;
        float4v y = part[0][j][l];
#pragma unroll
        for (int v = 1; v < NW; ++v) y += part[v][j][l];
        store4<YT>(a, m0 + (j % TM) * 16 + (l & 15), n0 + (j / TM) * 16 + (l >> 4) * 4, y);
    }
}

// ------------------------------------------------------------------------------------
// launches
// ------------------------------------------------------------------------------------
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <class T, int MODE, int YT>
int launch_tile(BlockArgs a, hipStream_t s) {
    a.tm = (int)ceil_div(a.M, T::BM);
    a.tn = (int)ceil_div(a.N, T::BN);
    if (!cham_launchable((int64_t)a.tm * a.tn, T::kWaves * T::KS * 64)) return CHAM_ESHAPE;
    hipLaunchKernelGGL((tile_kernel<T, MODE, YT>), dim3((unsigned)(a.tm * a.tn)), dim3(T::kWaves * T::KS * 64), 0, s, a);
    CHAM_CHECK_LAUNCH();
    return CHAM_OK;
}
template <int TM, int TN, int NW, int MODE, int YT>
int launch_few(BlockArgs a, hipStream_t s) {
    a.tm = (int)ceil_div(a.M, 16 * TM);
    a.tn = (int)ceil_div(a.N, 16 * TN);
    if (!cham_launchable((int64_t)a.tm * a.tn, NW * 64)) return CHAM_ESHAPE;
    hipLaunchKernelGGL((few_rows_kernel<TM, TN, NW, MODE, YT>), dim3((unsigned)(a.tm * a.tn)), dim3(NW * 64), 0, s, a);
    CHAM_CHECK_LAUNCH();
    return CHAM_OK;
}

// Modeled time (us) of one tile shape: the tiles of the busiest CU, each its k-steps and a fixed
// part (first loads, output).  8-bit instructions: a k-step among others is a little faster where
// the last round leaves CUs idle.  Against forced launches of every tile over 39 shapes (M 32 -
// 16384, N 512 - 10240, K 512 - 9216; 3 sets of operands in turn) the choice takes 0.8 % longer than
// the best tile on average and 9 % at worst (16384 x 640 x 640: 14.4 us against 13.2), with scales that
// are powers of two 0.6 % and 8 %, with f16 instructions 0.4 % and 7 % (120 x 4608 x 1152: 7.2 us against
// 6.7).
struct TileCost {
    int bm, bn, ks;
    double lone, step, fixed;  // us: a k-step alone on a CU, among others, and the fixed part
};
enum { kT256, kT192, kT128, kT64, kT64x2, kT32, kT32x2, kTWide, kTiles };
struct Costs {
    TileCost tile[kTiles];
    double idle;  // share of a k-step that a round without tiles would save
};
// 8-bit matrix instructions
constexpr Costs kCostCodes = {{{256, 256, 1, 1.13, 1.48, 7.0}, {256, 192, 1, 0.95, 1.25, 7.5}, {128, 128, 1, 0.535, 0.492, 1.7},
                               {64, 64, 1, 0.28, 0.20, 0.44}, {64, 64, 2, 0.375, 0.37, 1.3},
                               {32, 64, 1, 0.24, 0.138, 0.30}, {32, 64, 2, 0.318, 0.267, 0.82},
                               {0, 0, 0, 0, 0, 0}}, 0.2};
// f16 matrix instructions
constexpr Costs kCostHalf = {{{0, 0, 0, 0, 0, 0}, {0, 0, 0, 0, 0, 0}, {0, 0, 0, 0, 0, 0},
                              {64, 64, 1, 0.409, 0.298, 0.747}, {64, 64, 2, 0.685, 0.596, 1.264},
                              {32, 64, 1, 0.323, 0.192, 0.442}, {32, 64, 2, 0.484, 0.389, 0.99},
                              {64, 128, 1, 0.64, 0.534, 1.524}}, 0.0};

int plan_tile(const BlockArgs& a, const Costs& costs) {
    const int cus = cham_device_cus();
    int best = -1;
    double least = 0.0;
    for (int i = 0; i < kTiles; ++i) {
        const TileCost& c = costs.tile[i];
        if (c.bm == 0) continue;
        const int64_t tiles = ceil_div(a.M, c.bm) * ceil_div(a.N, c.bn), k = ceil_div(tiles, cus);
        const double idle = 1.0 - (double)tiles / (double)(k * cus);  // share of the CUs' rounds without a tile
        const double step = k == 1 ? c.lone : c.step * (1.0 - costs.idle * idle);
        const double t = (double)k * ((double)ceil_div(a.nkb, c.ks) * step + c.fixed);
        if (best < 0 || t < least) { best = i; least = t; }
    }
    return best;
}

// Few rows go without LDS where the launch is at most one workgroup per CU, or where the
// activations' repeated rows cost little, against the tiles of 32 x 64 with two k groups that the plan
// takes else: 1 x 10240 x 1280 4.5 us and 4.7 (f16 route 4.6 and 5.6), 32 x 1280 x 5120 6.8 and 8.4 (6.8
// and 12.9), 48 x 1152 x 4608 6.3 and 7.8; 8 x 10240 x 1280 5.0 and 4.8 (5.1 and 5.7), 16 x 10240 x 1280
// 5.6 and 4.9 (5.7 and 5.8), 17 x 10240 x 1280 8.1 and 4.9 (8.3 and 5.8), 16 x 8192 x 8192 16.9 and 13.7
// (17.1 and 19.1).
bool few_rows(const BlockArgs& a, bool half) {
    return ceil_div(a.M, 16) * ceil_div(a.N, 16) <= cham_device_cus() || a.M <= (half ? 16 : 8);
}

template <int MODE, int YT>
int launch_plan(const BlockArgs& a, hipStream_t s) {
    if (few_rows(a, exact(MODE))) return launch_few<1, 1, 8, MODE, YT>(a, s);
    const int tile = plan_tile(a, exact(MODE) ? kCostHalf : kCostCodes);
    if constexpr (exact(MODE)) {
        if (tile == kTWide) return launch_tile<Tile<2, 2, 2, 4, 1>, MODE, YT>(a, s);
    } else {
        if (tile == kT256) return launch_tile<Tile<4, 2, 4, 8, 1>, MODE, YT>(a, s);
        // three quarters of a 256 x 256 tile: fewer CUs idle in the last round at some widths (8192 x
        // 1152 x 4608 44.9 us against 50.1, 8192 x 1280 x 1280 18.4 against 20.3 in tiles of 128 x 128)
        if (tile == kT192) return launch_tile<Tile<4, 2, 4, 6, 1>, MODE, YT>(a, s);
        if (tile == kT128) return launch_tile<Tile<2, 2, 4, 4, 1>, MODE, YT>(a, s);
    }
    if (tile == kT64) return launch_tile<Tile<2, 2, 2, 2, 1>, MODE, YT>(a, s);
    if (tile == kT64x2) return launch_tile<Tile<2, 2, 2, 2, 2>, MODE, YT>(a, s);
    if (tile == kT32) return launch_tile<Tile<2, 2, 1, 2, 1>, MODE, YT>(a, s);
    return launch_tile<Tile<2, 2, 1, 2, 2>, MODE, YT>(a, s);
}

template <int YT>
int launch_codes(const BlockArgs& a, int pow2, hipStream_t s) {
    return pow2 ? launch_plan<kCodesPow2, YT>(a, s) : launch_plan<kCodes, YT>(a, s);
}
template <int YT>
int launch_half(const BlockArgs& a, int pow2, hipStream_t s) {
    return pow2 ? launch_plan<kHalfPow2, YT>(a, s) : launch_plan<kHalf, YT>(a, s);
}

// y_type without CHAM_T_EXACT, and whether the products take the f16 instructions
bool split_type(int32_t* y_type, bool* half) {
    *half = (*y_type & CHAM_T_EXACT) != 0;
    *y_type &= ~CHAM_T_EXACT;
    *half = *half || *y_type == CHAM_T_F32;
    return *y_type >= 0 && *y_type < CHAM_T_N;
}

// the last row of the last tile is still a 32-bit index
constexpr int64_t kMostRows = ((int64_t)1 << 31) - 257;

int block_check(const cham_bq* x, const cham_bw* w) {
    if (!x || !w || x->M < 0 || w->N < 1 || x->K < 1 || x->K != w->K) return CHAM_EINVAL;
    if (x->K % 32 != 0 || x->K > (1 << 20) || x->M > kMostRows || w->N > kMostRows) return CHAM_ESHAPE;
    if ((x->M > 0 && (!x->codes || !x->scale)) || !w->codes || !w->scale) return CHAM_EINVAL;
    if (((uintptr_t)x->codes & 15u) || ((uintptr_t)w->codes & 15u)) return CHAM_EINVAL;
    if ((!x->pow2 && ((uintptr_t)x->scale & 3u)) || (!w->pow2 && ((uintptr_t)w->scale & 3u))) return CHAM_EINVAL;
    if ((x->pow2 != 0 && x->pow2 != 1) || x->pow2 != w->pow2) return CHAM_EINVAL;
    return CHAM_OK;
}

}  // namespace
}  // namespace cham

using namespace cham;

extern "C" int cham_block_linear(const cham_bq* x, const cham_bw* w, void* Y, int32_t y_type, int64_t ldy,
                                 void* stream) {
    const int rc = block_check(x, w);
    if (rc != CHAM_OK) return rc;
    bool half;
    if (!split_type(&y_type, &half)) return CHAM_EFORMAT;
    const int size = y_type == CHAM_T_F32 ? 4 : 2;
    if (x->M == 0) return CHAM_OK;
    if (!Y || ldy < w->N || (uintptr_t)Y % size) return CHAM_EINVAL;
    BlockArgs a{};
    a.xc = x->codes;
    a.xs = x->scale;
    a.wc = w->codes;
    a.ws = w->scale;
    a.Y = Y;
    a.ldy = ldy;
    a.M = (int)x->M;
    a.N = (int)w->N;
    a.K = (int)x->K;
    a.nkb = (a.K + BK - 1) / BK;
    const uint64_t at = (uint64_t)(uintptr_t)Y | (uint64_t)ldy * size;
    a.vec = at % 16 == 0 ? 2 : at % 8 == 0 ? 1 : 0;
    const hipStream_t s = (hipStream_t)stream;
    if (y_type == CHAM_T_F32) return launch_half<CHAM_T_F32>(a, x->pow2, s);
    if (y_type == CHAM_T_F16) return half ? launch_half<CHAM_T_F16>(a, x->pow2, s) : launch_codes<CHAM_T_F16>(a, x->pow2, s);
    return half ? launch_half<CHAM_T_BF16>(a, x->pow2, s) : launch_codes<CHAM_T_BF16>(a, x->pow2, s);
}

extern "C" int cham_block_linear_plan(int64_t M, int64_t N, int64_t K, int32_t y_type, int32_t* out, int32_t out_len) {
    if (!out || out_len < 3 || M < 1 || N < 1 || K < 1) return CHAM_EINVAL;
    bool half;
    if (!split_type(&y_type, &half)) return CHAM_EFORMAT;
    if (K % 32 != 0 || K > (1 << 20) || M > kMostRows || N > kMostRows) return CHAM_ESHAPE;
    BlockArgs a{};
    a.M = (int)M;
    a.N = (int)N;
    a.K = (int)K;
    a.nkb = (a.K + BK - 1) / BK;
    if (few_rows(a, half)) {
        out[0] = out[1] = 16;
        out[2] = 8;
        return CHAM_OK;
    }
    const Costs& costs = half ? kCostHalf : kCostCodes;
    const TileCost& c = costs.tile[plan_tile(a, costs)];
    out[0] = c.bm;
    out[1] = c.bn;
    out[2] = c.ks;
    return CHAM_OK;
}

// Attention over packed sequences and over a paged cache.
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(s_ij - m_i) / sum_j exp(s_ij - m_i),  s_ij = scale <q_i, k_j>
//
// in one pass over the keys: a running reference m, the sum l and the output's sum o are rescaled
// by exp(m_old - m_new) where m grows.  p does not depend on m, so m need not be the largest score: it
// only has to keep the sums in their types' range, and most steps neither look for a maximum nor
// rescale anything.
//
// The rows of a key head's queries -- G = Hq / Hk heads of each token, token by token -- form one
// matrix, so grouped heads share the keys they read.  Products run transposed: scores as keys
// times queries, so that a lane holds the scores of one query (column), and outputs as values
// times probabilities, whose operand is then the scores' result as it lies in the registers: the
// matrix instructions sum over keys in any order, as long as both operands have the same, and the
// transposing LDS read brings the values in the order in which a lane holds its keys.
//
// The key axis of long sequences is split over workgroups so that all have about the same work;
// partial outputs go to a workspace and a second launch joins them.  Where the split lies follows
// from the lengths, which only the device knows: every workgroup derives it from them.
#include <algorithm>
#include <cmath>

#include "cham_chunk.h"
#include "cham_heads.h"

namespace cham {
namespace {

// Where keys and values come from: rows, 16-bit pages, E4M3 pages.  Probabilities are rounded to 16 bits for
// their product with the values.  Beside 16-bit values they take those's type, and their sum adds the rounded
// ones, so that a key that outweighs the others comes out as it is (bfloat16 errors against 64 bits stay below 1.5
// times those of a binary32 form, 0.0017).  E4M3 values are exact in float16, so there they take
// float16 whatever the queries' type, after the values' scale and a factor of the row's own, which keeps them in
// its range; the sum adds them unrounded (but for float16 outputs of single tokens).
enum { kPacked, kPages, kCodes };

constexpr float kLog2e = 1.44269504f;

// kCodes: what is rounded to float16 is a probability times its value's scale, and what counts among those of a
// row is how they compare with the row's largest, whatever the probabilities and the scales are
// alone (a scale may be anything in binary32).  2^r brings the largest to 2^kTop when it is set, so those down to
// 2^-16 of it keep 11 bits and none above 2^-27 is lost; it falls when one is past float16, 2^14 larger.
// Keys that the row does not see are 0 there and have no say in it; nor have other rows.  Chunks of 1100 new
// tokens over 36000, three draws: 300 to 338 us with 2^6, 295 to 312 with 2^2, 296 to 303 with 1.
constexpr int kTop = 2;
constexpr float kCodesGrow = 20.0f;  // log2 of how far probabilities may be above 1: only binary32 holds them alone
// The next r: of a row whose largest product is w where its reference moves up by `up`, a whole number or
// infinite.  Products behind the move keep their place or fall, so r grows with it at most.
CHAM_DEV int next_r(int r, float up, float w) {
    const int to = min(kTop + 1 - __builtin_amdgcn_frexp_expf(fmaxf(w, FLT_MIN)), 126);
    return up < 512.0f ? min(to, r + (int)up) : to;
}
CHAM_DEV float two_to(int r) { return __uint_as_float((uint32_t)(r + 127) << 23); }  // -126 <= r <= 127

constexpr int kNever = INT32_MAX / 2;  // steps that no sequence has: nothing is cut
constexpr int kRowsTile = 128, kKeysTile = 64;  // of a workgroup of the tiled kernel and its step
constexpr int kRowsFew = 16, kKeysFew = 128;    // of the single-token kernel (4 wavefronts x 32 keys)

struct AttnArgs {
    cham_attn a;
    cham_heads k, v;      // kPacked
    cham_cache c;         // kPages, kCodes
    const int32_t *cu_k, *table, *lens;
    int64_t Tk, width;
    int nq, nk;           // rows of each sequence where cu_q, cu_k are NULL
    int G, Hk;
    int shift;            // log2 of the page
    float c2;             // scale log2(e)
    uint32_t group_mul;   // division by G, see by_group
    int group_shift;
    float share;          // key heads over the pieces that the whole work is cut into
    int least;            // steps of keys a piece has at least
    int most;             // pieces the workspace holds
    float* part_o;        // [piece][rows][D] outputs of pieces
    float* part_s;        // [piece][rows][2] their references and sums
};

struct Piece {
    int q0, nq, k0, nk;   // the sequence's first row and rows, first key and keys
    int tile, first, end; // row tile; steps of keys [first, end)
    int pieces, index;    // pieces of this tile; this piece's place in the workspace
    int seq;
};

// ------------------------------------------------------------------------------------
// the pieces of the work
// ------------------------------------------------------------------------------------
struct Seq {
    int q0, nq, k0, nk;
};
template <int SRC>
CHAM_DEV Seq sequence(const AttnArgs& a, int b) {
    Seq s;
    const int T = (int)a.a.T;
    if (a.a.cu_q) {
        s.q0 = min(max(a.a.cu_q[b], 0), T);
        s.nq = min(max(a.a.cu_q[b + 1], s.q0), T) - s.q0;
    } else {
        s.q0 = b * a.nq;
        s.nq = a.nq;
    }
    if (SRC == kPacked) {
        const int Tk = (int)a.Tk;
        if (a.cu_k) {
            s.k0 = min(max(a.cu_k[b], 0), Tk);
            s.nk = min(max(a.cu_k[b + 1], s.k0), Tk) - s.k0;
        } else {
            s.k0 = b * a.nk;
            s.nk = a.nk;
        }
    } else {
        s.k0 = 0;
        s.nk = (int)min(min((int64_t)max(a.lens[b], 0), a.width << a.shift), kMaxRows);
    }
    return s;
}

CHAM_DEV float max_halves(float v) {  // over lanes l and l ^ 32
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
CHAM_DEV float add_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
CHAM_DEV float max_rows16(float v) {  // over lanes l and l ^ 16
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
CHAM_DEV float add_rows16(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// a value that all lanes share, in scalar registers
CHAM_DEV int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
// the sum of all lanes; in binary32, and the same bits in every lane
CHAM_DEV float wave_total(float v) {
    v += dpp<0xB1>(v);
    v += dpp<0x4E>(v);
    v += dpp<0x141>(v);
    v += dpp<0x140>(v);
    return add_halves(add_rows16(v));
}
CHAM_DEV int wave_scan(int v) {  // inclusive
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, true);  // row 0's last into row 1, 2's into 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, true);  // row 1's last into rows 2 and 3
    return v;
}

// n / G for n < 2^31: with M = ceil(2^(31 + l) / G), 2^(l-1) < G <= 2^l, the error M G - 2^(31 + l) < 2^l
CHAM_DEV int by_group(const AttnArgs& a, int n) { return (int)((uint64_t)(uint32_t)n * a.group_mul >> a.group_shift); }

// Piece `at` of key head `hk` (every wavefront works it out for itself); false past the last one.
// With tiles: `at` counts row tiles, and the piece is the tile's first.  SORT: sequences come in the order
// of their keys, the longest first, where there are at most 64: what starts last is short.
template <int SRC, int BM, int BN, bool SORT>
CHAM_DEV bool find_piece(const AttnArgs& a, int at, int hk, bool tiles, Piece* p) {
    const int lane = threadIdx.x % kWave, B = (int)a.a.B;
    float work = 0.0f;
    Seq s{};
    int nt = 0;
    if (B <= kWave || a.least < kNever) {
#pragma unroll 4
        for (int b0 = 0; b0 < B; b0 += kWave) {
            if (b0 + lane < B) {
                s = sequence<SRC>(a, b0 + lane);
                nt = (s.nq * a.G + BM - 1) / BM;
                work += (float)nt * (float)((s.nk + BN - 1) / BN);
            }
        }
    }
    // more than its share of all steps, however the sum is rounded
    const int steps = max(uniform((int)fminf(wave_total(work) * a.share, 1e9f)) + 1, a.least);
    int before = 0, split_before = 0;
    for (int b0 = 0; b0 < B; b0 += kWave) {
        int n = 0;
        if (B > kWave) {
            nt = 0;
            if (b0 + lane < B) {
                s = sequence<SRC>(a, b0 + lane);
                nt = (s.nq * a.G + BM - 1) / BM;
            }
        }
        if (b0 + lane < B) n = max(1, (int)(((uint32_t)((s.nk + BN - 1) / BN) + (uint32_t)steps - 1) / (uint32_t)steps));
        const int mine = tiles ? nt : nt * n, split = n > 1 ? nt * n : 0;
        int first = 0, split_first = 0;
        if (SORT && B <= kWave) {
            for (int j = 0; j < B; ++j) {
                const int other = __builtin_amdgcn_readlane(s.nk, j);
                const bool ahead = other > s.nk || (other == s.nk && j < lane);
                first += ahead ? __builtin_amdgcn_readlane(mine, j) : 0;
                split_first += ahead ? __builtin_amdgcn_readlane(split, j) : 0;
            }
        } else {
            const int upto = wave_scan(mine), split_upto = wave_scan(split);
            first = before + upto - mine;
            split_first = split_before + split_upto - split;
            before += __builtin_amdgcn_readlane(upto, kWave - 1);
            split_before += __builtin_amdgcn_readlane(split_upto, kWave - 1);
        }
        const uint64_t here = __ballot(first <= at && at < first + mine);
        if (here == 0) continue;
        const int l = __builtin_ctzll(here);
        const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
        p->seq = b0 + l;
        p->q0 = of(s.q0), p->nq = of(s.nq), p->k0 = of(s.k0), p->nk = of(s.nk);
        p->pieces = of(n);
        const int in = at - of(first);  // within the sequence
        const int tile = tiles ? in : (int)((uint32_t)in / (uint32_t)p->pieces), piece = tiles ? 0 : in - tile * p->pieces;
        // the last rows of a causal sequence see the most keys: they come first
        p->tile = of(nt) - 1 - tile;
        const int blocks = (p->nk + BN - 1) / BN, per = (int)(((uint32_t)blocks + p->pieces - 1) / (uint32_t)p->pieces);
        p->first = piece * per;
        p->end = min(blocks, p->first + per);
        p->index = (of(split_first) + tile * p->pieces + piece) * a.Hk + hk;
        return true;
    }
    return false;
}

// ------------------------------------------------------------------------------------
// element types
// ------------------------------------------------------------------------------------
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4v LdsShort4;

template <int T>
CHAM_DEV f16v mma32(u4 a, u4 b, f16v c) {  // 32 x 32 x 16
    if constexpr (T == CHAM_T_F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
}
template <int T>
CHAM_DEV f4 mma16(u4 a, u4 b, f4 c) {  // 16 x 16 x 32
    if constexpr (T == CHAM_T_F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
}

// two E4M3 codes (a word's lower or upper half) in 16 bits; every value is exact
template <int T, bool HI>
CHAM_DEV uint32_t widen2(uint32_t w) {
    if constexpr (T == CHAM_T_F16) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HI));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
}
// c plus two 16-bit values
template <int T>
CHAM_DEV float add2(uint32_t w, float c) {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    if constexpr (T == CHAM_T_F16) return __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, w), half2v{(_Float16)1, (_Float16)1}, c, false);
    else return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf2, w), bf2{(__bf16)1.0f, (__bf16)1.0f}, c, false);
}
template <int T>
CHAM_DEV u4 widen8(uint32_t lo, uint32_t hi) {
    return u4{widen2<T, false>(lo), widen2<T, true>(lo), widen2<T, false>(hi), widen2<T, true>(hi)};
}

CHAM_DEV u4 load16(const char* p) { return *(const u4*)p; }

// four transposed 16-bit values: a lane names 8 bytes of a row of LDS and receives, of the four rows
// that its 16 lanes name, the column of its own place among them
typedef __attribute__((address_space(3))) uint8_t Lds;
CHAM_DEV uint2 read_tr(const Lds* p) { return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4*)p)); }

template <int T>
CHAM_DEV void put4(const cham_heads& o, int64_t at, float a, float b, float c, float d) {
    *(uint2*)((char*)o.p + at * 2) = make_uint2(narrow<T>(a, b), narrow<T>(c, d));
}

// ------------------------------------------------------------------------------------
// the tiled kernel: 128 rows of queries, 32 a wavefront, against steps of 64 keys
// ------------------------------------------------------------------------------------
// KS: steps of 16 along D for the scores, DB: blocks of 32 along D for the outputs.  Keys and values
// lie in LDS as rows of CU chunks of 16 bytes, without gaps, so that 16-bit ones go there from memory
// directly; a chunk's place within its row is swizzled so that neither the 16 rows of a score
// operand nor the four of a transposing read fall on the same banks (no conflicts counted).  Two
// buffers; a step's loads are spread over the products of the step before (issued in one go they held a
// wavefront up for 400 to 600 cycles).
//
// What bounds it, per step of a wavefront and D = 72 / 128: 22 / 32 products of 34 cycles, and about 130
// vector instructions, 600 to 700 cycles with 32 exponentials of 8.6; two workgroups share a CU, and their
// steps together take 2.9 / 4.1 thousand cycles, 1.9 and 2.3 times the products' (matrix cores busy 43 % over
// 2 x 4096 x 4096, 16 heads of 72, bfloat16: 204 us, 758 TFLOP/s; 35 % over seven causal sequences of 8101
// tokens, 32 on 8 heads of 128: 185 us, 752).  A wavefront alone on its SIMD needs as long for one step as two
// for theirs, so it is the chain scores - exponentials - values in each that takes the time; priorities
// (s_setprio), three workgroups a CU and a staggered start changed nothing.  Tiles of ragged causal
// sequences end 18 % after the mean; the search for a piece takes 2 to 3 us of each.  E4M3 pages: 64 more
// products with scales, the row's factor and what finds the largest, the conversions and their way through
// registers make a step 1.5 times as long (1100 new tokens over 36000, 32 on 8 heads of 128: 289 + 23 us, 491 TFLOP/s).
typedef __attribute__((address_space(3))) u4 LdsU4;
typedef __attribute__((address_space(3))) f4 LdsF4;
typedef __attribute__((address_space(3))) float LdsFloat;
constexpr int kBufferFlags = 0x00020000;    // buffer descriptor word 3: 32-bit data, raw
constexpr uint32_t kOutside = 0x80000000u;  // an offset past every buffer: such loads give zeros

// 16 bytes a lane from offset `from` of a buffer into LDS, the wavefront's from `to` on
CHAM_DEV void load_lds(__amdgpu_buffer_rsrc_t b, Lds* to, uint32_t from) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (__attribute__((address_space(3))) void*)to, 16, from, 0, 0, 0);
}

template <int KS, int DB>
struct Tile {
    static constexpr int CU = KS == 4 ? 8 : KS <= 6 ? 12 : 16;
    static constexpr int kBytes = kKeysTile * CU * 16;  // of one buffer
    static constexpr int kLoads = CU / 4;               // of a wavefront's 16 rows, 1 KB each
    // place of chunk c of row r: c ^ key
    static CHAM_DEV int key_k(int r) { return CU == 16 ? r & 15 : CU == 8 ? (r >> 1) & 7 : (r >> 2) & 3; }
    static CHAM_DEV int key_v(int r) { return CU == 16 ? (r & 3) << 2 : CU == 8 ? (r << 1) & 4 : 0; }
};

template <int T, int KS, int DB, int SRC>
__global__ __launch_bounds__(256, 2) void tile_kernel(const AttnArgs a) {
    using L = Tile<KS, DB>;
    constexpr int VT = SRC == kCodes ? CHAM_T_F16 : T;  // of the values' products, see kPacked
    // each buffer a variable of its own: the compiler then knows that a step's reads do not touch what
    // the loads under way write, and does not wait for them
    __shared__ __align__(1024) uint8_t k0[L::kBytes], k1[L::kBytes], v0[L::kBytes], v1[L::kBytes];
    __shared__ __align__(16) float lds_ks[2][kKeysTile], lds_vs[2][kKeysTile];  // kCodes: scales
    const int hk = blockIdx.x % a.Hk;
    Piece p;
    if (!find_piece<SRC, kRowsTile, kKeysTile, true>(a, blockIdx.x / a.Hk, hk, false, &p)) return;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int col = lane & 31, h = lane >> 5, D = a.a.D;
    const int rows = p.nq * a.G, row0 = p.tile * kRowsTile;
    const bool causal = SRC != kPacked || a.a.causal;
    // keys that a row sees: the first `lim`
    const auto limit = [&](int row) { return causal ? min(max(p.nk - p.nq + by_group(a, row) + 1, 0), p.nk) : p.nk; };
    const int my_row = row0 + wave * 32 + col;
    const bool live = row0 + wave * 32 < rows;
    const int lim = my_row < rows ? limit(my_row) : 0;
    // of the wavefront's rows the fewest and the most, and of the tile's the most
    const int lim_lo = uniform(limit(row0 + wave * 32));
    const int lim_hi = uniform(limit(min(row0 + wave * 32 + 31, rows - 1)));
    const int lim_tile = uniform(limit(min(row0 + kRowsTile, rows) - 1));
    const int end = min(p.end, (lim_tile + kKeysTile - 1) / kKeysTile);

    // the queries: second operand of the scores' products
    u4 q[KS];
    const int token = by_group(a, my_row), head = hk * a.G + my_row - token * a.G;
    const int64_t q_at = (int64_t)(p.q0 + token) * a.a.q.token + (int64_t)head * a.a.q.head;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        q[s] = u4{0, 0, 0, 0};
        if (my_row < rows && 16 * s + 8 * h < D) q[s] = load16((const char*)a.a.q.p + (q_at + 16 * s + 8 * h) * 2);
    }

    // A wavefront brings 16 keys of a step, which lie in one page.  16-bit rows go to LDS directly:
    // load i takes the 64 chunks from 64 i on; rows past the last key and chunks past D are outside the
    // buffer and become zeros.  Codes go through registers, where they are widened.
    constexpr int kLoads = SRC == kCodes ? (16 * KS + kWave - 1) / kWave : L::kLoads;
    const int ldk = SRC == kPacked ? (int)(a.k.token * 2) : D * (SRC == kCodes ? 1 : 2);
    const int ldv = SRC == kPacked ? (int)(a.v.token * 2) : ldk;
    uint32_t off_k[kLoads], off_v[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int u = lane + kWave * i;
        if constexpr (SRC == kCodes) {
            const int row = u / KS, c = u % KS;
            off_k[i] = off_v[i] = row < 16 && 16 * c < D ? (uint32_t)(row * ldk + c * 16) : kOutside;
        } else {
            const int row = u / L::CU, ck = (u % L::CU) ^ L::key_k(row), cv = (u % L::CU) ^ L::key_v(row);
            off_k[i] = 8 * ck < D ? (uint32_t)(row * ldk + ck * 16) : kOutside;
            off_v[i] = 8 * cv < D ? (uint32_t)(row * ldv + cv * 16) : kOutside;
        }
    }
    // pages of the next step's keys (one a lane), a step ahead of their use.  No branch guards this load or
    // the scales' (what lies behind the last key is read from the last one's place): at a branch's end the
    // compiler would wait for them.
    const int32_t* table = SRC == kPacked ? nullptr : a.table + (int64_t)p.seq * a.width;
    const auto page_of = [&](int step) { return table[min(step * kKeysTile + lane, p.nk - 1) >> a.shift]; };
    u4 rk[SRC == kCodes ? kLoads : 1], rv[SRC == kCodes ? kLoads : 1];
    float k_scale = 0.0f, v_scale = 0.0f;
    int pages = -1;
    bool held = false;  // the lane's key of the step that is brought has a place
    uint32_t no_page = 0, no_page_next = 0;  // which 16 keys of the step have none
    // What the next step's loads need, kept short: its first key for this wavefront, and the rows' place
    // (kPacked: the place itself, which moves with the steps; pages: that of page 0's first token).
    const int row_bytes = D * (SRC == kCodes ? 1 : 2);
    int key_at = p.first * kKeysTile + 16 * wave;
    const char* kp = SRC == kPacked ? (const char*)a.k.p + ((int64_t)(p.k0 + key_at) * a.k.token + (int64_t)hk * a.k.head) * 2
                                    : (const char*)a.c.k + ((int64_t)hk << a.shift) * row_bytes;
    const char* vp = SRC == kPacked ? (const char*)a.v.p + ((int64_t)(p.k0 + key_at) * a.v.token + (int64_t)hk * a.v.head) * 2
                                    : (const char*)a.c.v + ((int64_t)hk << a.shift) * row_bytes;
    const uint32_t page_bytes = SRC == kPacked ? 0 : (uint32_t)row_bytes << a.shift;  // of one head: below 2^24
    const int full_k = 15 * ldk + row_bytes, full_v = 15 * ldv + row_bytes;
    __amdgpu_buffer_rsrc_t from_k, from_v;
    const auto fetch = [&](int step) __attribute__((always_inline)) {
        const char *k_from = kp, *v_from = vp;
        int size_k = full_k, size_v = full_v;
        if (step >= end) {  // the loads behind the last step bring nothing
            size_k = size_v = 0;
        } else if (key_at + 16 > p.nk) {  // row r < left lies wholly before `size`, row `left` behind it
            const int left = p.nk - key_at;
            size_k = left > 0 ? (left - 1) * ldk + row_bytes : 0;
            size_v = left > 0 ? (left - 1) * ldv + row_bytes : 0;
        }
        if constexpr (SRC == kPacked) {
            kp += (int64_t)kKeysTile * ldk;
            vp += (int64_t)kKeysTile * ldv;
        } else {
            const int key = step * kKeysTile + lane, in_page = key_at & ((1 << a.shift) - 1);
            const bool there = (uint32_t)pages < (uint32_t)a.c.pages;
            held = there && key < p.nk;
            const uint64_t none = __ballot(!there && key < p.nk);
            no_page_next = (none & 1) | (none >> 15 & 2) | (none >> 30 & 4) | (none >> 45 & 8);
            const int page = __builtin_amdgcn_readlane(there ? pages : -1, 16 * wave);
            if (page < 0) size_k = size_v = 0;
            const uint64_t at = (uint64_t)(uint32_t)max(page, 0) * a.Hk * page_bytes + (uint32_t)(in_page * row_bytes);
            k_from += at;
            v_from += at;
            if constexpr (SRC == kCodes) {
                const int64_t row = (((int64_t)(there ? pages : 0) * a.Hk + hk) << a.shift) + (key & ((1 << a.shift) - 1));
                k_scale = a.c.ks[row];
                v_scale = a.c.vs[row];
            }
            pages = page_of(step + 1);
        }
        key_at += kKeysTile;
        from_k = __builtin_amdgcn_make_buffer_rsrc((void*)k_from, (short)0, size_k, kBufferFlags);
        from_v = __builtin_amdgcn_make_buffer_rsrc((void*)v_from, (short)0, size_v, kBufferFlags);
    };
    const auto load_k = [&](int i, Lds* kb) __attribute__((always_inline)) {
        if constexpr (SRC == kCodes) rk[i] = __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(from_k, off_k[i], 0, 0));
        else load_lds(from_k, kb + (wave * L::kLoads + i) * 1024, off_k[i]);
    };
    const auto load_v = [&](int i, Lds* vb) __attribute__((always_inline)) {
        if constexpr (SRC == kCodes) rv[i] = __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(from_v, off_v[i], 0, 0));
        else load_lds(from_v, vb + (wave * L::kLoads + i) * 1024, off_v[i]);
    };
    const auto load_all = [&](Lds* kb, Lds* vb) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            load_k(i, kb);
            load_v(i, vb);
        }
    };
    const auto store = [&](int buf, Lds* kb, Lds* vb) __attribute__((always_inline)) {
        if constexpr (SRC == kCodes) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int u = lane + kWave * i, in = u / KS, c = 2 * (u % KS);
                if (16 * KS % kWave == 0 || in < 16) {
                    const int row = (16 * wave + in) * L::CU;
                    *(LdsU4*)(kb + 16 * (row + (c ^ L::key_k(in)))) = widen8<T>(rk[i][0], rk[i][1]);
                    *(LdsU4*)(kb + 16 * (row + ((c + 1) ^ L::key_k(in)))) = widen8<T>(rk[i][2], rk[i][3]);
                    *(LdsU4*)(vb + 16 * (row + (c ^ L::key_v(in)))) = widen8<VT>(rv[i][0], rv[i][1]);
                    *(LdsU4*)(vb + 16 * (row + ((c + 1) ^ L::key_v(in)))) = widen8<VT>(rv[i][2], rv[i][3]);
                }
            }
            if (wave == 0) *((LdsFloat*)lds_ks[buf] + lane) = held ? k_scale * a.c2 : 0.0f;
            if (wave == 1) *((LdsFloat*)lds_vs[buf] + lane) = held ? v_scale : 0.0f;
        }
    };

    f16v o[DB] = {};
    // the reference (in powers of two; none before a score), and this lane's part of the sum
    float m = -INFINITY, l = 0.0f;
    // kCodes: o is the sum times 2^r, a factor of each row's own
    int r = 0;
    // where the lane reads: row col of the keys, its chunks 2 t + h; rows 4 h + (lane & 15) / 4 of the
    // values, 8 bytes of their chunks 4 d ..
    const int k_at = col * L::CU * 16, k_key = (h ^ L::key_k(col)) << 4;
    const int v_row = 4 * h + ((lane & 15) >> 2);
    const int v_at = v_row * L::CU * 16 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8, v_key = L::key_v(v_row) << 4;

    // The reference is set kAbove powers of two above the largest score and stays until a lane's 32
    // probabilities (bfloat16: all up to here) add up to kBig: where they have not, none is as large.  float16 holds
    // 11 bits of a probability between 2^-14 and 2^16 and nothing below 2^-25, so there the largest is set to 2^2: none
    // above 2^-27 of it is lost, of which 2^15 make half a rounding of the output.  binary32 sums of bfloat16 ones and
    // values hold 24 bits for values from 2^-78 up, and are finite for the largest as the probabilities of a row's two
    // lanes stay below 1/2.  So a reference moves where scores grow by 2^14 (2^17 and more; codes: 2^kCodesGrow).
    // 2 x 4096 x 4096, 16 heads of 72, float16, scores of 4 nats' standard deviation: 221 us with 1, 226 with 2^2, 236
    // with 2^4, 243 with 2^6.
    constexpr float kAbove = T == CHAM_T_F16 ? -2.0f : 24.0f;
    constexpr float kBig = SRC == kCodes ? 0x1p20f : T == CHAM_T_F16 ? 61440.0f : 0.25f;

    // One step's keys against the wavefront's rows; masked: some row does not see all of them.  The
    // outputs' sums are touched in three places only, whatever branch made the probabilities, so that they
    // stay in their registers.
    const auto compute = [&](bool masked, bool bad, int step, int buf, const Lds* keys, const Lds* vals, Lds* next_k,
                             Lds* next_v) __attribute__((always_inline)) {
        const int key0 = step * kKeysTile;
        const Lds *kb = keys + k_at, *vb = vals + v_at;
        // the scores of 32 keys; element i: key 32 b + 8 (i / 4) + 4 h + i % 4
        f16v s[2];
        const auto score = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                s[b] = f16v{};
#pragma unroll
                for (int t = 0; t < KS; ++t) {
                    s[b] = mma32<T>(*(const LdsU4*)(kb + 32 * b * L::CU * 16 + ((t << 5) ^ k_key)), q[t], s[b]);
                    if (SRC != kCodes && b == 0 && t < kLoads) load_k(t, next_k);
                }
                if constexpr (SRC == kCodes) {
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const f4 k4 = *((const LdsF4*)lds_ks[buf] + 8 * b + i / 2 + h);
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[b][i + j] *= k4[j];
                    }
                }
            }
        };
        const int rel = lim - key0 - 4 * h;
        const auto seen = [&](int b, int i) {
            return 32 * b + 2 * (i & ~3) + (i & 3) < rel && !(no_page >> (2 * b + (i >> 3)) & 1);
        };
        const auto mask = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!seen(b, i)) s[b][i] = -INFINITY;
        };
        // their probabilities over the reference, and the lane's sum of them
        u4 pr[4];
        typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
        ushort2v most = {0, 0};  // kCodes: the largest (as integers: none is below 0)
        const auto weigh = [&](float ref, bool hide) __attribute__((always_inline)) {
            float sum[2] = {0.0f, 0.0f};
            const float by = two_to(r);
            most = ushort2v{0, 0};
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    float e[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        e[j] = __builtin_amdgcn_exp2f(SRC == kCodes ? s[b][i + j] - ref : __builtin_fmaf(s[b][i + j], a.c2, -ref));
                        if (SRC == kCodes) sum[j & 1] += e[j];
                    }
                    if constexpr (SRC == kCodes) {
                        const f4 v4 = *((const LdsF4*)lds_vs[buf] + 8 * b + i / 2 + h);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            e[j] = e[j] * v4[j] * by;
                            if (hide && !seen(b, i + j)) e[j] = 0.0f;  // its scale may be anything, NaN too
                        }
                    }
                    uint32_t lo = narrow<VT>(e[0], e[1]), hi = narrow<VT>(e[2], e[3]);
                    if constexpr (SRC == kCodes) asm("" : "+v"(lo), "+v"(hi));  // or the compiler rounds each once more, for `most`
                    const ushort2v l2 = __builtin_bit_cast(ushort2v, lo), h2 = __builtin_bit_cast(ushort2v, hi);
                    if constexpr (SRC != kCodes) sum[0] = add2<T>(hi, add2<T>(lo, sum[0]));
                    else most = __builtin_elementwise_max(most, __builtin_elementwise_max(l2, h2));
                    pr[2 * b + i / 8][i % 8 / 2] = lo;
                    pr[2 * b + i / 8][i % 8 / 2 + 1] = hi;
                }
            return sum[0] + sum[1];
        };
        float sum, f = 1.0f;
        int moved = 0;
        if (masked) {
            asm volatile("; some keys hidden");  // two forms, which the compiler is not to join again
            score();
            mask();
            sum = weigh(m, true);
            asm volatile("; some keys hidden");
        } else {
            asm volatile("; all keys seen");
            score();
            sum = weigh(m, false);
            asm volatile("; all keys seen");
        }
        constexpr bool kAll = SRC != kCodes && T == CHAM_T_BF16;
        bool big = !((kAll ? l + sum : sum) < kBig);  // a probability may be large, or there is no reference yet
        if constexpr (SRC == kCodes) big = big || max((uint32_t)most[0], (uint32_t)most[1]) >= 0x7c00;
        if (__builtin_expect(__any(big), 0)) {
            // every row's reference follows its largest score, and its probabilities with it
            if constexpr (SRC == kCodes) {  // the scores once more: kept until here they would not fit the registers
                asm volatile("" ::: "memory");
                score();
                if (masked) mask();
            }
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(fmaxf(top, s[0][i]), s[1][i]);
            if constexpr (SRC != kCodes) top *= a.c2;
            // (a row's own sums decide, so that no other row's keys change how it rounds)
            const bool mine = max_halves(big ? 1.0f : 0.0f) > 0.0f;
            top = max_halves(top);
            // (codes: whole numbers, so that factors between references are exact)
            float next = mine ? fmaxf(m, SRC == kCodes ? __builtin_ceilf(top) : top + kAbove) : m;
            if constexpr (kAll) {  // those before this step
                const float before = max_halves(l);
                if (mine && before > 0.5f * kBig) next = fmaxf(next, m + kAbove);
            }
            f = next > m ? __builtin_amdgcn_exp2f(m - next) : 1.0f;
            l *= f;
            if constexpr (SRC == kCodes) {
                float w = 0.0f;  // the row's largest product in this step; scales that are not finite have no say
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const f4 v4 = *((const LdsF4*)lds_vs[buf] + 8 * b + i / 2 + h);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float x = fabsf(__builtin_amdgcn_exp2f(s[b][i + j] - (next == -INFINITY ? 0.0f : next)) * v4[j]);
                            w = x < INFINITY ? fmaxf(w, x) : w;
                        }
                    }
                w = max_halves(w);
                const int to = mine ? next_r(r, next - m, w) : r;
                f = __builtin_amdgcn_ldexpf(f, to - r);
                r = to;
            }
            m = next;
            sum = weigh(m == -INFINITY ? 0.0f : m, masked);
            moved = 1;
        }
        l += sum;
        moved = uniform(moved);
        asm volatile("" : "+s"(moved));  // a branch of its own
        if (__builtin_expect(moved, 0)) {
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
        }
        // values of the lane's column of block d, keys as its probabilities lie
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (SRC != kCodes && t < kLoads) load_v(t, next_v);
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const Lds* at = vb + 16 * t * L::CU * 16 + ((64 * d) ^ v_key);
                const uint2 lo = read_tr(at), hi = read_tr(at + 8 * L::CU * 16);
                o[d] = mma32<VT>(u4{lo.x, lo.y, hi.x, hi.y}, pr[t], o[d]);
            }
        }
        if (__builtin_expect(bad, 0)) {
            // Values that are not finite: each row adds those that it sees, from memory (see `clean`).
            constexpr uint32_t inf = VT == CHAM_T_F16 ? 0x7c00u : 0x7f80u;
#pragma unroll 1
            for (int key = key0; key < min(key0 + kKeysTile, p.nk); ++key) {
                const bool see = key < lim && !(no_page >> ((key - key0) >> 4) & 1);
                const char* row;
                if constexpr (SRC == kPacked) {
                    row = (const char*)a.v.p + ((int64_t)(p.k0 + key) * a.v.token + (int64_t)hk * a.v.head) * 2;
                } else {
                    if (no_page >> ((key - key0) >> 4) & 1) continue;
                    const int page = a.table[(int64_t)p.seq * a.width + (key >> a.shift)];
                    const int64_t at = (((int64_t)page * a.Hk + hk) << a.shift) + (key & ((1 << a.shift) - 1));
                    row = (const char*)a.c.v + at * ldv;
                }
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const int e = 32 * d + 2 * i + 4 * h;
                        uint2 w = make_uint2(0, 0);
                        if (e < D) {
                            if constexpr (SRC == kCodes) {
                                const uint32_t c = *(const uint32_t*)(row + e);
                                w = make_uint2(widen2<VT, false>(c), widen2<VT, true>(c));
                            } else {
                                w = *(const uint2*)(row + 2 * e);
                            }
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t x = (j < 2 ? w.x : w.y) >> (16 * (j & 1)) & 0xffffu;
                            // an infinity or a NaN, widened: the exponent is all ones in either type
                            const uint32_t w32 = (x & 0x8000u) << 16 | 0x7f800000u | ((x & 0x7fffu) > inf ? 0x400000u : 0);
                            o[d][i + j] += see && (x & 0x7fffu) >= inf ? __uint_as_float(w32) : 0.0f;
                        }
                    }
            }
        }
    };

    // Values that are not finite among keys that some of the tile's rows do not see, though they exist: 0
    // times such a value would be NaN in those rows.  They are taken out of LDS (each wavefront its own 16
    // keys'), and added apart; the result: whether there are any.
    const auto clean = [&](Lds* vals) __attribute__((always_inline)) {
        constexpr uint32_t carry = VT == CHAM_T_F16 ? 0x04000400u : 0x00800080u;  // an exponent of ones overflows
        bool found = false;
#pragma unroll 1
        for (int i = 0; i < L::CU / 4; ++i) {
            LdsU4* at = (LdsU4*)(vals + wave * 16 * L::CU * 16) + lane + kWave * i;
            u4 w = *at;
            uint32_t all = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t c = ((w[j] & 0x7fff7fffu) + carry) & 0x80008000u;
                all |= c;
                w[j] &= ~((c >> 15) * 0xffffu);
            }
            if (all) *at = w;
            found |= all != 0;
        }
        return uniform(__syncthreads_or(found)) != 0;
    };

    const int lim_first = uniform(limit(row0));
    int step = p.first;
    const auto turn = [&](int buf, Lds* kb, Lds* vb, Lds* next_k, Lds* next_v) __attribute__((always_inline)) {
        __syncthreads();  // this step's keys are there; the other buffer's readers are done
        no_page = no_page_next;
        const int key0 = step * kKeysTile;
        bool bad = false;
        if (lim_first < min(key0 + kKeysTile, p.nk)) bad = clean(vb);
        fetch(step + 1);
        if constexpr (SRC == kCodes) load_all(next_k, next_v);  // into registers: no branch between them and their use
        if (live && key0 < lim_hi) compute(key0 + kKeysTile > lim_lo || no_page, bad, step, buf, kb, vb, next_k, next_v);
        else if constexpr (SRC != kCodes) load_all(next_k, next_v);
        ++step;
    };
    if (step < end) {
        if constexpr (SRC != kPacked) pages = page_of(step);
        fetch(step);
        load_all((Lds*)k0, (Lds*)v0);
        store(0, (Lds*)k0, (Lds*)v0);
    }
    while (step < end) {
        turn(0, (Lds*)k0, (Lds*)v0, (Lds*)k1, (Lds*)v1);
        if constexpr (SRC == kCodes) {
            if (step >= end) break;
            store(1, (Lds*)k1, (Lds*)v1);
            turn(1, (Lds*)k1, (Lds*)v1, (Lds*)k0, (Lds*)v0);
            if (step >= end) break;
            store(0, (Lds*)k0, (Lds*)v0);
        } else if (step < end) {
            turn(1, (Lds*)k1, (Lds*)v1, (Lds*)k0, (Lds*)v0);
        }
    }
    __builtin_amdgcn_s_waitcnt(7 << 4 | 15 << 8);  // vmcnt(0): no load is under way into LDS that another workgroup gets

    if (!live || my_row >= rows || (p.pieces > 1 && (unsigned)p.index >= (unsigned)a.most)) return;
    l = add_halves(l);
    const float f = l == 0.0f ? 0.0f : 1.0f / l;  // before 2^-r: the product stays in range
    m = m == -INFINITY ? 0.0f : m;
    const int64_t o_at = (int64_t)(p.q0 + token) * a.a.o.token + (int64_t)head * a.a.o.head;
    float* po = a.part_o + ((int64_t)p.index * kRowsTile + wave * 32 + col) * D;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int e = 32 * d + 2 * i + 4 * h;
            if (e >= D) continue;
            float y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = SRC == kCodes ? __builtin_amdgcn_ldexpf(o[d][i + j] * f, -r) : o[d][i + j] * f;
            if (p.pieces == 1) put4<T>(a.a.o, o_at + e, y[0], y[1], y[2], y[3]);
            else *(f4*)(po + e) = f4{y[0], y[1], y[2], y[3]};
        }
    if (p.pieces > 1 && h == 0)
        *(float2*)(a.part_s + ((int64_t)p.index * kRowsTile + wave * 32 + col) * 2) = make_float2(m, l);
}

// ------------------------------------------------------------------------------------
// the kernel of single tokens: up to 16 rows (heads of one token), over pages
// ------------------------------------------------------------------------------------
// The cache's bytes bound it.  Each of NW wavefronts takes every NW-th 32 keys of the piece, with no
// wait for the others: keys go from memory into the products' operand as they lie (a lane's 16 bytes
// of a row are a run of D, which only fixes the order of the sum), values through the wavefront's own
// LDS for the transposing read; the next 32 keys' loads are under way meanwhile.  At the end
// they join through LDS.  48 sequences of 200000 tokens, 8 key heads of 128, E4M3 pages of 64: 87 us, 4.8 TB/s
// (a copy reaches 5.1), and 7.6 for the join; 16-bit pages of one sequence of 700 tokens: 12.3, three steps of
// memory latency, 1.7 each, and 7 before and behind them.
template <int ND, int SRC, int NW>
struct Few {
    // rows of values 2 mod 4 chunks apart: 8 rows of 32 bytes fall on different banks
    static constexpr int SV = ND <= 5 ? 10 : ND == 6 ? 14 : 18;
    static constexpr int kKLoads = SRC == kCodes ? (ND + 3) / 4 : (ND + 1) / 2;  // of 16 keys
    static constexpr int kUnits = SRC == kCodes ? ND : 2 * ND;                   // chunks of a row of values
    static constexpr int kVLoads = (32 * kUnits + kWave - 1) / kWave;
    u4 v[NW][32][SV];
    float m[NW][kRowsFew], l[NW][kRowsFew];
    int r[NW][kRowsFew];
};

template <int T, int ND, int SRC, int NW>
__global__ __launch_bounds__(64 * NW, 2) void few_kernel(const AttnArgs a) {
    using L = Few<ND, SRC, NW>;
    constexpr int VT = SRC == kCodes ? CHAM_T_F16 : T;
    constexpr int kKeys = 32 * NW;
    __shared__ L lds;
    const int hk = blockIdx.x % a.Hk;
    Piece p;
    if (!find_piece<SRC, kRowsFew, kKeys, false>(a, blockIdx.x / a.Hk, hk, false, &p)) return;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int col = lane & 15, g = lane >> 4, D = a.a.D;
    const int rows = min(a.G - p.tile * kRowsFew, kRowsFew), head0 = hk * a.G + p.tile * kRowsFew;
    constexpr int kSize = SRC == kCodes ? 1 : 2;

    // the queries, along D as the keys' loads bring it: codes: load i holds d = 64 i + 16 g ..
    // + 15, two steps of the product; 16 bits: d = 32 i + 8 g .. + 7, one
    constexpr int kSteps = SRC == kCodes ? 2 * L::kKLoads : L::kKLoads;
    u4 q[kSteps];
    const int64_t q_at = (int64_t)p.q0 * a.a.q.token + (int64_t)(head0 + col) * a.a.q.head;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int d = SRC == kCodes ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
        q[s] = u4{0, 0, 0, 0};
        if (col < rows && d < D) q[s] = load16((const char*)a.a.q.p + (q_at + d) * 2);
    }

    struct Loads {
        u4 k[2][L::kKLoads], v[L::kVLoads];
        float ks[2][4], vs[2][4];  // scales of the lane's keys: 16 t + 4 g + i
        bool page[2];              // whether the 16 keys have a page
    };
    const int row_bytes = D * kSize;
    const auto fetch = [&](int key0, Loads& r) {
        int64_t at[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = key0 + 16 * t;
            const int page = key < p.nk ? a.table[(int64_t)p.seq * a.width + (key >> a.shift)] : -1;
            r.page[t] = page >= 0 && page < a.c.pages;
            at[t] = ((((int64_t)(r.page[t] ? page : 0) * a.Hk + hk)) << a.shift) + (key & ((1 << a.shift) - 1));
            const char* base = (const char*)a.c.k + at[t] * row_bytes;
#pragma unroll
            for (int i = 0; i < L::kKLoads; ++i) {
                const int byte = 64 * i + 16 * g;
                r.k[t][i] = u4{0, 0, 0, 0};
                if (r.page[t] && key + col < p.nk && byte < row_bytes) r.k[t][i] = load16(base + col * row_bytes + byte);
            }
            if constexpr (SRC == kCodes) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool in = r.page[t] && key + 4 * g + i < p.nk;
                    r.ks[t][i] = in ? a.c.ks[at[t] + 4 * g + i] : 0.0f;
                    r.vs[t][i] = in ? a.c.vs[at[t] + 4 * g + i] : 0.0f;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < L::kVLoads; ++i) {
            const int u = lane + kWave * i, row = u / L::kUnits, c = u % L::kUnits, t = row >> 4;
            r.v[i] = u4{0, 0, 0, 0};
            if (row < 32 && (t ? r.page[1] : r.page[0]) && key0 + row < p.nk && c * 16 < row_bytes)
                r.v[i] = load16((const char*)a.c.v + (t ? at[1] : at[0]) * row_bytes + (row & 15) * row_bytes + c * 16);
        }
    };

    f4 o[ND] = {};
    float m = 0.0f, l = 0.0f;
    bool any = false;
    int r = 0;  // kCodes: o is the sum times 2^r, see kTop
    u4(&vl)[32][L::SV] = lds.v[wave];
    const int end = min(p.end * kKeys, p.nk);
    int key0 = p.first * kKeys + 32 * wave;
    Loads now{};
    if (key0 < end) fetch(key0, now);
    for (; key0 < end; key0 += kKeys) {
        // values into LDS, and the scores, from this step's registers; then the next step's loads
#pragma unroll
        for (int i = 0; i < L::kVLoads; ++i) {
            const int u = lane + kWave * i, row = u / L::kUnits, c = u % L::kUnits;
            if (32 * L::kUnits % kWave == 0 || row < 32) {
                if constexpr (SRC == kCodes) {
                    vl[row][2 * c] = widen8<VT>(now.v[i][0], now.v[i][1]);
                    vl[row][2 * c + 1] = widen8<VT>(now.v[i][2], now.v[i][3]);
                } else {
                    vl[row][c] = now.v[i];
                }
            }
        }
        f4 s[2] = {};
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < L::kKLoads; ++i) {
                const u4 w = now.k[t][i];
                if constexpr (SRC == kCodes) {
                    s[t] = mma16<T>(widen8<T>(w[0], w[1]), q[2 * i], s[t]);
                    s[t] = mma16<T>(widen8<T>(w[2], w[3]), q[2 * i + 1], s[t]);
                } else {
                    s[t] = mma16<T>(w, q[i], s[t]);
                }
            }
        float vs[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (SRC == kCodes) s[t][i] *= now.ks[t][i];
                vs[t][i] = SRC == kCodes ? now.vs[t][i] : 1.0f;
                if (!now.page[t] || key0 + 16 * t + 4 * g + i >= p.nk) s[t][i] = -INFINITY;
            }
        if (key0 + kKeys < end) fetch(key0 + kKeys, now);
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][i]);
        top *= a.c2;
        float e[2][4], w[2][4];  // probabilities; kCodes: times their scales and 2^r
        const auto weigh = [&]() __attribute__((always_inline)) {
            const float by = two_to(r);
            float most = 0.0f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], a.c2, -m));
                    if constexpr (SRC == kCodes) {
                        w[t][i] = e[t][i] * vs[t][i] * by;
                        most = fmaxf(most, fabsf(w[t][i]));
                    }
                }
            return most;
        };
        if constexpr (SRC == kCodes) {
            const bool past = weigh() >= 65520.0f;  // infinite in float16
            const bool big = past || top > m + kCodesGrow || (!any && top > -INFINITY);
            if (__any(big)) {
                const bool mine = max_halves(max_rows16(big ? 1.0f : 0.0f)) > 0.0f;
                top = max_halves(max_rows16(top));
                const float next = mine && top > -INFINITY ? (any ? fmaxf(m, __builtin_ceilf(top)) : __builtin_ceilf(top)) : m;
                float most = 0.0f;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = fabsf(__builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], a.c2, -next)) * vs[t][i]);
                        most = x < INFINITY ? fmaxf(most, x) : most;
                    }
                most = max_halves(max_rows16(most));
                const int to = mine ? next_r(r, any ? next - m : INFINITY, most) : r;
                const float f = any ? __builtin_amdgcn_exp2f(m - next) : 0.0f;
                l *= f;
#pragma unroll
                for (int d = 0; d < ND; ++d) o[d] *= __builtin_amdgcn_ldexpf(f, to - r);
                m = next;
                r = to;
                any = any || top > -INFINITY;
                weigh();
            }
        } else {
            // the largest is set to 2^2 or 2^-16 (see the tiled kernel) and may grow to 2^kGrow; the sum of a row's four
            // lanes stays below 1/2 in bfloat16
            constexpr float kAbove = T == CHAM_T_F16 ? -2.0f : 16.0f, kGrow = T == CHAM_T_F16 ? 15.0f : -8.0f;
            const float full = T == CHAM_T_F16 ? INFINITY : 0x1p-4f;
            const bool big = top > m + kGrow || (!any && top > -INFINITY) || l > full;
            if (__any(big)) {
                // (a row's own scores decide, so that no other head's change how it rounds)
                const bool mine = max_halves(max_rows16(big ? 1.0f : 0.0f)) > 0.0f;
                top = max_halves(max_rows16(top)) + kAbove;
                if (max_halves(max_rows16(l)) > full) top = fmaxf(top, m + kAbove);
                const float f = !mine ? 1.0f : any ? __builtin_amdgcn_exp2f(m - top) : 0.0f;
                m = mine ? top : m;
                any = any || mine;
                l *= f;
#pragma unroll
                for (int d = 0; d < ND; ++d) o[d] *= f;
            }
            weigh();
        }
        u4 pr;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float(&x)[4] = SRC == kCodes ? w[t] : e[t];
            pr[2 * t] = narrow<VT>(x[0], x[1]);
            pr[2 * t + 1] = narrow<VT>(x[2], x[3]);
            if constexpr (SRC != kCodes) {
                l = add2<T>(pr[2 * t + 1], add2<T>(pr[2 * t], l));
            } else if constexpr (T == CHAM_T_F16) {
                // the rounded ones here too, without their scale: one key's rounding would be as large as the
                // output's.  But for those that float16 holds with fewer than 11 bits, or not at all: their products
                // are next to nothing beside the row's largest, which their probabilities may not be.
                const uint32_t p2[2] = {pr[2 * t], pr[2 * t + 1]};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p0 = i & 1 ? f16_hi(p2[i >> 1]) : f16_lo(p2[i >> 1]);
                    l += x[i] >= 0x1p-14f ? e[t][i] * (p0 * __builtin_amdgcn_rcpf(x[i])) : e[t][i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) l += e[t][i];
            }
        }
        // values of column 16 d + (lane & 15): keys 4 g .. + 3 and 16 + 4 g .. + 3
        __builtin_amdgcn_wave_barrier();
        const Lds* at = (const Lds*)&vl[4 * g + (col >> 2)][0] + (col & 3) * 8;
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            const uint2 lo = read_tr(at + 32 * d), hi = read_tr(at + 32 * d + 16 * L::SV * 16);
            o[d] = mma16<VT>(u4{lo.x, lo.y, hi.x, hi.y}, pr, o[d]);
        }
        __builtin_amdgcn_wave_barrier();
    }

    // the wavefronts' sums, each over its own reference: element i of block d is o[4 g + i of block d]
    l = add_halves(add_rows16(l));
    float* mine = (float*)&lds.v[wave][0][0];
#pragma unroll
    for (int d = 0; d < ND; ++d) *(f4*)(mine + col * (16 * ND) + 16 * d + 4 * g) = o[d];
    if (g == 0) {
        lds.m[wave][col] = any ? m : -INFINITY;
        lds.l[wave][col] = l;
        if (SRC == kCodes) lds.r[wave][col] = r;
    }
    __syncthreads();
    if (p.pieces > 1 && (unsigned)p.index >= (unsigned)a.most) return;
    for (int u = threadIdx.x; u < rows * (D / 4); u += 64 * NW) {
        const int row = u / (D / 4), e = u % (D / 4) * 4;
        float top = lds.m[0][row];
#pragma unroll
        for (int w = 1; w < NW; ++w) top = fmaxf(top, lds.m[w][row]);
        float weight[NW], total = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float mw = lds.m[w][row], lw = lds.l[w][row];
            weight[w] = mw > -INFINITY ? __builtin_amdgcn_exp2f(mw - top) : lw != lw ? lw : 0.0f;  // 0: saw no key
            total += weight[w] > 0.0f || weight[w] != weight[w] ? weight[w] * lw : 0.0f;
        }
        const float f = total == 0.0f ? 0.0f : 1.0f / total;
        f4 sum = {};
#pragma unroll
        for (int w = 0; w < NW; ++w)
            if (weight[w] != 0.0f) {
                f4 v = weight[w] * f * *(const f4*)((const float*)&lds.v[w][0][0] + row * (16 * ND) + e);
                if constexpr (SRC == kCodes) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_ldexpf(v[i], -lds.r[w][row]);
                }
                sum += v;
            }
        if (p.pieces == 1) {
            put4<T>(a.a.o, (int64_t)p.q0 * a.a.o.token + (int64_t)(head0 + row) * a.a.o.head + e, sum[0], sum[1], sum[2], sum[3]);
        } else {
            const int64_t r = (int64_t)p.index * kRowsFew + row;
            *(f4*)(a.part_o + r * D + e) = sum;
            if (e == 0) *(float2*)(a.part_s + r * 2) = make_float2(top == -INFINITY ? 0.0f : top, total);
        }
    }
}

// ------------------------------------------------------------------------------------
// joining the pieces of a row tile: o = sum_c w_c o_c / sum_c w_c, w_c = l_c 2^(m_c - max m)
// ------------------------------------------------------------------------------------
// A workgroup takes 8 rows, 32 lanes a row (4 elements a lane); where a tile has fewer, several groups of
// lanes share a row's pieces and are added in their order.  23 us for 1044 pieces of 128 rows of 128 (68 MB);
// one workgroup a tile took 90 for half of them.
constexpr int kRowsJoin = 8;
template <int T, int SRC, int BM, int BN>
__global__ __launch_bounds__(256) void join_kernel(const AttnArgs a) {
    __shared__ float4 sums[kRowsJoin][32];
    __shared__ float2 stats[kRowsJoin];  // reference and total
    const int hk = blockIdx.x % a.Hk;
    Piece p;
    if (!find_piece<SRC, BM, BN, BM == kRowsTile>(a, blockIdx.x / a.Hk, hk, true, &p) || p.pieces == 1) return;
    if ((unsigned)(p.index + (p.pieces - 1) * a.Hk) >= (unsigned)a.most) return;
    const int D = a.a.D, row0 = blockIdx.y * kRowsJoin, rows = min(min(p.nq * a.G - p.tile * BM, BM) - row0, kRowsJoin);
    if (rows <= 0) return;
    const int shift = rows > 4 ? 3 : rows > 2 ? 2 : rows > 1 ? 1 : 0;  // lane groups: 2^shift rows, the rest shares pieces
    const int group = threadIdx.x / 32, e = threadIdx.x % 32 * 4, row = group & ((1 << shift) - 1), part = group >> shift;
    const int parts = 8 >> shift;
    const bool live = row < rows && e < D;
    const int64_t at = (int64_t)p.index * BM + row0 + row, stride = (int64_t)a.Hk * BM;
    // every output is weighed with its share of the whole, so that sums of the largest values stay finite
    float top = -INFINITY, total = 0.0f;
    f4 sum = {};
    if (live) {
#pragma unroll 4
        for (int c = part; c < p.pieces; c += parts) {
            const float2 s = *(const float2*)(a.part_s + (at + c * stride) * 2);
            top = s.y != 0.0f ? fmaxf(top, s.x) : top;
        }
        const auto weight = [&](float2 s) {
            return s.y == 0.0f ? 0.0f : s.y * __builtin_amdgcn_exp2f(s.x - top);  // 0: saw no key, its output is 0
        };
#pragma unroll 4
        for (int c = part; c < p.pieces; c += parts) total += weight(*(const float2*)(a.part_s + (at + c * stride) * 2));
        const float f = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll 4
        for (int c = part; c < p.pieces; c += parts) {
            const f4 v = *(const f4*)(a.part_o + (at + c * stride) * D + e);
            sum += weight(*(const float2*)(a.part_s + (at + c * stride) * 2)) * f * v;
        }
    }
    if (parts > 1) {  // a group's sums are over its own largest reference
        sums[group][threadIdx.x % 32] = make_float4(sum[0], sum[1], sum[2], sum[3]);
        if (threadIdx.x % 32 == 0) stats[group] = make_float2(top, total);
        __syncthreads();
        if (part > 0) return;
        for (int c = 0; c < parts; ++c) top = fmaxf(top, stats[row + (c << shift)].x);
        const auto weight = [&](float2 s) {
            return s.x == top || s.y != s.y ? s.y : s.y == 0.0f ? 0.0f : s.y * __builtin_amdgcn_exp2f(s.x - top);
        };
        total = 0.0f;
        for (int c = 0; c < parts; ++c) total += weight(stats[row + (c << shift)]);
        const float f = total == 0.0f ? 0.0f : 1.0f / total;
        sum = f4{};
        for (int c = 0; c < parts; ++c) {
            const int g = row + (c << shift);
            const float4 v = sums[g][threadIdx.x % 32];
            sum += weight(stats[g]) * f * f4{v.x, v.y, v.z, v.w};
        }
    }
    if (!live) return;
    const int in = p.tile * BM + row0 + row, token = by_group(a, in);
    put4<T>(a.a.o, (int64_t)(p.q0 + token) * a.a.o.token + (int64_t)(hk * a.G + in - token * a.G) * a.a.o.head + e, sum[0], sum[1],
            sum[2], sum[3]);
}

// ------------------------------------------------------------------------------------
// launches
// ------------------------------------------------------------------------------------
// single tokens: one row of queries each, known on the host
bool few_rows(const cham_attn* a) { return !a->cu_q && a->T == a->B; }

// Pieces the work is cut into: four for each CU, of which two (three of the single-token kernel) run at once.
// 1100 new tokens over 36000 cached, two draws: 319 and 335 us a call with two, 294 and 311 with four, 304 and 320 with
// six; 48 single tokens over 200000 95, 97 and 93.
int slots() { return cham_device_cus() * 4; }

struct Space {
    int64_t pieces, rows, bytes;
};
// A tile is cut only where it is longer than a piece, so it has fewer than twice the pieces that its
// work would make: all together at most 2 slots.
Space space(const cham_attn* a, bool few) {
    Space s;
    s.pieces = 2 * (int64_t)slots();
    s.rows = few ? kRowsFew : kRowsTile;
    s.bytes = s.pieces * s.rows * (a->D + 2) * 4;
    return s;
}

int attn_check(const cham_attn* a, int32_t Hk) {
    if (!a || a->B < 0 || a->T < 0 || a->D < 1) return CHAM_EINVAL;
    if (a->D % 8 != 0 || a->D > kMaxD || a->B >= kMaxSeqs || a->T >= kMaxRows) return CHAM_ESHAPE;
    if (!float_type(a->q.type) || a->q.type == CHAM_T_F32 || a->o.type != a->q.type) return CHAM_EFORMAT;
    if (Hk < 1 || a->q.H < 1 || a->q.H % Hk != 0 || a->o.H != a->q.H) return CHAM_EINVAL;
    if (a->causal != 0 && a->causal != 1) return CHAM_EINVAL;
    if (!(a->scale >= FLT_MIN) || a->scale > FLT_MAX / 2) return CHAM_EINVAL;
    if ((uintptr_t)a->cu_q % 4 != 0 || (!a->cu_q && a->B > 0 && a->T % a->B != 0) || (!a->cu_q && a->B == 0 && a->T > 0))
        return CHAM_EINVAL;
    int rc = heads_check(&a->q, a->T, a->D);
    if (rc == CHAM_OK) rc = heads_check(&a->o, a->T, a->D);
    if (rc != CHAM_OK) return rc;
    if (a->T * (a->q.H / Hk) >= kMaxRows) return CHAM_ESHAPE;
    if (a->T > 0 && a->o.p == a->q.p) return CHAM_EINVAL;  // several workgroups read a row of q
    return CHAM_OK;
}

// Grid of the pieces: every tile is a piece, and the cuts make at most `slots` more.
template <int T, int SRC, int KS, int DB, int ND>
int launch(AttnArgs& a, bool few, int64_t tiles, bool may_split, hipStream_t s) {
    const int64_t all = tiles * a.Hk, grid = may_split ? all + slots() : all;
    const int64_t most = may_split ? std::max(grid, all * (few ? kRowsFew : kRowsTile) / kRowsJoin) : grid;
    if (!cham_launchable(most, few && !may_split ? 512 : 256)) return CHAM_ESHAPE;
    if constexpr (SRC != kPacked) {
        if (few) {
            if (may_split) hipLaunchKernelGGL((few_kernel<T, ND, SRC, 4>), dim3((unsigned)grid), dim3(256), 0, s, a);
            else hipLaunchKernelGGL((few_kernel<T, ND, SRC, 8>), dim3((unsigned)grid), dim3(512), 0, s, a);
            CHAM_CHECK_LAUNCH();
            const dim3 join((unsigned)all, a.G > kRowsJoin ? kRowsFew / kRowsJoin : 1);
            if (may_split) hipLaunchKernelGGL((join_kernel<T, SRC, kRowsFew, kKeysFew>), join, dim3(256), 0, s, a);
            CHAM_CHECK_LAUNCH();
            return CHAM_OK;
        }
    }
    hipLaunchKernelGGL((tile_kernel<T, KS, DB, SRC>), dim3((unsigned)grid), dim3(256), 0, s, a);
    CHAM_CHECK_LAUNCH();
    const dim3 join((unsigned)all, kRowsTile / kRowsJoin);
    if (may_split) hipLaunchKernelGGL((join_kernel<T, SRC, kRowsTile, kKeysTile>), join, dim3(256), 0, s, a);
    CHAM_CHECK_LAUNCH();
    return CHAM_OK;
}
template <int T, int SRC>
int launch_d(AttnArgs& a, bool few, int64_t tiles, bool may_split, hipStream_t s) {
    const int D = a.a.D;
    if (D <= 64) return launch<T, SRC, 4, 2, 4>(a, few, tiles, may_split, s);
    if (D <= 80) return launch<T, SRC, 5, 3, 5>(a, few, tiles, may_split, s);
    if (D <= 96) return launch<T, SRC, 6, 3, 6>(a, few, tiles, may_split, s);
    return launch<T, SRC, 8, 4, 8>(a, few, tiles, may_split, s);
}

int64_t up(int64_t n, int64_t d) { return (n + d - 1) / d; }

// nk_most: keys that no sequence has more of
template <int SRC>
int attend(AttnArgs& a, int64_t nk_most, void* ws, size_t ws_bytes, hipStream_t s) {
    const bool few = SRC != kPacked && few_rows(&a.a);
    const int BM = few ? kRowsFew : kRowsTile, BN = few ? kKeysFew : kKeysTile;
    const Space sp = space(&a.a, few);
    if (a.a.T == 0 || a.a.B == 0) return CHAM_OK;
    a.G = a.a.q.H / a.Hk;
    a.nq = (int)(a.a.T / a.a.B);
    a.c2 = a.a.scale * kLog2e;
    a.share = (float)a.Hk / (float)slots() * 1.001f;
    int l = 0;
    while ((1 << l) < a.G) ++l;
    a.group_shift = 31 + l;
    a.group_mul = (uint32_t)((((uint64_t)1 << a.group_shift) + a.G - 1) / a.G);
    a.least = few ? 1 : CHAM_ATTN_NO_WS / kKeysTile;
    a.most = (int)sp.pieces;
    a.part_o = (float*)ws;
    a.part_s = a.part_o + sp.pieces * sp.rows * a.a.D;
    const int64_t tiles = a.a.cu_q ? a.a.T * a.G / BM + a.a.B : a.a.B * up((int64_t)a.nq * a.G, BM);
    const int64_t blocks = up(nk_most, BN);
    bool may_split = blocks > a.least;
    // Tiles that fill the card twice are not cut: the long ones start first, and what a cut saves at the end is
    // less than the partial outputs and the second launch cost (8101 tokens, 2056 tiles: 44 us with nothing
    // to join).  A cache's sequences may be far longer than others: theirs are cut up to four times as many.
    if (!few && a.a.T * a.G / BM * a.Hk >= (int64_t)slots() * (SRC == kPacked ? 1 : 4)) may_split = false;
    // Up to 1024 keys are one piece, of eight wavefronts: a step of theirs takes about 1.7 us, a second launch
    // 4 and 3 more on the host (one sequence of 700 tokens, 8 key heads, 16-bit pages of 16: 12.3 us, in pieces
    // 7.2 and 4.2, which is less only where a graph spares the host).
    if (few && blocks <= CHAM_ATTN_NO_WS_ONE / kKeysFew) may_split = false;
    if (SRC == kPacked && !a.a.cu_q && !a.cu_k)  // every length is known here
        may_split = may_split && blocks > up(tiles * blocks * a.Hk, slots());
    if (!may_split) a.least = kNever;  // the device is to find the same
    if (may_split && (!ws || (uintptr_t)ws % 256 != 0 || ws_bytes < (size_t)sp.bytes)) return CHAM_EWORKSPACE;
    if (a.a.q.type == CHAM_T_F16) return launch_d<CHAM_T_F16, SRC>(a, few, tiles, may_split, s);
    return launch_d<CHAM_T_BF16, SRC>(a, few, tiles, may_split, s);
}

}  // namespace
}  // namespace cham

using namespace cham;

extern "C" size_t cham_attention_workspace_bytes(const cham_attn* a, int32_t Hk) {
    if (attn_check(a, Hk) != CHAM_OK) return 0;
    const size_t few = few_rows(a) ? (size_t)space(a, true).bytes : 0;
    return std::max(few, (size_t)space(a, false).bytes);
}

extern "C" int cham_attention(const cham_attn* a, const cham_heads* k, const cham_heads* v, int64_t Tk, const int32_t* cu_k,
                              void* ws, size_t ws_bytes, void* stream) {
    if (!k || !v || Tk < 0) return CHAM_EINVAL;
    int rc = attn_check(a, k->H);
    if (rc != CHAM_OK) return rc;
    if (v->H != k->H) return CHAM_EINVAL;
    if (k->type != a->q.type || v->type != a->q.type) return CHAM_EFORMAT;
    if (Tk >= kMaxRows) return CHAM_ESHAPE;
    rc = heads_check(k, Tk, a->D);
    if (rc == CHAM_OK) rc = heads_check(v, Tk, a->D);
    if (rc != CHAM_OK) return rc;
    if (Tk > 1 && (k->token >= kMaxStride || v->token >= kMaxStride)) return CHAM_ESHAPE;
    if ((uintptr_t)cu_k % 4 != 0 || (!cu_k && a->B > 0 && Tk % a->B != 0)) return CHAM_EINVAL;
    AttnArgs args{};
    args.a = *a;
    args.k = *k;
    args.v = *v;
    if (Tk <= 1) args.k.token = args.v.token = a->D;  // a single row's stride says nothing
    args.cu_k = cu_k;
    args.Tk = Tk;
    args.nk = a->B > 0 ? (int)(Tk / a->B) : 0;
    args.Hk = k->H;
    return attend<kPacked>(args, cu_k ? Tk : args.nk, ws, ws_bytes, (hipStream_t)stream);
}

extern "C" int cham_cache_attention(const cham_attn* a, const cham_cache* c, const int32_t* table, int64_t width,
                                    const int32_t* lens, void* ws, size_t ws_bytes, void* stream) {
    int rc = cache_check(c);
    if (rc == CHAM_OK) rc = attn_check(a, c->H);
    if (rc != CHAM_OK) return rc;
    if (c->D != a->D || width < 0) return CHAM_EINVAL;
    if (c->type != CHAM_T_E4M3 && c->type != a->q.type) return CHAM_EFORMAT;
    if (width >= (int64_t)1 << 31) return CHAM_ESHAPE;
    if (a->T > 0 && a->B > 0 && (!lens || (uintptr_t)lens % 4 != 0 || (width > 0 && (!table || (uintptr_t)table % 4 != 0))))
        return CHAM_EINVAL;
    AttnArgs args{};
    args.a = *a;
    args.c = *c;
    args.table = table;
    args.width = width;
    args.lens = lens;
    args.Hk = c->H;
    while ((1 << args.shift) < c->page) ++args.shift;
    const int64_t most = std::min(width * c->page, (int64_t)INT32_MAX);
    if (c->type == CHAM_T_E4M3) return attend<kCodes>(args, most, ws, ws_bytes, (hipStream_t)stream);
    return attend<kPages>(args, most, ws, ws_bytes, (hipStream_t)stream);
}

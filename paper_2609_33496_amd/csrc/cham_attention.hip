// Attention over packed sequences and over a paged cache.
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(s_ij - m_i) / sum_j exp(s_ij - m_i),  s_ij = scale <q_i, k_j>
//
// in one pass over the keys: a running reference m, the sum l and the output's sum o are rescaled
// by exp(m_old - m_new) where m grows.  p does not depend on m, so m only follows the largest
// score where that lies more than 2^8 above it, and most steps rescale nothing.
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

enum { kPacked, kPages, kCodes };  // where keys and values come from: rows, 16-bit pages, E4M3 pages

constexpr float kLog2e = 1.44269504f;
constexpr float kGrow = 8.0f;    // the reference follows scores more than 2^8 above it
constexpr float kVGrow = 16.0f;  // and the values' scale follows scales more than 16 times it

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
    int slots;            // pieces the whole work is cut into
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
        s.nk = (int)min((int64_t)max(a.lens[b], 0), a.width << a.shift);
    }
    return s;
}

CHAM_DEV int64_t wave_add(int64_t v) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) v += __shfl_xor((long long)v, d);
    return v;
}
CHAM_DEV int wave_scan(int v, int lane) {  // inclusive
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int o = __shfl_up(v, d);
        v += lane >= d ? o : 0;
    }
    return v;
}

// Piece `at` of key head `hk` (every wavefront works it out for itself); false past the last one.
// With tiles: `at` counts row tiles, and the piece is the tile's first.
template <int SRC, int BM, int BN>
CHAM_DEV bool find_piece(const AttnArgs& a, int at, int hk, bool tiles, Piece* p) {
    const int lane = threadIdx.x % kWave, B = (int)a.a.B;
    int64_t work = 0;
    for (int b0 = 0; b0 < B; b0 += kWave) {
        if (b0 + lane < B) {
            const Seq s = sequence<SRC>(a, b0 + lane);
            work += (int64_t)((s.nq * a.G + BM - 1) / BM) * ((s.nk + BN - 1) / BN);
        }
    }
    work = wave_add(work) * a.Hk;
    const int steps = (int)max((work + a.slots - 1) / a.slots, (int64_t)a.least);
    int before = 0, split_before = 0;
    for (int b0 = 0; b0 < B; b0 += kWave) {
        Seq s{};
        int nt = 0, n = 0;
        if (b0 + lane < B) {
            s = sequence<SRC>(a, b0 + lane);
            nt = (s.nq * a.G + BM - 1) / BM;
            n = max(1, ((s.nk + BN - 1) / BN + steps - 1) / steps);
        }
        const int mine = tiles ? nt : nt * n, split = n > 1 ? nt * n : 0;
        const int upto = wave_scan(mine, lane), split_upto = wave_scan(split, lane);
        const uint64_t past = __ballot(before + upto > at);
        if (past == 0) {
            before += __shfl(upto, kWave - 1);
            split_before += __shfl(split_upto, kWave - 1);
            continue;
        }
        const int l = __builtin_ctzll(past);
        const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
        p->seq = b0 + l;
        p->q0 = of(s.q0), p->nq = of(s.nq), p->k0 = of(s.k0), p->nk = of(s.nk);
        p->pieces = of(n);
        const int in = at - before - (of(upto) - of(mine));  // within the sequence
        const int tile = tiles ? in : in / p->pieces, piece = tiles ? 0 : in - tile * p->pieces;
        // the last rows of a causal sequence see the most keys: they come first
        p->tile = of(nt) - 1 - tile;
        const int blocks = (p->nk + BN - 1) / BN, per = (blocks + p->pieces - 1) / p->pieces;
        p->first = piece * per;
        p->end = min(blocks, p->first + per);
        p->index = (split_before + of(split_upto) - of(split) + tile * p->pieces + piece) * a.Hk + hk;
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
template <int T>
CHAM_DEV u4 widen8(uint32_t lo, uint32_t hi) {
    return u4{widen2<T, false>(lo), widen2<T, true>(lo), widen2<T, false>(hi), widen2<T, true>(hi)};
}

// whether a word's two 16-bit values hold an infinity or a NaN
template <int T>
CHAM_DEV bool not_finite(uint32_t w) {
    constexpr uint32_t e = T == CHAM_T_F16 ? 0x7c00u : 0x7f80u;
    return (w & e) == e || ((w >> 16) & e) == e;
}

CHAM_DEV u4 load16(const char* p) { return *(const u4*)p; }

// four transposed 16-bit values: a lane names 8 bytes of a row of LDS and receives, of the four rows
// that its 16 lanes name, the column of its own place among them
CHAM_DEV uint2 read_tr(const char* p) {
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4*)(__attribute__((address_space(3))) char*)p));
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

template <int T>
CHAM_DEV void put4(const cham_heads& o, int64_t at, float a, float b, float c, float d) {
    *(uint2*)((char*)o.p + at * 2) = make_uint2(narrow<T>(a, b), narrow<T>(c, d));
}

// ------------------------------------------------------------------------------------
// the tiled kernel: 128 rows of queries, 32 a wavefront, against steps of 64 keys
// ------------------------------------------------------------------------------------
// KS: steps of 16 along D for the scores, DB: blocks of 32 along D for the outputs.  Rows of keys lie
// 2 KS + 1 chunks of 16 bytes apart (an odd count: 16 rows fall on 16 different bank groups), rows of
// values SV, 4 mod 8 (a transposing read takes 64 bytes of four rows).
template <int KS, int DB>
struct Tile {
    static constexpr int SK = 2 * KS + 1, SV = DB == 4 ? 20 : 12;
    u4 k[2][kKeysTile][SK];
    u4 v[2][kKeysTile][SV];
    float ks[2][kKeysTile], vs[2][kKeysTile];  // scales of the keys and values
    float vmax[2][4];                          // the largest finite of each 16 values' scales
    int flags[2][4];                           // of each 16 keys: 1 a value is not finite, 2 no page
};

template <int T, int KS, int DB, int SRC>
__global__ __launch_bounds__(256, 2) void tile_kernel(const AttnArgs a) {
    using L = Tile<KS, DB>;
    __shared__ L lds;
    const int hk = blockIdx.x % a.Hk;
    Piece p;
    if (!find_piece<SRC, kRowsTile, kKeysTile>(a, blockIdx.x / a.Hk, hk, false, &p)) return;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int col = lane & 31, h = lane >> 5, D = a.a.D;
    const int rows = p.nq * a.G, row0 = p.tile * kRowsTile;
    const bool causal = SRC != kPacked || a.a.causal;
    // keys that a row sees: the first `lim`
    const auto limit = [&](int row) { return causal ? min(max(p.nk - p.nq + row / a.G + 1, 0), p.nk) : p.nk; };
    const int my_row = row0 + wave * 32 + col, last_row = min(row0 + kRowsTile, rows) - 1;
    const bool live = row0 + wave * 32 < rows;
    const int lim = my_row < rows ? limit(my_row) : 0;
    // of the wavefront's rows the fewest and the most, and of the tile's the most
    const int lim_lo = limit(row0 + wave * 32), lim_hi = limit(min(row0 + wave * 32 + 31, rows - 1));
    const int end = min(p.end, (limit(last_row) + kKeysTile - 1) / kKeysTile);

    // the queries: second operand of the scores' products
    u4 q[KS];
    const int token = my_row / a.G, head = hk * a.G + my_row - token * a.G;
    const int64_t q_at = (int64_t)(p.q0 + token) * a.a.q.token + (int64_t)head * a.a.q.head;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        q[s] = u4{0, 0, 0, 0};
        if (my_row < rows && 16 * s + 8 * h < D) q[s] = load16((const char*)a.a.q.p + (q_at + 16 * s + 8 * h) * 2);
    }

    // staging: a wavefront brings 16 keys of a step
    constexpr int kUnits = SRC == kCodes ? KS : 2 * KS;  // chunks of 16 bytes of a row, those behind D among them
    constexpr int kLoads = (16 * kUnits + kWave - 1) / kWave;
    const int row_units = SRC == kCodes ? D / 16 : D / 8;
    u4 rk[kLoads], rv[kLoads];
    float scale_in = 0.0f;
    int no_page = 0;
    const auto fetch = [&](int step) {
        const int key0 = step * kKeysTile + 16 * wave;
        const char *kp = nullptr, *vp = nullptr;
        int64_t ldk = 0, ldv = 0, at = 0;
        bool in = key0 < p.nk;
        no_page = 0;
        if constexpr (SRC == kPacked) {
            ldk = a.k.token * 2, ldv = a.v.token * 2;
            kp = (const char*)a.k.p + ((int64_t)(p.k0 + key0) * a.k.token + (int64_t)hk * a.k.head) * 2;
            vp = (const char*)a.v.p + ((int64_t)(p.k0 + key0) * a.v.token + (int64_t)hk * a.v.head) * 2;
        } else {
            const int page = in ? a.table[(int64_t)p.seq * a.width + (key0 >> a.shift)] : 0;
            if (page < 0 || page >= a.c.pages) {
                in = false;
                no_page = 2;
            }
            at = (((int64_t)page * a.Hk + hk) << a.shift) + (key0 & ((1 << a.shift) - 1));
            ldk = ldv = D * (SRC == kCodes ? 1 : 2);
            kp = (const char*)a.c.k + at * ldk;
            vp = (const char*)a.c.v + at * ldv;
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int u = lane + kWave * i, row = u / kUnits, c = u % kUnits;
            rk[i] = rv[i] = u4{0, 0, 0, 0};
            if (in && row < 16 && key0 + row < p.nk && c < row_units) {
                rk[i] = load16(kp + row * (int)ldk + c * 16);
                rv[i] = load16(vp + row * (int)ldv + c * 16);
            }
        }
        if constexpr (SRC == kCodes) {
            scale_in = 0.0f;
            if (in && lane < 32 && key0 + (lane & 15) < p.nk) scale_in = (lane < 16 ? a.c.ks : a.c.vs)[at + (lane & 15)];
        }
    };
    const auto store = [&](int step, int buf) {
        bool bad = false;
        const bool look = (step + 1) * kKeysTile > limit(row0);  // some row does not see all of these keys
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int u = lane + kWave * i, row = 16 * wave + u / kUnits, c = u % kUnits;
            if (16 * kUnits % kWave == 0 || u < 16 * kUnits) {
                if constexpr (SRC == kCodes) {
                    const u4 v0 = widen8<T>(rv[i][0], rv[i][1]), v1 = widen8<T>(rv[i][2], rv[i][3]);
                    lds.k[buf][row][2 * c] = widen8<T>(rk[i][0], rk[i][1]);
                    lds.k[buf][row][2 * c + 1] = widen8<T>(rk[i][2], rk[i][3]);
                    lds.v[buf][row][2 * c] = v0;
                    lds.v[buf][row][2 * c + 1] = v1;
                    if (look)
#pragma unroll
                        for (int j = 0; j < 4; ++j) bad |= not_finite<T>(v0[j]) || not_finite<T>(v1[j]);
                } else {
                    lds.k[buf][row][c] = rk[i];
                    lds.v[buf][row][c] = rv[i];
                    if (look)
#pragma unroll
                        for (int j = 0; j < 4; ++j) bad |= not_finite<T>(rv[i][j]);
                }
            }
        }
        if constexpr (SRC == kCodes) {
            if (lane < 16) lds.ks[buf][16 * wave + lane] = scale_in;
            else if (lane < 32) lds.vs[buf][16 * wave + lane - 16] = scale_in;
            uint32_t m = __float_as_uint(scale_in) & 0x7fffffffu;
            m = lane >= 16 && lane < 32 && m < kInfBits ? m : 0;
            m = dpp_maxu<0x140>(dpp_maxu<0x141>(dpp_maxu<0x4E>(dpp_maxu<0xB1>(m))));
            if (lane == 16) lds.vmax[buf][wave] = __uint_as_float(m);
        }
        const int f = (__ballot(bad) != 0 ? 1 : 0) | no_page;
        if (lane == 0) lds.flags[buf][wave] = f;
    };

    f16v o[DB] = {};
    float m = 0.0f, l = 0.0f;   // the reference (in powers of two), and this lane's part of the sum
    bool any = false;           // the reference has been set
    float vref = 0.0f, vinv = 0.0f;  // kCodes: o is the sum over vref
    int step = p.first;
    if (step < end) {
        fetch(step);
        store(step, 0);
    }
    for (int buf = 0; step < end; ++step, buf ^= 1) {
        __syncthreads();  // this step's keys are there; the other buffer's readers are done
        if (step + 1 < end) fetch(step + 1);
        const int key0 = step * kKeysTile;
        if (live && key0 < lim_hi) {
            f16v s[2] = {};
#pragma unroll
            for (int t = 0; t < KS; ++t)
#pragma unroll
                for (int b = 0; b < 2; ++b) s[b] = mma32<T>(lds.k[buf][32 * b + col][2 * t + h], q[t], s[b]);
            // element i of block b: key 32 b + 8 (i / 4) + 4 h + i % 4
            if constexpr (SRC == kCodes) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const f4 k4 = *(const f4*)&lds.ks[buf][32 * b + 2 * i + 4 * h];
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[b][i + j] *= k4[j];
                    }
            }
            int flags = 0;
            {
                const u4 f = *(const u4*)lds.flags[buf];
                flags = __builtin_amdgcn_readfirstlane(f[0] | f[1] << 2 | f[2] << 4 | f[3] << 6);
            }
            const auto seen = [&](int b, int i) {
                return key0 + 32 * b + 2 * (i & ~3) + 4 * h + (i & 3) < lim && !(flags >> (4 * b + (i >> 3) * 2 + 1) & 1);
            };
            const bool masked = key0 + kKeysTile > lim_lo || (flags & 0xaa);
            if (masked) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (!seen(b, i)) s[b][i] = -INFINITY;
            }
            float top = -INFINITY;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
            top *= a.c2;
            if (__any(top > m + kGrow || (!any && top > -INFINITY))) {
                top = max_halves(top);
                if (top > -INFINITY && (!any || top > m)) {
                    const float f = any ? __builtin_amdgcn_exp2f(m - top) : 0.0f;
                    m = top;
                    any = true;
                    l *= f;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[d][i] *= f;
                }
            }
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], a.c2, -m));
                    l += s[b][i];
                }
            if constexpr (SRC == kCodes) {
                const f4 v4 = *(const f4*)lds.vmax[buf];
                const float vm = fmaxf(fmaxf(v4[0], v4[1]), fmaxf(v4[2], v4[3]));
                if (vm > kVGrow * vref) {
                    const float f = vref / fmaxf(vm, FLT_MIN);
                    vref = fmaxf(vm, FLT_MIN);
                    vinv = 1.0f / vref;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[d][i] *= f;
                }
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const f4 k4 = *(const f4*)&lds.vs[buf][32 * b + 2 * i + 4 * h];
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[b][i + j] *= k4[j] * vinv;
                    }
                if (masked) {
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (!seen(b, i)) s[b][i] = 0.0f;
                }
            }
            u4 pr[4];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) pr[t][j] = narrow<T>(s[t >> 1][8 * (t & 1) + 2 * j], s[t >> 1][8 * (t & 1) + 2 * j + 1]);
            // values of the lane's column of block d, keys as its probabilities lie
            const int vr = 4 * h + ((lane & 15) >> 2), vc = ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
            const auto values = [&](int t, int d) {
                const char* at = (const char*)&lds.v[buf][16 * t + vr][4 * d] + vc;
                const uint2 lo = read_tr(at), hi = read_tr(at + 8 * L::SV * 16);
                return u4{lo.x, lo.y, hi.x, hi.y};
            };
            if (!(masked && (flags & 0x55))) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int d = 0; d < DB; ++d) o[d] = mma32<T>(values(t, d), pr[t], o[d]);
            } else {
                // A value that is not finite lies among keys that some rows do not see, and 0 times
                // it would be NaN there.  Such values count as 0, and then as infinities of either
                // sign (NaN as both) for the rows that see them: how many is a product with 0 and 1.
                constexpr uint32_t inf = T == CHAM_T_F16 ? 0x7c00u : 0x7f80u, one = T == CHAM_T_F16 ? 0x3c00u : 0x3f80u;
#pragma unroll 1
                for (int t = 0; t < 4; ++t) {
                    u4 vis, pt;
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (u == t) {
                            pt = pr[u];
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                vis[j] = (seen(u >> 1, 8 * (u & 1) + 2 * j) ? one : 0) | (seen(u >> 1, 8 * (u & 1) + 2 * j + 1) ? one << 16 : 0);
                        }
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        const u4 v = values(t, d);
                        u4 fin, up, down;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            fin[j] = up[j] = down[j] = 0;
#pragma unroll
                            for (int e = 0; e < 32; e += 16) {
                                const uint32_t x = (v[j] >> e) & 0xffffu, mag = x & 0x7fffu;
                                if (mag < inf) fin[j] |= x << e;
                                if (mag > inf || x == inf) up[j] |= one << e;
                                if (mag > inf || x == (inf | 0x8000u)) down[j] |= one << e;
                            }
                        }
                        o[d] = mma32<T>(fin, pt, o[d]);
                        const f16v zero = {}, nu = mma32<T>(up, vis, zero), nd = mma32<T>(down, vis, zero);
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            if (nu[i] > 0.0f) o[d][i] += INFINITY;
                            if (nd[i] > 0.0f) o[d][i] -= INFINITY;
                        }
                    }
                }
            }
        }
        if (step + 1 < end) store(step + 1, buf ^ 1);
    }

    if (!live || my_row >= rows || (p.pieces > 1 && (unsigned)p.index >= (unsigned)a.most)) return;
    l = add_halves(l);
    const float f = l == 0.0f ? 0.0f : (SRC == kCodes ? vref : 1.0f) / l;
    const int64_t o_at = (int64_t)(p.q0 + token) * a.a.o.token + (int64_t)head * a.a.o.head;
    float* po = a.part_o + ((int64_t)p.index * kRowsTile + wave * 32 + col) * D;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int e = 32 * d + 2 * i + 4 * h;
            if (e >= D) continue;
            if (p.pieces == 1) put4<T>(a.a.o, o_at + e, o[d][i] * f, o[d][i + 1] * f, o[d][i + 2] * f, o[d][i + 3] * f);
            else *(f4*)(po + e) = f4{o[d][i] * f, o[d][i + 1] * f, o[d][i + 2] * f, o[d][i + 3] * f};
        }
    if (p.pieces > 1 && h == 0)
        *(float2*)(a.part_s + ((int64_t)p.index * kRowsTile + wave * 32 + col) * 2) = make_float2(m, l);
}

// ------------------------------------------------------------------------------------
// the kernel of single tokens: up to 16 rows (heads of one token), over pages
// ------------------------------------------------------------------------------------
// The cache's bytes bound it.  Each of 4 wavefronts takes every fourth 32 keys of the piece, with no
// wait for the others: keys go from memory into the products' operand as they lie (a lane's 16 bytes
// of a row are a run of D, which only fixes the order of the sum), values through the wavefront's own
// LDS for the transposing read; the next 32 keys' loads are under way meanwhile.  At the end
// the four join through LDS.
template <int ND, int SRC>
struct Few {
    // rows of values 2 mod 4 chunks apart: 8 rows of 32 bytes fall on different banks
    static constexpr int SV = ND <= 5 ? 10 : ND == 6 ? 14 : 18;
    static constexpr int kKLoads = SRC == kCodes ? (ND + 3) / 4 : (ND + 1) / 2;  // of 16 keys
    static constexpr int kUnits = SRC == kCodes ? ND : 2 * ND;                   // chunks of a row of values
    static constexpr int kVLoads = (32 * kUnits + kWave - 1) / kWave;
    u4 v[4][32][SV];
    float m[4][kRowsFew], l[4][kRowsFew];
};

template <int T, int ND, int SRC>
__global__ __launch_bounds__(256, 2) void few_kernel(const AttnArgs a) {
    using L = Few<ND, SRC>;
    __shared__ L lds;
    const int hk = blockIdx.x % a.Hk;
    Piece p;
    if (!find_piece<SRC, kRowsFew, kKeysFew>(a, blockIdx.x / a.Hk, hk, false, &p)) return;
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
    float m = 0.0f, l = 0.0f, vref = 0.0f, vinv = 0.0f;
    bool any = false;
    u4(&vl)[32][L::SV] = lds.v[wave];
    const int end = min(p.end * kKeysFew, p.nk);
    int key0 = p.first * kKeysFew + 32 * wave;
    Loads now{};
    if (key0 < end) fetch(key0, now);
    for (; key0 < end; key0 += kKeysFew) {
        // values into LDS, and the scores, from this step's registers; then the next step's loads
#pragma unroll
        for (int i = 0; i < L::kVLoads; ++i) {
            const int u = lane + kWave * i, row = u / L::kUnits, c = u % L::kUnits;
            if (32 * L::kUnits % kWave == 0 || row < 32) {
                if constexpr (SRC == kCodes) {
                    vl[row][2 * c] = widen8<T>(now.v[i][0], now.v[i][1]);
                    vl[row][2 * c + 1] = widen8<T>(now.v[i][2], now.v[i][3]);
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
        if (key0 + kKeysFew < end) fetch(key0 + kKeysFew, now);
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][i]);
        top *= a.c2;
        if (__any(top > m + kGrow || (!any && top > -INFINITY))) {
            top = max_halves(max_rows16(top));
            if (top > -INFINITY && (!any || top > m)) {
                const float f = any ? __builtin_amdgcn_exp2f(m - top) : 0.0f;
                m = top;
                any = true;
                l *= f;
#pragma unroll
                for (int d = 0; d < ND; ++d) o[d] *= f;
            }
        }
        if constexpr (SRC == kCodes) {
            float vm = 0.0f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = fabsf(vs[t][i]);
                    vm = x < INFINITY ? fmaxf(vm, x) : vm;
                }
            if (__any(vm > kVGrow * vref)) {  // vref is one for the wavefront: its columns share the values
                vm = fmaxf(max_halves(max_rows16(vm)), FLT_MIN);
                const float f = vref / vm;
                vref = vm;
                vinv = 1.0f / vm;
#pragma unroll
                for (int d = 0; d < ND; ++d) o[d] *= f;
            }
        }
        u4 pr;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], a.c2, -m));
                l += e[i];
                if constexpr (SRC == kCodes) e[i] *= vs[t][i] * vinv;
            }
            pr[2 * t] = narrow<T>(e[0], e[1]);
            pr[2 * t + 1] = narrow<T>(e[2], e[3]);
        }
        // values of column 16 d + (lane & 15): keys 4 g .. + 3 and 16 + 4 g .. + 3
        __builtin_amdgcn_wave_barrier();
        const char* at = (const char*)&vl[4 * g + (col >> 2)][0] + (col & 3) * 8;
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            const uint2 lo = read_tr(at + 32 * d), hi = read_tr(at + 32 * d + 16 * L::SV * 16);
            o[d] = mma16<T>(u4{lo.x, lo.y, hi.x, hi.y}, pr, o[d]);
        }
        __builtin_amdgcn_wave_barrier();
    }

    // the wavefronts' sums, each over its own reference: element i of block d is o[4 g + i of block d]
    l = add_halves(add_rows16(l));
    float* mine = (float*)&lds.v[wave][0][0];
    const float back = SRC == kCodes ? vref : 1.0f;
#pragma unroll
    for (int d = 0; d < ND; ++d) *(f4*)(mine + col * (16 * ND) + 16 * d + 4 * g) = o[d] * back;
    if (g == 0) {
        lds.m[wave][col] = any ? m : -INFINITY;
        lds.l[wave][col] = l;
    }
    __syncthreads();
    if (p.pieces > 1 && (unsigned)p.index >= (unsigned)a.most) return;
    for (int u = threadIdx.x; u < rows * (D / 4); u += 256) {
        const int row = u / (D / 4), e = u % (D / 4) * 4;
        float top = lds.m[0][row];
#pragma unroll
        for (int w = 1; w < 4; ++w) top = fmaxf(top, lds.m[w][row]);
        f4 sum = {};
        float total = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = lds.m[w][row] > -INFINITY ? __builtin_amdgcn_exp2f(lds.m[w][row] - top) : 0.0f;
            if (lds.m[w][row] == -INFINITY && !(lds.l[w][row] != lds.l[w][row])) continue;  // saw no key
            total += f * lds.l[w][row];
            sum += f * *(const f4*)((const float*)&lds.v[w][0][0] + row * (16 * ND) + e);
        }
        const float f = total == 0.0f ? 0.0f : 1.0f / total;
        sum *= f;
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
template <int T, int SRC, int BM, int BN>
__global__ __launch_bounds__(256) void join_kernel(const AttnArgs a) {
    const int hk = blockIdx.x % a.Hk;
    Piece p;
    if (!find_piece<SRC, BM, BN>(a, blockIdx.x / a.Hk, hk, true, &p) || p.pieces == 1) return;
    if ((unsigned)(p.index + (p.pieces - 1) * a.Hk) >= (unsigned)a.most) return;
    const int D = a.a.D, rows = min(p.nq * a.G - p.tile * BM, BM);
    for (int u = threadIdx.x; u < rows * (D / 4); u += 256) {
        const int row = u / (D / 4), e = u % (D / 4) * 4;
        float top = -INFINITY;
        for (int c = 0; c < p.pieces; ++c) {
            const float2 s = *(const float2*)(a.part_s + ((int64_t)(p.index + c * a.Hk) * BM + row) * 2);
            if (s.y != 0.0f) top = fmaxf(top, s.x);
        }
        f4 sum = {};
        float total = 0.0f;
        for (int c = 0; c < p.pieces; ++c) {
            const int64_t r = (int64_t)(p.index + c * a.Hk) * BM + row;
            const float2 s = *(const float2*)(a.part_s + r * 2);
            if (s.y == 0.0f) continue;  // saw no key
            const float w = s.y * __builtin_amdgcn_exp2f(s.x - top);
            total += w;
            sum += w * *(const f4*)(a.part_o + r * D + e);
        }
        sum *= total == 0.0f ? 0.0f : 1.0f / total;
        const int at = p.tile * BM + row, token = at / a.G;
        put4<T>(a.a.o, (int64_t)(p.q0 + token) * a.a.o.token + (int64_t)(hk * a.G + at - token * a.G) * a.a.o.head + e, sum[0],
                sum[1], sum[2], sum[3]);
    }
}

// ------------------------------------------------------------------------------------
// launches
// ------------------------------------------------------------------------------------
// single tokens: one row of queries each, known on the host
bool few_rows(const cham_attn* a) { return !a->cu_q && a->T == a->B; }

// Pieces the work is cut into: what the card holds at once.
int slots_of(bool few) { return cham_device_cus() * (few ? 4 : 2); }

struct Space {
    int64_t pieces, rows, bytes;
};
// A tile is cut only where it is longer than a piece, so it has fewer than twice the pieces that its
// work would make: all together at most 2 slots.
Space space(const cham_attn* a, bool few) {
    Space s;
    s.pieces = 2 * (int64_t)slots_of(few);
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
    return CHAM_OK;
}

// Grid of the pieces: every tile is a piece, and the cuts make at most `slots` more.
template <int T, int SRC, int KS, int DB, int ND>
int launch(AttnArgs& a, bool few, int64_t tiles, bool may_split, hipStream_t s) {
    const int64_t all = tiles * a.Hk, grid = may_split ? all + a.slots : all;
    if (!cham_launchable(grid, 256)) return CHAM_ESHAPE;
    if constexpr (SRC != kPacked) {
        if (few) {
            hipLaunchKernelGGL((few_kernel<T, ND, SRC>), dim3((unsigned)grid), dim3(256), 0, s, a);
            CHAM_CHECK_LAUNCH();
            if (may_split) hipLaunchKernelGGL((join_kernel<T, SRC, kRowsFew, kKeysFew>), dim3((unsigned)all), dim3(256), 0, s, a);
            CHAM_CHECK_LAUNCH();
            return CHAM_OK;
        }
    }
    hipLaunchKernelGGL((tile_kernel<T, KS, DB, SRC>), dim3((unsigned)grid), dim3(256), 0, s, a);
    CHAM_CHECK_LAUNCH();
    if (may_split) hipLaunchKernelGGL((join_kernel<T, SRC, kRowsTile, kKeysTile>), dim3((unsigned)all), dim3(256), 0, s, a);
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
    if (!ws || (uintptr_t)ws % 256 != 0 || ws_bytes < (size_t)sp.bytes) return CHAM_EWORKSPACE;
    a.G = a.a.q.H / a.Hk;
    a.nq = (int)(a.a.T / a.a.B);
    a.c2 = a.a.scale * kLog2e;
    a.slots = slots_of(few);
    a.least = few ? 1 : 4;
    a.most = (int)sp.pieces;
    a.part_o = (float*)ws;
    a.part_s = a.part_o + sp.pieces * sp.rows * a.a.D;
    const int64_t tiles = a.a.cu_q ? a.a.T * a.G / BM + a.a.B : a.a.B * up((int64_t)a.nq * a.G, BM);
    const int64_t blocks = up(nk_most, BN);
    bool may_split = blocks > a.least;
    if (SRC == kPacked && !a.a.cu_q && !a.cu_k)  // every length is known here
        may_split = may_split && blocks > up(tiles * blocks * a.Hk, a.slots);
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

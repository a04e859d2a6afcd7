// Row passes that end in 8-bit codes: the residual's addition with the root-mean-square norm,
// the (gated) activation function, and the block quantizer of weights.
//
// All are bound by memory, or by their launch where they are small: each input is read once and
// each output written once (a copy of 1 GiB reaches 5.1 TB/s on this card).  A row is
// held in registers between the reduction that its scale needs and its codes, so nothing is
// read twice; a lane holds chunks of 8 consecutive elements, 16 lanes a block of 128, 4 lanes
// an MX block of 32, and block maxima are DPP rotations within 16 lanes (no LDS).
#include <algorithm>

#include "cham_chunk.h"

namespace cham {
namespace {

constexpr int kRowMax = 32768;

// Stored past the caches: the residual is not read before the block's end, and its lines would
// push out the codes that the next product reads (8192 x 1152, bfloat16 with a binary32 residual:
// 25.9 us -> 21.8; the codes stored the same way too: 19.9, but the block of four operators
// 172 -> 176).
template <int T>
CHAM_DEV void store8(void* p, int64_t i, const float (&v)[kChunk]) {
    typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
    uint4v* q = (uint4v*)at8<T>(p, i);
    if constexpr (T == CHAM_T_F32) {
        __builtin_nontemporal_store(uint4v{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}, q);
        __builtin_nontemporal_store(uint4v{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])}, q + 1);
    } else {
        __builtin_nontemporal_store(uint4v{narrow<T>(v[0], v[1]), narrow<T>(v[2], v[3]), narrow<T>(v[4], v[5]), narrow<T>(v[6], v[7])}, q);
    }
}

// ------------------------------------------------------------------------------------
// activation functions
// ------------------------------------------------------------------------------------
// Relative error: up to 1e-6 and 4e-7 of the exponent's argument (|x| for SiLU, x^2 for GELU,
// 1.6 |x + 0.044715 x^3| for its tanh form), which a rounding of the argument moves by as much.
// Where 1 + 2^v passes 2^126 the reciprocal instruction gives 0 (it has no subnormal results), so
// values below 2^-119 may come out as 0: SiLU below x = -87.3, the tanh form below -9.99.  The root of
// the exponential and a scaled denominator would keep them (8192 x 4608, tanh form, 28.1 us -> 29.8).
constexpr float kLog2e = 1.44269504f;

// x Phi(x).  With z = |x| and q = Phi(-z), it is -z q for x < 0 and x - z q otherwise, so that
// neither tail cancels.  q = exp(-z^2/2) t P(t), t = 1/(1 + 0.36 z), P a polynomial of degree 6
// fitted to the scaled complementary error function by reweighted least squares over
// 0 <= z <= 15 (the polynomial's largest relative error 1.1e-6; half a step of E4M3 is 6e-2).
CHAM_DEV float gelu(float x) {
    const float z = fabsf(x);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(z, 0.36f, 1.0f));
    float p = 0.046524156f;
    p = __builtin_fmaf(p, t, -0.17794086f);
    p = __builtin_fmaf(p, t, 0.178473085f);
    p = __builtin_fmaf(p, t, 0.028252916f);
    p = __builtin_fmaf(p, t, 0.1391006f);
    p = __builtin_fmaf(p, t, 0.14188439f);
    p = __builtin_fmaf(p, t, 0.1437052f);
    const float q = __builtin_amdgcn_exp2f(-0.5f * kLog2e * z * z) * (p * t);
    return __builtin_fmaf(-z, q, fmaxf(x, 0.0f));
}

CHAM_DEV float silu(float x) { return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * x)); }

CHAM_DEV float gelu_tanh(float x) {
    constexpr float c = -2.0f * 0.79788456f * kLog2e;  // 2 sqrt(2/pi) log2(e)
    const float w = x * __builtin_fmaf(x * x, 0.044715f * c, c);
    return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(w));
}

// one branch per chunk (8192 x 4608 with GELU's tanh form 28.4 us; with a branch per element 30.3)
CHAM_DEV void activate(float (&y)[kChunk], int act) {
    if (act == CHAM_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < kChunk; ++j) y[j] = silu(y[j]);
    } else if (act == CHAM_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < kChunk; ++j) y[j] = gelu(y[j]);
    } else if (act == CHAM_ACT_GELU_TANH) {
#pragma unroll
        for (int j = 0; j < kChunk; ++j) y[j] = gelu_tanh(y[j]);
    }
}

// ------------------------------------------------------------------------------------
// scales and codes of a chunk
// ------------------------------------------------------------------------------------
CHAM_DEV uint32_t max16(uint32_t v) {  // over aligned groups of 16 lanes (row rotations)
    return dpp_maxu<0x121>(dpp_maxu<0x122>(dpp_maxu<0x124>(dpp_maxu<0x128>(v))));
}
CHAM_DEV uint32_t max4(uint32_t v) { return dpp_maxu<0x4E>(dpp_maxu<0xB1>(v)); }  // of 4 lanes

template <int FMT>
CHAM_DEV uint2 codes8(const float (&y)[kChunk], float r, float z) {
    return make_uint2(act_codes4<FMT>(make_float4(y[0], y[1], y[2], y[3]), r, z),
                      act_codes4<FMT>(make_float4(y[4], y[5], y[6], y[7]), r, z));
}

// Where a row pass writes
struct Out {
    int64_t M;
    int K;
    int fmt;         // activation format (per token), unused by the block format
    int pow2;        // block format
    uint8_t* codes;  // [M][K]
    void* scale;     // block: [K / 128][M]; per token: float [M]
    float* zero;     // per token: [M]
    uint8_t* e8m0;   // MX: [M][K / 32]
};
enum { kOutBlock, kOutRow, kOutMx };

CHAM_DEV void put_codes(const Out& o, int64_t row, int c, uint2 w) {
    *(uint2*)(o.codes + row * o.K + (int64_t)c * kChunk) = w;
}

// A chunk of a block-format row; the 16 lanes of a block all come here (in: the chunk exists and
// is written; others take no part in the maximum).
CHAM_DEV void emit_block(const Out& o, int64_t row, int c, bool in, const float (&y)[kChunk]) {
    uint32_t stored;
    const float r = block_scale(max16(in ? chunk_amax(y) : 0u), o.pow2 != 0, &stored);
    const uint2 w = codes8_e4m3(y, r);
    if (in) {
        put_codes(o, row, c, w);
        if ((c & 15) == 0) {
            const int64_t i = (int64_t)(c >> 4) * o.M + row;
            if (o.pow2) ((uint8_t*)o.scale)[i] = (uint8_t)stored;
            else ((uint32_t*)o.scale)[i] = stored;
        }
    }
}

// A chunk of an MX row: 4 lanes hold a block of 32, which is whole (K % 32 == 0).  A block that
// holds a NaN or an infinity takes the scale NaN, and MXFP8 codes that are NaN themselves.
CHAM_DEV void emit_mx(const Out& o, int64_t row, int c, bool in, const float (&y)[kChunk]) {
    const uint32_t m = max4(chunk_amax(y));
    const bool bad = m >= kInfBits;
    const int E = mx_exponent(__uint_as_float(m), 0);
    uint2 w;
    if (o.fmt == CHAM_A_MXFP8_E4M3) {
        float v[kChunk];
#pragma unroll
        for (int j = 0; j < kChunk; ++j) v[j] = clampf(ldexpf(y[j], -E), -448.0f, 448.0f);
        w.x = pack_codes<CHAM_A_FP8_E4M3>(v[0], v[1], v[2], v[3], 0.0f);
        w.y = pack_codes<CHAM_A_FP8_E4M3>(v[4], v[5], v[6], v[7], 0.0f);
        if (bad) w = make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu);
    } else {
        uint32_t q[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < kChunk; ++j)
            q[j >> 2] |= ((uint32_t)(int)clampf(rne(ldexpf(y[j], 6 - E)), -127.0f, 127.0f) & 0xFFu) << (8 * (j & 3));
        w = make_uint2(q[0], q[1]);
    }
    if (in) {
        put_codes(o, row, c, w);
        if ((c & 3) == 0) o.e8m0[row * (o.K >> 5) + (c >> 2)] = bad ? (uint8_t)255 : (uint8_t)(E + 127);
    }
}

// ------------------------------------------------------------------------------------
// reductions over the T lanes that hold a row (T = 64: a wavefront; else the workgroup)
// ------------------------------------------------------------------------------------
template <int T, typename V, typename F>
CHAM_DEV V team_reduce(V v, V* sh, F f) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, kWave));
    if constexpr (T > kWave) {
        __syncthreads();  // sh is free again
        if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
        __syncthreads();
        v = sh[0];
#pragma unroll
        for (int i = 1; i < T / kWave; ++i) v = f(v, sh[i]);
    }
    return v;
}

// Lanes per row T, chunks per lane V: rows of up to T V 8 elements.
template <int T>
constexpr int rows_per_wg() { return T == kWave ? 4 : 1; }
template <int T>
constexpr int wg_threads() { return T == kWave ? 256 : T; }
constexpr int kV = 4;

// Codes of the row y (chunks v T + lane) in the per-token formats.
template <int T>
CHAM_DEV void emit_row(const Out& o, int64_t row, bool live, int lane, int nch, const float (&y)[kV][kChunk], void* sh) {
    float s, z = 0.0f;
    uint32_t m = 0;
    float lo = INFINITY, hi = -INFINITY;
#pragma unroll
    for (int v = 0; v < kV; ++v) {
        if (v * T < nch) {
            if (v * T + lane < nch) {
                const uint32_t a = chunk_amax(y[v]);
                m = m > a ? m : a;
#pragma unroll
                for (int j = 0; j < kChunk; ++j) {
                    lo = fminf(lo, y[v][j]);
                    hi = fmaxf(hi, y[v][j]);
                }
            }
        }
    }
    m = team_reduce<T>(m, (uint32_t*)sh, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
    const float amax = __uint_as_float(m);
    if (o.fmt == CHAM_A_INT8_ASYM) {
        lo = team_reduce<T>(lo, (float*)sh, [](float a, float b) { return fminf(a, b); });
        hi = team_reduce<T>(hi, (float*)sh, [](float a, float b) { return fmaxf(a, b); });
        int_asym_scale_zp(lo, hi, 255.0f, &s, &z);
    } else {
        s = floor_scale(amax / (o.fmt == CHAM_A_FP8_E4M3 ? 448.0f : 57344.0f));
    }
    const float r = 1.0f / s;
    if (m >= kInfBits) s = __uint_as_float(0x7fc00000u);
    if (live && lane == 0) {
        ((float*)o.scale)[row] = s;
        o.zero[row] = z;
    }
#pragma unroll
    for (int v = 0; v < kV; ++v) {
        const int c = v * T + lane;
        if (live && c < nch) {
            if (o.fmt == CHAM_A_INT8_ASYM) put_codes(o, row, c, codes8<CHAM_A_INT8_ASYM>(y[v], r, z));
            else if (o.fmt == CHAM_A_FP8_E4M3) put_codes(o, row, c, codes8_e4m3(y[v], r));
            else put_codes(o, row, c, codes8<CHAM_A_FP8_E5M2>(y[v], r, z));
        }
    }
}

template <int T, int OUT>
CHAM_DEV void emit(const Out& o, int64_t row, bool live, int lane, int nch, const float (&y)[kV][kChunk], void* sh) {
    if constexpr (OUT == kOutRow) {
        emit_row<T>(o, row, live, lane, nch, y, sh);
    } else {
        if (OUT == kOutMx && live && lane == 0) {
            ((float*)o.scale)[row] = 1.0f;
            o.zero[row] = 0.0f;
        }
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            const int c = v * T + lane;
            if (v * T < nch) {
                if (OUT == kOutBlock) emit_block(o, row, c, live && c < nch, y[v]);
                else emit_mx(o, row, c, live && c < nch, y[v]);
            }
        }
    }
}

// ------------------------------------------------------------------------------------
// the residual's addition and the norm
// ------------------------------------------------------------------------------------
struct NormArgs {
    const void* x;
    const void* r;
    void* h;
    const void* g;
    int64_t ldx, ldr, ldh;
    int g_type;
    float eps;
    Out o;
};

// h = x + r, y = h / sqrt(mean h^2 + eps) g, then the codes of y.  The whole row is loaded before
// its first use (up to 4 chunks a lane in flight), so one wavefront per row with no barrier holds
// rows up to 2048, and workgroups the longer ones and those of few rows.  h goes past the caches
// (nothing here reads it again soon), the codes stay in them for the product that follows.
// Measured in a graph: bfloat16 x, binary32 residual, 8192 x 1152, block output 20.0 us (104 MB, 5.2
// TB/s: memory); bfloat16 x and residual, 4096 x 5120, block output 31.4 us, MXFP8 30.4, MXINT8 31.0,
// INT8 per token 32.3 (147 MB, 4.6 to 4.8 TB/s); 1 x 1280 2.8 us (a launch).  binary32 x alone, 8100 x
// 640, E4M3 per token 9.2 us (26 MB, 2.8 TB/s): a launch's 2.7 us beside 5.1 of memory, and the chains
// of the two reductions, which all rows run at about the same time (block output, one reduction: 8.7).
// RT: type of the residual, or -1 for none
template <int XT, int RT, int T, int OUT>
__global__ __launch_bounds__(wg_threads<T>()) void norm_kernel(NormArgs a) {
    __shared__ double sh[T > kWave ? T / kWave : 1];
    const int lane = threadIdx.x & (T - 1), nch = a.o.K / kChunk;
    int64_t row = (int64_t)blockIdx.x * rows_per_wg<T>() + (T == kWave ? threadIdx.x / T : 0);
    const bool live = row < a.o.M;
    if (!live) row = a.o.M - 1;  // a repeat of the last row, not written
    constexpr int RR = RT < 0 ? XT : RT;
    Raw<XT> x[kV];
    Raw<RR> r[kV];
#pragma unroll
    for (int v = 0; v < kV; ++v) {
        if (v * T < nch) {
            const int64_t i = (int64_t)min(v * T + lane, nch - 1) * kChunk;
            x[v] = load8<XT>(a.x, row * a.ldx + i);
            if (RT >= 0) r[v] = load8<RR>(a.r, row * a.ldr + i);
        }
    }
    float h[kV][kChunk];
    double ss = 0.0;
#pragma unroll
    for (int v = 0; v < kV; ++v) {
        if (v * T < nch && v * T + lane < nch) {
            widen<XT>(x[v], h[v]);
            if (RT >= 0) {
                float t[kChunk];
                widen<RR>(r[v], t);
#pragma unroll
                for (int j = 0; j < kChunk; ++j) h[v][j] += t[j];
                if (a.h && live) store8<RR>(a.h, row * a.ldh + (int64_t)(v * T + lane) * kChunk, h[v]);
            }
#pragma unroll
            for (int j = 0; j < kChunk; ++j) {  // squares of binary32 are exact, and in range, in binary64
                const double d = (double)h[v][j];
                ss = __builtin_fma(d, d, ss);
            }
        }
    }
    ss = team_reduce<T>(ss, sh, [](double p, double q) { return p + q; });
    // rows near either end of binary32 have a factor outside its normal numbers: a power of two of
    // it goes to h first, exactly
    const double rs = 1.0 / sqrt(ss / (double)a.o.K + (double)a.eps);
    const float pre = rs < 0x1p-120 ? 0x1p-64f : rs > 0x1p120 ? 0x1p64f : 1.0f;
    const float rstd = (float)(rs < 0x1p-120 ? rs * 0x1p64 : rs > 0x1p120 ? rs * 0x1p-64 : rs);
#pragma unroll
    for (int v = 0; v < kV; ++v) {
        const int c = v * T + lane;
        if (v * T < nch && c < nch) {
            float g[kChunk];
            if (a.g) load_g(a.g, a.g_type, (int64_t)c * kChunk, g);
#pragma unroll
            for (int j = 0; j < kChunk; ++j) h[v][j] = a.g ? h[v][j] * pre * rstd * g[j] : h[v][j] * pre * rstd;
        }
    }
    emit<T, OUT>(a.o, row, live, lane, nch, h, sh);
}

// ------------------------------------------------------------------------------------
// the (gated) activation function
// ------------------------------------------------------------------------------------
struct GateArgs {
    const void* x;
    const void* u;
    int64_t ldx, ldu;
    int act;
    Out o;
};

template <int XT>
CHAM_DEV void gate_chunk(const Raw<XT>& x, const Raw<XT>& u, bool gated, int act, float (&y)[kChunk]) {
    widen<XT>(x, y);
    activate(y, act);
    if (gated) {
        float t[kChunk];
        widen<XT>(u, t);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) y[j] *= t[j];
    }
}

// One scale per token: the row in registers, as in the norm (a scale needs the whole row's range).
// Bound as the block form below, and by the range's reductions where rows are short.  Measured,
// bfloat16 gated SiLU, E4M3 and INT8 (two more reductions): 8192 x 4608 38.7 and 44.6 us (189 MB, 4.9
// TB/s), 8192 x 2560 28.1 and 33.5 (105 MB), 8192 x 1152 13.6 and 15.0 (47 MB), 2048 x 5120 12.7 and
// 14.3 (52 MB).
template <int XT, int T>
__global__ __launch_bounds__(wg_threads<T>()) void gate_row_kernel(GateArgs a) {
    __shared__ float sh[T > kWave ? T / kWave : 1];
    const int lane = threadIdx.x & (T - 1), nch = a.o.K / kChunk;
    int64_t row = (int64_t)blockIdx.x * rows_per_wg<T>() + (T == kWave ? threadIdx.x / T : 0);
    const bool live = row < a.o.M;
    if (!live) row = a.o.M - 1;
    // binary32 rows of 1024 lanes: the second factor is loaded after the first is used up (both
    // at once would not fit the 128 registers that 1024 lanes leave each)
    constexpr bool kLate = XT == CHAM_T_F32 && T == 1024;
    Raw<XT> x[kV], u[kV];
#pragma unroll
    for (int v = 0; v < kV; ++v) {
        if (v * T < nch) {
            const int64_t i = (int64_t)min(v * T + lane, nch - 1) * kChunk;
            x[v] = load8<XT>(a.x, row * a.ldx + i);
            if (!kLate && a.u) u[v] = load8<XT>(a.u, row * a.ldu + i);
        }
    }
    float y[kV][kChunk];
#pragma unroll
    for (int v = 0; v < kV; ++v) {
        const int64_t c = v * T + lane;
        if (v * T < nch && c < nch) {
            if (kLate && a.u) u[v] = load8<XT>(a.u, row * a.ldu + c * kChunk);
            gate_chunk<XT>(x[v], u[v], a.u != nullptr, a.act, y[v]);
        }
    }
    emit<T, kOutRow>(a.o, row, live, lane, nch, y, sh);
}

// Block and MX formats need no more than 16 neighbouring lanes: the tensor is a list of blocks
// of 128 (those of a row's ragged end are short), 16 lanes a block, any K.  A workgroup takes 32
// consecutive blocks; where its first one lies is found once, in scalar registers.
// Measured: bfloat16 gated GELU 2048 x 5120 14.0 us (53 MB, 3.8 TB/s, a launch's 2.7 us among
// them), plain GELU's tanh form 8192 x 4608 26 us (115 MB, 4.4 TB/s: memory), gated SiLU 8192 x 4608
// 37.2 us in block format, 36.5 in MXFP8, 37.3 in MXINT8 (190 MB, 5.1 TB/s), 240 x 4608 3.6 us (a launch).
constexpr int kGateThreads = 256;
constexpr int kGateBlocks = 2;  // blocks per 16 lanes, their loads in flight together
constexpr int kGatePer = kGateThreads / 16 * kGateBlocks;

template <int XT, int OUT>
__global__ __launch_bounds__(kGateThreads) void gate_block_kernel(GateArgs a) {
    const int nch = a.o.K / kChunk, nb = (nch + 15) >> 4;
    const int64_t b0 = (int64_t)blockIdx.x * kGatePer, row0 = b0 / nb;
    const int c0 = (int)(b0 - row0 * nb);
    const int recip = 65536 / min(nb, 65536) + 1;  // of nb < 32
    Raw<XT> x[kGateBlocks], u[kGateBlocks];
    int64_t row[kGateBlocks];
    int c[kGateBlocks];
    bool in[kGateBlocks];
#pragma unroll
    for (int v = 0; v < kGateBlocks; ++v) {
        const int i = c0 + v * (kGateThreads / 16) + (int)threadIdx.x / 16;  // blocks from row0's start, < nb + 32
        const int q = nb >= kGatePer ? (i >= nb ? 1 : 0) : (i * recip) >> 16;  // i / nb (i < 64 where nb < 32)
        row[v] = row0 + q;
        c[v] = (i - q * nb) * 16 + (threadIdx.x & 15);
        in[v] = row[v] < a.o.M && c[v] < nch;
        const int64_t r = min(row[v], a.o.M - 1), e = (int64_t)min(c[v], nch - 1) * kChunk;
        x[v] = load8<XT>(a.x, r * a.ldx + e);
        if (a.u) u[v] = load8<XT>(a.u, r * a.ldu + e);
    }
#pragma unroll
    for (int v = 0; v < kGateBlocks; ++v) {
        float y[kChunk];
        gate_chunk<XT>(x[v], u[v], a.u != nullptr, a.act, y);
        if (OUT == kOutBlock) {
            emit_block(a.o, row[v], c[v], in[v], y);
        } else {
            if (in[v] && c[v] == 0) {
                ((float*)a.o.scale)[row[v]] = 1.0f;
                a.o.zero[row[v]] = 0.0f;
            }
            emit_mx(a.o, row[v], c[v], in[v], y);
        }
    }
}

// ------------------------------------------------------------------------------------
// weights: one workgroup per 128 x 128 block
// ------------------------------------------------------------------------------------
// The block is held in registers (4 chunks a lane) between its maximum, one reduction over the
// workgroup, and its codes: W is read once.  Memory: bfloat16 10240 x 1280 9.4 us (39 MB, 4.2
// TB/s); binary32 640 x 1920, 75 blocks, 3.8 us (a launch).
constexpr int kWThreads = 512;
constexpr int kWRows = kWThreads / 16;      // rows of the block in one step
constexpr int kWSteps = 128 / kWRows;

template <int XT>
__global__ __launch_bounds__(kWThreads) void weights_block_kernel(const void* W, int64_t ldw, int64_t N, int K, int nb,
                                                                  int pow2, uint8_t* codes, void* scale) {
    __shared__ uint32_t sh[kWThreads / kWave];
    const int64_t bn = blockIdx.x / nb;
    const int bk = (int)(blockIdx.x - bn * nb);
    const int c = bk * 16 + (threadIdx.x & 15), nch = K / kChunk;
    const int64_t n0 = bn * 128 + threadIdx.x / 16;
    Raw<XT> raw[kWSteps];
#pragma unroll
    for (int v = 0; v < kWSteps; ++v)
        raw[v] = load8<XT>(W, min(n0 + v * kWRows, N - 1) * ldw + (int64_t)min(c, nch - 1) * kChunk);
    float y[kWSteps][kChunk];
    uint32_t m = 0;
#pragma unroll
    for (int v = 0; v < kWSteps; ++v) {  // past an end: repeats of the block's own elements
        widen<XT>(raw[v], y[v]);
        const uint32_t a = chunk_amax(y[v]);
        m = m > a ? m : a;
    }
    m = team_reduce<kWThreads>(m, sh, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
    uint32_t stored;
    const float r = block_scale(m, pow2 != 0, &stored);
    if (threadIdx.x == 0) {
        if (pow2) ((uint8_t*)scale)[blockIdx.x] = (uint8_t)stored;
        else ((uint32_t*)scale)[blockIdx.x] = stored;
    }
#pragma unroll
    for (int v = 0; v < kWSteps; ++v) {
        const int64_t n = n0 + v * kWRows;
        if (n < N && c < nch) *(uint2*)(codes + n * K + (int64_t)c * kChunk) = codes8_e4m3(y[v], r);
    }
}

// ------------------------------------------------------------------------------------
// launches
// ------------------------------------------------------------------------------------
bool type_ok(int t) { return t >= 0 && t < CHAM_T_N; }
int64_t type_size(int t) { return t == CHAM_T_F32 ? 4 : 2; }
bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
// a [M][K] matrix of row stride ld (in elements): whole rows, each 16-byte aligned
bool rows_ok(const void* p, int64_t ld, int64_t K, int type) {
    return p && aligned(p, 16) && ld >= K && (ld * type_size(type)) % 16 == 0;
}

int sizes_ok(int64_t M, int64_t K, int64_t most) {
    if (M < 0 || K < 1) return CHAM_EINVAL;
    if (K % 32 != 0 || K > most || M >= (int64_t)1 << 31) return CHAM_ESHAPE;
    return CHAM_OK;
}

int out_block(const cham_bq* q, int64_t M, int64_t K, Out* o) {
    if (!q || q->M != M || q->K != K) return CHAM_EINVAL;
    if (M > 0 && (!q->codes || !q->scale || !aligned(q->codes, 16) || !aligned(q->scale, 4))) return CHAM_EINVAL;
    if (q->pow2 != 0 && q->pow2 != 1) return CHAM_EINVAL;
    *o = Out{M, (int)K, 0, q->pow2, q->codes, q->scale, nullptr, nullptr};
    return CHAM_OK;
}
int out_token(int32_t fmt, cham_aq* q, int64_t M, int64_t K, Out* o) {
    if (!q || q->M != M || q->K != K) return CHAM_EINVAL;
    if (M > 0 && (!q->codes || !q->scale || !q->zero || !aligned(q->codes, 8))) return CHAM_EINVAL;
    if (q->nsamples != M) return CHAM_EINVAL;
    if (fmt < 0 || fmt >= CHAM_A_NFMT) return CHAM_EFORMAT;
    if (M > 0 && fmt >= CHAM_A_MXFP8_E4M3 && !q->e8m0) return CHAM_EINVAL;
    *o = Out{M, (int)K, fmt, 0, q->codes, q->scale, q->zero, q->e8m0};
    return CHAM_OK;
}

// Lanes per row: a wavefront where its registers hold the row (no barrier, four rows per workgroup),
// else 256 lanes, and 1024 for rows that 256 cannot hold.  Rows of more than a chunk per lane take 256
// lanes too where there are at most two of them per CU: latency counts there, and a lane's chunks are
// worked off in turn.  Norm of bfloat16 rows and residual, us with 64, 256 and 1024 lanes (block
// output / INT8 per token):
//   8100 x 640    10.5 14.7 50.1 / 11.8 19.8 91.9      8192 x 1152   15.6 16.7 50.8 / 16.8 21.5 92.7
//   1024 x 640     3.9  4.0  8.3 /  4.4  5.1 13.3      512 x 640      3.7  3.4  5.1 /  4.2  4.4  7.6
//   512 x 1152     4.5  3.5  5.2 /  4.9  4.5  7.8      1 x 1152       3.9  2.8  3.3 /  4.4  3.8  5.0
//   1 x 2048       4.5  2.8  3.4 /  5.0  3.8  5.0      4096 x 2048   13.0 12.7 27.6 / 13.6 15.3 47.8
//   1 x 4096          -  3.5  3.5 /    -  4.4  5.1     1 x 8192          -  4.8  4.1 /    -  5.7  5.8
//   4096 x 5120       - 31.4 37.7 /    - 32.2 59.7     4096 x 8192       - 50.9 50.7 /    - 50.7 71.7
// Gated SiLU, E4M3 per token: 1 x 2048 4.2 2.7 2.8, 1 x 4096 - 3.2 3.0, 1 x 8192 - 4.3 3.7, 2048 x 5120
// - 12.8 21.4.  So 1024 lanes would save a few rows of 4097 to 8192 elements up to 0.7 us, below the
// host's call; the rule has no line for them.
int team(int64_t M, int64_t K) {
    if (K <= kWave * kChunk || (K <= kWave * kV * kChunk && M > 2 * (int64_t)cham_device_cus())) return kWave;
    return K <= 256 * kV * kChunk ? 256 : 1024;
}
int64_t row_grid(int64_t M, int T) { return T == kWave ? (M + 3) / 4 : M; }
bool rows_launchable(int64_t M, int64_t K) {
    const int T = team(M, K);
    return cham_launchable(row_grid(M, T), std::max(T, 256));
}
// workgroups of the block and MX forms of the gate
int64_t gate_grid(int64_t M, int64_t K) { return (M * ((K + 127) / 128) + kGatePer - 1) / kGatePer; }

template <int XT, int RT, int OUT>
void launch_norm_t(const NormArgs& a, hipStream_t s) {
    const int T = team(a.o.M, a.o.K);
    const dim3 grid((unsigned)row_grid(a.o.M, T));
    if (T == kWave) hipLaunchKernelGGL((norm_kernel<XT, RT, kWave, OUT>), grid, dim3(256), 0, s, a);
    else if (T == 256) hipLaunchKernelGGL((norm_kernel<XT, RT, 256, OUT>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((norm_kernel<XT, RT, 1024, OUT>), grid, dim3(1024), 0, s, a);
}
template <int XT, int RT>
void launch_norm_o(const NormArgs& a, int out, hipStream_t s) {
    if (out == kOutBlock) launch_norm_t<XT, RT, kOutBlock>(a, s);
    else if (out == kOutRow) launch_norm_t<XT, RT, kOutRow>(a, s);
    else launch_norm_t<XT, RT, kOutMx>(a, s);
}
template <int XT>
void launch_norm_r(const NormArgs& a, int r_type, int out, hipStream_t s) {
    if (!a.r) launch_norm_o<XT, -1>(a, out, s);
    else if (r_type == XT) launch_norm_o<XT, XT>(a, out, s);
    else if constexpr (XT != CHAM_T_F32) launch_norm_o<XT, CHAM_T_F32>(a, out, s);
}

int out_kind(int fmt) { return fmt >= CHAM_A_MXFP8_E4M3 ? kOutMx : kOutRow; }

int norm_check(const cham_norm* n) {
    if (!n) return CHAM_EINVAL;
    const int rc = sizes_ok(n->M, n->K, kRowMax);
    if (rc != CHAM_OK) return rc;
    if (!type_ok(n->x_type) || (n->r && n->r_type != n->x_type && n->r_type != CHAM_T_F32) || (n->g && !type_ok(n->g_type)))
        return CHAM_EFORMAT;
    if (!(n->eps >= 0.0f) || n->eps > FLT_MAX) return CHAM_EINVAL;
    if (n->M == 0) return CHAM_OK;
    if (!rows_ok(n->x, n->ldx, n->K, n->x_type)) return CHAM_EINVAL;
    if (n->r && !rows_ok(n->r, n->ldr, n->K, n->r_type)) return CHAM_EINVAL;
    if (n->h && (!n->r || !rows_ok(n->h, n->ldh, n->K, n->r_type))) return CHAM_EINVAL;
    if (n->h && n->h == n->r && n->ldh != n->ldr) return CHAM_EINVAL;
    if (n->g && !aligned(n->g, 16)) return CHAM_EINVAL;
    return CHAM_OK;
}

int norm_launch(const cham_norm* n, const Out& o, int out, hipStream_t s) {
    if (n->M == 0) return CHAM_OK;
    if (!rows_launchable(n->M, n->K)) return CHAM_ESHAPE;
    const NormArgs a{n->x, n->r, n->h, n->g, n->ldx, n->ldr, n->ldh, n->g_type, n->eps, o};
    if (n->x_type == CHAM_T_F32) launch_norm_r<CHAM_T_F32>(a, n->r_type, out, s);
    else if (n->x_type == CHAM_T_F16) launch_norm_r<CHAM_T_F16>(a, n->r_type, out, s);
    else launch_norm_r<CHAM_T_BF16>(a, n->r_type, out, s);
    CHAM_CHECK_LAUNCH();
    return CHAM_OK;
}

int gate_check(const cham_gate* g, int64_t most) {
    if (!g) return CHAM_EINVAL;
    const int rc = sizes_ok(g->M, g->K, most);
    if (rc != CHAM_OK) return rc;
    if (!type_ok(g->type) || g->act < 0 || g->act >= CHAM_ACT_N) return CHAM_EFORMAT;
    if (g->M == 0) return CHAM_OK;
    if (!rows_ok(g->x, g->ldx, g->K, g->type)) return CHAM_EINVAL;
    if (g->u && !rows_ok(g->u, g->ldu, g->K, g->type)) return CHAM_EINVAL;
    return CHAM_OK;
}

template <int XT>
void launch_gate_t(const GateArgs& a, int out, hipStream_t s) {
    if (out == kOutRow) {
        const int T = team(a.o.M, a.o.K);
        const dim3 grid((unsigned)row_grid(a.o.M, T));
        if (T == kWave) hipLaunchKernelGGL((gate_row_kernel<XT, kWave>), grid, dim3(256), 0, s, a);
        else if (T == 256) hipLaunchKernelGGL((gate_row_kernel<XT, 256>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((gate_row_kernel<XT, 1024>), grid, dim3(1024), 0, s, a);
        return;
    }
    const dim3 grid((unsigned)gate_grid(a.o.M, a.o.K));
    if (out == kOutBlock) hipLaunchKernelGGL((gate_block_kernel<XT, kOutBlock>), grid, dim3(kGateThreads), 0, s, a);
    else hipLaunchKernelGGL((gate_block_kernel<XT, kOutMx>), grid, dim3(kGateThreads), 0, s, a);
}

int gate_launch(const cham_gate* g, const Out& o, int out, hipStream_t s) {
    if (g->M == 0) return CHAM_OK;
    if (out == kOutRow ? !rows_launchable(g->M, g->K) : !cham_launchable(gate_grid(g->M, g->K), kGateThreads)) return CHAM_ESHAPE;
    const GateArgs a{g->x, g->u, g->ldx, g->ldu, g->act, o};
    if (g->type == CHAM_T_F32) launch_gate_t<CHAM_T_F32>(a, out, s);
    else if (g->type == CHAM_T_F16) launch_gate_t<CHAM_T_F16>(a, out, s);
    else launch_gate_t<CHAM_T_BF16>(a, out, s);
    CHAM_CHECK_LAUNCH();
    return CHAM_OK;
}

}  // namespace
}  // namespace cham

using namespace cham;

extern "C" int cham_rms_norm_quantize_block(const cham_norm* n, cham_bq* out, void* stream) {
    Out o;
    int rc = norm_check(n);
    if (rc == CHAM_OK) rc = out_block(out, n->M, n->K, &o);
    return rc != CHAM_OK ? rc : norm_launch(n, o, kOutBlock, (hipStream_t)stream);
}

extern "C" int cham_rms_norm_quantize(const cham_norm* n, int32_t fmt, cham_aq* out, void* stream) {
    Out o;
    int rc = norm_check(n);
    if (rc == CHAM_OK) rc = out_token(fmt, out, n->M, n->K, &o);
    if (rc == CHAM_OK) rc = norm_launch(n, o, out_kind(fmt), (hipStream_t)stream);
    if (rc == CHAM_OK) out->fmt = fmt;
    return rc;
}

// Largest K of the block and MX forms of the gate: chunk indices stay within 32 bits.
static constexpr int64_t kGateMax = (int64_t)1 << 30;

extern "C" int cham_gated_quantize_block(const cham_gate* a, cham_bq* out, void* stream) {
    Out o;
    int rc = gate_check(a, kGateMax);
    if (rc == CHAM_OK) rc = out_block(out, a->M, a->K, &o);
    return rc != CHAM_OK ? rc : gate_launch(a, o, kOutBlock, (hipStream_t)stream);
}

extern "C" int cham_gated_quantize(const cham_gate* a, int32_t fmt, cham_aq* out, void* stream) {
    Out o;
    int rc = gate_check(a, fmt >= CHAM_A_MXFP8_E4M3 ? kGateMax : kRowMax);
    if (rc == CHAM_OK) rc = out_token(fmt, out, a->M, a->K, &o);
    if (rc == CHAM_OK) rc = gate_launch(a, o, out_kind(fmt), (hipStream_t)stream);
    if (rc == CHAM_OK) out->fmt = fmt;
    return rc;
}

extern "C" int cham_block_quantize_weights(const void* W, int32_t type, int64_t ldw, cham_bw* out, void* stream) {
    if (!out || out->N < 1) return CHAM_EINVAL;
    const int rc = sizes_ok(out->N, out->K, kGateMax);
    if (rc != CHAM_OK) return rc;
    if (!type_ok(type)) return CHAM_EFORMAT;
    if (!rows_ok(W, ldw, out->K, type) || !out->codes || !out->scale || !aligned(out->codes, 16) || !aligned(out->scale, 4))
        return CHAM_EINVAL;
    if (out->pow2 != 0 && out->pow2 != 1) return CHAM_EINVAL;
    const int64_t nb = (out->K + 127) / 128, blocks = (out->N + 127) / 128 * nb;
    if (!cham_launchable(blocks, kWThreads)) return CHAM_ESHAPE;
    const dim3 grid((unsigned)blocks);
    const hipStream_t s = (hipStream_t)stream;
#define CHAM_W(T)                                                                                                      \
    hipLaunchKernelGGL(weights_block_kernel<T>, grid, dim3(kWThreads), 0, s, W, ldw, out->N, (int)out->K, (int)nb,      \
                       out->pow2, out->codes, out->scale)
    if (type == CHAM_T_F32) CHAM_W(CHAM_T_F32);
    else if (type == CHAM_T_F16) CHAM_W(CHAM_T_F16);
    else CHAM_W(CHAM_T_BF16);
#undef CHAM_W
    CHAM_CHECK_LAUNCH();
    return CHAM_OK;
}

// Row passes over heads: the root-mean-square norm of each head with the rotation by the token's
// position, the same with keys and values written into the pages of a cache, and pages brought
// back into packed rows.
//
// All are bound by memory, or by their launch where they are small.  A vector is one head of one
// token; 8 or 16 lanes hold it, 8 consecutive elements each, from its load to its store.  A workgroup
// takes some tokens with all or a part of their vectors and makes the tokens' cosines and sines
// once, in LDS.  A group of lanes stays with one head of those tokens, so that addresses, weights and the
// branch by kind are worked out once, and has four tokens' loads under way.
//
// bfloat16, 8192 x 32 heads of 72, 48 elements turned: 22.3 us, 3.4 TB/s (with one vector at a time and a division
// for each 32, with sums in binary64 36; 2 % of it leave what lies behind R untouched); 8100 x 8 heads of 128
// into E4M3 pages 13.8, 3.6 TB/s; 30001 tokens of 8 heads of 128 out of them 43, 4.3 TB/s (a copy reaches
// 5.1).  One token of 40 heads: 3.8, a launch and the angle's chain.
#include <algorithm>

#include "cham_chunk.h"
#include "cham_heads.h"

namespace cham {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTok = 8;    // tokens of a workgroup
constexpr int kMaxHalf = 64;  // pairs of a head

// ------------------------------------------------------------------------------------
// reductions over the LP lanes of a vector: quads, then mirrors, so every lane adds the same
// two values at each step and all get the same bits
// ------------------------------------------------------------------------------------
template <int CTRL>
CHAM_DEV double dpp_add(double v) {
    const uint2 w = __builtin_bit_cast(uint2, v);
    const uint2 o = make_uint2((uint32_t)__builtin_amdgcn_mov_dpp((int)w.x, CTRL, 0xF, 0xF, true),
                               (uint32_t)__builtin_amdgcn_mov_dpp((int)w.y, CTRL, 0xF, 0xF, true));
    return v + __builtin_bit_cast(double, o);
}
template <int LP>
CHAM_DEV double vector_sum(double v) {
    v = dpp_add<0x141>(dpp_add<0x4E>(dpp_add<0xB1>(v)));  // 8 lanes
    return LP == 16 ? dpp_add<0x140>(v) : v;
}
template <int LP>
CHAM_DEV float vector_sum(float v) {
    v += dpp<0xB1>(v);
    v += dpp<0x4E>(v);
    v += dpp<0x141>(v);
    return LP == 16 ? v + dpp<0x140>(v) : v;
}
template <int LP>
CHAM_DEV uint32_t vector_max(uint32_t v) {
    v = dpp_maxu<0x141>(dpp_maxu<0x4E>(dpp_maxu<0xB1>(v)));
    return LP == 16 ? dpp_maxu<0x140>(v) : v;
}

// cos t and sin t.  t is reduced by multiples of pi/2 in binary64 (pi/2 in two parts: the rest is
// within 2^-53 |t|), the remainder's series, |r| <= pi/4, are cut off below 2^-29 and run in binary32.
// From 2^51 on a multiple's own rounding may leave several pi/2, which a second turn takes off; from 2^55 on
// every angle is within 2^-53 |t|, and 0 is taken.
CHAM_DEV float2 cos_sin(double t) {
    const auto reduce = [](double t, int* quarter) {
        const double n = __builtin_rint(t * 0.63661977236758134308);
        *quarter += (int)(n - 4.0 * __builtin_floor(n * 0.25));
        return __builtin_fma(-n, 0x1.1a62633145c07p-54, __builtin_fma(-n, 0x1.921fb54442d18p+0, t));
    };
    t = __builtin_fabs(t) < 0x1p55 ? t : t * 0.0;
    int quarter = 0;
    const double r = reduce(reduce(t, &quarter), &quarter);
    const float x = (float)r, z = x * x;
    float s = __builtin_fmaf(z, 1.0f / 362880.0f, -1.0f / 5040.0f);
    s = __builtin_fmaf(z, s, 1.0f / 120.0f);
    s = __builtin_fmaf(z, s, -1.0f / 6.0f);
    s = __builtin_fmaf(x * z, s, x);
    float c = __builtin_fmaf(z, -1.0f / 3628800.0f, 1.0f / 40320.0f);
    c = __builtin_fmaf(z, c, -1.0f / 720.0f);
    c = __builtin_fmaf(z, c, 1.0f / 24.0f);
    c = __builtin_fmaf(z, c, -0.5f);
    c = __builtin_fmaf(z, c, 1.0f);
    const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
    return make_float2((quarter + 1) & 2 ? -a : a, quarter & 2 ? -b : b);
}

struct RowsArgs {
    cham_heads in[3], out[2];  // q, k, v; q, k
    cham_rotate r;
    cham_cache c;
    const int32_t* slots;
    int tok, per;              // tokens of a workgroup, vectors of a workgroup's token
    int nv;                    // vectors of a token
    double inv_d;              // 1 / D
};

// XT: type of the inputs; CT: -1 (norm_rotate) or the cache's type
template <int XT, int LP, int CT>
__global__ __launch_bounds__(kThreads) void heads_kernel(const RowsArgs a) {
    constexpr int kGroups = kThreads / LP;
    __shared__ __align__(16) float cs[kMaxTok][2][kMaxHalf];    // cos, sin of each token's pairs
    __shared__ __align__(16) float rows[kGroups][LP * kChunk];  // a vector between its norm and its rotation
    const int lane = threadIdx.x % LP, group = threadIdx.x / LP, d0 = lane * kChunk;
    const int D = a.r.D, half = a.r.R >> 1;
    const int64_t t0 = (int64_t)blockIdx.x * a.tok;
    const int nt = (int)min((int64_t)a.tok, a.r.T - t0);
    const int first = blockIdx.y * a.per, per = min(a.per, a.nv - first);
    const bool live = d0 < D;

    // A group of lanes takes vectors first + group, + kGroups, ... of each token, a few tokens' loads at a
    // time, the first before the angles.
    constexpr int kBatch = XT == CHAM_T_F32 ? 2 : 4, kSize = XT == CHAM_T_F32 ? 4 : 2;
    Raw<XT> raw[kBatch];
    int which = 0, head = 0;
    const char* from = nullptr;
    int64_t step = 0;  // bytes from token to token
    const auto vector = [&](int vec) {
        const int hq = a.in[0].H, hk = a.in[1].H;
        which = vec < hq ? 0 : vec < hq + hk ? 1 : 2;
        head = vec - (which == 0 ? 0 : which == 1 ? hq : hq + hk);
        const cham_heads& h = which == 0 ? a.in[0] : which == 1 ? a.in[1] : a.in[2];
        step = h.token * kSize;
        from = (const char*)h.p + (t0 * h.token + (int64_t)head * h.head + d0) * kSize;
    };
    const auto fetch = [&](int tok) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            raw[i] = Raw<XT>{};
            if (live && tok + i < nt) raw[i] = load8<XT>(from + (tok + i) * step, 0);
        }
    };
    if (group < per) {
        vector(first + group);
        fetch(0);
    }
    if (half > 0) {
        for (int i = threadIdx.x; i < nt * kMaxHalf; i += kThreads) {
            const int k = i % kMaxHalf;
            float2 v = make_float2(1.0f, 0.0f);  // pairs behind R are read, but not turned
            if (k < half) {
                v = cos_sin((double)a.r.pos[t0 + i / kMaxHalf] * a.r.freq[k]);
                v.x *= a.r.amp;
                v.y *= a.r.amp;
            }
            cs[i / kMaxHalf][0][k] = v.x;
            cs[i / kMaxHalf][1][k] = v.y;
        }
    }
    __syncthreads();

    for (int vec = group; vec < per; vec += kGroups) {
        if (vec != group) vector(first + vec);
        const cham_heads& out = which == 0 ? a.out[0] : a.out[1];
        char* const to = (char*)out.p + (t0 * out.token + (int64_t)head * out.head + d0) * kSize;
        const int64_t to_step = out.token * kSize;
        float w[kChunk];  // the norm's weights
        if (a.r.norm && which < 2) {
            const void* g = which == 0 ? a.r.qg : a.r.kg;
#pragma unroll
            for (int j = 0; j < kChunk; ++j) w[j] = 1.0f;
            if (g && live) load_g(g, which == 0 ? a.r.qg_type : a.r.kg_type, d0, w);
        }
        for (int tok0 = 0; tok0 < nt; tok0 += kBatch) {
            if (vec != group || tok0 > 0) fetch(tok0);
#pragma unroll
            for (int v = 0; v < kBatch; ++v) {
                const int tok = tok0 + v;
                if (tok >= nt) break;
                float y[kChunk];
                widen<XT>(raw[v], y);
                if (which < 2) {
                    if (a.r.norm) {
                        // 16-bit elements: binary32 where the sum is far from its ends (twelve roundings, halved by the
                        // root: 6 2^-24); else, and for binary32 elements, binary64
                        float q32 = 0.0f;
                        bool wide = XT == CHAM_T_F32;
                        if constexpr (XT != CHAM_T_F32) {
                            float s = 0.0f;
#pragma unroll
                            for (int j = 0; j < kChunk; ++j) s = __builtin_fmaf(y[j], y[j], s);
                            s = __builtin_fmaf(vector_sum<LP>(s), (float)a.inv_d, a.r.eps);
                            q32 = __builtin_amdgcn_rsqf(s);
                            q32 = q32 * __builtin_fmaf(-0.5f * s * q32, q32, 1.5f);
                            wide = !(s > 0x1p-60f && s < 0x1p+100f);
                        }
                        if (wide) {
                            double s = 0.0;
#pragma unroll
                            for (int j = 0; j < kChunk; ++j) s = __builtin_fma((double)y[j], (double)y[j], s);
                            s = __builtin_fma(vector_sum<LP>(s), a.inv_d, (double)a.r.eps);
                            // 1 / sqrt(s): binary32's estimate for s brought into its range by a power of four,
                            // one Newton step in binary64; an infinite s gives 0
                            const int e = (__builtin_amdgcn_frexp_exp(s) + 1) & ~1;
                            const double m = __builtin_amdgcn_ldexp(s, -e);
                            double q = (double)__builtin_amdgcn_rsqf((float)m);
                            if (q != 0.0) q = __builtin_amdgcn_ldexp(q * __builtin_fma(-0.5 * m * q, q, 1.5), -e / 2);
#pragma unroll
                            for (int j = 0; j < kChunk; ++j) y[j] = (float)((double)y[j] * q) * w[j];
                        } else {
#pragma unroll
                            for (int j = 0; j < kChunk; ++j) y[j] = y[j] * q32 * w[j];
                        }
                    }
                    if (half > 0) {
                        const float *co = cs[tok][0], *si = cs[tok][1];
                        if (a.r.layout == CHAM_ROT_PAIRS) {
                            const float4 c4 = *(const float4*)(co + d0 / 2), s4 = *(const float4*)(si + d0 / 2);
                            const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
                            // (a pair behind R times (1, 0) would pass an infinity on to its neighbour)
                            const int turned = half - d0 / 2;
                            if (half % 4 == 0) {
                                if (turned > 0) {
#pragma unroll
                                    for (int j = 0; j < 4; ++j) {
                                        const float u = y[2 * j], v = y[2 * j + 1];
                                        y[2 * j] = u * c[j] - v * s[j];
                                        y[2 * j + 1] = v * c[j] + u * s[j];
                                    }
                                }
                            } else {
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    const float u = y[2 * j], v = y[2 * j + 1];
                                    y[2 * j] = j < turned ? u * c[j] - v * s[j] : u;
                                    y[2 * j + 1] = j < turned ? v * c[j] + u * s[j] : v;
                                }
                            }
                        } else if (half % kChunk == 0) {
                            // a partner is another lane's element of the same place
                            const bool low = d0 < half, turned = d0 < 2 * half;
                            const int i = turned ? (low ? d0 : d0 - half) : 0, from = turned ? (low ? d0 + half : i) : 0;
                            float* row = rows[group];
                            *(float4*)(row + d0) = make_float4(y[0], y[1], y[2], y[3]);
                            *(float4*)(row + d0 + 4) = make_float4(y[4], y[5], y[6], y[7]);
                            __builtin_amdgcn_wave_barrier();
                            float4 o4[2], c4[2], s4[2];
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                o4[j] = *(const float4*)(row + from + 4 * j);
                                c4[j] = *(const float4*)(co + i + 4 * j);
                                s4[j] = *(const float4*)(si + i + 4 * j);
                            }
                            __builtin_amdgcn_wave_barrier();
                            const float *o = (const float*)o4, *c = (const float*)c4, *s = (const float*)s4;
                            if (turned) {
#pragma unroll
                                for (int j = 0; j < kChunk; ++j) y[j] = y[j] * c[j] + (low ? -o[j] : o[j]) * s[j];
                            }
                        } else {
                            // partners lie R/2 elements apart, in another lane and, for odd R/2, at
                            // another place: through LDS, within the wavefront
                            float* row = rows[group];
                            *(float4*)(row + d0) = make_float4(y[0], y[1], y[2], y[3]);
                            *(float4*)(row + d0 + 4) = make_float4(y[4], y[5], y[6], y[7]);
                            __builtin_amdgcn_wave_barrier();
#pragma unroll
                            for (int j = 0; j < kChunk; ++j) {
                                const int d = d0 + j;
                                if (d < 2 * half) {
                                    const bool low = d < half;
                                    const int i = low ? d : d - half;
                                    const float o = row[low ? d + half : i], s = si[i];
                                    y[j] = y[j] * co[i] + (low ? -o : o) * s;
                                }
                            }
                            __builtin_amdgcn_wave_barrier();
                        }
                    }
                }
                if (CT < 0 || which == 0) {
                    if (live) put8<XT>(to + tok * to_step, 0, y);
                } else if constexpr (CT >= 0) {
                    const int32_t slot = a.slots[t0 + tok];
                    const bool in = slot >= 0 && slot < a.c.pages * a.c.page;
                    const int64_t row = in ? ((int64_t)(slot / a.c.page) * a.c.H + head) * a.c.page + slot % a.c.page : 0;
                    void* to = which == 1 ? a.c.k : a.c.v;
                    if constexpr (CT == CHAM_T_E4M3) {
                        uint32_t stored;
                        const float r = block_scale(vector_max<LP>(live ? chunk_amax(y) : 0u), false, &stored);
                        if (in && live) {
                            *(uint2*)((uint8_t*)to + row * D + d0) = codes8_e4m3(y, r);
                            if (lane == 0) ((uint32_t*)(which == 1 ? a.c.ks : a.c.vs))[row] = stored;
                        }
                    } else if (in && live) {
                        put8<CT>(to, row * D + d0, y);
                    }
                }
            }
        }
    }
}

// ------------------------------------------------------------------------------------
// pages back into rows
// ------------------------------------------------------------------------------------
struct ReadArgs {
    cham_cache c;
    cham_heads ko, vo;
    const int32_t *table, *cu;
    int64_t width, T;
    int B, tok, per;
};

template <int CT, int YT, int LP>
__global__ __launch_bounds__(kThreads) void read_kernel(const ReadArgs a) {
    constexpr int kGroups = kThreads / LP;
    __shared__ int page_of[kMaxTok], place[kMaxTok];  // of the workgroup's tokens; page -2: no sequence, -1: no page
    const int lane = threadIdx.x % LP, group = threadIdx.x / LP, d0 = lane * kChunk;
    const int64_t t0 = (int64_t)blockIdx.x * a.tok;
    const int nt = (int)min((int64_t)a.tok, a.T - t0);
    const int first = blockIdx.y * a.per, per = min(a.per, 2 * a.c.H - first);
    if (threadIdx.x < kWave) {
        // a token's sequence: how many of the starts behind the first lie at or below it
        int seq = 0;
        const int64_t mine = t0 + threadIdx.x;
        for (int b0 = 0; b0 < a.B; b0 += kWave) {
            const int b = b0 + (int)threadIdx.x;
            const int64_t end = b < a.B ? a.cu[b + 1] : INT64_MAX;
            for (int i = 0; i < nt; ++i) {
                const int n = __popcll(__ballot(end <= t0 + i));
                if ((int)threadIdx.x == i) seq += n;
            }
        }
        if ((int)threadIdx.x < nt) {
            int page = -2, in = 0;
            if (seq < a.B && mine >= a.cu[seq]) {
                const int64_t t = mine - a.cu[seq];
                page = t / a.c.page < a.width ? a.table[(int64_t)seq * a.width + t / a.c.page] : -1;
                if (page < 0 || page >= a.c.pages) page = -1;
                in = (int)(t % a.c.page);
            }
            page_of[threadIdx.x] = page;
            place[threadIdx.x] = in;
        }
    }
    __syncthreads();
    if (d0 >= a.c.D) return;
    // four vectors' loads are under way at a time
    for (int item0 = group; item0 < nt * per; item0 += 4 * kGroups) {
        Raw<CT == CHAM_T_E4M3 ? CHAM_T_BF16 : CT> raw[4];
        float scale[4];
        int page[4];
        int64_t to[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int item = min(item0 + i * kGroups, nt * per - 1);
            const int tok = (int)((uint32_t)item / (uint32_t)per), vec = item - tok * per + first;
            const bool v = vec >= a.c.H;
            const int head = v ? vec - a.c.H : vec;
            page[i] = item0 + i * kGroups < nt * per ? page_of[tok] : -2;
            const int64_t row = ((int64_t)max(page[i], 0) * a.c.H + head) * a.c.page + (page[i] >= 0 ? place[tok] : 0);
            const void* from = v ? a.c.v : a.c.k;
            if constexpr (CT == CHAM_T_E4M3) {
                const uint2 w = *(const uint2*)((const uint8_t*)from + row * a.c.D + d0);
                raw[i].a = make_uint4(w.x, w.y, 0, 0);
                scale[i] = (v ? a.c.vs : a.c.ks)[row];
            } else {
                raw[i] = load8<CT>(from, row * a.c.D + d0);
            }
            const cham_heads& h = v ? a.vo : a.ko;
            to[i] = (int64_t)(uintptr_t)h.p + ((t0 + tok) * h.token + (int64_t)head * h.head + d0) * (YT == CHAM_T_F32 ? 4 : 2);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (page[i] == -2) continue;
            float y[kChunk] = {};
            if (page[i] >= 0) {
                if constexpr (CT == CHAM_T_E4M3) {
                    decode8_e4m3(make_uint2(raw[i].a.x, raw[i].a.y), y);
#pragma unroll
                    for (int j = 0; j < kChunk; ++j) y[j] *= scale[i];
                } else {
                    widen<CT>(raw[i], y);
                }
            }
            put8<YT>((void*)(uintptr_t)to[i], 0, y);
        }
    }
}

// ------------------------------------------------------------------------------------
// launches
// ------------------------------------------------------------------------------------
// Tokens of a workgroup, and over how many workgroups a token's nv vectors go.  Few vectors: one for
// each group of lanes, so that the card is as full as it can be; else four and more for each, which
// share the tokens' angles (or pages) and load ahead.
void rows_plan(int64_t T, int nv, int groups, int* tok, int* split) {
    const int one = (nv + groups - 1) / groups;
    if (T * one <= 8 * (int64_t)cham_device_cus()) {
        *tok = 1;
        *split = one;
    } else {
        *tok = std::max(1, std::min(kMaxTok, 8 * groups / nv));
        *split = 1;
    }
}

int rotate_check(const cham_rotate* r) {
    if (!r || r->T < 0 || r->D < 1 || r->R < 0 || r->R > r->D || r->R % 2 != 0) return CHAM_EINVAL;
    if (r->D % 8 != 0 || r->D > kMaxD || r->T >= kMaxRows) return CHAM_ESHAPE;
    if (r->layout != CHAM_ROT_HALF && r->layout != CHAM_ROT_PAIRS) return CHAM_EFORMAT;
    if (r->norm != 0 && r->norm != 1) return CHAM_EINVAL;
    if (r->norm) {
        if (!(r->eps >= 0.0f) || r->eps > FLT_MAX) return CHAM_EINVAL;
        if ((r->qg && !float_type(r->qg_type)) || (r->kg && !float_type(r->kg_type))) return CHAM_EFORMAT;
        if ((uintptr_t)r->qg % 16 != 0 || (uintptr_t)r->kg % 16 != 0) return CHAM_EINVAL;
    }
    if (r->R > 0) {
        if (!(r->amp >= -FLT_MAX && r->amp <= FLT_MAX)) return CHAM_EINVAL;
        if (r->T > 0 && (!r->pos || !r->freq || (uintptr_t)r->pos % 4 != 0 || (uintptr_t)r->freq % 8 != 0)) return CHAM_EINVAL;
    }
    return CHAM_OK;
}

template <int XT, int CT>
int launch_rows(RowsArgs& a, hipStream_t s) {
    const int LP = a.r.D <= 64 ? 8 : 16;
    int split;
    rows_plan(a.r.T, a.nv, kThreads / LP, &a.tok, &split);
    a.per = (a.nv + split - 1) / split;
    const int64_t blocks = (a.r.T + a.tok - 1) / a.tok;
    if (split > 65535 || !cham_launchable(blocks * split, kThreads)) return CHAM_ESHAPE;
    const dim3 grid((unsigned)blocks, (unsigned)split);
    if (LP == 8) hipLaunchKernelGGL((heads_kernel<XT, 8, CT>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((heads_kernel<XT, 16, CT>), grid, dim3(kThreads), 0, s, a);
    CHAM_CHECK_LAUNCH();
    return CHAM_OK;
}
template <int CT>
int launch_rows_x(RowsArgs& a, int type, hipStream_t s) {
    if (a.r.T == 0 || a.nv == 0) return CHAM_OK;
    if (type == CHAM_T_F32) return launch_rows<CHAM_T_F32, CT>(a, s);
    if (type == CHAM_T_F16) return launch_rows<CHAM_T_F16, CT>(a, s);
    return launch_rows<CHAM_T_BF16, CT>(a, s);
}

template <int CT, int YT>
int launch_read(ReadArgs& a, hipStream_t s) {
    const int LP = a.c.D <= 64 ? 8 : 16;
    int split;
    rows_plan(a.T, 2 * a.c.H, kThreads / LP, &a.tok, &split);
    a.per = (2 * a.c.H + split - 1) / split;
    const int64_t blocks = (a.T + a.tok - 1) / a.tok;
    if (split > 65535 || !cham_launchable(blocks * split, kThreads)) return CHAM_ESHAPE;
    const dim3 grid((unsigned)blocks, (unsigned)split);
    if (LP == 8) hipLaunchKernelGGL((read_kernel<CT, YT, 8>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((read_kernel<CT, YT, 16>), grid, dim3(kThreads), 0, s, a);
    CHAM_CHECK_LAUNCH();
    return CHAM_OK;
}
template <int CT>
int launch_read_y(ReadArgs& a, hipStream_t s) {
    if (a.ko.type == CHAM_T_F32) return launch_read<CT, CHAM_T_F32>(a, s);
    if (a.ko.type == CHAM_T_F16) return launch_read<CT, CHAM_T_F16>(a, s);
    return launch_read<CT, CHAM_T_BF16>(a, s);
}

}  // namespace
}  // namespace cham

using namespace cham;

extern "C" int cham_norm_rotate(const cham_rotate* r, const cham_heads* q, const cham_heads* qo, const cham_heads* k,
                                const cham_heads* ko, void* stream) {
    int rc = rotate_check(r);
    if (rc != CHAM_OK) return rc;
    if (!q || !qo || !k || !ko || q->H != qo->H || k->H != ko->H) return CHAM_EINVAL;
    if (q->type != k->type || q->type != qo->type || q->type != ko->type) return CHAM_EFORMAT;
    for (const cham_heads* h : {q, qo, k, ko}) {
        rc = heads_check(h, r->T, r->D);
        if (rc != CHAM_OK) return rc;
    }
    if ((q->p == qo->p && (q->token != qo->token || q->head != qo->head) && r->T > 0 && q->H > 0) ||
        (k->p == ko->p && (k->token != ko->token || k->head != ko->head) && r->T > 0 && k->H > 0))
        return CHAM_EINVAL;
    RowsArgs a{{*q, *k, {}}, {*qo, *ko}, *r, {}, nullptr, 0, 0, q->H + k->H, 1.0 / r->D};
    return launch_rows_x<-1>(a, q->type, (hipStream_t)stream);
}

extern "C" int cham_cache_write(const cham_cache* c, const int32_t* slots, const cham_rotate* r, const cham_heads* k,
                                const cham_heads* v, const cham_heads* q, const cham_heads* qo, void* stream) {
    int rc = rotate_check(r);
    if (rc == CHAM_OK) rc = cache_check(c);
    if (rc != CHAM_OK) return rc;
    if (!k || !v || (q == nullptr) != (qo == nullptr) || c->D != r->D || k->H != c->H || v->H != c->H) return CHAM_EINVAL;
    if (k->type != v->type || (q && (q->type != k->type || qo->type != k->type))) return CHAM_EFORMAT;
    if (r->T > 0 && (!slots || (uintptr_t)slots % 4 != 0)) return CHAM_EINVAL;
    rc = heads_check(k, r->T, r->D);
    if (rc == CHAM_OK) rc = heads_check(v, r->T, r->D);
    if (rc == CHAM_OK && q) rc = heads_check(q, r->T, r->D);
    if (rc == CHAM_OK && q) rc = heads_check(qo, r->T, r->D);
    if (rc != CHAM_OK) return rc;
    if (q && (q->H != qo->H || (q->p == qo->p && (q->token != qo->token || q->head != qo->head) && r->T > 0 && q->H > 0)))
        return CHAM_EINVAL;
    const cham_heads none{};
    RowsArgs a{{q ? *q : none, *k, *v}, {q ? *qo : none, none}, *r, *c, slots, 0, 0, (q ? q->H : 0) + 2 * c->H,
               1.0 / r->D};
    if (c->type == CHAM_T_E4M3) return launch_rows_x<CHAM_T_E4M3>(a, k->type, (hipStream_t)stream);
    if (c->type == CHAM_T_F16) return launch_rows_x<CHAM_T_F16>(a, k->type, (hipStream_t)stream);
    return launch_rows_x<CHAM_T_BF16>(a, k->type, (hipStream_t)stream);
}

extern "C" int cham_cache_read(const cham_cache* c, const int32_t* table, int64_t width, const int32_t* cu, int64_t B,
                               int64_t T, const cham_heads* ko, const cham_heads* vo, void* stream) {
    int rc = cache_check(c);
    if (rc != CHAM_OK) return rc;
    if (!ko || !vo || B < 0 || T < 0 || width < 0 || ko->H != c->H || vo->H != c->H) return CHAM_EINVAL;
    if (ko->type != vo->type) return CHAM_EFORMAT;
    if (T >= kMaxRows || B >= kMaxSeqs || width >= (int64_t)1 << 31) return CHAM_ESHAPE;
    rc = heads_check(ko, T, c->D);
    if (rc == CHAM_OK) rc = heads_check(vo, T, c->D);
    if (rc != CHAM_OK) return rc;
    if (T == 0 || B == 0) return CHAM_OK;
    if (!cu || (uintptr_t)cu % 4 != 0 || (width > 0 && (!table || (uintptr_t)table % 4 != 0))) return CHAM_EINVAL;
    ReadArgs a{*c, *ko, *vo, table, cu, width, T, (int)B, 0, 0};
    if (c->type == CHAM_T_E4M3) return launch_read_y<CHAM_T_E4M3>(a, (hipStream_t)stream);
    if (c->type == CHAM_T_F16) return launch_read_y<CHAM_T_F16>(a, (hipStream_t)stream);
    return launch_read_y<CHAM_T_BF16>(a, (hipStream_t)stream);
}

// Rows of heads and caches: the checks of their descriptors.
#pragma once
#include "cham_device.h"

namespace cham {

constexpr int kMaxD = 128;
constexpr int64_t kMaxRows = ((int64_t)1 << 31) - 65536;  // a tile behind the last row is still a 32-bit index
constexpr int64_t kMaxSeqs = (int64_t)1 << 24;
constexpr int kMaxHeads = 65536;
constexpr int64_t kMaxStride = (int64_t)1 << 24;  // 16 rows of keys lie within 31 bits of offsets

inline bool float_type(int t) { return t >= 0 && t < CHAM_T_N; }

inline int heads_check(const cham_heads* h, int64_t T, int D) {
    if (h->H < 0) return CHAM_EINVAL;
    if (h->H > kMaxHeads) return CHAM_ESHAPE;
    if (!float_type(h->type)) return CHAM_EFORMAT;
    if (T == 0 || h->H == 0) return CHAM_OK;
    const int64_t size = h->type == CHAM_T_F32 ? 4 : 2;
    if (!h->p || (uintptr_t)h->p % 16 != 0) return CHAM_EINVAL;
    // a single row's or head's stride is not used
    if (T > 1 && (h->token < D || h->token * size % 16 != 0)) return CHAM_EINVAL;
    if (h->H > 1 && (h->head < D || h->head * size % 16 != 0)) return CHAM_EINVAL;
    return CHAM_OK;
}

inline int cache_check(const cham_cache* c) {
    if (!c || c->pages < 1 || c->H < 1 || c->D < 1) return CHAM_EINVAL;
    if (c->page < 16 || c->page > 32768 || (c->page & (c->page - 1)) != 0) return CHAM_ESHAPE;
    if (c->H > kMaxHeads || c->D > kMaxD || c->D % (c->type == CHAM_T_E4M3 ? 16 : 8) != 0 ||
        c->pages >= ((int64_t)1 << 31) / c->page)
        return CHAM_ESHAPE;
    if (c->type != CHAM_T_F16 && c->type != CHAM_T_BF16 && c->type != CHAM_T_E4M3) return CHAM_EFORMAT;
    if (!c->k || !c->v || (uintptr_t)c->k % 16 != 0 || (uintptr_t)c->v % 16 != 0) return CHAM_EINVAL;
    if ((c->type == CHAM_T_E4M3) != (c->ks != nullptr) || (c->type == CHAM_T_E4M3) != (c->vs != nullptr)) return CHAM_EINVAL;
    if ((uintptr_t)c->ks % 4 != 0 || (uintptr_t)c->vs % 4 != 0) return CHAM_EINVAL;
    return CHAM_OK;
}

}  // namespace cham

// Where the block product's loads into LDS lie: the arithmetic that keeps them in their buffer,
// shared by the kernel and the host's checks of it.
#pragma once
#include <stdint.h>

namespace cham {

constexpr int BK = 128;                     // one block of the format: bytes of a row per step
constexpr uint32_t kOutside = 0x80000000u;  // an offset past every buffer: such loads give zeros

// A buffer load reads `lane + wave` bytes from the buffer's base, and zeros where it is outside.
struct LoadAt {
    uint32_t lane, wave;
};

// whether chunk c (16 bytes) of the last of nkb k-steps lies past a row of K bytes
__host__ __device__ inline bool past_row(int nkb, int c, int K) { return (nkb - 1) * BK + c * 16 >= K; }

// The load of k-step kb whose row and chunk start `off` bytes into the buffer; last: past_row of
// its chunk.  Loads are issued up to two steps past the last one.  The range check compares `lane`
// with the buffer's size less `wave`, in 32 bits: `wave` stays within the buffer for those too,
// else the difference would wrap and kOutside would count as inside.
__host__ __device__ inline LoadAt load_at(uint32_t off, bool last, int kb, int nkb) {
    const bool past = kb >= nkb || (kb == nkb - 1 && last);
    return {past ? kOutside : off, (uint32_t)((kb < nkb ? kb : nkb - 1) * BK)};
}

}  // namespace cham

// Host model of the block product's loads into LDS (no GPU code runs): every load of a tile whose
// last rows end the matrix, against what it has to read.
#include "../../paper_2609_33496_amd/csrc/cham_block_load.h"

using namespace cham;

// The range check of a raw buffer load as it is documented: outside where the lane's offset is not
// below num_records - the scalar offset, a difference of 32 bits.
static bool outside(LoadAt l, uint32_t records) { return l.lane >= records - l.wave; }

// Tiles of bm rows (kLoads rows apart), the last one with `rows` rows of K codes, steps up to
// `ahead` past the last: the number of loads that read anything but their own chunk, or read it
// where zeros are due.
extern "C" long block_load_faults(int bm, int rows, int K, int ahead) {
    const int nkb = (K + BK - 1) / BK;
    const uint32_t records = (uint32_t)rows * K;
    long bad = 0;
    for (int kb = 0; kb < nkb + ahead; ++kb)
        for (int r = 0; r < bm; ++r)
            for (int c = 0; c < 8; ++c) {
                // a lane's first row and chunk, and the rows of its later loads
                LoadAt l = load_at((uint32_t)(r & 31) * K + c * 16, past_row(nkb, c, K), kb, nkb);
                l.lane += (uint32_t)(r & ~31) * K;
                const bool due = r < rows && kb < nkb && kb * BK + c * 16 < K;
                const uint64_t at = (uint64_t)l.lane + l.wave;
                if (outside(l, records) ? due : !due || at != (uint64_t)r * K + kb * BK + c * 16) ++bad;
            }
    return bad;
}

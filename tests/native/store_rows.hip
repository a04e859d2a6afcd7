// Host model of the linear layer's stores (no GPU code runs): every row that a tile of tm blocks of 32
// stores, where the last tile ends the matrix.
#include "../../paper_2609_33496_amd/csrc/cham_store.h"

using namespace cham;

// The range check of a raw buffer store as it is documented: dropped where the lane's offset is not
// below num_records - the scalar offset, a difference of 32 bits.  Counts the stores that are dropped
// and should not be, or the other way round, or go elsewhere.
extern "C" long store_faults(int tm, int rows, int N) {
    const uint32_t bytes = (uint32_t)N * 4, records = (uint32_t)rows * bytes;
    long bad = 0;
    for (int i = 0; i < tm; ++i)
        for (int h = 0; h < 2; ++h)
            for (int r = 0; r < 16; ++r)
                for (int n : {0, N / 2, N - 1}) {
                    const int row = 32 * i + 4 * h + 8 * (r >> 2) + (r & 3);
                    const uint32_t voff = (uint32_t)(32 * i + 4 * h) * bytes + n * 4;
                    const uint32_t soff = row_offset(8 * (r >> 2) + (r & 3), bytes, records);
                    const bool dropped = voff >= records - soff, due = row < rows;
                    if (dropped == due || (due && voff + soff != (uint32_t)row * bytes + n * 4)) ++bad;
                }
    return bad;
}

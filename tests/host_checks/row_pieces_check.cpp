// Host check of how the narrow forward kernel finds the row of a 16-byte piece (paper_2212_01185_amd/csrc/train_narrow.h, the source that
// the kernel compiles): against integer division, for every number of pieces that its launch lets through and every piece of a wave's rows.
// Prints one line "checked <n> failures <m>" and exits 0 iff m == 0.
#include <cstdio>

#include "train_narrow.h"

int main() {
    using namespace pcc_train;
    long checked = 0, failures = 0;
    for (int pieces = 1; pieces <= kMaxRowPieces; ++pieces)
        for (int id = 0; id < kNarrowRowsWave * pieces; ++id, ++checked) failures += row_of_piece(id, pieces_inverse(pieces)) != id / pieces;
    std::printf("checked %ld failures %ld\n", checked, failures);
    return failures != 0;
}

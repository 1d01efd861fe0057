// Which kernel a call of xc_scores_microscaled takes, by sizes alone.  Host code without HIP.
#pragma once

#include <stdint.h>

namespace xc {

enum MicroKernel {
    kMicroOnline,        // few queries in LDS, brought to 4 bits by every workgroup
    kMicroFew,           // few queries in LDS, from the workspace
    kMicroHeld,          // 512 labels in registers
    kMicroSmall,         // tiles of 128 x 128
    kMicroLarge          // tiles of 256 x 256
};

constexpr int kMicroCus = 256, kMicroXcds = 8;           // compute units of the device
constexpr int kMicroFewQueries = 16;                     // at most
constexpr int kMicroShortUnits = 8, kMicroFewUnits = 32; // units of 128 elements of a row of few queries: two sizes of their place in LDS
constexpr int64_t kMicroInline = 128;                    // units of queries: two rounds of a workgroup's loads (16 x 131072 x 4096, 512 of
                                                         // them: 81 us, in a launch of their own 64; 4 x 2487 x 3280, 104: 14.7 against 18.8 with one round)
constexpr int kMicroHeldLabels = 512, kMicroHeldUnits = 8, kMicroHeldQueries = 64 /* of a stage */;
constexpr int kMicroSmallSide = 128, kMicroSmallPerCu = 2, kMicroLargeSide = 256, kMicroLargePerCu = 1;           // tiles, workgroups of them to a compute unit

// Labels in registers: from four stages to a compute unit on, for more than 256 queries (a tile's labels cost a workgroup as much as several
// stages) and tiles for all XCDs.  Held against in tiles, d = 768: 64 x 670000 92 us and 82, 256 x 64000 19.9 and 17.6, 2000 x 8000 18.5 and
// 18.1, 2000 x 16000 25.0 and 26.0, 400 x 131072 43.5 and 49.9, 10000 x 2000 35 and 28, 10000 x 4000 38 and 46, 10000 x 64000 300 and 460.
// Other rows: d = 128: 2000 x 16000 19.1 and 17.9, 400 x 131072 23.4 and 23.2, 4096 x 131072 187 and 211; d = 256: 10000 x 64000 256 and 257,
// 300 x 140001 24.1 and 27.9; d = 1024: 2000 x 8000 23.1 and 20.9, 2000 x 16000 30.4 and 32.6, 300 x 140001 44 and 55, 4096 x 131072 296 and 473.
// To fp32 the sides differ by as much or more (d = 128: 2000 x 16000 26.2 and 26.1; d = 1024: 2000 x 16000 33.4 and 43.3, 2000 x 8000 24.3 and 26.6).
inline bool hold_labels(int64_t B, int64_t L, int units) {
    const int64_t tiles = (L + kMicroHeldLabels - 1) / kMicroHeldLabels, stages = (B + kMicroHeldQueries - 1) / kMicroHeldQueries;
    return units <= kMicroHeldUnits && B > 256 && tiles >= kMicroXcds && tiles * stages >= 4 * kMicroCus;
}
// Tiles of 128 x 128, two workgroups of them to a compute unit, or of 256 x 256: whichever's rounds take less, a round of large ones
// 5/3 of the others' (d = 2048, small against large: 2000 x 2000 18.3 us against 27.8, 300 x 50021 40.9 against 44.3, 2000 x 6000 29.0
// against 28.2, 4096 x 4096 35.3 against 29.5; 4096 x 131072 x 4096 1817 against 1346; d = 1152: 2000 x 2000 15.4 against 22.6, 300 x 50021 28.9
// against 33.3, 2000 x 6000 24.0 against 22.4, 4096 x 4096 29.8 against 25.3; d = 4096: 30.8 against 47.8, 69.0 against 76.1, 52.9 against 48.1,
// 65.1 against 53.1.  To bf16; to fp32 large tiles cost up to 20 % more: 2000 x 6000 x 4096 54.8 against 57.1, 4096 x 4096 x 1152 31.9 against 33.0).
inline bool small_tiles(int64_t B, int64_t L) {
    auto rounds = [&](int64_t side, int64_t at_once) { return ((B + side - 1) / side * ((L + side - 1) / side) + at_once - 1) / at_once; };
    return rounds(kMicroLargeSide, kMicroCus * kMicroLargePerCu) * 5 > rounds(kMicroSmallSide, kMicroCus * kMicroSmallPerCu) * 3;
}
// units: of 128 elements in a row.
inline MicroKernel choose_micro(int64_t B, int64_t L, int units) {
    if (B <= kMicroFewQueries && units <= kMicroFewUnits) return B * units <= kMicroInline ? kMicroOnline : kMicroFew;
    if (hold_labels(B, L, units)) return kMicroHeld;
    return small_tiles(B, L) ? kMicroSmall : kMicroLarge;
}

}  // namespace xc

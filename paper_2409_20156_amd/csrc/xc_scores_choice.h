// Which kernel a call of xc_scores_quantized takes, by sizes alone.  Host code without HIP.
#pragma once

#include <stdint.h>

namespace xc {

enum ScoresKernel {
    kScoresOnline,       // 16 x 128, queries brought to integers by every workgroup
    kScoresThin,         // 16 x 16
    kScoresNarrow,       // 32 x 32
    kScoresFew,          // 32 x 128
    kScoresLow,          // 64 x 32
    kScoresSmall,        // 64 x 64
    kScoresSome,         // 64 x 128
    kScoresHeld,         // 512 labels in registers
    kScoresMid,          // 128 x 128
    kScoresMany          // 256 x 256
};

constexpr int kScoresUnits = 256, kScoresXcds = 8;           // compute units of the device
constexpr int kOnlineQueries = 16, kOnlineBytes = 768;
constexpr int kHeldLabels = 512, kHeldBytes = 768;

// Up to 16 queries on rows of up to 768 bytes: one launch, every workgroup brings the queries to integers for itself (1 x 131072 x
// 768: 18.3 us a call, 21.0 with a launch of their own; 1 x 4000 x 768: 8.0 and 10.8; 16 x 131072 x 768: 23.5 and 24.2; with
// tiles of 32, 32 x 131072 x 768: 29.9 and 26.3, so not beyond 16).
// Which kernel.  Measured with rows of Q from memory (us, scores alone, on the sides of each rule):
//   up to 32 queries   32 x 128; fewer labels than 256 such tiles 32 x 32, and up to 16 queries or 256 of those 16 x 16: a compute unit
//                      keeps only so many lines of memory under way, so a short call wants many of them at it (32 x 30000 x 4096: 31,
//                      38 with 16 x 16; 32 x 6000 x 4096: 24 and 14; 12 x 10000 x 4096: 23 and 15, with 32 x 128 24)
//   up to 512 tiles of 64 x 64   these; up to 256 of 64 x 32 those (128 x 16000 x 768: 8.5 against 10.0 with 128 x 128 and 12 with 64 x 32;
//                      400 x 4000 x 4096: 25, 35 and 34; 128 x 4000 x 4096: 21, with 64 x 32 16)
//   up to 64 queries   64 x 128 (64 x 300000 x 768: 59; 128 x 128 70, 64 x 64 62)
//   more than 1792 tiles of 128 x 128, rows of up to 768 bytes and more than 384 queries, or up to 384 and 128   labels held in registers
//                      (4096 x 131072 x 768 to bf16: 360; 256 x 256 tiles 545; 700 x 74141 x 768: 67, 128 x 128 tiles 74; 340 x 526924 x
//                      320: 143 and 168; 700 x 34200 x 768, 1608 tiles: 43 and 36; 340 x 188544 x 512: 83 and 72)
//                      Whole tiles of 512 labels go to an XCD: not where the busiest has more than half as many again as the mean (1 to 5,
//                      9 and 10 tiles), which left up to seven XCDs without work (to fp32, bf16, held and 128 x 128: 65948 x 512 x 768:
//                      167, 145 and 50, 43; 22521 x 1499 x 768: 85, 78 and 62, 43; 7385 x 4571 x 768: 67, 61 and 61, 44; lost by it, to
//                      fp32: 34909 x 2523 x 768 143 and 152, 19000 x 5115 x 768 150 and 171).  To bf16, where 128 x 128 tiles store at less
//                      cost, the 1792 are counted with what the busiest XCD has eight times (4096 x 8700 x 768: 60 and 42; 2645 x 12763 x
//                      192: 32 and 26; on the other side 6901 x 12763 x 768: 94 and 97), to fp32 not (4096 x 9000 x 384: 45 and 54; 2001
//                      x 16859 x 768: 54 and 73)
//   else 128 x 128 tiles or, beyond 192 queries, 256 x 256 where that takes fewer rounds for its larger tiles (to bf16 512 x 209651 x
//                      1024: 137 against 185; 1000 x 93139 x 4096: 338 against 428; 256 x 188816 x 512: 44 against 56; 800 x
//                      17762 x 1536: 51 against 34, so not there; 130 x 141461 x 800: 71 against 55).  Short rows beyond 256 queries
//                      are no longer worth it (300 x 87520 x 384: 37 against 29).
// ppitch: bytes of a query's row in 8 bits, whole stages of 128; out_bytes: of a score.
inline ScoresKernel choose_scores(int64_t B, int64_t L, int ppitch, int out_bytes) {
    auto tiles = [&](int m, int n) { return (B + m - 1) / m * ((L + n - 1) / n); };
    if (B <= kOnlineQueries && ppitch <= kOnlineBytes) return kScoresOnline;
    if (B <= 32) {
        if (tiles(32, 128) >= kScoresUnits) return kScoresFew;
        return B <= 16 || tiles(32, 32) <= kScoresUnits ? kScoresThin : kScoresNarrow;
    }
    if (tiles(64, 32) <= kScoresUnits) return kScoresLow;
    if (tiles(64, 64) <= 2 * kScoresUnits) return kScoresSmall;
    if (B <= 64) return kScoresSome;
    const int64_t held = (L + kHeldLabels - 1) / kHeldLabels, busiest = (held + kScoresXcds - 1) / kScoresXcds * kScoresXcds;
    if (B > 128 && ppitch <= (B > 384 ? kHeldBytes : kHeldBytes / 2) && 2 * busiest <= 3 * held &&
        tiles(128, 128) * (out_bytes == 2 ? held : busiest) > 7 * kScoresUnits * busiest)
        return kScoresHeld;
    const int64_t mid = (tiles(128, 128) + 2 * kScoresUnits - 1) / (2 * kScoresUnits), many = (tiles(256, 256) + kScoresUnits - 1) / kScoresUnits;
    return B <= 192 || (ppitch <= kHeldBytes && B > 256) || 5 * mid <= 8 * many ? kScoresMid : kScoresMany;
}

}  // namespace xc

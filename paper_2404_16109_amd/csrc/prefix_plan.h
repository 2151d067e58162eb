// How attention behind a shared prefix is spread over the chip: rows to a workgroup, parts of the prefix and of each sequence's own keys.
// Plain C++: tests go through it on the host.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace zkmi {

static const uint32_t kPrefixTile = 64, kPrefixWorkgroups = 512;  // tokens; that the chip holds
inline uint64_t prefix_parts(uint64_t n, uint64_t each) { return (n + each - 1) / each; }

// Wavefronts to a workgroup, 32 rows to each: of many rows eight share what a tile costs to bring, where their sums fit the registers; with
// four there is room on a CU for a workgroup of the other kind beside, which few rows need more.
inline bool prefix_eight_waves(uint64_t rows, uint32_t head_dim) { return rows >= 1024 && head_dim <= 128; }
static const uint32_t kMostParts = 32;  // of the prefix, and of a sequence's own keys

// Whether a sequence's rows (of a head of the cache) go through the kernel of few rows, and its tiles of 16 rows; 0: many.
inline bool prefix_few(uint64_t rows) { return rows <= 32; }
inline int prefix_row_tiles(uint64_t rows) { return rows <= 16 ? 1 : prefix_few(rows) ? 2 : 0; }

// How a call is spread.  rows: of the batch and a head; most: of a sequence and a head.
struct PrefixPlan {
    uint32_t row_tile, front_tiles, front_splits, front_each, splits, each;
};
inline PrefixPlan prefix_plan(uint32_t seqs, uint64_t rows, uint64_t most, uint32_t kv_heads, uint32_t head_dim, uint32_t prefix, uint32_t max_len) {
    PrefixPlan p = {};
    p.front_tiles = prefix / kPrefixTile;
    p.row_tile = prefix_eight_waves(rows, head_dim) ? 256 : 128;
    const auto share = [](uint64_t groups, uint32_t tiles, uint32_t& splits, uint32_t& each) {
        uint64_t n = groups >= kPrefixWorkgroups / 2 ? 1 : prefix_parts(kPrefixWorkgroups, groups);
        if (n > prefix_parts(tiles, 4)) n = prefix_parts(tiles, 4);
        if (n > kMostParts) n = kMostParts;
        each = (uint32_t)prefix_parts(tiles, n);
        splits = (uint32_t)prefix_parts(tiles, each);
    };
    if (p.front_tiles) {
        // Time of the prefix by the number of parts, in us: as many rounds of a workgroup to each CU as it takes, 0.41 (0.57 with eight
        // wavefronts) a tile for each 32 dimensions and 1 to begin with, and the parts' way to memory and back at 4 TB/s.  Measured for 320
        // rows and 8 heads of 128 behind 8192 tokens, whole call: 4 parts 71 us, 8 46, 10 42, 16 44, 32 56.
        const uint64_t groups = kv_heads * prefix_parts(rows, p.row_tile);
        double best = 0.0;
        for (uint32_t n = 1; n <= kMostParts && n <= p.front_tiles; ++n) {
            const uint32_t each = (uint32_t)prefix_parts(p.front_tiles, n);
            if (prefix_parts(p.front_tiles, each) != n) continue;
            const double us = (double)prefix_parts(groups * n, kPrefixWorkgroups / 2) * ((p.row_tile == 256 ? 0.57 : 0.41) * each * (double)prefix_parts(head_dim, 32) + 1.0) +
                              (double)(kv_heads * rows * head_dim) * n * 8.0 / 4e6;
            if (n == 1 || us < best) {
                best = us;
                p.front_splits = n;
                p.front_each = each;
            }
        }
    }
    const uint32_t own = max_len > p.front_tiles * kPrefixTile ? (uint32_t)prefix_parts(max_len - p.front_tiles * kPrefixTile, kPrefixTile) : 1;
    share((uint64_t)seqs * kv_heads * (prefix_few(most) ? 1 : prefix_parts(most, p.row_tile)), own, p.splits, p.each);
    return p;
}

}  // namespace zkmi

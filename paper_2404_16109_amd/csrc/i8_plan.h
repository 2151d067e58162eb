// How a product of 8-bit integers is spread over the chip: which kernel and tile, and in how many parts of k.
// Plain C++: tests go through it on the host.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace zkmi {

static const uint32_t kStep = 128;  // of k
static const int kWaves = 8;        // of a workgroup of k_few
inline uint64_t i8_parts(uint64_t n, uint64_t each) { return (n + each - 1) / each; }

enum I8Tile { kFew, kShort, kMid, kWide, kLarge };
struct I8Plan {
    I8Tile tile;
    uint32_t nt, groups, splits, each;  // nt: tiles of 16 outputs to a workgroup of k_few
};
inline void i8_share_k(I8Plan& p, uint32_t steps, uint32_t splits) {
    p.each = (uint32_t)(i8_parts(i8_parts(steps, splits), 2) * 2);  // k_tiles takes two steps at a time
    p.splits = (uint32_t)i8_parts(steps, p.each);
}

// Up to 32 rows.  More outputs to a workgroup read x less often, fewer fill the chip.  Measured, us, weights from HBM, 16 / 32 / 64 outputs
// to a workgroup: one row by 13824 x 5120 16.8 18.6 19.1, 16 rows 25.2 23.6 20.9, 32 rows 38 29 23.7; 32 rows by 5120 x 13824 46 33 48, and
// with k shared by three 36 29 24.3; 32 rows by 5120 x 5120 16 11.9 16.4 (shared 15 13 12.3); 16 rows by 2000 x 8192 9.9 13.2.  Few outputs
// share a long k, which costs a launch: one row by 941 x 21856 11.9 us in one part, 7.9 in four, by 339 x 10768 7.2 and 5.7 in a graph, but 7.4
// and 9.3 called from Python, where launches count; by 500 x 4096 4.7 and 4.8.
inline I8Plan i8_plan_few(uint32_t rows, size_t n, uint32_t steps) {
    I8Plan p = {};
    p.tile = kFew;
    const bool shares = rows > 16 && steps >= 64;  // a part takes sixteen steps at least, and a launch to join them
    p.nt = rows <= 4 ? 1 : n >= 64 * 200 || (shares && n >= 64 * 32) ? 4 : n >= 32 * 128 ? 2 : 1;
    p.groups = (uint32_t)i8_parts(n, 16 * p.nt);
    uint32_t splits = p.groups < 128 ? 256 / p.groups : 1;
    const uint32_t most = p.nt == 4 || steps >= 96 ? steps / (2 * kWaves) : 1;
    if (splits > most) splits = most;
    i8_share_k(p, steps, splits ? splits : 1);
    return p;
}

// Tiles of more rows: rows and outputs, workgroups to a CU, and us a step of 128 with one, two or three of them there.  Measured with
// as many tiles as the chip takes at once, the difference between k 8192 and 2048.
struct I8Shape {
    uint32_t rows, outs, slots;
    double step[3];
};
static const I8Shape kShapes[] = {{}, {64, 128, 3, {0.57, 0.81, 0.90}}, {128, 128, 2, {0.66, 0.95}}, {192, 256, 1, {1.38}}, {256, 256, 1, {1.69}}};

// The tile and the parts of k that take least: rounds of the chip's 256 CUs, each with what a workgroup begins and ends with, and the parts'
// way to memory and back.  Measured and, in brackets, tiles of 128 x 128 in as many parts as are best: 2048 x 5120 x 5120 56.7 us (76.5), of
// 600 x 2000 x 27200 58.0 (58.0), of 1000 x 5120 x 5120 38.9 (38.9), of 8192 x 13824 x 5120 523.
inline I8Plan i8_plan_tiles(size_t rows, size_t n, uint32_t steps) {
    I8Plan best = {};
    double least = 0.0;
    for (int t = kShort; t <= kLarge; ++t) {
        const I8Shape& s = kShapes[t];
        const uint64_t groups = i8_parts(rows, s.rows) * i8_parts(n, s.outs);
        if (t < kLarge && groups >= (uint64_t)1 << 22) continue;  // a launch holds fewer than 2^32 threads
        for (uint32_t splits = 1; splits <= 16 && splits * 4 <= (steps < 4 ? 4 : steps); ++splits) {
            if (splits > 1 && groups * (splits - 1) >= 256 * s.slots) break;
            I8Plan p = {};
            p.tile = (I8Tile)t;
            p.groups = (uint32_t)groups;
            i8_share_k(p, steps, splits);
            const uint64_t all = groups * p.splits, chip = 256 * s.slots, rest = all % chip;
            const double rounds = (double)(all / chip) * (p.each * s.step[s.slots - 1] + 3.0) + (rest ? p.each * s.step[(rest - 1) / 256] + 3.0 : 0.0);
            const double us = rounds + (p.splits > 1 ? 2.0 + 8.0 * (double)rows * (double)n * p.splits / 8e6 : 0.0);
            if (!best.groups || us < least) {
                least = us;
                best = p;
            }
        }
    }
    return best;
}
inline I8Plan i8_plan(size_t rows, size_t n, size_t k) {
    const uint32_t steps = (uint32_t)i8_parts(k, kStep);
    return rows <= 32 ? i8_plan_few((uint32_t)rows, n, steps) : i8_plan_tiles(rows, n, steps);
}

}  // namespace zkmi

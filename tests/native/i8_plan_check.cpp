// Host build of how a product of 8-bit integers is spread (csrc/i8_plan.h).  Compiled with g++ by tests/test_i8_plan.py;
// nothing here runs on a GPU.
#include "../../paper_2404_16109_amd/csrc/i8_plan.h"

using namespace zkmi;

extern "C" void c_plan(size_t rows, size_t n, size_t k, uint32_t* out) {
    const I8Plan p = i8_plan(rows, n, k);
    const uint32_t v[5] = {(uint32_t)p.tile, p.nt, p.groups, p.splits, p.each};
    for (int j = 0; j < 5; ++j) out[j] = v[j];
}
extern "C" void c_tile(int tile, uint32_t* out) {
    out[0] = kShapes[tile].rows;
    out[1] = kShapes[tile].outs;
}

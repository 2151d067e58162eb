// Host build of how attention behind a shared prefix is spread (csrc/prefix_plan.h).  Compiled with g++ by tests/test_prefix_plan.py;
// nothing here runs on a GPU.
#include "../../paper_2404_16109_amd/csrc/prefix_plan.h"

using namespace zkmi;

// rows: of the batch and a head of the cache; most: of a sequence and a head
extern "C" void c_plan(uint32_t seqs, uint64_t rows, uint64_t most, uint32_t kv_heads, uint32_t head_dim, uint32_t prefix, uint32_t max_len, uint32_t* out) {
    const PrefixPlan p = prefix_plan(seqs, rows, most, kv_heads, head_dim, prefix, max_len);
    const uint32_t v[8] = {p.row_tile,  p.front_tiles, p.front_splits, p.front_each,
                           p.splits,    p.each,        (uint32_t)prefix_row_tiles(most), prefix_eight_waves(rows, head_dim) ? 8u : 4u};
    for (int j = 0; j < 8; ++j) out[j] = v[j];
}

// Host build of how k_attend_many's threads share out a tile (csrc/attend_pieces.h).  Compiled with g++ by
// tests/test_attend_pieces.py; nothing here runs on a GPU.
#include "../../paper_2404_16109_amd/csrc/attend_pieces.h"

using namespace zkmi;

template <int DT>
static void fill(uint32_t threads, uint32_t rounds, uint32_t* out) {
    for (uint32_t i = 0; i < rounds; ++i)
        for (uint32_t t = 0; t < threads; ++t) {
            const AttendPiece p = attend_piece<DT>(t, threads, i);
            const uint32_t v[6] = {p.p, p.slot, p.c, p.dim, p.run, attend_piece_kept<DT>(t, threads, i)};
            for (int j = 0; j < 6; ++j) out[(i * threads + t) * 6 + j] = v[j];
        }
}

extern "C" void c_pieces(int dt, uint32_t threads, uint32_t rounds, uint32_t* out) {
    switch (dt) {
        case 1: return fill<1>(threads, rounds, out);
        case 2: return fill<2>(threads, rounds, out);
        case 3: return fill<3>(threads, rounds, out);
        case 4: return fill<4>(threads, rounds, out);
        case 5: return fill<5>(threads, rounds, out);
        case 6: return fill<6>(threads, rounds, out);
        case 7: return fill<7>(threads, rounds, out);
        case 8: return fill<8>(threads, rounds, out);
    }
}

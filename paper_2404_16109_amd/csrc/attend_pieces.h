// How the threads of k_attend_many share out a tile of 64 tokens: which 16 codes of K, and which of V, a thread brings.
// Plain C++: tests go through it on the host.
#pragma once
#include "small_dev.h"

namespace zkmi {

// Piece p of a tile: of K, dimensions 16 c .. of token `slot`; of V, tokens 16 `run` .. of dimension `dim`.
struct AttendPiece {
    uint32_t p, slot, c, dim, run;
};
// DT: head_dim in units of 32, rounded up; a tile has 128 DT pieces.  Thread tid of `threads` brings piece tid + threads * i in
// round i; where there is none, one that another thread brings too: what is read lies inside the tile, and is not kept.
template <int DT>
ZK_SHD AttendPiece attend_piece(uint32_t tid, uint32_t threads, uint32_t i) {
    AttendPiece a;
    a.p = (tid + threads * i) % (128 * DT);
    a.slot = a.p / (2 * DT);
    a.c = a.p % (2 * DT);
    a.dim = a.p >> 2;
    a.run = a.p & 3;
    return a;
}
// Whether the thread's piece of round i is its own.
template <int DT>
ZK_SHD bool attend_piece_kept(uint32_t tid, uint32_t threads, uint32_t i) {
    return tid + threads * i < 128 * DT;
}

}  // namespace zkmi

// How the pieces of moved rows are dealt to threads (evict_accumulated.hip). A header of its own because it is checked on the host
// as well (tests/row_moves_check.cpp).
#pragma once

#include <hip/hip_runtime.h>

namespace audiokv {

// A thread's pieces: piece `piece` of moves first, first + step, ... `per` pieces to a move, a power of two that divides `threads`.
// (Moves are counted, not pieces: 2^25 moves of 64 pieces leave 32 bits.)
struct MoveWalk {
    int first, step, piece;
};
__host__ __device__ inline MoveWalk move_walk(int thread, int threads, int per) { return MoveWalk{thread / per, threads / per, thread % per}; }

}  // namespace audiokv

// Workgroups of latent_write: how many of each kind, and what one of them does.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ordermoe {

constexpr int LW_TOK = 64, LW_COLS = 64;             // tokens and ranks of an absorb workgroup
// pieces of a thread that are on their way together, in workgroups of one kind (one each, mixed in a wave: 152 us for 99)
constexpr int LW_COPIES = 4, LW_TURNS = 2;

struct WriteBlocks {
    int64_t absorb, rows, copies, turns;
    enum Kind { ABSORB, ROWS, COPY, TURN, NONE };
    // What workgroup blk does; blk becomes its number among those of its kind.  (NONE: a launch of more than 2^22
    // workgroups is rounded up, and what lies past the last of them may have no queries to turn.)
    __host__ __device__ Kind kind(int64_t& blk) const {
        if (blk < absorb) return ABSORB;
        blk -= absorb;
        if (blk < rows) return ROWS;
        blk -= rows;
        if (blk < copies) return COPY;
        blk -= copies;
        return blk < turns ? TURN : NONE;
    }
};
// T tokens with or without queries, absorbed or copied
inline WriteBlocks write_blocks(int64_t T, int n_q, int head_dim, int rank, int rot, bool queries, bool absorb) {
    const int64_t heads = queries ? T * n_q : 0;
    const int64_t per_copy = 256 / (head_dim / 8) * LW_COPIES, per_turn = 256 / (rot / 16) * LW_TURNS;
    return WriteBlocks{queries && absorb ? (T + LW_TOK - 1) / LW_TOK * n_q * (rank / LW_COLS) : 0, (T + 3) / 4,
                       absorb ? 0 : (heads + per_copy - 1) / per_copy, (heads + per_turn - 1) / per_turn};
}

}  // namespace ordermoe

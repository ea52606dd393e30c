// The products of the losses over a vocabulary: what their tiles read and write (see vocab_tiles.hip), and how they are launched.
#pragma once

#include "vocab.h"

namespace snn {

// What a call finds out about its rows on the device: how many count, and the powers of two that bring their gradients into the type's range
// and back.
struct LossHead {
    int count;
    float up, down;
};

// The four products.  Rows t are those that count, next to each other; tokens v are all (STATS) or a piece of the vocabulary.
//   STATS   z[v][t] = table[v] . x[t]; of a tile the largest and the sum of exponentials for each row, and the logits of the listed tokens
//   PROBS   z again; probs[t][v] = g[t] (2^(c z - lse2[t]) - the listed tokens' q), rounded to 16 bits
//   ROWS    sums over v of probs[t][v] table[v][c], fp32, in parts of the piece
//   TABLE   sums over t of probs[t][v] x[t][c]: rows of the table's gradient
enum { STATS, PROBS, ROWS, TABLE };

struct TilesArgs {
    const void *a, *b;                // the operands that give the tile's rows (M) and columns (N)
    int64_t lda, ldb;
    int M, N, K;                      // count limits N, in TABLE K
    const LossHead *head;             // nullptr: as given
    float c;                          // log2(e) / temperature
    int v0;                           // first token of the piece
    const int32_t *ids;               // token j of row t at t * id_row + j * id_k
    const float *q;                   // its share, likewise; nullptr: one
    int64_t id_row, id_k;
    int k;
    float2 *part;                     // STATS: [tile of tokens][part_ld]
    int64_t part_ld;
    float *picked;                    // [row of the call][k]
    const int *list;                  // the rows that count; nullptr: all
    const float *lse2, *g;
    void *probs;
    int64_t ldp;
    float *out;                       // ROWS: [split][N][M]
    int64_t out_split;
    int steps, most_splits, add;      // splits go by the first piece's steps; add: to what earlier pieces left
    void *dtable;                     // TABLE
    int accumulate;
};

// How many parts the contracted axis of ROWS is cut into: as many as leave the fewest turns of the chip's 256 workgroups for the work of one.
__host__ __device__ inline int row_splits(int tiles, int steps, int most)
{
    int best = 1;
    float least = 0.0f;
    for (int s = 1; s <= most && s <= (steps + 7) / 8; ++s) {
        const float turns = (float)((tiles * s + 255) / 256);
        const float cost = turns * ((float)((steps + s - 1) / s) + 6.0f) + 0.5f * (float)s;
        if (s == 1 || cost < least) {
            best = s;
            least = cost;
        }
    }
    return best;
}

// Tile shapes (tile rows x columns)
enum { TILE_256, TILE_128, TILE_FEW };
inline int tile_m(int form) { return form == TILE_256 ? 256 : 128; }
inline int tile_n(int form) { return form == TILE_256 ? 256 : form == TILE_128 ? 128 : 64; }

int launch_vocab_tiles(int kind, int form, int dtype, const TilesArgs &p, hipStream_t s);

}  // namespace snn

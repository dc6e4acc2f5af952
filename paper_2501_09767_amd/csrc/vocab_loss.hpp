// Parameter blocks and launchers of the loss over a vocabulary (vocab_loss.hip, vocab_loss_tiles.hip).
#pragma once
#include "gather_gemm.hpp"

namespace lemo {

// What turns logits into losses: u = softcap tanh(x / softcap) (0: u = x), hit = 1 - smoothing, all = smoothing / V.
struct VocabRule {
    float softcap, hit, all, z;
    int V;
};

// What the kernels that form G do beside it, for the products that follow.
//   parts     2: behind the M rows of G stand M more, of what rounding the first has left, which meet the same rows of X in the weight's gradient.  Where both
//             fit the one slab that its contraction is padded to, so at no product's cost; bf16 only.
//   rows [parts M + 1]   the rows of X for the weight's gradient, those without a label replaced by `past`, one past X's end, which the loads' range check
//             turns into zeros whatever such a row holds.  Entry parts M is one more of those, and row parts M of G zeros where the vocabulary does not fill
//             whole pieces of 16 bytes (zero_row): the last row of G that a product reads is then one of zeros, whose last piece of columns may
//             end in the operand's middle.
//   uniform   one gradient for all losses: G is formed for gradients of `uniform` each (1 / (1 - smoothing), which makes the label's share 1), the rest is
//             multiplied into the results.  0: gradients of their own.
struct VocabSide {
    const float* dloss;  // gradients of the losses
    long long stride;
    float uniform;
    int* rows;           // or null: not the first piece
    int past, zero_row, parts;
};

// A product of the rows with (a piece of) the head's weight and what is done with a tile of it.  GgParams: A = X [S, C], idx = the kept rows, B = the piece's
// first row of W, M, N = the piece's columns, K = C; for the planes A = G, B = W (contraction-major), K = the piece's columns, N = C; for the weight's
// gradient A = G, B = X (both contraction-major, X's rows by idx), M = the piece's columns, N = C, K = rows.
struct VocabTileParams : GgParams {
    VocabRule rule;
    const int* labels;     // [M]
    int v0;                // the piece's first column in the vocabulary
    float2* parts;         // statistics: [tiles_n][M] maximum, sum of exponentials
    float* sums;           // statistics: [tiles_n][M] sums of the logits, or null (no smoothing)
    float* picked;         // statistics: [M] the labels' logits
    const float* lse;      // probabilities: [M]
    VocabSide side;        // probabilities
    float* rest;           // probabilities: [M] what rounding the label's element has left
    void* G;               // probabilities: [M, ldg] bf16, columns from N up to a multiple of 8 are zeros
    long long ldg;
    float* planes;         // planes: [splits][M][N]
    int splits, k_split;   // planes: of the contraction, and its length of each (a multiple of 64)
    int add;               // planes: to what they hold
    const float* scale;    // the weight's gradient: a factor for all of it, times scale_by, or null
    float scale_by;
    long long n_labels;    // the weight's gradient with such a factor: rows, whose labels say whether any counts
};
enum { VOCAB_STATS, VOCAB_PROBS, VOCAB_PLANES, VOCAB_WEIGHT };
int prepare_vocab_tiles();
int launch_vocab_tiles(VocabTileParams p, int what, GgTile tile, hipStream_t st);
// tiles of a launch of one kind along the columns
int vocab_tile_cols(GgTile tile);

struct VocabLossParams {
    const void *X, *W;
    const int *idx, *labels;
    long long S, ldx, ldw, M;
    int C;
    VocabRule rule;
    float *loss, *lse, *total;  // total: or null
    void* workspace;
};
struct VocabGradParams {
    const void *X, *W;
    const int *idx, *labels;
    long long S, ldx, ldw, M;
    int C;
    VocabRule rule;
    const float *lse, *dloss;
    long long dloss_stride;
    void *dX, *dW;  // or null
    long long lddx, lddw;
    int piece;
    void* workspace;
};
int prepare_vocab_loss(lemo_dtype_t dt);
int prepare_vocab_grad(lemo_dtype_t dt);
size_t vocab_loss_workspace(long long M, int C, int V, lemo_dtype_t dt);
int launch_vocab_loss(const VocabLossParams& p, lemo_dtype_t dt, hipStream_t st);
// columns of a piece for a wanted number of them (0: this library's choice); 0: no piece fits the operands' 32-bit offsets
int vocab_piece(long long M, int C, int V, long long ldw, int wanted, lemo_dtype_t dt);
size_t vocab_grad_workspace(long long M, int C, int V, int piece, lemo_dtype_t dt);
int launch_vocab_grad(const VocabGradParams& p, lemo_dtype_t dt, hipStream_t st);

}  // namespace lemo

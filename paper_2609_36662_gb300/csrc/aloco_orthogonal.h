// Internal interface of the orthogonalised updates: what aloco_muon.cpp plans
// and what the kernels of aloco_orthogonal.cu take by value.
#pragma once

#include <cuda.h>
#include <cuda_fp16.h>

#include "aloco_internal.h"

namespace aloco {

// Matrices of one shape in a pass.  X is the matrix with its smaller side as
// rows (m <= n), as a sum of two fp16 values: the larger ones row by row, whose
// products are taken, and what they leave, which only what multiplies X itself
// sees, in blocks of 32 x 32 laid out as the epilogue's threads hold them.  The
// symmetric m x m matrices (A = X X^T, polynomials of it) are fp16 values with their
// diagonals beside them in fp32.  Rows lie ldx and lda elements apart (multiples
// of 8).
constexpr int kOrthoSyms = 4;        // places for symmetric matrices

// What a matrix's next operation is.
enum { kGram, kPoly, kProduct, kUpdate };
struct OrthoOp {
    // kGram     out = X X^T
    // kPoly     out = a + b L + c L L
    // kProduct  out = L R
    // kUpdate   X <- L X
    int8_t what;
    int8_t left, right, out;         // places of symmetric matrices
    int8_t step;                     // whose coefficients are taken
    int8_t x;                        // which of x[2] X is
    // kGram, kPoly: L is (to be) kept as L + b / 2c, as whose square the polynomial
    // comes out but for its diagonal
    int8_t shifted;
    int8_t bare;                     // out's diagonal lies beside it only (for kUpdate)
    int8_t last;                     // kUpdate: writes the result
    int8_t syms, ups;                // operations of either kind ahead of it
};
// Lists of operations: one step after another, or two at a time.
enum { kPlain, kMerged, kOrthoLists };
constexpr int kOrthoOps = 64;

struct OrthoGroup {
    int m, n, ldx, lda;
    int rows, cols;                  // as the caller has it
    int tall;                        // rows > cols: X is its transpose
    int count;                       // matrices of this pass
    int first, period, skip;         // the i-th: number first + (skip + i) % period
                                     // of worker (skip + i) / period
    int sym_tiles, up_tiles;         // tiles of a matrix: symmetric products, update
    int split[2];                    // parts of the depth of tiles of X X^T, and of the
                                     // other symmetric products'
    int chunks, chunk;               // norm blocks of a matrix, elements of each
    int norm0, prep0;                // the group's first block
    int small0;                      // its first cluster (launch_ortho_small)
    __half *x[2], *sym[kOrthoSyms];
    float *diag[kOrthoSyms];
    int list;                        // of operations: kPlain or kMerged
    uint4 *rest;                     // X - x, kBlockPieces a block: 8 columns of a row each
    int blocks_down, blocks_across;  // of a matrix
    double *partial;                 // [count][chunks] sums of squares
    int *done;                       // [count] blocks of 32 x 32 that are finished
    // where tiles have parts: their sums, a block as a warp holds it after the other,
    // and how many parts have left theirs for either half of a warp's blocks
    float4 *sums;                    // [count][sym_tiles][parts]
    int *came;                       // [count][sym_tiles][warps][2]
};

// What fits a CTA of launch_ortho_small: rows of X, and columns of it.
constexpr int kOrthoSmallSide = 128, kOrthoSmallCols = 256, kOrthoSmallCtas = 16;

constexpr int kOrthoCounters = 2;    // of a pass, ahead of its matrices' (OrthoArgs::next_tile)
constexpr int kOrthoGroups = 16;     // groups of a pass
constexpr int kOrthoMatrices = 1024; // places of a pass (a worker's)

constexpr int kBlockPieces = 32 * 32 / 8, kBlockQuads = 32 * 32 / 4;

// X is held times 2^8, so that fp16 keeps its values of any realistic size in
// its normal range (its largest value is at most about 1.2).
constexpr float kOrthoScale = 256.f;

enum OrthoSource { kSourceMatrix, kSourceMuon };

// Operands of the products: X, which alternates between two places, and the
// symmetric matrices.
enum { kMapX0, kMapX1, kMapSym, kOrthoMaps = kMapSym + kOrthoSyms };

struct OrthoArgs {
    CUtensorMap map[kOrthoMaps][kOrthoGroups];
    OrthoGroup g[kOrthoGroups];
    int64_t place[kOrthoMatrices];   // offset in a replica; kSourceMatrix: index in the batch
    int n_groups;
    OrthoOp ops[kOrthoLists][kOrthoOps];
    int n_ops[kOrthoLists];
    int tiles, norm_blocks, prep_blocks;   // all groups'
    float coef[ALOCO_MAX_NS_STEPS][3];     // the steps' coefficients
    int steps;
    int small_ctas;                  // launch_ortho_small: the CTAs of a matrix
    int *next_tile;                  // the next tile to take, how many pairs have given
    int counters;                    // up, `done` and `came`: zero when the products
                                     // begin, so many
    double eps;
    // where the matrices come from and go to
    int source;
    int in_bf16, out_bf16;
    int64_t batch_stride, row_stride;      // kSourceMatrix
    const void *in[ALOCO_MAX_WORKERS];     // gradients (kSourceMatrix: one)
    float *momentum[ALOCO_MAX_WORKERS];
    void *out[ALOCO_MAX_WORKERS];          // parameters (kSourceMatrix: one, bf16)
    float mu;
    int nesterov;
    float decay;                     // 1 - lr weight_decay
    float step[kOrthoGroups];        // -lr * scale of the group's shape
    int64_t test_stall1;             // testing only: 1 + the slot whose copies a
                                     // first block leaves out
};

int ortho_pair_tile();               // rows of a tile by two CTAs; half by one
int ortho_slot_depth();              // k-elements of a slot
int ortho_epilogue_warps();          // of a CTA
cudaError_t launch_ortho_norm(const OrthoArgs &a, cudaStream_t stream);
cudaError_t launch_ortho_prepare(const OrthoArgs &a, cudaStream_t stream);
// All steps' products; ctas: 1 or 2 CTAs share a tile (of 128 or 256 rows and
// columns).
cudaError_t launch_ortho_chain(const OrthoArgs &a, int ctas, int sm_count, cudaStream_t stream);
// All steps of matrices with m <= kOrthoSmallSide and n <= kOrthoSmallCols *
// a.small_ctas (1, 2, 4, 8 or 16, if the device has room for such a cluster).
cudaError_t ortho_small_setup(int ctas, bool *fits);
cudaError_t launch_ortho_small(const OrthoArgs &a, int matrices, cudaStream_t stream);

}  // namespace aloco

// Internal interface between the host side of the layer operators and their
// HIP kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "arena_layer.h"

namespace arena {

// Defined beside arena_ctx: the context's device, and its error text.
int ctx_device(const arena_ctx* c);
void ctx_clear(arena_ctx* c);
arena_status ctx_fail(arena_ctx* c, arena_status s, const char* fmt, ...) __attribute__((format(printf, 3, 4)));

namespace mm {

constexpr int kBK = 64;                 // k per step
constexpr int kMaxLd = 1 << 22;         // row stride limit, elements: 256 rows stay within 32-bit byte offsets

enum Epi { kPlain = 0, kGatedFwd = 1, kGatedBwd = 2, kPlainRest = 3, kWide = 4, kLossStats = 5, kLossGrad = 6 };
enum Out { kOut16 = 0, kOutF32 = 1, kOutBf16 = 2 };   // the operands' own type, float, bf16
enum Act { kSilu = 0, kGelu = 1, kRelu = 2, kGeluShort = 3 };
// Products whose rows or steps come in groups (experts) of lengths that only the
// device knows: rows offsets[g] .. offsets[g + 1] - 1 of A and C meet matrix g of B, or
// those steps of k of both operands make matrix g of C.
enum Group { kOneGroup = 0, kRowGroups = 1, kStepGroups = 2 };

// A token as the products of a loss's gradient read it.  target < 0: left out of the loss.
struct LossRow {
    float lse, factor;        // log sum exp of its logits; its gradient's factor
    int32_t target, unused;
};

struct GemmArgs {
    // segments of k (nseg = 2: the second operand pair follows the first), or
    // with pairs = 1 the operands of batch index 0 and 1, or the gate and up
    // matrices of the gated forward product (b)
    const void* a[2];
    const void* b[2];
    void* c[2];
    int64_t lda, ldb, ldc;    // elements
    int64_t ldb1;             // few tokens: of b[1]
    int64_t sa, sb, sc;       // batch strides, elements
    int32_t M, N, K;
    int32_t nseg, pairs, batch;
    // tiles of the product (sym: only those on and below the diagonal) and which
    // of them, over all batch indices, this launch takes: from `first` on, each
    // as 2^ratio x 2^ratio tiles of the kernel's size
    int32_t tiles_m, tiles_n, sym;
    int32_t first, ratio;
    // plain: C = alpha * product + beta * e - diag on the diagonal
    const void* e[2];
    int64_t lde, se;
    float alpha, beta, diag;
    int32_t out;
    // plain with a rest: what rounding took off e, times 2^11, laid out as e and C;
    // `rest_in` times it is added, and with rest_out C's own takes its place.  C is of
    // the operands' type, N a multiple of 8 and pad = N
    void* rest;
    float rest_in;
    int32_t rest_out;
    // gated, forward: c[0] = act(g) u, and g, u unless null; backward: c[0] and
    // c[1] the gradients of g and u.  Rows of ldc elements (c) and ldg values of
    // 24 bits (g, u: M rows of 16-bit heads, then M rows of 8-bit tails);
    // columns N .. pad - 1 are written as zeros
    void *g, *u;
    int64_t ldg;
    int32_t act, pad;
    // split k: block y of `splits` takes `per` steps and leaves its sums in part,
    // a place of tile size for each block
    int32_t splits, per;
    float* part;
};

// The products of groups and of a loss.  A struct of its own: what a kernel is handed is on
// the path of a short product, and the dense ones take up to 4 % longer with these fields
// among theirs (512 x 512 on 64 x 64 tiles 7.6 us, without 7.3).
struct GroupArgs : GemmArgs {
    int64_t sb1;              // matrices of b[1] lie so many values apart
    // groups: of rows, matrix g of b lies sb values on; of steps, matrix g of c (and e) sc
    // (se).  With pairs = 1 every group's two products are neighbouring batch indices
    const int32_t* offsets;   // [groups + 1], held inside 0 .. rows
    int32_t groups;
    int32_t tail;             // most parts of k for the tiles past the last whole round, in part too; 0: whole
    int32_t any;              // an operand's rows start on any value (tiles of 128 columns)
    // wide: C = alpha factor[0] product + beta e, e in 32 bits or in C's type
    const float* factor;      // nullable
    int32_t e_f32;
    // loss: columns are entries first_col + n of the vocabulary.  Statistics: of each tile
    // column and row the largest logit and the sum of exponentials beside it, at pair
    // stats[column * M + row], and the logit of target[row]; gradient: c[0], and what rounding took
    // off it `low` rows further on, unless 0 (64 x 128 tiles)
    const LossRow* rows;
    const void* target;
    float* stats;
    float* picked;            // [M]
    int32_t first_col, target_wide, low;
};

// Products by the layouts of their operands (rows: k contiguous; cols: m or n
// contiguous) and epilogue; those with a rest in float16 only.
enum Product { kRowsRows = 0, kRowsCols, kColsCols, kGateUp, kGateUpBack, kRowsRowsRest, kRowsColsRest,
               kLossLogits, kLossGradient };

// Tiles: 256 x 256 (8 waves, two buffers, one block on a compute unit), 128 x 128
// (4 waves) with two buffers (two blocks) or four (one block), 64 x 64 (4 waves,
// four buffers, two blocks).
enum TileKind { k256 = 0, k128, k128Deep, k64, kTileKinds };
constexpr int kTileSide[kTileKinds] = {256, 128, 128, 64};

// How a product is cut: tiles of kind `main`, the first `first` of them by
// themselves, in whole rounds over the compute units; the rest as tiles of kind
// `tail`, whose side divides main's, with k in `splits` parts of `per` steps.
struct Cut {
    int main, tail;
    int64_t first;
    int splits, per;
};

// part: `splits` times the tail's tiles, each of its side squared, if k is
// split.  The host has checked that operands are 16-byte aligned
// with strides and batch strides of multiples of 8, and that values between
// the matrix's edge and the next multiple of 8 along the contiguous axis are
// readable (and zero where that axis is k).
hipError_t launch_gemm(const GemmArgs& A, int dtype, Product what, const Cut& cut, hipStream_t s);

// Two independent products in one launch, both on 128 x 128 tiles: A of layout
// rows x cols (what: kGateUpBack or kRowsCols) with k in cut.splits parts, B of
// layout cols x cols.
hipError_t launch_pair(const GemmArgs& A, int dtype, Product what, const GemmArgs& B, const Cut& cut, hipStream_t s);

// Most tiles of `side` rows that `groups` groups of M rows in all make.
constexpr int64_t group_tiles(int64_t M, int64_t groups, int64_t side)
{
    return M / side + (groups < M ? groups : M);
}

// Tiles of the products of groups: 256 x 256 (8 waves, two buffers, one block on a compute
// unit), 128 x 128 (4 waves, two buffers, two blocks) and 64 x 128 (4 waves, three buffers,
// two blocks).
enum GroupKind { kGroup256 = 0, kGroup128, kGroup64x128, kGroupKinds };
constexpr int kGroupRows[kGroupKinds] = {256, 128, 64}, kGroupCols[kGroupKinds] = {256, 128, 128};

// The products of experts: C of groups of rows (gate and up, down, and the gradients of
// both operands' inner sides), C of groups of steps (the weights' gradients, wide: beta e
// and the type of C).  kind: of GroupKind; A.splits parts of k, joined in a launch of their own
// (not of gate and up, nor of groups of rows on the largest tiles).
hipError_t launch_groups(const GroupArgs& A, int dtype, Product what, int kind, hipStream_t s);

// Few rows, of groups or (offsets null) of one: C = A B^T without LDS tiles, plain, gated or
// the statistics of a loss (columns of 16: kSkinnyCols).  Operands of any alignment.
constexpr int kSkinnyCols = 16;
hipError_t launch_skinny_groups(const GroupArgs& A, int dtype, Product what, hipStream_t s);

// The products of a loss, on the same tiles: the logits' statistics, their gradient (what:
// kLossLogits, kLossGradient), and the gradients of both operands (wide; k in A.splits parts).
hipError_t launch_loss(const GroupArgs& A, int dtype, Product what, int kind, hipStream_t s);

constexpr int kSkinnyRows = 32;         // rows of A (tokens) that the kernel without LDS tiles takes

// C = A B^T with both operands' k contiguous, M <= kSkinnyRows; dual: the gated
// forward product.
hipError_t launch_skinny(const GemmArgs& A, int dtype, bool dual, hipStream_t s);

// Copies of matrices of 16-bit values, rows x cols, with zeros in columns cols ..
// ld_to - 1; one launch.
struct Pack {
    const void* from;
    void* to;
    int64_t ld_from, ld_to, rows, cols;
};
constexpr int kMaxPacks = 5;
hipError_t launch_packs(const Pack* packs, int n, hipStream_t s);

}  // namespace mm

// Loss: the passes beside the products.
struct LossArgs {
    int64_t tokens;
    int32_t vocabulary, model;
    const void* target;           // int64 or int32
    int32_t target_wide;
    int64_t ignore;
    // forward: the tiles' statistics, `columns` of them a token
    const float *stats, *picked;
    int32_t columns;
    float *loss, *lse;
    // backward
    const float* dloss;
    int64_t s_dloss;              // elements between tokens' gradients, 0 for one of all
    const float* lse_in;
    mm::LossRow* rows;
    float* scale;                 // [2] or null: a power of two for the factors, and its inverse
    const void* x;                // copied with zeros in rows that the loss leaves out
    int64_t ld_x;
    void* x_to;
    int64_t ld_to;
    int32_t twice;                // x_to has that copy twice
};

hipError_t launch_loss_join(const LossArgs& A, hipStream_t s);
hipError_t launch_loss_rows(const LossArgs& A, hipStream_t s);
// dx of dtype, rows of ld: the sum of `sum`'s first and second `tokens` rows.
hipError_t launch_loss_fold(const float* sum, void* dx, int64_t ld, int64_t tokens, int model, int dtype, hipStream_t s);

// Router and tokens to experts.
constexpr int kRouteMaxExperts = 1024;
constexpr int kRouteMaxChoices = 16;

struct RouteArgs {
    int64_t tokens;
    int32_t experts, k, normalise;
    float scale;
    const void* logits;
    int64_t ld_logits;
    void* index;                  // int32 [tokens][k]
    float* weight;                // [tokens][k]
    const float* dweight;
    int64_t ld_dweight;
    void* dlogits;
    int64_t ld_dlogits;
};

hipError_t launch_route_forward(const RouteArgs& A, int dtype, hipStream_t s);
hipError_t launch_route_backward(const RouteArgs& A, int dtype, hipStream_t s);

struct SortArgs {
    int64_t choices;
    int32_t experts, wide;        // wide: int64 indices
    const void* index;
    int32_t *offsets, *row;
    int32_t* counts;              // [blocks][experts], of more than one block
    int32_t blocks, each;         // choices of a block
};

constexpr int kSortThreads = 1024;
void sort_plan(int64_t choices, int* blocks, int* each);
hipError_t launch_sort(const SortArgs& A, hipStream_t s);

// One row of x (dispatch), y, dy or dx a token; one of xs, ys, dys or dxs a choice.
struct MoveArgs {
    int64_t tokens, rows;         // rows: of xs and ys, all that `row` may name
    int32_t model, k;
    const int32_t* row;           // [tokens][k]
    const float* weight;          // nullable
    int64_t ld_weight;
    const void *token, *choice;   // read: rows of tokens, rows of choices
    int64_t ld_token, ld_choice;
    void *to_token, *to_choice;
    int64_t ld_to_token, ld_to_choice;
    float* dweight;
};

hipError_t launch_dispatch(const MoveArgs& A, int dtype, hipStream_t s);
hipError_t launch_combine(const MoveArgs& A, int dtype, hipStream_t s);
hipError_t launch_combine_backward(const MoveArgs& A, int dtype, hipStream_t s);

// Norms around a block.
struct NormArgs {
    const void *x, *y, *gate, *w_post, *b_post, *w_pre, *b_pre;
    int64_t ld_x, ld_y, ld_gate, ld_r, ld_n;
    void *r, *n;
    float* stats;                 // [tokens][4]: mean and 1/deviation of the block's output, then of the stream
    int64_t first_token, tokens;  // rows first_token .. tokens - 1 (the backward: from 0)
    int64_t gate_rows;            // tokens of one gate row (all of them: tokens, at least 1)
    int32_t width, layer;         // layer: subtract the mean
    float eps, scale;
    // backward
    const void *dn, *dr, *res;    // gradients of n and r; res: r (x where there is no block output)
    int64_t ld_dn, ld_dr, ld_res, ld_dx, ld_dy;
    void *dx, *dy;
    void *dgate, *dw_post, *db_post, *dw_pre, *db_pre;
    float* part;                  // workers' column sums, see norm_plan
    float* means;                 // [tokens][2], rows wider than kNormSumsWidth
    int32_t workers, rows_each;   // workers of the backward, tokens of each
};

// Column sums that a worker keeps: of dw_pre, db_pre, dw_post, db_post and its
// first and last gate row's dgate.
constexpr int kNormSums = 6;
constexpr int kNormMaxWidth = 16384;
constexpr int kNormSumsWidth = 8192;       // wider rows' column sums take a pass of their own

void norm_plan(int64_t tokens, int64_t gate_rows, int width, int* workers, int* rows_each);
hipError_t launch_norm_forward(const NormArgs& A, int dtype, int stream_dtype, hipStream_t s);
hipError_t launch_norm_backward(const NormArgs& A, int dtype, int stream_dtype, hipStream_t s);

// Orthogonalised update: the passes over the gradient.
struct UpdateArgs {
    const void* grad;             // [batch][rows][cols]
    const float* momentum;        // nullable
    float* momentum_out;
    int64_t ld_grad, ld_mom, ld_mom_out, s_grad, s_mom, s_mom_out;
    int32_t rows, cols, batch, nesterov;
    float mu, eps;
    void* x;                      // float16 [batch][rows_p][ld_x], zero past rows and cols
    void* rest;                   // nullable: 2^11 times what rounding took off x, laid out as x
    int32_t rows_p, ld_x;
    double* part;                 // [batch][blocks] sums of squares
    int32_t blocks;
};

constexpr int kUpdateBlocks = 256;      // most blocks that share a matrix's sum of squares

hipError_t launch_update_sum(const UpdateArgs& A, int dtype, hipStream_t s);
hipError_t launch_update_scale(const UpdateArgs& A, int dtype, hipStream_t s);

}  // namespace arena

// Losses of the output layer (wind_loss.cu): sizes, workspace layout and the launcher that the entry points call.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "wind.h"

namespace wind {

constexpr int kLossMaxK = 256;            // teacher's entries of a row
constexpr long long kLossMaxLogits = 1ll << 40;   // N n_out
constexpr int kLossMaxRows = 1 << 24;
constexpr int kLossMaxOut = (1 << 24) - 1;
constexpr int kLossMaxH = 1 << 16;
constexpr size_t kLossPieceBytes = (size_t)512 << 20;   // the gradient's share of logits that is kept at a time (see loss_layout)

// Control words, first thing in the workspace.
struct LossCtrl {
    int32_t status;   // of the last call: WIND_OK or WIND_ERR_INVALID_ARG
    int32_t n_rows;   // rows with a loss
    // kLossTimedOut: a wait ran out, in this call or in an earlier one.  Only wind_loss_status takes it back: a gradient that reads what a
    // timed-out loss wrote is as wrong as that.  (64 bits: a workspace nobody has written yet should not say so by chance.)
    unsigned long long timed_out;
};
constexpr unsigned long long kLossTimedOut = 0x9c0e5d2b71f6a843ull;

// How a call is cut up, and the byte offsets of its workspace regions.  Host arithmetic on the sizes alone.
struct LossLayout {
    int planes;        // bf16 parts of an operand: 1 (bf16) or 3 (fp32)
    int kind;          // LossKind
    int g_planes;      // bf16 parts of the gradient's share of logits: 1, 2 (bf16, few rows) or 3 (fp32)
    int pack_w;        // W is laid out again: fp32, or rows that TMA cannot start on
    int where_ld;      // bytes of a row's index into its list of the teacher's entries
    int Hp, Npad;      // H up to a multiple of 64, N up to a multiple of 128
    int piece;         // outputs of a piece (gradient), a multiple of 256
    int pieces;
    int tn, parts;     // columns of a tile of logits; partial results of a row (loss)
    int tn_products;   // columns of a tile of dx and dW
    int pair, pair_products;   // whether two CTAs make a tile, of logits and of dx and dW
    int s_dx, s_dw;    // parts that the sums of dx (over a piece's outputs) and dW (over the rows) are cut into
    int slab_dx, slab_dw;   // whether dx / dW go through fp32 partial sums
    size_t ctrl, next, counts, mark, src, target, scale, nlse, list, where, ent, x, w, pm, ps, pq, g, dbp, sdx, sdw, total;
};

struct LossCall {
    wind_output_t o;
    const void* x; int64_t ldx; int N;
    const int32_t* target;                              // labels, or null:
    const int32_t* ids; const float* y; int K; float tau;   // the teacher's entries
    float* loss; float* lse_out;                        // forward
    const float* lse; const float* dloss;               // gradient
    void* dx; int64_t lddx; void* dw; int64_t lddw; float* db;
    int grad;
    uint8_t* ws;
    LossLayout lay;
    cudaStream_t stream;
};

// most_of_fewer: `total` is the most that a call of up to N rows needs (the offsets are not to be used).
LossLayout loss_layout(const wind_output_t& o, int N, int K, int grad, bool most_of_fewer = false);
cudaError_t loss_run(const LossCall& c);
int loss_set_stall(int which);   // test hook (wind_debug_stall_loss); the previous value

}  // namespace wind

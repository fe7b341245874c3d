// The dense layer with bias, activation, dropout and residual (dense_tile.hip, dense_few.hip, dense_grad.hip): what dense_api.hip calls.
#pragma once

#include "dropout.h"

namespace abt {

// Y = residual + drop(act(Z)), Z = alpha X W^T + bias
struct DenseProduct {
    const uint16_t* X; const uint16_t* W;  // [M, K], [Q, K]; K a multiple of 8
    uint16_t* Y;                           // [M, Q]; Q a multiple of 8
    const float* bias;                     // [Q], NULL: none
    const uint16_t* residual;              // [M, Q], NULL: none
    uint16_t* Z;                           // [M, Q], NULL: not kept
    int64_t M;
    int Q, K, act;
    float alpha;
    Drop drop;
    float* parts;                          // dense_part_bytes(M, Q, K)
    int piece;                             // set by the launchers: slabs of 64 columns of a piece of the contraction
};
size_t dense_part_bytes(int64_t M, int Q, int K);
hipError_t launch_dense(const DenseProduct& p, hipStream_t s);
// What it costs, us, without an epilogue, and with tiles of 64 x 64: the longest of them, and what they keep the chip busy
float dense_cost(int64_t M, int Q, int K);
struct SmallCost { float longest, load; };
SmallCost dense_small_cost(int64_t M, int Q, int K);
hipError_t launch_dense_few(const DenseProduct& p, hipStream_t s);        // M <= 64

// What the gradients are made of: dZ = slope(Z) drop(dY) [M, m] as the sum of one or three bf16 values.  Without an activation or with ABT_ACT_RELU one is
// exact (dropout's factor is left to the products).  Otherwise it takes three to have all of fp32.
// Beside it W^T, and sums of dZ over pieces of the rows.
struct DenseSlope {
    const uint16_t* dY; const uint16_t* Z; // Z NULL without an activation
    uint16_t* value[3];                    // NULL: dY itself is dZ; not kept
    float* sums;                           // [pieces, m] of dZ, without the factor where that is left out; NULL: not wanted
    const uint16_t* W; uint16_t* Wt;       // [m, n] -> [n, m]; NULL: not wanted
    int64_t M;
    int m, n, act, rows;                   // rows of a piece
    int scaled;                            // with dropout's factor
    Drop drop;
};
int dense_piece_rows(int64_t M, int m);
hipError_t launch_dense_slope(const DenseSlope& p, hipStream_t s);

// dW [m, n] (+)= alpha (sum of the values)^T X, and dbias [m] (+)= alpha times the sum of `sums`; either may be NULL
struct DenseGrads {
    const uint16_t* value[3]; const uint16_t* X;
    float* dW; float* partials;
    const float* sums; float* dbias;
    int64_t M;
    int m, n, pieces, accumulate;
    int values;                            // of dZ where dW is wanted: how the launches are made does not go by what is wanted
    float alpha;
};
size_t dense_grad_partial_bytes(int64_t M, int m, int n);
// dX (x.Y NULL: not wanted), dW and dbias in one launch, or each in its own
hipError_t launch_dense_bwd(const DenseProduct& x, const DenseGrads& g, hipStream_t s);

}  // namespace abt

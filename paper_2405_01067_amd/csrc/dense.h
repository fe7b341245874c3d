// The dense layer with bias, activation, dropout and residual (dense_tile.hip, dense_few.hip, dense_grad.hip): what dense_api.hip calls.
#pragma once

#include "dense_way.h"
#include "dropout.h"

namespace abt {

// Y = residual + drop(act(Z)), Z = alpha X W^T + bias
struct DenseProduct {
    const uint16_t* X; const uint16_t* W;  // [M, K], [Q, K]; K a multiple of 8, up to 2^21
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
hipError_t launch_dense(const DenseProduct& p, hipStream_t s);
hipError_t launch_dense_few(const DenseProduct& p, hipStream_t s);        // M <= 64

// What the gradients are made of: dZ = slope(Z) drop(dY) [M, m] as the sum of bf16 values.  Without an activation or with ABT_ACT_RELU one is exact (dropout's factor is
// left to the products).  Otherwise a value is cut into three parts of eight bits, which together have all of fp32, for dW, which is fp32.  dX, which is rounded to bf16, takes two: what they
// leave out is 2^-15 of dZ at most (and 2^-16.5 on average, towards 0), 1 / 128 of dX's own rounding.  With one, the rounding of dZ counted as much as dX's own: 2.34e-3 of dX off in all instead of 1.66e-3.
// The two lie beside each other, [M, 2 m], and W^T twice, [n, 2 m], so that dX is one product with a contraction of 2 m.
// All parts have dZ's sign, and none is 0 where dZ is not: it is 2^-133 then, the smallest there is, which an infinite X or W makes the infinity that it makes of dZ.
// Beside it W^T, and sums of dZ over pieces of the rows.
struct DenseSlope {
    const uint16_t* dY; const uint16_t* Z; // Z NULL without an activation
    uint16_t* value[3];                    // NULL: dY itself is dZ; not kept.  Rows of the first and second lie pitch_of(values) m values apart
    int values;                            // one or three
    float* sums;                           // [pieces, m] of dZ, without the factor where that is left out; NULL: not wanted
    const uint16_t* W; uint16_t* Wt;       // [m, n] -> [n, m], or twice beside each other; NULL: not wanted
    int64_t M;
    int m, n, act, rows;                   // rows of a piece
    int scaled;                            // with dropout's factor
    Drop drop;
};
// of the first two parts of dZ, and of W^T, in m values
constexpr int pitch_of(int values) { return values == 1 ? 1 : 2; }
int dense_piece_rows(int64_t M, int m);
hipError_t launch_dense_slope(const DenseSlope& p, hipStream_t s);

// dW [m, n] (+)= alpha (sum of the values)^T X, and dbias [m] (+)= alpha times the sum of `sums`; either may be NULL
struct DenseGrads {
    const uint16_t* value[3]; const uint16_t* X;
    float* dW; float* partials;
    const float* sums; float* dbias;
    int64_t M;
    int m, n, pieces, accumulate;
    int values;                            // that make dZ; how the launches are made does not go by what is wanted
    float alpha;
};
size_t dense_grad_partial_bytes(int64_t M, int m, int n);
// dX (x.Y NULL: not wanted), dW and dbias in one launch, or each in its own
hipError_t launch_dense_bwd(const DenseProduct& x, const DenseGrads& g, hipStream_t s);

}  // namespace abt

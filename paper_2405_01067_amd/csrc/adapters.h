// A frozen dense layer with low-rank adapters, row by row another one (adapters.hip, adapters_few.hip, adapters_grad.hip): what
// adapters_api.hip calls.
#pragma once

#include "common.h"

namespace abt {

// Out_i = Main_i . W^T + E_i . F_a^T for the rows i of adapter a = row_adapter[i]; an id outside [0, count) is no adapter.  Main or E may be absent.
struct AdapterProduct {
    const void* X; const void* W;          // [M, kmain], [Q, kmain], bf16 or 8-bit floats; X NULL: no main product
    const float* x_scale; const float* w_scale;      // 8 bits: per row of X and of W
    const uint16_t* E; const uint16_t* F;  // [M, e_pitch] of which ke columns count, [count, Q, ke]
    const int32_t* row_adapter; const int32_t* ranks; const float* scales;   // ranks, scales may be NULL: r, 1
    int64_t M;
    int Q, kmain, ke, e_pitch, count, r;
    // what is made of it:
    uint16_t* Y;                           // [M, Q] rounded (E holds T, rank columns of ke)
    float* T;                              // or, Q = r: T [M, r] fp32 (columns from the rank on zero), may be NULL
    uint16_t* Tb;                          // and scale times it, rounded, [M, r], may be NULL
    const float* T_in;                     // or, Q = r: planes of scale times the result, and of scale times T_in [M, r]: three bf16 values whose sum is the
    uint16_t* dT_planes; uint16_t* T_planes;   // fp32 value, [M, 3, rp], rp = plane_columns(r)
};
// r padded to what the factor gradients work in: a power of two of blocks of 16
inline __host__ __device__ int plane_columns(int r) { return r <= 16 ? 16 : r <= 32 ? 32 : r <= 64 ? 64 : 128; }

hipError_t launch_adapters_y(const AdapterProduct& p, bool fp8, hipStream_t s);
hipError_t launch_adapters_t(const AdapterProduct& p, hipStream_t s);         // X absent, Q = r <= 128
// T row by row: up to 1024 rows and this many values of T.  us, the forward by rows / by tiles of 32 rows, in runs of 100 and any order: 768 x 768, r = 16, 394 rows
// 12.5 / 13.7, 13.4 / 15.3; 2304 x 768, r = 64, 256 rows 16.1 / 16.9, 22.3 / 36.7, 394 rows 18.6 / 17.3, 24.6 / 36.9, 1024 rows 39.1 / 28.6, 51.5 / 48.9; 4096 x 4096,
// r = 128, 256 rows 44.8 / 47.7, 512 rows 64.8 / 53.0.
constexpr int64_t kAdapterRowsOfT = 24576;
hipError_t launch_adapters_t_rows(const AdapterProduct& p, hipStream_t s);

// Few rows: T (p.T, p.Tb, either may be NULL but for Tb = p.E) from X [M, n] and B, and Y, together.  sums: adapters_few_sums_bytes.
// The limit is where rows that lie together by adapter no longer gain (rows in any order gain longer, but the host does not see the order).  us, these kernels / T row by
// row and tiles, in runs of 100, 128 and 192 rows: 768 x 768, r = 16 10.9 / 10.7, 11.2 / 11.4; 2304 x 768, r = 64 13.9 / 13.9, 16.6 / 14.7; 4096 x 4096, r = 16
// 26.2 / 29.9, 43.3 / 30.3, in 8 bits 20.1 / 18.2, 29.2 / 19.4; in any order, 128 rows: 4096 x 4096, r = 64 36.5 / 51.5.
constexpr int kAdapterFewRows = 128;
size_t adapters_few_sums_bytes(int64_t M, int m, int n);
hipError_t launch_adapters_few(const AdapterProduct& p, const uint16_t* X, const uint16_t* B, float* sums, bool fp8, hipStream_t s);

// What the backward prepares beside dT: W^T, the transposes of every adapter's B, the rows of each adapter one after the other in
// `order` (rows ascending) with offsets[count + 1].
struct AdapterPrep {
    const uint16_t* W; uint16_t* Wt;       // [m, n] -> [n, m]; NULL: not wanted
    const uint16_t* B; uint16_t* Bt;       // [count, r, n] -> [count, n, r]; NULL: not wanted
    const int32_t* row_adapter; int32_t* order; int32_t* offsets;     // order NULL: not wanted
    int64_t M;
    int m, n, r, count;
};
// E = dY [M, m], F = A [count, m, r], ke = m, and the planes
hipError_t launch_adapters_dt(const AdapterProduct& p, const AdapterPrep& prep, hipStream_t s);

// dA[a] = sum of U_i V_i^T over the rows of adapter a, both sides in one launch, then their sums.
struct AdapterGrads {
    const uint16_t* dY; const uint16_t* T_planes; float* dA;      // dA [count, m, r], NULL: not wanted
    const uint16_t* X; const uint16_t* dT_planes; float* dB;      // dB [count, r, n]
    const int32_t* order; const int32_t* offsets;
    float* partials;
    int64_t M;
    int m, n, r, count, accumulate;
};
int adapters_grad_piece(int64_t M, int m, int n);      // rows of a piece
size_t adapters_grad_partial_bytes(int64_t M, int m, int n, int r, int count);
// With x, dX beside them in the same launch
hipError_t launch_adapters_grads(const AdapterGrads& p, const AdapterProduct* x, hipStream_t s);
// Few rows: no partials, and dX (or NULL) in the same launch.  At most what a work-group's list of rows holds; up to there it is faster, us, this / pieces: 768 x 768, r = 8
// 17.8 / 25.8 (394 rows), 20.0 / 27.3 (1024); 2304 x 768, r = 16 33.8 / 44.1, 34.9 / 44.5; 1024 x 1024, r = 64 27.1 / 39.8, 45.0 / 49.8.
constexpr int kAdapterFewGradRows = 1024;
hipError_t launch_adapters_few_dx_grads(const AdapterProduct* x, const AdapterGrads& p, hipStream_t s);
// Many rows and a narrow rank: is dX faster beside the gradients than before them?  And that launch.
bool adapters_dx_beside_grads(const AdapterProduct& x, const AdapterGrads& p);
hipError_t launch_adapters_dx_grad_pieces(const AdapterProduct& x, const AdapterGrads& p, int piece, hipStream_t s);

}  // namespace abt

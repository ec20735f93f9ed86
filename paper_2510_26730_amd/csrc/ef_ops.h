// Launch interface between the context-free operators' entry points (ef_ops.hip) and their kernels
// (ef_router.hip, ef_q8.hip, ef_q8_panel.hip, ef_q8_tiled.hip).
#pragma once
#include "../../include/expertflow.h"

#include <hip/hip_runtime.h>
#include <cstdint>

namespace ef {

// ---- routing from logits (ef_router.hip) -------------------------------------------------------
constexpr int kRouterSumTiles = 1024;   // tiles whose counts every workgroup of the scatter adds up by itself

struct RouterArgs {
    ef_router r;
    const void *logits;
    int type;
    long long ld;
    const float *bias;
    int T;
    int32_t *ids;
    float *w;
    int32_t *counts, *offsets, *perm, *inv_perm;   // inv_perm holds, between the launches, an assignment's rank in its tile
    int ntiles;            // token tiles of router_tile(r, T) tokens
    uint8_t *tile_counts;  // [ntiles][pitch] (scratch): assignments of a tile to an expert
    int pitch;             // E rounded up to 16
    int32_t *prefix;       // [ntiles][pitch] (scratch): their prefixes over the tiles; null for up to kRouterSumTiles tiles
};
int router_tile(const ef_router &r, int T);
constexpr int kRouterSmallTiles = 8192;   // most tokens that are in tiles of 16
hipError_t launch_router(const RouterArgs &a, hipStream_t s);

// ---- 8-bit products (ef_q8.hip) ----------------------------------------------------------------
struct QuantArgs {
    const void *x;
    int type;
    long long ldx;
    int rows, K;
    int8_t *codes;
    long long ldc, width;  // bytes from row to row; bytes of a row that may be written
    float *scales;         // null: x are codes already, only padded
};
hipError_t launch_quant_rows(const QuantArgs &a, hipStream_t s);

// `a`: codes whose rows are zero from K up to the next multiple of 64, or, where q8_product_quantises(), the caller's rows
struct Q8Args {
    const int8_t *a;
    long long lda;         // elements from row to row
    int a_type;            // EF_I8: codes
    const float *a_scale;  // of codes; null otherwise
    int a_rows;
    const int32_t *rows;
    int row_div, M;
    const int32_t *offsets;
    int G;
    const int8_t *w;
    long long ldw, w_group;
    const float *w_scale;
    int N, K, swiglu;
    void *out;
    int out_type;
    long long ldo;
};
bool q8_product_quantises(const Q8Args &a);
hipError_t launch_q8_product(const Q8Args &a, hipStream_t s);
// ef_q8_tiled.hip: `wide` = tiles of 256 x 256, otherwise of 128 x 128
hipError_t launch_q8_tiled(const Q8Args &a, bool wide, hipStream_t s);
// ef_q8_panel.hip
bool q8_panel_ok(const Q8Args &a);
hipError_t launch_q8_panel(const Q8Args &a, hipStream_t s);

struct CombineArgs {
    const void *y;
    int y_type;
    long long ldy;
    int y_rows;
    const float *w;
    const int32_t *inv_perm;
    int T, k, d;
    void *out;
    int out_type;
    long long ldo;
};
hipError_t launch_combine_rows(const CombineArgs &a, hipStream_t s);

}  // namespace ef

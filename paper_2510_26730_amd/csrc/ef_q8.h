// What the kernels of the 8-bit products share: which rows a workgroup takes, and how results leave.
#pragma once
#include "ef_device.h"
#include "ef_ops.h"

namespace ef {

// a tile of product rows: of one group, rows row0 .. row_end-1 at most `tile` of them
struct Q8Tile { int group, row0, row_end; };

// tiles of `tile` rows that M rows in G groups can make at most: the grid is sized without knowing the groups
inline int q8_tiles_bound(const Q8Args &p, int tile) {
    const int full = p.M / tile, ragged = p.G < p.M ? p.G : p.M;
    return p.G == 1 ? (p.M + tile - 1) / tile : full + ragged;
}

// Tile number `index` of the launch: every wave walks the offsets, 64 groups at a time.  Offsets are clamped to 0..M, and one that
// lies before an earlier one counts as that one: no tile leaves the M rows and no row is in two groups, whatever they hold.
__device__ __forceinline__ bool q8_find_tile(const Q8Args &p, int index, int tile, Q8Tile &t) {
    if (!p.offsets) {
        t = Q8Tile{0, index * tile, min(p.M, (index + 1) * tile)};
        return t.row0 < p.M;
    }
    const int lane = threadIdx.x & 63;
    int before = 0, end = 0;   // tiles and rows of the groups already walked
    for (int g0 = 0; g0 < p.G; g0 += 64) {
        const int g = g0 + lane;
        int lo = 0, hi = 0;
        if (g < p.G) {
            lo = min(max(p.offsets[g], 0), p.M);
            hi = min(max(p.offsets[g + 1], 0), p.M);
        }
        if (__ballot(g < p.G && (lo > hi || lo < end))) {
            lo = max(lo, end);
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int v = __shfl_up(lo, o);
                if (lane >= o) lo = max(lo, v);
            }
            hi = max(lo, hi);
        }
        const int n = (hi - lo + tile - 1) / tile;
        int incl = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(incl, o);
            if (lane >= o) incl += v;
        }
        const unsigned long long past = __ballot(before + incl > index);
        if (past) {
            const int l = __builtin_ctzll(past);
            const int first = before + __builtin_amdgcn_readlane(incl - n, l);
            const int glo = __builtin_amdgcn_readlane(lo, l), ghi = __builtin_amdgcn_readlane(hi, l);
            t.group = g0 + l;
            t.row0 = glo + (index - first) * tile;
            t.row_end = min(ghi, t.row0 + tile);
            return true;
        }
        before += __builtin_amdgcn_readlane(incl, 63);
        end = __builtin_amdgcn_readlane(hi, 63);
    }
    return false;
}

// the row of `a` behind a product row, and its scale; one that does not exist reads row 0 and counts as NaN
struct Q8Row { int row; float scale; };
__device__ __forceinline__ Q8Row q8_row(const Q8Args &p, int i) {
    int r = i;
    if (p.rows) {
        r = p.rows[i];
        r = r < 0 ? -1 : r / p.row_div;
    }
    if (r < 0 || r >= p.a_rows) return Q8Row{0, __builtin_nanf("")};
    return Q8Row{r, p.a_scale[r]};
}

template <int TYPE>
__device__ __forceinline__ void store_element(void *out, size_t at, float v) {
    if constexpr (TYPE == EF_F32) static_cast<float *>(out)[at] = v;
    else if constexpr (TYPE == EF_F16) static_cast<_Float16 *>(out)[at] = (_Float16)v;
    else static_cast<__bf16 *>(out)[at] = (__bf16)v;
}

// columns n .. n+3 of an output row, as far as they are below n_end
__device__ __forceinline__ void q8_store4(const Q8Args &p, int row, int n, int n_end, const float (&v)[4]) {
    const size_t at = (size_t)row * p.ldo + n;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (n + e >= n_end) return;
        if (p.out_type == EF_F32) store_element<EF_F32>(p.out, at + e, v[e]);
        else if (p.out_type == EF_F16) store_element<EF_F16>(p.out, at + e, v[e]);
        else store_element<EF_BF16>(p.out, at + e, v[e]);
    }
}

}  // namespace ef

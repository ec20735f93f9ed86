// What the kernels of the 8-bit products share: which rows a workgroup takes, and how results leave.
#pragma once
#include "ef_device.h"
#include "ef_kernels.h"
#include "ef_ops.h"

#include <type_traits>

namespace ef {

typedef int int4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int4v load16(const int8_t *p) { return *reinterpret_cast<const int4v *>(p); }

// a tile of product rows: rows row0 .. row_end-1 of a group, which has rows lo .. hi-1, `tiles` tiles and the first one's number
struct Q8Tile { int group, row0, row_end, lo, hi, first, tiles; };

// tiles of `tile` rows that M rows in G groups can make at most: the grid is sized without knowing the groups
inline int q8_tiles_bound(const Q8Args &p, int tile) {
    const int full = p.M / tile, ragged = p.G < p.M ? p.G : p.M;
    return p.G == 1 ? (p.M + tile - 1) / tile : full + ragged;
}

// rows of group g, 64 groups from g0 on, one per lane (none past the last group).  Offsets are clamped to 0..M, and one that lies
// before an earlier one counts as that one (`end`: the largest of the groups before g0), so no tile leaves the M rows and no row is
// in two groups, whatever they hold.
__device__ __forceinline__ void q8_group_rows(const Q8Args &p, int g0, int &end, int &lo, int &hi) {
    const int lane = threadIdx.x & 63, g = g0 + lane;
    lo = hi = 0;
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
    end = __builtin_amdgcn_readlane(hi, 63);
}

// Tile number `index` of the launch: every wave walks the offsets
__device__ __forceinline__ bool q8_find_tile(const Q8Args &p, int index, int tile, Q8Tile &t) {
    if (!p.offsets) {
        t = Q8Tile{0, index * tile, min(p.M, (index + 1) * tile), 0, p.M, 0, (p.M + tile - 1) / tile};
        return t.row0 < p.M;
    }
    const int lane = threadIdx.x & 63;
    int before = 0, end = 0;
    for (int g0 = 0; g0 < p.G; g0 += 64) {
        int lo, hi;
        q8_group_rows(p, g0, end, lo, hi);
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
            t.first = before + __builtin_amdgcn_readlane(incl - n, l);
            t.tiles = __builtin_amdgcn_readlane(n, l);
            t.lo = __builtin_amdgcn_readlane(lo, l);
            t.hi = __builtin_amdgcn_readlane(hi, l);
            t.group = g0 + l;
            t.row0 = t.lo + (index - t.first) * tile;
            t.row_end = min(t.hi, t.row0 + tile);
            return true;
        }
        before += __builtin_amdgcn_readlane(incl, 63);
    }
    return false;
}

// The unit (panel of matrix rows x tile of `tile` product rows) of workgroup `block`, of `npanels` panels: an even, contiguous share
// of all units for each XCD (workgroups go to the XCDs in turn), walked in the order of tiled_unit().  t.row0 / row_end are the
// tile's; false for workgroups past their XCD's share.
__device__ __forceinline__ bool q8_find_unit(const Q8Args &p, int block, int npanels, int tile, Q8Tile &t, int &panel) {
    const int part = block & 7, local = block >> 3;
    if (!p.offsets) {
        t.tiles = (p.M + tile - 1) / tile;
        t.group = t.first = t.lo = 0;
        t.hi = p.M;
    }
    int u;
    if (p.offsets && p.G <= 64) {      // one walk
        const int lane = threadIdx.x & 63;
        int end = 0, lo, hi;
        q8_group_rows(p, 0, end, lo, hi);
        const int n = (hi - lo + tile - 1) / tile;
        int incl = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(incl, o);
            if (lane >= o) incl += v;
        }
        const int units = __builtin_amdgcn_readlane(incl, 63) * npanels;
        u = tiled_xcd_begin(units, part) + local;
        if (u >= tiled_xcd_begin(units, part + 1)) return false;
        const int l = __builtin_ctzll(__ballot(incl > u / npanels));
        t.group = l;
        t.first = __builtin_amdgcn_readlane(incl - n, l);
        t.tiles = __builtin_amdgcn_readlane(n, l);
        t.lo = __builtin_amdgcn_readlane(lo, l);
        t.hi = __builtin_amdgcn_readlane(hi, l);
    } else {
        int total = t.tiles, end = 0;
        if (p.offsets) {
            total = 0;
            for (int g0 = 0; g0 < p.G; g0 += 64) {
                int lo, hi;
                q8_group_rows(p, g0, end, lo, hi);
                int n = (hi - lo + tile - 1) / tile;
                for (int o = 32; o >= 1; o >>= 1) n += __shfl_xor(n, o);
                total += __builtin_amdgcn_readfirstlane(n);
            }
        }
        const int units = total * npanels;
        u = tiled_xcd_begin(units, part) + local;
        if (u >= tiled_xcd_begin(units, part + 1)) return false;
        if (p.offsets && !q8_find_tile(p, u / npanels, tile, t)) return false;
    }
    const TiledUnit unit = tiled_unit(u - t.first * npanels, npanels, t.tiles);
    panel = unit.np;
    t.row0 = t.lo + unit.mp * tile;
    t.row_end = min(t.hi, t.row0 + tile);
    return true;
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
    return Q8Row{r, p.a_scale ? p.a_scale[r] : 0.f};
}

// The scales on a sum.  Sum times row scale passes 32 bits from a row scale of 2^97 on (values from 2e31), though the channel's scale may bring
// the result back, so a row scale of 2^64 and more gives 2^32 away, which the result gets back at its end: in between there is
// neither an overflow nor a subnormal number that the result has not.
constexpr float kLargeScale = 0x1p64f;
struct Q8Scale { float s, back; };
__device__ __forceinline__ Q8Scale q8_scale(float s) { return s >= kLargeScale ? Q8Scale{s * 0x1p-32f, 0x1p32f} : Q8Scale{s, 1.f}; }
__device__ __forceinline__ float q8_value(int sum, Q8Scale row, float channel) { return (float)sum * row.s * channel * row.back; }

// silu(g) * u.  silu_mul() gives 0 below a gate of -87.3, where the quotient is still a number of 32 bits (and, times a large u, not a small
// one): there it is g exp(g), which differs by exp(g); exp(-64) is taken out of the exponential.
constexpr float kDeepGate = -87.f;
__device__ __forceinline__ float q8_silu_mul_deep(float g, float u) {
    return g < kDeepGate ? g * __expf(g + 64.f) * u * 0x1.969d47321e4ccp-93f : silu_mul(g, u);
}
// v = silu(v) * u
__device__ __forceinline__ void q8_silu_mul4(float (&v)[4], const float (&u)[4]) {
    const bool deep = __any(fminf(fminf(v[0], v[1]), fminf(v[2], v[3])) < kDeepGate);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = deep ? q8_silu_mul_deep(v[e], u[e]) : silu_mul(v[e], u[e]);
}

// Four loads of a wave take 16 rows x 256 bytes, a step: lane 16g + 4q + c gets chunk c (16 bytes) of segment g (64 bytes) of row
// 4q + j in load j.  Neighbouring lanes have to be neighbours in memory: four lanes in one segment are one cycle of a compute unit's
// address unit, in four rows they are four (16 bytes a clock, less than the products need).  The matrix instruction wants rows in the
// lower lane bits, so four lanes and four loads change places: lane 16g + 4q + j then has the four chunks of segment g of row 4q + j,
// and product c takes every lane's chunk c, on both sides the same K.  With rows in neighbouring lanes of the loads: 32
// tokens of 64 experts, first half 64.7 against 60.6 us, second half 34.2 against 31.8; 64 x 2048 x 5632 9.7 against 8.2; 64 x 5632 x 1000
// 13.4 against 9.3.
__device__ __forceinline__ void transpose_quads(int4v (&v)[4], int lane) {
    const bool odd = lane & 1, high = lane & 2;
    const auto swap = [](int &lo, int &hi, bool up, auto move) {
        const int l = lo, h = hi, lm = move(l), hm = move(h);
        lo = up ? hm : l;
        hi = up ? h : lm;
    };
    const auto by1 = [](int x) { return __builtin_amdgcn_mov_dpp(x, 0xB1, 0xf, 0xf, true); };   // lane ^ 1
    const auto by2 = [](int x) { return __builtin_amdgcn_mov_dpp(x, 0x4E, 0xf, 0xf, true); };   // lane ^ 2
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        int a = v[0][e], b = v[1][e], c = v[2][e], d = v[3][e];
        swap(a, b, odd, by1);
        swap(c, d, odd, by1);
        swap(a, c, high, by2);
        swap(b, d, high, by2);
        v[0][e] = a, v[1][e] = b, v[2][e] = c, v[3][e] = d;
    }
}
constexpr int kStep = 256;                                                                       // codes of K
__device__ __forceinline__ int quad_row(int lane, int j) { return (lane & 12) + j; }            // of 16 rows, in load j
__device__ __forceinline__ int quad_code(int lane) { return (lane >> 4) * 64 + (lane & 3) * 16; }   // of a step

template <int TYPE>
__device__ __forceinline__ void store_element(void *out, size_t at, float v) {
    if constexpr (TYPE == EF_F32) static_cast<float *>(out)[at] = v;
    else if constexpr (TYPE == EF_F16) static_cast<_Float16 *>(out)[at] = (_Float16)v;
    else static_cast<__bf16 *>(out)[at] = (__bf16)v;
}

// four results, as the output type, into columns c .. c+3 of a row
template <int TYPE>
__device__ __forceinline__ void q8_put4(char *row, int c, const float (&v)[4]) {
    if constexpr (TYPE == EF_F32) *reinterpret_cast<float4 *>(row + c * 4) = make_float4(v[0], v[1], v[2], v[3]);
    else if constexpr (TYPE == EF_F16) {
        typedef _Float16 h4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<h4 *>(row + c * 2) = h4{(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
    } else {
        typedef __bf16 b4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<b4 *>(row + c * 2) = b4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
    }
}

// columns n .. n+3 of an output row, as far as they are below n_end: one store where the four are there and aligned
template <int TYPE>
__device__ __forceinline__ void q8_store4(const Q8Args &p, int row, int n, int n_end, const float (&v)[4]) {
    constexpr int size = TYPE == EF_F32 ? 4 : 2;
    const size_t at = (size_t)row * p.ldo + n;
    char *to = static_cast<char *>(p.out) + at * size;
    if (n + 4 <= n_end && (reinterpret_cast<size_t>(to) & (4 * size - 1)) == 0) {
        q8_put4<TYPE>(to, 0, v);
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < n_end) store_element<TYPE>(p.out, at + e, v[e]);
}

// calls f with the output type as a constant
template <class F>
__device__ __forceinline__ void q8_by_type(int type, F &&f) {
    if (type == EF_F32) f(std::integral_constant<int, EF_F32>{});
    else if (type == EF_F16) f(std::integral_constant<int, EF_F16>{});
    else f(std::integral_constant<int, EF_BF16>{});
}

}  // namespace ef

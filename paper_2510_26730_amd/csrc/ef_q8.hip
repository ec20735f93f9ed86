// Rows to 8 bits, products of 8-bit codes (streamed form), and the weighted sum of expert rows.
//
// out[i][n] = sa[row] * sw[n] * sum_k a[row][k] w[n][k]: the sum runs on the matrix cores in whole numbers, 32-bit and exact
// (K <= 131071), so neither the split of K nor the order of its parts changes a bit.  Three forms, all reading the codes as the
// caller has them, row by row:
//   streamed (here): few rows per matrix, bound by reading the weights.  Operands go from memory straight into the registers of
//   v_mfma_i32_16x16x64_i8; a load of a wave covers 256 bytes of 4 rows (ef_q8.h says how that becomes operands).
//   panels (ef_q8_panel.hip): too few tiles to fill the chip, or groups of some tens of rows.
//   tiled (ef_q8_tiled.hip): many rows, bound by the matrix cores.
#include "ef_device.h"
#include "ef_ops.h"
#include "ef_q8.h"

#include <algorithm>

namespace ef {

namespace {

// ------------------------------------------------------------------------------------------------
// rows to 8 bits
// ------------------------------------------------------------------------------------------------

// the whole number nearest x / s, ties to even, |x| / s <= 127.5.  The product with the reciprocal finds it to within one; the
// residual x - q s, which a multiply-add gives exactly here, says on which side of the halves x / s lies; twice it against s, since s / 2 need
// not be a number of 32 bits (s below 2^-125).
__device__ __forceinline__ int quant_code(float x, float s, float inv) {
    float q = __builtin_rintf(x * inv);
    const float r = 2.f * __builtin_fmaf(-q, s, x);
    const bool odd = (int)q & 1;
    if (r > s || (r == s && odd)) q += 1.f;
    else if (r < -s || (r == -s && odd)) q -= 1.f;
    return (int)q;
}

template <int TYPE> struct Element;
template <> struct Element<EF_F32> { using T = float; };
template <> struct Element<EF_BF16> { using T = uint16_t; };
template <> struct Element<EF_F16> { using T = uint16_t; };
template <int TYPE>
__device__ __forceinline__ float to_float(typename Element<TYPE>::T v) {
    if constexpr (TYPE == EF_F32) return v;
    else if constexpr (TYPE == EF_BF16) return __builtin_bit_cast(float, (uint32_t)v << 16);
    else return (float)__builtin_bit_cast(_Float16, v);
}

// 16 bytes of a row of type TYPE as 32-bit values
template <int TYPE>
__device__ __forceinline__ void unpack16(uint4 u, float (&v)[TYPE == EF_F32 ? 4 : 8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (TYPE == EF_F32) v[i] = __builtin_bit_cast(float, w[i]);
        else {
            v[2 * i] = to_float<TYPE>((uint16_t)w[i]);
            v[2 * i + 1] = to_float<TYPE>((uint16_t)(w[i] >> 16));
        }
    }
}

// the larger magnitudes of two words of one or two elements each, as bits: those order magnitudes, infinities and NaN on top
template <int TYPE>
__device__ __forceinline__ uint32_t larger(uint32_t most, uint32_t w) {
    if constexpr (TYPE == EF_F32) return max(most, w & 0x7FFFFFFFu);
    else {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, most), __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu)));
    }
}

// Four codes in a word.  x * inv + 1.5 * 2^23 leaves the nearest whole number, ties to even, in the low byte of the sum's bits; it is
// x / s rounded unless the residual says otherwise (a quotient next to a half, as x = max / 2 has), then the codes are formed again.
__device__ __forceinline__ uint32_t quant_four(const float *v, float s, float inv) {
    uint32_t y[4];
    float off = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float sum = __builtin_fmaf(v[i], inv, 12582912.f);
        off = fmaxf(off, fabsf(__builtin_fmaf(12582912.f - sum, s, v[i])));
        y[i] = __builtin_bit_cast(uint32_t, sum);
    }
    if (off >= 0.5f * s) {      // (an s / 2 that has to round separates the same residuals)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (uint32_t)quant_code(v[i], s, inv);
    }
    const uint32_t lo = __builtin_amdgcn_perm(y[1], y[0], 0x0C0C0400), hi = __builtin_amdgcn_perm(y[3], y[2], 0x0C0C0400);
    return hi << 16 | lo;
}

// Rows that are read once: a row's NC pieces of 16 bytes per lane stay in registers between the search for the largest magnitude
// and the codes.  WPR waves share a row.  Bound by reading and writing: 8192 rows of 4096 bf16 25-32 us, 3.1-4 TB/s
// (82 us where the row was read twice, an element per lane).
template <int TYPE, int NC, int WPR>
__global__ __launch_bounds__(256) void quant_rows_kernel(QuantArgs a) {
    constexpr int kPer = TYPE == EF_F32 ? 4 : 8;     // elements of a piece
    __shared__ uint32_t wave_most[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = blockIdx.x * (4 / WPR) + wave / WPR, l = (wave % WPR) * 64 + lane;
    const char *x = static_cast<const char *>(a.x) + (size_t)min(row, a.rows - 1) * a.ldx * (TYPE == EF_F32 ? 4 : 2);
    uint4 p[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int e = (c * 64 * WPR + l) * kPer;
        p[c] = e < a.K ? *reinterpret_cast<const uint4 *>(x + (size_t)e * (16 / kPer)) : make_uint4(0, 0, 0, 0);
    }
    uint32_t most = 0;
#pragma unroll
    for (int c = 0; c < NC; ++c) most = larger<TYPE>(larger<TYPE>(larger<TYPE>(larger<TYPE>(most, p[c].x), p[c].y), p[c].z), p[c].w);
    if constexpr (TYPE != EF_F32) most = __builtin_bit_cast(uint32_t, to_float<TYPE>((uint16_t)max(most & 0xFFFFu, most >> 16)));
    for (int off = 32; off >= 1; off >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off));
    if constexpr (WPR > 1) {
        if (lane == 0) wave_most[wave] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WPR; ++w) most = max(most, wave_most[wave / WPR * WPR + w]);
    }
    if (row >= a.rows) return;
    const bool bad = most >= 0x7F800000u;
    const float s = fmaxf(__builtin_bit_cast(float, most) / 127.f, 0x1p-126f), inv = 1.f / s;
    if (l == 0) a.scales[row] = bad ? __builtin_nanf("") : s;
    int8_t *out = a.codes + (size_t)row * a.ldc;
    const int padded = (a.K + 63) / 64 * 64;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int e = (c * 64 * WPR + l) * kPer;
        if (e >= padded) break;
        float v[kPer];
        unpack16<TYPE>(p[c], v);
        uint32_t q[kPer / 4];
#pragma unroll
        for (int w = 0; w < kPer / 4; ++w) q[w] = bad ? 0 : quant_four(v + 4 * w, s, inv);
        if constexpr (kPer == 8) *reinterpret_cast<uint2 *>(out + e) = make_uint2(q[0], q[1]);
        else *reinterpret_cast<uint32_t *>(out + e) = q[0];
    }
}

// Any row: strides, alignments and lengths that the kernel above does not take.  A workgroup takes a row and reads it twice, an element per
// lane: 8192 rows of 4097 bf16 36 us, 38 in 32 bits, from the caches, where 4104 bf16 take 18 in the kernel above.
template <int TYPE>
__global__ __launch_bounds__(256) void quant_any_kernel(QuantArgs a) {
    using T = typename Element<TYPE>::T;
    __shared__ uint32_t wave_most[4];
    const int row = blockIdx.x, tid = threadIdx.x;
    const T *x = static_cast<const T *>(a.x) + (size_t)row * a.ldx;
    int8_t *out = a.codes + (size_t)row * a.ldc;
    uint32_t most = 0;
    for (int i0 = 0; i0 < a.K; i0 += 8 * 256) {
        T v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = x[min(i0 + j * 256 + tid, a.K - 1)];
#pragma unroll
        for (int j = 0; j < 8; ++j) most = max(most, __builtin_bit_cast(uint32_t, to_float<TYPE>(v[j])) & 0x7FFFFFFFu);
    }
    for (int off = 32; off >= 1; off >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off));
    if ((tid & 63) == 0) wave_most[tid >> 6] = most;
    __syncthreads();
    most = max(max(wave_most[0], wave_most[1]), max(wave_most[2], wave_most[3]));
    const bool bad = most >= 0x7F800000u;
    const float s = fmaxf(__builtin_bit_cast(float, most) / 127.f, 0x1p-126f), inv = 1.f / s;
    if (tid == 0) a.scales[row] = bad ? __builtin_nanf("") : s;
    const int padded = (int)min((long long)(a.K + 63) / 64 * 64, a.width);
    for (int i0 = 0; i0 < padded; i0 += 8 * 256) {
        T v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = x[min(i0 + j * 256 + tid, a.K - 1)];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = i0 + j * 256 + tid;
            if (i < padded) out[i] = i < a.K && !bad ? (int8_t)quant_code(to_float<TYPE>(v[j]), s, inv) : 0;
        }
    }
}

// codes into rows whose bytes from K to the next multiple of 64 are zero, a byte per lane: 8192 rows of 4100 28 us
__global__ __launch_bounds__(256) void pad_rows_kernel(QuantArgs a) {
    const int8_t *x = static_cast<const int8_t *>(a.x) + (size_t)blockIdx.x * a.ldx;
    int8_t *out = a.codes + (size_t)blockIdx.x * a.ldc;
    for (int i = threadIdx.x; i < (a.K + 63) / 64 * 64; i += 256) out[i] = i < a.K ? x[i] : 0;
}

// ------------------------------------------------------------------------------------------------
// products, streamed
// ------------------------------------------------------------------------------------------------

// Bytes from row to row of the codes in LDS: whole steps, and 16 more that put neighbouring rows on different banks
__host__ __device__ inline int q8_tile_pitch(int K) { return (K + kStep - 1) / kStep * kStep + 16; }

// Quantises the n product rows from row0 on into LDS, zero from K to the end of the last step; a wave takes 64 pieces of 16 bytes of a
// row at a time.  Returns the scale of row (lane % 16).  Rows are read twice, the second time from the caches.
template <int NW, int TYPE>
__device__ __forceinline__ void quant_tile_codes(const Q8Args &p, int row0, int n, int pitch, int8_t *codes, uint32_t *most) {
    constexpr int kPer = TYPE == EF_F32 ? 4 : 8;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per_row = ((pitch - 16) / kPer + 63) / 64, units = n * per_row;
    const auto piece = [&](int unit, int &r, int &e) {
        r = unit / per_row;
        e = ((unit - r * per_row) * 64 + lane) * kPer;
        const Q8Row src = q8_row(p, row0 + r);
        return e < p.K ? *reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(p.a) + ((size_t)src.row * p.lda + e) * (16 / kPer))
                       : make_uint4(0, 0, 0, 0);
    };
    for (int u = wave; u < units; u += NW) {
        int r, e;
        const uint4 v = piece(u, r, e);
        uint32_t m = larger<TYPE>(larger<TYPE>(larger<TYPE>(larger<TYPE>(0, v.x), v.y), v.z), v.w);
        if constexpr (TYPE != EF_F32) m = __builtin_bit_cast(uint32_t, to_float<TYPE>((uint16_t)max(m & 0xFFFFu, m >> 16)));
        for (int off = 32; off >= 1; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off));
        if (lane == 0) atomicMax(&most[r], m);
    }
    __syncthreads();
    for (int u = wave; u < units; u += NW) {
        int r, e;
        const uint4 q = piece(u, r, e);
        const uint32_t m = most[r];
        const float s = fmaxf(__builtin_bit_cast(float, m) / 127.f, 0x1p-126f), inv = 1.f / s;
        float v[kPer];
        unpack16<TYPE>(q, v);
        if (e < pitch - 16)
#pragma unroll
            for (int w = 0; w < kPer / 4; ++w)
                reinterpret_cast<uint32_t *>(codes + r * pitch + e)[w] = m >= 0x7F800000u ? 0 : quant_four(v + 4 * w, s, inv);
    }
}
template <int NW>
__device__ __forceinline__ float quant_tile(const Q8Args &p, int row0, int n, int pitch, int8_t *codes, uint32_t *most) {
    if (threadIdx.x < 16) most[threadIdx.x] = 0;
    __syncthreads();
    if (p.a_type == EF_F32) quant_tile_codes<NW, EF_F32>(p, row0, n, pitch, codes, most);
    else if (p.a_type == EF_BF16) quant_tile_codes<NW, EF_BF16>(p, row0, n, pitch, codes, most);
    else quant_tile_codes<NW, EF_F16>(p, row0, n, pitch, codes, most);
    __syncthreads();
    const int r = min((int)threadIdx.x & 15, n - 1);
    const uint32_t m = most[r];
    const Q8Row src = q8_row(p, row0 + r);
    return m >= 0x7F800000u || src.scale != src.scale ? __builtin_nanf("") : fmaxf(__builtin_bit_cast(float, m) / 127.f, 0x1p-126f);
}

// A wave: NB blocks of 16 matrix rows (swiglu: 16 gate and their 16 up rows) for TT tiles of 16 product rows, in steps of 256 codes,
// DEPTH steps in flight; K in KS parts over the waves of a workgroup, which are added in LDS.
//
// QUANT: `a` is not codes yet.  The workgroup quantises its tile's rows into LDS itself, while its first weights are on their way, and
// the launch that would have done so is saved; every workgroup repeats it, so it is for a few rows.
template <int TT, bool PAIR, int NB, int KS, int DEPTH, bool QUANT>
__global__ __launch_bounds__(64 * (KS > 4 ? KS : 4)) void q8_stream_kernel(Q8Args p) {
    static_assert(!PAIR || NB == 2, "gate and up");
    static_assert(!QUANT || TT == 1, "few rows");
    constexpr int kWaves = KS > 4 ? KS : 4;
    extern __shared__ __attribute__((aligned(16))) int8_t tile_codes[];   // QUANT: M rows of q8_tile_pitch bytes
    __shared__ uint32_t tile_most[QUANT ? 16 : 1];
    __shared__ int4v sums[KS > 1 ? kWaves : 1][NB * TT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Q8Tile t;
    if (!q8_find_tile(p, blockIdx.y, 16 * TT, t)) return;
    const int part = wave & (KS - 1), cw = wave / KS;
    const int F = p.N >> 1;
    const int n0 = (blockIdx.x * (kWaves / KS) + cw) * (PAIR ? 16 : 16 * NB), n_end = PAIR ? F : p.N;
    const int i = lane & 15, g = lane >> 4;
    const int steps = (p.K + kStep - 1) / kStep;
    const int s0 = steps * part / KS, s1 = steps * (part + 1) / KS;
    const bool run = n0 < n_end && s0 < s1;

    // columns past the end and rows past the group's read a neighbour's codes; their results are dropped
    const int8_t *w[NB][4];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const int c = min(n0 + (PAIR ? 0 : 16 * b) + quad_row(lane, h), n_end - 1);
            w[b][h] = p.w + (size_t)t.group * p.w_group + (size_t)(PAIR && b ? F + c : c) * p.ldw;
        }
    const int k_last = ((p.K + 15) & ~15) - 16;   // last 16 codes that a weight row holds
    int4v wb[DEPTH][NB][4], xb[DEPTH][TT][4];
    const auto fetch_w = [&](int u, int s) {
        const int k = min(min(s, s1 - 1) * kStep + quad_code(lane), k_last);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int h = 0; h < 4; ++h) wb[u][b][h] = load16(w[b][h] + k);
    };
    if (run)
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) fetch_w(u, s0 + u);

    const int8_t *x[TT][4];
    float xs[TT], ws[NB][4];
    if constexpr (QUANT) {
        const int n = t.row_end - t.row0, pitch = q8_tile_pitch(p.K);
        xs[0] = quant_tile<kWaves>(p, t.row0, n, pitch, tile_codes, tile_most);
        x[0][0] = tile_codes + min(i, n - 1) * pitch + 64 * g;
    } else {
#pragma unroll
        for (int j = 0; j < TT; ++j) {
#pragma unroll
            for (int h = 0; h < 4; ++h) x[j][h] = p.a + (size_t)q8_row(p, min(t.row0 + 16 * j + quad_row(lane, h), t.row_end - 1)).row * p.lda;
            xs[j] = q8_row(p, min(t.row0 + 16 * j + i, t.row_end - 1)).scale;
        }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = min(n0 + (PAIR ? 0 : 16 * b) + 4 * g + e, n_end - 1);
            ws[b][e] = p.w_scale[(size_t)t.group * p.N + (PAIR && b ? F + c : c)];
        }
    // Rows of `a` are zero from K up to x_end, a multiple of 64; chunks behind it are read from before it and cleared
    const int x_end = (p.K + 63) & ~63;
    const auto fetch_x = [&](int u, int s) {
        if constexpr (QUANT) {
#pragma unroll
            for (int c = 0; c < 4; ++c) xb[u][0][c] = load16(x[0][0] + min(s, s1 - 1) * kStep + 16 * c);
            return;
        }
        const int k = min(min(s, s1 - 1) * kStep + quad_code(lane), x_end - 16);
#pragma unroll
        for (int j = 0; j < TT; ++j)
#pragma unroll
            for (int h = 0; h < 4; ++h) xb[u][j][h] = load16(x[j][h] + k);
    };

    int4v acc[NB][TT];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < TT; ++j) acc[b][j] = int4v{0, 0, 0, 0};
    if (run) {
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) fetch_x(u, s0 + u);
        const auto multiply = [&](int u, int s) {
            if constexpr (!QUANT) {
#pragma unroll
                for (int j = 0; j < TT; ++j) transpose_quads(xb[u][j], lane);
                if (s * kStep + 64 * g >= x_end) {
#pragma unroll
                    for (int j = 0; j < TT; ++j)
#pragma unroll
                        for (int c = 0; c < 4; ++c) xb[u][j][c] = int4v{0, 0, 0, 0};
                }
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                transpose_quads(wb[u][b], lane);
#pragma unroll
                for (int j = 0; j < TT; ++j)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[b][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wb[u][b][c], xb[u][j][c], acc[b][j], 0, 0, 0);
            }
        };
        // loads without a branch between them keep the compiler's wait counts exact; past the end they repeat the last step
        int s = s0;
        for (; s + DEPTH < s1; s += DEPTH) {
#pragma unroll
            for (int u = 0; u < DEPTH; ++u) {
                multiply(u, s + u);
                fetch_w(u, s + u + DEPTH);
                fetch_x(u, s + u + DEPTH);
            }
        }
#pragma unroll
        for (int u = 0; u < DEPTH; ++u)
            if (s + u < s1) multiply(u, s + u);
    }
    if constexpr (KS > 1) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int j = 0; j < TT; ++j) sums[wave][b * TT + j][lane] = acc[b][j];
        __syncthreads();
        if (part != 0) return;
#pragma unroll
        for (int q = 1; q < KS; ++q)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int j = 0; j < TT; ++j) acc[b][j] += sums[wave + q][b * TT + j][lane];
    }
    if (n0 >= n_end) return;
    // lane 16g + i holds product row i, matrix rows 4g .. 4g+3 of each 16
    q8_by_type(p.out_type, [&](auto TYPE) {
#pragma unroll
        for (int j = 0; j < TT; ++j) {
            const int row = t.row0 + 16 * j + i;
            if (row >= t.row_end) continue;
            const Q8Scale scale = q8_scale(xs[j]);
            float v[NB][4];
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[b][e] = q8_value(acc[b][j][e], scale, ws[b][e]);
            if constexpr (PAIR) q8_silu_mul4(v[0], v[1]);
#pragma unroll
            for (int b = 0; b < (PAIR ? 1 : NB); ++b) q8_store4<decltype(TYPE)::value>(p, row, n0 + 16 * b + 4 * g, n_end, v[b]);
        }
    });
}

// Waves that a streamed launch has without a split of K, for tiles of 16*TT rows
long long stream_waves(const Q8Args &p, int TT) {
    const int cols = p.swiglu ? p.N / 2 : p.N, per = p.swiglu ? 16 : 32;
    return (long long)((cols + per - 1) / per) * q8_tiles_bound(p, 16 * TT);
}

// From 2048 waves (two per SIMD) on K stays whole; below, four waves share it; below 512, eight, with 16 columns each, so that twice
// the workgroups share the columns (1 x 4096 x 4096 8.6 -> 7.0 us).
template <int TT, bool PAIR, bool QUANT>
hipError_t launch_stream(const Q8Args &p, hipStream_t s) {
    const int cols = PAIR ? p.N / 2 : p.N, tiles = q8_tiles_bound(p, 16 * TT);
    const int b16 = (cols + 15) / 16, b32 = (cols + 31) / 32, wide = PAIR ? b16 : b32;
    const size_t lds = QUANT ? (size_t)p.M * q8_tile_pitch(p.K) : 0;
    if (tiles > 65535) return hipErrorInvalidValue;
    const long long waves = stream_waves(p, TT);
    if (TT < 4 && waves >= 2048) {
        if constexpr (TT < 4) hipLaunchKernelGGL((q8_stream_kernel<TT, PAIR, 2, 1, 1, QUANT>), dim3((wide + 3) / 4, tiles), dim3(256), lds, s, p);
    } else if (PAIR || TT > 1 || waves >= 512) {
        hipLaunchKernelGGL((q8_stream_kernel<TT, PAIR, 2, 4, 1, QUANT>), dim3(wide, tiles), dim3(256), lds, s, p);
    } else if constexpr (!PAIR && TT == 1) {
        hipLaunchKernelGGL((q8_stream_kernel<1, false, 1, 8, 2, QUANT>), dim3(b16, tiles), dim3(512), lds, s, p);
    }
    return hipGetLastError();
}
template <int TT, bool QUANT>
hipError_t launch_stream(const Q8Args &p, hipStream_t s) {
    return p.swiglu ? launch_stream<TT, true, QUANT>(p, s) : launch_stream<TT, false, QUANT>(p, s);
}

// ------------------------------------------------------------------------------------------------
// weighted sum of the expert rows of a token
// ------------------------------------------------------------------------------------------------
// A lane takes W columns (16 bytes of y), the rows of up to four slots in flight; sums in the order of the slots.  Bound by reading y:
// 1056 tokens, six rows of 2048 in 32 bits each, 10.2 us = 5.5 TB/s (an element per lane 16.4).
template <int YT, int OT, int W>
__global__ __launch_bounds__(256) void combine_rows_kernel(CombineArgs a) {
    using Y = typename Element<YT>::T;
    const Y *y = static_cast<const Y *>(a.y);
    const int t = blockIdx.x, c = (blockIdx.y * 256 + threadIdx.x) * W;
    if (c >= a.d) return;
    float sum[W];
    // a row that does not exist reads row 0 and counts as NaN; without rows there is not even that one
    const int slots = a.y_rows ? a.k : 0;
#pragma unroll
    for (int e = 0; e < W; ++e) sum[e] = a.y_rows ? 0.f : __builtin_nanf("");
    const long long slot0 = (long long)t * a.k;
    for (int j0 = 0; j0 < slots; j0 += 4) {
        Y v[4][W];
        float w[4];
        bool live[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const long long slot = slot0 + min(j0 + q, a.k - 1);
            long long r = a.inv_perm ? a.inv_perm[slot] : slot;
            live[q] = r >= 0 && r < a.y_rows;
            if (!live[q]) r = 0;
            w[q] = a.w[slot];
            if constexpr (W > 1) *reinterpret_cast<uint4 *>(v[q]) = *reinterpret_cast<const uint4 *>(y + r * a.ldy + c);
            else v[q][0] = y[r * a.ldy + c];
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (j0 + q < a.k)
#pragma unroll
                for (int e = 0; e < W; ++e) sum[e] = __builtin_fmaf(w[q], live[q] ? to_float<YT>(v[q][e]) : __builtin_nanf(""), sum[e]);
    }
    const size_t at = (size_t)t * a.ldo + c;
    if constexpr (W == 1) store_element<OT>(a.out, at, sum[0]);
    else {
#pragma unroll
        for (int e = 0; e < W; e += 4) {
            const float f[4] = {sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
            q8_put4<OT>(static_cast<char *>(a.out) + (at + e) * (OT == EF_F32 ? 4 : 2), 0, f);
        }
    }
}

template <int YT, int OT>
hipError_t launch_combine_rows(const CombineArgs &a, hipStream_t s) {
    constexpr int W = YT == EF_F32 ? 4 : 8, out = OT == EF_F32 ? 4 : 2;
    const bool whole = a.d % W == 0 && a.ldy % W == 0 && reinterpret_cast<size_t>(a.y) % 16 == 0 && a.ldo % 4 == 0 &&
                       reinterpret_cast<size_t>(a.out) % (4 * out) == 0;
    if (whole) hipLaunchKernelGGL((combine_rows_kernel<YT, OT, W>), dim3(a.T, (a.d / W + 255) / 256), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((combine_rows_kernel<YT, OT, 1>), dim3(a.T, (a.d + 255) / 256), dim3(256), 0, s, a);
    return hipGetLastError();
}
template <int YT>
hipError_t launch_combine_y(const CombineArgs &a, hipStream_t s) {
    return a.out_type == EF_BF16 ? launch_combine_rows<YT, EF_BF16>(a, s) : a.out_type == EF_F16 ? launch_combine_rows<YT, EF_F16>(a, s)
                                                                                                 : launch_combine_rows<YT, EF_F32>(a, s);
}

}  // namespace

namespace {

template <int TYPE>
hipError_t launch_quant(const QuantArgs &a, hipStream_t s) {
    constexpr int kPer = TYPE == EF_F32 ? 4 : 8;
    const int pieces = (a.K + kPer - 1) / kPer;      // of 16 bytes
    const bool whole = a.K % kPer == 0 && a.ldx % kPer == 0 && reinterpret_cast<size_t>(a.x) % 16 == 0 && a.ldc % 16 == 0 &&
                       a.width >= (a.K + 63) / 64 * 64 && reinterpret_cast<size_t>(a.codes) % 16 == 0;
    const dim3 block(256);
    if (!whole || pieces > 64 * 4 * 16) hipLaunchKernelGGL(quant_any_kernel<TYPE>, dim3(a.rows), block, 0, s, a);
    // a wave per row while that keeps eight pieces of a lane or fewer and there are rows for every compute unit, else four
    else if (pieces <= 64 * 2 && a.rows >= 1024) hipLaunchKernelGGL((quant_rows_kernel<TYPE, 2, 1>), dim3((a.rows + 3) / 4), block, 0, s, a);
    else if (pieces <= 64 * 4 && a.rows >= 1024) hipLaunchKernelGGL((quant_rows_kernel<TYPE, 4, 1>), dim3((a.rows + 3) / 4), block, 0, s, a);
    else if (pieces <= 64 * 8 && a.rows >= 1024) hipLaunchKernelGGL((quant_rows_kernel<TYPE, 8, 1>), dim3((a.rows + 3) / 4), block, 0, s, a);
    else if (pieces <= 64 * 4) hipLaunchKernelGGL((quant_rows_kernel<TYPE, 1, 4>), dim3(a.rows), block, 0, s, a);
    else if (pieces <= 64 * 4 * 2) hipLaunchKernelGGL((quant_rows_kernel<TYPE, 2, 4>), dim3(a.rows), block, 0, s, a);
    else if (pieces <= 64 * 4 * 4) hipLaunchKernelGGL((quant_rows_kernel<TYPE, 4, 4>), dim3(a.rows), block, 0, s, a);
    else if (pieces <= 64 * 4 * 8) hipLaunchKernelGGL((quant_rows_kernel<TYPE, 8, 4>), dim3(a.rows), block, 0, s, a);
    else hipLaunchKernelGGL((quant_rows_kernel<TYPE, 16, 4>), dim3(a.rows), block, 0, s, a);
    return hipGetLastError();
}

}  // namespace

// A launch has fewer than 2^32 lanes, and some forms take 256 for a row
constexpr int kRowsPerLaunch = 1 << 23;

hipError_t launch_quant_rows(const QuantArgs &all, hipStream_t s) {
    QuantArgs a = all;
    for (; a.rows > kRowsPerLaunch;) {
        QuantArgs part = a;
        part.rows = kRowsPerLaunch;
        const hipError_t e = launch_quant_rows(part, s);
        if (e != hipSuccess) return e;
        a.x = static_cast<const char *>(a.x) + kRowsPerLaunch * a.ldx * (a.type == EF_F32 ? 4 : a.type == EF_I8 ? 1 : 2);
        a.codes += kRowsPerLaunch * a.ldc;
        if (a.scales) a.scales += kRowsPerLaunch;
        a.rows -= kRowsPerLaunch;
    }
    if (a.rows <= 0) return hipSuccess;
    switch (a.type) {
        case EF_I8: hipLaunchKernelGGL(pad_rows_kernel, dim3(a.rows), dim3(256), 0, s, a); return hipGetLastError();
        case EF_BF16: return launch_quant<EF_BF16>(a, s);
        case EF_F16: return launch_quant<EF_F16>(a, s);
        default: return launch_quant<EF_F32>(a, s);
    }
}

// Whether the product quantises rows itself (p.a: the rows as they are): up to four rows, one matrix, aligned to 16 bytes, whose codes
// fit LDS.  1 x 4096 x 4096: 6.4 us in one launch against 3 + 6 and the gap between two.  Not for groups, whose tiles need LDS for 16
// rows each and run four instead of five to a compute unit: 32 tokens of 64 experts, first half, 74 against 4.7 + 60.9 us.
bool q8_product_quantises(const Q8Args &p) {
    const int per = p.a_type == EF_F32 ? 4 : 8;
    return p.a_type != EF_I8 && p.G == 1 && p.M <= 4 && p.K % per == 0 && p.lda % per == 0 && reinterpret_cast<size_t>(p.a) % 16 == 0 &&
           p.M * q8_tile_pitch(p.K) <= 64 * 1024;
}

// Which form a product takes, by its sizes alone (the groups' own sizes are on the device).  Measured with codes in place; us of the
// form taken / the next best:
//   streamed   one matrix, up to 32 rows of any width: 32 x 4096 x 14336 16.2 / 24.7 (panels); tiles of 32 rows that give every compute unit
//              one workgroup: 64 x 4096 x 4096 8.4 / 16.9 (128 x 128 tiles), 256 x 5632 x 1000 9.9 / 14.0 (tiles of 64); of 64 rows while two
//              workgroups a unit take all: 256 x 4096 x 4096 14.8 / 17.4, 1024 x 5632 x 1000 19.5 / 27.6, 64 x 4096 x 14336 20.7 / 25.5; past
//              that 384 x 4096 x 4096 21.4 against 17.0, 517 x 5640 x 2049 43.9 against 35.0, though 384 x 1408 x 2048, 9.3 against 8.5.
//              Groups of few rows where K is short, because a panel takes longer to start: 256 groups of 12, 1024 x 512, 28.4 / 32.2, of
//              16 33.7 against 32.5; 64 of 8, 2048 x 2816, 65.2 / 68.6, of 16 84.2 against 69.9.  Few groups at work, as with one token: 8 of
//              8, 14336 x 4096, 80.7 / 84.8, of 16 103.2 against 84.4.
//   panels     groups of up to 40 rows: 8 of 12, 4096 x 28672, 158.1 / 171.2; 64 of 64, 1408 x 2048, 43.3 against 35.4.  One matrix and one
//              round of panels, of up to 128 rows (4096 x 14336 21.0 / 28.0; 192 rows, two rounds, 31.1 against 27.3), with a long K
//              (384 x 4096 x 4096 17.0 / 18.0, 2048 x 5632 x 1000 23.1 / 27.2; 768 x 2048 x 2048 11.4 against 11.0) or with rows that are
//              not aligned to 64 bytes (517 x 5640 x 2049 35.0 / 44.1).
//   256 x 256  where rows per group times K make up for the start and end of a tile, and tiles fill half of the chip and more:
//              64 groups of 384, 2048 x 2816, 223 / 233, of 192 145 against 142; 64 of 384, 1408 x 2048, 148 against 136; 768 x 4096 x
//              14336 (168 tiles) 55.0 / 72.5, 384 (112) 47.1 against 44.2.
//   128 x 128  the rest.
hipError_t launch_q8_product(const Q8Args &p, hipStream_t s) {
    if (p.M <= 0) return hipSuccess;
    const int per = (p.M + p.G - 1) / p.G, cols = p.swiglu ? p.N / 2 : p.N;
    if (p.a_type != EF_I8) return q8_product_quantises(p) ? launch_stream<1, true>(p, s) : hipErrorInvalidValue;
    const auto panels = [&](int width) { return (long long)((cols + width - 1) / width); };
    if (p.G == 1) {
        if (p.M <= 16) return launch_stream<1, false>(p, s);
        if (p.M <= 32 || stream_waves(p, 2) <= 256) return launch_stream<2, false>(p, s);
        if (stream_waves(p, 4) <= 512) return launch_stream<4, false>(p, s);
        if (q8_panel_ok(p) && (p.M <= 128 || p.K >= 4096 || p.ldw % 64 != 0) &&
            panels(p.swiglu ? 64 : 128) * q8_tiles_bound(p, 64) <= 256)
            return launch_q8_panel(p, s);
    } else {
        if (per <= (p.K <= 1024 ? 12 : p.K <= 2048 ? 8 : 0) || (per <= 8 && stream_waves(p, 1) <= 2048)) return launch_stream<1, false>(p, s);
        if (q8_panel_ok(p) && per <= 40) return launch_q8_panel(p, s);
    }
    const long long tiles = std::max((p.M + 255) / 256, std::min(p.G, p.M));
    return launch_q8_tiled(p, (long long)per * p.K >= 512 * 1024 && tiles * panels(p.swiglu ? 128 : 256) >= 160, s);
}

hipError_t launch_combine_rows(const CombineArgs &all, hipStream_t s) {
    CombineArgs a = all;
    for (; a.T > kRowsPerLaunch;) {
        CombineArgs part = a;
        part.T = kRowsPerLaunch;
        const hipError_t e = launch_combine_rows(part, s);
        if (e != hipSuccess) return e;
        const long long slots = (long long)kRowsPerLaunch * a.k;
        if (a.inv_perm) a.inv_perm += slots;
        else {
            a.y = static_cast<const char *>(a.y) + slots * a.ldy * (a.y_type == EF_F32 ? 4 : 2);
            a.y_rows -= (int)slots;
        }
        a.w += slots;
        a.out = static_cast<char *>(a.out) + kRowsPerLaunch * a.ldo * (a.out_type == EF_F32 ? 4 : 2);
        a.T -= kRowsPerLaunch;
    }
    if (a.T <= 0) return hipSuccess;
    return a.y_type == EF_BF16 ? launch_combine_y<EF_BF16>(a, s) : a.y_type == EF_F16 ? launch_combine_y<EF_F16>(a, s)
                                                                                      : launch_combine_y<EF_F32>(a, s);
}

}  // namespace ef

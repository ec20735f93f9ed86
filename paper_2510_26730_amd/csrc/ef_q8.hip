// Rows to 8 bits, products of 8-bit codes (streamed form), and the weighted sum of expert rows.
//
// out[i][n] = sa[row] * sw[n] * sum_k a[row][k] w[n][k]: the sum runs on the matrix cores in whole numbers, 32-bit and exact
// (K <= 131071), so neither the split of K nor the order of its parts changes a bit.  Two forms, both reading the codes as the
// caller has them, row by row:
//   streamed (here): few rows per matrix, bound by reading the weights.  Operands go from memory straight into the registers of
//   v_mfma_i32_16x16x64_i8 (lane 16g + i: row i, 16 bytes of K at 16g), so a load of a wave covers 64 consecutive bytes of 16 rows.
//   tiled (ef_q8_tiled.hip): many rows, bound by the matrix cores.
#include "ef_device.h"
#include "ef_ops.h"
#include "ef_q8.h"

namespace ef {

namespace {

// ------------------------------------------------------------------------------------------------
// rows to 8 bits
// ------------------------------------------------------------------------------------------------

// the whole number nearest x / s, ties to even, |x| / s <= 127.5.  The product with the reciprocal finds it to within one; the
// residual x - q s, which a multiply-add gives exactly here, says on which side of the halves x / s lies.
__device__ __forceinline__ int quant_code(float x, float s, float inv) {
    float q = __builtin_rintf(x * inv);
    const float r = __builtin_fmaf(-q, s, x), h = 0.5f * s;
    const bool odd = (int)q & 1;
    if (r > h || (r == h && odd)) q += 1.f;
    else if (r < -h || (r == -h && odd)) q -= 1.f;
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
    if (off >= 0.5f * s) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (uint32_t)quant_code(v[i], s, inv);
    }
    const uint32_t lo = __builtin_amdgcn_perm(y[1], y[0], 0x0C0C0400), hi = __builtin_amdgcn_perm(y[3], y[2], 0x0C0C0400);
    return hi << 16 | lo;
}

// Rows that are read once: a row's NC pieces of 16 bytes per lane stay in registers between the search for the largest magnitude
// and the codes.  WPR waves share a row.  Bound by reading and writing, 8192 rows of 4096 bf16 MEASURED_HERE.
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

// Any row: strides, alignments and lengths that the kernel above does not take.  A workgroup takes a row and reads it twice.
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
    const int padded = (int)min((long long)(a.K + 63) / 64 * 64, a.ldc);
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

// codes into rows whose bytes from K to the next multiple of 64 are zero
__global__ __launch_bounds__(256) void pad_rows_kernel(QuantArgs a) {
    const int8_t *x = static_cast<const int8_t *>(a.x) + (size_t)blockIdx.x * a.ldx;
    int8_t *out = a.codes + (size_t)blockIdx.x * a.ldc;
    for (int i = threadIdx.x; i < (a.K + 63) / 64 * 64; i += 256) out[i] = i < a.K ? x[i] : 0;
}

// ------------------------------------------------------------------------------------------------
// products, streamed
// ------------------------------------------------------------------------------------------------
typedef int int4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int4v load16(const int8_t *p) { return *reinterpret_cast<const int4v *>(p); }
__device__ __forceinline__ int4v load16_stream(const int8_t *p) { return __builtin_nontemporal_load(reinterpret_cast<const int4v *>(p)); }

// A wave: 32 columns of the matrix (swiglu: 16 gate and their 16 up columns) for TT tiles of 16 rows, K in KS parts over the
// waves of a workgroup, which are added in LDS.
constexpr int kStreamDepth = 4;    // K steps of 64 in flight per wave

template <int TT, bool PAIR, int KS>
__global__ __launch_bounds__(256) void q8_stream_kernel(Q8Args p) {
    __shared__ int4v sums[KS > 1 ? 4 : 1][2 * TT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Q8Tile t;
    if (!q8_find_tile(p, blockIdx.y, 16 * TT, t)) return;
    const int part = wave & (KS - 1), cw = wave / KS;
    const int F = p.N >> 1;
    const int n0 = (blockIdx.x * (4 / KS) + cw) * (PAIR ? 16 : 32), n_end = PAIR ? F : p.N;
    const int i = lane & 15, g = lane >> 4;
    const int steps = (p.K + 63) >> 6;
    const int s0 = steps * part / KS, s1 = steps * (part + 1) / KS;

    // columns past the end and rows past the group's read a neighbour's codes; their results are dropped
    const int c0 = min(n0 + i, n_end - 1), c1 = PAIR ? F + c0 : min(n0 + 16 + i, n_end - 1);
    const int8_t *w = p.w + (size_t)t.group * p.w_group;
    const int8_t *w0 = w + (size_t)c0 * p.ldw, *w1 = w + (size_t)c1 * p.ldw;
    const int8_t *x[TT];
    float xs[TT];
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        const Q8Row r = q8_row(p, min(t.row0 + 16 * j + i, t.row_end - 1));
        x[j] = p.a + (size_t)r.row * p.lda + 16 * g;
        xs[j] = r.scale;
    }
    const int k_last = ((p.K + 15) & ~15) - 16;   // last 16 codes that a weight row holds; beyond K the rows of `a` are zero

    int4v acc[2][TT];
#pragma unroll
    for (int j = 0; j < TT; ++j) acc[0][j] = acc[1][j] = int4v{0, 0, 0, 0};
    int4v wb[2][kStreamDepth], xb[TT][kStreamDepth];
    const auto fetch = [&](int u, int s) {
        const int k = min(s, s1 - 1) * 64;
        const int kw = min(k + 16 * g, k_last);
        wb[0][u] = load16_stream(w0 + kw);
        wb[1][u] = load16_stream(w1 + kw);
#pragma unroll
        for (int j = 0; j < TT; ++j) xb[j][u] = load16(x[j] + k);
    };
    if (n0 < n_end && s0 < s1) {
#pragma unroll
        for (int u = 0; u < kStreamDepth; ++u) fetch(u, s0 + u);
        for (int s = s0; s < s1; s += kStreamDepth) {
#pragma unroll
            for (int u = 0; u < kStreamDepth; ++u) {
                if (s + u < s1) {
#pragma unroll
                    for (int j = 0; j < TT; ++j) {
                        acc[0][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wb[0][u], xb[j][u], acc[0][j], 0, 0, 0);
                        acc[1][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wb[1][u], xb[j][u], acc[1][j], 0, 0, 0);
                    }
                }
                fetch(u, s + u + kStreamDepth);
            }
        }
    }
    if constexpr (KS > 1) {
#pragma unroll
        for (int j = 0; j < TT; ++j) {
            sums[wave][2 * j][lane] = acc[0][j];
            sums[wave][2 * j + 1][lane] = acc[1][j];
        }
        __syncthreads();
        if (part != 0) return;
#pragma unroll
        for (int j = 0; j < TT; ++j)
#pragma unroll
            for (int q = 1; q < KS; ++q) {
                acc[0][j] += sums[wave + q][2 * j][lane];
                acc[1][j] += sums[wave + q][2 * j + 1][lane];
            }
    }
    if (n0 >= n_end) return;
    // lane 16g + i holds row (token) i, columns 4g .. 4g+3 of each 16
    const float *ws = p.w_scale + (size_t)t.group * p.N;
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        const int row = t.row0 + 16 * j + i;
        if (row >= t.row_end) continue;
        if constexpr (PAIR) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int f = min(n0 + 4 * g + e, F - 1);
                v[e] = silu_mul((float)acc[0][j][e] * xs[j] * ws[f], (float)acc[1][j][e] * xs[j] * ws[F + f]);
            }
            q8_store4(p, row, n0 + 4 * g, F, v);
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (float)acc[h][j][e] * xs[j] * ws[min(n0 + 16 * h + 4 * g + e, p.N - 1)];
                q8_store4(p, row, n0 + 16 * h + 4 * g, p.N, v);
            }
        }
    }
}

template <int TT, bool PAIR>
hipError_t launch_stream(const Q8Args &p, hipStream_t s) {
    const int per_wave = PAIR ? 16 : 32, cols = PAIR ? p.N / 2 : p.N;
    const int waves = (cols + per_wave - 1) / per_wave, tiles = q8_tiles_bound(p, 16 * TT);
    if ((long long)waves * tiles >= 2048) hipLaunchKernelGGL((q8_stream_kernel<TT, PAIR, 1>), dim3((waves + 3) / 4, tiles), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((q8_stream_kernel<TT, PAIR, 4>), dim3(waves, tiles), dim3(256), 0, s, p);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// weighted sum of the expert rows of a token
// ------------------------------------------------------------------------------------------------
template <int YT, int OT>
__global__ __launch_bounds__(256) void combine_rows_kernel(CombineArgs a) {
    using Y = typename Element<YT>::T;
    const Y *y = static_cast<const Y *>(a.y);
    const int t = blockIdx.x;
    for (int i = blockIdx.y * 256 + threadIdx.x; i < a.d; i += gridDim.y * 256) {
        float sum = 0.f;
        for (int j = 0; j < a.k; ++j) {
            const long long slot = (long long)t * a.k + j, r = a.inv_perm ? a.inv_perm[slot] : slot;
            const float v = r >= 0 && r < a.y_rows ? to_float<YT>(y[r * a.ldy + i]) : __builtin_nanf("");
            sum = __builtin_fmaf(a.w[slot], v, sum);
        }
        store_element<OT>(a.out, (size_t)t * a.ldo + i, sum);
    }
}

template <int YT>
hipError_t launch_combine_y(const CombineArgs &a, hipStream_t s) {
    const dim3 grid(a.T, (a.d + 255) / 256);
    switch (a.out_type) {
        case EF_BF16: hipLaunchKernelGGL((combine_rows_kernel<YT, EF_BF16>), grid, dim3(256), 0, s, a); break;
        case EF_F16: hipLaunchKernelGGL((combine_rows_kernel<YT, EF_F16>), grid, dim3(256), 0, s, a); break;
        default: hipLaunchKernelGGL((combine_rows_kernel<YT, EF_F32>), grid, dim3(256), 0, s, a); break;
    }
    return hipGetLastError();
}

}  // namespace

namespace {

template <int TYPE>
hipError_t launch_quant(const QuantArgs &a, hipStream_t s) {
    constexpr int kPer = TYPE == EF_F32 ? 4 : 8;
    const int pieces = (a.K + kPer - 1) / kPer;      // of 16 bytes
    const bool whole = a.K % kPer == 0 && a.ldx % kPer == 0 && reinterpret_cast<size_t>(a.x) % 16 == 0 && a.ldc % 16 == 0 &&
                       a.ldc >= (a.K + 63) / 64 * 64 && reinterpret_cast<size_t>(a.codes) % 16 == 0;
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

hipError_t launch_quant_rows(const QuantArgs &a, hipStream_t s) {
    if (a.rows <= 0) return hipSuccess;
    switch (a.type) {
        case EF_I8: hipLaunchKernelGGL(pad_rows_kernel, dim3(a.rows), dim3(256), 0, s, a); return hipGetLastError();
        case EF_BF16: return launch_quant<EF_BF16>(a, s);
        case EF_F16: return launch_quant<EF_F16>(a, s);
        default: return launch_quant<EF_F32>(a, s);
    }
}

hipError_t launch_q8_product(const Q8Args &p, hipStream_t s) {
    if (p.M <= 0) return hipSuccess;
    const int per = (p.M + p.G - 1) / p.G;
    if (per > 64) return launch_q8_tiled(p, per > 512, s);
    if (p.swiglu) return per <= 16 ? launch_stream<1, true>(p, s) : per <= 32 ? launch_stream<2, true>(p, s) : launch_stream<4, true>(p, s);
    return per <= 16 ? launch_stream<1, false>(p, s) : per <= 32 ? launch_stream<2, false>(p, s) : launch_stream<4, false>(p, s);
}

hipError_t launch_combine_rows(const CombineArgs &a, hipStream_t s) {
    if (a.T <= 0) return hipSuccess;
    return a.y_type == EF_BF16 ? launch_combine_y<EF_BF16>(a, s) : a.y_type == EF_F16 ? launch_combine_y<EF_F16>(a, s)
                                                                                      : launch_combine_y<EF_F32>(a, s);
}

}  // namespace ef

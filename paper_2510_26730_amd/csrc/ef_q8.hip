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

// A workgroup takes a row.  First pass: the largest magnitude (as bits, which order magnitudes and put infinities and NaN on
// top); second: codes.
template <int TYPE>
__global__ __launch_bounds__(256) void quant_rows_kernel(QuantArgs a) {
    using T = typename Element<TYPE>::T;
    __shared__ uint32_t wave_most[4];
    const int row = blockIdx.x, tid = threadIdx.x;
    const T *x = static_cast<const T *>(a.x) + (size_t)row * a.ldx;
    int8_t *out = a.codes + (size_t)row * a.ldc;
    uint32_t most = 0;
    for (int i = tid; i < a.K; i += 256) most = max(most, __builtin_bit_cast(uint32_t, to_float<TYPE>(x[i])) & 0x7FFFFFFFu);
    for (int off = 32; off >= 1; off >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off));
    if ((tid & 63) == 0) wave_most[tid >> 6] = most;
    __syncthreads();
    most = max(max(wave_most[0], wave_most[1]), max(wave_most[2], wave_most[3]));
    const bool bad = most >= 0x7F800000u;
    const float s = fmaxf(__builtin_bit_cast(float, most) / 127.f, 0x1p-126f), inv = 1.f / s;
    if (tid == 0) a.scales[row] = bad ? __builtin_nanf("") : s;
    const int padded = (int)min((long long)(a.K + 63) / 64 * 64, a.ldc);
    for (int i = tid; i < padded; i += 256) out[i] = i < a.K && !bad ? (int8_t)quant_code(to_float<TYPE>(x[i]), s, inv) : 0;
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

hipError_t launch_quant_rows(const QuantArgs &a, hipStream_t s) {
    if (a.rows <= 0) return hipSuccess;
    const dim3 grid(a.rows), block(256);
    switch (a.type) {
        case EF_I8: hipLaunchKernelGGL(pad_rows_kernel, grid, block, 0, s, a); break;
        case EF_BF16: hipLaunchKernelGGL(quant_rows_kernel<EF_BF16>, grid, block, 0, s, a); break;
        case EF_F16: hipLaunchKernelGGL(quant_rows_kernel<EF_F16>, grid, block, 0, s, a); break;
        default: hipLaunchKernelGGL(quant_rows_kernel<EF_F32>, grid, block, 0, s, a); break;
    }
    return hipGetLastError();
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

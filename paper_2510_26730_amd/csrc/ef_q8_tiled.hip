// Products of 8-bit codes, tiled: many rows per matrix, bound by the matrix cores.
//
// A workgroup of four waves owns 64*RA matrix rows (output columns) x 64*RB product rows, a wave a quarter of it: RA x RB
// accumulators of v_mfma_i32_32x32x32_i8, 32-bit whole numbers.  Both operands come row by row as the caller has them, so the rows
// of `a` are gathered by the routing for free: direct global -> LDS loads of 16 rows x 64 bytes (a wave's 64 lanes x 16 bytes, a
// "slab") fill a ring of four stages of 64 codes of K, three ahead of the one that feeds the matrix cores, one barrier per stage.
// Rows of 64 bytes would put every second row of an operand read into the same LDS banks, so lane 4r + p of a load fetches chunk
// p ^ fold(r) of its row instead of p: the 16-byte chunks of a slab lie permuted within their row, and a read of 32 rows at one
// chunk touches all banks evenly.
// The results go through LDS on their way out, so that a wave stores whole runs of a row.
// What it measured: 8192 x 4096 x 14336 in tiles of 256 x 256 444-509 us, 1.9-2.17 POP/s; the same kernel without its loads took 82 % of
// that, with its matrix products alone 63 %.  1056 tokens x 6 of 64 experts, 1408 -> 2048, in tiles of 128 x 128: 67 us.
#include "ef_device.h"
#include "ef_kernels.h"
#include "ef_ops.h"
#include "ef_q8.h"

namespace ef {

namespace {

typedef int int16v __attribute__((ext_vector_type(16)));

constexpr int kStages = 4;
constexpr int wait_vm(int n) { return ((n >> 4) << 14) | (0x7 << 4) | (0xF << 8) | (n & 15); }   // s_waitcnt vmcnt(n) alone
__device__ __forceinline__ int fold(int r) { return (r >> 1 ^ r >> 3) & 3; }

// 64 lanes x 16 bytes straight into LDS at a wave-uniform byte offset; in inline assembly so that the compiler neither moves it
// against the LDS reads nor waits for it: every wait for these loads is an explicit vmcnt
#define EF_Q8_DMA(gptr, lds_off) \
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(gptr), "s"(lds_off) : "memory")

// After matrix product m of a K step: which operand reads (of 8 / 4, in the order a0 b0 a1 b1 ..) and which loads go out there.
// 16 products: reads in the first ten slots, so the next step never waits; loads evenly, because a burst stalls at the issue.
template <int RA, int RB> struct Slots;
template <> struct Slots<4, 4> {
    static constexpr int read(int m) { constexpr int r[16] = {0, 1, -1, 2, 3, 4, -1, 5, 6, 7, -1, -1, -1, -1, -1, -1}; return r[m]; }
    static constexpr int load(int m) { return m % 4 == 2 ? m / 4 : -1; }
};
template <> struct Slots<2, 2> {
    static constexpr int read(int m) { return m; }
    static constexpr int load(int m) { return m % 2 == 0 ? m / 2 : -1; }
};

template <int I, int N, class F>
__device__ __forceinline__ void static_for(F &&f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<I + 1, N>(f);
    }
}

template <int RA, int RB, bool PAIR>
__global__ __launch_bounds__(256, RA *RB >= 16 ? 1 : 2) void q8_tiled_kernel(Q8Args p, int npanels) {
    static_assert(RA == RB, "reads alternate between the operands");
    constexpr int kSlabs = 4 * (RA + RB), kStageBytes = kSlabs * 1024, kLoads = RA + RB;
    __shared__ __attribute__((aligned(16))) char lds[kStages * kStageBytes];
    __shared__ __attribute__((aligned(16))) float wscale[64 * RA], xscale[64 * RB];   // of the rows in the order of their slabs
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wf = wave & 1, wt = wave >> 1;

    Q8Tile t;
    int panel;
    if (!q8_find_unit(p, blockIdx.x, npanels, 64 * RB, t, panel)) return;
    const int F = p.N >> 1, n_end = PAIR ? F : p.N;
    const int n0 = panel * (PAIR ? 32 * RA : 64 * RA);
    const int nstage = (p.K + 63) >> 6;

    // this lane's rows; columns past the end and rows past the group's read a neighbour's codes, their results are dropped
    const int8_t *wsrc[RA], *xsrc[RB];
#pragma unroll
    for (int q = 0; q < RA; ++q) {
        const int local = (q * 4 + wave) * 16 + (lane >> 2), i = local & 31, ab = local >> 5;
        const int row = PAIR ? (ab & 1) * F + min(n0 + (ab >> 1) * 32 + i, F - 1) : min(n0 + local, p.N - 1);
        wsrc[q] = p.w + (size_t)t.group * p.w_group + (size_t)row * p.ldw;
    }
#pragma unroll
    for (int q = 0; q < RB; ++q) {
        const int local = (q * 4 + wave) * 16 + (lane >> 2);
        xsrc[q] = p.a + (size_t)q8_row(p, min(t.row0 + local, t.row_end - 1)).row * p.lda;
    }
    const int chunk = ((lane & 3) ^ fold(lane >> 2)) * 16;
    const int k_last = ((p.K + 15) & ~15) - 16;   // last 16 codes that a weight row holds; beyond K the rows of `a` are zero
    const unsigned lds_base = (unsigned)(size_t)&lds[0];
    // load `q` of stage `st` (past the end the last stage again, in bounds): waits count loads, so every wave issues all of them
    const auto load = [&](int st, auto q) {
        constexpr int n = decltype(q)::value;
        const int k = min(st, nstage - 1) * 64 + chunk;
        const int8_t *from = n < RA ? wsrc[n < RA ? n : 0] + min(k, k_last) : xsrc[n < RA ? 0 : n - RA] + k;
        const unsigned to = lds_base + (st & (kStages - 1)) * kStageBytes + (n < RA ? n * 4 : 4 * RA + (n - RA) * 4) * 1024 + wave * 1024;
        EF_Q8_DMA(from, to);
    };
    // operand fragment `blk` of 32 rows, K step ks of a stage: row i of the fragment, 16 bytes at 32 ks + 16 (lane / 32)
    const int i = lane & 31, row_at = (i >> 4) * 1024 + (i & 15) * 64;
    const int at0 = row_at + (((lane >> 5) ^ fold(i & 15)) << 4), at1 = at0 ^ 32;
    const int abase = wf * RA * 2048, bbase = (4 * RA + wt * RB * 2) * 1024;
    const auto frag = [&](int st, int ks, int base, int blk) {
        return *reinterpret_cast<const int4v *>(lds + (st & (kStages - 1)) * kStageBytes + base + blk * 2048 + (ks ? at1 : at0));
    };

    int16v acc[RA][RB];
#pragma unroll
    for (int x = 0; x < RA; ++x)
#pragma unroll
        for (int y = 0; y < RB; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[x][y][v] = 0;
    int4v a0[RA], b0[RB], a1[RA], b1[RB];

    // scales ahead of the first loads: what waits for them is the waits' first round at most
    for (int r = tid; r < 64 * RA; r += 256) {
        const int i = r & 31, ab = r >> 5;
        wscale[r] = p.w_scale[(size_t)t.group * p.N + (PAIR ? (ab & 1) * F + min(n0 + (ab >> 1) * 32 + i, F - 1) : min(n0 + r, p.N - 1))];
    }
    for (int r = tid; r < 64 * RB; r += 256) xscale[r] = q8_row(p, min(t.row0 + r, t.row_end - 1)).scale;
    static_for<0, kStages - 1>([&](auto st) { static_for<0, kLoads>([&](auto q) { load(decltype(st)::value, q); }); });
    __builtin_amdgcn_s_waitcnt(wait_vm(kLoads * (kStages - 2)));   // my part of stage 0 has landed
    __syncthreads();
#pragma unroll
    for (int x = 0; x < RA; ++x) a0[x] = frag(0, 0, abase, x);
#pragma unroll
    for (int y = 0; y < RB; ++y) b0[y] = frag(0, 0, bbase, y);

    // one K step: the products of (ac, bc), the reads of the next step's (an, bn), half of the loads of stage `ld`.  Only the
    // first `LIVE` of the wave's row tiles exist; the products of the others are left out (power is what limits a full chip).
    const auto step = [&](auto LIVE, int4v(&ac)[RA], int4v(&bc)[RB], int4v(&an)[RA], int4v(&bn)[RB], int rd, int rks, int ld, auto half) {
        constexpr int live = decltype(LIVE)::value;
        static_for<0, RA * RB>([&](auto M) {
            constexpr int m = decltype(M)::value, x = m / RB, y = m % RB, r = Slots<RA, RB>::read(m), l = Slots<RA, RB>::load(m);
            if constexpr (y < live) acc[x][y] = __builtin_amdgcn_mfma_i32_32x32x32_i8(ac[x], bc[y], acc[x][y], 0, 0, 0);
            if constexpr (r >= 0 && r % 2 == 0) an[r / 2] = frag(rd, rks, abase, r / 2);
            if constexpr (r >= 0 && r % 2 == 1 && r / 2 < live) bn[r / 2] = frag(rd, rks, bbase, r / 2);
            if constexpr (l >= 0) load(ld, std::integral_constant<int, decltype(half)::value * (kLoads / 2) + l>{});
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    const auto loop = [&](auto LIVE) {
        for (int st = 0; st < nstage; ++st) {
            // the buffer of stage st+3 held stage st-1, whose last reads every wave finished before the previous barrier
            step(LIVE, a0, b0, a1, b1, st, 1, st + kStages - 1, std::integral_constant<int, 0>{});
            __builtin_amdgcn_s_waitcnt(wait_vm(kLoads * (kStages - 3) + kLoads / 2));   // stage st+1 has landed
            __syncthreads();
            __builtin_amdgcn_sched_barrier(0);
            step(LIVE, a1, b1, a0, b0, st + 1, 0, st + kStages - 1, std::integral_constant<int, 1>{});
        }
    };
    const int live = max(0, min(RB, (t.row_end - t.row0 - wt * 32 * RB + 31) / 32));
    if (live == RB) loop(std::integral_constant<int, RB>{});
    else if (RB > 3 && live == 3) loop(std::integral_constant<int, (RB > 3 ? 3 : 1)>{});
    else if (RB > 2 && live == 2) loop(std::integral_constant<int, (RB > 2 ? 2 : 1)>{});
    else if (live == 1) loop(std::integral_constant<int, 1>{});
    else loop(std::integral_constant<int, 0>{});
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();

    // Lane 32g + i holds product row i of its tile, columns 8q + 4g .. +3 of each fragment.  Tile by tile through this wave's
    // share of the ring: 16 bytes per lane back, neighbouring lanes neighbouring pieces of a row.
    constexpr int kCols = PAIR ? 16 * RA : 32 * RA;        // output columns of the wave
    const int g = lane >> 5, col0 = n0 + wf * kCols;
    float sc[RA][16];
#pragma unroll
    for (int x = 0; x < RA; ++x)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float4 f = *reinterpret_cast<const float4 *>(&wscale[(wf * RA + x) * 32 + 8 * q + 4 * g]);
            sc[x][4 * q] = f.x, sc[x][4 * q + 1] = f.y, sc[x][4 * q + 2] = f.z, sc[x][4 * q + 3] = f.w;
        }
    char *mine = lds + wave * (kStages * kStageBytes / 4);
    static_assert(32 * (kCols * 4 + 16) <= kStages * kStageBytes / 4, "a tile of results fits a wave's share of the ring");
    // Returns whether a result needs CAREFUL, the forms for gates and row scales that the plain ones are not right for
    const auto leave = [&](auto TYPE, auto CAREFUL) {
        constexpr bool careful = decltype(CAREFUL)::value;
        float lowest = 0.f, largest = 0.f;
        constexpr int type = decltype(TYPE)::value, size = type == EF_F32 ? 4 : 2, pitch = kCols * size + 16;
        constexpr int kPieces = kCols * size / 16, kTurns = 32 * kPieces / 64;    // 16-byte pieces of a row; of a tile, for each lane
        const bool whole = ((reinterpret_cast<size_t>(p.out) | (size_t)p.ldo * size) & 15) == 0 && (col0 * size & 15) == 0 && col0 + kCols <= n_end;
#pragma unroll
        for (int y = 0; y < RB; ++y) {
            const int row0 = t.row0 + (wt * RB + y) * 32;
            if (row0 >= t.row_end) break;
            const float xs = xscale[(wt * RB + y) * 32 + i];
            largest = fmaxf(largest, xs);
            const auto value = [&](int sum, float channel) { return careful ? q8_value(sum, q8_scale(xs), channel) : (float)sum * xs * channel; };
#pragma unroll
            for (int x = 0; x < RA; x += PAIR ? 2 : 1)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[e] = value(acc[x][y][4 * q + e], sc[x][4 * q + e]);
                        if constexpr (PAIR) {
                            const float u = value(acc[x + 1][y][4 * q + e], sc[x + 1][4 * q + e]);
                            lowest = fminf(lowest, v[e]);
                            v[e] = careful ? q8_silu_mul_deep(v[e], u) : silu_mul(v[e], u);
                        }
                    }
                    q8_put4<type>(mine + i * pitch, (PAIR ? x / 2 : x) * 32 + 8 * q + 4 * g, v);
                }
            wave_lds_sync();
            const int rows = min(32, t.row_end - row0);
            char *to = static_cast<char *>(p.out) + ((size_t)row0 * p.ldo + col0) * size;
            if (whole) {
                const int r0 = lane / kPieces, piece = (lane & (kPieces - 1)) * 16;
                const char *from = mine + r0 * pitch + piece;
                to += (size_t)r0 * p.ldo * size + piece;
                const size_t hop = (size_t)p.ldo * (size * 64 / kPieces);      // 64 / kPieces rows further on
                uint4 v[kTurns];
#pragma unroll
                for (int z = 0; z < kTurns; ++z) v[z] = *reinterpret_cast<const uint4 *>(from + z * (64 / kPieces) * pitch);
#pragma unroll
                for (int z = 0; z < kTurns; ++z, to += hop)
                    if (r0 + z * (64 / kPieces) < rows) *reinterpret_cast<uint4 *>(to) = v[z];
            } else {      // an element per lane: rows that start anywhere, the last columns
                using T = std::conditional_t<type == EF_F32, float, uint16_t>;
                const int cols = min(kCols, n_end - col0);
                for (int r = 0; r < rows; r += 8)
#pragma unroll
                    for (int c = lane; c < kCols; c += 64) {
                        T v[8];
#pragma unroll
                        for (int q = 0; q < 8; ++q) v[q] = reinterpret_cast<const T *>(mine + (r + q) * pitch)[c];
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            if (c < cols && r + q < rows) reinterpret_cast<T *>(to)[(size_t)(r + q) * p.ldo + c] = v[q];
                    }
            }
            wave_lds_sync();
        }
        return largest >= kLargeScale || lowest < kDeepGate;
    };
    // once more where needed; a branch for every four gates or a third factor on every sum cost the large products up to 3 %
    q8_by_type(p.out_type, [&](auto TYPE) {
        if (__any(leave(TYPE, std::false_type{}))) leave(TYPE, std::true_type{});
    });
}

template <int R, bool PAIR>
hipError_t launch(const Q8Args &p, hipStream_t s) {
    const int cols = PAIR ? p.N / 2 : p.N, per = PAIR ? 32 * R : 64 * R, npanels = (cols + per - 1) / per;
    const long long units = (long long)q8_tiles_bound(p, 64 * R) * npanels;
    if (units > 0x7FFFFFF0ll) return hipErrorInvalidValue;
    hipLaunchKernelGGL((q8_tiled_kernel<R, R, PAIR>), dim3((unsigned)((units + 7) / 8 * 8)), dim3(256), 0, s, p, npanels);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_q8_tiled(const Q8Args &p, bool wide, hipStream_t s) {
    if (p.swiglu) return wide ? launch<4, true>(p, s) : launch<2, true>(p, s);
    return wide ? launch<4, false>(p, s) : launch<2, false>(p, s);
}

}  // namespace ef

// Products of 8-bit codes, panels: one tile of 64 product rows x 128 matrix rows per workgroup, for products whose larger tiles would
// leave compute units idle; bound by what a step's reads, moves between lanes and matrix products take one after another.
//
// Four waves share the 64 product rows and have 32 matrix rows each (swiglu: 16 gate, 16 up), in steps of 256 codes.  A weight is
// needed by one wave only, so it goes from memory straight into that wave's operand registers; the tokens are needed by all four and
// come through LDS by direct loads; both are requested D steps ahead (more gained nothing).  At most one panel per compute unit: two
// teams of four waves take half of K each, one's products beside the other's waits, and add their sums in LDS.
// 517 x 5640 x 2049, 153 panels: 26.5 us, 33.4 with one team (37-42 in tiles of 128 x 128, 81 in tiles of 256 x 256); its rows are not
// aligned to 64 bytes, and a compute unit's address unit then takes a lane at a time, not four.
// A slab of 1 KiB of LDS is 8 rows x 128 codes; lane 8r + p of a load fetches chunk p ^ r, so that 16 rows at one chunk are read from
// all banks evenly.
#include "ef_device.h"
#include "ef_kernels.h"
#include "ef_ops.h"
#include "ef_q8.h"

namespace ef {

namespace {

constexpr int RA = 2, RB = 4;        // blocks of 16 matrix rows of a wave, of 16 product rows
constexpr int D = 2;                 // steps on their way

template <bool PAIR, int KS>
__global__ __launch_bounds__(256 * KS) void q8_panel_kernel(Q8Args p, int npanels) {
    constexpr int kStage = RB * 4096, kBuffers = D + 1, kLoads = RB + 4 * RA;   // loads of a step and wave
    __shared__ __attribute__((aligned(16))) char lds[KS * kBuffers * kStage];
    __shared__ __attribute__((aligned(16))) float wscale[64 * RA], xscale[16 * RB];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6 & 3), team = __builtin_amdgcn_readfirstlane(tid >> 8);
    Q8Tile t;
    int panel;
    if (!q8_find_unit(p, blockIdx.x, npanels, 16 * RB, t, panel)) return;
    const int F = p.N >> 1, n_end = PAIR ? F : p.N;
    const int n0 = panel * (PAIR ? 32 * RA : 64 * RA), col0 = n0 + wave * (PAIR ? 8 * RA : 16 * RA);
    const int i = lane & 15, g = lane >> 4;
    const int steps = ((p.K + kStep - 1) / kStep + KS - 1) / KS, first = team * steps, end = first + steps;   // of this team; past K they add nothing
    // matrix row behind row r (0..15) of the wave's block b; columns past the end read a neighbour's codes, their results are dropped
    const auto matrix_row = [&](int first, int b, int r) {
        if constexpr (PAIR) return (b < RA / 2 ? 0 : F) + min(first + (b % (RA / 2)) * 16 + r, F - 1);
        else return min(first + b * 16 + r, p.N - 1);
    };

    const int8_t *w = p.w + (size_t)t.group * p.w_group;
    unsigned woff[RA][4];
#pragma unroll
    for (int b = 0; b < RA; ++b)
#pragma unroll
        for (int h = 0; h < 4; ++h) woff[b][h] = (unsigned)matrix_row(col0, b, quad_row(lane, h)) * (unsigned)p.ldw;
    const int k_last = ((p.K + 15) & ~15) - 16, x_last = ((p.K + 63) & ~63) - 16;
    int4v wb[D][RA][4];
    const auto fetch_w = [&](int u, int s) {
        const unsigned k = min(min(s, end - 1) * kStep + quad_code(lane), k_last);
#pragma unroll
        for (int b = 0; b < RA; ++b)
#pragma unroll
            for (int h = 0; h < 4; ++h) wb[u][b][h] = load16(w + (woff[b][h] + k));
    };

    // slabs 2r and 2r + 1 hold the halves of a step of rows 8r .. 8r+7
    const int8_t *xsrc[RB];
#pragma unroll
    for (int q = 0; q < RB; ++q) xsrc[q] = p.a + (size_t)q8_row(p, min(t.row0 + (q * 2 + (wave >> 1)) * 8 + (lane >> 3), t.row_end - 1)).row * p.lda;
    char *ring = lds + team * kBuffers * kStage;
    const unsigned lds_base = (unsigned)(size_t)ring;
    const int xchunk = (wave & 1) * 128 + ((lane & 7) ^ (lane >> 3)) * 16;
    const auto load_x = [&](int buf, int s) {
#pragma unroll
        for (int q = 0; q < RB; ++q) {
            const int8_t *from = xsrc[q] + min(min(s, end - 1) * kStep + xchunk, x_last);
            const unsigned to = __builtin_amdgcn_readfirstlane(lds_base + buf * kStage + (q * 4 + wave) * 1024);
            asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "memory");
        }
    };
    // in the order of the loop, whose waits count on it
#pragma unroll
    for (int u = 0; u < D; ++u) {
        load_x(u, first + u);
        __builtin_amdgcn_sched_barrier(0);
        fetch_w(u, first + u);
        __builtin_amdgcn_sched_barrier(0);
    }
    for (int r = tid; r < 64 * RA; r += 256 * KS)
        wscale[r] = p.w_scale[(size_t)t.group * p.N + matrix_row(n0 + (r / (16 * RA)) * (PAIR ? 8 * RA : 16 * RA), (r / 16) % RA, r & 15)];
    for (int r = tid; r < 16 * RB; r += 256 * KS) xscale[r] = q8_row(p, min(t.row0 + r, t.row_end - 1)).scale;

    int4v acc[RA][RB];
#pragma unroll
    for (int b = 0; b < RA; ++b)
#pragma unroll
        for (int j = 0; j < RB; ++j) acc[b][j] = int4v{0, 0, 0, 0};
    const int row_at = (i >> 3) * 2048 + (g >> 1) * 1024 + (i & 7) * 128, chunk0 = 4 * (g & 1);
    // the products of step s, weights in wb[u], tokens in LDS buffer `buf`
    const auto multiply = [&](int u, int buf, int s) {
#pragma unroll
        for (int b = 0; b < RA; ++b) {
            transpose_quads(wb[u][b], lane);
            if (s * kStep + 64 * g > x_last)   // past the tokens' end
#pragma unroll
                for (int y = 0; y < 4; ++y) wb[u][b][y] = int4v{0, 0, 0, 0};
        }
        const char *from = ring + buf * kStage;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int at = row_at + (((chunk0 + y) ^ (i & 7)) << 4);
            int4v x[RB];
#pragma unroll
            for (int j = 0; j < RB; ++j) x[j] = *reinterpret_cast<const int4v *>(from + j * 4096 + at);
#pragma unroll
            for (int j = 0; j < RB; ++j)
#pragma unroll
                for (int b = 0; b < RA; ++b) acc[b][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wb[u][b][y], x[j], acc[b][j], 0, 0, 0);
        }
    };
    // Step s waits for its own tokens alone: its weights, and tokens and weights of the D - 1 steps behind it, may be on their way.  The
    // compiler waits for the weights; it does not know of the loads into LDS between them, so it waits for somewhat more than it
    // needs to.  Requests past the end repeat the last step; what is left then runs without requests.
    int s = first, buf = 0;
    const auto next = [&](int b) { return b + 1 == kBuffers ? 0 : b + 1; };
    for (; s + D < end; s += D) {
#pragma unroll
        for (int u = 0; u < D; ++u) {
            constexpr int behind = 4 * RA + (D - 1) * kLoads;
            static_assert(behind < 64, "vmcnt is a 6-bit counter");
            __builtin_amdgcn_s_waitcnt((behind >> 4) << 14 | 0x0F70 | (behind & 15));
            __syncthreads();            // everybody's part has landed, and nobody reads the buffer of step s + u - 1 any more
            load_x(buf == 0 ? kBuffers - 1 : buf - 1, s + u + D);
            __builtin_amdgcn_sched_barrier(0);
            multiply(u, buf, s + u);
            __builtin_amdgcn_sched_barrier(0);
            fetch_w(u, s + u + D);
            __builtin_amdgcn_sched_barrier(0);
            buf = next(buf);
        }
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < D; ++u) {
        if (s + u < end) multiply(u, buf, s + u);
        buf = next(buf);
    }

    // the teams' sums: every team gives away the tiles that the other finishes
    constexpr int kOwn = RB / KS;
    if constexpr (KS == 2) {
        static_assert(4 * RA * RB / 2 * 1024 * KS <= sizeof(lds), "the sums fit the ring");
        int4v *away = reinterpret_cast<int4v *>(lds) + wave * 64 + lane;
        __syncthreads();
#pragma unroll
        for (int b = 0; b < RA; ++b)
#pragma unroll
            for (int j = 0; j < kOwn; ++j) away[((team * RA + b) * kOwn + j) * 256] = team ? acc[b][j] : acc[b][kOwn + j];
        __syncthreads();
#pragma unroll
        for (int b = 0; b < RA; ++b)
#pragma unroll
            for (int j = 0; j < kOwn; ++j) acc[b][j] = (team ? acc[b][kOwn + j] : acc[b][j]) + away[(((team ^ 1) * RA + b) * kOwn + j) * 256];
    }
    // lane 16g + i holds product row i of its tile, matrix rows 4g .. 4g+3 of each block
    const float *sc = wscale + wave * 16 * RA + 4 * g;
    q8_by_type(p.out_type, [&](auto TYPE) {
#pragma unroll
        for (int j = 0; j < kOwn; ++j) {
            const int tile = team * kOwn + j, row = t.row0 + 16 * tile + i;
            const Q8Scale xs = q8_scale(xscale[16 * tile + i]);
            if (row >= t.row_end) continue;
#pragma unroll
            for (int b = 0; b < (PAIR ? RA / 2 : RA); ++b) {
                float v[4], up[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = q8_value(acc[b][j][e], xs, sc[16 * b + e]);
                    if constexpr (PAIR) up[e] = q8_value(acc[b + RA / 2][j][e], xs, sc[16 * (b + RA / 2) + e]);
                }
                if constexpr (PAIR) q8_silu_mul4(v, up);
                q8_store4<decltype(TYPE)::value>(p, row, col0 + 16 * b + 4 * g, n_end, v);
            }
        }
    });
}

template <bool PAIR>
hipError_t launch(const Q8Args &p, hipStream_t s) {
    const int cols = PAIR ? p.N / 2 : p.N, per = PAIR ? 32 * RA : 64 * RA, npanels = (cols + per - 1) / per;
    const long long units = (long long)q8_tiles_bound(p, 16 * RB) * npanels;
    if (units > 0x7FFFFFF0ll || !q8_panel_ok(p)) return hipErrorInvalidValue;
    const dim3 grid((unsigned)((units + 7) / 8 * 8));
    if (units <= 256) hipLaunchKernelGGL((q8_panel_kernel<PAIR, 2>), grid, dim3(512), 0, s, p, npanels);
    else hipLaunchKernelGGL((q8_panel_kernel<PAIR, 1>), grid, dim3(256), 0, s, p, npanels);
    return hipGetLastError();
}

}  // namespace

bool q8_panel_ok(const Q8Args &p) { return (long long)p.N * p.ldw < 0x7FFFFFFFll; }      // offsets within a matrix in 32 bits

hipError_t launch_q8_panel(const Q8Args &p, hipStream_t s) { return p.swiglu ? launch<true>(p, s) : launch<false>(p, s); }

}  // namespace ef

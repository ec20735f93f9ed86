// Routing from logits: scores, balance bias, groups of experts, top-k, weights, and the stable grouping of the assignments.
//
// A wave takes one token: expert e sits in lane e % 64, register e / 64.  The choice values c become whole numbers of the same
// order ("keys": a float's bits, negative ones inverted), so a maximum over the wave is six DPP steps on 32-bit numbers.  Top-k
// is k such maxima; the lowest expert with the maximum's key is found by ballots, so ties need no second key.
// Without a bias (and without sums of two) the order of the logits is the order of the scores, and the logits themselves are
// compared, exactly.  Otherwise c is formed in 32 bits, where it is off by up to ~1e-6 of the largest score and of the bias; a
// token whose border (the last chosen against the best left out, of experts or of groups) is closer than that is decided again in
// 64 bits: with 256 experts one token in some thousands, where forming every score in 64 bits would cost more than the logits' bytes.
//
// Grouping: a workgroup takes one tile of 16 or 64 tokens, and every expert has a bit per token of the tile in LDS.  The bits
// below a token's own are its rank among the tile's assignments to that expert, their number the tile's count.  One tile:
// everything in one launch.  Otherwise the counts' prefixes over the tiles, a wave per expert, and a scatter, a tile per workgroup.
#include "ef_device.h"
#include "ef_ops.h"

namespace ef {

hipError_t launch_fill_i32(int32_t *p, int n, int32_t v, hipStream_t s);

namespace {

// DPP moves within a wave; lanes without a source get 0
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint32_t dpp0(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
constexpr int kShr1 = 0x111, kShr2 = 0x112, kShr4 = 0x114, kShr8 = 0x118, kBcast15 = 0x142, kBcast31 = 0x143;

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    x = max(x, dpp0<kShr1>(x));
    x = max(x, dpp0<kShr2>(x));
    x = max(x, dpp0<kShr4>(x));
    x = max(x, dpp0<kShr8>(x));
    x = max(x, dpp0<kBcast15>(x));
    x = max(x, dpp0<kBcast31>(x));
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ __forceinline__ uint64_t wave_max(uint64_t x) {
    const uint32_t hi = wave_max((uint32_t)(x >> 32));
    const uint32_t lo = wave_max((uint32_t)(x >> 32) == hi ? (uint32_t)x : 0u);
    return (uint64_t)hi << 32 | lo;
}
// sum over the wave in a fixed order
__device__ __forceinline__ float wave_sum(float x) {
    const auto add = [](float v, uint32_t o) { return v + __builtin_bit_cast(float, o); };
    x = add(x, dpp0<kShr1>(__builtin_bit_cast(uint32_t, x)));
    x = add(x, dpp0<kShr2>(__builtin_bit_cast(uint32_t, x)));
    x = add(x, dpp0<kShr4>(__builtin_bit_cast(uint32_t, x)));
    x = add(x, dpp0<kShr8>(__builtin_bit_cast(uint32_t, x)));
    x = add(x, dpp0<kBcast15, 0xa>(__builtin_bit_cast(uint32_t, x)));
    x = add(x, dpp0<kBcast31, 0xc>(__builtin_bit_cast(uint32_t, x)));
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ __forceinline__ double wave_sum(double x) {
    for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off);
    return x;
}
__device__ __forceinline__ float lane_value(float x, int lane) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}
__device__ __forceinline__ double lane_value(double x, int lane) {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// whole numbers in the order of the values (no NaN); 0 lies below every one of them
__device__ __forceinline__ uint32_t key_of(float f) {
    const uint32_t u = __builtin_bit_cast(uint32_t, f);
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __builtin_bit_cast(float, k >> 31 ? k & 0x7FFFFFFFu : ~k); }
__device__ __forceinline__ uint64_t key_of(double f) {
    const uint64_t u = __builtin_bit_cast(uint64_t, f);
    return u >> 63 ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ double of_key(uint64_t k) {
    return __builtin_bit_cast(double, k >> 63 ? k & 0x7FFFFFFFFFFFFFFFull : ~k);
}

__device__ __forceinline__ float load_element(const void *p, int type, size_t i) {
    if (type == EF_F32) return static_cast<const float *>(p)[i];
    const uint16_t b = static_cast<const uint16_t *>(p)[i];
    return type == EF_BF16 ? __builtin_bit_cast(float, (uint32_t)b << 16) : (float)__builtin_bit_cast(_Float16, b);
}

constexpr float kMinusInf = -__builtin_inff();

struct Groups {
    int n, size, kept, best;
    int lanes;             // lanes that share a group (a power of two, lanes * n <= 64)
};

// Chooses a token's experts by their choice values c (expert r*64 + lane; `mine`: bits of the registers that hold an expert).
// Returns the bits of the lane's chosen registers; `near`: a border is closer than `margin`.  cl: this wave's LDS, for the groups.
template <int R, class V>
__device__ __forceinline__ uint32_t choose(const V (&c)[R], uint32_t mine, int k, const Groups &g, V *cl, V margin, bool &near) {
    const int lane = threadIdx.x & 63;
    uint32_t live = mine;
    near = false;
    if (g.n > 1) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (mine >> r & 1) cl[r * 64 + lane] = c[r];
        wave_lds_sync();
        const int grp = lane / g.lanes, q = lane & (g.lanes - 1);
        V b1 = (V)kMinusInf, b2 = (V)kMinusInf;
        if (grp < g.n)
            for (int x = q; x < g.size; x += g.lanes) {
                const V v = cl[grp * g.size + x];
                b2 = fmax(b2, fmin(b1, v));
                b1 = fmax(b1, v);
            }
        wave_lds_sync();
        for (int off = 1; off < g.lanes; off <<= 1) {
            const V o1 = __shfl_xor(b1, off), o2 = __shfl_xor(b2, off);
            b2 = fmax(fmin(b1, o1), fmax(b2, o2));
            b1 = fmax(b1, o1);
        }
        const V v = g.best == 1 ? b1 : b2 == (V)kMinusInf ? b2 : b1 + b2;
        int rank = 0;
        for (int o = 0; o < g.n; ++o) {
            const V ov = lane_value(v, o * g.lanes);
            rank += ov > v || (ov == v && o < grp);
        }
        const bool leads = q == 0 && grp < g.n;
        const unsigned long long kept = __ballot(leads && rank < g.kept);
        if (g.kept < g.n) {
            const unsigned long long last = __ballot(leads && rank == g.kept - 1), next = __ballot(leads && rank == g.kept);
            near = lane_value(v, __builtin_ctzll(last)) - lane_value(v, __builtin_ctzll(next)) <= margin;
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (mine >> r & 1 && !(kept >> ((r * 64 + lane) / g.size * g.lanes) & 1)) live &= ~(1u << r);
    }
    using Key = decltype(key_of(c[0]));
    Key key[R];
#pragma unroll
    for (int r = 0; r < R; ++r) key[r] = live >> r & 1 ? key_of(c[r]) : 0;
    uint32_t chosen = 0;
    Key last = 0;
    for (int j = 0; j < k; ++j) {
        Key m = key[0];
#pragma unroll
        for (int r = 1; r < R; ++r) m = max(m, key[r]);
        last = wave_max(m);
        bool found = false;   // uniform
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const unsigned long long eq = __ballot(!found && key[r] == last);
            if (eq && lane == __builtin_ctzll(eq)) {
                chosen |= 1u << r;
                key[r] = 0;
            }
            found |= eq != 0;
        }
    }
    if (margin >= 0) {   // uniform
        Key m = key[0];
#pragma unroll
        for (int r = 1; r < R; ++r) m = max(m, key[r]);
        const Key next = wave_max(m);
        near |= next != 0 && of_key(last) - of_key(next) <= margin;
    }
    return chosen;
}

// exclusive prefix sum of the experts' counts (register r of a wave: expert r*64 + lane); returns the sum
template <int R>
__device__ __forceinline__ int expert_offsets(const int (&cnt)[R], int (&off)[R]) {
    const int lane = threadIdx.x & 63;
    int before = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        int incl = cnt[r];
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(incl, o);
            if (lane >= o) incl += v;
        }
        off[r] = before + incl - cnt[r];
        before += __shfl(incl, 63);
    }
    return before;
}

template <int TT> struct TileBits { using type = unsigned long long; };
template <> struct TileBits<16> { using type = uint32_t; };

template <int R, int TT>
__global__ __launch_bounds__(64 * kRouterWaves) void router_kernel(RouterArgs a) {
    using Bits = typename TileBits<TT>::type;
    constexpr int kE = 64 * R;
    __shared__ Bits bits[kE];
    __shared__ uint16_t chosen_ids[TT * EF_ROUTER_MAX_TOPK];
    __shared__ int first[kE];
    __shared__ double group_values[kRouterWaves][kE];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int E = a.r.n_experts, k = a.r.top_k;
    const int t0 = blockIdx.x * TT, n = min(TT, a.T - t0);
    for (int e = tid; e < kE; e += 64 * kRouterWaves) bits[e] = 0;
    __syncthreads();

    Groups g{a.r.n_groups, E / a.r.n_groups, a.r.groups_kept, a.r.group_best, 64};
    while (g.lanes * g.n > 64) g.lanes >>= 1;
    const bool softmax = a.r.score == EF_SCORE_SOFTMAX;
    const bool by_logit = !a.bias && (g.n == 1 || g.best == 1);
    uint32_t mine = 0;
    float b[R], bmax = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int e = r * 64 + lane;
        b[r] = 0.f;
        if (e < E) {
            mine |= 1u << r;
            if (a.bias) {
                b[r] = a.bias[e];
                if (b[r] != b[r]) b[r] = kMinusInf;
                if (fabsf(b[r]) < __builtin_inff()) bmax = fmaxf(bmax, fabsf(b[r]));
            }
        }
    }
    if (a.bias) bmax = __builtin_bit_cast(float, wave_max(__builtin_bit_cast(uint32_t, bmax)));

    float zn[R];   // the next token's logits
    const auto fetch = [&](int t) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            zn[r] = mine >> r & 1 ? load_element(a.logits, a.type, (size_t)(t0 + t) * a.ld + r * 64 + lane) : kMinusInf;
    };
    if (wave < n) fetch(wave);
    for (int t = wave; t < n; t += kRouterWaves) {
        float z[R];
#pragma unroll
        for (int r = 0; r < R; ++r) z[r] = zn[r] != zn[r] ? kMinusInf : zn[r] + 0.f;   // -0 and 0 are one value
        if (t + kRouterWaves < n) fetch(t + kRouterWaves);

        // scores in 32 bits
        float s[R], top = 1.f;
        if (softmax) {
            uint32_t mk = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) mk = max(mk, key_of(z[r]));
            const float m = of_key(wave_max(mk));
            float part = 0.f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                s[r] = z[r] == kMinusInf ? 0.f : z[r] == m ? 1.f : expf(z[r] - m);   // m = inf: the others are 0
                part += s[r];
            }
            const float sum = wave_sum(part);
            const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
            for (int r = 0; r < R; ++r) s[r] *= inv;
            top = inv;
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) s[r] = 1.f / (1.f + expf(-z[r]));
        }

        uint32_t chosen;
        bool near;
        if (by_logit) {
            chosen = choose<R, float>(z, mine, k, g, reinterpret_cast<float *>(group_values[wave]), -1.f, near);
        } else {
            float c[R];
#pragma unroll
            for (int r = 0; r < R; ++r) c[r] = z[r] == kMinusInf ? kMinusInf : s[r] + b[r];
            // a choice value is off by at most 1.2e-6 of the largest score and 2^-24 of itself, a sum of two by twice that
            chosen = choose<R, float>(c, mine, k, g, reinterpret_cast<float *>(group_values[wave]), 8e-6f * top + 1e-6f * bmax, near);
            if (near) {
                double d[R];
                if (softmax) {
                    float m = kMinusInf;
#pragma unroll
                    for (int r = 0; r < R; ++r) m = fmaxf(m, z[r]);
                    m = of_key(wave_max(key_of(m)));
                    double part = 0;
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        d[r] = z[r] == kMinusInf ? 0 : z[r] == m ? 1 : exp((double)z[r] - (double)m);
                        part += d[r];
                    }
                    const double sum = wave_sum(part);
#pragma unroll
                    for (int r = 0; r < R; ++r) d[r] = sum > 0 ? d[r] / sum : 0;
                } else {
#pragma unroll
                    for (int r = 0; r < R; ++r) d[r] = 1 / (1 + exp(-(double)z[r]));
                }
#pragma unroll
                for (int r = 0; r < R; ++r) d[r] = z[r] == kMinusInf ? (double)kMinusInf : d[r] + (double)b[r];
                chosen = choose<R, double>(d, mine, k, g, group_values[wave], -1.0, near);
            }
        }

        float part = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) part += chosen >> r & 1 ? s[r] : 0.f;
        const float sum = wave_sum(part);
        int before = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool on = chosen >> r & 1;
            const unsigned long long all = __ballot(on);
            if (on) {
                const int e = r * 64 + lane, j = before + __popcll(all & ((1ull << lane) - 1));
                const size_t at = (size_t)(t0 + t) * k + j;
                const float w = !a.r.renorm ? s[r] : sum > 0.f ? s[r] / sum : 0.f;
                a.ids[at] = e;
                a.w[at] = w * a.r.scale;
                chosen_ids[t * k + j] = (uint16_t)e;
                atomicOr(&bits[e], (Bits)1 << t);
            }
            before += __popcll(all);
        }
    }
    __syncthreads();

    if (a.ntiles > 1) {
        for (int e = tid; e < E; e += 64 * kRouterWaves) a.tile_counts[(size_t)e * a.ntiles + blockIdx.x] = __popcll(bits[e]);
        for (int x = tid; x < n * k; x += 64 * kRouterWaves)
            a.rank[(size_t)t0 * k + x] = (uint8_t)__popcll(bits[chosen_ids[x]] & (((Bits)1 << (x / k)) - 1));
        return;
    }
    if (wave == 0) {
        int cnt[R], off[R];
#pragma unroll
        for (int r = 0; r < R; ++r) cnt[r] = __popcll(bits[r * 64 + lane]);
        const int all = expert_offsets<R>(cnt, off);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int e = r * 64 + lane;
            first[e] = off[r];
            if (e < E) {
                a.counts[e] = cnt[r];
                a.offsets[e] = off[r];
            }
        }
        if (lane == 0) a.offsets[E] = all;
    }
    __syncthreads();
    for (int x = tid; x < n * k; x += 64 * kRouterWaves) {
        const int e = chosen_ids[x];
        const int pos = first[e] + __popcll(bits[e] & (((Bits)1 << (x / k)) - 1));
        a.perm[pos] = x;
        a.inv_perm[x] = pos;
    }
}

// the tiles' counts of an expert -> their exclusive prefix, in place, and the expert's total; a wave per expert
__global__ __launch_bounds__(256) void router_scan_kernel(int32_t *__restrict__ tile_counts, int ntiles, int E, int32_t *__restrict__ counts) {
    const int e = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (e >= E) return;
    int32_t *row = tile_counts + (size_t)e * ntiles;
    int before = 0;
    for (int c0 = 0; c0 < ntiles; c0 += 64) {
        const int v = c0 + lane < ntiles ? row[c0 + lane] : 0;
        int incl = v;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(incl, o);
            if (lane >= o) incl += x;
        }
        if (c0 + lane < ntiles) row[c0 + lane] = before + incl - v;
        before += __shfl(incl, 63);
    }
    if (lane == 0) counts[e] = before;
}

template <int R>
__global__ __launch_bounds__(256) void router_scatter_kernel(RouterArgs a, int tile) {
    __shared__ int first[64 * R];
    const int E = a.r.n_experts, k = a.r.top_k, tid = threadIdx.x, lane = tid & 63;
    if (tid < 64) {
        int cnt[R], off[R];
#pragma unroll
        for (int r = 0; r < R; ++r) cnt[r] = r * 64 + lane < E ? a.counts[r * 64 + lane] : 0;
        const int all = expert_offsets<R>(cnt, off);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int e = r * 64 + lane;
            if (e < E) {
                first[e] = off[r] + a.tile_counts[(size_t)e * a.ntiles + blockIdx.x];
                if (blockIdx.x == 0) a.offsets[e] = off[r];
            }
        }
        if (blockIdx.x == 0 && lane == 0) a.offsets[E] = all;
    }
    __syncthreads();
    const size_t a0 = (size_t)blockIdx.x * tile * k;
    const int n = min(tile, a.T - (int)blockIdx.x * tile) * k;
    for (int x = tid; x < n; x += 256) {
        const int pos = first[a.ids[a0 + x]] + a.rank[a0 + x];
        a.perm[pos] = (int)(a0 + x);
        a.inv_perm[a0 + x] = pos;
    }
}

template <int R>
hipError_t launch_r(const RouterArgs &a, hipStream_t s) {
    const int tile = router_tile(a.T);
    if (tile == 16) hipLaunchKernelGGL((router_kernel<R, 16>), dim3(a.ntiles), dim3(64 * kRouterWaves), 0, s, a);
    else hipLaunchKernelGGL((router_kernel<R, 64>), dim3(a.ntiles), dim3(64 * kRouterWaves), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.ntiles == 1) return e;
    hipLaunchKernelGGL(router_scan_kernel, dim3((a.r.n_experts + 3) / 4), dim3(256), 0, s, a.tile_counts, a.ntiles, a.r.n_experts, a.counts);
    hipLaunchKernelGGL(router_scatter_kernel<R>, dim3(a.ntiles), dim3(256), 0, s, a, tile);
    return hipGetLastError();
}

}  // namespace

// up to 64 tokens are one tile (one launch); beyond, tiles of 16 until the grid of 64s fills the chip
int router_tile(int T) { return T > 64 && T <= 8192 ? 16 : 64; }

hipError_t launch_router(const RouterArgs &a, hipStream_t s) {
    const int E = a.r.n_experts;
    if (a.T <= 0) {
        const hipError_t e = launch_fill_i32(a.counts, E, 0, s);
        return e != hipSuccess ? e : launch_fill_i32(a.offsets, E + 1, 0, s);
    }
    if (a.ntiles != (a.T + router_tile(a.T) - 1) / router_tile(a.T)) return hipErrorInvalidValue;
    return E <= 64 ? launch_r<1>(a, s) : E <= 128 ? launch_r<2>(a, s) : E <= 256 ? launch_r<4>(a, s) : launch_r<8>(a, s);
}

}  // namespace ef

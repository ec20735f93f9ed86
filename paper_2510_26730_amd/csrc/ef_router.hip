// Routing from logits: scores, balance bias, groups of experts, top-k, weights, and the stable grouping of the assignments.
//
// A wave takes four tokens, 16 lanes each; lane l of a token holds the experts l*V .. l*V+V-1, V = ceil(E / 16).  A choice value
// becomes a whole number of the same order (a float's bits, negative ones inverted) whose low nine bits are replaced by 511 - e:
// keys are distinct, a maximum names its expert and ties go to the lowest.  Top-k is k rounds of "the largest key below the last
// one": key - last, modulo 2^32, is largest for exactly that key, so nothing has to be removed between rounds, and a round is 1.5
// instructions per key and four DPP steps for four tokens.
// The nine bits, and forming scores in 32 bits (not needed without a bias, where the order of the logits is that of the scores, and
// exact where logits have 16 bits), can hide which of two close values is larger.  That matters at a border only: the last expert
// chosen against the best left out, the last group kept against the best dropped.  A token whose border is closer than the error is
// decided again by the whole wave, from its logits' full bits or from scores in 64 bits ("exact" below): with 256 experts and 32-bit
// logits some tokens in a thousand.  16-bit logits of 256 experts are equal at the border of a top 8 in 9 % (bf16) or 1 % (f16) of normally
// distributed tokens; where scores are compared (a bias, sums of two best) those go the exact way too: 32768 tokens, 8 groups by their two
// best, no bias, 50 us in bf16 and 42 in 32 bits.  More than 16 groups go that way always, and so do groups of more than
// 32 experts a lane.  Groups that do not fill their lanes leave the rest empty: 32768 tokens of 200 experts in 8 groups 42 us, 124 with a
// wave per token.
//
// 32768 tokens of 256 experts (sigmoid, bias, eight groups, top 8) take 32-33 us.  About half of that is the issue of vector instructions:
// 319 per token, 42 thousand cycles of each SIMD, 17.5 us at 2.4 GHz.  A wave spends 31 % of its life issuing, 31 % ready and waiting for
// its turn, 38 % waiting for data, with four waves a SIMD; the rest of the time is a launch's start and end, when SIMDs have fewer.  48
// tokens take 12 us on the one compute unit that keeps their grouping in the launch.
//
// Grouping: a workgroup takes one tile of 16 or 64 tokens, and every expert has a bit per token of the tile in LDS.  The bits
// below a token's own are its rank among the tile's assignments to that expert, their number the tile's count.  One tile:
// everything in one launch.  Otherwise a second launch adds up the tiles' counts, all of them and those before its own tile, in
// every workgroup, and scatters.
#include "ef_device.h"
#include "ef_ops.h"

#include <type_traits>

namespace ef {

hipError_t launch_fill_i32(int32_t *p, int n, int32_t v, hipStream_t s);

namespace {

// DPP moves within a wave; lanes without a source get 0
template <int CTRL>
__device__ __forceinline__ uint32_t dpp0(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false);
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

template <int TYPE, class T>
__device__ __forceinline__ float value_of(T b) {
    if constexpr (TYPE == EF_F32) return b;
    else if constexpr (TYPE == EF_BF16) return __builtin_bit_cast(float, (uint32_t)b << 16);
    else return (float)__builtin_bit_cast(_Float16, b);
}
__device__ __forceinline__ float load_element(const void *p, int type, size_t i) {
    if (type == EF_F32) return static_cast<const float *>(p)[i];
    const uint16_t b = static_cast<const uint16_t *>(p)[i];
    return type == EF_BF16 ? value_of<EF_BF16>(b) : value_of<EF_F16>(b);
}

constexpr float kMinusInf = -__builtin_inff();
// NaN counts as -inf, -0 and 0 are one value
__device__ __forceinline__ float clean(float x) { return x != x ? kMinusInf : x + 0.f; }

// maximum of numbers that are not NaN, without the canonicalising that fmaxf brings
__device__ __forceinline__ float max_of(float x, float y) { return __builtin_amdgcn_fmed3f(x, y, __builtin_inff()); }
__device__ __forceinline__ float min_of(float x, float y) { return __builtin_amdgcn_fmed3f(x, y, -__builtin_inff()); }

// keeps a value out of a branch that the compiler would make of a selection behind it
__device__ __forceinline__ float pinned(float x) {
    asm volatile("" : "+v"(x));
    return x;
}

template <int I, int N, class F>
__device__ __forceinline__ void static_for(F &&f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<I + 1, N>(f);
    }
}

struct Groups {
    int n, size, kept, best;
    int lanes;             // lanes that share a group (a power of two, lanes * n <= 64)
};

// Chooses a token's experts by their choice values c (expert r*64 + lane; `mine`: bits of the registers that hold an expert).
// Returns the bits of the lane's chosen registers.  cl: this wave's LDS, for the groups.
template <int R, class V>
__device__ __forceinline__ uint32_t choose(const V (&c)[R], uint32_t mine, int k, const Groups &g, V *cl) {
    const int lane = threadIdx.x & 63;
    uint32_t live = mine;
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
        const unsigned long long kept = __ballot(q == 0 && grp < g.n && rank < g.kept);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (mine >> r & 1 && !(kept >> ((r * 64 + lane) / g.size * g.lanes) & 1)) live &= ~(1u << r);
    }
    using Key = decltype(key_of(c[0]));
    Key key[R];
#pragma unroll
    for (int r = 0; r < R; ++r) key[r] = live >> r & 1 ? key_of(c[r]) : 0;
    uint32_t chosen = 0;
    for (int j = 0; j < k; ++j) {
        Key m = key[0];
#pragma unroll
        for (int r = 1; r < R; ++r) m = max(m, key[r]);
        m = wave_max(m);
        bool found = false;   // uniform
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const unsigned long long eq = __ballot(!found && key[r] == m);
            if (eq && lane == __builtin_ctzll(eq)) {
                chosen |= 1u << r;
                key[r] = 0;
            }
            found |= eq != 0;
        }
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

// ---- the exact way: a whole wave decides one token; expert r*64 + lane in register r -----------------------------------------

// ids and weights of token t (in the batch; `bit` its number in the tile)
template <int R, class Bits>
__device__ __forceinline__ void exact_token(const RouterArgs &a, size_t t, int bit, const Groups &g, double *cl, uint16_t *chosen_ids, Bits *bits) {
    const int lane = threadIdx.x & 63, E = a.r.n_experts, k = a.r.top_k;
    const bool softmax = a.r.score == EF_SCORE_SOFTMAX;
    float z[R];
    uint32_t mine = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int e = r * 64 + lane;
        z[r] = kMinusInf;
        if (e < E) {
            mine |= 1u << r;
            z[r] = clean(load_element(a.logits, a.type, t * a.ld + e));
        }
    }
    uint32_t mk = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) mk = max(mk, key_of(z[r]));
    const float m = of_key(wave_max(mk));
    uint32_t chosen;
    double total = 0;      // softmax: sum of exp(z - m)
    if (softmax) {
#pragma unroll
        for (int r = 0; r < R; ++r) total += z[r] == kMinusInf ? 0 : z[r] == m ? 1 : exp((double)z[r] - (double)m);
        total = wave_sum(total);
    }
    const auto score = [&](float x) -> double {
        if (!softmax) return 1 / (1 + exp(-(double)x));
        return x == kMinusInf ? 0 : (x == m ? 1 : exp((double)x - (double)m)) / total;   // m = inf: the others are 0
    };
    if (a.bias || (g.n > 1 && g.best == 2)) {
        double c[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const double b = a.bias && mine >> r & 1 ? (double)clean(a.bias[r * 64 + lane]) : 0;
            c[r] = z[r] == kMinusInf ? (double)kMinusInf : score(z[r]) + b;
        }
        chosen = choose<R, double>(c, mine, k, g, cl);
    } else {
        chosen = choose<R, float>(z, mine, k, g, reinterpret_cast<float *>(cl));
    }
    double part = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) part += chosen >> r & 1 ? score(z[r]) : 0;
    const double sum = wave_sum(part);
    int before = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool on = chosen >> r & 1;
        const unsigned long long all = __ballot(on);
        if (on) {
            const int e = r * 64 + lane, j = before + __popcll(all & ((1ull << lane) - 1));
            const double w = score(z[r]);
            a.ids[t * k + j] = e;
            a.w[t * k + j] = (float)(!a.r.renorm ? w : sum > 0 ? w / sum : 0) * a.r.scale;
            chosen_ids[bit * k + j] = (uint16_t)e;
            atomicOr(&bits[e], (Bits)1 << bit);
        }
        before += __popcll(all);
    }
}

// ---- the fast way: four tokens per wave ------------------------------------------------------------------------------------

// moves within 16 lanes in which every lane has a source
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, true); }
constexpr int kRor = 0x120;      // rotation: lane i gets lane i - n
template <class Op>
__device__ __forceinline__ uint32_t row_all(uint32_t x, Op op) {
    x = op(x, dpp<kRor + 8>(x));
    x = op(x, dpp<kRor + 4>(x));
    x = op(x, dpp<kRor + 2>(x));
    return op(x, dpp<kRor + 1>(x));
}
__device__ __forceinline__ uint32_t bits_of(float x) { return __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ float of_bits(uint32_t x) { return __builtin_bit_cast(float, x); }
// maximum, minimum, sum over the 16 lanes of a token
__device__ __forceinline__ uint32_t row_max(uint32_t x) { return row_all(x, [](uint32_t p, uint32_t q) { return max(p, q); }); }
__device__ __forceinline__ float row_max(float x) { return of_bits(row_all(bits_of(x), [](uint32_t p, uint32_t q) { return bits_of(max_of(of_bits(p), of_bits(q))); })); }
__device__ __forceinline__ float row_min(float x) { return of_bits(row_all(bits_of(x), [](uint32_t p, uint32_t q) { return bits_of(min_of(of_bits(p), of_bits(q))); })); }
__device__ __forceinline__ float row_sum(float x) { return of_bits(row_all(bits_of(x), [](uint32_t p, uint32_t q) { return bits_of(of_bits(p) + of_bits(q)); })); }

constexpr uint32_t kIndexBits = 511;      // low bits of a key: 511 - expert
constexpr float kDeep = -80.f;            // scores above exp(kDeep) are normal numbers of 32 bits, a softmax's share of 512 too

// Rows of logits (or the bias) come 16 neighbouring lanes after 16 neighbouring quads or elements, go through LDS, and are read
// back V at a time: a lane that fetched its own V from memory would touch a line of its own with every load, and the address unit
// takes a line at a time (64 tokens of 256 experts in one workgroup: 31 of 47 thousand cycles went into those loads).
// A group's `size` experts are the V each of 2^shift lanes, the last of which may have fewer; expert e of a group lies at (e / V) * pitch +
// e % V behind the group's first lane; `pitch` keeps the lanes' reads on different banks.
struct RowShape {
    int E, V, pitch, shift, size;
    unsigned per_v;       // (e * per_v) >> 16 = e / V for e below 512, V up to 32
    unsigned per_size;    // (e * per_size) >> 20 = e / size for e below 512; 0: lanes have V experts each, or there is one group
    bool quads;           // four elements at a time: aligned, V, E and size multiples of four
    __device__ __forceinline__ int at(int e) const {
        int l0 = 0;
        if (per_size) {
            const int g = (int)((unsigned)e * per_size >> 20);
            e -= g * size;
            l0 = g << shift;
        }
        const int l = (int)((unsigned)e * per_v >> 16);
        return (l0 + l) * pitch + e - l * V;
    }
};
template <int TYPE, int VT>
__device__ __forceinline__ void fetch_row(const void *p, size_t row, const RowShape &r, int l, float (&z)[VT]) {
    using T = std::conditional_t<TYPE == EF_F32, float, uint16_t>;
    const T *x = static_cast<const T *>(p) + row;
    if (r.quads) {
        using T4 = std::conditional_t<TYPE == EF_F32, float4, ushort4>;
        T4 q[VT / 4];
#pragma unroll
        for (int v = 0; v < VT / 4; ++v) q[v] = *reinterpret_cast<const T4 *>(x + min(64 * v + 4 * l, r.E - 4));
#pragma unroll
        for (int v = 0; v < VT / 4; ++v) {
            z[4 * v] = value_of<TYPE>(q[v].x), z[4 * v + 1] = value_of<TYPE>(q[v].y);
            z[4 * v + 2] = value_of<TYPE>(q[v].z), z[4 * v + 3] = value_of<TYPE>(q[v].w);
        }
    } else {
        T h[VT];
#pragma unroll
        for (int v = 0; v < VT; ++v) h[v] = x[min(16 * v + l, r.E - 1)];
#pragma unroll
        for (int v = 0; v < VT; ++v) z[v] = value_of<TYPE>(h[v]);
    }
}
template <int VT>
__device__ __forceinline__ void fetch_row(const void *p, int type, size_t row, const RowShape &r, int l, float (&z)[VT]) {
    if (type == EF_F32) fetch_row<EF_F32>(p, row, r, l, z);
    else if (type == EF_BF16) fetch_row<EF_BF16>(p, row, r, l, z);
    else fetch_row<EF_F16>(p, row, r, l, z);
}
template <int VT>
__device__ __forceinline__ void put_row(float *to, const RowShape &r, int l, const float (&z)[VT]) {
    if (r.quads) {
#pragma unroll
        for (int v = 0; v < VT / 4; ++v) {
            const int e = 64 * v + 4 * l;
            if (e < r.E) *reinterpret_cast<float4 *>(to + r.at(e)) = make_float4(clean(z[4 * v]), clean(z[4 * v + 1]), clean(z[4 * v + 2]), clean(z[4 * v + 3]));
        }
    } else {
#pragma unroll
        for (int v = 0; v < VT; ++v) {
            const int e = 16 * v + l;
            if (e < r.E) to[r.at(e)] = clean(z[v]);
        }
    }
}
// this lane's V; what lies behind them is of no use
template <int VT>
__device__ __forceinline__ void get_row(const float *from, const RowShape &r, int l, float (&z)[VT]) {
    if (r.quads) {
#pragma unroll
        for (int v = 0; v < VT; v += 4) {
            const float4 q = *reinterpret_cast<const float4 *>(from + l * r.pitch + v);
            z[v] = q.x, z[v + 1] = q.y, z[v + 2] = q.z, z[v + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int v = 0; v < VT; ++v) z[v] = from[l * r.pitch + v];
    }
}

template <int TT> struct TileBits { using type = unsigned long long; };
template <> struct TileBits<16> { using type = uint32_t; };

// a tile of TT tokens per workgroup of NW waves, four tokens per wave at a time
template <int VT, int TT, int NW>
__global__ __launch_bounds__(64 * NW, VT <= 16 ? 4 : 2) void router_kernel(RouterArgs a, RowShape shape, bool fast) {
    using Bits = typename TileBits<TT>::type;
    constexpr int R = VT / 4, kE = 16 * VT, kThreads = 64 * NW;
    constexpr int kRow = 16 * (VT + 4);
    __shared__ Bits bits[kE], undecided;
    __shared__ uint16_t chosen_ids[TT * EF_ROUTER_MAX_TOPK];
    __shared__ int first[kE];
    __shared__ __attribute__((aligned(16))) float rows[NW][4][kRow], bias[kRow];
    static_assert(sizeof(rows[0]) >= kE * sizeof(double), "room for a token's values in 64 bits");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int E = a.r.n_experts, k = a.r.top_k, V = shape.V;
    const int t0 = blockIdx.x * TT, n = min(TT, a.T - t0);
    float zn[VT];          // the next tokens' logits
    const auto fetch = [&](int w0, int l) {
        fetch_row<VT>(a.logits, a.type, (size_t)(t0 + min(w0 + (lane >> 4), n - 1)) * a.ld, shape, l, zn);
    };
    if (fast) fetch(wave * 4, lane & 15);
    for (int e = tid; e < kE; e += kThreads) bits[e] = 0;
    if (tid == 0) undecided = fast ? 0 : n == 8 * (int)sizeof(Bits) ? ~(Bits)0 : ((Bits)1 << n) - 1;
    if (a.bias)
        for (int e = tid; e < E; e += kThreads) bias[shape.at(e)] = clean(a.bias[e]);
    __syncthreads();

    const bool softmax = a.r.score == EF_SCORE_SOFTMAX;
    const bool by_logit = !a.bias && (a.r.n_groups == 1 || a.r.group_best == 1);
    for (int w0 = fast ? wave * 4 : n; w0 < n; w0 += NW * 4) {
        // opaque: what follows from a lane's number is worked out in every pass instead of being kept, spilled, over all of them
        int l = lane & 15;
        asm volatile("" : "+v"(l));
        const int g0 = shape.per_size ? (l >> shape.shift) * shape.size : 0, e0 = g0 + (shape.per_size ? l & ((1 << shape.shift) - 1) : l) * V;
        float *mine_rows = rows[wave][lane >> 4];
        const int tok = w0 + (lane >> 4);
        const size_t t = (size_t)t0 + min(tok, n - 1);
        float c[VT], b[VT];     // logits, then choice values; bias
        put_row<VT>(mine_rows, shape, l, zn);
        if (TT > NW * 4 && w0 + NW * 4 < n) fetch(w0 + NW * 4, l);
        wave_lds_sync();
        get_row<VT>(mine_rows, shape, l, c);
        if (a.bias) get_row<VT>(bias, shape, l, b);
        else
#pragma unroll
            for (int v = 0; v < VT; ++v) b[v] = 0.f;
        const int own = max(0, min(V, min(E, g0 + shape.size) - e0));      // experts of this lane
        float m = kMinusInf;
#pragma unroll
        for (int v = 0; v < VT; ++v) {
            c[v] = v < own ? c[v] : kMinusInf;
            m = max_of(m, c[v]);
        }
        float top = 1.f, total = 0.f, bmax = 0.f;
        if (softmax) {
            m = row_max(m);
            const float same = m > 0.f ? 0.f : kMinusInf;     // for inf - inf, and -inf - -inf
            float x[VT];
#pragma unroll
            for (int v = 0; v < VT; ++v) {
                const float d = c[v] - m;
                x[v] = pinned(__expf(d != d ? same : d));
                total += x[v];
            }
            total = row_sum(total);
            top = total > 0.f ? 1.f / total : 0.f;
            if (!by_logit)
#pragma unroll
                for (int v = 0; v < VT; ++v) c[v] = c[v] == kMinusInf ? kMinusInf : x[v] * top;
        } else if (!by_logit) {
#pragma unroll
            for (int v = 0; v < VT; ++v) {
                const float s = pinned(__builtin_amdgcn_rcpf(1.f + __expf(-c[v])));
                c[v] = c[v] == kMinusInf ? kMinusInf : s;
            }
        }
        if (!by_logit) {
#pragma unroll
            for (int v = 0; v < VT; ++v) {
                bmax = max_of(bmax, v < own && fabsf(b[v]) < __builtin_inff() ? fabsf(b[v]) : 0.f);
                c[v] = c[v] == kMinusInf ? kMinusInf : c[v] + b[v];
            }
            bmax = row_max(bmax);
        }
        // A choice value is off by at most 5e-7 (sigmoid: exp, sum, reciprocal) or 1.6e-6 (softmax: the sum's error too) of the
        // largest score and 2^-24 of itself, a sum of two by twice that; a margin is two such errors.
        const float margin = by_logit ? -1.f : (softmax ? 8e-6f : 2.5e-6f) * top + 1e-6f * bmax;

        bool near = false, kept = true;
        if (a.r.n_groups > 1) {
            const int P = 1 << shape.shift;     // lanes of a group; those behind the last group have no experts and lose to every group
            float b1 = kMinusInf, b2 = kMinusInf;
#pragma unroll
            for (int v = 0; v < VT; ++v) {
                b2 = __builtin_amdgcn_fmed3f(b1, b2, c[v]);
                b1 = max_of(b1, c[v]);
            }
            const auto join = [&](uint32_t o1b, uint32_t o2b) {
                const float o1 = of_bits(o1b), o2 = of_bits(o2b);
                b2 = fmaxf(fminf(b1, o1), fmaxf(b2, o2));
                b1 = fmaxf(b1, o1);
            };
            if (P >= 2) join(dpp<0xB1>(bits_of(b1)), dpp<0xB1>(bits_of(b2)));         // lanes in pairs,
            if (P >= 4) join(dpp<0x4E>(bits_of(b1)), dpp<0x4E>(bits_of(b2)));         // fours,
            if (P >= 8) join(dpp<0x141>(bits_of(b1)), dpp<0x141>(bits_of(b2)));       // eights (mirrored)
            const float value = a.r.group_best == 1 ? b1 : b2 == kMinusInf ? kMinusInf : b1 + b2;
            int rank = 0;
            const auto rank_groups = [&](auto lanes) {      // a lane of every other group; a lower lane is of a lower group
                constexpr int p = decltype(lanes)::value;
                static_for<1, 16 / p>([&](auto o) {
                    const float ov = of_bits(dpp<kRor + decltype(o)::value * p>(bits_of(value)));
                    rank += l >= decltype(o)::value * p ? ov >= value : ov > value;
                });
            };
            if (P == 1) rank_groups(std::integral_constant<int, 1>{});
            else if (P == 2) rank_groups(std::integral_constant<int, 2>{});
            else if (P == 4) rank_groups(std::integral_constant<int, 4>{});
            else rank_groups(std::integral_constant<int, 8>{});
            kept = rank < a.r.groups_kept;
            if (a.r.groups_kept < a.r.n_groups && margin >= 0.f) {
                const float worst = row_min(kept ? value : __builtin_inff()), best = row_max(kept ? kMinusInf : value);
                // a sum of two that passes 32 bits: the wave's tokens are decided in 64
                const float inf = __builtin_inff();
                near = worst - best <= margin;
                if (__builtin_expect(__any(fabsf(value) == inf), 0)) near |= __any(fabsf(value) == inf && fabsf(b1) < inf && fabsf(b2) < inf);
            }
        }
        uint32_t key[VT];
        const int live = kept ? own : 0;
#pragma unroll
        for (int v = 0; v < VT; ++v) key[v] = v < live ? (key_of(c[v]) & ~kIndexBits) | (kIndexBits - (uint32_t)(e0 + v)) : 0u;
        const auto below = [&](uint32_t last) {     // the largest key below `last`
            uint32_t d = key[0] - last;
#pragma unroll
            for (int v = 1; v < VT; ++v) d = max(d, key[v] - last);
            return row_max(d) + last;
        };
        uint32_t prev = 0, last = 0, won = 0;
        for (int j = 0; j < k; ++j) {
            prev = last;
            last = below(last);
            if (l == j) won = last;
        }
        if (a.type == EF_F32 || !by_logit) {
            // the keys' upper bits hold a value to 2^-14 of itself: the best expert left out may be ahead of the last one chosen.
            // Where no third one is as close, their values in full decide between the two
            const uint32_t next = below(last);
            const auto close = [&](uint32_t hi, uint32_t lo) {      // 0 and what below() gives behind the last key are not values
                const float x = of_key(hi & ~kIndexBits), y = of_key(lo & ~kIndexBits);
                return lo > kIndexBits && lo < hi && (((hi ^ lo) & ~kIndexBits) == 0 || x - y <= margin + 0x1p-14f * (fabsf(x) + fabsf(y)));
            };
            const bool border = close(last, next);
            if (__ballot(border)) {
                const uint32_t third = below(next);
                if (border) {
                    near |= (k > 1 && close(prev, last)) || (next < last && close(next, third));
                    const int ea = (int)(kIndexBits - (last & kIndexBits)), eb = (int)(kIndexBits - (next & kIndexBits));
                    const float za = mine_rows[shape.at(ea)], zb = mine_rows[shape.at(eb)];
                    const auto choice = [&](float z, int e) {
                        if (by_logit || z == kMinusInf) return z;
                        const float d = z - m;
                        const float s = softmax ? __expf(d != d ? 0.f : d) * top : __builtin_amdgcn_rcpf(1.f + __expf(-z));
                        return a.bias ? s + bias[shape.at(e)] : s;
                    };
                    const float ca = choice(za, ea), cb = choice(zb, eb);
                    if (!by_logit) near |= fabsf(ca - cb) <= margin;
                    if (cb > ca || (cb == ca && eb < ea)) {
                        if (l == k - 1) won = next;
                    }
                }
            }
        }
        if (tok < n && near && l == 0) atomicOr(&undecided, (Bits)1 << tok);
        // lanes 0..k-1: one chosen expert each, its place among them, its score
        const bool mine = l < k && tok < n && !near;
        const int e = (int)(kIndexBits - (won & kIndexBits));
        int place = 0;
        static_for<1, 16>([&](auto o) { place += dpp<kRor + decltype(o)::value>(l < k ? (uint32_t)e : 1u << 16) < (uint32_t)e; });
        const float z = mine ? mine_rows[shape.at(e)] : kMinusInf;
        const float depth = softmax ? z - m : z, x0 = expf(softmax ? depth : -fabsf(z));
        float w = softmax ? (z == m ? top : x0 * top) : (z < 0.f ? x0 : 1.f) / (1.f + x0);
        if (a.r.renorm) {
            if (__builtin_expect(__any(mine && depth < kDeep), 0)) {
                // Scores that 32 bits do not hold, or in part, keep their quotients without their common factor exp(zc): zc the largest
                // chosen logit (sigmoid: 0 unless all are negative).  What is 0 in 64 bits counts as 0.
                const float most = row_max(z), zc = softmax ? most : min_of(most, 0.f);
                const float x = z == most ? 1.f : expf((softmax ? z : min_of(z, 0.f)) - zc);
                const bool none = z == kMinusInf || (softmax ? depth < -745.1332f : z <= -709.7827f);
                w = none ? 0.f : softmax ? x : x / (1.f + x0);
            }
            const float sum = row_sum(w);
            w = sum > 0.f ? w / sum : 0.f;
        }
        if (mine) {
            a.ids[t * k + place] = e;
            a.w[t * k + place] = w * a.r.scale;
            chosen_ids[tok * k + place] = (uint16_t)e;
            atomicOr(&bits[e], (Bits)1 << tok);
        }
    }
    __syncthreads();
    if (undecided) {       // uniform; a wave per token
        Groups g{a.r.n_groups, E / a.r.n_groups, a.r.groups_kept, a.r.group_best, 64};
        while (g.lanes * g.n > 64) g.lanes >>= 1;
        int nth = 0;
        for (Bits todo = undecided; todo; todo &= todo - 1, ++nth)
            if (nth % NW == wave) {
                const int x = __builtin_ctzll(todo);
                exact_token<R>(a, (size_t)t0 + x, x, g, reinterpret_cast<double *>(&rows[wave][0][0]), chosen_ids, bits);
                wave_lds_sync();
            }
        __syncthreads();
    }

    if (a.ntiles > 1) {
        for (int e = tid; e < a.pitch; e += kThreads) a.tile_counts[(size_t)blockIdx.x * a.pitch + e] = (uint8_t)__popcll(bits[e]);
        for (int x = tid; x < n * k; x += kThreads)
            a.inv_perm[(size_t)t0 * k + x] = __popcll(bits[chosen_ids[x]] & (((Bits)1 << (x / k)) - 1));
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
    for (int x = tid; x < n * k; x += kThreads) {
        const int e = chosen_ids[x];
        const int pos = first[e] + __popcll(bits[e] & (((Bits)1 << (x / k)) - 1));
        a.perm[pos] = x;
        a.inv_perm[x] = pos;
    }
}

// Adds up the tiles' counts of every expert, over all tiles and over those before `tile`.  A thread takes 16 experts of every
// (256 / threads per tile)-th tile, eight loads of 16 bytes in flight, and adds the bytes in pairs of 16 bits, which hold the sum
// of its tiles.
template <int R>
__device__ __forceinline__ void add_counts(const RouterArgs &a, int tile, int *total, int *before) {
    constexpr int kPer = 4 * R, kStep = 256 / kPer;      // threads per tile, tiles per round
    static_assert(kRouterSumTiles / kStep * 64 < 65536, "16 bits per sum");
    const int tid = threadIdx.x, sixteen = tid % kPer;
    for (int e = tid; e < 64 * R; e += 256) total[e] = before[e] = 0;
    __syncthreads();
    const uint4 *counts = reinterpret_cast<const uint4 *>(a.tile_counts) + sixteen;
    const auto add = [&](int b0, int b1, int *to, int *and_to) {
        uint32_t even[4] = {0, 0, 0, 0}, odd[4] = {0, 0, 0, 0};
        for (int b = b0 + tid / kPer; b < b1; b += kStep * 8) {
            uint4 x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = counts[(size_t)min(b + i * kStep, b1 - 1) * (a.pitch / 16)];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t mask = b + i * kStep < b1 ? 0x00FF00FFu : 0u, w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    even[q] += w[q] & mask;
                    odd[q] += w[q] >> 8 & mask;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int x = (i & 1 ? odd[i >> 2] : even[i >> 2]) >> (i & 2 ? 16 : 0) & 0xFFFF;
            if (x) {
                atomicAdd(to + sixteen * 16 + i, x);
                if (and_to) atomicAdd(and_to + sixteen * 16 + i, x);
            }
        }
    };
    if (sixteen * 16 < a.pitch) {
        add(0, tile, before, total);
        add(tile, a.ntiles, total, nullptr);
    }
    __syncthreads();
}

// scatter of a tile; `scanned`: the prefixes over the tiles and the totals are there already
template <int R>
__global__ __launch_bounds__(256) void router_scatter_kernel(RouterArgs a, int tile, bool scanned) {
    __shared__ int first[64 * R], total[64 * R];
    const int E = a.r.n_experts, k = a.r.top_k, tid = threadIdx.x, lane = tid & 63;
    if (scanned) {
        for (int e = tid; e < 64 * R; e += 256) {
            total[e] = e < E ? a.counts[e] : 0;
            first[e] = e < E ? a.prefix[(size_t)blockIdx.x * a.pitch + e] : 0;
        }
        __syncthreads();
    } else {
        add_counts<R>(a, blockIdx.x, total, first);
    }
    if (tid < 64) {
        int cnt[R], off[R];
#pragma unroll
        for (int r = 0; r < R; ++r) cnt[r] = total[r * 64 + lane];
        const int all = expert_offsets<R>(cnt, off);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int e = r * 64 + lane;
            first[e] += off[r];
            if (blockIdx.x == 0 && e < E) {
                a.offsets[e] = off[r];
                if (!scanned) a.counts[e] = cnt[r];
            }
        }
        if (blockIdx.x == 0 && lane == 0) a.offsets[E] = all;
    }
    __syncthreads();
    const size_t a0 = (size_t)blockIdx.x * tile * k;
    const int n = min(tile, a.T - (int)blockIdx.x * tile) * k;
    for (int x = tid; x < n; x += 256) {
        const int pos = first[a.ids[a0 + x]] + a.inv_perm[a0 + x];     // its rank in the tile, from the first launch
        a.perm[pos] = (int)(a0 + x);
        a.inv_perm[a0 + x] = pos;
    }
}

// many tiles: their counts' exclusive prefixes, an expert per workgroup of 256
__global__ __launch_bounds__(256) void router_scan_kernel(RouterArgs a) {
    __shared__ int part[256];
    const int e = blockIdx.x, tid = threadIdx.x, per = (a.ntiles + 255) / 256;
    const int b0 = min(a.ntiles, tid * per), b1 = min(a.ntiles, b0 + per);
    int sum = 0;
    for (int b = b0; b < b1; ++b) sum += a.tile_counts[(size_t)b * a.pitch + e];
    part[tid] = sum;
    __syncthreads();
    int before = 0, all = 0;
    for (int i = 0; i < 256; ++i) {
        before += i < tid ? part[i] : 0;
        all += part[i];
    }
    for (int b = b0; b < b1; ++b) {
        a.prefix[(size_t)b * a.pitch + e] = before;
        before += a.tile_counts[(size_t)b * a.pitch + e];
    }
    if (tid == 0) a.counts[e] = all;
}

// How 16 lanes share a token's experts: 2^shift lanes a group, V experts a lane.  More groups than lanes, or more than 32 experts a
// lane: the exact way.
struct LaneShares { bool fast; int shift, V; };
LaneShares lane_shares(const ef_router &r) {
    int shift = 4;
    while (shift >= 0 && (r.n_groups << shift) > 16) --shift;
    const int V = shift < 0 ? 33 : (r.n_experts / r.n_groups + (1 << shift) - 1) >> shift;
    return V <= 32 ? LaneShares{true, shift, V} : LaneShares{false, 4, (r.n_experts + 15) / 16};
}

template <int VT>
hipError_t launch_v(const RouterArgs &a, hipStream_t s) {
    const int tile = router_tile(a.r, a.T), E = a.r.n_experts, n = a.r.n_groups, size = n == 1 ? E : E / n;
    const LaneShares share = lane_shares(a.r);
    const bool fast = share.fast;
    const int V = share.V;
    const size_t bytes = a.type == EF_F32 ? 4 : 2;
    const bool quads = V % 4 == 0 && E % 4 == 0 && size % 4 == 0 && a.ld % 4 == 0 && reinterpret_cast<size_t>(a.logits) % (4 * bytes) == 0 &&
                       reinterpret_cast<size_t>(a.bias) % 16 == 0;
    const unsigned per_size = fast && n > 1 && size != V << share.shift ? ((1u << 20) + size - 1) / size : 0;
    const RowShape shape{E, V, quads ? V + 4 : V | 1, share.shift, per_size ? size : E, (65536u + V - 1) / V, per_size, quads};
    // one tile of 64: a wave for every four tokens; many: two passes per wave, so that two workgroups fit a compute unit's LDS
    if (tile == 16) hipLaunchKernelGGL((router_kernel<VT, 16, 4>), dim3(a.ntiles), dim3(256), 0, s, a, shape, fast);
    else if (VT > 16 || a.ntiles > 1) hipLaunchKernelGGL((router_kernel<VT, 64, 8>), dim3(a.ntiles), dim3(512), 0, s, a, shape, fast);
    else if constexpr (VT <= 16) hipLaunchKernelGGL((router_kernel<VT, 64, 16>), dim3(1), dim3(1024), 0, s, a, shape, fast);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.ntiles == 1) return e;
    const bool scan = a.prefix != nullptr;
    if (scan) hipLaunchKernelGGL(router_scan_kernel, dim3(E), dim3(256), 0, s, a);
    hipLaunchKernelGGL((router_scatter_kernel<VT / 4>), dim3(a.ntiles), dim3(256), 0, s, a, tile, scan);
    return hipGetLastError();
}

}  // namespace

// Up to 64 tokens are one tile (one launch, on one compute unit); beyond, tiles of 16 until the grid of 64s fills the chip.  With many
// experts a lane a second launch costs less than the one unit: 64 tokens of 256 experts in 8 groups 11.8 us against 13.7 (48: 11.6
// against 11.9), of 200 10.6 against 10.0; 17 of 512 13.4 against 16.4.
int router_tile(const ef_router &r, int T) {
    const int V = lane_shares(r).V;
    return T > (V > 16 ? 0 : V > 13 ? 48 : 64) && T <= kRouterSmallTiles ? 16 : 64;
}

hipError_t launch_router(const RouterArgs &a, hipStream_t s) {
    const int E = a.r.n_experts;
    if (a.T <= 0) {
        const hipError_t e = launch_fill_i32(a.counts, E, 0, s);
        return e != hipSuccess ? e : launch_fill_i32(a.offsets, E + 1, 0, s);
    }
    const int tile = router_tile(a.r, a.T);
    if (a.ntiles != (a.T + tile - 1) / tile || a.pitch < E || a.pitch % 4 != 0) return hipErrorInvalidValue;
    const int V = lane_shares(a.r).V;
    return V <= 4 ? launch_v<4>(a, s) : V <= 8 ? launch_v<8>(a, s) : V <= 16 ? launch_v<16>(a, s) : launch_v<32>(a, s);
}

}  // namespace ef

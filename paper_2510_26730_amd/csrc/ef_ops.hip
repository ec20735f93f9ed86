// Entry points of the context-free operators: routing from logits, rows to 8 bits, products of 8-bit codes, weighted sum of
// expert rows.  Argument checks and scratch layout; the kernels are in ef_router.hip, ef_q8.hip, ef_q8_panel.hip
// and ef_q8_tiled.hip.
#include "ef_ctx.h"
#include "ef_ops.h"

using namespace efi;

namespace {

constexpr size_t kAlign = 256;
size_t rounded(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }
bool is_float_type(int t) { return t == EF_BF16 || t == EF_F16 || t == EF_F32; }
// tensors of elements are used at their natural alignment
bool aligned_to_type(const void *p, int type) {
    return (reinterpret_cast<uintptr_t>(p) & (type == EF_F32 ? 3u : type == EF_I8 ? 0u : 1u)) == 0;
}
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

const char *router_fault(const ef_router *r) {
    if (!r) return "null router";
    if (r->n_experts < 1 || r->n_experts > EF_ROUTER_MAX_EXPERTS) return "n_experts out of range";
    if (r->score != EF_SCORE_SOFTMAX && r->score != EF_SCORE_SIGMOID) return "unknown score";
    if (r->n_groups < 1 || r->n_groups > EF_ROUTER_MAX_GROUPS || r->n_experts % r->n_groups != 0)
        return "n_groups must divide n_experts and be at most EF_ROUTER_MAX_GROUPS";
    if (r->groups_kept < 1 || r->groups_kept > r->n_groups) return "groups_kept outside 1..n_groups";
    const int size = r->n_experts / r->n_groups;
    if (r->group_best != 1 && r->group_best != 2) return "group_best must be 1 or 2";
    if (r->n_groups > 1 && r->group_best > size) return "group_best 2 needs groups of two experts";
    if (r->top_k < 1 || r->top_k > EF_ROUTER_MAX_TOPK || r->top_k > size * r->groups_kept) return "top_k out of range";
    if (r->renorm != 0 && r->renorm != 1) return "renorm must be 0 or 1";
    return nullptr;
}
// a launch has fewer than 2^32 lanes: eight for a token at most
bool router_tokens_ok(const ef_router *r, int T) { return T >= 0 && T <= (1 << 29) - 64 && (long long)T * r->top_k <= 0x7FFFFFFFll; }

int router_tiles(const ef_router *r, int T) {
    const int tile = ef::router_tile(*r, T);
    return (T + tile - 1) / tile;
}
int router_pitch(const ef_router *r) { return (r->n_experts + 15) / 16 * 16; }
size_t router_counts_bytes(const ef_router *r, int T) { return rounded((size_t)router_pitch(r) * router_tiles(r, T)); }
size_t router_prefix_bytes(const ef_router *r, int T) { return router_tiles(r, T) > ef::kRouterSumTiles ? 4 * router_counts_bytes(r, T) : 0; }

}  // namespace

extern "C" size_t ef_route_scores_work(const ef_router *r, int T) {
    if (router_fault(r) || !router_tokens_ok(r, T)) return 0;
    const auto bytes = [&](int t) { return router_counts_bytes(r, t) + router_prefix_bytes(r, t) + kAlign; };
    return std::max(bytes(T), bytes(std::min(T, ef::kRouterSmallTiles)));   // fewer tokens never need more
}

extern "C" int ef_route_scores(const ef_router *r, const void *logits, int type, int64_t ld, const float *bias, int T,
                               int32_t *topk_ids, float *topk_w, int32_t *counts, int32_t *offsets, int32_t *perm,
                               int32_t *inv_perm, void *work, size_t work_bytes, void *stream) {
    if (const char *why = router_fault(r)) return fail(nullptr, EF_EINVAL, "ef_route_scores: %s", why);
    if (!router_tokens_ok(r, T)) return fail(nullptr, EF_EINVAL, "ef_route_scores: T=%d out of range", T);
    if (!is_float_type(type)) return fail(nullptr, EF_EINVAL, "ef_route_scores: logits of type %d", type);
    if (!counts || !offsets) return fail(nullptr, EF_EINVAL, "ef_route_scores: null pointer");
    if (T > 0) {
        if (!logits || !topk_ids || !topk_w || !perm || !inv_perm || !work) return fail(nullptr, EF_EINVAL, "ef_route_scores: null pointer");
        if (ld < r->n_experts) return fail(nullptr, EF_EINVAL, "ef_route_scores: rows of %lld elements for %d experts", (long long)ld, r->n_experts);
        if (!aligned_to_type(logits, type) || !aligned4(bias) || !aligned4(topk_ids) || !aligned4(topk_w) || !aligned4(perm) ||
            !aligned4(inv_perm) || !aligned16(work))
            return fail(nullptr, EF_EINVAL, "ef_route_scores: misaligned pointer");
        if (work_bytes < ef_route_scores_work(r, T)) return fail(nullptr, EF_EINVAL, "ef_route_scores: %zu bytes of scratch, %zu needed", work_bytes, ef_route_scores_work(r, T));
    }
    if (!aligned4(counts) || !aligned4(offsets)) return fail(nullptr, EF_EINVAL, "ef_route_scores: misaligned pointer");
    ef::RouterArgs a{};
    a.r = *r;
    a.logits = logits;
    a.type = type;
    a.ld = ld;
    a.bias = bias;
    a.T = T;
    a.ids = topk_ids;
    a.w = topk_w;
    a.counts = counts;
    a.offsets = offsets;
    a.perm = perm;
    a.inv_perm = inv_perm;
    a.ntiles = router_tiles(r, T);
    a.tile_counts = static_cast<uint8_t *>(work);
    a.pitch = router_pitch(r);
    a.prefix = router_prefix_bytes(r, T) ? reinterpret_cast<int32_t *>(a.tile_counts + router_counts_bytes(r, T)) : nullptr;
    EF_HIP(nullptr, ef::launch_router(a, static_cast<hipStream_t>(stream)));
    return EF_OK;
}

extern "C" int ef_route_scores_of(const ef_router *r, const ef_route_operands *o, void *stream) {
    if (!o) return fail(nullptr, EF_EINVAL, "ef_route_scores: null operands");
    return ef_route_scores(r, o->logits, o->type, o->ld, o->bias, o->T, o->topk_ids, o->topk_w, o->counts, o->offsets, o->perm, o->inv_perm,
                           o->work, o->work_bytes, stream);
}

extern "C" int ef_quant_rows(const void *x, int type, int64_t ldx, int rows, int K, int8_t *codes, int64_t ldc, float *scales,
                             void *stream) {
    return ef_quant_rows_within(x, type, ldx, rows, K, codes, ldc, ldc, scales, stream);
}

extern "C" int ef_quant_rows_within(const void *x, int type, int64_t ldx, int rows, int K, int8_t *codes, int64_t width, int64_t ldc,
                                    float *scales, void *stream) {
    if (!is_float_type(type)) return fail(nullptr, EF_EINVAL, "ef_quant_rows: rows of type %d", type);
    if (rows < 0 || K < 1) return fail(nullptr, EF_EINVAL, "ef_quant_rows: %d rows of %d", rows, K);
    if (rows == 0) return EF_OK;
    if (!x || !codes || !scales) return fail(nullptr, EF_EINVAL, "ef_quant_rows: null pointer");
    if (ldx < K || ldc < K) return fail(nullptr, EF_EINVAL, "ef_quant_rows: rows of %d overlap (ldx %lld, ldc %lld)", K, (long long)ldx, (long long)ldc);
    if (width < K || width > ldc) return fail(nullptr, EF_EINVAL, "ef_quant_rows: width %lld outside K=%d..ldc=%lld", (long long)width, K, (long long)ldc);
    if (!aligned_to_type(x, type) || !aligned4(scales)) return fail(nullptr, EF_EINVAL, "ef_quant_rows: misaligned pointer");
    const ef::QuantArgs a{x, type, ldx, rows, K, codes, ldc, width, scales};
    EF_HIP(nullptr, ef::launch_quant_rows(a, static_cast<hipStream_t>(stream)));
    return EF_OK;
}

namespace {

constexpr int kMaxQ8K = 131071;   // 128 * 128 * K stays below 2^31

const char *q8_shape_fault(const ef_q8_product *p) {
    if (!p) return "null product";
    if (p->a_type != EF_I8 && !is_float_type(p->a_type)) return "unknown a_type";
    if (!is_float_type(p->out_type)) return "unknown out_type";
    if (p->M < 0 || p->a_rows < 0 || p->N < 1 || p->K < 1 || p->K > kMaxQ8K) return "M, a_rows, N or K out of range";
    if (p->G < 1 || p->G > EF_ROUTER_MAX_EXPERTS) return "G out of range";
    if (p->swiglu != 0 && p->swiglu != 1) return "swiglu must be 0 or 1";
    if (p->swiglu && p->N % 2 != 0) return "swiglu needs an even N";
    if (p->lda < p->K) return "rows of a overlap";
    return nullptr;
}
// codes are used where they are if the kernels can read whole steps of 64 of them
bool q8_in_place(const ef_q8_product *p) { return p->a_type == EF_I8 && p->K % 64 == 0 && p->lda % 16 == 0 && aligned16(p->a); }
long long q8_pitch(int K) { return ((long long)K + 63) / 64 * 64; }

}  // namespace

extern "C" size_t ef_matmul_q8_work(const ef_q8_product *p) {
    if (q8_shape_fault(p)) return 0;
    return rounded((size_t)p->a_rows * q8_pitch(p->K)) + rounded((size_t)p->a_rows * 4) + kAlign;
}

extern "C" int ef_matmul_q8(const ef_q8_product *p, void *work, size_t work_bytes, void *stream) {
    if (const char *why = q8_shape_fault(p)) return fail(nullptr, EF_EINVAL, "ef_matmul_q8: %s", why);
    if (p->M == 0) return EF_OK;
    if (!p->a || !p->w || !p->w_scale || !p->out) return fail(nullptr, EF_EINVAL, "ef_matmul_q8: null pointer");
    if ((p->a_type == EF_I8) != (p->a_scale != nullptr)) return fail(nullptr, EF_EINVAL, "ef_matmul_q8: a_scale comes with codes and only with them");
    if (!p->offsets && p->G != 1) return fail(nullptr, EF_EINVAL, "ef_matmul_q8: %d groups without offsets", p->G);
    if (p->row_div < 1) return fail(nullptr, EF_EINVAL, "ef_matmul_q8: row_div=%d", p->row_div);
    if (p->a_rows < 1 || (!p->rows && p->M > p->a_rows)) return fail(nullptr, EF_EINVAL, "ef_matmul_q8: %d product rows of %d rows of a", p->M, p->a_rows);
    const long long kw = ((long long)p->K + 15) / 16 * 16, cols = p->swiglu ? p->N / 2 : p->N;
    if (p->ldw < kw || p->ldw % 16 != 0 || p->w_group % 16 != 0 || !aligned16(p->w))
        return fail(nullptr, EF_EINVAL, "ef_matmul_q8: weight rows must be 16-byte aligned and hold K rounded up to 16 (ldw %lld, w_group %lld)", (long long)p->ldw, (long long)p->w_group);
    if (p->G > 1 && p->w_group < (p->N - 1) * p->ldw + kw) return fail(nullptr, EF_EINVAL, "ef_matmul_q8: matrices overlap (w_group %lld)", (long long)p->w_group);
    if (p->ldo < cols) return fail(nullptr, EF_EINVAL, "ef_matmul_q8: rows of out overlap");
    if (!aligned_to_type(p->a, p->a_type) || !aligned_to_type(p->out, p->out_type) || !aligned4(p->a_scale) || !aligned4(p->rows) ||
        !aligned4(p->offsets) || !aligned4(p->w_scale))
        return fail(nullptr, EF_EINVAL, "ef_matmul_q8: misaligned pointer");
    ef::Q8Args q{};
    q.a = static_cast<const int8_t *>(p->a);
    q.lda = p->lda;
    q.a_type = p->a_type;
    q.a_scale = p->a_scale;
    q.a_rows = p->a_rows;
    q.rows = p->rows;
    q.row_div = p->row_div;
    q.M = p->M;
    q.offsets = p->offsets;
    q.G = p->G;
    q.w = static_cast<const int8_t *>(p->w);
    q.ldw = p->ldw;
    q.w_group = p->w_group;
    q.w_scale = p->w_scale;
    q.N = p->N;
    q.K = p->K;
    q.swiglu = p->swiglu;
    q.out = p->out;
    q.out_type = p->out_type;
    q.ldo = p->ldo;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (!q8_in_place(p)) {
        if (!work || !aligned16(work)) return fail(nullptr, EF_EINVAL, "ef_matmul_q8: scratch is null or not 16-byte aligned");
        if (work_bytes < ef_matmul_q8_work(p)) return fail(nullptr, EF_EINVAL, "ef_matmul_q8: %zu bytes of scratch, %zu needed", work_bytes, ef_matmul_q8_work(p));
        if (!ef::q8_product_quantises(q)) {
            int8_t *codes = static_cast<int8_t *>(work);
            float *scales = reinterpret_cast<float *>(codes + rounded((size_t)p->a_rows * q8_pitch(p->K)));
            const ef::QuantArgs qa{p->a, p->a_type, p->lda, p->a_rows, p->K, codes, q8_pitch(p->K), q8_pitch(p->K), scales};
            EF_HIP(nullptr, ef::launch_quant_rows(qa, s));
            q.a = codes;
            q.lda = q8_pitch(p->K);
            q.a_type = EF_I8;
            if (p->a_type != EF_I8) q.a_scale = scales;
        }
    }
    EF_HIP(nullptr, ef::launch_q8_product(q, s));
    return EF_OK;
}

extern "C" int ef_combine(const void *y, int y_type, int64_t ldy, int y_rows, const float *w, const int32_t *inv_perm, int T, int k,
                          int d, void *out, int out_type, int64_t ldo, void *stream) {
    if (!is_float_type(y_type) || !is_float_type(out_type)) return fail(nullptr, EF_EINVAL, "ef_combine: unknown type");
    if (T < 0 || k < 1 || d < 1 || y_rows < 0 || (long long)T * k > 0x7FFFFFFFll) return fail(nullptr, EF_EINVAL, "ef_combine: T, k, d or y_rows out of range");
    if (T == 0) return EF_OK;
    if ((!y && y_rows > 0) || !w || !out) return fail(nullptr, EF_EINVAL, "ef_combine: null pointer");
    if (ldy < d || ldo < d) return fail(nullptr, EF_EINVAL, "ef_combine: rows of %d overlap", d);
    if (!inv_perm && y_rows < (long long)T * k) return fail(nullptr, EF_EINVAL, "ef_combine: %d rows for %d x %d", y_rows, T, k);
    if (!aligned_to_type(y, y_type) || !aligned_to_type(out, out_type) || !aligned4(w) || !aligned4(inv_perm))
        return fail(nullptr, EF_EINVAL, "ef_combine: misaligned pointer");
    const ef::CombineArgs a{y, y_type, ldy, y_rows, w, inv_perm, T, k, d, out, out_type, ldo};
    EF_HIP(nullptr, ef::launch_combine_rows(a, static_cast<hipStream_t>(stream)));
    return EF_OK;
}

// extern "C" entry points of the 8-bit key/value cache (declared in
// include/skm.h): argument checks on the host, workspace carving, launches.
#include <algorithm>

#include "skm_kv.cuh"

namespace skm {

namespace {

constexpr int64_t KV_MOST = int64_t(1) << 30;  // tokens of a call, positions of a sequence

cudaStream_t S(void *s) { return static_cast<cudaStream_t>(s); }
bool aligned(const void *p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

int check_cache(const skm_kv_cache *c) {
    if (!c) return set_error(SKM_ERR_INVALID_ARG, "skm_kv_cache is NULL");
    if (c->heads < 1 || c->pages < 1)
        return set_error(SKM_ERR_INVALID_ARG, "heads = %d, pages = %d: both must be positive", c->heads, c->pages);
    if (c->d < 1 || c->page < 1) return set_error(SKM_ERR_INVALID_ARG, "d = %d, page = %d", c->d, c->page);
    if (c->d % KV_B || c->d > 256)
        return set_error(SKM_ERR_UNSUPPORTED, "d = %d: a multiple of 16 up to 256", c->d);
    if (c->page % KV_B) return set_error(SKM_ERR_UNSUPPORTED, "page = %d: a multiple of 16", c->page);
    if (cdiv((int64_t(1) << 31) - 1, (int64_t)c->heads * (c->page / KV_B)) <= c->pages)
        return set_error(SKM_ERR_UNSUPPORTED, "pages * heads * page / 16 must be below 2^31");
    if (!c->k || !c->v || !c->scales) return set_error(SKM_ERR_INVALID_ARG, "the cache's k, v or scales is NULL");
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->scales, 8))
        return set_error(SKM_ERR_INVALID_ARG, "k and v must be 16-byte, scales 8-byte aligned");
    return SKM_OK;
}

int check_seqs(const skm_kv_cache *c, const skm_kv_seqs *s) {
    if (!s) return set_error(SKM_ERR_INVALID_ARG, "skm_kv_seqs is NULL");
    if (s->batch < 1 || s->cols < 1)
        return set_error(SKM_ERR_INVALID_ARG, "batch = %d, cols = %d: both must be positive", s->batch, s->cols);
    if (s->tokens < 0 || s->max_tokens < 0)
        return set_error(SKM_ERR_INVALID_ARG, "tokens = %d, max_tokens = %d", s->tokens, s->max_tokens);
    if (s->tokens >= KV_MOST || (int64_t)s->cols * c->page >= KV_MOST)
        return set_error(SKM_ERR_UNSUPPORTED, "tokens and cols * page must be below 2^30");
    if (!s->table || !s->pos || !s->cu) return set_error(SKM_ERR_INVALID_ARG, "table, pos or cu is NULL");
    return SKM_OK;
}

int check_dtype(int dtype) {
    if (dtype != SKM_DTYPE_F32 && dtype != SKM_DTYPE_BF16 && dtype != SKM_DTYPE_F16)
        return set_error(SKM_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    return SKM_OK;
}

int most_tokens(const skm_kv_seqs *s) { return std::min(s->max_tokens, s->tokens); }

size_t elem_of(int dtype) { return dtype == SKM_DTYPE_F32 ? 4 : 2; }

KvCacheArgs cache_args(const skm_kv_cache *c, const skm_kv_seqs *s) {
    KvCacheArgs a = {};
    a.k = c->k;
    a.v = c->v;
    a.scales = reinterpret_cast<float2 *>(c->scales);
    a.table = s->table;
    a.pos = s->pos;
    a.cu = s->cu;
    a.heads = c->heads;
    a.d = c->d;
    a.page = c->page;
    a.pages = c->pages;
    a.bpp = c->page / KV_B;
    a.batch = s->batch;
    a.cols = s->cols;
    a.tokens = s->tokens;
    a.max_tokens = most_tokens(s);
    return a;
}

// a launch's warps must fit a grid
int check_grid(const skm_kv_cache *c, const skm_kv_seqs *s) {
    const int64_t blocks = (most_tokens(s) + 2 * KV_B - 2) / KV_B;
    if ((double)s->batch * blocks * c->heads > 1e9)
        return set_error(SKM_ERR_UNSUPPORTED, "batch * max_tokens * heads is too large");
    return SKM_OK;
}

KvTokens tokens_of(const void *x, int64_t token, int64_t head, int dtype) {
    const size_t e = elem_of(dtype);
    return KvTokens{x, token, head, aligned(x, 16) && token * e % 16 == 0 && head * e % 16 == 0};
}

int check_attn(const skm_kv_cache *c, const skm_kv_seqs *s, const skm_kv_attn *a) {
    if (!a) return set_error(SKM_ERR_INVALID_ARG, "skm_kv_attn is NULL");
    SKM_TRY(check_dtype(a->dtype));
    if (a->heads_q < 1 || a->heads_q % c->heads)
        return set_error(SKM_ERR_INVALID_ARG, "heads_q = %d is not a multiple of the cache's %d heads", a->heads_q, c->heads);
    if (a->window < 0) return set_error(SKM_ERR_INVALID_ARG, "window = %d", a->window);
    if (a->window > 0 && !a->causal) return set_error(SKM_ERR_INVALID_ARG, "a window needs causal");
    if (!(a->scale - a->scale == 0.0f)) return set_error(SKM_ERR_INVALID_ARG, "scale is not finite");
    if (s->max_len < 0) return set_error(SKM_ERR_INVALID_ARG, "max_len = %d", s->max_len);
    if ((int64_t)most_tokens(s) * a->heads_q >= KV_MOST)
        return set_error(SKM_ERR_UNSUPPORTED, "max_tokens * heads_q must be below 2^30");
    return SKM_OK;
}

// positions that a row tile's items may span
int64_t span_of(const skm_kv_cache *c, const skm_kv_seqs *s, const skm_kv_attn *a) {
    int64_t span = std::min<int64_t>(s->max_len, (int64_t)s->cols * c->page);
    if (a->window > 0) span = std::min<int64_t>(span, (int64_t)a->window + most_tokens(s) + KV_B);
    return span;
}

// How a call runs, and its parts of the workspace
struct AttendPlan {
    bool prompt;
    int seqs;  // of a launch
    KvRowsPlan rows = {};
    KvPromptPlan many = {};
    float *part_cta = nullptr, *part_warp = nullptr;
};

AttendPlan plan_attend(const skm_kv_cache *c, const skm_kv_seqs *s, const skm_kv_attn *a, Carver &cv) {
    AttendPlan p;
    const int nb = p.seqs = std::min<int>(s->batch, KV_MAX_SEQS), group = a->heads_q / c->heads, most = most_tokens(s);
    p.prompt = kv_prompt_ok(a->dtype, nb, c->heads, c->d, (int64_t)most * group, span_of(c, s, a));
    if (p.prompt) {
        p.many = kv_prompt_plan(nb, c->heads, group, c->d, most, span_of(c, s, a));
        if (p.many.part) p.part_cta = cv.take<float>(p.many.part / 4);
    } else {
        p.rows = kv_rows_plan(nb, c->heads, group, c->d, a->dtype, most, span_of(c, s, a));
        p.seqs = p.rows.seqs;
        if (p.rows.part_cta) p.part_cta = cv.take<float>(p.rows.part_cta / 4);
        if (p.rows.part_warp) p.part_warp = cv.take<float>(p.rows.part_warp / 4);
    }
    return p;
}

int check_attend(const skm_kv_cache *c, const skm_kv_seqs *s, const skm_kv_attn *a) {
    SKM_TRY(check_cache(c));
    SKM_TRY(check_seqs(c, s));
    return check_attn(c, s, a);
}

}  // namespace

}  // namespace skm

using namespace skm;

extern "C" {

int skm_kv_write(const skm_kv_cache *c, const skm_kv_seqs *s, int dtype, const void *K, int64_t k_token,
                 int64_t k_head, const void *V, int64_t v_token, int64_t v_head, void *stream) {
    SKM_TRY(check_cache(c));
    SKM_TRY(check_seqs(c, s));
    SKM_TRY(check_dtype(dtype));
    SKM_TRY(check_grid(c, s));
    if (most_tokens(s) == 0) return SKM_OK;
    if (!K || !V) return set_error(SKM_ERR_INVALID_ARG, "K or V is NULL");
    if (!aligned(K, elem_of(dtype)) || !aligned(V, elem_of(dtype)))
        return set_error(SKM_ERR_INVALID_ARG, "K and V must be aligned to their elements");
    KvCacheArgs a = cache_args(c, s);
    a.K = tokens_of(K, k_token, k_head, dtype);
    a.V = tokens_of(V, v_token, v_head, dtype);
    SKM_CUDA_TRY(launch_kv_write(a, dtype, S(stream)));
    return SKM_OK;
}

int skm_kv_read(const skm_kv_cache *c, const skm_kv_seqs *s, int dtype, void *K, void *V, void *stream) {
    SKM_TRY(check_cache(c));
    SKM_TRY(check_seqs(c, s));
    SKM_TRY(check_dtype(dtype));
    SKM_TRY(check_grid(c, s));
    if (most_tokens(s) == 0) return SKM_OK;
    if (!K && !V) return set_error(SKM_ERR_INVALID_ARG, "K and V are both NULL");
    if (!aligned(K, 16) || !aligned(V, 16)) return set_error(SKM_ERR_INVALID_ARG, "K and V must be 16-byte aligned");
    KvCacheArgs a = cache_args(c, s);
    a.outk = K;
    a.outv = V;
    SKM_CUDA_TRY(launch_kv_read(a, dtype, S(stream)));
    return SKM_OK;
}

size_t skm_kv_attend_workspace_size(const skm_kv_cache *c, const skm_kv_seqs *s, const skm_kv_attn *a) {
    if (check_attend(c, s, a) != SKM_OK) return (size_t)-1;
    if (most_tokens(s) == 0) return 0;
    // the most that any call of these sizes or smaller ones takes: fewer rows may
    // mean another tile, or more CTAs that share a row
    const int64_t span = std::min<int64_t>(s->max_len, (int64_t)s->cols * c->page);
    const int64_t rows = (int64_t)most_tokens(s) * (a->heads_q / c->heads);
    size_t most = kv_rows_part_most(std::min<int>(s->batch, KV_MAX_SEQS), c->heads, c->d, a->dtype, rows, span);
    if (a->dtype != SKM_DTYPE_F32 && rows > KV_ROWS_MOST) most = std::max(most, kv_prompt_part_most(c->d, span));
    return most;
}

int skm_kv_attend(const skm_kv_cache *c, const skm_kv_seqs *s, const skm_kv_attn *a, void *ws, size_t ws_bytes,
                  void *stream) {
    SKM_TRY(check_attend(c, s, a));
    if (most_tokens(s) == 0) return SKM_OK;
    const size_t e = elem_of(a->dtype);
    if (!a->Q || !a->out) return set_error(SKM_ERR_INVALID_ARG, "Q or out is NULL");
    if (!aligned(a->Q, e) || !aligned(a->out, 16) || !aligned(a->lse, 4) || !aligned(a->status, 4))
        return set_error(SKM_ERR_INVALID_ARG, "out must be 16-byte aligned, Q, lse and status to their elements");
    Carver cv(ws, ws_bytes);
    const AttendPlan p = plan_attend(c, s, a, cv);
    if (cv.off && !ws) return set_error(SKM_ERR_INVALID_ARG, "workspace is NULL (%zu bytes needed)", cv.off);
    if (!aligned(ws, 256)) return set_error(SKM_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    if (!cv.fits() || fault_take(SKM_FAULT_WORKSPACE))
        return set_error(SKM_ERR_NO_MEMORY, "workspace of %zu bytes, %zu needed", ws_bytes, cv.off);
    const int64_t ctas = p.prompt ? p.many.units * std::max(p.many.splits, 32) : p.rows.units;
    if (ctas > 0x7fffffff) return set_error(SKM_ERR_UNSUPPORTED, "too many row tiles");
    KvAttnArgs k = {};
    k.k = c->k;
    k.v = c->v;
    k.scales = reinterpret_cast<const float2 *>(c->scales);
    k.table = s->table;
    k.pos = s->pos;
    k.cu = s->cu;
    k.heads = c->heads;
    k.d = c->d;
    k.page = c->page;
    k.pages = c->pages;
    k.bpp = c->page / KV_B;
    k.cols = s->cols;
    k.tokens = s->tokens;
    k.max_tokens = most_tokens(s);
    k.group = a->heads_q / c->heads;
    k.by_heads = FastDiv(k.heads);
    k.by_group = FastDiv(k.group);
    k.by_bpp = FastDiv(k.bpp);
    k.causal = a->causal != 0;
    k.window = (int)std::min<int64_t>(a->window, KV_MOST);
    k.dtype = a->dtype;
    k.scale_log2 = (float)(a->scale * 1.4426950408889634);
    k.Q = a->Q;
    k.q_token = a->q_token;
    k.q_head = a->q_head;
    k.q_wide = aligned(a->Q, 4 * e) && a->q_token % 4 == 0 && a->q_head % 4 == 0;
    k.out = a->out;
    k.lse = a->lse;
    k.status = a->status;
    k.part_cta = p.part_cta;
    k.part_warp = p.part_warp;
    k.max_tiles = p.prompt ? p.many.max_tiles : (int)cdiv((int64_t)k.max_tokens * k.group, p.rows.rt);
    k.whole = p.rows.whole;
    k.wait_ns = KV_WAIT_NS;
    k.stuck = -1;
    if (!p.prompt && fault_take(SKM_FAULT_WAIT)) {
        k.wait_ns = KV_WAIT_NS_INJECTED;
        k.stuck = skm_fault_armed(SKM_FAULT_WAIT);
    }
    for (k.b0 = 0; k.b0 < s->batch; k.b0 += p.seqs) {
        k.nb = std::min(s->batch - k.b0, p.seqs);
        if (p.prompt) {
            KvPromptPlan q = p.many;
            q.units = (int64_t)k.nb * k.heads * k.max_tiles;
            SKM_CUDA_TRY(launch_kv_prompt(k, q, S(stream)));
        } else {
            KvRowsPlan q = p.rows;
            q.units = (int64_t)k.nb * k.max_tiles * k.heads;
            if (q.whole) q.grid = q.units;
            SKM_CUDA_TRY(launch_kv_rows(k, q, S(stream)));
        }
    }
    return SKM_OK;
}

}  // extern "C"

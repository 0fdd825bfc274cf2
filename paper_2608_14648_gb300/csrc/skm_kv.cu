// extern "C" entry points of the key/value caches (8-bit, 4-bit) and of rotary positions (declared
// in include/skm.h): argument checks on the host, workspace carving, launches.
#include <algorithm>

#include "skm_kv.cuh"

namespace skm {

namespace {

constexpr int64_t KV_MOST = int64_t(1) << 30;  // tokens of a call, positions of a sequence

cudaStream_t S(void *s) { return static_cast<cudaStream_t>(s); }
bool aligned(const void *p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// A cache of either format: what the checks and launches of both need of it
struct Cache {
    int heads, d, page, pages;
    uint8_t *k, *v;  // 4-bit: the blocks, not used
    float *scales;   // 4-bit: not used
    bool four;
};
Cache view(const skm_kv_cache &c) { return Cache{c.heads, c.d, c.page, c.pages, c.k, c.v, c.scales, false}; }
Cache view(const skm_kv4_cache &c) { return Cache{c.heads, c.d, c.page, c.pages, c.blocks, nullptr, nullptr, true}; }

int check_cache(const Cache *c) {
    if (!c) return set_error(SKM_ERR_INVALID_ARG, "the cache is NULL");
    if (c->heads < 1 || c->pages < 1)
        return set_error(SKM_ERR_INVALID_ARG, "heads = %d, pages = %d: both must be positive", c->heads, c->pages);
    if (c->d < 1 || c->page < 1) return set_error(SKM_ERR_INVALID_ARG, "d = %d, page = %d", c->d, c->page);
    if (c->d % KV_B || c->d > 256)
        return set_error(SKM_ERR_UNSUPPORTED, "d = %d: a multiple of 16 up to 256", c->d);
    if (c->page % KV_B) return set_error(SKM_ERR_UNSUPPORTED, "page = %d: a multiple of 16", c->page);
    if (cdiv((int64_t(1) << 31) - 1, (int64_t)c->heads * (c->page / KV_B)) <= c->pages)
        return set_error(SKM_ERR_UNSUPPORTED, "pages * heads * page / 16 must be below 2^31");
    if (c->four) {
        if (!c->k) return set_error(SKM_ERR_INVALID_ARG, "the cache's blocks are NULL");
        if (!aligned(c->k, 16)) return set_error(SKM_ERR_INVALID_ARG, "blocks must be 16-byte aligned");
        return SKM_OK;
    }
    if (!c->k || !c->v || !c->scales) return set_error(SKM_ERR_INVALID_ARG, "the cache's k, v or scales is NULL");
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->scales, 8))
        return set_error(SKM_ERR_INVALID_ARG, "k and v must be 16-byte, scales 8-byte aligned");
    return SKM_OK;
}

int check_seqs(const Cache *c, const skm_kv_seqs *s) {
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

KvCacheArgs cache_args(const Cache *c, const skm_kv_seqs *s) {
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
int check_grid(const Cache *c, const skm_kv_seqs *s) {
    const int64_t blocks = (most_tokens(s) + 2 * KV_B - 2) / KV_B;
    if ((double)s->batch * blocks * c->heads > 1e9)
        return set_error(SKM_ERR_UNSUPPORTED, "batch * max_tokens * heads is too large");
    return SKM_OK;
}

KvTokens tokens_of(const void *x, int64_t token, int64_t head, int dtype) {
    const size_t e = elem_of(dtype);
    return KvTokens{x, token, head, aligned(x, 16) && token * e % 16 == 0 && head * e % 16 == 0};
}

int check_attn(const Cache *c, const skm_kv_seqs *s, const skm_kv_attn *a) {
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
int64_t span_of(const Cache *c, const skm_kv_seqs *s, const skm_kv_attn *a) {
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

AttendPlan plan_attend(const Cache *c, const skm_kv_seqs *s, const skm_kv_attn *a, Carver &cv) {
    AttendPlan p;
    const int nb = p.seqs = std::min<int>(s->batch, KV_MAX_SEQS), group = a->heads_q / c->heads, most = most_tokens(s);
    p.prompt = kv_prompt_ok(a->dtype, nb, c->heads, c->d, (int64_t)most * group, span_of(c, s, a));
    if (p.prompt) {
        p.many = kv_prompt_plan(nb, c->heads, group, c->d, most, span_of(c, s, a));
        if (p.many.part) p.part_cta = cv.take<float>(p.many.part / 4);
    } else {
        p.rows = (c->four ? kv4_rows_plan : kv_rows_plan)(nb, c->heads, group, c->d, a->dtype, most, span_of(c, s, a));
        p.seqs = p.rows.seqs;
        if (p.rows.part_cta) p.part_cta = cv.take<float>(p.rows.part_cta / 4);
        if (p.rows.part_warp) p.part_warp = cv.take<float>(p.rows.part_warp / 4);
    }
    return p;
}

int check_attend(const Cache *c, const skm_kv_seqs *s, const skm_kv_attn *a) {
    SKM_TRY(check_cache(c));
    SKM_TRY(check_seqs(c, s));
    return check_attn(c, s, a);
}

int write_rows(const Cache *c, const skm_kv_seqs *s, int dtype, const void *K, int64_t k_token, int64_t k_head,
               const void *V, int64_t v_token, int64_t v_head, void *stream) {
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
    SKM_CUDA_TRY((c->four ? launch_kv4_write : launch_kv_write)(a, dtype, S(stream)));
    return SKM_OK;
}

int read_rows(const Cache *c, const skm_kv_seqs *s, int dtype, void *K, void *V, void *stream) {
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
    SKM_CUDA_TRY((c->four ? launch_kv4_read : launch_kv_read)(a, dtype, S(stream)));
    return SKM_OK;
}

size_t attend_workspace_size(const Cache *c, const skm_kv_seqs *s, const skm_kv_attn *a) {
    if (check_attend(c, s, a) != SKM_OK) return (size_t)-1;
    if (most_tokens(s) == 0) return 0;
    // the most that any call of these sizes or smaller ones takes: fewer rows may
    // mean another tile, or more CTAs that share a row
    const int64_t span = std::min<int64_t>(s->max_len, (int64_t)s->cols * c->page);
    const int64_t rows = (int64_t)most_tokens(s) * (a->heads_q / c->heads);
    size_t most = (c->four ? kv4_rows_part_most : kv_rows_part_most)(std::min<int>(s->batch, KV_MAX_SEQS), c->heads, c->d, a->dtype, rows, span);
    if (a->dtype != SKM_DTYPE_F32 && rows > KV_ROWS_MOST) most = std::max(most, kv_prompt_part_most(c->d, span));
    return most;
}

int attend(const Cache *c, const skm_kv_seqs *s, const skm_kv_attn *a, void *ws, size_t ws_bytes, void *stream) {
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
    // a 4-bit vector's largest code may stand for more than f16 holds, and so may a mean of them
    k.most = c->four ? 65504.0f : INFINITY;
    k.part_cta = p.part_cta;
    k.part_warp = p.part_warp;
    k.max_tiles = p.prompt ? p.many.max_tiles : (int)cdiv((int64_t)k.max_tokens * k.group, p.rows.rt);
    k.whole = p.rows.whole;
    k.wait_ns = KV_WAIT_NS;
    k.stuck = -1;
    if ((!p.prompt || c->four) && fault_take(SKM_FAULT_WAIT)) {
        k.wait_ns = KV_WAIT_NS_INJECTED;
        k.stuck = skm_fault_armed(SKM_FAULT_WAIT);
    }
    for (k.b0 = 0; k.b0 < s->batch; k.b0 += p.seqs) {
        k.nb = std::min(s->batch - k.b0, p.seqs);
        if (p.prompt) {
            KvPromptPlan q = p.many;
            q.units = (int64_t)k.nb * k.heads * k.max_tiles;
            SKM_CUDA_TRY((c->four ? launch_kv4_prompt : launch_kv_prompt)(k, q, S(stream)));
        } else {
            KvRowsPlan q = p.rows;
            q.units = (int64_t)k.nb * k.max_tiles * k.heads;
            if (q.whole) q.grid = q.units;
            SKM_CUDA_TRY((c->four ? launch_kv4_rows : launch_kv_rows)(k, q, S(stream)));
        }
    }
    return SKM_OK;
}

// The entry points of a cache: on a view of it, or on nothing
template <class C, class F>
auto with(const C *c, F &&f) {
    if (!c) return f(static_cast<const Cache *>(nullptr));
    const Cache v = view(*c);
    return f(&v);
}

constexpr int ROTARY_D_MOST = 1024;

// Whether two of a tensor's rows (tokens x heads, d elements each) share an element.  Rows (t, h) and (t + i, h + j) do where
// |i token + j head| < d: of each j >= 0 the i on either side of -j head / token are looked at, unless one stride spans
// all that the other does
bool rows_overlap(int64_t tokens, int64_t heads, int64_t token, int64_t head, int64_t d) {
    using Wide = __int128;
    const auto size = [](Wide x) { return x < 0 ? -x : x; };
    const Wide t = tokens > 1 ? size(token) : 0, h = heads > 1 ? size(head) : 0;
    if ((tokens > 1 && t < d) || (heads > 1 && h < d)) return true;
    if (tokens == 1 || heads == 1 || t >= (heads - 1) * h + d || h >= (tokens - 1) * t + d) return false;
    for (int64_t j = 1; j < heads; ++j) {  // (the sign of either stride only mirrors the rows)
        const Wide i = j * h / t;
        if ((i < tokens && j * h - i * t < d) || (i + 1 < tokens && (i + 1) * t - j * h < d)) return true;
    }
    return false;
}

}  // namespace

}  // namespace skm

using namespace skm;

extern "C" {

int skm_kv_write(const skm_kv_cache *c, const skm_kv_seqs *s, int dtype, const void *K, int64_t k_token,
                 int64_t k_head, const void *V, int64_t v_token, int64_t v_head, void *stream) {
    return with(c, [&](const Cache *v) { return write_rows(v, s, dtype, K, k_token, k_head, V, v_token, v_head, stream); });
}
int skm_kv4_write(const skm_kv4_cache *c, const skm_kv_seqs *s, int dtype, const void *K, int64_t k_token,
                  int64_t k_head, const void *V, int64_t v_token, int64_t v_head, void *stream) {
    return with(c, [&](const Cache *v) { return write_rows(v, s, dtype, K, k_token, k_head, V, v_token, v_head, stream); });
}

int skm_kv_read(const skm_kv_cache *c, const skm_kv_seqs *s, int dtype, void *K, void *V, void *stream) {
    return with(c, [&](const Cache *v) { return read_rows(v, s, dtype, K, V, stream); });
}
int skm_kv4_read(const skm_kv4_cache *c, const skm_kv_seqs *s, int dtype, void *K, void *V, void *stream) {
    return with(c, [&](const Cache *v) { return read_rows(v, s, dtype, K, V, stream); });
}

size_t skm_kv_attend_workspace_size(const skm_kv_cache *c, const skm_kv_seqs *s, const skm_kv_attn *a) {
    return with(c, [&](const Cache *v) { return attend_workspace_size(v, s, a); });
}
size_t skm_kv4_attend_workspace_size(const skm_kv4_cache *c, const skm_kv_seqs *s, const skm_kv_attn *a) {
    return with(c, [&](const Cache *v) { return attend_workspace_size(v, s, a); });
}

int skm_kv_attend(const skm_kv_cache *c, const skm_kv_seqs *s, const skm_kv_attn *a, void *ws, size_t ws_bytes,
                  void *stream) {
    return with(c, [&](const Cache *v) { return attend(v, s, a, ws, ws_bytes, stream); });
}
int skm_kv4_attend(const skm_kv4_cache *c, const skm_kv_seqs *s, const skm_kv_attn *a, void *ws, size_t ws_bytes,
                   void *stream) {
    return with(c, [&](const Cache *v) { return attend(v, s, a, ws, ws_bytes, stream); });
}

int skm_rotary_turns(const skm_rotary_config *cfg, uint64_t *turns, float *gain) {
    if (!cfg || !turns || !gain) return set_error(SKM_ERR_INVALID_ARG, "cfg, turns or gain is NULL");
    const int dims = cfg->dims;
    if (dims < 2 || dims % 2 || dims > ROTARY_D_MOST)
        return set_error(SKM_ERR_INVALID_ARG, "dims = %d: an even number up to %d", dims, ROTARY_D_MOST);
    if (cfg->scaling < SKM_ROTARY_NONE || cfg->scaling > SKM_ROTARY_TURNS)
        return set_error(SKM_ERR_INVALID_ARG, "unknown scaling %d", cfg->scaling);
    const auto above = [](double x, double least) { return x > least && x - x == 0.0; };
    if (!above(cfg->base, 1.0)) return set_error(SKM_ERR_INVALID_ARG, "base must be above 1 and finite");
    if (cfg->scaling != SKM_ROTARY_NONE && !above(cfg->factor, 0.0))
        return set_error(SKM_ERR_INVALID_ARG, "factor must be positive and finite");
    const bool parts = cfg->scaling == SKM_ROTARY_INDEX || cfg->scaling == SKM_ROTARY_TURNS;
    if (parts && !(above(cfg->trained, 0.0) && above(cfg->low, 0.0) && above(cfg->high, cfg->low)))
        return set_error(SKM_ERR_INVALID_ARG, "trained, low and high must be finite, with 0 < trained and 0 < low < high");
    constexpr double CIRCLE = 6.283185307179586476925;
    double base = cfg->base;
    if (cfg->scaling == SKM_ROTARY_BASE && dims > 2) base *= pow(cfg->factor, (double)dims / (dims - 2));
    if (!above(base, 1.0)) return set_error(SKM_ERR_INVALID_ARG, "the scaled base must be above 1 and finite");
    const auto pair_of = [&](double turns_trained) {  // the pair that turns so often over the trained length
        return dims * log(cfg->trained / (turns_trained * CIRCLE)) / (2 * log(cfg->base));
    };
    double first = 0.0, width = 1.0;
    *gain = 1.0f;
    if (cfg->scaling == SKM_ROTARY_INDEX) {
        first = fmax(floor(pair_of(cfg->high)), 0.0);
        width = fmax(fmin(ceil(pair_of(cfg->low)), dims - 1.0) - first, 0.001);
        *gain = (float)(cfg->factor > 1.0 ? 0.1 * log(cfg->factor) + 1.0 : 1.0);
    }
    for (int i = 0; i < dims / 2; ++i) {
        double f = pow(base, -2.0 * i / dims), keep = 1.0;
        if (cfg->scaling == SKM_ROTARY_LINEAR) keep = 0.0;
        if (cfg->scaling == SKM_ROTARY_INDEX) keep = 1.0 - fmin(fmax((i - first) / width, 0.0), 1.0);
        if (cfg->scaling == SKM_ROTARY_TURNS)
            keep = fmin(fmax((cfg->trained * f / CIRCLE - cfg->low) / (cfg->high - cfg->low), 0.0), 1.0);
        if (keep < 1.0) f = f * keep + f / cfg->factor * (1.0 - keep);
        // of a turn a position, the part below one, in units of 2^-64
        const double turn = f / CIRCLE, part = turn - floor(turn);
        const double units = nearbyint(ldexp(part, 64));
        turns[i] = units < 18446744073709551616.0 ? (uint64_t)units : 0;
    }
    return SKM_OK;
}

int skm_kv_rotate(const skm_kv_seqs *s, const skm_rotary *r, int d, int dtype, const skm_rotary_rows *rows, int count,
                  void *stream) {
    if (!s || !r || !rows) return set_error(SKM_ERR_INVALID_ARG, "skm_kv_seqs, skm_rotary or skm_rotary_rows is NULL");
    if (s->batch < 1) return set_error(SKM_ERR_INVALID_ARG, "batch = %d must be positive", s->batch);
    if (s->tokens < 0 || s->max_tokens < 0)
        return set_error(SKM_ERR_INVALID_ARG, "tokens = %d, max_tokens = %d", s->tokens, s->max_tokens);
    if (s->tokens >= KV_MOST || s->batch >= KV_MOST) return set_error(SKM_ERR_UNSUPPORTED, "tokens and batch must be below 2^30");
    if (!s->pos || !s->cu) return set_error(SKM_ERR_INVALID_ARG, "pos or cu is NULL");
    SKM_TRY(check_dtype(dtype));
    if (d < 1 || d > ROTARY_D_MOST) return set_error(SKM_ERR_INVALID_ARG, "d = %d: up to %d", d, ROTARY_D_MOST);
    if (r->dims < 2 || r->dims % 2 || r->dims > d) return set_error(SKM_ERR_INVALID_ARG, "dims = %d: an even number up to d = %d", r->dims, d);
    if (r->layout != SKM_ROTARY_HALF && r->layout != SKM_ROTARY_INTERLEAVED)
        return set_error(SKM_ERR_INVALID_ARG, "unknown layout %d", r->layout);
    if (!(r->gain - r->gain == 0.0f)) return set_error(SKM_ERR_INVALID_ARG, "gain is not finite");
    if (!r->turns || !aligned(r->turns, 8)) return set_error(SKM_ERR_INVALID_ARG, "turns is NULL or not 8-byte aligned");
    if (count < 1 || count > 2) return set_error(SKM_ERR_INVALID_ARG, "count = %d: one or two tensors", count);
    const size_t e = elem_of(dtype);
    RotaryArgs a = {};
    int vec = (int)(16 / e);  // elements that every vector of the call is aligned to
    const auto narrow = [&](int64_t multiple) {
        while (vec > 1 && multiple % vec) vec /= 2;
    };
    bool in_place = true;
    for (int i = 0; i < count; ++i) {
        const skm_rotary_rows &p = rows[i];
        if (p.heads < 1 || p.heads > 65536) return set_error(SKM_ERR_INVALID_ARG, "heads = %d", p.heads);
        if (most_tokens(s) == 0) continue;
        if (!p.x || !p.y) return set_error(SKM_ERR_INVALID_ARG, "x or y is NULL");
        if (!aligned(p.x, e) || !aligned(p.y, e)) return set_error(SKM_ERR_INVALID_ARG, "x and y must be aligned to their elements");
        if (p.x == p.y && (p.x_token != p.y_token || p.x_head != p.y_head))
            return set_error(SKM_ERR_INVALID_ARG, "in place, x and y must have the same strides");
        if (rows_overlap(s->tokens, p.heads, p.y_token, p.y_head, d))
            return set_error(SKM_ERR_INVALID_ARG, "y's rows overlap: strides %lld and %lld for rows of %d", (long long)p.y_token, (long long)p.y_head, d);
        if (i == 1 && (p.y == rows[0].y || p.y == rows[0].x || p.x == rows[0].y))
            return set_error(SKM_ERR_INVALID_ARG, "y of one tensor is x or y of the other");
        if (p.x != p.y) in_place = false;
        narrow((int64_t)(reinterpret_cast<uintptr_t>(p.x) / e));
        narrow((int64_t)(reinterpret_cast<uintptr_t>(p.y) / e));
        for (const int64_t stride : {p.x_token, p.x_head, p.y_token, p.y_head}) narrow(stride);
        a.part[i] = RotaryPart{p.x, p.y, p.x_token, p.x_head, p.y_token, p.y_head, p.heads};
        a.heads = std::max(a.heads, p.heads);
    }
    if (most_tokens(s) == 0) return SKM_OK;
    a.copied = in_place ? 0 : d - r->dims;  // (a tensor that is in place beside one that is not: its dims onto themselves)
    narrow(r->layout == SKM_ROTARY_HALF ? r->dims / 2 : r->dims);
    narrow(a.copied);
    if ((double)s->tokens * a.heads > 5e8) return set_error(SKM_ERR_UNSUPPORTED, "tokens * heads is too large");
    a.pos = s->pos;
    a.cu = s->cu;
    a.turns = r->turns;
    a.batch = s->batch;
    a.tokens = s->tokens;
    a.max_tokens = most_tokens(s);
    a.dims = r->dims;
    a.interleaved = r->layout == SKM_ROTARY_INTERLEAVED;
    a.gain = r->gain;
    a.sine = r->transpose ? -r->gain : r->gain;
    SKM_CUDA_TRY(launch_rotary(a, dtype, vec, S(stream)));
    return SKM_OK;
}

}  // extern "C"

// C ABI of attention and of the paged cache: argument checks and launches.
#include "eigenpro.h"
#include "attn.h"
#include "ep_host.h"
#include "ep_internal.h"

#include <cmath>

using namespace ep;

namespace {

constexpr int64_t kMaxTokens = int64_t(1) << 30;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

#define REQUIRE(cond, ...)                                \
    do {                                                  \
        if (!(cond)) return fail(EP_EINVAL, __VA_ARGS__); \
    } while (0)

int check_attn(const ep_attn* a, bool packed_keys) {
    REQUIRE(a, "NULL arguments");
    REQUIRE(a->type == EP_BF16 || a->type == EP_FP16, "type must be EP_BF16 or EP_FP16");
    REQUIRE(a->batch >= 1 && a->batch < (1 << 24), "batch must be in [1, 2^24)");
    REQUIRE(a->kv_heads >= 1 && a->kv_heads < (1 << 16), "kv_heads must be in [1, 65535]");
    REQUIRE(a->heads >= 1 && a->heads % a->kv_heads == 0 && a->heads / a->kv_heads <= 1024,
            "heads must be a multiple of kv_heads, at most 1024 times as many");
    REQUIRE(a->dim >= 8 && a->dim <= 128 && a->dim % 8 == 0,
            "dim must be a multiple of 8 in [8, 128]");
    REQUIRE(a->tokens_q >= 0 && a->tokens_q < kMaxTokens, "tokens_q must be in [0, 2^30)");
    const int64_t group = a->heads / a->kv_heads;
    REQUIRE(a->tokens_q * group < kMaxTokens && a->tokens_q * group * group < int64_t(1) << 32,
            "with group = heads / kv_heads, tokens_q * group must be below 2^30 and tokens_q * "
            "group^2 below 2^32");
    REQUIRE(attn_groups(a->kv_heads, a->tokens_q * group, kFewRows, a->batch) <= kMaxGroups &&
                (!packed_keys ||
                 attn_groups(a->kv_heads, a->tokens_k, kRowTile, a->batch) <= kMaxGroups / 2),
            "too many workgroups: kv_heads * (tokens_q * (heads / kv_heads) / 32 + batch) must be "
            "below 2^24, kv_heads * (tokens_k / 128 + batch) below 2^23");
    REQUIRE(std::isfinite(a->scale * kLog2e) && a->scale > 0.f,
            "scale must be positive, scale * log2(e) finite");
    REQUIRE(a->causal == 0 || a->causal == 1, "causal must be 0 or 1");
    REQUIRE(a->window >= 0 && a->window < kMaxTokens, "window must be in [0, 2^30)");
    REQUIRE(a->window == 0 || a->causal, "a window needs causal");
    REQUIRE(a->start_q, "start_q is NULL");
    if (packed_keys) {
        REQUIRE(a->tokens_k >= 0 && a->tokens_k < kMaxTokens, "tokens_k must be in [0, 2^30)");
        REQUIRE(a->start_k, "start_k is NULL");
    }
    return EP_OK;
}

// Whether rows of dim elements meet, where neither axis' stride is below dim:
// token t of head i + h and token t + s of head i, s row within dim of h head.
// Strides of which one spans the whole other axis are apart at a glance.
bool rows_meet(const ep_rows& r, int64_t tokens, int64_t heads, int64_t dim) {
    if (tokens == 1 || heads == 1) return false;
    // (row < 2^24 and tokens < 2^30, so nothing here passes 64 bits)
    if (r.head >= (tokens - 1) * r.row + dim) return false;
    if (r.head <= r.row && r.row >= (heads - 1) * r.head + dim) return false;
    for (int64_t h = 1; h < heads; ++h) {
        const int64_t at = h * r.head, s = at / r.row;
        if (s >= tokens) return false;
        if ((s >= 1 && at - s * r.row < dim) || (s + 1 < tokens && (s + 1) * r.row - at < dim)) return true;
    }
    return false;
}

// (data may be NULL where there are no rows)
// dim: of an output, whose rows must lie apart; 0: of an input.
int check_rows(const char* name, const ep_rows& r, int64_t tokens, int64_t heads, int64_t dim) {
    if (tokens == 0) return EP_OK;
    REQUIRE(r.data, "%s is NULL", name);
    REQUIRE(aligned16(r.data), "%s must be 16-byte aligned", name);
    // (the stride of an axis of one element counts for nothing)
    REQUIRE(tokens == 1 || (r.row % 8 == 0 && r.row >= dim && r.row < (1 << 24)),
            "%s: the rows' stride must be a multiple of 8 elements in [%d, 2^24)", name, (int)dim);
    REQUIRE(heads == 1 || (r.head % 8 == 0 && r.head >= dim),
            "%s: the heads' stride must be a multiple of 8 elements, at least %d", name, (int)dim);
    REQUIRE(dim == 0 || !rows_meet(r, tokens, heads, dim),
            "%s: its rows overlap: strides of %lld and %lld elements for %lld tokens of %lld heads",
            name, (long long)r.row, (long long)r.head, (long long)tokens, (long long)heads);
    return EP_OK;
}

int check_cache(const ep_cache* c, const ep_pages* p, int type) {
    REQUIRE(c && p, "NULL cache or pages");
    REQUIRE(type == EP_BF16 || type == EP_FP16, "type must be EP_BF16 or EP_FP16");
    REQUIRE(c->type == EP_E4M3 || c->type == type,
            "the cache must hold the call's type or EP_E4M3");
    REQUIRE(c->pages >= 1 && c->pages < int64_t(1) << 31, "pages must be in [1, 2^31)");
    REQUIRE(c->page_size >= 1 && c->page_size <= 65536 && (c->page_size & (c->page_size - 1)) == 0,
            "page_size must be a power of two in [1, 65536]");
    REQUIRE(c->kv_heads >= 1 && c->kv_heads < (1 << 16), "kv_heads must be in [1, 65535]");
    REQUIRE(c->dim >= 8 && c->dim <= 128 && c->dim % 8 == 0,
            "dim must be a multiple of 8 in [8, 128]");
    REQUIRE(c->k && c->v && aligned16(c->k) && aligned16(c->v),
            "the pages must be 16-byte aligned and not NULL");
    REQUIRE(c->type != EP_E4M3 || (c->k_scale && c->v_scale), "an EP_E4M3 cache needs scales");
    REQUIRE(p->batch >= 1 && p->batch < (1 << 24), "batch must be in [1, 2^24)");
    REQUIRE(p->cols >= 1 && p->cols < kMaxTokens / c->page_size,
            "cols * page_size must be positive and below 2^30");
    REQUIRE(p->table && p->lengths, "table or lengths is NULL");
    return EP_OK;
}

#define TRY(expr)                     \
    do {                              \
        const int rc_ = (expr);       \
        if (rc_ != EP_OK) return rc_; \
    } while (0)

Rows rows_of(const ep_rows& r) { return {static_cast<char*>(r.data), 2 * r.row, 2 * r.head}; }

int shift_of(int64_t page_size) {
    int s = 0;
    while ((int64_t(1) << s) < page_size) ++s;
    return s;
}

AttnArgs args_of(const ep_attn* a) {
    AttnArgs g{};
    g.start_q = a->start_q;
    g.start_k = a->start_k;
    g.tokens_q = a->tokens_q;
    g.tokens_k = a->tokens_k;
    g.batch = (int)a->batch;
    g.heads = (int)a->heads;
    g.kv_heads = (int)a->kv_heads;
    g.group = (int)(a->heads / a->kv_heads);
    g.group_magic = group_magic(g.group);
    g.dim = (int)a->dim;
    g.scale = a->scale;
    g.scale_log2 = a->scale * kLog2e;
    g.causal = a->causal;
    g.window = (int)a->window;
    return g;
}

// Where a plan's partial results go.
void set_plan(AttnArgs& g, const AttnPlan& p, void* work) {
    g.splits = p.splits;
    g.part = static_cast<float*>(work);
    g.part_lse = g.part + (p.splits > 1 ? p.splits * g.tokens_q * g.heads * g.dim : 0);
}

int launched(hipError_t e) {
    if (e != hipSuccess) return fail(EP_EDEVICE, "launch: %s", hipGetErrorString(e));
    return EP_OK;
}

// keys: of a sequence, as far as the host can tell.
AttnPlan plan_of(const ep_attn* a, int64_t keys) {
    if (a->window) keys = std::min(keys, a->window + kRowTile);
    return attn_plan(a->batch, a->tokens_q, a->heads, a->kv_heads, a->dim, keys);
}
// Packed sequences: twice the average, for ragged ones.
AttnPlan plan_packed(const ep_attn* a) {
    return plan_of(a, std::min(a->tokens_k, 2 * ceil_div(a->tokens_k, a->batch)));
}

// The gradients' work: log-sums and D, then partial sums of dk and dv, then of
// dq.
struct GradientWork {
    int key_splits, row_splits;
    int64_t part_kv, part_q, bytes;      // where they start, and the end
};
GradientWork gradient_work(const ep_attn* a) {
    GradientWork w;
    w.key_splits = attn_key_splits(a->batch, a->tokens_q, a->tokens_k, a->heads, a->kv_heads);
    w.row_splits = attn_row_splits(a->batch, a->tokens_q, a->tokens_k, a->heads, a->kv_heads);
    w.part_kv = round_up(a->tokens_q * a->heads * 8, 16);
    w.part_q = w.part_kv + (w.row_splits > 1 ? w.row_splits * a->tokens_k * a->kv_heads * a->dim * 8 : 0);
    w.bytes = w.part_q + (w.key_splits > 1 ? w.key_splits * a->tokens_q * a->heads * a->dim * 4 : 0);
    return w;
}

int check_work(const void* work, int64_t bytes, int64_t need) {
    REQUIRE(bytes >= need && (work || need == 0) && aligned16(work),
            "work must be 16-byte aligned and hold %lld bytes", (long long)need);
    return EP_OK;
}

CacheArgs cache_args(const ep_cache* c, const ep_pages* p, const ep_rows& k, const ep_rows& v,
                     int64_t tokens, const int32_t* start) {
    CacheArgs g{};
    g.k = rows_of(k);
    g.v = rows_of(v);
    g.kp = static_cast<char*>(c->k);
    g.vp = static_cast<char*>(c->v);
    g.ks = c->k_scale;
    g.vs = c->v_scale;
    g.table = p->table;
    g.cols = p->cols;
    g.lengths = p->lengths;
    g.start = start;
    g.tokens = tokens;
    g.batch = (int)p->batch;
    g.kv_heads = (int)c->kv_heads;
    g.dim = (int)c->dim;
    g.pages = (int)c->pages;
    g.page_shift = shift_of(c->page_size);
    g.err = p->err;
    return g;
}

int check_move(const ep_cache* c, const ep_pages* p, int type, const ep_rows& k, const ep_rows& v,
               int64_t tokens, const int32_t* start, bool out) {
    TRY(check_cache(c, p, type));
    REQUIRE(tokens >= 0 && tokens < kMaxTokens, "tokens must be in [0, 2^30)");
    REQUIRE(start, "start is NULL");
    TRY(check_rows("k", k, tokens, c->kv_heads, out ? c->dim : 0));
    TRY(check_rows("v", v, tokens, c->kv_heads, out ? c->dim : 0));
    return EP_OK;
}

int check_cached(const ep_attn* a, const ep_cache* c, const ep_pages* p) {
    TRY(check_attn(a, false));
    TRY(check_cache(c, p, a->type));
    REQUIRE(c->kv_heads == a->kv_heads && c->dim == a->dim && p->batch == a->batch,
            "cache and call differ in kv_heads, dim or batch");
    return EP_OK;
}

}  // namespace

extern "C" int64_t ep_attention_bytes(const ep_attn* a) {
    TRY(check_attn(a, true));
    return plan_packed(a).bytes;
}

extern "C" int ep_attention(const ep_attn* a, ep_rows q, ep_rows k, ep_rows v, ep_rows out,
                            float* lse, void* work, int64_t work_bytes, void* hip_stream) {
    TRY(check_attn(a, true));
    TRY(check_rows("q", q, a->tokens_q, a->heads, 0));
    TRY(check_rows("out", out, a->tokens_q, a->heads, a->dim));
    TRY(check_rows("k", k, a->tokens_k, a->kv_heads, 0));
    TRY(check_rows("v", v, a->tokens_k, a->kv_heads, 0));
    const AttnPlan plan = plan_packed(a);
    TRY(check_work(work, work_bytes, plan.bytes));
    if (a->tokens_q == 0) return EP_OK;
    AttnArgs g = args_of(a);
    set_plan(g, plan, work);
    g.q = rows_of(q);
    g.k = rows_of(k);
    g.v = rows_of(v);
    g.o = rows_of(out);
    g.lse = lse;
    return launched(attn_forward_launch(g, plan, a->type == EP_BF16, kPacked,
                                        static_cast<hipStream_t>(hip_stream)));
}

extern "C" int64_t ep_attention_backward_bytes(const ep_attn* a) {
    TRY(check_attn(a, true));
    return gradient_work(a).bytes;
}

extern "C" int ep_attention_backward(const ep_attn* a, ep_rows dout, ep_rows q, ep_rows k,
                                     ep_rows v, ep_rows out, const float* lse, ep_rows dq,
                                     ep_rows dk, ep_rows dv, void* work, int64_t work_bytes,
                                     void* hip_stream) {
    TRY(check_attn(a, true));
    const ep_rows* of_q[] = {&dout, &q, &out, &dq};
    const ep_rows* of_k[] = {&k, &v, &dk, &dv};
    const char* names[] = {"dout", "q", "out", "dq", "k", "v", "dk", "dv"};
    for (int i = 0; i < 4; ++i) {
        TRY(check_rows(names[i], *of_q[i], a->tokens_q, a->heads, i == 3 ? a->dim : 0));
        TRY(check_rows(names[4 + i], *of_k[i], a->tokens_k, a->kv_heads, i >= 2 ? a->dim : 0));
    }
    REQUIRE(lse || a->tokens_q == 0, "lse is NULL");
    const GradientWork w = gradient_work(a);
    TRY(check_work(work, work_bytes, w.bytes));
    AttnArgs g = args_of(a);
    g.dout = rows_of(dout);
    g.q = rows_of(q);
    g.k = rows_of(k);
    g.v = rows_of(v);
    g.o = rows_of(out);
    g.lse = const_cast<float*>(lse);
    g.dq = rows_of(dq);
    g.dk = rows_of(dk);
    g.dv = rows_of(dv);
    g.lse2 = static_cast<float*>(work);
    g.delta = g.lse2 + a->tokens_q * a->heads;
    g.row_splits = w.row_splits;
    g.part_kv = reinterpret_cast<float*>(static_cast<char*>(work) + w.part_kv);
    g.key_splits = w.key_splits;
    g.part_q = reinterpret_cast<float*>(static_cast<char*>(work) + w.part_q);
    return launched(attn_backward_launch(g, a->type == EP_BF16,
                                         static_cast<hipStream_t>(hip_stream)));
}

extern "C" int ep_cache_write(const ep_cache* c, const ep_pages* p, int type, ep_rows k, ep_rows v,
                              int64_t tokens, const int32_t* start, void* hip_stream) {
    TRY(check_move(c, p, type, k, v, tokens, start, false));
    if (tokens == 0) return EP_OK;
    return launched(cache_write_launch(cache_args(c, p, k, v, tokens, start), type == EP_BF16,
                                       c->type == EP_E4M3, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int ep_cache_read(const ep_cache* c, const ep_pages* p, int type, ep_rows k, ep_rows v,
                             int64_t tokens, const int32_t* start, void* hip_stream) {
    TRY(check_move(c, p, type, k, v, tokens, start, true));
    if (tokens == 0) return EP_OK;
    return launched(cache_read_launch(cache_args(c, p, k, v, tokens, start), type == EP_BF16,
                                      c->type == EP_E4M3, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int64_t ep_cache_attention_bytes(const ep_attn* a, const ep_cache* c,
                                            const ep_pages* p) {
    TRY(check_cached(a, c, p));
    return plan_of(a, p->cols * c->page_size).bytes;
}

extern "C" int ep_cache_attention(const ep_attn* a, const ep_cache* c, const ep_pages* p,
                                  ep_rows q, ep_rows out, float* lse, void* work,
                                  int64_t work_bytes, void* hip_stream) {
    TRY(check_cached(a, c, p));
    TRY(check_rows("q", q, a->tokens_q, a->heads, 0));
    TRY(check_rows("out", out, a->tokens_q, a->heads, a->dim));
    const AttnPlan plan = plan_of(a, p->cols * c->page_size);
    TRY(check_work(work, work_bytes, plan.bytes));
    if (a->tokens_q == 0) return EP_OK;
    AttnArgs g = args_of(a);
    set_plan(g, plan, work);
    const int64_t bytes = c->type == EP_E4M3 ? 1 : 2;
    g.q = rows_of(q);
    g.o = rows_of(out);
    g.lse = lse;
    g.k = {static_cast<char*>(c->k), c->kv_heads * c->dim * bytes, c->dim * bytes};
    g.v = {static_cast<char*>(c->v), c->kv_heads * c->dim * bytes, c->dim * bytes};
    g.k_scale = c->k_scale;
    g.v_scale = c->v_scale;
    g.table = p->table;
    g.cols = p->cols;
    g.lengths = p->lengths;
    g.pages = (int)c->pages;
    g.page_shift = shift_of(c->page_size);
    g.err = p->err;
    const bool small = g.page_shift < 4;
    const int source = c->type == EP_E4M3 ? (small ? kE4m3Small : kE4m3) : (small ? kPagedSmall : kPaged);
    return launched(attn_forward_launch(g, plan, a->type == EP_BF16, source,
                                        static_cast<hipStream_t>(hip_stream)));
}

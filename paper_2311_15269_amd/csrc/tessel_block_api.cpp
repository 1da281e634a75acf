// Host side of include/tessel_block_ops.h: argument checks, tiles of packed sequences, launches.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include "tessel_block.h"

using namespace tessel;

struct tessel_packing {
    int64_t tokens = 0;
    int64_t longest = 0, steps = 0;         // steps of 64 keys of the longest sequence's last tile, and of all tiles
    std::vector<AttendTile> tiles;
    const AttendTile *table = nullptr;      // device copy
};

namespace {

thread_local int last_hip = 0;

int hip_result(int e)
{
    if (e == 0) return TESSEL_OK;
    last_hip = e;
    return TESSEL_E_HIP;
}

constexpr int64_t kMostThreads = UINT32_MAX;         // of a launch
constexpr int64_t kMostStride = (int64_t)1 << 40;    // (elements; a product with a token's number stays far inside 64 bits)

constexpr int64_t kMostNear = (int64_t)1 << 24;      // (where a kernel takes 32-bit offsets over 64 rows)

int size_of(int type) { return type == TESSEL_F32 ? 4 : 2; }
bool is_type(int type) { return type == TESSEL_BF16 || type == TESSEL_F16 || type == TESSEL_F32; }
bool aligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// ---- attention
bool heads_ok(const tessel_heads &h, bool written, int heads, int dim)
{
    if (!h.data || !aligned(h.data, 16) || h.token_stride < 0 || h.head_stride < 0 || h.token_stride % 8 || h.head_stride % 8) return false;
    if (h.token_stride > kMostStride || h.head_stride > kMostStride) return false;
    return !written || (h.token_stride >= dim && (heads == 1 || h.head_stride >= dim));
}

int attention_ok(const tessel_packing *p, const tessel_attention *a)
{
    if (!p || !a || a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads || a->dim < 1) return TESSEL_E_INVALID_ARG;
    if (!(a->scale >= 0x1p-100f && a->scale <= 0x1p100f)) return TESSEL_E_INVALID_ARG;        // (the kernels divide by it)
    if ((a->type != TESSEL_BF16 && a->type != TESSEL_F16) || a->dim % 8 || a->dim > 128) return TESSEL_E_UNSUPPORTED;
    if ((int64_t)p->tiles.size() > kMostThreads / kAttendThreads / a->heads) return TESSEL_E_TOOBIG;
    return TESSEL_OK;
}

AttendLaunch attend_launch(const tessel_packing *p, const tessel_attention *a)
{
    AttendLaunch l = {};
    l.a = *a;
    l.tiles = p->table;
    l.num_tiles = (int32_t)p->tiles.size();
    l.tokens = p->tokens;
    return l;
}

// How the forward pass and dq (of which two workgroups are resident on a compute unit) and dk, dv (one) are split: over the 64-key steps of a
// tile, and the 64-query steps of a tile for all heads on its keys (of which there are as many in all).
int query_splits(const tessel_packing *p, const tessel_attention *a)
{
    return attend_splits(p->longest, p->steps * a->heads, 512, 1.6, 4.0 * p->tokens * a->heads * a->dim);
}
int key_splits(const tessel_packing *p, const tessel_attention *a)
{
    return attend_splits(p->longest * (a->heads / a->kv_heads), p->steps * a->heads, 256, 2.6, 8.0 * p->tokens * a->kv_heads * a->dim);
}

// whether launches over all tiles for `heads` heads in so many splits hold their threads, that which joins the splits among them
bool launchable(const tessel_packing *p, int heads, int splits, int threads)
{
    const int64_t blocks = (int64_t)p->tiles.size() * heads;      // (2^24 at most: attention_ok)
    return blocks * splits <= kMostThreads / threads && (splits == 1 || blocks * (kAttendRows / kJoinRows) <= kMostThreads / kAttendThreads);
}
int forward_ok(const tessel_packing *p, const tessel_attention *a)
{
    const int e = attention_ok(p, a);
    return e == TESSEL_OK && !launchable(p, a->heads, query_splits(p, a), kAttendThreads) ? TESSEL_E_TOOBIG : e;
}
int backward_ok(const tessel_packing *p, const tessel_attention *a)
{
    const int e = forward_ok(p, a);
    return e == TESSEL_OK && !launchable(p, a->kv_heads, key_splits(p, a), kDkvThreads) ? TESSEL_E_TOOBIG : e;
}

size_t forward_workspace(const tessel_packing *p, const tessel_attention *a)
{
    const int s = query_splits(p, a);
    return s > 1 ? (size_t)s * p->tokens * a->heads * (a->dim + 2) * sizeof(float) : 0;
}

// delta, then the parts of dq and after them those of dk and dv
size_t gradient_words(const tessel_packing *p, const tessel_attention *a) { return ((size_t)p->tokens * a->heads + 3) / 4 * 4; }
size_t backward_workspace(const tessel_packing *p, const tessel_attention *a)
{
    const size_t q = query_splits(p, a), k = key_splits(p, a), row = (size_t)p->tokens * a->dim;
    const size_t parts = std::max(q > 1 ? q * row * a->heads : 0, k > 1 ? k * 2 * row * a->kv_heads : 0);
    return (gradient_words(p, a) + parts) * sizeof(float);
}

bool workspace_ok(const void *p, size_t have, size_t need) { return need == 0 || (p && aligned(p, 16) && have >= need); }

// ---- rows
bool rows_ok(const tessel_rows &r, int type, int64_t tokens, int channels, bool written)
{
    if (tokens == 0) return true;
    if (!r.data || !aligned(r.data, size_of(type)) || r.stride < 0 || r.stride > kMostStride) return false;
    return !written || r.stride >= channels;
}

int checkpoint_ok(const tessel_checkpoint *c)
{
    if (!c || c->tokens < 0 || c->channels < 1) return TESSEL_E_INVALID_ARG;
    if (!is_type(c->type)) return TESSEL_E_UNSUPPORTED;
    const int64_t groups = ((int64_t)c->channels + TESSEL_CHECKPOINT_GROUP - 1) / TESSEL_CHECKPOINT_GROUP;
    if (c->tokens > INT32_MAX || (double)c->tokens * groups * 8 > 4e9) return TESSEL_E_TOOBIG;
    if (c->tokens == 0) return TESSEL_OK;
    if (!c->values || !c->exponents || !aligned(c->values, 16) || c->value_stride % TESSEL_CHECKPOINT_GROUP || c->value_stride < c->channels ||
        c->value_stride > kMostStride || c->exponent_stride < groups || c->exponent_stride > kMostStride) return TESSEL_E_INVALID_ARG;
    return TESSEL_OK;
}

int norm_ok(const tessel_residual_norm *a)
{
    if (!a || a->tokens < 0 || a->channels < 1 || a->gate_kind < TESSEL_GATE_NONE || a->gate_kind > TESSEL_GATE_TOKEN) return TESSEL_E_INVALID_ARG;
    if (!(a->eps >= 0.0f) || !std::isfinite(a->eps) || !std::isfinite(a->scale)) return TESSEL_E_INVALID_ARG;
    if (!is_type(a->type)) return TESSEL_E_UNSUPPORTED;
    if (a->channels > 16384 || a->tokens > INT32_MAX) return TESSEL_E_TOOBIG;
    if (!a->pre || !aligned(a->pre, 4) || !aligned(a->post, 4)) return TESSEL_E_INVALID_ARG;
    if (a->gate_kind == TESSEL_GATE_CHANNEL && (!a->gate.data || !aligned(a->gate.data, 4))) return TESSEL_E_INVALID_ARG;
    if (a->gate_kind == TESSEL_GATE_TOKEN && !rows_ok(a->gate, a->type, a->tokens, a->channels, false)) return TESSEL_E_INVALID_ARG;
    if (!rows_ok(a->x, a->type, a->tokens, a->channels, false) || !rows_ok(a->y, a->type, a->tokens, a->channels, false)) return TESSEL_E_INVALID_ARG;
    if (a->tokens && (!a->stats || !aligned(a->stats, 4))) return TESSEL_E_INVALID_ARG;
    return TESSEL_OK;
}

size_t norm_workspace(const tessel_residual_norm *a) { return (size_t)norm_parts(*a) * 2 * a->channels * sizeof(float); }

int weight_ok(const tessel_weight_grad *a)
{
    if (!a || a->outputs < 1) return TESSEL_E_INVALID_ARG;
    const int e = checkpoint_ok(&a->x);
    if (e) return e;
    if (a->x.type == TESSEL_F32) return TESSEL_E_UNSUPPORTED;
    if (weight_tiles(*a) > kMostThreads / kWeightThreads / weight_parts(*a)) return TESSEL_E_TOOBIG;
    if (a->outputs > kMostNear || a->dy.stride > kMostNear || a->x.value_stride > kMostNear || a->x.exponent_stride > kMostNear) return TESSEL_E_TOOBIG;
    if (!a->dw || !aligned(a->dw, 4) || a->dw_stride < a->x.channels || a->dw_stride > kMostStride) return TESSEL_E_INVALID_ARG;
    return rows_ok(a->dy, a->x.type, a->x.tokens, a->outputs, false) ? TESSEL_OK : TESSEL_E_INVALID_ARG;
}

size_t weight_workspace(const tessel_weight_grad *a)
{
    const int parts = weight_parts(*a);
    return parts > 1 ? (size_t)parts * a->outputs * a->x.channels * sizeof(float) : 0;
}

// ---- between the tokens and the attention
// chunks of eight channels: of as many as a launch has threads, by workgroups of 256, the kernels take several a lane where rows leave lanes over
bool chunks_ok(int64_t tokens, int channels) { return tokens * (((int64_t)channels + 7) / 8) <= kMostThreads / 256 * 256; }

int drop_ok(const tessel_dropout &d, DropLaunch &l)
{
    if (!(d.rate >= 0.0f && d.rate < 1.0f) || !aligned(d.step, 8)) return TESSEL_E_INVALID_ARG;
    // (exact: the largest rate below 1 is 1 - 2^-24)
    l = {(uint32_t)((double)d.rate * 0x1p32), (float)(1.0 / (1.0 - (double)d.rate)), d.seed, d.number, d.step};
    return TESSEL_OK;
}

int dropout_ok(const tessel_dropout_rows *a, DropLaunch &l)
{
    if (!a || a->tokens < 0 || a->channels < 1) return TESSEL_E_INVALID_ARG;
    if (!is_type(a->type)) return TESSEL_E_UNSUPPORTED;
    const int e = drop_ok(a->drop, l);
    if (e) return e;
    if (a->tokens > INT32_MAX || a->channels > 1 << 30 || !chunks_ok(a->tokens, a->channels)) return TESSEL_E_TOOBIG;
    return rows_ok(a->x, a->type, a->tokens, a->channels, false) && rows_ok(a->y, a->type, a->tokens, a->channels, true) ? TESSEL_OK : TESSEL_E_INVALID_ARG;
}

bool index_ok(const void *p, int type, int64_t tokens) { return tokens == 0 || (p && aligned(p, type == TESSEL_I64 ? 8 : 4)); }

int embedding_sizes_ok(const tessel_embedding *a)
{
    if (!a || a->tokens < 0 || a->rows < 1 || a->channels < 1) return TESSEL_E_INVALID_ARG;
    if (a->tokens > INT32_MAX || a->rows > 1 << 24 || a->channels > 1 << 24 || !chunks_ok(a->tokens, a->channels)) return TESSEL_E_TOOBIG;
    return TESSEL_OK;
}

int embedding_ok(const tessel_embedding *a, DropLaunch &l)
{
    int e = embedding_sizes_ok(a);
    if (e) return e;
    if (!is_type(a->type) || (a->index_type != TESSEL_I32 && a->index_type != TESSEL_I64)) return TESSEL_E_UNSUPPORTED;
    if (a->first < 0 || a->first > (int64_t)1 << 62 || !std::isfinite(a->scale) || !index_ok(a->token, a->index_type, a->tokens)) return TESSEL_E_INVALID_ARG;
    return drop_ok(a->drop, l);
}

// strides of any multiple; what is written must not lie on itself
bool any_heads_ok(const tessel_heads &h, int type, bool written, int64_t tokens, int heads, int dim)
{
    if (!h.data || !aligned(h.data, size_of(type)) || h.token_stride < 0 || h.head_stride < 0) return false;
    if (h.token_stride > kMostStride || h.head_stride > kMostStride) return false;
    if (!written) return true;
    const bool by_token = heads == 1 || (tokens > 1 && h.token_stride >= h.head_stride);       // heads lie inside a token
    const int64_t near = by_token ? h.head_stride : h.token_stride, far = by_token ? h.token_stride : h.head_stride;
    const int64_t inner = by_token ? heads : tokens, outer = by_token ? tokens : heads;
    return (inner == 1 || near >= dim) && (outer == 1 || far >= (inner - 1) * near + dim);
}

int rotation_sizes_ok(const tessel_rotation *a)
{
    if (!a || a->tokens < 0 || a->heads < 1 || a->kv_heads < 1 || a->dim < 2 || a->dim % 2 || a->turning < 0 || a->turning > a->dim || a->turning % 2)
        return TESSEL_E_INVALID_ARG;
    if (a->dim > 256 || a->tokens > INT32_MAX || a->heads > 1 << 24 || a->kv_heads > 1 << 24) return TESSEL_E_TOOBIG;
    if (rotate_waves(*a) > kMostThreads / 256 * 4) return TESSEL_E_TOOBIG;       // (workgroups of four waves)
    return TESSEL_OK;
}

int rotation_ok(const tessel_rotation *a)
{
    const int e = rotation_sizes_ok(a);
    if (e) return e;
    if (!is_type(a->type) || (a->index_type != TESSEL_I32 && a->index_type != TESSEL_I64)) return TESSEL_E_UNSUPPORTED;
    if (!(a->eps >= 0.0f) || !std::isfinite(a->eps) || !a->wq != !a->wk || !aligned(a->wq, 4) || !aligned(a->wk, 4)) return TESSEL_E_INVALID_ARG;
    if (a->turning && (!a->frequency || !aligned(a->frequency, 8) || !index_ok(a->position, a->index_type, a->tokens))) return TESSEL_E_INVALID_ARG;
    if (a->tokens && (!any_heads_ok(a->q, a->type, false, a->tokens, a->heads, a->dim) || !any_heads_ok(a->k, a->type, false, a->tokens, a->kv_heads, a->dim)))
        return TESSEL_E_INVALID_ARG;
    return TESSEL_OK;
}

size_t rotation_workspace(const tessel_rotation *a) { return a->wq ? (size_t)rotate_parts(*a) * 2 * a->dim * sizeof(float) : 0; }

}  // namespace

extern "C" {

int tessel_block_last_hip_error(void) { return last_hip; }

int tessel_packing_create(const int32_t *lengths, int32_t num_sequences, int64_t total_tokens, tessel_packing **out)
{
    if (!out) return TESSEL_E_INVALID_ARG;
    *out = nullptr;
    if (num_sequences < 0 || total_tokens < 0 || (num_sequences > 0 && !lengths)) return TESSEL_E_INVALID_ARG;
    if (total_tokens > INT32_MAX) return TESSEL_E_TOOBIG;
    int64_t sum = 0;
    for (int32_t i = 0; i < num_sequences; i++) {
        if (lengths[i] < 0) return TESSEL_E_INVALID_ARG;
        sum += lengths[i];
    }
    if (sum > total_tokens) return TESSEL_E_INVALID_ARG;
    try {
        tessel_packing *p = new tessel_packing;
        try {
            p->tokens = total_tokens;
            int32_t begin = 0;
            for (int32_t i = 0; i < num_sequences; i++) {
                const int32_t tiles = (int32_t)(((int64_t)lengths[i] + kAttendRows - 1) / kAttendRows);
                for (int32_t t = 0; t < tiles; t++) {
                    const int64_t steps = (std::min<int64_t>((int64_t)(t + 1) * kAttendRows, lengths[i]) + 63) / 64;
                    p->tiles.push_back({begin, lengths[i], t, tiles});
                    p->steps += steps;
                    p->longest = std::max(p->longest, steps);
                }
                begin += lengths[i];
            }
            // a tile's work is the number of tiles up to it
            std::stable_sort(p->tiles.begin(), p->tiles.end(), [](const AttendTile &a, const AttendTile &b) { return a.tile > b.tile; });
            for (int64_t at = sum; at < total_tokens; at += kAttendRows)
                p->tiles.push_back({(int32_t)at, -(int32_t)std::min<int64_t>(kAttendRows, total_tokens - at), 0, 1});
        } catch (...) {
            delete p;
            throw;
        }
        *out = p;
    } catch (const std::bad_alloc &) {
        return TESSEL_E_TOOBIG;
    }
    return TESSEL_OK;
}

void tessel_packing_destroy(tessel_packing *p) { delete p; }

int tessel_packing_table_bytes(const tessel_packing *p, size_t *bytes)
{
    if (!p || !bytes) return TESSEL_E_INVALID_ARG;
    *bytes = std::max<size_t>(1, p->tiles.size()) * sizeof(AttendTile);
    return TESSEL_OK;
}

int tessel_packing_bind(tessel_packing *p, void *table_dev, size_t table_bytes, void *hip_stream)
{
    if (!p) return TESSEL_E_INVALID_ARG;
    const size_t need = p->tiles.size() * sizeof(AttendTile);
    if (!table_dev || !aligned(table_dev, 16) || table_bytes < need) return TESSEL_E_WORKSPACE;
    if (need) {
        hipError_t e = hipMemcpyAsync(table_dev, p->tiles.data(), need, hipMemcpyHostToDevice, (hipStream_t)hip_stream);
        if (e == hipSuccess) e = hipStreamSynchronize((hipStream_t)hip_stream);
        if (e != hipSuccess) {
            (void)hipGetLastError();
            return hip_result((int)e);
        }
    }
    p->table = (const AttendTile *)table_dev;
    return TESSEL_OK;
}

int tessel_attention_forward_workspace_bytes(const tessel_packing *p, const tessel_attention *a, size_t *bytes)
{
    if (!bytes) return TESSEL_E_INVALID_ARG;
    const int e = forward_ok(p, a);
    if (e) return e;
    *bytes = forward_workspace(p, a);
    return TESSEL_OK;
}

int tessel_attention_forward(const tessel_packing *p, const tessel_attention *a, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    int e = forward_ok(p, a);
    if (e) return e;
    if (p->tokens == 0) return TESSEL_OK;
    if (!heads_ok(a->q, false, a->heads, a->dim) || !heads_ok(a->k, false, a->kv_heads, a->dim) || !heads_ok(a->v, false, a->kv_heads, a->dim) ||
        !heads_ok(a->o, true, a->heads, a->dim) || !a->lse || !aligned(a->lse, 4)) return TESSEL_E_INVALID_ARG;
    if (!p->table || !workspace_ok(workspace_dev, workspace_bytes, forward_workspace(p, a))) return TESSEL_E_WORKSPACE;
    AttendLaunch l = attend_launch(p, a);
    l.splits = query_splits(p, a);
    l.parts = (float *)workspace_dev;
    if (l.splits > 1) l.tops = l.parts + (size_t)l.splits * p->tokens * a->heads * a->dim;
    return hip_result(launch_attend(l, hip_stream));
}

int tessel_attention_backward_workspace_bytes(const tessel_packing *p, const tessel_attention *a, size_t *bytes)
{
    if (!bytes) return TESSEL_E_INVALID_ARG;
    const int e = backward_ok(p, a);
    if (e) return e;
    *bytes = backward_workspace(p, a);
    return TESSEL_OK;
}

int tessel_attention_backward(const tessel_packing *p, const tessel_attention *a, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    int e = backward_ok(p, a);
    if (e) return e;
    if (p->tokens == 0) return TESSEL_OK;
    if (!heads_ok(a->q, false, a->heads, a->dim) || !heads_ok(a->k, false, a->kv_heads, a->dim) || !heads_ok(a->v, false, a->kv_heads, a->dim) ||
        !heads_ok(a->o, false, a->heads, a->dim) || !heads_ok(a->d_o, false, a->heads, a->dim) || !heads_ok(a->dq, true, a->heads, a->dim) ||
        !heads_ok(a->dk, true, a->kv_heads, a->dim) || !heads_ok(a->dv, true, a->kv_heads, a->dim) || !a->lse || !aligned(a->lse, 4))
        return TESSEL_E_INVALID_ARG;
    if (!p->table || !workspace_ok(workspace_dev, workspace_bytes, backward_workspace(p, a))) return TESSEL_E_WORKSPACE;
    AttendLaunch l = attend_launch(p, a);
    l.delta = (float *)workspace_dev;
    l.parts = l.delta + gradient_words(p, a);
    l.splits = query_splits(p, a);
    e = launch_attend_dq(l, hip_stream);
    l.splits = key_splits(p, a);
    if (e == 0) e = launch_attend_dkv(l, hip_stream);
    return hip_result(e);
}

int tessel_residual_norm_forward(const tessel_residual_norm *a, void *hip_stream)
{
    const int e = norm_ok(a);
    if (e) return e;
    if (!rows_ok(a->r, a->type, a->tokens, a->channels, true) || !rows_ok(a->h, a->type, a->tokens, a->channels, true)) return TESSEL_E_INVALID_ARG;
    return hip_result(launch_norm(*a, hip_stream));
}

int tessel_residual_norm_backward_workspace_bytes(const tessel_residual_norm *a, size_t *bytes)
{
    if (!bytes || !a || a->tokens < 0 || a->channels < 1) return TESSEL_E_INVALID_ARG;
    if (a->channels > 16384 || a->tokens > INT32_MAX) return TESSEL_E_TOOBIG;
    *bytes = norm_workspace(a);
    return TESSEL_OK;
}

int tessel_residual_norm_backward(const tessel_residual_norm *a, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    const int e = norm_ok(a);
    if (e) return e;
    if (!rows_ok(a->dr, a->type, a->tokens, a->channels, false) || !rows_ok(a->dh, a->type, a->tokens, a->channels, false) ||
        !rows_ok(a->dx, a->type, a->tokens, a->channels, true) || !rows_ok(a->dy, a->type, a->tokens, a->channels, true)) return TESSEL_E_INVALID_ARG;
    if (!a->dpre || !aligned(a->dpre, 4) || (a->post && (!a->dpost || !aligned(a->dpost, 4)))) return TESSEL_E_INVALID_ARG;
    if (a->gate_kind == TESSEL_GATE_CHANNEL && (!a->dgate_channel || !aligned(a->dgate_channel, 4))) return TESSEL_E_INVALID_ARG;
    if (a->gate_kind == TESSEL_GATE_TOKEN && !rows_ok(a->dgate, a->type, a->tokens, a->channels, true)) return TESSEL_E_INVALID_ARG;
    if (!workspace_ok(workspace_dev, workspace_bytes, norm_workspace(a))) return TESSEL_E_WORKSPACE;
    return hip_result(launch_norm_backward(*a, (float *)workspace_dev, hip_stream));
}

int tessel_checkpoint_store(const tessel_checkpoint *c, const tessel_rows *x, void *hip_stream)
{
    const int e = checkpoint_ok(c);
    if (e) return e;
    if (!x || !rows_ok(*x, c->type, c->tokens, c->channels, false)) return TESSEL_E_INVALID_ARG;
    return c->tokens == 0 ? TESSEL_OK : hip_result(launch_store(*c, *x, hip_stream));
}

int tessel_checkpoint_restore(const tessel_checkpoint *c, const tessel_rows *x, void *hip_stream)
{
    const int e = checkpoint_ok(c);
    if (e) return e;
    if (!x || !rows_ok(*x, c->type, c->tokens, c->channels, true)) return TESSEL_E_INVALID_ARG;
    return c->tokens == 0 ? TESSEL_OK : hip_result(launch_restore(*c, *x, hip_stream));
}

static int gated_ok(int act, const tessel_checkpoint *g, const tessel_checkpoint *u)
{
    if (act != TESSEL_SILU && act != TESSEL_GELU) return TESSEL_E_INVALID_ARG;
    int e = checkpoint_ok(g);
    if (e == 0) e = checkpoint_ok(u);
    if (e) return e;
    return g->tokens == u->tokens && g->channels == u->channels && g->type == u->type ? TESSEL_OK : TESSEL_E_INVALID_ARG;
}

int tessel_gated_forward(int act, const tessel_rows *g, const tessel_rows *u, const tessel_rows *a, const tessel_checkpoint *kept_g,
                         const tessel_checkpoint *kept_u, void *hip_stream)
{
    const int e = gated_ok(act, kept_g, kept_u);
    if (e) return e;
    const int64_t n = kept_g->tokens;
    const int c = kept_g->channels, t = kept_g->type;
    if (!g || !u || !a || !rows_ok(*g, t, n, c, false) || !rows_ok(*u, t, n, c, false) || !rows_ok(*a, t, n, c, true)) return TESSEL_E_INVALID_ARG;
    return n == 0 ? TESSEL_OK : hip_result(launch_gated(act, *g, *u, *a, *kept_g, *kept_u, hip_stream));
}

int tessel_gated_backward(int act, const tessel_rows *da, const tessel_checkpoint *kept_g, const tessel_checkpoint *kept_u, const tessel_rows *dg,
                          const tessel_rows *du, const tessel_rows *a, void *hip_stream)
{
    const int e = gated_ok(act, kept_g, kept_u);
    if (e) return e;
    const int64_t n = kept_g->tokens;
    const int c = kept_g->channels, t = kept_g->type;
    if (!da || !dg || !du || !rows_ok(*da, t, n, c, false) || !rows_ok(*dg, t, n, c, true) || !rows_ok(*du, t, n, c, true)) return TESSEL_E_INVALID_ARG;
    const tessel_rows none = {nullptr, 0};
    if (a && a->data && !rows_ok(*a, t, n, c, true)) return TESSEL_E_INVALID_ARG;
    return n == 0 ? TESSEL_OK : hip_result(launch_gated_backward(act, *da, *kept_g, *kept_u, *dg, *du, a ? *a : none, hip_stream));
}

int tessel_weight_gradient_workspace_bytes(const tessel_weight_grad *a, size_t *bytes)
{
    if (!bytes || !a || a->outputs < 1 || a->x.channels < 1 || a->x.tokens < 0) return TESSEL_E_INVALID_ARG;
    if (a->x.tokens > INT32_MAX) return TESSEL_E_TOOBIG;
    *bytes = weight_workspace(a);
    return TESSEL_OK;
}

int tessel_weight_gradient(const tessel_weight_grad *a, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    const int e = weight_ok(a);
    if (e) return e;
    if (!workspace_ok(workspace_dev, workspace_bytes, weight_workspace(a))) return TESSEL_E_WORKSPACE;
    return hip_result(launch_weight_gradient(*a, (float *)workspace_dev, hip_stream));
}

int tessel_dropout_apply(const tessel_dropout_rows *a, void *hip_stream)
{
    DropLaunch l;
    const int e = dropout_ok(a, l);
    if (e) return e;
    return a->tokens == 0 ? TESSEL_OK : hip_result(launch_dropout(*a, l, hip_stream));
}

int tessel_embedding_forward(const tessel_embedding *a, void *hip_stream)
{
    DropLaunch l;
    const int e = embedding_ok(a, l);
    if (e) return e;
    if (!rows_ok(a->table, a->type, a->rows, a->channels, false) || !rows_ok(a->out, a->type, a->tokens, a->channels, true)) return TESSEL_E_INVALID_ARG;
    return a->tokens == 0 ? TESSEL_OK : hip_result(launch_embed(*a, l, hip_stream));
}

int tessel_embedding_backward_workspace_bytes(const tessel_embedding *a, size_t *bytes)
{
    if (!bytes) return TESSEL_E_INVALID_ARG;
    const int e = embedding_sizes_ok(a);
    if (e) return e;
    *bytes = embed_workspace(*a);
    return TESSEL_OK;
}

int tessel_embedding_backward(const tessel_embedding *a, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    DropLaunch l;
    const int e = embedding_ok(a, l);
    if (e) return e;
    if (!rows_ok(a->d_out, a->type, a->tokens, a->channels, false) || !a->dtable || !aligned(a->dtable, 4) || a->dtable_stride < a->channels ||
        a->dtable_stride > kMostStride) return TESSEL_E_INVALID_ARG;
    if (!workspace_ok(workspace_dev, workspace_bytes, embed_workspace(*a))) return TESSEL_E_WORKSPACE;
    return hip_result(launch_embed_backward(*a, l, workspace_dev, hip_stream));
}

int tessel_rotation_forward(const tessel_rotation *a, void *hip_stream)
{
    const int e = rotation_ok(a);
    if (e || a->tokens == 0) return e;
    if (!any_heads_ok(a->q_out, a->type, true, a->tokens, a->heads, a->dim) || !any_heads_ok(a->k_out, a->type, true, a->tokens, a->kv_heads, a->dim))
        return TESSEL_E_INVALID_ARG;
    return hip_result(launch_rotate(*a, hip_stream));
}

int tessel_rotation_backward_workspace_bytes(const tessel_rotation *a, size_t *bytes)
{
    if (!bytes) return TESSEL_E_INVALID_ARG;
    const int e = rotation_sizes_ok(a);
    if (e) return e;
    *bytes = rotation_workspace(a);
    return TESSEL_OK;
}

int tessel_rotation_backward(const tessel_rotation *a, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    const int e = rotation_ok(a);
    if (e) return e;
    if (a->wq && (!a->dwq || !a->dwk || !aligned(a->dwq, 4) || !aligned(a->dwk, 4))) return TESSEL_E_INVALID_ARG;
    if (a->tokens && (!any_heads_ok(a->dq_out, a->type, false, a->tokens, a->heads, a->dim) || !any_heads_ok(a->dk_out, a->type, false, a->tokens, a->kv_heads, a->dim) ||
                      !any_heads_ok(a->dq, a->type, true, a->tokens, a->heads, a->dim) || !any_heads_ok(a->dk, a->type, true, a->tokens, a->kv_heads, a->dim)))
        return TESSEL_E_INVALID_ARG;
    if (!workspace_ok(workspace_dev, workspace_bytes, rotation_workspace(a))) return TESSEL_E_WORKSPACE;
    return hip_result(launch_rotate_backward(*a, (float *)workspace_dev, hip_stream));
}

}  // extern "C"

// kv_attend: attention of the new tokens over a paged cache (host side).
//
// For a row (a new token and a query head) with scores s_t over the tokens it sees, out = sum exp(s_t - m) v_t / sum
// exp(s_t - m) in one pass over the tokens: m is the largest score so far (up to a factor of 2^8), and what was
// summed under a smaller one is scaled down when it grows.  Sequences of few rows per KV head go to the step kernel,
// others to the tail kernel; both split a long sequence over workgroups where the batch alone does not fill the chip.
#include <algorithm>
#include <cmath>

#include "kvx_attend_kernels.h"

namespace kvx {

namespace {

constexpr int64_t kMaxWorkgroups = int64_t{1} << 22;  // of the tail kernel: 2^31 lanes
constexpr int64_t kMaxScoreBytes = int64_t{1} << 30;

// The factor of q . k.
float scale_of(const kv_cache *cache, const kv_attend_options *o) {
    return (o->scale == 0.f ? 1.f / std::sqrt(static_cast<float>(cache->layout.head_dim)) : o->scale) *
           (o->k_scale == 0.f ? 1.f : o->k_scale);
}

// The checks of kv_attend that need no stream.
kv_status check_attend(const kv_cache *cache, const kv_batch *batch, const kv_attend_options *o, const kv_rows *q) {
    if (!cache)
        return fail(KV_EINVAL, "cache must not be NULL");
    kv_status st = check_layer(cache, 0);
    if (st != KV_OK)
        return st;
    if (!o)
        return fail(KV_EINVAL, "options must not be NULL");
    st = check_dtype(cache, o->cache_dtype);
    if (st == KV_OK)
        st = check_batch(cache, batch);
    if (st == KV_OK)
        st = check_rows(cache, batch, q, "q");
    if (st != KV_OK)
        return st;
    const int H = cache->layout.num_kv_heads;
    if (q->heads % H != 0)
        return fail(KV_EINVAL, "%d query heads for %d KV heads", q->heads, H);
    if (q->heads > 16383)
        return fail(KV_EUNSUPPORTED, "%d query heads (at most 16,383)", q->heads);
    const bool quantised = o->cache_dtype == KV_DTYPE_E4M3;
    if (!quantised && q->dtype != o->cache_dtype)
        return fail(KV_EINVAL, "rows of type %d for a cache of type %d", q->dtype, o->cache_dtype);
    if (!(o->scale >= 0.f && std::isfinite(o->scale)) || !(o->softcap >= 0.f && std::isfinite(o->softcap)) ||
        o->window < 0)
        return fail(KV_EINVAL, "scale, softcap and window must not be negative (got %g, %g, %d)", o->scale, o->softcap,
                    o->window);
    const float ks = o->k_scale == 0.f ? 1.f : o->k_scale, vs = o->v_scale == 0.f ? 1.f : o->v_scale;
    if (!(ks > 0.f && std::isfinite(ks)) || !(vs > 0.f && std::isfinite(vs)) ||
        (!quantised && (ks != 1.f || vs != 1.f)))
        return fail(KV_EINVAL, "scales must be positive, and 1 for a cache of 2-byte elements (got %g and %g)", ks, vs);
    // What the kernels multiply scores by has to be a normal number.
    const float product = scale_of(cache, o), inv = o->softcap > 0.f ? product / o->softcap : 1.f;
    if (!(product >= 1e-36f && product <= 1e36f) || !(inv >= 1e-36f && inv <= 1e36f))
        return fail(KV_EUNSUPPORTED, "scale %g with k_scale %g and softcap %g is beyond 32-bit scores", o->scale,
                    o->k_scale, o->softcap);
    if ((o->full_weights != 0 && o->full_weights != 1) || o->reserved != 0)
        return fail(KV_EINVAL, "full_weights must be 0 or 1 and reserved 0 (got %d and %d)", o->full_weights,
                    o->reserved);
    if (o->weights_in && !o->weights_out)
        return fail(KV_EINVAL, "weights_in without weights_out");
    // Rows are counted in 32 bits, and the tail kernel's workgroups by what one launch takes.
    const int64_t queries = std::min(batch->max_queries, batch->num_queries), group = q->heads / H;
    if (queries * group > INT32_MAX / 2 || (queries * group > kStepRows &&
                                            tail_tiles(queries, group) * H * batch->num_seqs > kMaxWorkgroups))
        return fail(KV_EUNSUPPORTED, "up to %lld new tokens in each of %d sequences of %d query heads are too many for "
                    "one call", static_cast<long long>(queries), batch->num_seqs, q->heads);
    if (o->weights_out && (o->weights_seq_stride < 0 || o->weights_head_stride < 0 ||
                           (batch->num_seqs > 0 && H > 1 && o->weights_head_stride < batch->max_len) ||
                           (batch->num_seqs > 1 && o->weights_seq_stride < batch->max_len)))
        return fail(KV_EINVAL, "rows of weights (strides %lld and %lld) are shorter than max_len %d",
                    static_cast<long long>(o->weights_seq_stride), static_cast<long long>(o->weights_head_stride),
                    batch->max_len);
    return KV_OK;
}

// How a call is cut, and what its workspace holds.  Only the host's numbers count.
struct Plan {
    int32_t max_queries, max_rows;  // of a sequence; rows per KV head in the step kernel
    bool tail;                      // some sequence may have more than kStepRows rows
    bool scores;                    // weights_out from the step kernel's scores
    bool listed;                    // the step kernel's parts are listed by a kernel
    int64_t score_len, lists, step_stats, step_sums, tail_stats, tail_sums, scores_at, bytes;
    Shares shares;
    Parts tail_parts;
};

int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// The tail kernel's parts, for `have` tiles of rows (of the `launched`, others are empty).  512 of its workgroups run
// at once (2 per CU; 256 where D > 128), so they may leave the last round nearly empty, and tiles that see less than
// others end it early: the number of parts is the one whose rounds (between those of equal parts, and those without
// an edge and half a part idle at the end) and joining take least, at the 0.2 ns per token and column that such a
// round takes and the 5 TB/s at which parts are written and read again (a session turn of 656 tiles: 1.99 ms whole,
// 1.54 in 3 parts, joining included).  Parts have no fewer than 256 tokens and no more than 256 MB between them.
Parts tail_parts_for(int64_t longest, int64_t have, int64_t launched, int64_t head_dim) {
    const int64_t at_once = head_dim > 128 ? 256 : 512;
    const double tokens_us = 0.2e-3 * static_cast<double>(head_dim) * static_cast<double>(longest);
    const double parts_bytes = static_cast<double>(have) * kTailRows * static_cast<double>(head_dim) * 4;
    int64_t best = 1;
    double best_us = 0.;
    for (int64_t splits = 1; splits <= 64; ++splits) {
        const double n = static_cast<double>(splits);
        if (splits > 1 && (longest < 256 * splits || parts_bytes * n > 256e6 || launched * splits > kMaxWorkgroups))
            break;
        const double rounds = 0.5 * (static_cast<double>((have * splits + at_once - 1) / at_once) +
                                     static_cast<double>(have * splits) / static_cast<double>(at_once) + 0.5);
        const double us = rounds / n * tokens_us + (splits > 1 ? 5. + n * parts_bytes * 2 / 5e6 : 0.);
        if (splits == 1 || us < 0.97 * best_us) {
            best = splits;
            best_us = us;
        }
    }
    Parts p{};
    p.len = static_cast<int32_t>(round_up((longest + best - 1) / best, 64));
    p.splits = static_cast<int32_t>((longest + p.len - 1) / p.len);
    return p;
}

Plan plan_of(const kv_cache *cache, const kv_batch *batch, const kv_attend_options *o, const kv_rows *q) {
    const int64_t H = cache->layout.num_kv_heads, D = cache->layout.head_dim, group = q->heads / H;
    const int64_t heads = batch->num_seqs * H;
    Plan p{};
    p.max_queries = std::min(batch->max_queries, batch->num_queries);
    if (heads == 0 || p.max_queries == 0)
        return p;
    const int64_t all_rows = p.max_queries * group;
    p.max_rows = static_cast<int32_t>(std::min<int64_t>(all_rows, kStepRows));
    p.tail = all_rows > kStepRows;
    // With more rows than a tile has the scores would outgrow K itself: they are taken again instead.  So they are
    // where the host's bounds, which may be far above what the sequences hold, would ask for more than 1 GiB of them.
    p.score_len = round_up(batch->max_len, 32);
    p.scores = o->weights_out && all_rows <= 16 && p.score_len <= kMaxScoreBytes / (4 * heads * all_rows);
    // The step kernel: as many workgroups as run at once (by its registers 2 per CU, 3 up to 64 columns, 1 with wide
    // 2-byte rows), or one for each sequence where that is more.
    const int64_t tile = step_tile_rows(p.max_rows, static_cast<int>(D)), tiles = (p.max_rows + tile - 1) / tile;
    const int64_t at_once = D <= 64 ? 768 : D > 128 && cache->layout.elem_bytes == 2 ? 256 : 512;
    const int64_t window = o->window > 0 ? o->window + int64_t{kStepRows} + 31 : batch->max_len;
    const int64_t longest = std::max<int64_t>(std::min<int64_t>(window, batch->max_len), 1);
    // A part has 32 tokens a wave at least; where the sequences alone fill the chip, enough that splitting and joining
    // take less than the wait for a long one does (2,000 sequences of up to 300 tokens: 82 us whole, 129 in parts).
    Shares &s = p.shares;
    s.shortest = heads * tiles >= at_once ? 512 : 128;
    const int64_t most = (longest + s.shortest - 1) / s.shortest * batch->num_seqs;  // parts that can be
    s.num_seqs = batch->num_seqs;
    // (Many sequences are cut for three rounds of workgroups, of which the last may be nearly empty: 64 of up to 4,096
    // tokens on 8 heads take 143 us in one to one and a half rounds, 136 in three.)
    const int64_t rounds = 2 * heads * tiles >= at_once ? 3 : 1;
    s.target = static_cast<int32_t>(
        std::min(std::max<int64_t>(rounds * at_once / (H * tiles), s.num_seqs), most));
    s.alone = longest <= s.shortest || s.target == 1;
    s.items = s.alone || s.num_seqs == 1 ? std::max(s.num_seqs, s.alone ? 1 : s.target) : s.target + s.num_seqs;
    s.row_cap = p.max_rows;
    if (p.tail) {
        const int64_t seen = o->window > 0 ? o->window + int64_t{kTailRows} + 31 : batch->max_len;
        const int64_t tiles_each = tail_tiles(p.max_queries, group);
        const int64_t tiles_all = (batch->num_queries * group + kTailRows - 1) / kTailRows + batch->num_seqs;
        p.tail_parts = tail_parts_for(std::max<int64_t>(std::min<int64_t>(seen, batch->max_len), 1),
                                      H * std::min(batch->num_seqs * tiles_each, tiles_all), heads * tiles_each, D);
    }
    int64_t at = round_up(static_cast<int64_t>(batch->num_queries) * q->heads * 4, 16);
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += round_up(bytes, 16);
        return here;
    };
    const int64_t shared = s.alone ? 0 : H * s.items * s.row_cap;
    p.listed = !s.alone && s.num_seqs > kShareSeqs;
    p.lists = take(p.listed ? (2 + 2 * (int64_t{s.num_seqs} + s.items)) * 4 : 0);
    p.step_stats = take(shared * 8);
    p.step_sums = take(shared * D * 4);
    const int64_t split =
        p.tail_parts.splits > 1 ? static_cast<int64_t>(batch->num_queries) * q->heads * p.tail_parts.splits : 0;
    p.tail_stats = take(split * 8);
    p.tail_sums = take(split * D * 4);
    p.scores_at = take(p.scores ? heads * all_rows * p.score_len * 4 : 0);
    p.bytes = at;
    return p;
}

kv_status attend(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_attend_options *o,
                 const kv_rows *q, const kv_rows *out, float *lse, void *workspace, int64_t workspace_bytes,
                 hipStream_t stream) {
    kv_status st = check_layer(cache, layer);
    if (st == KV_OK)
        st = check_attend(cache, batch, o, q);
    if (st == KV_OK)
        st = check_rows(cache, batch, out, "out");
    if (st != KV_OK)
        return st;
    if (out->heads != q->heads || out->dtype != q->dtype)
        return fail(KV_EINVAL, "out has %d heads of type %d, q %d of type %d", out->heads, out->dtype, q->heads,
                    q->dtype);
    const int D = cache->layout.head_dim;
    if (batch->num_seqs > 0 && ((batch->num_queries > 1 && out->token_stride < D) ||
                                (batch->num_queries > 0 && out->heads > 1 && out->head_stride < D)))
        return fail(KV_EINVAL, "rows of out (strides %lld and %lld) are shorter than %d elements",
                    static_cast<long long>(out->token_stride), static_cast<long long>(out->head_stride), D);
    const Plan plan = plan_of(cache, batch, o, q);
    const int64_t need = plan.bytes;
    if (workspace_bytes < need || (need > 0 && !workspace))
        return fail(KV_EINVAL, "workspace of %lld bytes; %lld are needed", static_cast<long long>(workspace_bytes),
                    static_cast<long long>(need));
    if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
        return fail(KV_EUNSUPPORTED, "workspace is not 16-byte aligned");
    if (batch->num_seqs == 0)
        return KV_OK;
    int32_t *err = nullptr;
    st = check_on_current_device(cache);
    if (st == KV_OK)
        st = error_word(&err);
    if (st != KV_OK)
        return st;
    AttendArgs a{};
    a.pages = pages_of(cache, layer, err);
    a.batch = batch_of(batch);
    a.q = Rows{static_cast<uint8_t *>(q->data), q->token_stride * 2, q->head_stride * 2};
    a.out = Rows{static_cast<uint8_t *>(out->data), out->token_stride * 2, out->head_stride * 2};
    uint8_t *space = static_cast<uint8_t *>(workspace);
    a.lse = lse ? lse : reinterpret_cast<float *>(space);
    const auto at = [&](int64_t offset) { return reinterpret_cast<float *>(space + offset); };
    Shares step = plan.shares;
    Parts tail = plan.tail_parts;
    step.stats = at(plan.step_stats);
    step.sums = at(plan.step_sums);
    step.items_of = plan.listed ? reinterpret_cast<int32_t *>(space + plan.lists) : nullptr;
    tail.stats = at(plan.tail_stats);
    tail.sums = at(plan.tail_sums);
    a.scores = plan.scores ? at(plan.scores_at) : nullptr;
    a.score_len = plan.score_len;
    a.score_cap = plan.max_rows;
    a.slopes = o->slopes;
    a.weights_in = o->weights_in;
    a.weights_out = o->weights_out;
    a.weights_seq_stride = o->weights_seq_stride;
    a.weights_head_stride = o->weights_head_stride;
    a.scale = scale_of(cache, o);
    a.softcap = o->softcap;
    a.v_scale = o->v_scale == 0.f ? 1.f : o->v_scale;
    a.window = o->window < batch->max_len ? o->window : 0;  // a window of every token hides none
    a.heads = q->heads;
    a.group = q->heads / cache->layout.num_kv_heads;
    a.num_seqs = batch->num_seqs;
    a.q_type = q->dtype;
    a.cache_type = o->cache_dtype;
    a.full_weights = o->full_weights;
    a.by_group = divisor(a.group);
    if (plan.max_queries > 0) {
        if (plan.listed)
            KVX_HIP(launch_share(a, step, stream));
        KVX_HIP(launch_step(a, step, plan.max_queries, stream));
        if (!step.alone)
            KVX_HIP(launch_join_step(a, step, plan.max_queries, stream));
        if (plan.tail) {
            KVX_HIP(launch_tail(a, tail, plan.max_queries, stream));
            if (tail.splits > 1)
                KVX_HIP(launch_join_tail(a, tail, plan.max_queries, stream));
        }
    }
    if (a.weights_out && batch->max_len > 0)
        KVX_HIP(a.scores ? launch_weigh_step(a, stream) : launch_weigh(a, stream));
    return KV_OK;
}

}  // namespace

}  // namespace kvx

extern "C" {

int64_t kv_attend_workspace(const kv_cache *cache, const kv_batch *batch, const kv_attend_options *options,
                            const kv_rows *q) {
    int64_t bytes = 0;
    const kv_status st = kvx::guarded([&]() -> kv_status {
        const kv_status checked = kvx::check_attend(cache, batch, options, q);
        if (checked == KV_OK)
            bytes = kvx::plan_of(cache, batch, options, q).bytes;
        return checked;
    });
    return st == KV_OK ? bytes : st;
}

kv_status kv_attend(const kv_cache *cache, int32_t layer, const kv_batch *batch, const kv_attend_options *options,
                    const kv_rows *q, const kv_rows *out, float *lse, void *workspace, int64_t workspace_bytes,
                    void *stream) {
    return kvx::guarded([&]() -> kv_status {
        return kvx::attend(cache, layer, batch, options, q, out, lse, workspace, workspace_bytes,
                           static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"

// Host side of the entry points over pages that a server calls around the attention: checks of arguments, division of the work,
// launches.
#include <algorithm>
#include <cmath>

#include "octopus_internal.h"

namespace octopus {
namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

// of the partial results' (reference, sum) pairs and rows
size_t prefix_bytes(int64_t partials, int32_t d) {
    return 256 + up256(partials * 2 * sizeof(float)) + up256(partials * static_cast<size_t>(d) * sizeof(float));
}

bool pages_ok(const void *table, int32_t pages) {
    return table != nullptr && aligned(table, 4) && pages >= 1 && pages <= INT32_MAX / OCTOPUS_TILE;
}

int prefix_args(const octopus_codebooks_t *cb, int32_t n_seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t n_q, int64_t max_prefix,
                int64_t max_len) {
    if (cb == nullptr) return OCTOPUS_EINVAL;
    if (n_seq < 1 || n_q_heads < 1 || n_kv_heads < 1 || n_q < 1 || n_q_heads % n_kv_heads != 0) return OCTOPUS_EINVAL;
    if (max_prefix < 0 || max_prefix > INT32_MAX - OCTOPUS_TILE || max_len < 0 || max_len > INT32_MAX - OCTOPUS_TILE) return OCTOPUS_EINVAL;
    // rows, segments and threads of a launch are counted in 32 bits
    if (static_cast<int64_t>(n_seq) * n_q > (1 << 24) || static_cast<int64_t>(n_seq) * n_q * n_q_heads > (1 << 26)) return OCTOPUS_EINVAL;
    if (!plan_well_formed(cb->plan)) return OCTOPUS_EINVAL;
    if (!plan_supported(cb->plan)) return OCTOPUS_EUNSUPPORTED;
    return OCTOPUS_OK;
}

// Partial results of the prefix, and of the own tokens, that ranges may make beyond one per row.  The workspace is sized by this limit
// and not by the division, which can make fewer of a larger call, so that a workspace serves every smaller call.  2^18 are
// 130 MB at d = 128; of 6000 random shapes 23 divide worse than without a limit, by 1.8 % of the cost below at most (2^17: 71 of them, 13 %).
constexpr int64_t kRangePartials = 1 << 18;
constexpr int64_t kMostRanges = 128;

int64_t prefix_round_keys(const octopus_plan_t &plan) { return 32 * prefix_waves(plan.head_dim); }
int64_t most_ranges(int64_t rows) { return std::min(std::max<int64_t>(kRangePartials / rows, 1), kMostRanges); }

// octopus_append_paged (axes NULL) and octopus_append_paged_axes (rope NULL).
int append(const octopus_codebooks_t *cb, const void *k, int64_t k_stride_seq, int64_t k_stride_tok, int64_t k_stride_head,
           const void *v, int64_t v_stride_seq, int64_t v_stride_tok, int64_t v_stride_head, int32_t kv_dtype, int32_t n_seq,
           int32_t n_kv_heads, int32_t n_new, const int32_t *new_lens, const octopus_rope_t *rope, const octopus_rope_axes_t *axes, const void *q,
           int32_t q_dtype, int64_t q_stride_seq, int64_t q_stride_tok, int64_t q_stride_head, int32_t n_q_heads, void *q_out,
           int32_t q_out_dtype, const uint8_t *signs, void *k_pool, void *v_pool, int32_t v_bits, int32_t v_group,
           int32_t n_pages, const int32_t *block_table, int32_t max_pages_per_seq, const int32_t *start_pos, void *stream) {
    if (cb == nullptr || signs == nullptr || k_pool == nullptr || v_pool == nullptr) return OCTOPUS_EINVAL;
    if (n_new != 0 && (k == nullptr || v == nullptr)) return OCTOPUS_EINVAL;   // (an empty tensor may have no address)
    if (n_seq < 1 || n_kv_heads < 1 || n_new < 0 || n_seq > 65535 || n_kv_heads > 65535 || n_pages < 1) return OCTOPUS_EINVAL;
    if (!pages_ok(block_table, max_pages_per_seq) || !plan_well_formed(cb->plan)) return OCTOPUS_EINVAL;
    const int32_t d = cb->plan.head_dim;
    auto type_ok = [](int32_t t) { return t == OCTOPUS_DTYPE_F32 || t == OCTOPUS_DTYPE_BF16; };
    if (!type_ok(kv_dtype) || !plan_supported(cb->plan) || !encoder_takes(*cb) || !corner_levels(*cb)) return OCTOPUS_EUNSUPPORTED;
    if (v_bits != 0 && (v_bits < 2 || v_bits > 4 || (v_group != 16 && v_group != 32))) return OCTOPUS_EUNSUPPORTED;
    auto strides_ok = [](int64_t a, int64_t b, int64_t c) { return a >= 0 && b >= 0 && c >= 0 && a % 8 == 0 && b % 8 == 0 && c % 8 == 0; };
    if (!strides_ok(k_stride_seq, k_stride_tok, k_stride_head) || !strides_ok(v_stride_seq, v_stride_tok, v_stride_head)) return OCTOPUS_EINVAL;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k_pool, 16) || !aligned(v_pool, 16) || !aligned(new_lens, 4) || !aligned(start_pos, 4))
        return OCTOPUS_EINVAL;
    AppendCall a{};
    if (q != nullptr) {
        if (q_out == nullptr || n_q_heads < 1 || n_q_heads % n_kv_heads != 0) return OCTOPUS_EINVAL;
        if (!type_ok(q_dtype) || !type_ok(q_out_dtype)) return OCTOPUS_EUNSUPPORTED;
        if (!strides_ok(q_stride_seq, q_stride_tok, q_stride_head) || !aligned(q, 16) || !aligned(q_out, 16)) return OCTOPUS_EINVAL;
        a.n_q_heads = n_q_heads;
    }
    if (rope != nullptr) {
        if (rope->table == nullptr || !aligned(rope->table, 16) || rope->n_pos < 1 || !aligned(rope->pos, 4)) return OCTOPUS_EINVAL;
        if (rope->dim < 16 || rope->dim > d || rope->dim % 16 != 0 || (rope->interleaved != 0 && rope->interleaved != 1)) return OCTOPUS_EINVAL;
        a.rope = RopeCall{rope->table, rope->n_pos, rope->pos, rope->dim, rope->interleaved};
    }
    AxesCall many{};
    if (axes != nullptr) {
        if (axes->table == nullptr || !aligned(axes->table, 16) || axes->n_pos < 1 || (n_new != 0 && axes->pos == nullptr) || !aligned(axes->pos, 4))
            return OCTOPUS_EINVAL;
        if (axes->dim < 16 || axes->dim > d || axes->dim % 16 != 0 || (axes->interleaved != 0 && axes->interleaved != 1)) return OCTOPUS_EINVAL;
        // (the table is addressed by 32 bits of bytes, rows by a product of 24 bits each, a token's positions by one of 32)
        if (axes->n_pos > (int64_t{1} << 32) / (4 * axes->dim) || axes->n_pos > (1 << 24)) return OCTOPUS_EINVAL;
        if (axes->stride_seq < 0 || axes->stride_tok < 0 || axes->stride_tok > INT32_MAX || axes->stride_axis < 0 || axes->stride_axis > INT64_MAX / (8 * kMaxAxes))
            return OCTOPUS_EINVAL;
        if (axes->n_axes < 1 || axes->n_axes > kMaxAxes || axes->axis == nullptr) return OCTOPUS_EINVAL;
        for (int i = 0; i < axes->dim / 2; ++i) {
            if (axes->axis[i] >= axes->n_axes) return OCTOPUS_EINVAL;
            many.axis_of[i / 16] |= static_cast<uint32_t>(axes->axis[i]) << (2 * (i % 16));
        }
        many.pos = axes->pos;
        many.stride_seq = axes->stride_seq;
        many.stride_tok = static_cast<int32_t>(axes->stride_tok);
        for (int k = 1; k < axes->n_axes; ++k) many.axis_at[k - 1] = k * axes->stride_axis;
        many.last_pos = static_cast<int32_t>(axes->n_pos - 1);
        a.rope = RopeCall{axes->table, axes->n_pos, nullptr, axes->dim, axes->interleaved};
        a.axes = &many;
    }
    if (start_pos == nullptr && n_new > static_cast<int64_t>(max_pages_per_seq) * OCTOPUS_TILE) return OCTOPUS_EINVAL;
    // the launch: 2^22 workgroups at most, of tiles and of runs of at least 16 tokens by eight rows
    const int64_t tiles = (static_cast<int64_t>(n_new) / 64 + 2) * n_kv_heads * n_seq;
    const int64_t rows = (static_cast<int64_t>(n_kv_heads) + a.n_q_heads) / 8 + 1, runs = (static_cast<int64_t>(n_new) / 16 + 1) * n_seq;
    if (tiles > (1 << 21) || rows > (1 << 21) || rows * runs > (1 << 21)) return OCTOPUS_EINVAL;
    if (v_bits != 0 && static_cast<int64_t>(n_kv_heads) * (d / v_group) > 4096) return OCTOPUS_EINVAL;
    if (n_new == 0) return OCTOPUS_OK;
    a.k = k;
    a.v = v;
    a.q = q;
    a.k_seq = k_stride_seq;
    a.k_tok = k_stride_tok;
    a.k_head = k_stride_head;
    a.v_seq = v_stride_seq;
    a.v_tok = v_stride_tok;
    a.v_head = v_stride_head;
    a.q_seq = q_stride_seq;
    a.q_tok = q_stride_tok;
    a.q_head = q_stride_head;
    a.k_pool = k_pool;
    a.v_pool = v_bits == 0 ? v_pool : nullptr;
    a.q_out = q_out;
    a.signs = signs;
    a.start_pos = start_pos;
    a.new_lens = new_lens;
    a.pt = PageTable{block_table, max_pages_per_seq, n_pages};
    a.n_seq = n_seq;
    a.n_kv_heads = n_kv_heads;
    a.n_new = n_new;
    a.kv_is_bf16 = kv_dtype == OCTOPUS_DTYPE_BF16;
    a.q_is_bf16 = q_dtype == OCTOPUS_DTYPE_BF16;
    a.q_out_is_bf16 = q_out_dtype == OCTOPUS_DTYPE_BF16;
    int err = launch_append(*cb, a, stream);
    if (err == 0 && v_bits != 0) err = launch_append_values(a, d, v_bits, v_group, v_pool, stream);
    return err == 0 ? OCTOPUS_OK : OCTOPUS_EHIP;
}

}  // namespace

int64_t prefix_room(const octopus_plan_t &plan, int64_t rows, int64_t max_prefix, int64_t max_len) {
    int64_t room = 0;
    for (const int64_t tokens : {max_prefix, max_len}) {
        const int64_t rounds = (tokens + prefix_round_keys(plan) - 1) / prefix_round_keys(plan);
        if (rounds > 0) room += std::max(rows, std::min(rows * std::min(rounds, kMostRanges), kRangePartials));
    }
    return room;
}

// Ranges of tokens: a workgroup's segment takes rounds of one step per wavefront and a start of its own (queries, results), the
// workgroups run in rounds of 256, and every range writes a partial result per query row that the merge reads again.  The number of
// rounds a segment has at most is, of those tried (each a sixteenth above the one before), the one that makes the least of all that.
// The two constants are flat: of 13 shapes (one to 200 sequences, 1 to 70 000 tokens, every head dimension) a start of 1.25 rounds instead
// of 2.5 made one slower, by 3 %, and 5 none; 5e-6 a partial result made none slower, 8e-5 one, by 3 %.  Without a start four took 1.1
// to 2 times as long.
PrefixShape make_prefix_shape(const octopus_plan_t &plan, int32_t n_seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t n_q,
                              int64_t max_prefix, int64_t max_len) {
    PrefixShape s{};
    s.n_seq = n_seq;
    s.n_q_heads = n_q_heads;
    s.n_kv_heads = n_kv_heads;
    s.n_q = n_q;
    s.max_prefix = static_cast<int32_t>(max_prefix);
    s.max_len = static_cast<int32_t>(max_len);
    const int64_t hpk = n_q_heads / n_kv_heads, own_rows = n_q * hpk, all_rows = own_rows * n_seq;
    const int64_t group = prefix_rows(plan.head_dim);
    s.prefix_groups = static_cast<int32_t>((all_rows + group - 1) / group);
    s.own_groups = static_cast<int32_t>((own_rows + group - 1) / group);
    const int64_t round_keys = prefix_round_keys(plan), ranges_cap = most_ranges(all_rows * n_kv_heads);
    const int64_t prefix_rounds = (max_prefix + round_keys - 1) / round_keys, own_rounds = (max_len + round_keys - 1) / round_keys;
    const int64_t prefix_units = static_cast<int64_t>(n_kv_heads) * s.prefix_groups, own_units = static_cast<int64_t>(n_seq) * n_kv_heads * s.own_groups;
    auto ranges = [&](int64_t rounds, int64_t most) { return rounds == 0 ? 0 : std::min((rounds + most - 1) / most, ranges_cap); };
    double best = INFINITY;
    for (int64_t most = 1; most <= std::max<int64_t>(1, std::max(prefix_rounds, own_rounds)); most += std::max<int64_t>(1, most / 16)) {
        const int64_t a = ranges(prefix_rounds, most), b = ranges(own_rounds, most);
        const int64_t segments = prefix_units * a + own_units * b;
        if (segments > INT32_MAX / 2) continue;
        // (a workgroup takes every 256th segment: the busiest has one of each kind too many, or none of the prefix's and one more own)
        const double start = 2.5, shared = a > 0 ? start + (prefix_rounds + a - 1) / a : 0.0, mine = b > 0 ? start + (own_rounds + b - 1) / b : 0.0;
        const int64_t n_shared = prefix_units * a, full = n_shared / 256, some = (n_shared + 255) / 256, all = (segments + 255) / 256;
        const double cost = std::max(some * shared + std::max<int64_t>(all - some, 0) * mine, full * shared + (all - full) * mine) +
                            static_cast<double>(all_rows) * n_kv_heads * (a + b) * 2e-5;
        if (cost < best) {
            best = cost;
            s.prefix_splits = static_cast<int32_t>(a);
            s.own_splits = static_cast<int32_t>(b);
            s.prefix_segments = static_cast<int32_t>(prefix_units * a);
            s.n_segments = static_cast<int32_t>(segments);
        }
    }
    s.own_partials = all_rows * n_kv_heads * s.prefix_splits;
    return s;
}

}  // namespace octopus

using namespace octopus;

extern "C" {

size_t octopus_attn_prefix_workspace(const octopus_codebooks_t *cb, int32_t n_seq, int32_t n_q_heads, int32_t n_kv_heads, int32_t n_q,
                                     int64_t max_prefix, int64_t max_len) {
    if (prefix_args(cb, n_seq, n_q_heads, n_kv_heads, n_q, max_prefix, max_len) != OCTOPUS_OK) return 0;
    return prefix_bytes(prefix_room(cb->plan, static_cast<int64_t>(n_seq) * n_q * n_q_heads, max_prefix, max_len), cb->plan.head_dim);
}

int octopus_attn_decode_paged_prefix(const octopus_codebooks_t *cb, const void *q, int32_t q_dtype, int32_t n_seq, int32_t n_q_heads,
                                     int32_t n_kv_heads, int32_t n_q, const int32_t *q_lens, int32_t causal, const uint8_t *signs,
                                     const void *k_pool, const void *v_pool, int32_t n_pages, const int32_t *prefix_table,
                                     int32_t prefix_pages, const int32_t *prefix_len, int64_t max_prefix, const int32_t *block_table,
                                     int32_t max_pages_per_seq, const int32_t *seq_lens, int64_t max_len, float scale, float *out,
                                     void *workspace, size_t workspace_bytes, void *stream) {
    void *before = nullptr, *after = nullptr;
    take_profile_events(&before, &after);
    const int ok = prefix_args(cb, n_seq, n_q_heads, n_kv_heads, n_q, max_prefix, max_len);
    if (ok != OCTOPUS_OK) return ok;
    if (q == nullptr || signs == nullptr || k_pool == nullptr || v_pool == nullptr || out == nullptr || n_pages < 1) return OCTOPUS_EINVAL;
    if (causal != 0 && causal != 1) return OCTOPUS_EINVAL;
    if (max_prefix > 0) {
        if (!pages_ok(prefix_table, prefix_pages) || prefix_len == nullptr || !aligned(prefix_len, 4)) return OCTOPUS_EINVAL;
        if (max_prefix > static_cast<int64_t>(prefix_pages) * OCTOPUS_TILE) return OCTOPUS_EINVAL;
    }
    if (max_len > 0) {
        if (!pages_ok(block_table, max_pages_per_seq) || seq_lens == nullptr || !aligned(seq_lens, 4)) return OCTOPUS_EINVAL;
        if (max_len > static_cast<int64_t>(max_pages_per_seq) * OCTOPUS_TILE) return OCTOPUS_EINVAL;
    }
    if (q_dtype != OCTOPUS_DTYPE_F32 && q_dtype != OCTOPUS_DTYPE_BF16) return OCTOPUS_EUNSUPPORTED;
    if (!aligned(q, 4) || !aligned(out, 4) || !aligned(k_pool, 16) || !aligned(v_pool, 16) ||
        !aligned(q_lens, 4) || !std::isfinite(scale))
        return OCTOPUS_EINVAL;
    const int64_t partials = prefix_room(cb->plan, static_cast<int64_t>(n_seq) * n_q * n_q_heads, max_prefix, max_len);
    PrefixShape s = make_prefix_shape(cb->plan, n_seq, n_q_heads, n_kv_heads, n_q, max_prefix, max_len);
    if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < prefix_bytes(partials, cb->plan.head_dim)) return OCTOPUS_EWORKSPACE;
    s.max_pages = max_pages_per_seq;
    s.n_pages = n_pages;
    s.causal = causal;
    s.q = q;
    s.q_is_bf16 = q_dtype == OCTOPUS_DTYPE_BF16 ? 1 : 0;
    s.signs = signs;
    // (the tables' entries are 256 rho n, scores are in units of log2)
    int exponent = 0;
    s.scale_part = static_cast<float>(std::frexp(scale * 1.4426950408889634 / (256.0 * std::sqrt(static_cast<double>(cb->plan.head_dim))), &exponent));
    s.scale_exp = exponent;
    float *part_ml = static_cast<float *>(workspace);
    float *part_acc = reinterpret_cast<float *>(static_cast<char *>(workspace) + up256(partials * 2 * sizeof(float)));
    int err = before != nullptr ? record_event(before, stream) : 0;
    if (err == 0 && s.n_segments > 0)
        err = launch_prefix(*cb, s, k_pool, v_pool, prefix_table, prefix_len, block_table, seq_lens, q_lens, part_ml, part_acc, stream);
    if (err == 0 && after != nullptr) err = record_event(after, stream);
    if (err == 0) err = launch_prefix_merge(cb->plan, s, prefix_len, seq_lens, q_lens, part_ml, part_acc, out, stream);
    return err == 0 ? OCTOPUS_OK : OCTOPUS_EHIP;
}

int octopus_append_paged(const octopus_codebooks_t *cb, const void *k, int64_t k_stride_seq, int64_t k_stride_tok, int64_t k_stride_head,
                         const void *v, int64_t v_stride_seq, int64_t v_stride_tok, int64_t v_stride_head, int32_t kv_dtype, int32_t n_seq,
                         int32_t n_kv_heads, int32_t n_new, const int32_t *new_lens, const octopus_rope_t *rope, const void *q,
                         int32_t q_dtype, int64_t q_stride_seq, int64_t q_stride_tok, int64_t q_stride_head, int32_t n_q_heads, void *q_out,
                         int32_t q_out_dtype, const uint8_t *signs, void *k_pool, void *v_pool, int32_t v_bits, int32_t v_group,
                         int32_t n_pages, const int32_t *block_table, int32_t max_pages_per_seq, const int32_t *start_pos, void *stream) {
    return append(cb, k, k_stride_seq, k_stride_tok, k_stride_head, v, v_stride_seq, v_stride_tok, v_stride_head, kv_dtype, n_seq,
                  n_kv_heads, n_new, new_lens, rope, nullptr, q, q_dtype, q_stride_seq, q_stride_tok, q_stride_head, n_q_heads, q_out,
                  q_out_dtype, signs, k_pool, v_pool, v_bits, v_group, n_pages, block_table, max_pages_per_seq, start_pos, stream);
}

int octopus_append_paged_axes(const octopus_codebooks_t *cb, const void *k, int64_t k_stride_seq, int64_t k_stride_tok, int64_t k_stride_head,
                              const void *v, int64_t v_stride_seq, int64_t v_stride_tok, int64_t v_stride_head, int32_t kv_dtype, int32_t n_seq,
                              int32_t n_kv_heads, int32_t n_new, const int32_t *new_lens, const octopus_rope_axes_t *rope, const void *q,
                              int32_t q_dtype, int64_t q_stride_seq, int64_t q_stride_tok, int64_t q_stride_head, int32_t n_q_heads, void *q_out,
                              int32_t q_out_dtype, const uint8_t *signs, void *k_pool, void *v_pool, int32_t v_bits, int32_t v_group,
                              int32_t n_pages, const int32_t *block_table, int32_t max_pages_per_seq, const int32_t *start_pos, void *stream) {
    if (rope == nullptr) return OCTOPUS_EINVAL;
    return append(cb, k, k_stride_seq, k_stride_tok, k_stride_head, v, v_stride_seq, v_stride_tok, v_stride_head, kv_dtype, n_seq,
                  n_kv_heads, n_new, new_lens, nullptr, rope, q, q_dtype, q_stride_seq, q_stride_tok, q_stride_head, n_q_heads, q_out,
                  q_out_dtype, signs, k_pool, v_pool, v_bits, v_group, n_pages, block_table, max_pages_per_seq, start_pos, stream);
}

int octopus_read_paged(const octopus_codebooks_t *cb, const uint8_t *signs, const void *k_pool, const void *v_pool, int32_t v_bits,
                       int32_t v_group, int32_t n_pages, const int32_t *block_table, int32_t max_pages_per_seq, int32_t n_seq,
                       int32_t n_kv_heads, const int32_t *start_pos, int32_t n_tok, const int32_t *lens, void *k_out, void *v_out,
                       int32_t out_dtype, void *stream) {
    if (cb == nullptr || (n_tok != 0 && k_out == nullptr && v_out == nullptr)) return OCTOPUS_EINVAL;
    if ((k_out != nullptr && (k_pool == nullptr || signs == nullptr)) || (v_out != nullptr && v_pool == nullptr)) return OCTOPUS_EINVAL;
    if (n_seq < 1 || n_kv_heads < 1 || n_tok < 0 || n_seq > 65535 || n_kv_heads > 65535 || n_pages < 1) return OCTOPUS_EINVAL;
    if (!pages_ok(block_table, max_pages_per_seq) || !plan_well_formed(cb->plan)) return OCTOPUS_EINVAL;
    if (!plan_supported(cb->plan) || (out_dtype != OCTOPUS_DTYPE_F32 && out_dtype != OCTOPUS_DTYPE_BF16)) return OCTOPUS_EUNSUPPORTED;
    if (v_bits != 0 && (v_bits < 2 || v_bits > 4 || (v_group != 16 && v_group != 32))) return OCTOPUS_EUNSUPPORTED;
    if (!aligned(k_pool, 16) || !aligned(v_pool, 16) || !aligned(k_out, 16) || !aligned(v_out, 16) || !aligned(start_pos, 4) || !aligned(lens, 4))
        return OCTOPUS_EINVAL;
    if (start_pos == nullptr && n_tok > static_cast<int64_t>(max_pages_per_seq) * OCTOPUS_TILE) return OCTOPUS_EINVAL;
    // (workgroups; and a launch counts the threads along its tiles, one more than the tokens fill, in 32 bits)
    if ((static_cast<int64_t>(n_tok) / 64 + 2) * n_kv_heads * n_seq > (1 << 23)) return OCTOPUS_EINVAL;
    if (((static_cast<int64_t>(n_tok) + 63) / 64 + 1) * 64 * read_waves(cb->plan.head_dim) > UINT32_MAX) return OCTOPUS_EINVAL;
    if (n_tok == 0) return OCTOPUS_OK;
    ReadCall a{};
    a.k_pool = k_pool;
    a.v_pool = v_pool;
    a.k_out = k_out;
    a.v_out = v_out;
    a.signs = signs;
    a.start_pos = start_pos;
    a.lens = lens;
    a.pt = PageTable{block_table, max_pages_per_seq, n_pages};
    a.n_seq = n_seq;
    a.n_kv_heads = n_kv_heads;
    a.n_tok = n_tok;
    a.v_bits = v_bits;
    a.v_group = v_group;
    a.out_is_bf16 = out_dtype == OCTOPUS_DTYPE_BF16;
    const int err = launch_read(*cb, a, stream);
    return err == 0 ? OCTOPUS_OK : OCTOPUS_EHIP;
}

}  // extern "C"

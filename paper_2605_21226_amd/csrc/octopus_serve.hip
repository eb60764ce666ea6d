// Dispatch of the kernels over pages that a server calls around the attention (shared prefixes, appending, reading back), and the
// merge of a shared-prefix call.
#include "octopus_decode.hpp"

namespace octopus {

#define OCTOPUS_DECL(D)                                                                                                   \
    int launch_prefix_d##D(const octopus_codebooks_t &, const PrefixShape &, const void *, const void *, const int32_t *, \
                           const int32_t *, const int32_t *, const int32_t *, const int32_t *, float *, float *, void *); \
    int launch_append_d##D(const octopus_codebooks_t &, const AppendCall &, void *);                                      \
    int launch_read_d##D(const octopus_codebooks_t &, const ReadCall &, void *);
OCTOPUS_DECL(64)
OCTOPUS_DECL(128)
OCTOPUS_DECL(256)
#undef OCTOPUS_DECL

#define OCTOPUS_BY_HEAD_DIM(plan, fn, ...)             \
    switch ((plan).head_dim) {                         \
        case 64: return fn##_d64(__VA_ARGS__);         \
        case 128: return fn##_d128(__VA_ARGS__);       \
        case 256: return fn##_d256(__VA_ARGS__);       \
        default: return static_cast<int>(hipErrorInvalidValue); \
    }

int launch_prefix(const octopus_codebooks_t &cb, const PrefixShape &s, const void *k_pool, const void *v_pool, const int32_t *prefix_table,
                  const int32_t *prefix_len, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens, float *part_ml,
                  float *part_acc, void *stream) {
    OCTOPUS_BY_HEAD_DIM(cb.plan, launch_prefix, cb, s, k_pool, v_pool, prefix_table, prefix_len, block_table, seq_lens, q_lens, part_ml,
                        part_acc, stream)
}

int launch_append(const octopus_codebooks_t &cb, const AppendCall &a, void *stream) {
    OCTOPUS_BY_HEAD_DIM(cb.plan, launch_append, cb, a, stream)
}

int launch_read(const octopus_codebooks_t &cb, const ReadCall &a, void *stream) {
    OCTOPUS_BY_HEAD_DIM(cb.plan, launch_read, cb, a, stream)
}

// One wavefront per output row: out = sum_i 2^(m_i - M) acc_i / sum_i 2^(m_i - M) l_i over the row's partial results, the prefix's and
// the own ones; zeros where no token was seen.  Rows past a sequence's q_lens are left as they were.
template <int D>
__global__ __launch_bounds__(256) void prefix_merge_kernel(PrefixShape s, const int32_t *__restrict__ prefix_len,
                                                           const int32_t *__restrict__ seq_lens, const int32_t *__restrict__ q_lens,
                                                           const float *__restrict__ part_ml, const float *__restrict__ part_acc,
                                                           float *__restrict__ out) {
    constexpr int EPL = D / 64;
    const int lane = threadIdx.x & 63;
    const int64_t orow = static_cast<int64_t>(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t rows = static_cast<int64_t>(s.n_seq) * s.n_q * s.n_q_heads;
    if (orow >= rows) return;
    const int head = static_cast<int>(orow % s.n_q_heads);
    const int sq = static_cast<int>(orow / s.n_q_heads), qi = sq % s.n_q, seq = sq / s.n_q;
    if (q_lens != nullptr && qi >= q_lens[seq]) return;
    const int hpk = s.n_q_heads / s.n_kv_heads, kvh = head / hpk;
    auto ranges = [](int len, int splits) {      // those that have tokens, as the attention kernel divides them
        const int steps = (len + 31) / 32, per = splits > 0 ? (steps + splits - 1) / splits : 0;
        return per > 0 ? (steps + per - 1) / per : 0;
    };
    const int n_shared = s.prefix_splits > 0 ? ranges(min(max(prefix_len[0], 0), s.max_prefix), s.prefix_splits) : 0;
    const int n_own = s.own_splits > 0 ? ranges(min(max(seq_lens[seq], 0), s.max_len), s.own_splits) : 0;
    const int64_t first = (static_cast<int64_t>(kvh) * s.n_seq * s.n_q * hpk + static_cast<int64_t>(sq) * hpk + head % hpk) * s.prefix_splits;
    const int64_t second = s.own_partials + ((static_cast<int64_t>(seq) * s.n_kv_heads + kvh) * s.n_q * hpk + qi * hpk + head % hpk) * s.own_splits - n_shared;
    const int total = n_shared + n_own;

    float m_run = -INFINITY, l_run = 0.0f, acc[EPL];
#pragma unroll
    for (int j = 0; j < EPL; ++j) acc[j] = 0.0f;
    for (int i0 = 0; i0 < total; i0 += 64) {
        const int mine = min(i0 + lane, total - 1), count = min(64, total - i0);
        const int64_t p = (mine < n_shared ? first : second) + mine;
        const float2 ml = *reinterpret_cast<const float2 *>(part_ml + 2 * p);
        float m_new = lane < count ? ml.x : -INFINITY;
        static_for<0, 6>([&](auto bb) { m_new = fmaxf(m_new, lane_xor<(1 << decltype(bb)::value)>(m_new, lane)); });
        m_new = fmaxf(m_new, m_run);
        const float keep = exp2_raw(m_run - m_new), weight = lane < count ? exp2_raw(ml.x - m_new) : 0.0f;
        l_run = l_run * keep + wave_sum(lane < count ? weight * ml.y : 0.0f);
        m_run = m_new;
#pragma unroll
        for (int j = 0; j < EPL; ++j) acc[j] *= keep;
        for (int i = 0; i < count; i += 8) {
            float x[8][EPL];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int at = min(i0 + i + u, total - 1);
                const float *row = part_acc + ((at < n_shared ? first : second) + at) * D;
#pragma unroll
                for (int j = 0; j < EPL; ++j) x[u][j] = row[lane + 64 * j];
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (i + u >= count) break;
                const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(weight), i + u));
#pragma unroll
                for (int j = 0; j < EPL; ++j) acc[j] = fmaf(w, x[u][j], acc[j]);
            }
        }
    }
    const float inv = l_run == 0.0f ? 0.0f : 1.0f / l_run;   // (a sum that is no number stays none)
#pragma unroll
    for (int j = 0; j < EPL; ++j) out[orow * D + lane + 64 * j] = acc[j] * inv;
}

int launch_prefix_merge(const octopus_plan_t &plan, const PrefixShape &s, const int32_t *prefix_len, const int32_t *seq_lens,
                        const int32_t *q_lens, const float *part_ml, const float *part_acc, float *out, void *stream) {
    const int64_t rows = static_cast<int64_t>(s.n_seq) * s.n_q * s.n_q_heads;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>((rows + 3) / 4)), dim3(256), 0, static_cast<hipStream_t>(stream), s, prefix_len,
                           seq_lens, q_lens, part_ml, part_acc, out);
        return static_cast<int>(hipGetLastError());
    };
    switch (plan.head_dim) {
        case 64: return go(prefix_merge_kernel<64>);
        case 128: return go(prefix_merge_kernel<128>);
        case 256: return go(prefix_merge_kernel<256>);
        default: return static_cast<int>(hipErrorInvalidValue);
    }
}

}  // namespace octopus

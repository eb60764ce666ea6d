// Dispatch of the kernels over pages that a server calls around the attention (shared prefixes, appending, reading back), and the
// merge of a shared-prefix call.
#include "octopus_decode.hpp"

namespace octopus {

#define OCTOPUS_DECL(D)                                                                                                   \
    int launch_prefix_d##D(const octopus_codebooks_t &, const PrefixShape &, const void *, const void *, const int32_t *, \
                           const int32_t *, const int32_t *, const int32_t *, const int32_t *, float *, float *, void *); \
    int launch_append_d##D(const octopus_codebooks_t &, const AppendCall &, void *);                                      \
    int launch_append_axes_d##D(const octopus_codebooks_t &, const AppendCall &, void *);                                 \
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
    if (a.axes != nullptr) {
        OCTOPUS_BY_HEAD_DIM(cb.plan, launch_append_axes, cb, a, stream)
    }
    OCTOPUS_BY_HEAD_DIM(cb.plan, launch_append, cb, a, stream)
}

int launch_read(const octopus_codebooks_t &cb, const ReadCall &a, void *stream) {
    OCTOPUS_BY_HEAD_DIM(cb.plan, launch_read, cb, a, stream)
}

// out = sum_i 2^(m_i - M) acc_i / sum_i 2^(m_i - M) l_i over an output row's partial results, the prefix's and the own ones; zeros where
// no token was seen.  Rows past a sequence's q_lens are left as they were.  A workgroup per row, whose time is the latency of three
// dependent reads: D / 4 threads read a partial result, 16 bytes each, and the 512 / D groups of them take every so manieth, 16 on their way at once; the groups'
// sums meet in LDS.  512 rows of 17 partial results at d = 128 (4.5 MB) take 5.3 us; a wavefront per row took 9.0.
constexpr int kMergeThreads = 128;
template <int D>
__global__ __launch_bounds__(kMergeThreads) void prefix_merge_kernel(PrefixShape s, const int32_t *__restrict__ prefix_len,
                                                           const int32_t *__restrict__ seq_lens, const int32_t *__restrict__ q_lens,
                                                           const float *__restrict__ part_ml, const float *__restrict__ part_acc,
                                                           float *__restrict__ out) {
    typedef float f4_t __attribute__((ext_vector_type(4)));
    constexpr int LANES = D / 4, GROUPS = kMergeThreads / LANES, AHEAD = 16 / GROUPS;
    __shared__ __attribute__((aligned(16))) float sums[GROUPS][D];
    __shared__ float ml_of[GROUPS][2];
    const int c = threadIdx.x % LANES, grp = threadIdx.x / LANES;
    const int64_t rows = static_cast<int64_t>(s.n_seq) * s.n_q * s.n_q_heads;
    for (int64_t orow = blockIdx.x; orow < rows; orow += gridDim.x) {
        const int head = static_cast<int>(orow % s.n_q_heads);
        const int sq = static_cast<int>(orow / s.n_q_heads), qi = sq % s.n_q, seq = sq / s.n_q;
        if (q_lens != nullptr && qi >= q_lens[seq]) continue;
        const int hpk = s.n_q_heads / s.n_kv_heads, kvh = head / hpk;
        auto ranges = [](int len, int splits) {  // those that have tokens, as the attention kernel divides them
            const int steps = (len + 31) / 32, per = splits > 0 ? (steps + splits - 1) / splits : 0;
            return per > 0 ? (steps + per - 1) / per : 0;
        };
        const int n_shared = s.prefix_splits > 0 ? ranges(min(max(prefix_len[0], 0), s.max_prefix), s.prefix_splits) : 0;
        const int n_own = s.own_splits > 0 ? ranges(min(max(seq_lens[seq], 0), s.max_len), s.own_splits) : 0;
        const int64_t first = (static_cast<int64_t>(kvh) * s.n_seq * s.n_q * hpk + static_cast<int64_t>(sq) * hpk + head % hpk) * s.prefix_splits;
        const int64_t second = s.own_partials + ((static_cast<int64_t>(seq) * s.n_kv_heads + kvh) * s.n_q * hpk + qi * hpk + head % hpk) * s.own_splits - n_shared;
        const int total = n_shared + n_own;

        float m = kNoTokenSeen, l = 0.0f;
        f4_t acc = f4_t{0.0f, 0.0f, 0.0f, 0.0f};
        for (int i0 = grp; i0 < total; i0 += AHEAD * GROUPS) {
            f4_t x[AHEAD];
            float2 ml[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int at = min(i0 + u * GROUPS, total - 1);
                const int64_t p = (at < n_shared ? first : second) + at;
                ml[u] = *reinterpret_cast<const float2 *>(part_ml + 2 * p);
                x[u] = *reinterpret_cast<const f4_t *>(part_acc + p * D + 4 * c);
            }
            float m_new = m;
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) m_new = fmaxf(m_new, ml[u].x);     // (the last one again is no larger)
            const float keep = exp2_raw(m - m_new);
            m = m_new;
            l *= keep;
            acc *= keep;
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (i0 + u * GROUPS < total) {
                    const float w = exp2_raw(ml[u].x - m);
                    l = fmaf(w, ml[u].y, l);
                    acc += w * x[u];
                }
        }
        *reinterpret_cast<f4_t *>(&sums[grp][4 * c]) = acc;
        if (c == 0) {
            ml_of[grp][0] = m;
            ml_of[grp][1] = l;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < D; e += kMergeThreads) {
            float m_all = kNoTokenSeen, l_all = 0.0f, sum = 0.0f;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) m_all = fmaxf(m_all, ml_of[g][0]);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const float w = exp2_raw(ml_of[g][0] - m_all);
                l_all = fmaf(w, ml_of[g][1], l_all);
                sum = fmaf(w, sums[g][e], sum);
            }
            const float inv = l_all == 0.0f ? 0.0f : 1.0f / l_all;   // (a sum that is no number stays none)
            out[orow * D + e] = sum * inv;
        }
        __syncthreads();
    }
}

int launch_prefix_merge(const octopus_plan_t &plan, const PrefixShape &s, const int32_t *prefix_len, const int32_t *seq_lens,
                        const int32_t *q_lens, const float *part_ml, const float *part_acc, float *out, void *stream) {
    const int64_t rows = static_cast<int64_t>(s.n_seq) * s.n_q * s.n_q_heads;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(rows < 65536 ? rows : 65536)), dim3(kMergeThreads), 0, static_cast<hipStream_t>(stream), s,
                           prefix_len, seq_lens, q_lens, part_ml, part_acc, out);
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

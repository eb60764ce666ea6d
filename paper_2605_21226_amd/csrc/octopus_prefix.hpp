// Attention of sequences that share a prefix, over pages: the prefix's tokens are read once for the rows of all sequences, each
// sequence's own tokens by itself (Alg. 2, with the flash-decoding identity joining the two).
//
// With q_rot = H diag(s) q and a key k^ = gamma D_s H u^ the score of row r and token t is
//     scale q . k^ = scale gamma_t sum_i rho_i (q_rot,i . n_i)           (Eq. (score-exact)),
// and a row's output is sum_t p_t v_t / sum_t p_t over the prefix's tokens and the own ones the row may see.
//
// Both products run on the matrix cores and a key is decoded straight into the operand registers: the dot product does not care in
// which order its terms come, so the terms are laid out as the table of (direction, norm) codes holds them -- (x, y, z, 0) of a
// triplet as four fp16 numbers and their four remainders, one 16-byte entry, half an operand of each.  A lane of group g = lane / 16
// decodes the g-th quarter of the triplets of key lane % 16.  No decoded key is written anywhere, no barrier is in the loop: a
// wavefront owns steps of 32 tokens (its records and value rows staged in LDS of its own) and 32 query rows, the wavefronts of a
// workgroup take the steps of a segment in turn, and their (m, l, acc) join at its end.
#ifndef OCTOPUS_PREFIX_HPP_
#define OCTOPUS_PREFIX_HPP_

#include "octopus_decode.hpp"

namespace octopus {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 prefix_bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t prefix_u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

constexpr int kPrefixKeys = 32;      // tokens of a step
constexpr int kPrefixRows = 32;      // query rows of a wavefront: two blocks of 16
constexpr float kUnitScale = 256.0f; // the table's numbers are 256 rho n: the remainders of small ones stay above fp16's denormals

template <class P>
struct PrefixCfg {
    static constexpr int D = P::D;
    static constexpr int NW = D <= 128 ? 8 : 4;                    // wavefronts of a workgroup: what LDS and registers hold
    static constexpr int NT = kWave * NW;
    // triplets of each class that a lane group decodes; one class: padded to whole operands
    static constexpr int T0 = P::NCLASS == 1 ? ((P::NTRI + 7) / 8) * 2 : (P::NT0 + 3) / 4;
    static constexpr int T1 = P::NCLASS == 2 ? (P::NT1 + 3) / 4 : 0;
    static constexpr int TPL = T0 + T1;
    static constexpr int KS = (TPL + 1) / 2;                       // operands (of two triplets) a key
    static constexpr bool J0 = joint_codes(P::BD0, P::BN0);
    static constexpr bool J1 = P::NCLASS == 2 && joint_codes(P::BD1, P::BN1);
    static_assert(P::NCLASS == 1 || (J0 && J1), "two classes have joint tables");
    static constexpr int E0 = J0 ? 1 << (2 * P::BD0 + P::BN0) : 1 << (2 * P::BD0);
    static constexpr int E1 = P::NCLASS == 2 ? 1 << (2 * P::BD1 + P::BN1) : 0;
    static constexpr int rep(int bytes, int budget) { return bytes * 8 <= budget ? 8 : (bytes * 4 <= budget ? 4 : (bytes * 2 <= budget ? 2 : 1)); }
    static constexpr int R0 = rep(E0 * 16, P::NCLASS == 2 ? 32768 : 65536);
    static constexpr int R1 = P::NCLASS == 2 ? rep(E1 * 16, 16384) : 1;
    static constexpr int log2i(int x) { return x <= 1 ? 0 : 1 + log2i(x / 2); }
    static constexpr int REC = P::GRANULES * kPrefixKeys * 16;     // bytes of a step's records
    static constexpr int VST = 2 * D + 32;                         // bytes of a staged value row: four rows lie on 32 different banks
    static constexpr int STAGE = REC + kPrefixKeys * VST;          // bytes of a wavefront's staging area
    static constexpr int NREC = (REC + 1023) / 1024;               // 16-byte pieces per lane
    static constexpr int NVAL = D / 16;
    static constexpr int QOP = kPrefixRows * 4 * KS * 16;          // bytes of the query operands, leading parts (the remainders as many)
    static_assert(2 * QOP <= NW * STAGE, "the query operands share the staging areas");
    static_assert(NW * 16 * D * 4 <= NW * STAGE + 0 * D, "so do the wavefronts' results");
};

template <class P>
struct PrefixSmem {
    using C = PrefixCfg<P>;
    uint4 tab0[C::E0 * C::R0];
    uint4 tab1[P::NCLASS == 2 ? C::E1 * C::R1 : 1];
    unsigned char stage[C::NW][C::STAGE];
    float ml[C::NW][kPrefixRows][2];
    float factor[kPrefixRows];         // of a row's scores
    float c_xi[P::NCLASS][1 << (P::BD0 > P::BD1 ? P::BD0 : P::BD1)];
    float c_rho[P::NCLASS][1 << (P::BN0 > P::BN1 ? P::BN0 : P::BN1)];
};

// 256 (x, y, z, 0) as fp16 and the remainders as fp16: together 22 bits of each (a product drops the remainders' product only).
__device__ __forceinline__ uint4 half_triplet(float x, float y, float z) {
    auto two = [](float a, float b) {
        const auto h = __builtin_amdgcn_cvt_pkrtz(a, b);
        return __builtin_bit_cast(uint32_t, h);
    };
    auto lower = [](uint32_t w) { return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(w))); };
    uint4 r;
    r.x = two(x, y);
    r.y = two(z, 0.0f);
    r.z = two(x - lower(r.x), y - lower(r.x >> 16));
    r.w = two(z - lower(r.y), 0.0f);
    return r;
}

template <class P>
__device__ __forceinline__ void build_prefix_tables(PrefixSmem<P> &sm, int tid) {
    using C = PrefixCfg<P>;
    auto one = [&](auto bd_, auto bn_, auto joint_, uint4 *tab, const float *c_xi, const float *c_rho, auto entries_, auto rep_) {
        constexpr int BD = decltype(bd_)::value, BN = decltype(bn_)::value, E = decltype(entries_)::value, REP = decltype(rep_)::value;
        constexpr bool JOINT = decltype(joint_)::value;
#pragma unroll 1
        for (int e = tid; e < E; e += C::NT) {
            const int dir = JOINT ? e >> BN : e;
            const float4 n = oct_decode(c_xi[dir & ((1 << BD) - 1)], c_xi[dir >> BD]);
            uint4 val;
            if constexpr (JOINT) {
                const float rho = c_rho[e & ((1 << BN) - 1)] * kUnitScale;
                val = half_triplet(rho * n.x, rho * n.y, rho * n.z);
            } else {
                val = make_uint4(__float_as_uint(n.x), __float_as_uint(n.y), __float_as_uint(n.z), 0u);
            }
#pragma unroll
            for (int r = 0; r < REP; ++r) tab[e * REP + ((r + tid) & (REP - 1))] = val;   // (neighbouring threads on different banks)
        }
    };
    using std::integral_constant;
    one(integral_constant<int, P::BD0>{}, integral_constant<int, P::BN0>{}, integral_constant<bool, C::J0>{}, sm.tab0, sm.c_xi[0], sm.c_rho[0],
        integral_constant<int, C::E0>{}, integral_constant<int, C::R0>{});
    if constexpr (P::NCLASS == 2)
        one(integral_constant<int, P::BD1>{}, integral_constant<int, P::BN1>{}, integral_constant<bool, C::J1>{}, sm.tab1, sm.c_xi[1],
            sm.c_rho[1], integral_constant<int, C::E1>{}, integral_constant<int, C::R1>{});
}

// N consecutive bits-wide fields of a lane group's quarter of a stream, in words of its own: word j holds bits 32 j .. of the quarter.
template <int START, int QUARTER_BITS>
struct QuarterStream {
    static constexpr int WORDS = (QUARTER_BITS + 31) / 32;
    static constexpr bool ALIGNED = START % 32 == 0 && QUARTER_BITS % 32 == 0;
    static constexpr int READ = ALIGNED ? WORDS : WORDS + 1;
};

template <class P>
__global__ __launch_bounds__(PrefixCfg<P>::NT) __attribute__((amdgpu_waves_per_eu(PrefixCfg<P>::D <= 128 ? 2 : 1))) void prefix_attention_kernel(
    DeviceBooks books, PrefixShape shp, const unsigned char *__restrict__ k_pool, const unsigned char *__restrict__ v_pool,
    const int32_t *__restrict__ prefix_table, const int32_t *__restrict__ prefix_len, const int32_t *__restrict__ block_table,
    const int32_t *__restrict__ seq_lens, const int32_t *__restrict__ q_lens, float *__restrict__ part_ml,
    float *__restrict__ part_acc) {
    using C = PrefixCfg<P>;
    constexpr int D = P::D, NW = C::NW, KS = C::KS;
    constexpr int CB = D / 16;                       // blocks of 16 channels
    constexpr int64_t TILEB = P::GRANULES * kWave * 16, VTILEB = static_cast<int64_t>(kWave) * D * 2;
    __shared__ __attribute__((aligned(16))) PrefixSmem<P> sm;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, g = lane >> 4;

    // levels, a lane each, then the tables
    {
        typedef const float __attribute__((address_space(4))) *arg_t;
        arg_t arg = (arg_t)__builtin_amdgcn_kernarg_segment_ptr();
        constexpr int NX = sizeof(sm.c_xi[0]) / 4, NR = sizeof(sm.c_rho[0]) / 4;
        if (wave < P::NCLASS) {
            const float xi = arg[offsetof(DeviceBooks, c_xi) / 4 + wave * kMaxLevels + lane], rho = arg[offsetof(DeviceBooks, c_rho) / 4 + wave * kMaxLevels + lane];
            if (lane < NX) sm.c_xi[wave][lane] = xi;
            if (lane < NR) sm.c_rho[wave][lane] = rho * (C::J0 ? 1.0f : kUnitScale);
        }
    }
    __syncthreads();
    build_prefix_tables<P>(sm, tid);

    unsigned char *stage = sm.stage[wave];
    // where this lane's code words lie in the staged records (of key n; + 256 for key 16 + n)
    constexpr int DQ0 = C::T0 * 2 * P::BD0, NQ0 = C::T0 * P::BN0, DQ1 = C::T1 * 2 * P::BD1, NQ1 = C::T1 * P::BN1;
    using SD0 = QuarterStream<P::DIR0_BIT, DQ0>;
    using SN0 = QuarterStream<P::NRM0_BIT, NQ0>;
    using SD1 = QuarterStream<P::DIR1_BIT, (DQ1 > 0 ? DQ1 : 32)>;
    using SN1 = QuarterStream<P::NRM1_BIT, (NQ1 > 0 ? NQ1 : 32)>;
    auto word_at = [&](int w) { return ((w >> 2) * (kPrefixKeys * 16)) + (w & 3) * 4 + n * 16; };
    // (the last quarter's padding may lie past the record: words past it are its last one, and their terms meet zeros)
    auto quarter = [&](auto stream_, int start, int quarter_bits, auto &words, int block) __attribute__((always_inline)) {
        using S = decltype(stream_);
        const int bit = start + g * quarter_bits;
        const int first = bit >> 5;
        uint32_t raw[S::READ];
#pragma unroll
        for (int j = 0; j < S::READ; ++j)
            raw[j] = *reinterpret_cast<const uint32_t *>(stage + word_at(min(first + j, P::NWORDS - 1)) + block * 256);
        if constexpr (S::ALIGNED) {
#pragma unroll
            for (int j = 0; j < S::WORDS; ++j) words[j] = raw[j];
        } else {
#pragma unroll
            for (int j = 0; j < S::WORDS; ++j) words[j] = __builtin_amdgcn_alignbit(raw[j + 1], raw[j], bit & 31);
        }
    };

    const int hpk = shp.n_q_heads / shp.n_kv_heads;
    const int all_rows = shp.n_seq * shp.n_q * hpk, own_rows = shp.n_q * hpk;
    // what a factor of 256 in the keys and the units of log2 make of the caller's scale
    const float norm = shp.scale * kLog2e * (D == 64 ? 0.125f : (D == 128 ? 0.08838834764831845f : 0.0625f)) / kUnitScale;

    for (int seg = blockIdx.x; seg < shp.n_segments; seg += gridDim.x) {
        // ---- which (prefix or sequence, KV head, row group, split) this is ----
        const bool shared = seg < shp.prefix_segments;
        int i = shared ? seg : seg - shp.prefix_segments;
        const int groups = shared ? shp.prefix_groups : shp.own_groups, splits = shared ? shp.prefix_splits : shp.own_splits;
        const int grp = i % groups;
        i /= groups;
        const int split = i % splits;
        i /= splits;
        const int kvh = i % shp.n_kv_heads, seq = i / shp.n_kv_heads;   // (seq: 0 for the prefix)
        const int len = shared ? min(max(prefix_len[0], 0), shp.max_prefix) : min(max(seq_lens[seq], 0), shp.max_len);
        const int steps = (len + kPrefixKeys - 1) / kPrefixKeys, per = (steps + splits - 1) / splits;
        const int begin = split * per, end = min(begin + per, steps);
        if (begin >= end) continue;   // (nothing of it is written and the merge reads nothing of it; uniform over the workgroup)
        const int32_t *pages = shared ? prefix_table : block_table + static_cast<int64_t>(seq) * shp.max_pages;
        const int rows = shared ? all_rows : own_rows, row0 = grp * kPrefixRows;
        const int live = min(2, (rows - row0 + 15) / 16);               // blocks of 16 rows with rows

        // ---- a step's records and values: from memory to registers ----
        prefix_u32x4_t rec[C::NREC], val[C::NVAL];
        auto page_of = [&](int step) __attribute__((always_inline)) {
            return min(max(pages[min(step, end - 1) / 2], 0), shp.n_pages - 1);
        };
        auto load_step = [&](int step, int page) __attribute__((always_inline)) {
            const int64_t tile = static_cast<int64_t>(page) * shp.n_kv_heads + kvh;
            const int first = (step & 1) * kPrefixKeys;   // of the page's tokens
            const unsigned char *src = k_pool + tile * TILEB + first * 16;
#pragma unroll
            for (int e = 0; e < C::NREC; ++e) {
                const int piece = min(lane + 64 * e, P::GRANULES * kPrefixKeys - 1);
                rec[e] = *reinterpret_cast<const prefix_u32x4_t *>(src + (piece / kPrefixKeys) * (kWave * 16) + (piece % kPrefixKeys) * 16);
            }
            // (value rows past the end are the last one: their probabilities are zero, but what lies there may be no number)
            const unsigned char *vsrc = v_pool + tile * VTILEB;
            const int last = len - 1 - step * kPrefixKeys;
#pragma unroll
            for (int e = 0; e < C::NVAL; ++e) {
                const int piece = lane + 64 * e, row = first + min(piece / (D / 8), last);
                val[e] = *reinterpret_cast<const prefix_u32x4_t *>(vsrc + row * (2 * D) + (piece % (D / 8)) * 16);
            }
        };
        auto store_step = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < C::NREC; ++e)
                if (C::REC % 1024 == 0 || lane + 64 * e < P::GRANULES * kPrefixKeys)
                    *reinterpret_cast<prefix_u32x4_t *>(stage + (lane + 64 * e) * 16) = rec[e];
#pragma unroll
            for (int e = 0; e < C::NVAL; ++e) {
                const int piece = lane + 64 * e;
                *reinterpret_cast<prefix_u32x4_t *>(stage + C::REC + (piece / (D / 8)) * C::VST + (piece % (D / 8)) * 16) = val[e];
            }
        };
        const bool work = begin + wave < end;
        int next_page = 0;
        if (work) {
            load_step(begin + wave, page_of(begin + wave));
            next_page = page_of(begin + wave + NW);
        }

        // ---- the segment's queries: rotated, then as operands through LDS ----
        __syncthreads();                 // tables complete; the last segment's results have been read
        unsigned char *qop = sm.stage[0];
        for (int e = tid; e < 2 * C::QOP / 16; e += C::NT) reinterpret_cast<uint4 *>(qop)[e] = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
        {
            constexpr int EPL = D / 64, RPW = kPrefixRows / NW;
            int slot[EPL];
#pragma unroll
            for (int j = 0; j < EPL; ++j) {
                const int c = lane + 64 * j, t = c / 3;
                const bool second = P::NCLASS == 2 && t >= P::NT0;
                const int of = second ? t - P::NT0 : t, each = second ? (C::T1 > 0 ? C::T1 : 1) : C::T0;
                const int at = of % each + (second ? C::T0 : 0);
                slot[j] = ((of / each) * KS + at / 2) * 16 + ((at % 2) * 4 + c % 3) * 2;
            }
            float x[RPW][EPL];
#pragma unroll
            for (int r = 0; r < RPW; ++r) {
                const int row = min(row0 + wave * RPW + r, rows - 1);
                const int64_t sq = static_cast<int64_t>(seq) * shp.n_q + row / hpk;
                const int64_t at = (sq * shp.n_q_heads + kvh * hpk + row % hpk) * D;
#pragma unroll
                for (int j = 0; j < EPL; ++j) {
                    const int64_t e = at + lane + 64 * j;
                    x[r][j] = shp.q_is_bf16 ? __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t *>(shp.q)[e]) << 16)
                                            : static_cast<const float *>(shp.q)[e];
                }
            }
            uint32_t neg[EPL];
#pragma unroll
            for (int j = 0; j < EPL; ++j) neg[j] = static_cast<uint32_t>(shp.signs[kvh * (D / 8) + (lane + 64 * j) / 8] >> (lane % 8)) << 31;
#pragma unroll
            for (int r = 0; r < RPW; ++r) {
                const bool there = row0 + wave * RPW + r < rows;
#pragma unroll
                for (int j = 0; j < EPL; ++j) x[r][j] = there ? __uint_as_float(__float_as_uint(x[r][j]) ^ neg[j]) : 0.0f;
            }
            static_for<0, 6>([&](auto bb) {
                constexpr int m = 1 << decltype(bb)::value;
#pragma unroll
                for (int r = 0; r < RPW; ++r)
#pragma unroll
                    for (int j = 0; j < EPL; ++j) {
                        const float other = lane_xor<m>(x[r][j], lane);
                        x[r][j] = (lane & m) ? other - x[r][j] : x[r][j] + other;
                    }
            });
#pragma unroll
            for (int m = 1; m < EPL; m <<= 1)
#pragma unroll
                for (int r = 0; r < RPW; ++r)
#pragma unroll
                    for (int j = 0; j < EPL; ++j)
                        if ((j & m) == 0) {
                            const float a = x[r][j], b = x[r][j | m];
                            x[r][j] = a + b;
                            x[r][j | m] = a - b;
                        }
#pragma unroll
            for (int r = 0; r < RPW; ++r) {
                // a power of two brings the row's largest number into [1/2, 1): fp16 has no range to spare
                float top = 0.0f;
#pragma unroll
                for (int j = 0; j < EPL; ++j) top = fmaxf(top, fabsf(x[r][j]));
                static_for<0, 6>([&](auto bb) { top = fmaxf(top, lane_xor<(1 << decltype(bb)::value)>(top, lane)); });
                const int e = top > 0.0f && top < INFINITY ? __builtin_amdgcn_frexp_expf(top) : 0;
                const int row = wave * RPW + r;
                if (lane == 0) sm.factor[row] = ldexpf(norm, e);
#pragma unroll
                for (int j = 0; j < EPL; ++j) {
                    const float y = ldexpf(x[r][j], -e);
                    const _Float16 hi = static_cast<_Float16>(y);
                    const _Float16 lo = static_cast<_Float16>(y - static_cast<float>(hi));
                    unsigned char *to = qop + row * (4 * KS * 16) + slot[j];
                    *reinterpret_cast<_Float16 *>(to) = hi;
                    *reinterpret_cast<_Float16 *>(to + C::QOP) = lo;
                }
            }
        }
        __syncthreads();
        half8_t qh[2][KS], ql[2][KS];
        float factor[2];
        int limit[2];                    // tokens that the row sees
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) {
            const unsigned char *from = qop + ((rb * 16 + n) * 4 + g) * (KS * 16);
#pragma unroll
            for (int kk = 0; kk < KS; ++kk) {
                qh[rb][kk] = *reinterpret_cast<const half8_t *>(from + kk * 16);
                ql[rb][kk] = *reinterpret_cast<const half8_t *>(from + C::QOP + kk * 16);
            }
            factor[rb] = sm.factor[rb * 16 + n];
            limit[rb] = len;
            const int row = row0 + rb * 16 + n;
            if (!shared && shp.causal && row < rows) {
                const int nq = q_lens != nullptr ? min(max(q_lens[seq], 0), shp.n_q) : shp.n_q;
                limit[rb] = min(max(len - nq + row / hpk + 1, 0), len);
            }
        }
        __syncthreads();                 // the operands have been read: the staging areas are the wavefronts' own now

        // ---- the steps ----
        float m_ref[2] = {-1e30f, -1e30f}, l_run[2] = {0.0f, 0.0f};   // (-1e30: no token seen yet)
        f32x4_t oacc[2][CB];
#pragma unroll
        for (int rb = 0; rb < 2; ++rb)
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) oacc[rb][cb] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

        for (int step = begin + wave; step < end; step += NW) {
            __builtin_amdgcn_wave_barrier();
            store_step();
            __builtin_amdgcn_wave_barrier();
            if (step + NW < end) {
                load_step(step + NW, next_page);
                next_page = page_of(step + 2 * NW);
            }
            f32x4_t score[2][2];         // [key block][row block]: lane (n, g) has keys 4 g .. + 3 of row n
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                uint32_t wd0[SD0::WORDS], wn0[SN0::WORDS];
                quarter(SD0{}, P::DIR0_BIT, DQ0, wd0, kb);
                quarter(SN0{}, P::NRM0_BIT, NQ0, wn0, kb);
                [[maybe_unused]] uint32_t wd1[SD1::WORDS], wn1[SN1::WORDS];
                if constexpr (P::NCLASS == 2) {
                    quarter(SD1{}, P::DIR1_BIT, DQ1, wd1, kb);
                    quarter(SN1{}, P::NRM1_BIT, NQ1, wn1, kb);
                }
                score[kb][0] = score[kb][1] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
                static_for<0, KS>([&](auto kk_) {
                    constexpr int kk = decltype(kk_)::value;
                    auto entry = [&](auto at_) __attribute__((always_inline)) -> uint4 {
                        constexpr int at = decltype(at_)::value;
                        if constexpr (at >= C::TPL) {
                            return make_uint4(0u, 0u, 0u, 0u);
                        } else if constexpr (at < C::T0) {
                            const uint32_t dir = field_clamped<at * 2 * P::BD0, 2 * P::BD0>(wd0), nrm = field_clamped<at * P::BN0, P::BN0>(wn0);
                            if constexpr (C::J0) {
                                constexpr int NS = C::log2i(C::R0);
                                return sm.tab0[(dir << (NS + P::BN0)) + (nrm << NS) + (lane & (C::R0 - 1))];
                            } else {
                                const uint4 d4 = sm.tab0[dir * C::R0 + (lane & (C::R0 - 1))];
                                const float rho = sm.c_rho[0][nrm];
                                return half_triplet(rho * __uint_as_float(d4.x), rho * __uint_as_float(d4.y), rho * __uint_as_float(d4.z));
                            }
                        } else if constexpr (P::NCLASS == 2) {
                            constexpr int a1 = at - C::T0, NS = C::log2i(C::R1);
                            const uint32_t dir = field_clamped<a1 * 2 * P::BD1, 2 * P::BD1>(wd1), nrm = field_clamped<a1 * P::BN1, P::BN1>(wn1);
                            return sm.tab1[(dir << (NS + P::BN1)) + (nrm << NS) + (lane & (C::R1 - 1))];
                        }
                    };
                    const uint4 a = entry(std::integral_constant<int, 2 * kk>{}), b = entry(std::integral_constant<int, 2 * kk + 1>{});
                    const half8_t kh = __builtin_bit_cast(half8_t, make_uint4(a.x, a.y, b.x, b.y));
                    const half8_t kl = __builtin_bit_cast(half8_t, make_uint4(a.z, a.w, b.z, b.w));
#pragma unroll
                    for (int rb = 0; rb < 2; ++rb) {
                        if (rb >= live) break;   // (uniform)
                        score[kb][rb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh, qh[rb][kk], score[kb][rb], 0, 0, 0);
                        score[kb][rb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh, ql[rb][kk], score[kb][rb], 0, 0, 0);
                        score[kb][rb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kl, qh[rb][kk], score[kb][rb], 0, 0, 0);
                    }
                });
            }
            float gamma[2][4];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 4; ++e) gamma[kb][e] = *reinterpret_cast<const float *>(stage + (kb * 16 + 4 * g + e) * 16);

            uint32_t ph[2][4], pl[2][4];
#pragma unroll
            for (int rb = 0; rb < 2; ++rb) {
                if (rb >= live) break;
                float t[8];
                float top = -INFINITY;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    t[e] = score[e / 4][rb][e % 4] * gamma[e / 4][e % 4];
                    const int tok = step * kPrefixKeys + (e / 4) * 16 + 4 * g + e % 4;
                    t[e] = tok < limit[rb] ? t[e] * factor[rb] : -INFINITY;
                    top = fmaxf(top, t[e]);
                }
                // probabilities are 2^(score - m_ref); the reference moves when a score exceeds it by more than 8
                if (__ballot(top > m_ref[rb] + 8.0f) != 0) {
                    top = fmaxf(top, lane_xor<16>(top, lane));
                    top = fmaxf(top, lane_xor<32>(top, lane));
                    const float m_new = fmaxf(m_ref[rb], top);
                    const float alpha = exp2_raw(m_ref[rb] - m_new);
                    m_ref[rb] = m_new;
                    l_run[rb] *= alpha;
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb) oacc[rb][cb] *= alpha;
                }
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float p0 = exp2_raw(t[e] - m_ref[rb]), p1 = exp2_raw(t[e + 1] - m_ref[rb]);
                    l_run[rb] += p0 + p1;
                    // two bf16 numbers whose sum is p to 2^-16: the values are bf16
                    const uint32_t b0 = __float_as_uint(p0), b1 = __float_as_uint(p1);
                    const float r0 = p0 - __uint_as_float(b0 & 0xffff0000u), r1 = p1 - __uint_as_float(b1 & 0xffff0000u);
                    ph[rb][e / 2] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
                    pl[rb][e / 2] = bf16_rne(r0) | (bf16_rne(r1) << 16);
                }
            }
            // O^T += V^T P^T: k-slots 8 g .. + 3 are keys 4 g .. + 3 of the first block, the next four those of the second
            typedef __attribute__((address_space(3))) s16x4_t *tr_t;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                unsigned char *at = stage + C::REC + (4 * g + n / 4) * C::VST + (16 * cb + 4 * (n % 4)) * 2;
                union { s16x4_t h[2]; prefix_bf16x8_t b; } v;
                v.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)at);
                v.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)(at + 16 * C::VST));
#pragma unroll
                for (int rb = 0; rb < 2; ++rb) {
                    if (rb >= live) break;
                    oacc[rb][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.b, __builtin_bit_cast(prefix_bf16x8_t, make_uint4(ph[rb][0], ph[rb][1], ph[rb][2], ph[rb][3])), oacc[rb][cb], 0, 0, 0);
                    oacc[rb][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.b, __builtin_bit_cast(prefix_bf16x8_t, make_uint4(pl[rb][0], pl[rb][1], pl[rb][2], pl[rb][3])), oacc[rb][cb], 0, 0, 0);
                }
            }
        }

        // ---- the wavefronts' results join ----
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) {
            l_run[rb] += lane_xor<16>(l_run[rb], lane);
            l_run[rb] += lane_xor<32>(l_run[rb], lane);
            if (g == 0) {
                sm.ml[wave][rb * 16 + n][0] = m_ref[rb];
                sm.ml[wave][rb * 16 + n][1] = l_run[rb];
            }
        }
        __syncthreads();                 // (the staging areas are free from here on, too)
        float *out = reinterpret_cast<float *>(sm.stage[0]);   // [wavefront][16 rows][D]
        const int64_t prow0 = shared ? static_cast<int64_t>(kvh) * all_rows * splits
                                     : shp.own_partials + (static_cast<int64_t>(seq) * shp.n_kv_heads + kvh) * own_rows * splits;
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) {
            if (rb >= live) break;
            float m_all = -1e30f;
#pragma unroll
            for (int w = 0; w < NW; ++w) m_all = fmaxf(m_all, sm.ml[w][rb * 16 + n][0]);
            const float weight = exp2_raw(m_ref[rb] - m_all);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                *reinterpret_cast<f32x4_t *>(out + (wave * 16 + n) * D + 16 * cb + 4 * g) = oacc[rb][cb] * weight;
            __syncthreads();
            for (int e = tid; e < 16 * D / 4; e += C::NT) {
                const int r = e / (D / 4), row = row0 + rb * 16 + r;
                if (row >= rows) continue;
                f32x4_t sum = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int w = 0; w < NW; ++w) sum += *reinterpret_cast<const f32x4_t *>(out + (w * 16 + r) * D + (e % (D / 4)) * 4);
                const int64_t prow = prow0 + static_cast<int64_t>(row) * splits + split;
                *reinterpret_cast<f32x4_t *>(part_acc + prow * D + (e % (D / 4)) * 4) = sum;
                if (e % (D / 4) == 0) {
                    float m = -1e30f, l = 0.0f;
#pragma unroll
                    for (int w = 0; w < NW; ++w) m = fmaxf(m, sm.ml[w][rb * 16 + r][0]);
#pragma unroll
                    for (int w = 0; w < NW; ++w) l += sm.ml[w][rb * 16 + r][1] * exp2_raw(sm.ml[w][rb * 16 + r][0] - m);
                    part_ml[prow * 2] = m;
                    part_ml[prow * 2 + 1] = l;
                }
            }
            __syncthreads();
        }
    }
}

template <class P>
int launch_prefix_plan(const octopus_codebooks_t &cb, const PrefixShape &s, const void *k_pool, const void *v_pool, const int32_t *prefix_table,
                       const int32_t *prefix_len, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens, float *part_ml,
                       float *part_acc, hipStream_t stream) {
    const DeviceBooks books = device_books(cb);
    const int grid = s.n_segments < 256 ? s.n_segments : 256;
    hipLaunchKernelGGL(prefix_attention_kernel<P>, dim3(grid), dim3(PrefixCfg<P>::NT), 0, stream, books, s,
                       static_cast<const unsigned char *>(k_pool), static_cast<const unsigned char *>(v_pool), prefix_table, prefix_len,
                       block_table, seq_lens, q_lens, part_ml, part_acc);
    return static_cast<int>(hipGetLastError());
}

}  // namespace octopus

#endif

// Attention of sequences that share a prefix, over pages: the prefix's tokens are read once for the rows of all sequences, each
// sequence's own tokens by itself (Alg. 2, with the flash-decoding identity joining the two).
//
// With q_rot = H diag(s) q and a key k^ = gamma D_s H u^ the score of row r and token t is
//     scale q . k^ = scale gamma_t sum_i rho_i (q_rot,i . n_i)           (Eq. (score-exact)),
// and a row's output is sum_t p_t v_t / sum_t p_t over the prefix's tokens and the own ones the row may see.
//
// Both products run on the matrix cores and a key is decoded straight into the operand registers: the dot product does not care in
// which order its terms come, so a lane of group g = lane / 16 decodes the g-th quarter of the triplets of key lane % 16 and puts their
// coordinates one after the other into the eight places that it has in each operand.  A table by (direction, norm) codes holds
// (x, y, z, 0) of a triplet as four fp16 numbers and their four remainders, a 16-byte entry; three products -- leading parts, and either
// one with the other's remainders -- give 22 bits of each factor.  Probabilities are three bf16 numbers each, values are bf16 as they are.
//
// No decoded key is written anywhere and no barrier is in the loop: a wavefront owns steps of 32 tokens (its records and value rows
// staged in LDS of its own) and 32 query rows, 16 at head dimension 256; the wavefronts of a workgroup take the steps of a segment in
// turn, and their (m, l, acc) join at its end.  At most 256 workgroups, one a compute unit (the tables fill LDS and are built once),
// walk the segments: the prefix's first, then the own ones; the row groups that read the same tokens on one die.
//
// What bounds it: the vector units, the matrix cores and LDS, in turns, with two wavefronts a SIMD to hide one behind the other (the
// accumulators and the queries' operands leave room for no third).  16 sequences of 32 heads behind 65531 tokens with 512 own ones, d = 128,
// 3 bits: 186 MB in 75 us (2.5 TB/s; at a plain read's rate, 7.07, it would be 26), vector units active 52 % of it, matrix cores 39 %, LDS
// 38 %.  A step of 32 tokens and 32 rows is 108 matrix instructions (1730 clocks) and some 440 vector ones (1760).
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
constexpr float kUnitScale = 256.0f; // the table's numbers are 256 rho n: the remainders of small ones stay above fp16's denormals (the host
                                     // takes the factor out of the scale again)

template <class P>
struct PrefixCfg {
    static constexpr int D = P::D;
    // Wavefronts of a workgroup (two per SIMD, or one with all its registers) and blocks of 16 query rows of each: a key is decoded
    // once for a wavefront's rows.
    static constexpr int NW = prefix_waves(D);
    static constexpr int RB = prefix_rows(D) / 16;
    static constexpr int ROWS = 16 * RB;
    static constexpr int NT = kWave * NW;
    // triplets of each class that a lane group decodes
    static constexpr int T0 = ((P::NCLASS == 1 ? P::NTRI : P::NT0) + 3) / 4;
    static constexpr int T1 = P::NCLASS == 2 ? (P::NT1 + 3) / 4 : 0;
    static constexpr int TPL = T0 + T1;
    static constexpr int KS = (3 * TPL + 7) / 8;                   // operands of a key: eight coordinates each, a lane group's one after the other
    static constexpr bool J0 = joint_codes(P::BD0, P::BN0);
    static constexpr bool J1 = P::NCLASS == 2 && joint_codes(P::BD1, P::BN1);
    static_assert(P::NCLASS == 1 || (J0 && J1), "two classes have joint tables");
    static constexpr int E0 = J0 ? 1 << (2 * P::BD0 + P::BN0) : 1 << (2 * P::BD0);
    static constexpr int E1 = P::NCLASS == 2 ? 1 << (2 * P::BD1 + P::BN1) : 0;
    static constexpr int rep(int bytes, int budget) { return bytes * 16 <= budget ? 16 : bytes * 8 <= budget ? 8 : (bytes * 4 <= budget ? 4 : (bytes * 2 <= budget ? 2 : 1)); }
    static constexpr int log2i(int x) { return x <= 1 ? 0 : 1 + log2i(x / 2); }
    // bytes of a staged record, an odd number of sixteens: 16 keys' words at one place of the record lie on 16 different sets of banks
    // (at head dimension 256 eight sixteens cost 2000 clocks a step, a quarter of it)
    static constexpr int RST = ((P::GRANULES + 1) | 1) * 16;
    static constexpr int REC = RST * kPrefixKeys;                  // bytes of a step's records
    static constexpr int NREC = (P::GRANULES + 1) / 2;              // 16-byte pieces per lane
    // A step's value rows go from memory to LDS directly, 1 KB per instruction: instruction i takes rows i, i + NVAL, ..; 32 bytes
    // between the instructions' pieces put four rows that follow each other on 32 different banks (the transposed reads take four).
    static constexpr int NVAL = D / 16;
    static constexpr int VST = 1024 + 32;
    static constexpr bool VREG = D == 256;
    static constexpr int VAL = NVAL * VST;                         // bytes of a step's values
    // Query operands in LDS: a row's leading parts and its remainders; rows 16 bytes apart beyond their size, so that the 16 rows read
    // at once lie on all banks.  The wavefronts' results, which take the values' place: rows 16 bytes apart for the same reason.
    static constexpr int QST = 2 * 4 * KS * 16 + 16;
    static constexpr int OST = D + 4;                              // floats
    static constexpr int STAGED = ROWS * QST > NW * REC ? ROWS * QST : NW * REC;
    static constexpr int PLACE = NW * VAL > NW * 16 * OST * 4 ? NW * VAL : NW * 16 * OST * 4;
    // Copies of the tables' entries, 16 bytes apart, in what is left of LDS (4 KB of it for what is small).
    static constexpr int LEFT = 160 * 1024 - PLACE - STAGED - 4096;
    static constexpr int R0 = rep(E0 * 16, P::NCLASS == 2 ? 32768 : (LEFT < 65536 ? LEFT : 65536));
    static constexpr int R1 = P::NCLASS == 2 ? rep(E1 * 16, 16384) : 1;
    // The transform of the queries: eight coordinates a thread.
    static constexpr int QLANES = D / 8, QROWS = NT / QLANES, QPASS = (ROWS + QROWS - 1) / QROWS;
};

template <class P>
struct PrefixTables {
    using C = PrefixCfg<P>;
    uint4 tab0[C::E0 * C::R0];
    uint4 tab1[P::NCLASS == 2 ? C::E1 * C::R1 : 1];
};

template <class P>
struct PrefixSmem {
    using C = PrefixCfg<P>;
    float ml[C::NW][C::ROWS][2];
    float factor[C::ROWS];         // of a row's scores
    float c_xi[P::NCLASS][1 << (P::BD0 > P::BD1 ? P::BD0 : P::BD1)];
    float c_rho[P::NCLASS][1 << (P::BN0 > P::BN1 ? P::BN0 : P::BN1)];
};

// 256 (x, y, z, 0) as fp16 and the remainders as fp16, each rounded to the nearest: together 22 bits of each (a product drops the
// remainders' product only).
__device__ __forceinline__ uint4 half_triplet(float x, float y, float z) {
    auto two = [](float a, float b) {
        typedef float f32x2_t __attribute__((ext_vector_type(2)));
        typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), half2_t));
    };
    auto lower = [](uint32_t w) { return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(w))); };
    uint4 r;
    r.x = two(x, y);
    r.y = two(z, 0.0f);
    r.z = two(x - lower(r.x), y - lower(r.x >> 16));
    r.w = two(z - lower(r.y), 0.0f);
    return r;
}

// fp32 numbers as bf16, cut off: one as fp32 again, two in a word, the first in the lower half.
__device__ __forceinline__ float bf16_cut(float a) { return __uint_as_float(__float_as_uint(a) & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf16_cut_pair(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }

// Until at most N of the loads from memory asked for are on their way (they arrive in order), and until LDS has answered.
template <int N>
__device__ __forceinline__ void wait_loads() {
    static_assert(N < 64, "six bits");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70);
    __asm__ volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_lds() {
    __builtin_amdgcn_s_waitcnt(0xc07f);
    __asm__ volatile("" ::: "memory");
}

// The workgroup's barrier for what is in LDS. (__syncthreads waits for every load and store to memory as well: for the partial results on
// their way out, whose acknowledgement takes 2000 clocks and more, and for the records and pages asked for ahead.)
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <class P>
__device__ __forceinline__ void build_prefix_tables(PrefixSmem<P> &sm, PrefixTables<P> &tb, int tid) {
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
    one(integral_constant<int, P::BD0>{}, integral_constant<int, P::BN0>{}, integral_constant<bool, C::J0>{}, tb.tab0, sm.c_xi[0], sm.c_rho[0],
        integral_constant<int, C::E0>{}, integral_constant<int, C::R0>{});
    if constexpr (P::NCLASS == 2)
        one(integral_constant<int, P::BD1>{}, integral_constant<int, P::BN1>{}, integral_constant<bool, C::J1>{}, tb.tab1, sm.c_xi[1],
            sm.c_rho[1], integral_constant<int, C::E1>{}, integral_constant<int, C::R1>{});
}

// N consecutive bits-wide fields of a lane group's quarter of a stream, in words of its own: word j holds bits 32 j .. of the quarter.
template <int START, int QUARTER_BITS>
struct QuarterStream {
    static constexpr int WORDS = (QUARTER_BITS + 31) / 32;
    static constexpr bool ALIGNED = START % 32 == 0 && QUARTER_BITS % 32 == 0;
    static constexpr int READ = ALIGNED ? WORDS : WORDS + 1;
    static constexpr int END = ((START + 3 * QUARTER_BITS) / 32 + READ) * 4;   // bytes of a record that the last group's quarter reaches
};

// CAUSAL: rows of a sequence may see fewer of its tokens than others.  (A kernel of its own: what it takes to keep values that are no
// numbers from the rows that do not see them costs the other one 4 to 10 % in registers.)
template <class P, bool CAUSAL>
__global__ __launch_bounds__(PrefixCfg<P>::NT) __attribute__((amdgpu_waves_per_eu(PrefixCfg<P>::NW / 4))) void prefix_attention_kernel(
    DeviceBooks books, PrefixShape shp, const unsigned char *__restrict__ k_pool, const unsigned char *__restrict__ v_pool,
    const int32_t *__restrict__ prefix_table, const int32_t *__restrict__ prefix_len, const int32_t *__restrict__ block_table,
    const int32_t *__restrict__ seq_lens, const int32_t *__restrict__ q_lens, float *__restrict__ part_ml,
    float *__restrict__ part_acc) {
    using C = PrefixCfg<P>;
    constexpr int D = P::D, NW = C::NW, KS = C::KS, RB = C::RB;
    constexpr int CB = D / 16;                       // blocks of 16 channels
    constexpr int64_t TILEB = P::GRANULES * kWave * 16, VTILEB = static_cast<int64_t>(kWave) * D * 2;
    __shared__ __attribute__((aligned(16))) PrefixSmem<P> sm;
    __shared__ __attribute__((aligned(16))) PrefixTables<P> tb;
    __shared__ __attribute__((aligned(16))) unsigned char staged[C::STAGED];   // a segment's query operands, then the wavefronts' staged records
    __shared__ __attribute__((aligned(16))) unsigned char place[C::PLACE];   // (an object of its own: reads of the tables need not wait for it)
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);

    unsigned char *stage = staged + wave * C::REC, *vals = place + wave * C::VAL;
    constexpr int DQ0 = C::T0 * 2 * P::BD0, NQ0 = C::T0 * P::BN0, DQ1 = C::T1 * 2 * P::BD1, NQ1 = C::T1 * P::BN1;
    using SD0 = QuarterStream<P::DIR0_BIT, DQ0>;
    using SN0 = QuarterStream<P::NRM0_BIT, NQ0>;
    using SD1 = QuarterStream<P::DIR1_BIT, (DQ1 > 0 ? DQ1 : 32)>;
    using SN1 = QuarterStream<P::NRM1_BIT, (NQ1 > 0 ? NQ1 : 32)>;
    static_assert(SD0::END <= C::RST && SN0::END <= C::RST && SD1::END <= C::RST && SN1::END <= C::RST, "within a staged record and its padding");
    const int hpk = shp.n_q_heads / shp.n_kv_heads;
    const int all_rows = shp.n_seq * shp.n_q * hpk, own_rows = shp.n_q * hpk;

    bool built = false;                  // the tables
    for (int seg = blockIdx.x; seg < shp.n_segments; seg += gridDim.x) {
        // (opaque: what follows from a lane's number is computed for each segment, not kept -- in scratch memory, whose reads would
        // wait for the values on their way -- from the kernel's start)
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
        const int lane = tid & 63, n = lane & 15, g = lane >> 4;
        // ---- which (prefix or sequence, KV head, row group, split) this is ----
        const bool shared = seg < shp.prefix_segments;
        // (neighbours in the grid lie on different dies: each die takes a run of the prefix's segments, so that the row groups that read
        // the same tokens find them in its L2 cache)
        int i = seg - shp.prefix_segments;
        if (shared) {
            const int die = seg % 8, each = shp.prefix_segments / 8, more = shp.prefix_segments % 8;
            i = die * each + min(die, more) + seg / 8;
        }
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
        const int rows = shared ? all_rows : own_rows, row0 = grp * C::ROWS;
        const int live = min(RB, (rows - row0 + 15) / 16);              // blocks of 16 rows with rows

        // ---- the levels and the segment's queries, asked for with the pages ----
        float xi = 0.0f, rho = 0.0f;
        if (!built && wave < P::NCLASS) {
            typedef const float __attribute__((address_space(4))) *arg_t;
            arg_t arg = (arg_t)__builtin_amdgcn_kernarg_segment_ptr();
            xi = arg[offsetof(DeviceBooks, c_xi) / 4 + wave * kMaxLevels + lane];
            rho = arg[offsetof(DeviceBooks, c_rho) / 4 + wave * kMaxLevels + lane];
        }
        const int qc = tid % C::QLANES;                  // coordinates 8 qc .. + 7
        prefix_u32x4_t asked[C::QPASS][2];
        uint32_t sbits = shp.signs[kvh * (D / 8) + qc];
#pragma unroll
        for (int p = 0; p < C::QPASS; ++p) {
            typedef uint32_t u32x4a_t __attribute__((ext_vector_type(4), aligned(4)));
            const int row = min(row0 + tid / C::QLANES + p * C::QROWS, rows - 1);
            const int64_t at = ((static_cast<int64_t>(seq) * shp.n_q + row / hpk) * shp.n_q_heads + kvh * hpk + row % hpk) * D + 8 * qc;
            const unsigned char *src = static_cast<const unsigned char *>(shp.q) + at * (shp.q_is_bf16 ? 2 : 4);
            asked[p][0] = *reinterpret_cast<const u32x4a_t *>(src);
            asked[p][1] = *reinterpret_cast<const u32x4a_t *>(src + (shp.q_is_bf16 ? 0 : 16));
        }
        // ---- a step's records, from memory to registers and from there to LDS; its values, from memory to LDS ----
        prefix_u32x4_t rec[C::NREC], second[C::NREC];
        // the pages of the wavefront's next 64 steps, one a lane
        int held = 0, held_from = 0;
        auto hold_pages = [&](int step) __attribute__((always_inline)) {
            held_from = step;
            held = pages[min(step + lane * NW, end - 1) / 2];
        };
        auto page_of = [&](int step) __attribute__((always_inline)) {
            return min(max(__builtin_amdgcn_readlane(held, (step - held_from) / NW), 0), shp.n_pages - 1);
        };
        constexpr bool HALF = P::GRANULES % 2 != 0;       // (an odd number of granules: the last piece is half the lanes')
        const uint32_t rec_at = (lane / kPrefixKeys) * (kWave * 16) + (lane % kPrefixKeys) * 16;
        auto load_records = [&](prefix_u32x4_t (&rec)[C::NREC], int step, int page) __attribute__((always_inline)) {
            const unsigned char *src = k_pool + (static_cast<int64_t>(page) * shp.n_kv_heads + kvh) * TILEB + (step & 1) * (kPrefixKeys * 16);
#pragma unroll
            for (int e = 0; e < C::NREC; ++e)
                if (!HALF || e + 1 < C::NREC || lane < 32)
                    rec[e] = *reinterpret_cast<const prefix_u32x4_t *>(src + (rec_at + e * (2 * kWave * 16)));
        };
        auto store_records = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < C::NREC; ++e)
                if (!HALF || e + 1 < C::NREC || lane < 32)
                    *reinterpret_cast<prefix_u32x4_t *>(stage + (lane % kPrefixKeys) * C::RST + (lane / kPrefixKeys + 2 * e) * 16) = rec[e];
        };
        constexpr int LPR = D / 8;                       // lanes per value row
        const uint32_t val_at = (lane / LPR) * (C::NVAL * 2 * D) + (lane % LPR) * 16;
        [[maybe_unused]] prefix_u32x4_t val[C::VREG ? C::NVAL : 1];
        auto load_values = [&](int step, int page) __attribute__((always_inline)) {
            const unsigned char *src = v_pool + (static_cast<int64_t>(page) * shp.n_kv_heads + kvh) * VTILEB + (step & 1) * (kPrefixKeys * 2 * D);
#pragma unroll
            for (int e = 0; e < C::NVAL; ++e)
                if constexpr (C::VREG)
                    val[e] = *reinterpret_cast<const prefix_u32x4_t *>(src + (val_at + e * (2 * D)));
                else
                    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(src + (val_at + e * (2 * D))),
                                                     (__attribute__((address_space(3))) void *)(vals + e * C::VST), 16, 0, 0);
        };
        [[maybe_unused]] auto store_values = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < C::NVAL; ++e) *reinterpret_cast<prefix_u32x4_t *>(vals + e * C::VST + lane * 16) = val[e];
        };
        const bool work = begin + wave < end;
        if (work) hold_pages(begin + wave);
        if (!built && wave < P::NCLASS) {    // (they have arrived with the pages; a lane each)
            constexpr int NX = sizeof(sm.c_xi[0]) / 4, NR = sizeof(sm.c_rho[0]) / 4;
            if (lane < NX) sm.c_xi[wave][lane] = xi;
            if (lane < NR) sm.c_rho[wave][lane] = rho * (C::J0 ? 1.0f : kUnitScale);
        }
        // (all of it is waited for here, where the pages are, and not behind the records and values)
        asm volatile("" : "+v"(xi), "+v"(rho), "+v"(held), "+v"(sbits));
#pragma unroll
        for (int p = 0; p < C::QPASS; ++p) asm volatile("" : "+v"(asked[p][0]), "+v"(asked[p][1]));
        if (work) {
            load_records(rec, begin + wave, page_of(begin + wave));
            // (of the second step, too: before the first values, which the loop's waits for records are not to wait for)
            if (begin + wave + NW < end) load_records(second, begin + wave + NW, page_of(begin + wave + NW));
            if constexpr (C::VREG) load_values(begin + wave, page_of(begin + wave));
        }

        // (the last quarter may reach past the record, into its padding: those terms meet zeros)
        auto quarter = [&](auto stream_, int start, int quarter_bits, auto &words, int block) __attribute__((always_inline)) {
            using S = decltype(stream_);
            const int bit = start + g * quarter_bits;
            const unsigned char *first = stage + n * C::RST + (bit >> 5) * 4 + block * (16 * C::RST);
            uint32_t raw[S::READ];
    #pragma unroll
            for (int j = 0; j < S::READ; ++j) raw[j] = *reinterpret_cast<const uint32_t *>(first + 4 * j);
            if constexpr (S::ALIGNED) {
    #pragma unroll
                for (int j = 0; j < S::WORDS; ++j) words[j] = raw[j];
            } else {
    #pragma unroll
                for (int j = 0; j < S::WORDS; ++j) words[j] = __builtin_amdgcn_alignbit(raw[j + 1], raw[j], bit & 31);
            }
        };

        // ---- the tables, while the records and values are on their way; the queries rotated, and as operands through LDS ----
        if (!built) {
            lds_barrier();
            build_prefix_tables<P>(sm, tb, tid);
            built = true;
        }
#pragma unroll
        for (int p = 0; p < C::QPASS; ++p) {
            const int local = tid / C::QLANES + p * C::QROWS;
            const bool there = row0 + local < rows;
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t two = asked[p][0][e / 2], own = asked[p][e / 4][e % 4];
                const uint32_t bits = shp.q_is_bf16 ? ((e & 1) ? two & 0xffff0000u : two << 16) : own;
                x[e] = there ? __uint_as_float(bits ^ ((sbits << (31 - e)) & 0x80000000u)) : 0.0f;
            }
#pragma unroll
            for (int m = 1; m < 8; m <<= 1)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if ((e & m) == 0) {
                        const float a = x[e], b = x[e | m];
                        x[e] = a + b;
                        x[e | m] = a - b;
                    }
            static_for<0, C::log2i(C::QLANES)>([&](auto bb) {
                constexpr int m = 1 << decltype(bb)::value;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float other = lane_xor<m>(x[e], lane);
                    x[e] = (lane & m) ? other - x[e] : x[e] + other;
                }
            });
            // The scale's sign and mantissa go into the queries.  What is left of it is a row's factor, a power of two: factor score is exact,
            // so the largest score's probability is 1 whatever its size (a product rounded before the reference is taken from it would
            // leave up to half a step of the score, which is no number's exponent any more from 2^31 on).  Another power of two brings
            // the row's largest number into [1/2, 1): fp16 has no range to spare.
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= shp.scale_part;
            float top = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
            static_for<0, C::log2i(C::QLANES)>([&](auto bb) { top = fmaxf(top, lane_xor<(1 << decltype(bb)::value)>(top, lane)); });
            const int ex = top > 0.0f && top < INFINITY ? __builtin_amdgcn_frexp_expf(top) : 0;
            if (C::ROWS % C::QROWS == 0 || local < C::ROWS) {
                // (neither zero nor infinity: what a row does not see has a score of minus infinity, and stays there, and a score of
                // zero stays one)
                if (qc == 0) sm.factor[local] = ldexpf(1.0f, min(max(ex + shp.scale_exp, -126), 127));
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int c = 8 * qc + e, t = c / 3;
                    const bool second = P::NCLASS == 2 && t >= P::NT0;
                    const int of = second ? t - P::NT0 : t, each = second ? (C::T1 > 0 ? C::T1 : 1) : C::T0;
                    const int at = of % each + (second ? C::T0 : 0);
                    unsigned char *to = staged + local * C::QST + (of / each) * (KS * 16) + (3 * at + c % 3) * 2;
                    const float y = ldexpf(x[e], -ex);
                    const _Float16 hi = static_cast<_Float16>(y), lo = static_cast<_Float16>(y - static_cast<float>(hi));
                    *reinterpret_cast<_Float16 *>(to) = hi;
                    *reinterpret_cast<_Float16 *>(to + 4 * KS * 16) = lo;
                }
            }
        }
        // (not before: writes to LDS wait for what comes to LDS from memory)
        if (!C::VREG && work) load_values(begin + wave, page_of(begin + wave));
        lds_barrier();
        auto walk = [&](auto live_) __attribute__((always_inline)) {
        constexpr int LIVE = decltype(live_)::value;   // blocks of 16 rows with rows
        half8_t qh[LIVE][KS], ql[LIVE][KS];
        float factor[LIVE];
        int limit[LIVE];                   // tokens that the row sees
        int all_see = len;               // tokens that every row sees
#pragma unroll
        for (int rb = 0; rb < LIVE; ++rb) {
            // (places that no coordinate has: those of triplets past a class's last, of coordinates past the last and behind a lane
            // group's triplets; what lies there is left over)
            const unsigned char *from = staged + (rb * 16 + n) * C::QST + g * (KS * 16);
            static_for<0, KS>([&](auto kk_) {
                constexpr int kk = decltype(kk_)::value;
                uint4 h = *reinterpret_cast<const uint4 *>(from + kk * 16), l = *reinterpret_cast<const uint4 *>(from + 4 * KS * 16 + kk * 16);
                auto keep = [&](auto at_, uint32_t &hi, uint32_t &lo) __attribute__((always_inline)) {
                    static_for<0, 2>([&](auto half_) {
                        constexpr int place = decltype(at_)::value + decltype(half_)::value, at = place / 3;
                        constexpr uint32_t others = decltype(half_)::value ? 0xffffu : 0xffff0000u;
                        constexpr bool two = P::NCLASS == 2 && at >= C::T0;
                        constexpr int each = two ? C::T1 : C::T0, count = two ? P::NT1 : P::NT0, within = two ? at - C::T0 : at;
                        constexpr int base = two ? P::NT0 : 0;
                        if constexpr (at >= C::TPL) {
                            hi &= others;
                            lo &= others;
                        } else if constexpr (3 * each + within >= count - 1) {   // (some lane groups have none, or the last)
                            const int t = g * each + within;
                            if (t >= count || place % 3 >= D - 3 * (base + t)) {
                                hi &= others;
                                lo &= others;
                            }
                        }
                    });
                };
                keep(std::integral_constant<int, 8 * kk>{}, h.x, l.x);
                keep(std::integral_constant<int, 8 * kk + 2>{}, h.y, l.y);
                keep(std::integral_constant<int, 8 * kk + 4>{}, h.z, l.z);
                keep(std::integral_constant<int, 8 * kk + 6>{}, h.w, l.w);
                qh[rb][kk] = __builtin_bit_cast(half8_t, h);
                ql[rb][kk] = __builtin_bit_cast(half8_t, l);
            });
            factor[rb] = sm.factor[rb * 16 + n];
            limit[rb] = len;
            const int row = row0 + rb * 16 + n;
            if (CAUSAL && !shared && row < rows) {
                const int nq = q_lens != nullptr ? min(max(q_lens[seq], 0), shp.n_q) : shp.n_q;
                limit[rb] = min(max(len - nq + row / hpk + 1, 0), len);
                all_see = min(max(len - nq + row0 / hpk + 1, 0), len);
            }
        }
        all_see = __builtin_amdgcn_readfirstlane(all_see);
        lds_barrier();                 // the operands have been read: the staging areas are the wavefronts' own now

        // ---- the steps ----
        float m_ref[LIVE], l_run[LIVE];
        f32x4_t oacc[LIVE][CB];
#pragma unroll
        for (int rb = 0; rb < LIVE; ++rb) {
            m_ref[rb] = kNoTokenSeen;
            l_run[rb] = 0.0f;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) oacc[rb][cb] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        }
        // the code words of a step's keys n and 16 + n
        uint32_t wd0[2][SD0::WORDS], wn0[2][SN0::WORDS];
        [[maybe_unused]] uint32_t wd1[2][SD1::WORDS], wn1[2][SN1::WORDS];
        auto read_words = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                quarter(SD0{}, P::DIR0_BIT, DQ0, wd0[kb], kb);
                quarter(SN0{}, P::NRM0_BIT, NQ0, wn0[kb], kb);
                if constexpr (P::NCLASS == 2) {
                    quarter(SD1{}, P::DIR1_BIT, DQ1, wd1[kb], kb);
                    quarter(SN1{}, P::NRM1_BIT, NQ1, wn1[kb], kb);
                }
            }
        };
        // (the next step's are read before the values' products, or, where that spills, behind the last of the channels' reads: 4 bits at
        // head dimension 128, 64 sequences behind 8192 tokens 101 against 98.9 us, causal drafts 87.5 against 83.4; 1.5 bits 71 against 77)
        constexpr bool WORDS_LATE = D == 128 && !C::J0;
        if (work) {
            store_records();
            __builtin_amdgcn_wave_barrier();
            if constexpr (C::VREG) store_values();
            read_words();
#pragma unroll
            for (int e = 0; e < C::NREC; ++e) rec[e] = second[e];
            if constexpr (C::VREG) {
                if (begin + wave + NW < end) load_values(begin + wave + NW, page_of(begin + wave + NW));
            }
        }
        for (int step = begin + wave; step < end; step += NW) {
            const bool more = step + NW < end, two_more = step + 2 * NW < end;
            f32x4_t score[2][LIVE];      // [key block][row block]: lane (n, g) has keys 4 g .. + 3 of row n
            // The remainders' products have sums of their own where registers are left for them: a sum that is already large takes off
            // their last bits (4 beams of 4 rows behind 700 tokens: the output off by 0.62e-6 of its root mean square instead of 0.86e-6,
            // fp32 torch 0.72e-6; at d = 64 two row blocks 0.76e-6 instead of 1.15e-6; 1 % of the time).  With two row blocks at d = 128 they spill
            // (16 sequences behind 65531 tokens: 78 -> 100 us) and the error, 1.3e-6 over a long prefix, is below fp32 torch's 2.1e-6 as it is.
            constexpr bool APART = LIVE == 1 || D == 64;
            f32x4_t rest[2][LIVE];
            float gamma[2][4];
            // An operand of a key block at a time; the entries of the next one (triplets that begin there) are asked for before the
            // products of this one, as LDS takes longer to answer than a product.
            auto entry = [&](auto kb_, auto at_) __attribute__((always_inline)) -> uint4 {
                constexpr int kb = decltype(kb_)::value, at = decltype(at_)::value;
                if constexpr (at < C::T0) {
                    const uint32_t nrm = field_clamped<at * P::BN0, P::BN0>(wn0[kb]);
                    if constexpr (C::J0 && 2 * P::BD0 == 8 && C::R0 * 16 << P::BN0 == 256) {
                        // the code is a whole byte and the entry's offset has it as its second byte, above norm code and copy
                        const uint32_t low = nrm << (4 + C::log2i(C::R0)) | static_cast<uint32_t>(lane & (C::R0 - 1)) << 4;
                        const uint32_t at_byte = __builtin_amdgcn_perm(wd0[kb][at / 4], low, 0x0c0c0400u + ((at % 4) << 8));
                        return *reinterpret_cast<const uint4 *>(reinterpret_cast<const unsigned char *>(tb.tab0) + at_byte);
                    } else if constexpr (C::J0) {
                        constexpr int NS = C::log2i(C::R0);
                        const uint32_t dir = field_clamped<at * 2 * P::BD0, 2 * P::BD0>(wd0[kb]);
                        return tb.tab0[(dir << (NS + P::BN0)) + (nrm << NS) + (lane & (C::R0 - 1))];
                    } else {
                        const uint32_t dir = field_clamped<at * 2 * P::BD0, 2 * P::BD0>(wd0[kb]);
                        uint4 d4 = tb.tab0[dir * C::R0 + (lane & (C::R0 - 1))];
                        d4.w = __float_as_uint(sm.c_rho[0][nrm]);
                        return d4;
                    }
                } else if constexpr (P::NCLASS == 2) {
                    constexpr int a1 = at - C::T0, NS = C::log2i(C::R1);
                    const uint32_t dir = field_clamped<a1 * 2 * P::BD1, 2 * P::BD1>(wd1[kb]), nrm = field_clamped<a1 * P::BN1, P::BN1>(wn1[kb]);
                    return tb.tab1[(dir << (NS + P::BN1)) + (nrm << NS) + (lane & (C::R1 - 1))];
                }
            };
            // (tables without norms: the triplet is put together here)
            auto triplet = [&](uint4 e) __attribute__((always_inline)) -> uint4 {
                if constexpr (C::J0) return e;
                const float rho = __uint_as_float(e.w);
                return half_triplet(rho * __uint_as_float(e.x), rho * __uint_as_float(e.y), rho * __uint_as_float(e.z));
            };
            // (one row block: both key blocks at once, as a product that adds to the last one's result waits for it)
            constexpr int NB = LIVE == 1 ? 2 : 1, NS = 2 * KS / NB;
            uint4 ent[2][C::TPL];            // (unrolled: an entry lives from being asked for to the operand that it ends in)
            auto starts = [](int kk) constexpr { return (8 * kk + 2) / 3 < C::TPL ? (8 * kk + 2) / 3 : C::TPL; };
            auto ask = [&](auto s_) __attribute__((always_inline)) {
                constexpr int s = decltype(s_)::value, kk = s % KS;
                static_for<0, NB>([&](auto b_) {
                    constexpr int kb = decltype(b_)::value + s / KS;
                    static_for<starts(kk), starts(kk + 1)>([&](auto at_) { ent[kb][decltype(at_)::value] = entry(std::integral_constant<int, kb>{}, at_); });
                });
            };
            // halves 2 w and 2 w + 1 of a lane group's coordinates of a key: of the leading parts or of the remainders
            auto word = [&](auto kb_, auto w_, auto low_) __attribute__((always_inline)) -> uint32_t {
                constexpr int kb = decltype(kb_)::value, at = 2 * decltype(w_)::value / 3, c = 2 * decltype(w_)::value % 3;
                constexpr bool low = decltype(low_)::value;
                if constexpr (at >= C::TPL) {
                    return 0u;
                } else {
                    const uint32_t xy = low ? ent[kb][at].z : ent[kb][at].x, z = low ? ent[kb][at].w : ent[kb][at].y;
                    if constexpr (c == 0) return xy;
                    else if constexpr (c == 1) return __builtin_amdgcn_alignbit(z, xy, 16);
                    else if constexpr (at + 1 >= C::TPL) return z;
                    else return __builtin_amdgcn_perm(low ? ent[kb][at + 1].z : ent[kb][at + 1].x, z, 0x05040100u);
                }
            };
            ask(std::integral_constant<int, 0>{});
            static_for<0, NS>([&](auto s_) {
                constexpr int s = decltype(s_)::value, kk = s % KS;
                if constexpr (s + 1 < NS) {
                    ask(std::integral_constant<int, s + 1>{});
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) gamma[e / 4][e % 4] = *reinterpret_cast<const float *>(stage + ((e / 4) * 16 + 4 * g + e % 4) * C::RST);
                }
                __builtin_amdgcn_sched_barrier(0);
                half8_t kh[NB], kl[NB];
                static_for<0, NB>([&](auto b_) {
                    constexpr int b = decltype(b_)::value, kb = b + s / KS;
                    static_for<starts(kk), starts(kk + 1)>([&](auto at_) { ent[kb][decltype(at_)::value] = triplet(ent[kb][decltype(at_)::value]); });
                    auto four = [&](auto low_) __attribute__((always_inline)) {
                        using K = std::integral_constant<int, kb>;
                        return make_uint4(word(K{}, std::integral_constant<int, 4 * kk>{}, low_), word(K{}, std::integral_constant<int, 4 * kk + 1>{}, low_),
                                          word(K{}, std::integral_constant<int, 4 * kk + 2>{}, low_), word(K{}, std::integral_constant<int, 4 * kk + 3>{}, low_));
                    };
                    kh[b] = __builtin_bit_cast(half8_t, four(std::false_type{}));
                    kl[b] = __builtin_bit_cast(half8_t, four(std::true_type{}));
                });
                // (each of these loops has products that do not wait for each other)
                constexpr int first = s / KS;
                const f32x4_t zero = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int e = 0; e < NB * LIVE; ++e)
                    score[first + e / LIVE][e % LIVE] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh[e / LIVE], qh[e % LIVE][kk], kk == 0 ? zero : score[first + e / LIVE][e % LIVE], 0, 0, 0);
#pragma unroll
                for (int e = 0; e < NB * LIVE; ++e) {
                    f32x4_t &to = APART ? rest[first + e / LIVE][e % LIVE] : score[first + e / LIVE][e % LIVE];
                    to = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh[e / LIVE], ql[e % LIVE][kk], APART && kk == 0 ? zero : to, 0, 0, 0);
                }
#pragma unroll
                for (int e = 0; e < NB * LIVE; ++e) {
                    f32x4_t &to = APART ? rest[first + e / LIVE][e % LIVE] : score[first + e / LIVE][e % LIVE];
                    to = __builtin_amdgcn_mfma_f32_16x16x32_f16(kl[e / LIVE], qh[e % LIVE][kk], to, 0, 0, 0);
                }
            });
#pragma unroll
            for (int rb = 0; rb < LIVE; ++rb)
#pragma unroll
                for (int e = 0; e < 8; ++e) score[e / 4][rb][e % 4] = (APART ? score[e / 4][rb][e % 4] + rest[e / 4][rb][e % 4] : score[e / 4][rb][e % 4]) * gamma[e / 4][e % 4];
            // tokens past the sequence's end, or that a row does not see for causality
            if ((step + 1) * kPrefixKeys > all_see) {
#pragma unroll
                for (int rb = 0; rb < LIVE; ++rb)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (step * kPrefixKeys + (e / 4) * 16 + 4 * g + e % 4 >= limit[rb]) score[e / 4][rb][e % 4] = -INFINITY;
            }
            // probabilities are 2^(factor score - m_ref); a row's reference moves when a score exceeds it by more than 8
            float top[LIVE];
            bool higher = false;
#pragma unroll
            for (int rb = 0; rb < LIVE; ++rb) {
                top[rb] = score[0][rb][0];
#pragma unroll
                for (int e = 1; e < 8; ++e) top[rb] = fmaxf(top[rb], score[e / 4][rb][e % 4]);
                top[rb] *= factor[rb];
                higher = higher || top[rb] > m_ref[rb] + 8.0f;
            }
            if (__ballot(higher) != 0) {
#pragma unroll
                for (int rb = 0; rb < LIVE; ++rb) {
                    top[rb] = fmaxf(top[rb], lane_xor<16>(top[rb], lane));
                    top[rb] = fmaxf(top[rb], lane_xor<32>(top[rb], lane));
                    const float m_new = fmaxf(m_ref[rb], top[rb]);
                    const float alpha = exp2_raw(m_ref[rb] - m_new);
                    m_ref[rb] = m_new;
                    l_run[rb] *= alpha;
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb) oacc[rb][cb] *= alpha;
                }
            }
            prefix_bf16x8_t p_hi[LIVE], p_mid[LIVE], p_lo[LIVE];
#pragma unroll
            for (int rb = 0; rb < LIVE; ++rb) {
                uint32_t ph[4], pm[4], pl[4];
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float p0 = exp2_raw(fmaf(score[e / 4][rb][e % 4], factor[rb], -m_ref[rb]));
                    const float p1 = exp2_raw(fmaf(score[e / 4][rb][e % 4 + 1], factor[rb], -m_ref[rb]));
                    l_run[rb] += p0 + p1;
                    // Three bf16 numbers of eight bits each, whose sum is p to its last bit; the values are bf16.  (Two, rounded to the
                    // nearest, are off by up to 2^-17, and the output by 1.6e-6 to 2.0e-6 of its root mean square, fp32 torch by 0.6e-6 to
                    // 2.9e-6; three make it 0.3e-6 to 0.5e-6 and cost 1 to 10 %: 64 sequences behind 8192 tokens
                    // 71 -> 74.5 us, 16 behind 65531 72 -> 78, 32 at d = 256 behind 16384 70 -> 71.5.)
                    ph[e / 2] = bf16_cut_pair(p0, p1);
                    const float r0 = p0 - bf16_cut(p0), r1 = p1 - bf16_cut(p1);
                    pm[e / 2] = bf16_cut_pair(r0, r1);
                    pl[e / 2] = bf16_cut_pair(r0 - bf16_cut(r0), r1 - bf16_cut(r1));
                }
                p_hi[rb] = __builtin_bit_cast(prefix_bf16x8_t, make_uint4(ph[0], ph[1], ph[2], ph[3]));
                p_mid[rb] = __builtin_bit_cast(prefix_bf16x8_t, make_uint4(pm[0], pm[1], pm[2], pm[3]));
                p_lo[rb] = __builtin_bit_cast(prefix_bf16x8_t, make_uint4(pl[0], pl[1], pl[2], pl[3]));
            }
            // nothing reads this step's records any more: the next step's take their place
            if (more) {
                __builtin_amdgcn_wave_barrier();
                store_records();
                __builtin_amdgcn_wave_barrier();
                if (!WORDS_LATE) read_words();
            }
            // The values have arrived. Rows past the last token are made zeros: their probabilities are zero, but what lies there may
            // be no number.
            if constexpr (!C::VREG) wait_loads<0>();
            const int last = len - 1 - step * kPrefixKeys;
            if (last < kPrefixKeys - 1) {
#pragma unroll
                for (int e = 0; e < C::NVAL; ++e)
                    if ((lane / LPR) * C::NVAL + e > last)
                        *reinterpret_cast<uint4 *>(vals + e * C::VST + lane * 16) = make_uint4(0u, 0u, 0u, 0u);
                __builtin_amdgcn_wave_barrier();
            }
            // A value that is no finite number makes its channel NaN for the rows that see its token, and a zero for the others: what
            // they do not see would reach them through the product otherwise.
            if (CAUSAL && min((step + 1) * kPrefixKeys, len) > all_see) {
                auto none = [](uint32_t two, int j) { return (two >> (16 * j) & 0x7f80u) == 0x7f80u; };
                uint32_t odd = 0;                // keys that have such a value
#pragma unroll
                for (int e = 0; e < C::NVAL; ++e) {
                    const uint4 piece = *reinterpret_cast<const uint4 *>(vals + e * C::VST + lane * 16);
                    const uint32_t two[4] = {piece.x, piece.y, piece.z, piece.w};
                    bool any = false;
#pragma unroll
                    for (int j = 0; j < 8; ++j) any = any || none(two[j / 2], j % 2);
                    const uint64_t lanes = __ballot(any);
#pragma unroll
                    for (int part = 0; part < kWave / LPR; ++part)
                        if ((lanes >> (part * LPR) & ((1ull << (LPR - 1)) * 2 - 1)) != 0) odd |= 1u << (part * C::NVAL + e);
                }
                if (odd != 0) {
                    for (uint32_t left = odd; left != 0; left &= left - 1) {
                        const int key = __ffs(static_cast<int>(left)) - 1;
                        const unsigned char *row = vals + (key % C::NVAL) * C::VST + (key / C::NVAL) * (2 * D) + 8 * g;
#pragma unroll
                        for (int cb = 0; cb < CB; ++cb) {
                            const uint2 four = *reinterpret_cast<const uint2 *>(row + 32 * cb);
#pragma unroll
                            for (int rb = 0; rb < LIVE; ++rb)
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    if (none(j < 2 ? four.x : four.y, j % 2) && step * kPrefixKeys + key < limit[rb]) oacc[rb][cb][j] = NAN;
                        }
                    }
                    __builtin_amdgcn_wave_barrier();
                    for (int e = 0; e < C::NVAL; ++e) {
                        uint16_t *piece = reinterpret_cast<uint16_t *>(vals + e * C::VST + lane * 16);
                        for (int j = 0; j < 8; ++j)
                            if (none(piece[j], 0)) piece[j] = 0;
                    }
                    __builtin_amdgcn_wave_barrier();
                }
            }
            // O^T += V^T P^T: k-slots 8 g .. + 3 are keys 4 g .. + 3 of the first block, the next four those of the second
            constexpr int AHEAD_V = 3;                   // (channels of this and the next two products are held)
            typedef __attribute__((address_space(3))) s16x4_t *tr_t;
            const int row = 4 * g + n / 4;               // of the four that a lane group reads transposed, 16 channels of each
            unsigned char *vat = vals + (row % C::NVAL) * C::VST + (row / C::NVAL) * (2 * D) + (n % 4) * 8;
            constexpr int SECOND = (16 / C::NVAL) * (2 * D);   // 16 rows on
            static_assert(16 % C::NVAL == 0, "16 rows on is a whole number of pieces on");
            union channels_t { s16x4_t h[2]; prefix_bf16x8_t b; } v[AHEAD_V];
            auto ask_values = [&](int cb) __attribute__((always_inline)) {
                v[cb % AHEAD_V].h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)(vat + 32 * cb));
                v[cb % AHEAD_V].h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)(vat + 32 * cb + SECOND));
            };
#pragma unroll
            for (int cb = 0; cb < AHEAD_V - 1; ++cb) ask_values(cb);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                if (cb + AHEAD_V - 1 < CB) ask_values(cb + AHEAD_V - 1);
                if (WORDS_LATE && cb + AHEAD_V - 1 == CB && more) read_words();
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int rb = 0; rb < LIVE; ++rb) oacc[rb][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[cb % AHEAD_V].b, p_hi[rb], oacc[rb][cb], 0, 0, 0);
#pragma unroll
                for (int rb = 0; rb < LIVE; ++rb) oacc[rb][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[cb % AHEAD_V].b, p_mid[rb], oacc[rb][cb], 0, 0, 0);
#pragma unroll
                for (int rb = 0; rb < LIVE; ++rb) oacc[rb][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[cb % AHEAD_V].b, p_lo[rb], oacc[rb][cb], 0, 0, 0);
            }
            wait_lds();                  // (the reads are done before anything new is asked for in their place)
            if (more) {
                if constexpr (C::VREG) {
                    __builtin_amdgcn_wave_barrier();
                    store_values();
                    __builtin_amdgcn_wave_barrier();
                }
                // (the records first: they are waited for first, and a wait for them is not one for the values)
                if (two_more) {
                    if (step + 2 * NW - held_from >= 64 * NW) hold_pages(step + NW);
                    load_records(rec, step + 2 * NW, page_of(step + 2 * NW));
                    if constexpr (C::VREG) load_values(step + 2 * NW, page_of(step + 2 * NW));
                }
                if constexpr (!C::VREG) load_values(step + NW, page_of(step + NW));
            }
        }

        // ---- the wavefronts' results join ----
#pragma unroll
        for (int rb = 0; rb < LIVE; ++rb) {
            l_run[rb] += lane_xor<16>(l_run[rb], lane);
            l_run[rb] += lane_xor<32>(l_run[rb], lane);
            if (g == 0) {
                sm.ml[wave][rb * 16 + n][0] = m_ref[rb];
                sm.ml[wave][rb * 16 + n][1] = l_run[rb];
            }
        }
        lds_barrier();                 // (the staging areas are free from here on, too)
        float *out = reinterpret_cast<float *>(place);   // [wavefront][16 rows][OST]
        const int64_t prow0 = shared ? static_cast<int64_t>(kvh) * all_rows * splits
                                     : shp.own_partials + (static_cast<int64_t>(seq) * shp.n_kv_heads + kvh) * own_rows * splits;
#pragma unroll
        for (int rb = 0; rb < LIVE; ++rb) {
            float m_all = kNoTokenSeen;
#pragma unroll
            for (int w = 0; w < NW; ++w) m_all = fmaxf(m_all, sm.ml[w][rb * 16 + n][0]);
            const float weight = exp2_raw(m_ref[rb] - m_all);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                *reinterpret_cast<f32x4_t *>(out + (wave * 16 + n) * C::OST + 16 * cb + 4 * g) = oacc[rb][cb] * weight;
            lds_barrier();
            for (int e = tid; e < 16 * D / 4; e += C::NT) {
                const int r = e / (D / 4), row = row0 + rb * 16 + r;
                if (row >= rows) continue;
                f32x4_t sum = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int w = 0; w < NW; ++w) sum += *reinterpret_cast<const f32x4_t *>(out + (w * 16 + r) * C::OST + (e % (D / 4)) * 4);
                const int64_t prow = prow0 + static_cast<int64_t>(row) * splits + split;
                *reinterpret_cast<f32x4_t *>(part_acc + prow * D + (e % (D / 4)) * 4) = sum;
                if (e % (D / 4) == 0) {
                    float m = kNoTokenSeen, l = 0.0f;
#pragma unroll
                    for (int w = 0; w < NW; ++w) m = fmaxf(m, sm.ml[w][rb * 16 + r][0]);
#pragma unroll
                    for (int w = 0; w < NW; ++w) l += sm.ml[w][rb * 16 + r][1] * exp2_raw(sm.ml[w][rb * 16 + r][0] - m);
                    part_ml[prow * 2] = m;
                    part_ml[prow * 2 + 1] = l;
                }
            }
            lds_barrier();
        }
        };
        static_assert(RB <= 2, "a walk for each count of blocks with rows");
        if (RB == 1 || live == 1) walk(std::integral_constant<int, 1>{});
        else walk(std::integral_constant<int, RB>{});
    }
}

template <class P>
int launch_prefix_plan(const octopus_codebooks_t &cb, const PrefixShape &s, const void *k_pool, const void *v_pool, const int32_t *prefix_table,
                       const int32_t *prefix_len, const int32_t *block_table, const int32_t *seq_lens, const int32_t *q_lens, float *part_ml,
                       float *part_acc, hipStream_t stream) {
    const DeviceBooks books = device_books(cb);
    const int grid = s.n_segments < 256 ? s.n_segments : 256;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(PrefixCfg<P>::NT), 0, stream, books, s, static_cast<const unsigned char *>(k_pool),
                           static_cast<const unsigned char *>(v_pool), prefix_table, prefix_len, block_table, seq_lens, q_lens, part_ml, part_acc);
    };
    if (s.causal) go(prefix_attention_kernel<P, true>);
    else go(prefix_attention_kernel<P, false>);
    return static_cast<int>(hipGetLastError());
}

}  // namespace octopus

#endif

// A step's new tokens into pages, as the projection leaves them: keys and queries rotated by position, keys encoded into their
// pages (Alg. 1), values written into theirs as bf16 or quantised.
//
// The rotation turns pairs of channels (a, b) of a row at position p by the caller's (cos, sin) of that position:
//     a' = a cos - b sin,   b' = a sin + b cos,
// pairs being channels i and i + dim / 2, or 2 i and 2 i + 1, i < dim / 2; channels from dim on stay.  It is applied in fp32 to the
// key that the encoder takes: what octopus_encode_paged computes of rotated keys, without their rounding to bf16 in between.
// A token of an image or a video has a position on each of several axes (frame, row, column), and pair i goes by the one that the
// caller's map gives it: (cos, sin) = table[p_axis(i)][i].  Those kernels (append_*_axes_kernel) differ in nothing else.  A pair's entry is
// read by itself there, whatever the map, twice as many reads as of one position's row: 15840 patches take 104 to 111 us where tokens in a row
// take 96 (94 if the reads were as wide and no positions had to be read), 64 single tokens 7.8 instead of 7.4.  Wide reads for maps that allow
// them, beside these by a branch, cost more than they saved (113 in place of 111), by threads too (114).
//
// What bounds it: memory, for long prompts -- queries, keys and values come and go once, the records are a quarter of the keys -- and
// latency for a few tokens.  Measured at d = 128, 3 bits, 32 query and 8 KV heads, bf16: 15877 tokens, 366 MB, in 97 us, 3.8 TB/s
// where a copy reaches 5.0; a token of each of 64 sequences, 0.7 MB, in 6.6 us, all latency.
#ifndef OCTOPUS_APPEND_HPP_
#define OCTOPUS_APPEND_HPP_

#include "octopus_encode.hpp"

namespace octopus {

// Eight channels of a row, fp32.
__device__ __forceinline__ void load_eight(const void *base, int64_t at, int is_bf16, float (&x)[8]) {
    if (is_bf16) {
        const uint4 r = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(base) + at);
        x[0] = bf16_lo(r.x); x[1] = bf16_hi(r.x); x[2] = bf16_lo(r.y); x[3] = bf16_hi(r.y);
        x[4] = bf16_lo(r.z); x[5] = bf16_hi(r.z); x[6] = bf16_lo(r.w); x[7] = bf16_hi(r.w);
    } else {
        const float4 a = *reinterpret_cast<const float4 *>(static_cast<const float *>(base) + at);
        const float4 b = *reinterpret_cast<const float4 *>(static_cast<const float *>(base) + at + 4);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
}
// ... stored: bf16 rounded to the nearest.
__device__ __forceinline__ void store_eight(void *base, int64_t at, int is_bf16, const float (&x)[8]) {
    if (is_bf16) {
        typedef float f32x8_t __attribute__((ext_vector_type(8)));
        typedef __bf16 bf16x8v_t __attribute__((ext_vector_type(8)));
        const f32x8_t v = {x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
        *reinterpret_cast<bf16x8v_t *>(static_cast<uint16_t *>(base) + at) = __builtin_convertvector(v, bf16x8v_t);
    } else {
        float4 *p = reinterpret_cast<float4 *>(static_cast<float *>(base) + at);
        p[0] = make_float4(x[0], x[1], x[2], x[3]);
        p[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
}

// The table's rows of a token's positions on its axes, in bytes from its start.  (Four numbers, and handed on by value: the compiler
// puts into LDS what elements are chosen from by address, and reads the dispatch packet, in host memory, to find it there: 12 us.)
struct AxisRows {
    uint32_t r0, r1, r2, r3;
};
static_assert(kMaxAxes == 4, "");

// A thread's eight channels' (cos, sin) of a position, and the rotation of its share of a row.  Rows lie LPR lanes side by side, so
// that a channel's partner half a rotation away is half a rotation / 8 lanes away.
template <int LPR>
struct RowRotation {
    float2 cs[8];
    int half;         // dim / 2; 0: nothing of this thread is rotated
    bool pairs;       // channels 2 i and 2 i + 1
    bool upper;       // this thread has the second channels of its pairs
    __device__ __forceinline__ void load(const RopeCall &r, int64_t pos, int col) {
        half = r.table != nullptr && col < r.dim ? r.dim / 2 : 0;
        pairs = r.interleaved != 0;
        upper = col >= half;
        if (half == 0) return;
        pos = min(max(pos, static_cast<int64_t>(0)), r.n_pos - 1);
        const float2 *row = reinterpret_cast<const float2 *>(r.table) + pos * half;
        const int first = pairs ? col / 2 : (upper ? col - half : col);
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            if (j >= 4 && pairs) break;
            const float4 two = *reinterpret_cast<const float4 *>(row + first + j);
            cs[j] = make_float2(two.x, two.y);
            cs[j + 1] = make_float2(two.z, two.w);
        }
    }
    // The first of a thread's pairs, and the axes of its eight (two bits each).
    __device__ __forceinline__ static int first_pair(const RopeCall &r, int col) {
        return r.interleaved != 0 ? col / 2 : (col >= r.dim / 2 ? col - r.dim / 2 : col);
    }
    __device__ __forceinline__ static uint32_t axes_of(const RopeCall &r, const AxesCall &x, int col) {
        const int first = first_pair(r, col);
        uint32_t axes = x.axis_of[0];            // 16 pairs a word
#pragma unroll
        for (int w = 1; w < LPR / 4; ++w) axes = first / 16 == w ? x.axis_of[w] : axes;
        return axes >> (2 * (first % 16));
    }
    // ... of a token's positions on several axes, of which the table's rows are
    __device__ __forceinline__ void load(const RopeCall &r, uint32_t axes, AxisRows rows, int col) {
        half = col < r.dim ? r.dim / 2 : 0;
        pairs = r.interleaved != 0;
        upper = col >= half;
        if (half == 0) return;
        const int first = first_pair(r, col);
        const uint32_t r0 = rows.r0 + 8 * first, r1 = rows.r1 + 8 * first, r2 = rows.r2 + 8 * first, r3 = rows.r3 + 8 * first;
        auto bit = [axes](int i) { return static_cast<uint32_t>(static_cast<int32_t>(axes << (31 - i)) >> 31); };      // all ones or none
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (j >= 4 && pairs) break;
            const uint32_t odd = bit(2 * j), upper_two = bit(2 * j + 1);      // (selected bit by bit, see AxisRows)
            const uint32_t lo = (r1 & odd) | (r0 & ~odd), hi = (r3 & odd) | (r2 & ~odd), at = (hi & upper_two) | (lo & ~upper_two);
            cs[j] = *reinterpret_cast<const float2 *>(reinterpret_cast<const char *>(r.table) + at + 8 * j);
        }
    }
    // (all lanes of a row call this: the partners' channels come from other lanes.  One rounding order, whatever the caller: a key has
    // the same codes in a prompt and by itself)
    __device__ __forceinline__ void apply(float (&x)[8], int lane) const {
        if (pairs) {
            if (half == 0) return;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float a = x[2 * j], b = x[2 * j + 1];
                x[2 * j] = fmaf(a, cs[j].x, -__fmul_rn(b, cs[j].y));
                x[2 * j + 1] = fmaf(a, cs[j].y, __fmul_rn(b, cs[j].x));
            }
            return;
        }
        const int from = half == 0 ? lane : (upper ? lane - half / 8 : lane + half / 8);
        float other[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) other[j] = __shfl(x[j], from, kWave);
        if (half == 0) return;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            x[j] = upper ? fmaf(other[j], cs[j].y, __fmul_rn(x[j], cs[j].x)) : fmaf(x[j], cs[j].x, -__fmul_rn(other[j], cs[j].y));
    }
};

__device__ __forceinline__ int64_t append_start(const AppendCall &a, int seq) { return a.start_pos ? max(a.start_pos[seq], 0) : 0; }
__device__ __forceinline__ int append_count(const AppendCall &a, int seq) {
    return a.new_lens ? min(max(a.new_lens[seq], 0), a.n_new) : a.n_new;
}
__device__ __forceinline__ int64_t append_position(const AppendCall &a, int seq, int64_t start) {
    return a.rope.pos ? static_cast<int64_t>(a.rope.pos[seq]) : start;
}
__device__ __forceinline__ int64_t append_page(const AppendCall &a, int seq, int64_t tile) {
    return min(max(a.pt.table[static_cast<int64_t>(seq) * a.pt.stride + tile], 0), a.pt.n_pages - 1);
}

// Where a token's rotation comes from: one position, or one on each axis.  `at` reads the positions of a slot, `load` the (cos, sin) there:
// what else a caller reads goes in between, since the one waits for the other.
struct OneAxis {
    static constexpr bool LATE = false;     // nothing is waited for
    struct Sequence {
        using Place = int64_t;
        int64_t pos0;      // the position of slot 0, if it were there
        __device__ __forceinline__ Place at(const AppendCall &, int64_t slot) const { return pos0 + slot; }
        template <int LPR>
        __device__ __forceinline__ void load(RowRotation<LPR> &rot, const AppendCall &a, const Place &place, int col) const { rot.load(a.rope, place, col); }
    };
    template <int LPR>
    __device__ __forceinline__ Sequence of(const AppendCall &a, int seq, int64_t start, int) const { return {append_position(a, seq, start) - start}; }
};
struct ManyAxes {
    static constexpr bool LATE = true;
    AxesCall x;
    struct Sequence {
        using Place = AxisRows;
        const AxesCall &x;
        const int32_t *pos;
        int64_t start;
        int last;          // token that has positions
        uint32_t axes;     // of the thread's pairs
        __device__ __forceinline__ Place at(const AppendCall &a, int64_t slot) const {
            // (a tile's slots in front of the first token and behind the last one ask as well, and get the nearest token's; an axis past the last
            // reads the first one's position: four reads that wait for nothing but each other are one wait)
            const uint32_t tok = min(max(static_cast<int32_t>(slot - start), 0), last);
            const int32_t *p = pos + static_cast<uint64_t>(tok) * static_cast<uint32_t>(x.stride_tok);
            const int32_t p0 = p[0], p1 = p[x.axis_at[0]], p2 = p[x.axis_at[1]], p3 = p[x.axis_at[2]];
            auto row = [&](int32_t at) { return static_cast<uint32_t>(__umul24(min(max(at, 0), x.last_pos), 4 * a.rope.dim)); };
            return Place{row(p0), row(p1), row(p2), row(p3)};
        }
        template <int LPR>
        __device__ __forceinline__ void load(RowRotation<LPR> &rot, const AppendCall &a, Place place, int col) const { rot.load(a.rope, axes, place, col); }
    };
    template <int LPR>
    __device__ __forceinline__ Sequence of(const AppendCall &a, int seq, int64_t start, int col) const {
        uint32_t axes = RowRotation<LPR>::axes_of(a.rope, x, col);
        asm("" : "+v"(axes));      // (kept, and not read again for every token)
        return {x, x.pos + seq * x.stride_seq, start, append_count(a, seq) - 1, axes};
    }
};

// Few tokens (a decode step appends one per sequence): a wavefront per (token, KV head), which takes the key, the value and the
// head's queries as rows side by side, eight channels a lane, and encodes the key a triplet per lane.
// (the call by value: by reference the compiler copies loads of the rows' loop, 236 bytes and two registers more at d = 128, and a single
// token takes 5.36 us instead of 5.22)
template <class P, class Turn>
__device__ __forceinline__ void append_token(const AppendCall a, const Turn &turn) {
    constexpr int D = P::D, LPR = D / 8, ROWS = kWave / LPR;
    constexpr int NX = P::BD0 > 2 || P::BD1 > 2 ? 1 << (P::BD0 > P::BD1 ? P::BD0 : P::BD1) : 4;
    constexpr int NR = 1 << (P::BN0 > P::BN1 ? P::BN0 : P::BN1);
    __shared__ __attribute__((aligned(16))) float u[3 * P::NTRI + 16];
    __shared__ __attribute__((aligned(16))) uint32_t rec[P::NWORDS + 4];
    __shared__ float c_xi[P::NCLASS][NX], c_rho[P::NCLASS][NR];
    const int lane = threadIdx.x, col = (lane % LPR) * 8;
    const int kvh = blockIdx.y, seq = blockIdx.z, tok = blockIdx.x;
    if (tok >= append_count(a, seq)) return;
    const int64_t start = append_start(a, seq), slot = start + tok;
    // (a token past what the table reaches is written nowhere; its queries are rotated all the same)
    const bool reached = slot < static_cast<int64_t>(a.pt.stride) * kWave;
    const int64_t tile = reached ? (append_page(a, seq, slot / kWave) * a.n_kv_heads + kvh) : 0;
    const auto turns = turn.template of<LPR>(a, seq, start, col);
    const auto place = turns.at(a, slot);
    RowRotation<LPR> rot;
    if constexpr (!Turn::LATE) turns.load(rot, a, place, col);

    const int hpk = a.q != nullptr ? a.n_q_heads / a.n_kv_heads : 0;
    float key[8];
    for (int r0 = 0; r0 < 2 + hpk; r0 += ROWS) {
        const int row = r0 + lane / LPR;     // 0: the key, 1: the value, then the queries
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.0f;
        const int64_t qrow = (static_cast<int64_t>(seq) * a.n_new + tok) * a.n_q_heads + kvh * hpk + row - 2;
        if (row == 0) load_eight(a.k, seq * a.k_seq + tok * a.k_tok + kvh * a.k_head + col, a.kv_is_bf16, x);
        else if (row == 1 && a.v_pool != nullptr) load_eight(a.v, seq * a.v_seq + tok * a.v_tok + kvh * a.v_head + col, a.kv_is_bf16, x);
        else if (row > 1 && row < 2 + hpk) load_eight(a.q, seq * a.q_seq + tok * a.q_tok + (kvh * hpk + row - 2) * a.q_head + col, a.q_is_bf16, x);
        if constexpr (Turn::LATE)
            if (r0 == 0) turns.load(rot, a, place, col);
        if (row == 1 && a.v_pool != nullptr && reached) store_eight(a.v_pool, (tile * kWave + slot % kWave) * D + col, 1, x);
        rot.apply(x, lane);
        if (row > 1 && row < 2 + hpk) store_eight(a.q_out, qrow * D + col, a.q_out_is_bf16, x);
        if (r0 == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) key[e] = lane < LPR ? x[e] : 0.0f;
        }
    }
    if (!reached) return;

#pragma unroll
    for (int c = 0; c < P::NCLASS; ++c) {   // (levels by lane; the arguments hold kMaxLevels of each)
        typedef const float __attribute__((address_space(4))) *arg_t;
        arg_t arg = (arg_t)__builtin_amdgcn_kernarg_segment_ptr();
        const float xi = arg[offsetof(DeviceBooks, c_xi) / 4 + c * kMaxLevels + lane], rho = arg[offsetof(DeviceBooks, c_rho) / 4 + c * kMaxLevels + lane];
        if (lane < NX) c_xi[c][lane] = xi;
        if (lane < NR) c_rho[c][lane] = rho;
    }
    if (lane < P::NWORDS) rec[lane] = 0u;
    const uint32_t sbits = lane < LPR ? a.signs[kvh * LPR + lane] : 0u;

    // E1-E3: norm, sign flip, transform (eight coordinates per lane, then lane by lane)
    float ss = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(key[e], key[e], ss);
    ss = row_sum<LPR>(ss);
    const float gamma = sqrtf(__int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(ss))));
    const float norm = (1.0f / fmaxf(gamma, kEps)) * inv_sqrt_dim<D>();
#pragma unroll
    for (int e = 0; e < 8; ++e) key[e] = ((sbits >> e) & 1u) ? -key[e] : key[e];
    butterflies<8>(key);
    static_for<0, (D == 64 ? 3 : (D == 128 ? 4 : 5))>([&](auto bb) {
        constexpr int m = 1 << decltype(bb)::value;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float other = lane_xor<m>(key[e], lane);
            key[e] = (lane & m) ? other - key[e] : key[e] + other;
        }
    });
    if (lane < LPR) {
#pragma unroll
        for (int e = 0; e < 8; ++e) u[lane * 8 + e] = key[e];
    }
    __syncthreads();

    // E4-E8: a triplet per lane
    for (int i = lane; i < P::NTRI; i += kWave) {
        float x = u[3 * i] * norm, y = 3 * i + 1 < D ? u[3 * i + 1] * norm : 0.0f, z = 3 * i + 2 < D ? u[3 * i + 2] * norm : 0.0f;
        asm("" : "+v"(x), "+v"(y), "+v"(z));   // (the rounded products: none is to be fused into a later sum)
        uint32_t dir, nrm;
        int dir_bit, nrm_bit, dir_bits, nrm_bits;
        if (P::NCLASS == 1 || i < P::NT0) {
            encode_triplet_alone<P::BD0, P::BN0>(x, y, z, 3 * i + 1 >= D, c_xi[0], c_rho[0], &dir, &nrm);
            dir_bits = 2 * P::BD0;
            nrm_bits = P::BN0;
            dir_bit = P::DIR0_BIT + i * dir_bits;
            nrm_bit = P::NRM0_BIT + i * nrm_bits;
        } else {
            constexpr int BD1 = P::BD1 > 0 ? P::BD1 : 1, BN1 = P::BN1 > 0 ? P::BN1 : 1;
            encode_triplet_alone<BD1, BN1>(x, y, z, 3 * i + 1 >= D, c_xi[P::NCLASS - 1], c_rho[P::NCLASS - 1], &dir, &nrm);
            dir_bits = 2 * BD1;
            nrm_bits = BN1;
            dir_bit = P::DIR1_BIT + (i - P::NT0) * dir_bits;
            nrm_bit = P::NRM1_BIT + (i - P::NT0) * nrm_bits;
        }
        atomicOr(&rec[dir_bit >> 5], dir << (dir_bit & 31));
        if ((dir_bit & 31) + dir_bits > 32) atomicOr(&rec[(dir_bit >> 5) + 1], dir >> (32 - (dir_bit & 31)));
        atomicOr(&rec[nrm_bit >> 5], nrm << (nrm_bit & 31));
        if ((nrm_bit & 31) + nrm_bits > 32) atomicOr(&rec[(nrm_bit >> 5) + 1], nrm >> (32 - (nrm_bit & 31)));
    }
    if (lane == 0) rec[0] = __float_as_uint(gamma);   // (no field reaches into word 0)
    __syncthreads();
    if (lane < P::GRANULES)
        *(static_cast<uint4 *>(a.k_pool) + tile * (P::GRANULES * kWave) + lane * kWave + slot % kWave) =
            make_uint4(rec[4 * lane], rec[4 * lane + 1], rec[4 * lane + 2], rec[4 * lane + 3]);
}

template <class P>
__global__ __launch_bounds__(kWave) void append_token_kernel(DeviceBooks books, AppendCall a) { append_token<P>(a, OneAxis{}); }
template <class P>
__global__ __launch_bounds__(kWave) void append_token_axes_kernel(DeviceBooks books, AppendCall a, ManyAxes turn) { append_token<P>(a, turn); }

// Prompts.  Some workgroups encode: a run of 64-token tiles of one (sequence, KV head), eight coordinates a thread while the keys are
// loaded and rotated, a key per lane from the transform on (the phases of encode_kernel, with four candidates per triplet).  The
// others take rows that are not encoded, queries and bf16 values, eight channels a thread and the rows of its token one after the
// other, so that the position's (cos, sin) are read once.  The two kinds alternate: one is bound by the vector units, the
// other by memory.
constexpr int kAppendRows = 8;       // rows of a token per workgroup of the second kind
constexpr int kAhead = 4;            // of them asked for at once

template <class P, class Turn>
__device__ __forceinline__ void append_tile(const AppendCall &a, const Turn &turn, int32_t key_blocks, int32_t tile_runs, int32_t tiles_per_group,
                                            int32_t every) {
    constexpr int D = P::D, LPR = D / 8;
    constexpr int NWV = encode_waves<P>(), NT = encode_threads<P>(), RPP = NT / LPR, NPASS = kWave / RPP;
    using Smem = EncodeSmem<P, false, true>;
    constexpr int REP = Smem::REP;
    __shared__ Smem sm;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = (tid % LPR) * 8;
    const int id = blockIdx.x, before = min(key_blocks, (id + every - 1) / every);   // workgroups of the first kind before this one

    if (id % every != 0 || id / every >= key_blocks) {
        // ---- rows that are not encoded ----
        const int values = a.v_pool != nullptr ? a.n_kv_heads : 0, rows = values + (a.q != nullptr ? a.n_q_heads : 0);
        const int chunks = (rows + kAppendRows - 1) / kAppendRows;
        int i = id - before;
        const int chunk = i % chunks;
        i /= chunks;
        const int runs = (a.n_new + RPP - 1) / RPP;
        const int tok = (i % runs) * RPP + tid / LPR, seq = i / runs;
        if (tok >= append_count(a, seq)) return;     // (whole rows of LPR lanes)
        const int64_t start = append_start(a, seq), slot = start + tok;
        const int first = chunk * kAppendRows, last = min(first + kAppendRows, rows);
        if (first < values && slot < static_cast<int64_t>(a.pt.stride) * kWave) {
            const int64_t page = append_page(a, seq, slot / kWave);
            for (int h0 = first; h0 < min(last, values); h0 += kAhead) {
                float x[kAhead][8];
#pragma unroll
                for (int j = 0; j < kAhead; ++j)     // (rows past the last: the last again)
                    load_eight(a.v, seq * a.v_seq + tok * a.v_tok + min(h0 + j, min(last, values) - 1) * a.v_head + col, a.kv_is_bf16, x[j]);
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
                    if (h0 + j < min(last, values))
                        store_eight(a.v_pool, ((page * a.n_kv_heads + h0 + j) * kWave + slot % kWave) * D + col, 1, x[j]);
            }
        }
        if (last > values) {
            const auto turns = turn.template of<LPR>(a, seq, start, col);
            RowRotation<LPR> rot;
            turns.load(rot, a, turns.at(a, slot), col);
            const int64_t out = (static_cast<int64_t>(seq) * a.n_new + tok) * a.n_q_heads;
            for (int h0 = max(first - values, 0); h0 < last - values; h0 += kAhead) {
                float x[kAhead][8];
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
                    load_eight(a.q, seq * a.q_seq + tok * a.q_tok + min(h0 + j, last - values - 1) * a.q_head + col, a.q_is_bf16, x[j]);
#pragma unroll
                for (int j = 0; j < kAhead; ++j) {
                    rot.apply(x[j], lane);
                    if (h0 + j < last - values) store_eight(a.q_out, (out + h0 + j) * D + col, a.q_out_is_bf16, x[j]);
                }
            }
        }
        return;
    }

    // ---- keys ----
    const int kvh = (id / every) % a.n_kv_heads, run = (id / every) / a.n_kv_heads % tile_runs, seq = (id / every) / a.n_kv_heads / tile_runs;
    const int64_t start = append_start(a, seq);
    const int64_t tok_end = min(start + append_count(a, seq), static_cast<int64_t>(a.pt.stride) * kWave);
    const int64_t first_tile = start / kWave + static_cast<int64_t>(run) * tiles_per_group;
    if (max(first_tile * kWave, start) >= tok_end) return;
    const int64_t head_base = seq * a.k_seq + kvh * a.k_head + col;
    auto turns = turn.template of<LPR>(a, seq, start, col);
    const uint32_t sbits = a.signs[kvh * LPR + col / 8];

    // a tile's key rows: eight coordinates per thread and pass, rotated; rows outside [start, tok_end) are zeros
    {
        typedef const float __attribute__((address_space(4))) *arg_t;
        arg_t arg = (arg_t)__builtin_amdgcn_kernarg_segment_ptr();
        if (wave == 0) {
#pragma unroll
            for (int c = 0; c < P::NCLASS; ++c) {
                const float xi = arg[offsetof(DeviceBooks, c_xi) / 4 + c * kMaxLevels + lane], rho = arg[offsetof(DeviceBooks, c_rho) / 4 + c * kMaxLevels + lane];
                if (lane < Smem::NX) sm.c_xi[c][lane] = xi;
                if (lane < Smem::NR) sm.c_rho[c][lane] = rho;
            }
        }
    }
    __syncthreads();
    build_boundaries<P::BD0>(sm.bnd_xi[0], nullptr, sm.c_xi[0], tid);
    if constexpr (P::NCLASS == 2) build_boundaries<P::BD1>(sm.bnd_xi[1], nullptr, sm.c_xi[1], tid);
    build_encode_lut<P::BD0, REP, true>(sm.lut0, sm.nbx0, sm.nby0, sm.c_xi[0], tid, NT);
    if constexpr (P::NCLASS == 2) build_encode_lut<P::BD1, REP, true>(sm.lut1, sm.nbx1, sm.nby1, sm.c_xi[1], tid, NT);
    if (tid < P::NCLASS * Smem::NR) {
        const int c = tid / Smem::NR, k = tid % Smem::NR;
        const int levels = 1 << (c ? (P::BN1 > 0 ? P::BN1 : 1) : P::BN0);
        sm.bnd_rho[c][k] = (k < levels - 1) ? 0.5f * (sm.c_rho[c][k] + sm.c_rho[c][k + 1]) : INFINITY;
    }
    for (int e = tid; e < (3 * P::NTRI - D) * kWave; e += NT) sm.u[D + e / kWave][e % kWave] = 0.0f;

    for (int tg = 0; tg < tiles_per_group; ++tg) {
        const int64_t tile = first_tile + tg;
        const int64_t tok_lo = max(tile * kWave, start), tok_hi = min((tile + 1) * kWave, tok_end);
        if (tok_lo >= tok_hi) break;   // uniform over the workgroup
        const int64_t page = append_page(a, seq, tile);
        __syncthreads();               // the previous tile's records have been stored; tables are complete
        for (int e = kWave + tid; e < P::NWORDS * kWave; e += NT) sm.rec[e / kWave][e % kWave] = 0u;

        // E1-E2 and the first three stages of E3
        float rows[NPASS][8];
#pragma unroll
        for (int pass = 0; pass < NPASS; ++pass) {
            const int64_t tok = tile * kWave + pass * RPP + tid / LPR;
#pragma unroll
            for (int e = 0; e < 8; ++e) rows[pass][e] = 0.0f;
            if (tok >= tok_lo && tok < tok_hi) load_eight(a.k, head_base + (tok - start) * a.k_tok, a.kv_is_bf16, rows[pass]);
        }
#pragma unroll
        for (int pass = 0; pass < NPASS; ++pass) {
            const int key = pass * RPP + tid / LPR;
            float (&x)[8] = rows[pass];
            RowRotation<LPR> rot;
            turns.load(rot, a, turns.at(a, tile * kWave + key), col);
            rot.apply(x, lane);
            float ss = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
            ss = row_sum<LPR>(ss);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = ((sbits >> e) & 1u) ? -x[e] : x[e];
            butterflies<8>(x);
#pragma unroll
            for (int e = 0; e < 8; ++e) sm.u[col + e][key] = x[e];
            if (tid % LPR == 0) sm.sumsq[key] = ss;
        }
        __syncthreads();

        // E3: the other stages, one key per lane; the triplets take the coordinates unscaled and multiply by the key's factor
        {
            constexpr int R = D / 8;
            if (wave == NWV - 1) {
                const float gamma = sqrtf(sm.sumsq[lane]);
                sm.rec[0][lane] = __float_as_uint(gamma);
                sm.sumsq[lane] = (1.0f / fmaxf(gamma, kEps)) * inv_sqrt_dim<D>();
            }
            for (int lo = wave; lo < 8; lo += NWV) {
                float x[R];
#pragma unroll
                for (int e = 0; e < R; ++e) x[e] = sm.u[e * 8 + lo][lane];
                butterflies<R>(x);
#pragma unroll
                for (int e = 0; e < R; ++e) sm.u[e * 8 + lo][lane] = x[e];
            }
            __syncthreads();
        }

        // E4-E8: triplets, an equal share of them per wavefront, one key per lane
        {
            constexpr int CHUNK = (P::NTRI + NWV - 1) / NWV;
            const int i_first = wave * CHUNK, i_end = min(P::NTRI, (wave + 1) * CHUNK);
            constexpr bool THR0_REG = P::BN0 <= 3, THR1_REG = P::NCLASS == 2 && P::BN1 >= 1 && P::BN1 <= 3;
            float thr0_reg[THR0_REG ? (1 << P::BN0) : 1], thr1_reg[THR1_REG ? (1 << P::BN1) : 1];
            if constexpr (THR0_REG) {
#pragma unroll
                for (int k = 0; k < (1 << P::BN0) - 1; ++k) thr0_reg[k] = sm.bnd_rho[0][k];
            }
            if constexpr (THR1_REG) {
#pragma unroll
                for (int k = 0; k < (1 << P::BN1) - 1; ++k) thr1_reg[k] = sm.bnd_rho[1][k];
            }
            const float *thr0 = THR0_REG ? thr0_reg : sm.bnd_rho[0];
            const float *thr1 = THR1_REG ? thr1_reg : sm.bnd_rho[P::NCLASS - 1];
            using Grid1 = CornerGrid<(P::BD1 > 0 ? P::BD1 : 1)>;
            const uint32_t corner0 = CornerGrid<P::BD0>::template corner_start<REP>(lane);
            [[maybe_unused]] uint32_t corner1 = 0u;
            if constexpr (P::NCLASS == 2) corner1 = Grid1::template corner_start<REP>(lane);
            const float norm = sm.sumsq[lane];
            const bool valid = tile * kWave + lane >= tok_lo && tile * kWave + lane < tok_hi;
            FieldWriter<true> dir, nrm;
            dir.bit = (P::NCLASS == 1 || i_first < P::NT0) ? P::DIR0_BIT + i_first * 2 * P::BD0 : P::DIR1_BIT + (i_first - P::NT0) * 2 * P::BD1;
            nrm.bit = (P::NCLASS == 1 || i_first < P::NT0) ? P::NRM0_BIT + i_first * P::BN0 : P::NRM1_BIT + (i_first - P::NT0) * P::BN1;
            for (int i = i_first; i < i_end; ++i) {
                float x = sm.u[3 * i][lane] * norm, y = sm.u[3 * i + 1][lane] * norm, z = sm.u[3 * i + 2][lane] * norm;
                asm("" : "+v"(x), "+v"(y), "+v"(z));   // (the rounded products: none is to be fused into a later sum)
                uint32_t dir_field, nrm_index;
                if (P::NCLASS == 1 || i < P::NT0) {
                    encode_triplet_corners<P::BD0, P::BN0, REP, 3 * P::NTRI - D == 2>(x, y, z, sm.lut0, corner0, sm.bnd_xi[0], thr0, lane, valid,
                                                                                     3 * i + 3 - D, &dir_field, &nrm_index);
                    dir.put(sm.rec, lane, 2 * P::BD0, dir_field);
                    nrm.put(sm.rec, lane, P::BN0, nrm_index);
                } else if constexpr (P::NCLASS == 2) {
                    encode_triplet_corners<P::BD1, P::BN1, REP, 3 * P::NTRI - D == 2>(x, y, z, sm.lut1, corner1, sm.bnd_xi[1], thr1, lane, valid,
                                                                                     3 * i + 3 - D, &dir_field, &nrm_index);
                    if (i == P::NT0 && i > i_first) {   // the second class has its own streams
                        dir.finish(sm.rec, lane);
                        nrm.finish(sm.rec, lane);
                        dir = FieldWriter<true>{0u, P::DIR1_BIT};
                        nrm = FieldWriter<true>{0u, P::NRM1_BIT};
                    }
                    dir.put(sm.rec, lane, 2 * P::BD1, dir_field);
                    nrm.put(sm.rec, lane, P::BN1, nrm_index);
                }
            }
            dir.finish(sm.rec, lane);
            nrm.finish(sm.rec, lane);
        }
        __syncthreads();

        // E8: store the tile, 16 bytes per (granule, key), coalesced over keys
        uint4 *dst = static_cast<uint4 *>(a.k_pool) + (page * a.n_kv_heads + kvh) * (P::GRANULES * kWave);
        for (int e = tid; e < P::GRANULES * kWave; e += NT) {
            const int g = e / kWave, key = e % kWave;
            const int64_t tok = tile * kWave + key;
            if (tok >= tok_lo && tok < tok_hi)
                dst[e] = make_uint4(sm.rec[4 * g][key], sm.rec[4 * g + 1][key], sm.rec[4 * g + 2][key], sm.rec[4 * g + 3][key]);
        }
    }
}

#define OCTOPUS_TILE_KERNEL                          \
    __global__ __launch_bounds__(encode_threads<P>()) \
    __attribute__((amdgpu_waves_per_eu(encode_waves_per_simd<P, false, true>(), encode_waves_per_simd<P, false, true>()))) void
template <class P>
OCTOPUS_TILE_KERNEL append_tile_kernel(DeviceBooks books, AppendCall a, int32_t key_blocks, int32_t tile_runs, int32_t tiles_per_group, int32_t every) {
    append_tile<P>(a, OneAxis{}, key_blocks, tile_runs, tiles_per_group, every);
}
template <class P>
OCTOPUS_TILE_KERNEL append_tile_axes_kernel(DeviceBooks books, AppendCall a, ManyAxes turn, int32_t key_blocks, int32_t tile_runs, int32_t tiles_per_group,
                                            int32_t every) {
    append_tile<P>(a, turn, key_blocks, tile_runs, tiles_per_group, every);
}
#undef OCTOPUS_TILE_KERNEL

// The launch of a call: token(grid, threads) for few tokens, else tile(grid, threads, key blocks, runs, tiles a run, every).
template <class P, class Token, class Tile>
int launch_append_shape(const AppendCall &a, Token token, Tile tile) {
    if (few_keys<P::D>(a.n_seq, a.n_kv_heads, a.n_new)) {
        token(dim3(a.n_new, a.n_kv_heads, a.n_seq), dim3(kWave));
        return static_cast<int>(hipGetLastError());
    }
    constexpr int RPP = encode_threads<P>() / (P::D / 8);
    const int tiles = (a.n_new + kWave - 1) / kWave + (a.start_pos ? 1 : 0);   // (a start inside a tile: one tile more)
    const int per = encode_tiles_per_group(tiles, a.n_kv_heads, a.n_seq), runs = (tiles + per - 1) / per;
    const int64_t key_blocks = static_cast<int64_t>(runs) * a.n_kv_heads * a.n_seq;
    const int rows = (a.v_pool != nullptr ? a.n_kv_heads : 0) + (a.q != nullptr ? a.n_q_heads : 0);
    const int64_t row_blocks = static_cast<int64_t>((rows + kAppendRows - 1) / kAppendRows) * ((a.n_new + RPP - 1) / RPP) * a.n_seq;
    const int64_t blocks = key_blocks + row_blocks;
    if (blocks > (1 << 22)) return static_cast<int>(hipErrorInvalidValue);   // (threads of a launch; the host has checked it)
    tile(dim3(static_cast<unsigned>(blocks)), dim3(encode_threads<P>()), static_cast<int32_t>(key_blocks), runs, per,
         static_cast<int32_t>(blocks / key_blocks));
    return static_cast<int>(hipGetLastError());
}

template <class P>
int launch_append_plan(const octopus_codebooks_t &cb, const AppendCall &a, hipStream_t stream) {
    const DeviceBooks books = device_books(cb);
    return launch_append_shape<P>(
        a, [&](dim3 grid, dim3 threads) { hipLaunchKernelGGL(append_token_kernel<P>, grid, threads, 0, stream, books, a); },
        [&](dim3 grid, dim3 threads, int32_t key_blocks, int32_t runs, int32_t per, int32_t every) {
            hipLaunchKernelGGL(append_tile_kernel<P>, grid, threads, 0, stream, books, a, key_blocks, runs, per, every);
        });
}

template <class P>
int launch_append_axes_plan(const octopus_codebooks_t &cb, const AppendCall &a, hipStream_t stream) {
    const DeviceBooks books = device_books(cb);
    const ManyAxes turn{*a.axes};
    return launch_append_shape<P>(
        a, [&](dim3 grid, dim3 threads) { hipLaunchKernelGGL(append_token_axes_kernel<P>, grid, threads, 0, stream, books, a, turn); },
        [&](dim3 grid, dim3 threads, int32_t key_blocks, int32_t runs, int32_t per, int32_t every) {
            hipLaunchKernelGGL(append_tile_axes_kernel<P>, grid, threads, 0, stream, books, a, turn, key_blocks, runs, per, every);
        });
}

}  // namespace octopus

#endif

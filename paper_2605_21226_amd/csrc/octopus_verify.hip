// Verification of drafted tokens: how many of a sequence's drafts stand by the target's probabilities, and the token that follows them.
//
// Draft x_i, drawn from q_i, stands if u_i q_i(x_i) < p_i(x_i); a is the number of drafts before the first that does not.  The token
// after them is drawn from the weights r = max(p_a - q_a, 0) if draft a fell (tokens come out distributed as the target's), from p_a
// if all of them stand: the first token whose running sum of r exceeds u times the whole sum.
//
// A call reads a handful of numbers to find a, and then the target's row, and the drafter's where a draft fell.  What bounds it is latency: for few
// sequences four reads that wait for each other (1 x 8000 tokens 5.5 us), for many the same chain in front of each wavefront's one piece (256 x
// 128256 tokens in fp32, a third of whose drafts fall, 172 MB, 38 us with other inputs each call, 4.5 TB/s of a plain read's 7.07; 31 us with
// the same inputs, which the last-level cache holds).  A row is
// cut into pieces, a wavefront each, that are summed; then a wavefront finds the piece in which the running sum gets there, reads it once
// more and finds the token.  Differences and sums are 64-bit numbers: u has 24 bits, and a running sum over 10^5 tokens has to tell neighbours
// apart that differ by less.  Rows that are subtracted from and rows that are not have code of their own, and pieces inside a row need no
// comparison with its end: with both in one loop 1 x 8000 tokens took 7.8 us, 256 x 128256 40.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "octopus_internal.h"
#include "octopus_scan.hpp"

namespace octopus {
namespace {

constexpr int kLanes = kScanLanes;

// A probability that counts: a positive finite number, or none.
__device__ __forceinline__ float counted(float p) {
    constexpr int kPositiveDenormal = 1 << 7, kPositiveNormal = 1 << 8;
    return __builtin_amdgcn_classf(p, kPositiveDenormal | kPositiveNormal) ? p : 0.0f;
}
__device__ __forceinline__ double uniform(float u) { return u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0; }   // [0, 1)

// One of the distributions' rows.
template <bool BF16>
struct Row {
    using Word = typename std::conditional<BF16, uint16_t, float>::type;
    static constexpr int AT_ONCE = 16 / sizeof(Word);      // tokens of a 16-byte read
    const Word *p;
    __device__ __forceinline__ static Row of(const void *base, int64_t at) { return Row{static_cast<const Word *>(base) + at}; }
    __device__ __forceinline__ float operator[](int64_t i) const {
        if constexpr (BF16) return counted(__uint_as_float(static_cast<uint32_t>(p[i]) << 16));
        else return counted(p[i]);
    }
    // tokens i .. i + AT_ONCE - 1 (rows begin at any element: the reads are as aligned as those)
    __device__ __forceinline__ void load(int i, float (&x)[AT_ONCE]) const {
        typedef uint32_t words_t __attribute__((ext_vector_type(4), aligned(2)));
        const words_t w = *reinterpret_cast<const words_t *>(p + i);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            if constexpr (BF16) x[k] = counted(__uint_as_float(k % 2 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16));
            else x[k] = counted(__uint_as_float(w[k]));
        }
    }
    // ... none from `end` on
    __device__ __forceinline__ void load(int i, int end, float (&x)[AT_ONCE]) const {
        if (i + AT_ONCE <= end) return load(i, x);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) x[k] = 0.0f;
        if (i < end) {
#pragma unroll
            for (int k = 0; k < AT_ONCE - 1; ++k)
                if (i + k < end) x[k] = (*this)[i + k];
        }
    }
};

template <bool BF16>
__device__ __forceinline__ Row<BF16> target_row(const VerifyCall &c, int s, int i) {
    return Row<BF16>::of(c.target, s * c.target_seq + i * c.target_pos);
}
template <bool BF16>
__device__ __forceinline__ Row<BF16> draft_row(const VerifyCall &c, int s, int i) {
    return Row<BF16>::of(c.draft, s * c.draft_seq + i * c.draft_pos);
}

// The drafts of sequence s, those that stand, and the one that fell.  Every wavefront looks for itself, a draft per lane: a read of what was drafted
// and one of the probabilities that it goes by.
struct Drafts {
    int n, a, fell;
};
__device__ __forceinline__ int draft_count(const VerifyCall &c, int s) {
    return c.draft_lens != nullptr ? min(max(c.draft_lens[s], 0), c.n_draft) : c.n_draft;
}
template <bool BF16>
__device__ __forceinline__ Drafts standing(const VerifyCall &c, int s) {
    const int lane = threadIdx.x % kLanes;
    Drafts d{0, 0, -1};
    for (int i0 = 0; i0 == 0 || i0 < d.n; i0 += kLanes) {
        const int i = i0 + lane;
        int x = -1;
        float u = 0.0f;
        if (i < c.n_draft) {
            x = c.tokens[static_cast<int64_t>(s) * c.n_draft + i];
            u = c.uniforms[static_cast<int64_t>(s) * (c.n_draft + 1) + i];
        }
        if (i0 == 0) d.n = draft_count(c, s);
        const bool is = i < d.n && x >= 0 && x < c.vocab;
        const float p = is ? target_row<BF16>(c, s, i)[x] : 0.0f;
        const float q = c.draft == nullptr ? 1.0f : (is ? draft_row<BF16>(c, s, i)[x] : 0.0f);
        const unsigned long long fallen = __ballot(i < d.n && !(uniform(u) * q < p));     // (a product of two 24-bit numbers is exact in 64 bits)
        if (fallen != 0) {
            const int at = __ffsll(fallen) - 1;
            d.a = i0 + at;
            d.fell = __builtin_amdgcn_readlane(x, at);
            return d;
        }
    }
    d.a = d.n;
    return d;
}

constexpr int kRound = 1024;     // tokens that a wavefront has in registers

// Of the lanes that have something the first that is past the goal, without one the last; -1: none has.
__device__ __forceinline__ int first_past(bool some, bool past) {
    const unsigned long long has = __ballot(some), hits = __ballot(some && past);
    return hits != 0 ? __ffsll(hits) - 1 : (has != 0 ? 63 - __clzll(static_cast<long long>(has)) : -1);
}

// What the token after the drafts is drawn from: p less q (LESS: a draft of q fell), or p, without the token that fell if it had no
// probabilities.
template <bool BF16, bool LESS>
struct Weights {
    static constexpr int AT_ONCE = Row<BF16>::AT_ONCE;
    Row<BF16> p, q;
    int vocab;
    int without;         // that token, -1: none
    __device__ __forceinline__ static Weights of(const VerifyCall &c, int s, const Drafts &d) {
        return Weights{target_row<BF16>(c, s, d.a), LESS ? draft_row<BF16>(c, s, d.a) : Row<BF16>{}, c.vocab, c.draft == nullptr ? d.fell : -1};
    }
    __device__ __forceinline__ static double rest(float x, float y) {
        return LESS ? fmax(static_cast<double>(x) - static_cast<double>(y), 0.0) : static_cast<double>(x);
    }
    // A round of tokens from `at` on, none from `end` on: those of this lane, in a run of their own (RUN; for the one that goes on to
    // look for a token) or 16 bytes at a time side by side with the other lanes'.
    template <bool RUN>
    struct Round {
        static constexpr int READS = kRound / kLanes / AT_ONCE;
        float x[READS][AT_ONCE], y[READS][AT_ONCE];
        float left_out = 0.0f;       // what `without` had
        __device__ __forceinline__ static int offset(int i) { return i * AT_ONCE * (RUN ? 1 : kLanes); }
        __device__ __forceinline__ Round(const Weights &w, int at, int end, int without) {
            const int first = at + static_cast<int>(threadIdx.x % kLanes) * (RUN ? kRound / kLanes : AT_ONCE);
            if (at + kRound <= end) {
#pragma unroll
                for (int i = 0; i < READS; ++i) w.p.load(first + offset(i), x[i]);
                if constexpr (LESS) {
#pragma unroll
                    for (int i = 0; i < READS; ++i) w.q.load(first + offset(i), y[i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < READS; ++i) {
                    w.p.load(first + offset(i), end, x[i]);
                    if constexpr (LESS) w.q.load(first + offset(i), end, y[i]);
                }
            }
            if constexpr (!LESS) {
                if (without < at || without >= at + kRound) return;
#pragma unroll
                for (int i = 0; i < READS; ++i)
#pragma unroll
                    for (int k = 0; k < AT_ONCE; ++k)
                        if (first + offset(i) + k == without) {
                            left_out = x[i][k];
                            x[i][k] = 0.0f;
                        }
            }
        }
    };
    // A lane's sums over its tokens of [first, end).
    __device__ __forceinline__ RowSums sum(int first, int end) const {
        RowSums sum{0.0, 0.0};
        for (int at = first; at < end; at += kRound) {
            const Round<false> r(*this, at, end, without);
#pragma unroll
            for (int i = 0; i < r.READS; ++i)
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) {
                    if constexpr (LESS) sum.whole += r.x[i][k];
                    sum.rest += rest(r.x[i][k], r.y[i][k]);
                }
            if constexpr (!LESS) sum.whole += r.left_out;
        }
        if constexpr (!LESS) sum.whole += sum.rest;
        return sum;
    }
    // The first token of [first, end) whose weight is positive and whose running sum, from `before` on, exceeds the goal; without one
    // the last one with a positive weight (sums in another order may miss the goal by their last bits), -1 where there is none.  First the
    // lane whose run of tokens it is, and then a lane per token of that run, which is little code: code that runs once costs its fetch.
    __device__ __forceinline__ int find(int first, int end, double before, double goal, bool of_rest) const {
        constexpr int RUN = kRound / kLanes;
        const int left_out = of_rest ? without : -1;
        int token = -1;
        for (int at = first; at < end; at += kRound) {
            double own = 0.0;
            {
                const Round<true> r(*this, at, end, left_out);
#pragma unroll
                for (int i = 0; i < r.READS; ++i)
#pragma unroll
                    for (int k = 0; k < AT_ONCE; ++k) own += of_rest ? rest(r.x[i][k], r.y[i][k]) : static_cast<double>(r.x[i][k]);
            }
            const double upto = wave_scan(own);
            const int lane = first_past(own > 0.0, before + upto > goal);
            if (lane >= 0) {
                const int v = at + lane * RUN + static_cast<int>(threadIdx.x % kLanes);
                const bool there = threadIdx.x % kLanes < RUN && v < end && v != left_out;
                const float x = there ? p[v] : 0.0f, y = LESS && there ? q[v] : 0.0f;
                const double weight = of_rest ? rest(x, y) : static_cast<double>(x);
                token = at + lane * RUN + first_past(weight > 0.0, before + wave_lane(upto - own, lane) + wave_scan(weight) > goal);
                if (before + wave_lane(upto, lane) > goal) break;
            }
            before += wave_last(upto);
        }
        return token;
    }
};

// The piece in which the running sum exceeds the goal, as Weights::find has it, and the sum before it, in the same way: sums[i], i < pieces,
// kLanePieces of them a lane.
constexpr int kLanePieces = kMostPieces / kLanes;
struct Found {
    int piece;
    bool of_rest;
    double before, goal;
};
__device__ __forceinline__ Found find_piece(const RowSums *sums, int pieces, float u) {
    const int lane = threadIdx.x % kLanes;
    RowSums sum{0.0, 0.0};
#pragma unroll
    for (int i = 0; i < kLanePieces; ++i) {
        const int at = lane * kLanePieces + i;
        const RowSums piece = sums[min(at, pieces - 1)];
        sum.whole += at < pieces ? piece.whole : 0.0;
        sum.rest += at < pieces ? piece.rest : 0.0;
    }
    const double whole = wave_scan(sum.whole), rest = wave_scan(sum.rest);
    Found f;
    f.of_rest = wave_last(rest) > 0.0;     // (nothing left of a row, whose drafts were as likely as they were to be: all of it counts)
    f.goal = uniform(u) * wave_last(f.of_rest ? rest : whole);
    const double own = f.of_rest ? sum.rest : sum.whole, upto = f.of_rest ? rest : whole;
    const int first = first_past(own > 0.0, upto > f.goal), at = max(first, 0) * kLanePieces + lane;
    const RowSums mine = sums[min(at, pieces - 1)];
    const double piece = lane < kLanePieces && at < pieces ? (f.of_rest ? mine.rest : mine.whole) : 0.0;
    const double run = wave_lane(upto - own, max(first, 0)) + wave_scan(piece);
    const int nth = first_past(piece > 0.0, run > f.goal);
    f.piece = first < 0 ? -1 : first * kLanePieces + nth;
    f.before = wave_lane(run - piece, max(nth, 0));
    return f;
}

__device__ __forceinline__ void answer(const VerifyCall &c, int s, int a, int token) {
    for (int i = threadIdx.x % kLanes; i <= c.n_draft; i += kLanes)
        c.tokens_out[static_cast<int64_t>(s) * (c.n_draft + 1) + i] = i < a ? c.tokens[static_cast<int64_t>(s) * c.n_draft + i] : (i == a ? token : -1);
    if (threadIdx.x % kLanes == 0) c.accepted[s] = a;
}
__device__ __forceinline__ float last_uniform(const VerifyCall &c, int s) {
    return c.uniforms[static_cast<int64_t>(s) * (c.n_draft + 1) + c.n_draft];
}

// f(weights) by the kind that the drafts leave.
template <bool BF16, class F>
__device__ __forceinline__ void with_weights(const VerifyCall &c, int s, const Drafts &d, F f) {
    if (d.a < d.n && c.draft != nullptr) f(Weights<BF16, true>::of(c, s, d));
    else f(Weights<BF16, false>::of(c, s, d));
}

// A workgroup per sequence; its wavefronts take the pieces in turns.
constexpr int kRowWaves = 16;
template <bool BF16>
__global__ __launch_bounds__(kRowWaves * kLanes) void verify_row_kernel(VerifyCall c) {
    __shared__ RowSums sums[kMostPieces];
    const int s = blockIdx.x, lane = threadIdx.x % kLanes, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const float u = last_uniform(c, s);
    const Drafts d = standing<BF16>(c, s);
    with_weights<BF16>(c, s, d, [&](const auto &w) {
        for (int i = wave; i < c.pieces; i += kRowWaves) {
            const RowSums sum = w.sum(i * c.piece, min((i + 1) * c.piece, c.vocab));
            const double whole = wave_scan(sum.whole), rest = wave_scan(sum.rest);
            if (lane == kLanes - 1) sums[i] = RowSums{whole, rest};
        }
        __syncthreads();
        if (wave != 0) return;
        const Found f = find_piece(sums, c.pieces, u);
        const int first = f.piece * c.piece;
        answer(c, s, d.a, f.piece < 0 ? -1 : w.find(first, min(first + c.piece, c.vocab), f.before, f.goal, f.of_rest));
    });
}

// A wavefront per piece ...
template <bool BF16>
__global__ __launch_bounds__(kLanes) void verify_sums_kernel(VerifyCall c) {
    const int s = blockIdx.y;
    const Drafts d = standing<BF16>(c, s);
    with_weights<BF16>(c, s, d, [&](const auto &w) {
        const int first = blockIdx.x * c.piece;
        const RowSums sum = w.sum(first, min(first + c.piece, c.vocab));
        const double whole = wave_scan(sum.whole), rest = wave_scan(sum.rest);
        if (threadIdx.x == kLanes - 1) c.sums[static_cast<int64_t>(s) * c.pieces + blockIdx.x] = RowSums{whole, rest};
    });
    if (blockIdx.x == 0 && threadIdx.x == 0) c.accepted[s] = d.a;
}

// ... and one for the token.
template <bool BF16>
__global__ __launch_bounds__(kLanes) void verify_pick_kernel(VerifyCall c) {
    const int s = blockIdx.x;
    const float u = last_uniform(c, s);
    Drafts d{draft_count(c, s), c.accepted[s], -1};
    if (c.draft == nullptr && d.a < d.n) d.fell = c.tokens[static_cast<int64_t>(s) * c.n_draft + d.a];
    with_weights<BF16>(c, s, d, [&](const auto &w) {
        const Found f = find_piece(c.sums + static_cast<int64_t>(s) * c.pieces, c.pieces, u);
        const int first = f.piece * c.piece;
        answer(c, s, d.a, f.piece < 0 ? -1 : w.find(first, min(first + c.piece, c.vocab), f.before, f.goal, f.of_rest));
    });
}

}  // namespace

int launch_verify(VerifyCall c, void *stream) {
    const hipStream_t on = static_cast<hipStream_t>(stream);
    c.piece = (c.vocab / (kMostPieces * kRound) + 1) * kRound;
    c.pieces = (c.vocab + c.piece - 1) / c.piece;
    // Rows of up to 64 pieces in one launch, the others in two.  us a call, fp32, one launch / two, of sequences whose drafts all fell (two rows each
    // are read; of one row each, where all stood or have no probabilities, in brackets):
    //                    captured                     eager
    //   1 x 8000         5.5 / 6.7   (4.6 / 5.9)      5.9 / 8.2   (6.1 / 8.9)
    //   1 x 32000        7.5 / 6.2   (5.8 / 5.7)      7.3 / 9.5   (6.4 / 9.4)
    //   512 x 32000      28.7 / 30.7 (14.7 / 17.6)    27.9 / 30.4 (14.2 / 17.2)
    //   8 x 50257        9.3 / 6.9   (7.0 / 6.5)      9.1 / 9.4   (7.0 / 9.4)
    //   256 x 50257      22.5 / 25.7 (12.2 / 15.2)    22.2 / 25.2 (11.8 / 14.8)
    //   1 x 64000        10.5 / 6.3  (7.7 / 5.8)      10.4 / 9.2  (7.5 / 9.5)
    //   64 x 64000       13.2 / 13.0 (9.4 / 9.8)      12.7 / 12.8 (9.1 / 9.8)
    //   1 x 128256       16.5 / 6.2  (11.4 / 5.7)     16.5 / 9.1  (11.1 / 9.3)
    //   64 x 128256      24.2 / 17.4 (13.2 / 11.9)    23.6 / 16.9 (12.8 / 11.8)
    // The limit is where eager calls come out even, whose caller needs 3 us for a second launch; many sequences gain by it in graphs as well, and a
    // captured call of a few sequences pays for it, at most 4.2 us (1 x 64000).
    if (c.pieces <= 64) {
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(c.n_seq), dim3(kRowWaves * kLanes), 0, on, c); };
        if (c.is_bf16) go(verify_row_kernel<true>);
        else go(verify_row_kernel<false>);
    } else {
        auto go = [&](auto sums, auto pick) {
            hipLaunchKernelGGL(sums, dim3(c.pieces, c.n_seq), dim3(kLanes), 0, on, c);
            hipLaunchKernelGGL(pick, dim3(c.n_seq), dim3(kLanes), 0, on, c);
        };
        if (c.is_bf16) go(verify_sums_kernel<true>, verify_pick_kernel<true>);
        else go(verify_sums_kernel<false>, verify_pick_kernel<false>);
    }
    return static_cast<int>(hipGetLastError());
}

}  // namespace octopus

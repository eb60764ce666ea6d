// Verification of drafted tokens: how many of a sequence's drafts stand by the target's probabilities, and the token that follows them.
//
// Draft x_i, drawn from q_i, stands if u_i q_i(x_i) < p_i(x_i); a is the number of drafts before the first that does not.  The token
// after them is drawn from the weights r = max(p_a - q_a, 0) if draft a fell (tokens come out distributed as the target's), from p_a
// if all of them stand: the first token whose running sum of r exceeds u times the whole sum.
//
// A call reads a handful of numbers to find a, and then one row of each of the two distributions: memory bounds it for many sequences,
// latency for few.  The row is cut into pieces, a workgroup each, that write their sums; a second launch finds the piece in which the
// running sum gets there, and the token inside it.  Differences and sums are 64-bit numbers: u has 24 bits, and a running sum over
// 10^5 tokens has to tell neighbours apart that differ by less.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "octopus_internal.h"

namespace octopus {
namespace {

constexpr int kLanes = 64, kThreads = 256, kWaves = kThreads / kLanes;

// A probability that counts: a positive finite number, or none.
__device__ __forceinline__ float counted(float p) { return p > 0.0f && p < INFINITY ? p : 0.0f; }
__device__ __forceinline__ double uniform(float u) { return u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0; }   // [0, 1)

template <bool BF16>
struct Row {
    using Word = typename std::conditional<BF16, uint16_t, float>::type;
    static constexpr int AT_ONCE = 16 / sizeof(Word);      // of a 16-byte read
    const Word *p;
    __device__ __forceinline__ static Row of(const void *base, int64_t at) { return Row{static_cast<const Word *>(base) + at}; }
    __device__ __forceinline__ float operator[](int64_t i) const {
        if constexpr (BF16) return counted(__uint_as_float(static_cast<uint32_t>(p[i]) << 16));
        else return counted(p[i]);
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
__device__ __forceinline__ int draft_count(const VerifyCall &c, int s) {
    return c.draft_lens != nullptr ? min(max(c.draft_lens[s], 0), c.n_draft) : c.n_draft;
}

// Drafts of sequence s that stand; every wavefront finds them for itself, a draft per lane.
template <bool BF16>
__device__ __forceinline__ int standing(const VerifyCall &c, int s, int n) {
    const int lane = threadIdx.x % kLanes;
    for (int i0 = 0; i0 < n; i0 += kLanes) {
        const int i = i0 + lane;
        bool stands = true;
        if (i < n) {
            const int x = c.tokens[static_cast<int64_t>(s) * c.n_draft + i];
            const double u = uniform(c.uniforms[static_cast<int64_t>(s) * (c.n_draft + 1) + i]);
            const bool is = x >= 0 && x < c.vocab;
            const float p = is ? target_row<BF16>(c, s, i)[x] : 0.0f;
            const float q = c.draft == nullptr ? 1.0f : (is ? draft_row<BF16>(c, s, i)[x] : 0.0f);
            stands = u * q < p;       // (a product of two 24-bit numbers is exact in 64 bits)
        }
        const uint64_t fallen = __ballot(!stands);
        if (fallen != 0) return i0 + __ffsll(static_cast<unsigned long long>(fallen)) - 1;
    }
    return n;
}

// What the token after the drafts is drawn from.
template <bool BF16>
struct Weights {
    Row<BF16> p, q;
    bool less;           // q is subtracted
    int without;         // a token without weight (a draft that fell and has no probabilities), -1: none
    __device__ __forceinline__ static Weights of(const VerifyCall &c, int s, int a, int n) {
        Weights w;
        w.p = target_row<BF16>(c, s, a);
        w.less = a < n && c.draft != nullptr;
        w.q = w.less ? draft_row<BF16>(c, s, a) : w.p;
        w.without = a < n && c.draft == nullptr ? c.tokens[static_cast<int64_t>(s) * c.n_draft + a] : -1;
        return w;
    }
    // of token v: p(v), and what is left of it
    __device__ __forceinline__ double2 at(int v) const {
        const double p = this->p[v];
        return make_double2(p, v == without ? 0.0 : (less ? fmax(p - static_cast<double>(q[v]), 0.0) : p));
    }
};

// Inclusive sums over a wavefront's lanes, 64 bits.
__device__ __forceinline__ double wave_scan(double x, int lane) {
#pragma unroll
    for (int m = 1; m < kLanes; m *= 2) {
        const double other = __shfl_up(x, m, kLanes);
        x += lane >= m ? other : 0.0;
    }
    return x;
}
// ... over a workgroup's threads; everybody's sum.  (all threads call this; one order of sums, whatever runs beside it)
__device__ __forceinline__ double block_scan(double x, double *room, double *total) {
    const int lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes;
    const double upto = wave_scan(x, lane);
    __syncthreads();
    if (lane == kLanes - 1) room[wave] = upto;
    __syncthreads();
    double before = 0.0, all = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        before += w < wave ? room[w] : 0.0;
        all += room[w];
    }
    *total = all;
    return before + upto;
}

// A piece's two sums.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void verify_sums_kernel(VerifyCall c) {
    __shared__ double room[kWaves];
    const int s = blockIdx.y, n = draft_count(c, s), a = standing<BF16>(c, s, n);
    const Weights<BF16> w = Weights<BF16>::of(c, s, a, n);
    const int first = blockIdx.x * c.piece, last = min(first + c.piece, c.vocab);
    double2 sum = make_double2(0.0, 0.0), total;
    for (int v = first + threadIdx.x; v < last; v += kThreads) {
        const double2 x = w.at(v);
        sum.x += x.x;
        sum.y += x.y;
    }
    block_scan(sum.x, room, &total.x);
    block_scan(sum.y, room, &total.y);
    if (threadIdx.x == 0) {
        c.sums[static_cast<int64_t>(s) * c.pieces + blockIdx.x] = RowSums{total.x, total.y};
        if (blockIdx.x == 0) c.accepted[s] = a;
    }
}

// The token, and what the call says of the sequence.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void verify_pick_kernel(VerifyCall c) {
    static_assert(kMostPieces <= kThreads, "a piece per thread");
    __shared__ double room[kWaves], upto;
    __shared__ int hit, last;
    const int s = blockIdx.x, tid = threadIdx.x, n = draft_count(c, s), a = c.accepted[s];
    const Weights<BF16> w = Weights<BF16>::of(c, s, a, n);
    const RowSums mine = tid < c.pieces ? c.sums[static_cast<int64_t>(s) * c.pieces + tid] : RowSums{0.0, 0.0};
    double2 total;
    block_scan(mine.whole, room, &total.x);
    block_scan(mine.rest, room, &total.y);
    const bool rest = total.y > 0.0;         // (nothing left of a row, whose drafts were as likely as they were to be: all of it counts)
    const double goal = uniform(c.uniforms[static_cast<int64_t>(s) * (c.n_draft + 1) + c.n_draft]) * (rest ? total.y : total.x);

    // The first of the threads' values that is positive and whose running sum, from `before` on, exceeds the goal; without one the last
    // positive one (sums in another order may miss the goal by their last bits); -1 where none is positive.  `upto`: the sum before it.
    auto find = [&](double own, double before) {
        double all;
        const double run = before + block_scan(own, room, &all);
        if (tid == 0) {
            hit = kThreads;
            last = -1;
        }
        __syncthreads();
        if (own > 0.0) {
            if (run > goal) atomicMin(&hit, tid);
            atomicMax(&last, tid);
        }
        __syncthreads();
        const int at = hit < kThreads ? hit : last;
        if (tid == at) upto = run - own;
        __syncthreads();
        return at;
    };
    const int piece = find(rest ? mine.rest : mine.whole, 0.0);
    int token = -1;
    if (piece >= 0) {
        const double before = upto;
        const int each = c.piece / kThreads, first = piece * c.piece + tid * each, end = min(first + each, c.vocab);
        double own = 0.0;
        for (int v = first; v < end; ++v) {
            const double2 x = w.at(v);
            own += rest ? x.y : x.x;
        }
        if (find(own, before) == tid) {
            double run = upto;
            for (int v = first; v < end; ++v) {
                const double2 both = w.at(v);
                const double x = rest ? both.y : both.x;
                if (x <= 0.0) continue;
                token = v;
                run += x;
                if (run > goal) break;
            }
            last = token;
        }
        __syncthreads();
        token = last;
    }
    for (int i = tid; i <= c.n_draft; i += kThreads)
        c.tokens_out[static_cast<int64_t>(s) * (c.n_draft + 1) + i] = i < a ? c.tokens[static_cast<int64_t>(s) * c.n_draft + i] : (i == a ? token : -1);
}

}  // namespace

int launch_verify(const VerifyCall &c, void *stream) {
    const hipStream_t on = static_cast<hipStream_t>(stream);
    auto go = [&](auto sums, auto pick) {
        hipLaunchKernelGGL(sums, dim3(c.pieces, c.n_seq), dim3(kThreads), 0, on, c);
        hipLaunchKernelGGL(pick, dim3(c.n_seq), dim3(kThreads), 0, on, c);
        return static_cast<int>(hipGetLastError());
    };
    return c.is_bf16 ? go(verify_sums_kernel<true>, verify_pick_kernel<true>) : go(verify_sums_kernel<false>, verify_pick_kernel<false>);
}

}  // namespace octopus

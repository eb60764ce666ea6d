// Tokens of a paged cache as values again: k^ = gamma D_s H u^ (Sec. 3.1: the rotation is its own inverse up to the signs), and the
// value rows, dequantised where they are quantised.
//
// A workgroup takes a 64-token tile of one (sequence, KV head), the encoder's phases the other way round: records unpacked a key per
// lane, a share of the triplets per wavefront; the transform's far stages a key per lane; its near ones eight coordinates a thread,
// which then have the order of the output row.  Bound by memory (a row out is 256 bytes at d = 128 in bf16, its record 64): 15877
// tokens of 8 KV heads, 106 MB, take 21.8 us, 4.8 TB/s; at d = 256 with quantised values to fp32, 41 MB of ragged tails, 15.9.
#ifndef OCTOPUS_READ_HPP_
#define OCTOPUS_READ_HPP_

#include "octopus_append.hpp"

namespace octopus {

template <class P>
struct ReadSmem {
    float u[3 * P::NTRI][kWave + 1];
    float4 dir0[1 << (2 * P::BD0)];
    float4 dir1[P::NCLASS == 2 ? 1 << (2 * P::BD1) : 1];
    float c_xi[P::NCLASS][kMaxLevels];
    float c_rho[P::NCLASS][kMaxLevels];
};

template <class P>
__global__ __launch_bounds__(read_waves(P::D) * 64) void read_tokens_kernel(DeviceBooks books, ReadCall a) {
    constexpr int D = P::D, NWV = read_waves(D), NT = NWV * 64, LPR = D / 8, RPP = NT / LPR;
    __shared__ ReadSmem<P> sm;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kvh = blockIdx.y, seq = blockIdx.z;
    const int64_t start = a.start_pos ? max(a.start_pos[seq], 0) : 0;
    const int count = a.lens ? min(max(a.lens[seq], 0), a.n_tok) : a.n_tok;
    const int64_t end = min(start + count, static_cast<int64_t>(a.pt.stride) * kWave);
    const int64_t tile = start / kWave + blockIdx.x, lo = max(tile * kWave, start), hi = min((tile + 1) * kWave, end);
    if (lo >= hi) return;
    const int64_t page = min(max(a.pt.table[static_cast<int64_t>(seq) * a.pt.stride + tile], 0), a.pt.n_pages - 1);
    const int64_t slab = page * a.n_kv_heads + kvh;
    const int col = (tid % LPR) * 8;

    if (a.k_out != nullptr) {
        uint32_t w[P::NWORDS];
        const uint4 *src = static_cast<const uint4 *>(a.k_pool) + slab * (P::GRANULES * kWave) + lane;
#pragma unroll
        for (int g = 0; g < P::GRANULES; ++g) {
            const uint4 x = src[g * kWave];
            w[4 * g] = x.x; w[4 * g + 1] = x.y; w[4 * g + 2] = x.z; w[4 * g + 3] = x.w;
        }
        {   // a level per lane, of one array per wavefront
            typedef const float __attribute__((address_space(4))) *arg_t;
            const float level = ((arg_t)__builtin_amdgcn_kernarg_segment_ptr())[offsetof(DeviceBooks, c_xi) / 4 + (wave % 4) * kMaxLevels + lane];
            if (wave < 4 && wave % 2 < P::NCLASS) (wave < 2 ? sm.c_xi[wave % P::NCLASS] : sm.c_rho[wave % P::NCLASS])[lane] = level;
        }
        __syncthreads();
        build_dir_lut<P::BD0>(sm.dir0, sm.c_xi[0], tid, NT);
        if constexpr (P::NCLASS == 2) build_dir_lut<P::BD1>(sm.dir1, sm.c_xi[P::NCLASS - 1], tid, NT);
        __syncthreads();
        const float gamma = __uint_as_float(w[0]) * inv_sqrt_dim<D>();
        auto unpack = [&](auto wv_) __attribute__((always_inline)) {
            constexpr int wv = decltype(wv_)::value, EACH = (P::NTRI + NWV - 1) / NWV;
            static_for<wv * EACH, ((wv + 1) * EACH < P::NTRI ? (wv + 1) * EACH : P::NTRI)>([&](auto ii) {
                constexpr int i = decltype(ii)::value, c = P::cls(i);
                const float4 n = (c ? sm.dir1 : sm.dir0)[field<P::dir_bit(i), 2 * P::bdir(i)>(w)];
                const float rho = gamma * sm.c_rho[c][field<P::nrm_bit(i), P::bnrm(i)>(w)];
                sm.u[3 * i][lane] = rho * n.x;
                sm.u[3 * i + 1][lane] = rho * n.y;
                sm.u[3 * i + 2][lane] = rho * n.z;
            });
        };
        static_for<0, NWV>([&](auto wv_) {
            if (wave == decltype(wv_)::value) unpack(wv_);
        });
        __syncthreads();
        constexpr int R = D / 8;
        for (int low = wave; low < 8; low += NWV) {
            float x[R];
#pragma unroll
            for (int e = 0; e < R; ++e) x[e] = sm.u[e * 8 + low][lane];
            butterflies<R>(x);
#pragma unroll
            for (int e = 0; e < R; ++e) sm.u[e * 8 + low][lane] = x[e];
        }
        __syncthreads();
        const uint32_t sbits = a.signs[kvh * LPR + col / 8];
        for (int key = tid / LPR; key < kWave; key += RPP) {
            const int64_t slot = tile * kWave + key;
            if (slot < lo || slot >= hi) continue;
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = sm.u[col + e][key];
            butterflies<8>(x);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = ((sbits >> e) & 1u) ? -x[e] : x[e];
            store_eight(a.k_out, ((static_cast<int64_t>(seq) * a.n_tok + slot - start) * a.n_kv_heads + kvh) * D + col, a.out_is_bf16, x);
        }
    }
    if (a.v_out != nullptr) {
        constexpr int KEYS = kWave / RPP;        // rows a thread reads eight channels of: all of them asked for, then written
        const int first = static_cast<int>(lo - tile * kWave), last = static_cast<int>(hi - 1 - tile * kWave);
        auto write = [&](int key, const float (&x)[8]) __attribute__((always_inline)) {
            if (key >= first && key <= last)
                store_eight(a.v_out, ((static_cast<int64_t>(seq) * a.n_tok + tile * kWave + key - start) * a.n_kv_heads + kvh) * D + col, a.out_is_bf16, x);
        };
        float x[8];
        if (a.v_bits == 0) {
            uint4 row[KEYS];
#pragma unroll
            for (int i = 0; i < KEYS; ++i) {
                const int key = min(max(tid / LPR + i * RPP, first), last);
                row[i] = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.v_pool) + (slab * kWave + key) * D + col);
            }
#pragma unroll
            for (int i = 0; i < KEYS; ++i) {
                const uint32_t two[4] = {row[i].x, row[i].y, row[i].z, row[i].w};
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = __uint_as_float((e & 1) ? two[e / 2] & 0xffff0000u : two[e / 2] << 16);
                write(tid / LPR + i * RPP, x);
            }
        } else {
            // v^ = zero + scale code: channel j's code at bit v_bits j of the row, scale and zero of its group after the codes (so that
            // four bytes from any code's are the row's)
            typedef uint32_t word_t __attribute__((aligned(1)));
            const int code_bytes = a.v_bits * D / 8, row_bytes = code_bytes + D / a.v_group * 8;
            uint32_t codes[KEYS];
            float2 meta[KEYS];
#pragma unroll
            for (int i = 0; i < KEYS; ++i) {
                const int key = min(max(tid / LPR + i * RPP, first), last);
                const unsigned char *row = static_cast<const unsigned char *>(a.v_pool) + (slab * kWave + key) * row_bytes;
                codes[i] = *reinterpret_cast<const word_t *>(row + col / 8 * a.v_bits);
                meta[i] = *reinterpret_cast<const float2 *>(row + code_bytes + col / a.v_group * 8);
            }
#pragma unroll
            for (int i = 0; i < KEYS; ++i) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[e] = fmaf(meta[i].x, static_cast<float>((codes[i] >> (a.v_bits * e)) & ((1u << a.v_bits) - 1u)), meta[i].y);
                write(tid / LPR + i * RPP, x);
            }
        }
    }
}

template <class P>
int launch_read_plan(const octopus_codebooks_t &cb, const ReadCall &a, hipStream_t stream) {
    const int tiles = (a.n_tok + kWave - 1) / kWave + (a.start_pos ? 1 : 0);
    hipLaunchKernelGGL(read_tokens_kernel<P>, dim3(tiles, a.n_kv_heads, a.n_seq), dim3(read_waves(P::D) * 64), 0, stream, device_books(cb), a);
    return static_cast<int>(hipGetLastError());
}

}  // namespace octopus

#endif

// Says how the library's host side divides calls of octopus_attn_decode_paged_prefix, without a GPU: the launchers are stubs that keep
// the shape they are handed.  Arguments, eight per call: head_dim, bits per coordinate, n_seq, n_q_heads, n_kv_heads, n_q, max_prefix,
// max_len; one line per call: rows per group, wavefronts, prefix groups, prefix splits, own groups, own splits, prefix segments,
// segments, first own partial result, partial results the workspace has room for.
// Built by tests/test_serve_host.py from this file plus csrc/octopus_host.cpp and csrc/octopus_serve_host.cpp.
#include <cstdio>
#include <cstdlib>

#include "octopus_internal.h"

namespace octopus {
static PrefixShape g_shape;
static int64_t g_room;
int launch_prefix(const octopus_codebooks_t &, const PrefixShape &s, const void *, const void *, const int32_t *, const int32_t *,
                  const int32_t *, const int32_t *, const int32_t *, float *, float *, void *) { return s.n_segments > 0 ? 0 : 1; }
int launch_prefix_merge(const octopus_plan_t &, const PrefixShape &s, const int32_t *, const int32_t *, const int32_t *, const float *part_ml,
                        const float *part_acc, float *, void *) {
    g_shape = s;
    g_room = (reinterpret_cast<const char *>(part_acc) - reinterpret_cast<const char *>(part_ml)) / 8;
    return 0;
}
int launch_append(const octopus_codebooks_t &, const AppendCall &, void *) { return 0; }
int launch_append_values(const AppendCall &, int32_t, int32_t, int32_t, void *, void *) { return 0; }
int launch_read(const octopus_codebooks_t &, const ReadCall &, void *) { return 0; }

int launch_rotate_queries(const octopus_plan_t &, const void *, int, const uint8_t *, const DecodeShape &, float, float *,
                          const int32_t *, int32_t *, const uint8_t *, float *, void *) { return 0; }
int launch_decode(const octopus_codebooks_t &, const DecodeShape &, const float *, const void *, const void *, int,
                  const int32_t *, float *, float *, float *, int32_t *, void *) { return 0; }
int launch_decode_paged(const octopus_codebooks_t &, const DecodeShape &, const float *, const void *, const void *,
                        const PageTable &, const int32_t *, float *, float *, int32_t *, void *) { return 0; }
int launch_decode_qjl(const octopus_codebooks_t &, const DecodeShape &, const float *, const void *, const void *,
                      const float *, const void *, const int32_t *, float *, float *, float *, int32_t *, void *) { return 0; }
int launch_decode_paged_qjl(const octopus_codebooks_t &, const DecodeShape &, const float *, const void *, const void *,
                            const float *, const void *, const PageTable &, const int32_t *, float *, float *, int32_t *, void *) { return 0; }
int launch_decode_vq(const octopus_codebooks_t &, const DecodeShape &, const float *, const void *, const void *, int,
                     int, const int32_t *, float *, float *, float *, int32_t *, void *, PageTable) { return 0; }
int launch_merge(const octopus_plan_t &, const DecodeShape &, const float *, const float *, const int32_t *, float *, void *) { return 0; }
int launch_encode(const octopus_codebooks_t &, const void *, int, int64_t, int64_t, int64_t, int32_t, int32_t, int32_t,
                  const uint8_t *, void *, int64_t, const int32_t *, const uint8_t *, void *, void *) { return 0; }
int launch_encode_paged(const octopus_codebooks_t &, const void *, int, int64_t, int64_t, int64_t, int32_t, int32_t,
                        int32_t, const uint8_t *, void *, const PageTable &, const int32_t *, void *, const uint8_t *, void *) { return 0; }
int launch_encode_rounding(const octopus_codebooks_t &, const void *, int, int64_t, int64_t, int64_t, int32_t, int32_t,
                           int32_t, const uint8_t *, void *, int64_t, const int32_t *, int32_t, void *) { return 0; }
int launch_encode_values(const void *, int, int64_t, int64_t, int64_t, int32_t, int32_t, int32_t, int32_t, int32_t,
                         int32_t, void *, int64_t, const int32_t *, void *, PageTable) { return 0; }
int launch_probe_read(const void *, int64_t, int, int, void *, void *) { return 0; }
int record_event(void *, void *) { return 0; }
bool plan_supported(const octopus_plan_t &) { return true; }
bool plan_sweep_only(const octopus_plan_t &) { return false; }
int qjl_rows_cap(const octopus_plan_t &) { return 8; }
int vq_mfma_available(const octopus_plan_t &, int32_t, int32_t, int32_t) { return 0; }
}  // namespace octopus

int main(int argc, char **argv) {
    alignas(256) static unsigned char fake[256];    // satisfies the alignment checks; the stubs never look behind it
    const int32_t *ip = reinterpret_cast<const int32_t *>(fake);
    for (int a = 1; a + 7 < argc; a += 8) {
        octopus_codebooks_t cb;
        const int d = std::atoi(argv[a]), n_seq = std::atoi(argv[a + 2]), n_qh = std::atoi(argv[a + 3]), n_kv = std::atoi(argv[a + 4]);
        const int n_q = std::atoi(argv[a + 5]);
        const int64_t max_prefix = std::atoll(argv[a + 6]), max_len = std::atoll(argv[a + 7]);
        if (octopus_build_codebooks(d, std::atof(argv[a + 1]), &cb) != OCTOPUS_OK) return 2;
        const size_t bytes = octopus_attn_prefix_workspace(&cb, n_seq, n_qh, n_kv, n_q, max_prefix, max_len);
        const int rc = octopus_attn_decode_paged_prefix(&cb, fake, OCTOPUS_DTYPE_BF16, n_seq, n_qh, n_kv, n_q, nullptr, 0, fake, fake, fake, 1, ip,
                                                        static_cast<int32_t>((max_prefix + 63) / 64), ip, max_prefix, ip,
                                                        static_cast<int32_t>((max_len + 63) / 64), ip, max_len, 1.0f,
                                                        reinterpret_cast<float *>(fake), fake, bytes, nullptr);
        if (rc != OCTOPUS_OK) {
            std::printf("error %d\n", rc);
            continue;
        }
        const octopus::PrefixShape &s = octopus::g_shape;
        // of the workspace's bytes the partial results' rows take what (maximum, sum) pairs and the slack leave
        const int64_t rows = (static_cast<int64_t>(bytes) - 256 - octopus::g_room * 8) / (d * 4);
        std::printf("%d %d %d %d %d %d %d %d %lld %lld\n", octopus::prefix_rows(d), octopus::prefix_waves(d), s.prefix_groups, s.prefix_splits,
                    s.own_groups, s.own_splits, s.prefix_segments, s.n_segments, static_cast<long long>(s.own_partials),
                    static_cast<long long>(rows < octopus::g_room ? rows : octopus::g_room));
    }
    return 0;
}

// Host side of octopus_verify_drafts: checks of arguments, division of the rows, launches.
#include <algorithm>

#include "octopus_internal.h"

namespace octopus {
namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

bool shape_ok(int32_t n_seq, int32_t n_draft, int32_t vocab) {
    return n_seq >= 1 && n_seq <= 65535 && n_draft >= 0 && n_draft <= (1 << 20) && vocab >= 1 && vocab <= (1 << 30);
}

}  // namespace
}  // namespace octopus

using namespace octopus;

extern "C" {

size_t octopus_verify_workspace(int32_t n_seq, int32_t n_draft, int32_t vocab) {
    return shape_ok(n_seq, n_draft, vocab) ? static_cast<size_t>(n_seq) * kMostPieces * sizeof(RowSums) : 0;
}

int octopus_verify_drafts(const void *target, int32_t dtype, int64_t target_stride_seq, int64_t target_stride_pos, const void *draft,
                          int64_t draft_stride_seq, int64_t draft_stride_pos, const int32_t *draft_tokens, const int32_t *draft_lens,
                          const float *uniforms, int32_t n_seq, int32_t n_draft, int32_t vocab, int32_t *tokens_out, int32_t *n_accepted,
                          void *workspace, size_t workspace_bytes, void *stream) {
    if (target == nullptr || uniforms == nullptr || tokens_out == nullptr || n_accepted == nullptr || !shape_ok(n_seq, n_draft, vocab)) return OCTOPUS_EINVAL;
    if (n_draft > 0 && draft_tokens == nullptr) return OCTOPUS_EINVAL;
    if (dtype != OCTOPUS_DTYPE_F32 && dtype != OCTOPUS_DTYPE_BF16) return OCTOPUS_EUNSUPPORTED;
    const size_t word = dtype == OCTOPUS_DTYPE_BF16 ? 2 : 4;
    if (target_stride_seq < 0 || target_stride_pos < 0 || (draft != nullptr && (draft_stride_seq < 0 || draft_stride_pos < 0))) return OCTOPUS_EINVAL;
    if (!aligned(target, word) || !aligned(draft, word) || !aligned(draft_tokens, 4) || !aligned(draft_lens, 4) || !aligned(uniforms, 4) ||
        !aligned(tokens_out, 4) || !aligned(n_accepted, 4))
        return OCTOPUS_EINVAL;
    if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < octopus_verify_workspace(n_seq, n_draft, vocab)) return OCTOPUS_EWORKSPACE;
    VerifyCall c{};
    c.target = target;
    c.target_seq = target_stride_seq;
    c.target_pos = target_stride_pos;
    c.draft = draft;
    c.draft_seq = draft_stride_seq;
    c.draft_pos = draft_stride_pos;
    c.tokens = draft_tokens;
    c.draft_lens = draft_lens;
    c.uniforms = uniforms;
    c.tokens_out = tokens_out;
    c.accepted = n_accepted;
    c.sums = static_cast<RowSums *>(workspace);
    c.n_seq = n_seq;
    c.n_draft = n_draft;
    c.vocab = vocab;
    c.is_bf16 = dtype == OCTOPUS_DTYPE_BF16;
    return launch_verify(c, stream) == 0 ? OCTOPUS_OK : OCTOPUS_EHIP;
}

}  // extern "C"

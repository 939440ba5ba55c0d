// Host side of the beam selection: argument checks and launches.
#include "fnpu_internal.h"

namespace fnpu {
namespace {

int shape_ok(const fnpu_beam_desc *d) {
    if (!d || d->num_groups < 0 || d->num_beams < 1 || d->vocab < 1 || d->num_select < 1) return FNPU_EINVAL;
    if ((d->dtype != FNPU_LOGITS_BF16 && d->dtype != FNPU_LOGITS_FP32) || d->end_token < -1 || d->end_token >= d->vocab) return FNPU_EINVAL;
    if (d->num_beams > 128 || d->num_select > 64 || d->vocab > (1 << 24)) return FNPU_EUNSUPPORTED;
    // (the grid and each row's parent are 32-bit)
    return static_cast<int64_t>(d->num_groups) * d->num_beams * beam_slices(d) > INT32_MAX ? FNPU_EUNSUPPORTED : FNPU_OK;
}

// Bytes of the slices' parts (8 each), then of their lists.
int64_t parts_bytes(const fnpu_beam_desc *d, int slices) {
    return (static_cast<int64_t>(d->num_groups) * d->num_beams * slices * 8 + 15) / 16 * 16;
}
int64_t workspace_bytes_of(const fnpu_beam_desc *d) {
    const int slices = beam_slices(d);
    return parts_bytes(d, slices) + static_cast<int64_t>(d->num_groups) * d->num_beams * slices * d->num_select * 8;
}

}  // namespace
}  // namespace fnpu

using namespace fnpu;

extern "C" {

int fnpu_beam_select_workspace(const fnpu_beam_desc *desc, int64_t *bytes) {
    if (!bytes) return FNPU_EINVAL;
    const int rc = shape_ok(desc);
    if (rc == FNPU_OK) *bytes = workspace_bytes_of(desc);
    return rc;
}

int fnpu_beam_select(const fnpu_beam_desc *desc, const void *logits, int64_t row_stride, const float *scores, const uint8_t *finished,
                     float *out_scores, int32_t *out_parents, int32_t *out_tokens, void *workspace, int64_t workspace_bytes,
                     void *stream) {
    const int rc = shape_ok(desc);
    if (rc != FNPU_OK) return rc;
    if (desc->num_groups == 0) return FNPU_OK;
    const bool fp32 = desc->dtype == FNPU_LOGITS_FP32;
    if (!logits || !scores || !out_scores || !out_parents || !out_tokens || !workspace || row_stride < desc->vocab) return FNPU_EINVAL;
    if ((reinterpret_cast<uintptr_t>(logits) & (fp32 ? 3u : 1u)) ||
        ((reinterpret_cast<uintptr_t>(scores) | reinterpret_cast<uintptr_t>(out_scores) | reinterpret_cast<uintptr_t>(out_parents) |
          reinterpret_cast<uintptr_t>(out_tokens)) & 3u) ||
        (reinterpret_cast<uintptr_t>(workspace) & 15u))
        return FNPU_EINVAL;
    if (workspace_bytes < workspace_bytes_of(desc)) return FNPU_EINVAL;
    BeamArgs a = {};
    a.slices = beam_slices(desc);
    a.logits = logits;
    a.stride = row_stride;
    a.scores = scores;
    a.finished = finished;
    a.parts = static_cast<float2 *>(workspace);
    a.keys = reinterpret_cast<uint64_t *>(static_cast<uint8_t *>(workspace) + parts_bytes(desc, a.slices));
    a.out_scores = out_scores;
    a.out_parents = out_parents;
    a.out_tokens = out_tokens;
    a.groups = desc->num_groups;
    a.beams = desc->num_beams;
    a.vocab = desc->vocab;
    a.select = desc->num_select;
    a.end_token = desc->end_token;
    return launch_beam_select(a, fp32, stream);
}

}  // extern "C"

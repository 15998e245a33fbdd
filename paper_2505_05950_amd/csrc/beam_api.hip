// C entry points of the beam search's selection (declared in include/floe.h): argument checks, workspace, launches.
#include "beam.h"
#include "host_call.h"

using namespace floe;

namespace {

int check_beam(const floe_beam* b) {
    if (!b || b->groups < 0 || b->beams <= 0 || b->vocab <= 0 || b->take <= 0 || b->eos < -1 || b->eos >= b->vocab) return FLOE_EINVAL;
    if (b->take > kBeamTake || b->beams > kBeamRows || b->vocab >= (1 << 28) || (int64_t)b->groups * b->beams > (1 << 20)) return FLOE_EUNSUPPORTED;
    if (b->dtype != FLOE_FP16 && b->dtype != FLOE_BF16 && b->dtype != FLOE_FP32) return FLOE_EUNSUPPORTED;
    const BeamCut cut = beam_cut(b->groups * b->beams, b->vocab, b->dtype);
    return (int64_t)b->groups * b->beams * cut.slices > kMaxGrid ? FLOE_EUNSUPPORTED : FLOE_OK;
}
struct BeamWs {
    size_t best, total;
};
BeamWs beam_ws(const floe_beam* b, const BeamCut& cut) {
    const size_t lists = (size_t)b->groups * b->beams * cut.slices;
    BeamWs w;
    w.best = align_up(lists * sizeof(BeamSum));
    w.total = w.best + align_up(lists * b->take * 8);
    return w;
}

}  // namespace

extern "C" {

size_t floe_beam_workspace_bytes(const floe_beam* b) {
    return check_beam(b) == FLOE_OK && b->groups ? beam_ws(b, beam_cut(b->groups * b->beams, b->vocab, b->dtype)).total : 0;
}

int floe_beam_select(const floe_beam* b, const void* logits, int64_t row_stride, const float* score, const uint8_t* done, float* score_out,
                     int32_t* parent, int32_t* token, uint8_t* done_out, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_beam(b);
    if (rc) return rc;
    if (row_stride < b->vocab || (done && b->eos < 0)) return FLOE_EINVAL;
    if (row_stride > (int64_t)1 << 40) return FLOE_EUNSUPPORTED;
    if (b->groups == 0) return FLOE_OK;
    if (!logits || !score || !score_out || !parent || !token || !workspace) return FLOE_EINVAL;
    if (!aligned(logits, b->dtype == FLOE_FP32 ? 4 : 2) || !aligned(score, 4) || !aligned(score_out, 4) || !aligned(parent, 4) || !aligned(token, 4) ||
        !aligned(workspace, kAlign))
        return FLOE_EINVAL;
    const BeamCut cut = beam_cut(b->groups * b->beams, b->vocab, b->dtype);
    const BeamWs w = beam_ws(b, cut);
    if (workspace_bytes < w.total) return FLOE_EWORKSPACE;
    char* base = static_cast<char*>(workspace);
    const BeamArgs a{logits, row_stride, score, done, b->groups, b->beams, b->vocab, b->take, b->eos, cut.slices, cut.slice, score_out, parent, token,
                     done_out, reinterpret_cast<BeamSum*>(base), reinterpret_cast<uint64_t*>(base + w.best)};
    hipStream_t st = (hipStream_t)stream;
    FLOE_LAUNCH(FLOE_KERNEL_BEAM_ROWS, st, launch_beam_rows(a, b->dtype, cut.loads, st));
    FLOE_LAUNCH(FLOE_KERNEL_BEAM_GROUPS, st, launch_beam_groups(a, st));
    return FLOE_OK;
}

}  // extern "C"

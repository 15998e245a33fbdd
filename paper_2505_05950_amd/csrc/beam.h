// Beam search's selection (include/floe.h): what its two kernels share, and their launcher.  Arguments are checked in beam_api.hip.
#pragma once

#include "kv_cache.h"
#include "launch.h"

namespace floe {

constexpr int kBeamTake = 64;       // candidates of a group, at most: a lane each
constexpr int kBeamThreads = 256, kBeamWaves = kBeamThreads / kWave;
constexpr int kBeamRows = 256;      // rows of a group, at most

// What the groups' kernel gets to know of a slice and its row: it reads no input, so a group's results may lie over those of other groups.
struct BeamSum {
    float top;    // the largest logit
    float score;  // of the row
    double sum;   // of exp(x - top); kBeamDone of a row that is done
};
constexpr double kBeamDone = -1.0;
struct BeamArgs {
    const void* logits;
    int64_t stride;
    const float* score;
    const uint8_t* done;
    int groups, beams, vocab, take, eos;
    int slices, slice;  // of a row, and the tokens of one
    float* score_out;
    int32_t *parent, *token;
    uint8_t* done_out;
    // [rows][slices]; [rows][slices][take]: the best tokens, in no order, 0 where there are fewer
    BeamSum* sums;
    uint64_t* best;
};

struct BeamCut {
    int slices, slice, loads;  // loads: of sixteen bytes per lane and tile
};
BeamCut beam_cut(int rows, int vocab, int dtype);  // dtype: floe_dtype
hipError_t launch_beam_rows(const BeamArgs& a, int dtype, int loads, hipStream_t st);
hipError_t launch_beam_groups(const BeamArgs& a, hipStream_t st);

}  // namespace floe

// What the library's translation units share on the host: the record of a failed HIP call, per-kernel timing, the check of an
// encoding's configuration.  Defined in cngp_api.hip.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/cngp.h"

namespace cngp {

enum KernelId { K_FWD = 0, K_BWD_DIRECT, K_BWD_PREP, K_BWD_SLICED, K_BWD_SLICED_V, K_BWD_GRID_DRAIN,
                K_BAKE, K_ZERO, K_DEBUG, K_ADAM, K_MLP_FWD, K_MLP_BWD,
                K_BWD_BIN_OFFSETS, K_BWD_BIN_SCATTER, K_BWD_BIN_DRAIN, K_BWD_INPUT, K_FUSED_FWD, K_PLANES, K_FWD_ROWS, K_BWD_SMALL, K_BWD_CELLS, K_BWD_MERGE, K_BWD_PARTIAL,
                K_RECUR_FWD, K_RECUR_BWD, K_RECUR_CARRY, K_EMBED_FWD, K_EMBED_SORT, K_EMBED_SUMS, K_BALANCE,
                K_ATTEND_WALK, K_ATTEND_STATES, K_ATTEND_STEP, K_ATTEND_DECAY, K_ROTATE, K_ROTATE_BWD, K_ORTHO, K_ORTHO_PRODUCT, K_COUNT };

// A launch has less than 2^32 work-items: workgroups of 256 lanes that fit.
constexpr int64_t kMostGroups256 = 0xffffff;

int record_hip_failure(hipError_t e, const char *what);
int launch_status(const char *what);              // of the launch just made
int validate(const cngp_config *c);

struct LaunchTimer {
    hipStream_t s; int id; hipEvent_t t0 = nullptr, t1 = nullptr; bool on;
    LaunchTimer(hipStream_t s_, int id_);
    ~LaunchTimer();
};

}  // namespace cngp

// Linear attention with decays: the walks of fp32 storage.
#include "cngp_attend_walk.h"

int cngp::attend_walk_f32(const WalkArgs &a, bool states_only, hipStream_t s) { return attend::launch_tiles<float>(a, states_only, s); }

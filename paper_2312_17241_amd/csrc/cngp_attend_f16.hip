// Linear attention with decays: the walks of fp16 storage.
#include "cngp_attend_walk.h"

int cngp::attend_walk_f16(const WalkArgs &a, bool states_only, hipStream_t s) { return attend::launch_tiles<_Float16>(a, states_only, s); }

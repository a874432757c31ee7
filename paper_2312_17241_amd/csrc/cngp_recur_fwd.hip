// The forward launches of the gated linear recurrence.
#include "cngp_recur_scan.h"

template int cngp::recur_launch<false>(const cngp_recur_config *, cngp::RecurArgs, const cngp::RecurPlan &, const cngp::RecurSpace &, char *, hipStream_t);

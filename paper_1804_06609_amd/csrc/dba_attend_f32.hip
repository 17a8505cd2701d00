// libdba: attention over a paged cache, f32.
#include "tree_attend_launch.hpp"

template hipError_t dba::attend_launch<0>(const AttendParams &, const AttendPlan &, int, hipStream_t);
template hipError_t dba::shared_launch<0>(const SharedParams &, const AttendPlan &, const AttendPlan &, int, hipStream_t);

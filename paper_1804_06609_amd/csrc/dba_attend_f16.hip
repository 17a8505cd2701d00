// libdba: attention over a paged cache, f16.
#include "tree_attend_launch.hpp"

template hipError_t dba::attend_launch<1>(const AttendParams &, const AttendPlan &, int, hipStream_t);

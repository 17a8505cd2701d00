// libdba: attention over a paged cache, bf16.
#include "tree_attend_launch.hpp"

template hipError_t dba::attend_launch<2>(const AttendParams &, const AttendPlan &, int, hipStream_t);

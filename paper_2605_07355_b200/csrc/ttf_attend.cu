// Which kernel attends.
#include "ttf_paged.cuh"

namespace ttf {

cudaError_t launch_attend(const AttendArgs& a, int dtype, cudaStream_t st) {
    if (attend_tc_takes(a, dtype)) return launch_attend_tc(a, st);
    return launch_attend_simple(a, dtype, st);
}

}  // namespace ttf

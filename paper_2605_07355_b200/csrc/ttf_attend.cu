// Which kernel attends.
#include "ttf_paged.cuh"

namespace ttf {

cudaError_t launch_attend(const AttendArgs& a, int dtype, cudaStream_t st) {
    const bool few = (long long)a.seq.rows * a.group <= 32LL * a.seq.seqs;
    if (!few && attend_tc_takes(a, dtype)) return launch_attend_tc(a, st);
    if (attend_few_takes(a, dtype)) return launch_attend_few(a, st);
    if (attend_mma_takes(a, dtype)) return launch_attend_mma(a, st);
    return launch_attend_simple(a, dtype, st);
}

}  // namespace ttf

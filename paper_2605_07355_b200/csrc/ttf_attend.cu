// Which kernel attends.
#include "ttf_paged.cuh"

namespace ttf {

cudaError_t launch_attend(const AttendArgs& a, int dtype, cudaStream_t st) {
    // Few: at most 32 packed rows a sequence on the average.  Each, over 3000 slots, 8 heads of 128 (few / many rows' kernel):
    //   bf16, 16 sequences: 42.6 / 52.5 us at 16 rows, 49.5 / 52.7 at 32, 53.7 / 52.9 at 48, 140 / 53 at 128
    //   bf16, one sequence: 12.7 / 19.2 us at 32 rows, 15.7 / 19.3 at 64, 20.9 / 19.3 at 128 (one long sequence among short ones
    //   would pay more for a higher bound than this gains)
    //   fp32, 16 sequences: 391 / 473 us at 32 rows, 519 / 487 at 48
    // One kernel takes the whole call: 63 sequences of 2001 slots with one row and a prompt of 2048 rows, 194 us, are 97 and 49 apart.
    const bool few = (long long)a.seq.rows * a.group <= 32LL * a.seq.seqs;
    if (!few && attend_tc_takes(a, dtype)) return launch_attend_tc(a, st);
    if (attend_f32_takes(a, dtype)) return few ? launch_attend_few32(a, st) : launch_attend_f32(a, st);
    if (attend_few_takes(a, dtype)) return launch_attend_few(a, st);
    if (attend_mma_takes(a, dtype)) return launch_attend_mma(a, st);
    return launch_attend_simple(a, dtype, st);
}

}  // namespace ttf

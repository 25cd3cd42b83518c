// Attention of few new rows over a paged cache, fp32: decoding and a few tokens at a time.  Bound by the bytes of the cache as long
// as the fp32 pipes and the exchanges between lanes keep up.
//
//   t_s = scale log2(e) <q, k_s>,   o = sum_s exp2(t_s - m) v_s / sum_s exp2(t_s - m)
//
// A CTA takes 8 packed rows (tokens x query heads of a group) of one sequence and key head.  Its four warps take the blocks of 16
// slots in turn.  Lanes hold the channels (four in a row each, so that a key or value is read as whole lines): four slots times
// eight rows are 32 partial dot products per lane, which a butterfly of 31 exchanges turns into one finished score per lane; the
// weights go back to all lanes by a shuffle each.  A lane reads what it has fetched itself, so the ring needs no barrier.
// A block's products are summed apart from the running sums: a single chain would lose digits over thousands of slots.
// m only moves when a score exceeds it by more than 8 (in powers of two); warps and the CTAs of a cluster join their sums through
// shared memory (ttf_attend_few.cuh).
//
// Bound by the latency of a group of four slots (650 instructions in one warp, 2800 cycles) times the 12 warps that fit an SM:
// 32 sequences of 500 to 12000 slots, 8 heads of 128, groups of 4, take 326 us (2.7 TB/s) against 1837 us with 32 rows per CTA;
// with keys and values fetched into registers 624, with two CTAs and four groups in the ring per SM 381.
//
// Slots that no row of the tile sees are not read.
#include "ttf_attend_few.cuh"

namespace ttf {

constexpr int kF32Rows = 8, kF32Slots = 16, kF32Groups = kF32Slots / 4;

template <int VN> struct F32Ring {
    static constexpr int DEPTH = 3;                        // groups of four slots, keys and values
    static constexpr int GROUP = 2 * 4 * 128 * VN;         // floats
    static constexpr int WARP = DEPTH * GROUP;
};

template <int VN>                                          // groups of 128 channels
__global__ void __launch_bounds__(kMmaThreads, VN == 1 ? 3 : 1)
k_attend_few32(const __grid_constant__ AttendArgs a, int lsplit)
{
    constexpr int DP = 128 * VN;
    __shared__ JoinSpace<DP> jn;
    __shared__ __align__(16) float s_q[kF32Rows][DP];
    extern __shared__ __align__(16) float f32_smem[];      // the warps' rings; then [warp][row][DP + 4]: their weighted values
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int D = a.cache.dim;
    const int rank = lsplit ? (int)cluster_rank() : 0;
    const int work = blockIdx.x >> lsplit, hk = work % a.cache.heads;

    pdl_wait();
    Tile t;
    // (every CTA of a cluster has the same tile, and so the same answer)
    if (!find_tile(a, Cut{Divisor{0, 0, 0}, 3}, work / a.cache.heads, blockIdx.x == 0, t)) return;
    if (lsplit) cluster_arrive();                          // (waited for before anything is sent to another rank)
    const SeqRange r = t.r;
    const int* const table = a.seq.table + (long long)t.seq * a.seq.table_stride;
    const int row0 = t.tile * kF32Rows;
    const long long packed = (long long)r.n * a.group;
    const int nrow = packed - row0 < kF32Rows ? (int)(packed - row0) : kF32Rows;

    // this rank's blocks; this warp's are j_lo + warp, j_lo + warp + 4, ...
    const int tok_a = row0 / a.group, tok_z = (row0 + nrow - 1) / a.group;
    const int lo = seen_by(r, tok_a, a.causal, a.window).lo, hi = seen_by(r, tok_z, a.causal, a.window).hi;    // seen by some row
    const int b_lo = lo / kF32Slots, b_hi = hi > lo ? (hi + kF32Slots - 1) / kF32Slots : b_lo;
    const int j_lo = b_lo + (int)((long long)(b_hi - b_lo) * rank >> lsplit);
    const int j_hi = b_lo + (int)((long long)(b_hi - b_lo) * (rank + 1) >> lsplit);

    // queries, with the scale in them; rows that are not there are zeros
    for (int e = tid; e < kF32Rows * (DP / 4); e += kMmaThreads) {
        const int row = e / (DP / 4), d = (e - row * (DP / 4)) * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row < nrow && d < D) {
            const int token = (row0 + row) / a.group, head = hk * a.group + (row0 + row) - token * a.group;
            v = __ldcg(reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.q.data) + (long long)(r.first + token) * a.q.row + (long long)head * a.q.head + d));
        }
        const float c = a.scale * 1.4426950408889634f;
        *reinterpret_cast<float4*>(&s_q[row][d]) = make_float4(v.x * c, v.y * c, v.z * c, v.w * c);
    }
    __syncthreads();

    const int my_row = lane & 7;                           // of the finished scores: slot lane / 8 of four, row lane % 8
    const Seen mine = my_row < nrow ? seen_by(r, (row0 + my_row) / a.group, a.causal, a.window) : Seen{0, 0};
    float m = -INFINITY, l = 0.f;
    float4 acc[kF32Rows][VN];
#pragma unroll
    for (int i = 0; i < kF32Rows; ++i)
#pragma unroll
        for (int v = 0; v < VN; ++v) acc[i][v] = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* const kb = reinterpret_cast<const float*>(a.cache.k) + (long long)hk * a.cache.k_head;
    const float* const vb = reinterpret_cast<const float*>(a.cache.v) + (long long)hk * a.cache.v_head;
    bool bad = false;

    // Four slots' keys and values make a group; a lane fetches what it will read itself, so a wait for its own copies is enough.
    float* const ring = f32_smem + warp * F32Ring<VN>::WARP + 4 * lane;
    constexpr int DEPTH = F32Ring<VN>::DEPTH;
    int pg = 0, in = 0;                                    // lane i: page (as the table has it) and row of slot i of the block after
    auto look_up = [&](int j) {
        const int s = j * kF32Slots + lane;
        pg = 0; in = 0;
        if (lane < kF32Slots && j < j_hi && s >= lo && s < hi) {
            const int index = quotient(s, a.cache.page);
            pg = __ldcg(table + index);
            in = s - index * (int)a.cache.page.d;
        }
    };
    int f_blk = j_lo + warp, f_grp = 0, f_at = 0;          // the next group to fetch, and its place in the ring
    long long k_at = 0, v_at = 0;
    look_up(f_blk);
    auto fetch = [&]() {
        if (f_blk < j_hi) {
            if (f_grp == 0) {
                if ((unsigned)pg >= (unsigned)a.cache.pages) { bad = true; pg = 0; }
                k_at = pg * a.cache.k_page + in * a.cache.k_row; v_at = pg * a.cache.v_page + in * a.cache.v_row;
                look_up(f_blk + kMmaWarps);
            }
            float* const to = ring + f_at * F32Ring<VN>::GROUP;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int s = f_blk * kF32Slots + 4 * f_grp + i;
                const bool on = s >= lo && s < hi;
                const float* const kp = kb + __shfl_sync(0xffffffffu, k_at, 4 * f_grp + i);
                const float* const vp = vb + __shfl_sync(0xffffffffu, v_at, 4 * f_grp + i);
#pragma unroll
                for (int x = 0; x < VN; ++x) {
                    const int d = 128 * x + 4 * lane;
                    const bool read = on && d < D;         // (zeros elsewhere)
                    cp_async16(smem_u32(to + i * DP + 128 * x), read ? kp + d : kb, read ? 16 : 0);
                    cp_async16(smem_u32(to + (4 + i) * DP + 128 * x), read ? vp + d : vb, read ? 16 : 0);
                }
            }
            if (++f_grp == kF32Groups) { f_grp = 0; f_blk += kMmaWarps; }
            f_at = f_at + 1 == DEPTH ? 0 : f_at + 1;
        }
        cp_async_commit();                                 // (empty at the end, so that the count stays)
    };
#pragma unroll
    for (int i = 0; i < DEPTH - 1; ++i) fetch();
    int at = 0;
    for (int j = j_lo + warp; j < j_hi; j += kMmaWarps) {
        const int s0 = j * kF32Slots;
        float4 part[kF32Rows][VN];
#pragma unroll
        for (int i = 0; i < kF32Rows; ++i)
#pragma unroll
            for (int x = 0; x < VN; ++x) part[i][x] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int b = 0; b < kF32Groups; ++b) {
            cp_async_wait<DEPTH - 2>();
            fetch();                                       // (into the place that was read last)
            const float* const from = ring + at * F32Ring<VN>::GROUP;
            at = at + 1 == DEPTH ? 0 : at + 1;
            float4 k[4][VN], v[4][VN];
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
                for (int x = 0; x < VN; ++x) k[y][x] = *reinterpret_cast<const float4*>(from + y * DP + 128 * x);
            float dot[32];                                 // [slot][row]
#pragma unroll
            for (int i = 0; i < kF32Rows; ++i) {
                float4 q[VN];
#pragma unroll
                for (int x = 0; x < VN; ++x) q[x] = *reinterpret_cast<const float4*>(&s_q[i][128 * x + 4 * lane]);
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    float d = q[0].x * k[y][0].x;
                    d = fmaf(q[0].y, k[y][0].y, d); d = fmaf(q[0].z, k[y][0].z, d); d = fmaf(q[0].w, k[y][0].w, d);
                    if (VN > 1) {
                        d = fmaf(q[VN - 1].x, k[y][VN - 1].x, d); d = fmaf(q[VN - 1].y, k[y][VN - 1].y, d);
                        d = fmaf(q[VN - 1].z, k[y][VN - 1].z, d); d = fmaf(q[VN - 1].w, k[y][VN - 1].w, d);
                    }
                    dot[y * kF32Rows + i] = d;
                }
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)               // lane L ends up with the sum of dot[L]
#pragma unroll
                for (int i = 0; i < o; ++i) {
                    const bool up = lane & o;
                    const float keep = up ? dot[i + o] : dot[i], send = up ? dot[i] : dot[i + o];
                    dot[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                }
            const int s = s0 + 4 * b + (lane >> 3);
            const bool on = s >= mine.lo && s < mine.hi;
            const float score = on ? dot[0] : -INFINITY;
            if (__any_sync(0xffffffffu, score > m + 8.f)) {
                float top = fmaxf(score, __shfl_xor_sync(0xffffffffu, score, 8));
                top = fmaxf(fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16)), m);
                const float f = m == top ? 1.f : exp2f(m - top);
                m = top;
                l *= f;
#pragma unroll
                for (int i = 0; i < kF32Rows; ++i) {
                    const float fi = __shfl_sync(0xffffffffu, f, i);
#pragma unroll
                    for (int x = 0; x < VN; ++x) {
                        acc[i][x].x *= fi; acc[i][x].y *= fi; acc[i][x].z *= fi; acc[i][x].w *= fi;
                        part[i][x].x *= fi; part[i][x].y *= fi; part[i][x].z *= fi; part[i][x].w *= fi;
                    }
                }
            }
            const float p = on ? exp2f(score - (m == -INFINITY ? 0.f : m)) : 0.f;
            l += p;
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
                for (int x = 0; x < VN; ++x) v[y][x] = *reinterpret_cast<const float4*>(from + (4 + y) * DP + 128 * x);
            const unsigned seen = __ballot_sync(0xffffffffu, on);
            auto add = [&](int y, int i) {
                const float w = __shfl_sync(0xffffffffu, p, y * kF32Rows + i);
#pragma unroll
                for (int x = 0; x < VN; ++x) {
                    part[i][x].x = fmaf(w, v[y][x].x, part[i][x].x); part[i][x].y = fmaf(w, v[y][x].y, part[i][x].y);
                    part[i][x].z = fmaf(w, v[y][x].z, part[i][x].z); part[i][x].w = fmaf(w, v[y][x].w, part[i][x].w);
                }
            };
            if (seen == 0xffffffffu) {
#pragma unroll
                for (int y = 0; y < 4; ++y)
#pragma unroll
                    for (int i = 0; i < kF32Rows; ++i) add(y, i);
            } else {                                       // rows that are not there, slots that some rows do not see
#pragma unroll
                for (int y = 0; y < 4; ++y)
#pragma unroll
                    for (int i = 0; i < kF32Rows; ++i)
                        if (seen >> (y * kF32Rows + i) & 1) add(y, i);
            }
        }
#pragma unroll
        for (int i = 0; i < kF32Rows; ++i)
#pragma unroll
            for (int x = 0; x < VN; ++x) {
                acc[i][x].x += part[i][x].x; acc[i][x].y += part[i][x].y; acc[i][x].z += part[i][x].z; acc[i][x].w += part[i][x].w;
            }
    }
    pdl_launch_dependents();
    if (bad) report_paged(a.hdr, 2);
    cp_async_wait<0>();
    __syncthreads();                                       // the rings are read; their memory takes the warps' sums

    // ---- join the warps -------------------------------------------------------------------------------------------------
    l += __shfl_xor_sync(0xffffffffu, l, 8);
    l += __shfl_xor_sync(0xffffffffu, l, 16);
    if (lane < kF32Rows) { jn.m[warp][lane] = m; jn.l[warp][lane] = l; }
    if (tid == 0) jn.o = f32_smem;
#pragma unroll
    for (int i = 0; i < kF32Rows; ++i)
#pragma unroll
        for (int x = 0; x < VN; ++x)
            *reinterpret_cast<float4*>(f32_smem + (warp * kMmaRows + i) * JoinSpace<DP>::OP + 128 * x + 4 * lane) = acc[i][x];
    __syncthreads();
    join_rows<DP, float>(a, jn, r, row0, nrow, hk, lsplit, rank);
}

template <int VN> static cudaError_t launch_few32_t(const AttendArgs& a, cudaStream_t st) {
    const void* fn = reinterpret_cast<const void*>(k_attend_few32<VN>);
    const size_t ring = (size_t)kMmaWarps * F32Ring<VN>::WARP * 4, sums = (size_t)kMmaWarps * kMmaRows * JoinSpace<128 * VN>::OP * 4;
    const size_t smem = ring > sums ? ring : sums;
    cudaError_t e = ensure_dynamic_smem(fn, smem);
    if (e != cudaSuccess) return e;
    const long long ctas = most_tiles(a, kF32Rows, 0) * a.cache.heads;
    int ls = few_split(a, ctas);
    if (ls > 3 && !large_cluster_fits(fn, kMmaThreads, smem)) ls = 3;
    if ((ctas << ls) > 0x7fffffffLL) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(ctas << ls)); cfg.blockDim = dim3(kMmaThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1u << ls; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = ls ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, k_attend_few32<VN>, a, ls);
}
cudaError_t launch_attend_few32(const AttendArgs& a, cudaStream_t st) {
    return a.cache.dim <= 128 ? launch_few32_t<1>(a, st) : launch_few32_t<2>(a, st);
}

}  // namespace ttf

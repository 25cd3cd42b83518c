// Attention of few new rows over a paged cache, bf16: decoding, a few tokens at a time, and heads or pages that the tcgen05
// kernel does not take.  Bound by the bytes of the cache.
//
//   S = Q K^T,  t = scale log2(e) S,  P = exp2(t - m),  O += P V,  l += sum P,  o = O / l
//
// A CTA takes 16 packed rows (tokens x query heads of a group) of one sequence and key head: the 16 rows of an m16n8k16 MMA.
// Its four warps take the blocks of 16 slots in turn, each on its own: a lane fetches with cp.async exactly the 16-byte pieces
// whose elements it feeds to the MMAs, into slots of shared memory that no other lane touches, so that there is no barrier in
// the loop and everything but the present block is in flight (two stages of 8 KB per warp at 128 channels, three CTAs per SM:
// 190 KB, where 45 KB cover the latency of memory).  64 sequences of 500 to 16000 slots, 8 heads of 128: 270 us, 4.2 TB/s; the
// load unit bounds it (the form with TMA tiles, ttf_attend_few.cu, takes 186, but only pages of whole blocks and heads up to 128).
//   K: the sum over channels does not care for their order.  Lane (g, c) = (lane / 4, lane % 4) holds channels 32 b + 8 c .. + 7 of
//      slots g and g + 8; their four pairs are the operand registers of two MMAs over the 32 channels of b, with Q's
//      fragments cut the same way.
//   V: the columns of O may come in any order too.  The lane holds channels 64 h + 8 g .. + 7 of slots 2c, 2c + 1, 2c + 8, 2c + 9;
//      a byte permutation of two slots' registers is the operand of the columns 64 h + 8 n + j, n = 0 .. 7, and the accumulators
//      of a lane end up as 16 consecutive channels.
// m only moves when a score exceeds it by more than 8 (in powers of two), so that a block usually needs no exchange between lanes;
// sums are kept per lane until the end.
// Warps and the CTAs of a cluster, which share the slots of long sequences, join their sums through shared memory.
//
// P is rounded to bf16 for the second product, l adds up the weights before that (as in ttf_attend_tc.cu, with the same error).
//
// Slots that no row of the tile sees are fetched as zeros, whatever the page holds there.
#include "ttf_paged.cuh"
#include "ttf_attend_few.cuh"

namespace ttf {

template <int DC> struct MmaShape {                        // DC: 32-channel pieces of a head (even)
    static constexpr int D = DC * 32;
    static constexpr int PIECES = 4 * DC;                  // 16-byte pieces of a lane in a stage: 2 slots x DC of K, 4 x DC / 2 of V
    static constexpr int STAGE = PIECES * 32 * 16;
    static constexpr int STAGES = DC <= 4 ? 2 : 3;
    static constexpr int SMEM = kMmaWarps * STAGES * STAGE;
    static constexpr int OP = D + 4;                       // floats of a row that warps exchange
};

__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

template <int DC, bool PAGE16, bool FULL>
__global__ void __launch_bounds__(kMmaThreads, DC <= 2 ? 4 : (DC <= 4 ? 3 : 1))
k_attend_mma(const __grid_constant__ AttendArgs a, int lsplit)
{
    using S = MmaShape<DC>;
    constexpr int HC = DC / 2;                             // 64-channel pieces
    extern __shared__ __align__(128) unsigned char mma_smem[];
    __shared__ JoinSpace<S::D> jn;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const int D = a.cache.dim;
    const int rank = lsplit ? (int)cluster_rank() : 0;
    const int work = blockIdx.x >> lsplit, hk = work % a.cache.heads;

    pdl_wait();
    Tile t;
    // (every CTA of a cluster has the same tile, and so the same answer)
    if (!find_tile(a, Cut{Divisor{0, 0, 0}, 4}, work / a.cache.heads, blockIdx.x == 0, t)) return;
    if (lsplit) cluster_arrive();                          // (waited for before anything is sent to another rank)
    const SeqRange r = t.r;
    const int* const table = a.seq.table + (long long)t.seq * a.seq.table_stride;
    const int row0 = t.tile * kMmaRows;
    const long long packed = (long long)r.n * a.group;
    const int nrow = packed - row0 < kMmaRows ? (int)(packed - row0) : kMmaRows;

    // this rank's blocks; this warp's are j_lo + warp, j_lo + warp + 4, ...
    const int tok_a = row0 / a.group, tok_z = (row0 + nrow - 1) / a.group;
    const Seen sa = seen_by(r, tok_a, a.causal, a.window), sz = seen_by(r, tok_z, a.causal, a.window);
    const int lo = sa.lo, hi = sz.hi;                      // seen by some row
    const int b_lo = lo / kMmaSlots, b_hi = hi > lo ? (hi + kMmaSlots - 1) / kMmaSlots : b_lo;
    const int j_lo = b_lo + (int)((long long)(b_hi - b_lo) * rank >> lsplit);
    const int j_hi = b_lo + (int)((long long)(b_hi - b_lo) * (rank + 1) >> lsplit);
    const int all_lo = sz.lo, all_hi = sa.hi;              // seen by every row

    const uint32_t ring = smem_u32(mma_smem) + (uint32_t)(warp * S::STAGES * S::STAGE) + (uint32_t)lane * 16;
    bool bad = false;
    const bf16_t* const kb = reinterpret_cast<const bf16_t*>(a.cache.k) + (long long)hk * a.cache.k_head;
    const bf16_t* const vb = reinterpret_cast<const bf16_t*>(a.cache.v) + (long long)hk * a.cache.v_head;

    // Pages.  Pages of whole blocks: lane i holds the page of this warp's block 32 w + i, asked for 32 blocks at a time.  Others:
    // lane i holds page and row of slot i % 16 of the next block.  What the table says is only looked at when it is used, so
    // that its latency passes behind the blocks in flight.
    int pg = 0, in = 0;
    auto look_up = [&](int n) {                            // n: the warp's n-th block
        const int j = j_lo + warp + (PAGE16 ? (n + lane) : n) * kMmaWarps;
        const int s = j * kMmaSlots + (PAGE16 ? 0 : lane & 15);
        pg = 0; in = 0;
        if (j < j_hi && (PAGE16 || (s >= lo && s < hi))) {
            const int index = quotient(s, a.cache.page);
            pg = __ldcg(table + index);
            in = s - index * (int)a.cache.page.d;
        }
    };
    // this lane's pieces of a block of consecutive rows; a piece beyond the head (FULL: there is none) is fetched as zeros
    // from its first channels
    long long k_off[2], v_off[4];
#pragma unroll
    for (int u = 0; u < 2; ++u) k_off[u] = PAGE16 ? (long long)(g + 8 * u) * a.cache.k_row : 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) v_off[u] = PAGE16 ? (long long)(2 * c + (u & 1) + 8 * (u >> 1)) * a.cache.v_row : 0;
    auto fetch = [&](int n, int stage) {
        const int j = j_lo + warp + n * kMmaWarps;
        const uint32_t dst = ring + (uint32_t)(stage * S::STAGE);
        if (PAGE16 && (n & 31) == 0) look_up(n);
        int id = PAGE16 ? __shfl_sync(0xffffffffu, pg, n & 31) : pg;
        const int row = PAGE16 ? __shfl_sync(0xffffffffu, in, n & 31) : in;
        if ((unsigned)id >= (unsigned)a.cache.pages) { bad = true; id = 0; }
        const long long kp = id * a.cache.k_page + row * a.cache.k_row, vp = id * a.cache.v_page + row * a.cache.v_row;
        const int first = j < j_hi ? lo - j * kMmaSlots : kMmaSlots, end = hi - j * kMmaSlots;      // rows that are seen
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int i = g + 8 * u, bytes = i >= first && i < end ? 16 : 0;
            const bf16_t* src = kb + (PAGE16 ? kp + k_off[u] : __shfl_sync(0xffffffffu, kp, i));
#pragma unroll
            for (int b = 0; b < DC; ++b) {
                const bool over = !FULL && 32 * b + 8 * c >= D;
                cp_async16(dst + (uint32_t)(u * DC + b) * 512, src + (over ? 0 : 32 * b + 8 * c), over ? 0 : bytes);
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = 2 * c + (u & 1) + 8 * (u >> 1), bytes = i >= first && i < end ? 16 : 0;
            const bf16_t* src = vb + (PAGE16 ? vp + v_off[u] : __shfl_sync(0xffffffffu, vp, i));
#pragma unroll
            for (int h = 0; h < HC; ++h) {
                const bool over = !FULL && 64 * h + 8 * g >= D;
                cp_async16(dst + (uint32_t)(2 * DC + u * HC + h) * 512, src + (over ? 0 : 64 * h + 8 * g), over ? 0 : bytes);
            }
        }
        cp_async_commit();
        if (!PAGE16) look_up(n + 1);
    };
    if (!PAGE16) look_up(0);
    int next = 0;                                          // the next block to fetch
#pragma unroll
    for (int s = 0; s < S::STAGES - 1; ++s) fetch(next++, s);

    // Q: channels 32 b + 8 c .. + 7 of rows g and g + 8
    uint4 q[2][DC];
    Seen mine[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int row = g + 8 * u;
        const bool on = row < nrow;
        const int token = on ? (row0 + row) / a.group : 0, head = hk * a.group + (on ? (row0 + row) - token * a.group : 0);
        const bf16_t* src = reinterpret_cast<const bf16_t*>(a.q.data) + (long long)(r.first + token) * a.q.row + (long long)head * a.q.head;
#pragma unroll
        for (int b = 0; b < DC; ++b)
            q[u][b] = on && 32 * b + 8 * c < D ? __ldcg(reinterpret_cast<const uint4*>(src + 32 * b + 8 * c)) : make_uint4(0, 0, 0, 0);
        mine[u] = on ? seen_by(r, token, a.causal, a.window) : Seen{0, 0};
    }
    const float scale = a.scale * 1.4426950408889634f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    float o[HC][8][4];
#pragma unroll
    for (int h = 0; h < HC; ++h)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[h][j][e] = 0.f;

    int stage = 0;
    for (int j = j_lo + warp; j < j_hi; j += kMmaWarps) {
        int last = stage + S::STAGES - 1;
        if (last >= S::STAGES) last -= S::STAGES;
        fetch(next++, last);
        cp_async_wait<S::STAGES - 1>();
        const uint32_t at = ring + (uint32_t)(stage * S::STAGE);
        if (++stage == S::STAGES) stage = 0;

        float s[2][4], s1[2][4];                           // (four chains of MMAs, none longer than half the channels)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[u][e] = s1[u][e] = 0.f;
#pragma unroll
        for (int b = 0; b < DC; ++b) {
            uint4 k[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) k[u] = lds128(at + (uint32_t)(u * DC + b) * 512);
#pragma unroll
            for (int u = 0; u < 2; ++u) mma_bf16(s[u], q[0][b].x, q[1][b].x, q[0][b].y, q[1][b].y, k[u].x, k[u].y);
#pragma unroll
            for (int u = 0; u < 2; ++u) mma_bf16(s1[u], q[0][b].z, q[1][b].z, q[0][b].w, q[1][b].w, k[u].z, k[u].w);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[u][e] += s1[u][e];
        // s[u][0, 1]: row g, slots 8 u + 2 c + {0, 1}; s[u][2, 3]: row g + 8
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[u][e] *= scale;
        const int s0 = j * kMmaSlots;
        if (s0 < all_lo || s0 + kMmaSlots > all_hi) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int slot = s0 + 8 * u + 2 * c + (e & 1);
                    const Seen& v = mine[e >> 1];
                    s[u][e] = slot >= v.lo && slot < v.hi ? s[u][e] : -INFINITY;
                }
        }
        float top[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) top[w] = fmaxf(fmaxf(s[0][2 * w], s[0][2 * w + 1]), fmaxf(s[1][2 * w], s[1][2 * w + 1]));
        if (__any_sync(0xffffffffu, top[0] > m[0] + 8.f || top[1] > m[1] + 8.f)) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                float x = fmaxf(top[w], __shfl_xor_sync(0xffffffffu, top[w], 1));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
                x = fmaxf(x, m[w]);
                const float f = m[w] == x ? 1.f : exp2f(m[w] - x);
                m[w] = x;
                l[w] *= f;
#pragma unroll
                for (int h = 0; h < HC; ++h)
#pragma unroll
                    for (int jj = 0; jj < 8; ++jj) { o[h][jj][2 * w] *= f; o[h][jj][2 * w + 1] *= f; }
            }
        }
        const float ref[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
        uint32_t p[4];                                     // (rows g, g + 8) x (slots 2c, 2c + 1; 2c + 8, 2c + 9)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                float p0, p1;
                asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(p0) : "f"(s[u][2 * w] - ref[w]));
                asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(p1) : "f"(s[u][2 * w + 1] - ref[w]));
                l[w] += p0 + p1;
                p[2 * u + w] = bf16_pair(p0, p1);
            }
#pragma unroll
        for (int h = 0; h < HC; ++h) {
            uint4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = lds128(at + (uint32_t)(2 * DC + u * HC + h) * 512);
            const uint32_t* v0 = reinterpret_cast<const uint32_t*>(&v[0]);
            const uint32_t* v1 = reinterpret_cast<const uint32_t*>(&v[1]);
            const uint32_t* v2 = reinterpret_cast<const uint32_t*>(&v[2]);
            const uint32_t* v3 = reinterpret_cast<const uint32_t*>(&v[3]);
#pragma unroll
            for (int jj = 0; jj < 8; ++jj) {
                const uint32_t sel = jj & 1 ? 0x7632 : 0x5410;
                mma_bf16(o[h][jj], p[0], p[1], p[2], p[3], __byte_perm(v0[jj / 2], v1[jj / 2], sel), __byte_perm(v2[jj / 2], v3[jj / 2], sel));
            }
        }
    }
    cp_async_wait<0>();
    pdl_launch_dependents();
    if (bad) report_paged(a.hdr, 2);

    // ---- join the warps: o[h][j][e]: row g + 8 (e / 2), channel 64 h + 16 c + 8 (e % 2) + j -----------------------------------
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        l[w] += __shfl_xor_sync(0xffffffffu, l[w], 1);
        l[w] += __shfl_xor_sync(0xffffffffu, l[w], 2);
        if (c == 0) { jn.m[warp][g + 8 * w] = m[w]; jn.l[warp][g + 8 * w] = l[w]; }
    }
    __syncthreads();                                       // (every warp is through with its ring)
    float* const so = reinterpret_cast<float*>(mma_smem);
    if (tid == 0) jn.o = so;
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int h = 0; h < HC; ++h)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float* dst = so + (warp * kMmaRows + g + 8 * w) * S::OP + 64 * h + 16 * c + 8 * e;
                *reinterpret_cast<float4*>(dst) = make_float4(o[h][0][2 * w + e], o[h][1][2 * w + e], o[h][2][2 * w + e], o[h][3][2 * w + e]);
                *reinterpret_cast<float4*>(dst + 4) = make_float4(o[h][4][2 * w + e], o[h][5][2 * w + e], o[h][6][2 * w + e], o[h][7][2 * w + e]);
            }
    __syncthreads();
    join_rows<S::D>(a, jn, r, row0, nrow, hk, lsplit, rank);
}

// ---- host side ------------------------------------------------------------------------------------------------------
bool attend_mma_takes(const AttendArgs& a, int dtype) {
    auto eight = [](const void* p, long long s0, long long s1, long long s2) {
        return reinterpret_cast<uintptr_t>(p) % 16 == 0 && s0 % 8 == 0 && s1 % 8 == 0 && s2 % 8 == 0;
    };
    return dtype == TTF_DTYPE_BF16 && a.cache.dim % 8 == 0 && eight(a.q.data, a.q.row, a.q.head, 0) &&
           eight(a.out.data, a.out.row, a.out.head, 0) && eight(a.cache.k, a.cache.k_page, a.cache.k_row, a.cache.k_head) &&
           eight(a.cache.v, a.cache.v_page, a.cache.v_row, a.cache.v_head);
}

template <int DC, bool PAGE16, bool FULL> static cudaError_t launch_mma_f(const AttendArgs& a, cudaStream_t st) {
    using S = MmaShape<DC>;
    const void* fn = reinterpret_cast<const void*>(k_attend_mma<DC, PAGE16, FULL>);
    const size_t join = (size_t)kMmaWarps * kMmaRows * S::OP * 4, smem = S::SMEM > join ? S::SMEM : join;
    cudaError_t e = ensure_dynamic_smem(fn, smem);
    if (e != cudaSuccess) return e;
    const long long ctas = most_tiles(a, kMmaRows, 0) * a.cache.heads;
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
    return cudaLaunchKernelEx(&cfg, k_attend_mma<DC, PAGE16, FULL>, a, ls);
}
template <int DC, bool PAGE16> static cudaError_t launch_mma_t(const AttendArgs& a, cudaStream_t st) {
    return a.cache.dim == 32 * DC ? launch_mma_f<DC, PAGE16, true>(a, st) : launch_mma_f<DC, PAGE16, false>(a, st);
}
cudaError_t launch_attend_mma(const AttendArgs& a, cudaStream_t st) {
    const bool whole = a.cache.page.d % kMmaSlots == 0;
    switch ((a.cache.dim + 63) / 64) {
        case 1: return whole ? launch_mma_t<2, true>(a, st) : launch_mma_t<2, false>(a, st);
        case 2: return whole ? launch_mma_t<4, true>(a, st) : launch_mma_t<4, false>(a, st);
        case 3: return whole ? launch_mma_t<6, true>(a, st) : launch_mma_t<6, false>(a, st);
        default: return whole ? launch_mma_t<8, true>(a, st) : launch_mma_t<8, false>(a, st);
    }
}

}  // namespace ttf

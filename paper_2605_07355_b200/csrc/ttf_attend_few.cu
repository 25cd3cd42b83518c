// Attention of few new rows over a paged cache, bf16, heads of up to 128 channels and pages of whole blocks of 16 slots: decoding
// and a few tokens at a time.  Bound by the bytes of the cache: 64 sequences of 500 to 16000 slots, 8 heads of 128, take 186 us,
// 6.1 TB/s.  A single sequence of 2760 slots takes 9.3 us, of which its bytes would be 1.7: finding the tile and the pages, the
// first tiles' latency and the join of 16 CTAs follow one another.
//
//   S = Q K^T,  t = scale log2(e) S,  P = exp2(t - m),  O += P V,  l += sum P,  o = O / l
//
// A CTA takes 16 packed rows (tokens x query heads of a group) of one sequence and key head: the 16 rows of an m16n8k16 MMA.
// Its four warps take the blocks of 16 slots in turn, each on its own with a ring of TMA tiles (64 channels x 16 slots, 128-byte
// swizzle) that its first lane keeps filled: no barrier in the loop, nothing between a block's arrival and the warp that reads it.
// Operands come out of the tiles with ldmatrix (the values transposed).  (The same with a cp.async of 16 bytes per lane and piece,
// ttf_attend_mma.cu, takes in 35 GB/s per SM whatever is resident: every piece is 4 to 8 lines for the load unit.)
// m only moves when a score exceeds it by more than 8 (in powers of two), so that a block usually needs no exchange between lanes;
// sums are kept per lane until the end.  Warps, and the CTAs of a cluster that share the slots of long sequences, join their sums
// through shared memory.
//
// P is rounded to bf16 for the second product, l adds up the weights before that (as in ttf_attend_tc.cu, with the same error).
//
// Values of slots that no row of the tile sees are zeroed in shared memory, whatever the page holds there.
//
// Every mbarrier wait is bounded: a warp whose wait runs out reports it and stops; what its copies in flight still write is waited
// for (bounded) before it goes on to the join.
#include <cuda.h>

#include "ttf_attend_few.cuh"
#include "ttf_tensormap.cuh"

namespace ttf {

template <int DP, int STAGES> struct FewShape {
    static constexpr int HALVES = DP / 64;                 // tiles of 64 channels
    static constexpr int TILE = kMmaSlots * 128;           // 2 KB
    static constexpr int STAGE = 2 * HALVES * TILE;        // keys, values
    static constexpr int RING = kMmaWarps * STAGES * STAGE;
    static constexpr int JOIN = kMmaWarps * kMmaRows * (DP + 4) * 4;
    static constexpr int SMEM = RING > JOIN ? RING : JOIN;
};
struct FewMaps { CUtensorMap k, v; };

__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

template <int DP, int STAGES>
__global__ void __launch_bounds__(kMmaThreads, 3)
k_attend_few(const __grid_constant__ FewMaps maps, const __grid_constant__ AttendArgs a, int lsplit)
{
    using S = FewShape<DP, STAGES>;
    extern __shared__ unsigned char few_raw[];
    __shared__ JoinSpace<DP> jn;
    __shared__ uint64_t bar[kMmaWarps][STAGES];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const int D = a.cache.dim;
    const int rank = lsplit ? (int)cluster_rank() : 0;
    const int work = blockIdx.x >> lsplit, hk = work % a.cache.heads;
    if (lane == 0) {
        for (int s = 0; s < STAGES; ++s) mbar_init(&bar[warp][s], 1);
        mbar_init_fence();
        if (warp == 0) { tensormap_prefetch(&maps.k); tensormap_prefetch(&maps.v); }
    }
    __syncwarp();

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
    const int mine_n = j_hi - j_lo > warp ? (j_hi - j_lo - warp + kMmaWarps - 1) / kMmaWarps : 0;      // this warp's blocks

    const uint32_t base = (smem_u32(few_raw) + 1023u) & ~1023u;
    unsigned char* const smem = few_raw + (base - smem_u32(few_raw));
    const uint32_t ring = base + (uint32_t)(warp * STAGES * S::STAGE);
    bool bad = false;
    // lane i holds page and first row in it of this warp's block 32 w + i, asked for 32 blocks at a time
    int pg = 0, in = 0;
    auto fetch = [&](int n) {                              // the warp's n-th block; the whole warp
        if ((n & 31) == 0) {
            const int j = j_lo + warp + (n + lane) * kMmaWarps;
            pg = 0; in = 0;
            if (j < j_hi) {
                const int index = quotient(j * kMmaSlots, a.cache.page);
                pg = __ldcg(table + index);
                in = j * kMmaSlots - index * (int)a.cache.page.d;
            }
        }
        int id = __shfl_sync(0xffffffffu, pg, n & 31);
        const int row = __shfl_sync(0xffffffffu, in, n & 31);
        if ((unsigned)id >= (unsigned)a.cache.pages) { bad = true; id = 0; }
        if (lane == 0) {
            const int stage = n % STAGES;
            uint64_t* const b = &bar[warp][stage];
            unsigned char* const dst = smem + (warp * STAGES + stage) * S::STAGE;
            mbar_arrive_expect_tx(b, (uint32_t)(S::STAGE + a.tx_extra));
#pragma unroll
            for (int h = 0; h < S::HALVES; ++h) tma_load_4d(dst + h * S::TILE, &maps.k, h * 64, row, hk, id, b);
#pragma unroll
            for (int h = 0; h < S::HALVES; ++h) tma_load_4d(dst + (S::HALVES + h) * S::TILE, &maps.v, h * 64, row, hk, id, b);
        }
    };
    int issued = 0;
    for (; issued < STAGES && issued < mine_n; ++issued) fetch(issued);

    // Q: rows g and g + 8, channels 16 k + 2c, + 1 and 16 k + 8 + 2c, + 1
    uint32_t q[DP / 16][4];
    Seen mine[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int row = g + 8 * u;
        const bool on = row < nrow;
        const int token = on ? (row0 + row) / a.group : 0, head = hk * a.group + (on ? (row0 + row) - token * a.group : 0);
        const bf16_t* src = reinterpret_cast<const bf16_t*>(a.q.data) + (long long)(r.first + token) * a.q.row + (long long)head * a.q.head;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const int d = 16 * k + 8 * w + 2 * c;
                q[k][u + 2 * w] = on && d < D ? __ldcg(reinterpret_cast<const uint32_t*>(src + d)) : 0u;
            }
        mine[u] = on ? seen_by(r, token, a.causal, a.window) : Seen{0, 0};
    }
    const float scale = a.scale * 1.4426950408889634f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    float o[DP / 8][4];
#pragma unroll
    for (int j = 0; j < DP / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = 0.f;

    // ldmatrix addresses within a tile of 16 rows x 128 bytes, 16-byte pieces at (piece ^ (row & 7)).  Keys: matrices (slots 0 - 7,
    // pieces p, p + 1), (slots 8 - 15, pieces p, p + 1); values: (slots 0 - 7, 8 - 15) of piece p, then of piece p + 1.
    const int k_row = (lane & 7) + ((lane >> 4) << 3), k_piece = (lane >> 3) & 1;
    const int v_row = lane & 15, v_piece = lane >> 4;
    bool ok = true;
    for (int n = 0; n < mine_n; ++n) {
        const int stage = n % STAGES;
        const uint32_t at = ring + (uint32_t)(stage * S::STAGE);
        if (!__all_sync(0xffffffffu, mbar_wait(&bar[warp][stage], (n / STAGES) & 1, a.wait_limit))) { ok = false; break; }
        float s[2][4], s1[2][4];                           // (four chains of MMAs)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[u][e] = s1[u][e] = 0.f;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
            uint32_t b[4];
            ldmatrix_x4(b, at + (uint32_t)((k / 4) * S::TILE + k_row * 128 + (((k % 4) * 2 + k_piece) ^ (k_row & 7)) * 16));
            if (k & 1) {
                mma_bf16(s1[0], q[k][0], q[k][1], q[k][2], q[k][3], b[0], b[1]);
                mma_bf16(s1[1], q[k][0], q[k][1], q[k][2], q[k][3], b[2], b[3]);
            } else {
                mma_bf16(s[0], q[k][0], q[k][1], q[k][2], q[k][3], b[0], b[1]);
                mma_bf16(s[1], q[k][0], q[k][1], q[k][2], q[k][3], b[2], b[3]);
            }
        }
        // s[u][0, 1]: row g, slots 8 u + 2 c + {0, 1}; s[u][2, 3]: row g + 8
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[u][e] = (s[u][e] + s1[u][e]) * scale;
        const int s0 = (j_lo + warp + n * kMmaWarps) * kMmaSlots;
        if (s0 < all_lo || s0 + kMmaSlots > all_hi) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int slot = s0 + 8 * u + 2 * c + (e & 1);
                    const Seen& v = mine[e >> 1];
                    s[u][e] = slot >= v.lo && slot < v.hi ? s[u][e] : -INFINITY;
                }
            if (s0 < lo || s0 + kMmaSlots > hi) {          // values of slots that no row sees
                for (int i = lane; i < kMmaSlots * 8 * S::HALVES; i += 32) {
                    const int row = (i >> 3) % kMmaSlots;
                    if (s0 + row < lo || s0 + row >= hi)
                        *reinterpret_cast<uint4*>(smem + (at - base) + S::HALVES * S::TILE + i * 16) = make_uint4(0, 0, 0, 0);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");           // (before the ring's next copy into them)
                __syncwarp();
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
                for (int j = 0; j < DP / 8; ++j) { o[j][2 * w] *= f; o[j][2 * w + 1] *= f; }
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
        for (int j = 0; j < DP / 16; ++j) {                // columns 16 j .. + 15
            uint32_t b[4];
            ldmatrix_x4_trans(b, at + (uint32_t)((S::HALVES + j / 4) * S::TILE + v_row * 128 + (((j % 4) * 2 + v_piece) ^ (v_row & 7)) * 16));
            mma_bf16(o[2 * j], p[0], p[1], p[2], p[3], b[0], b[1]);
            mma_bf16(o[2 * j + 1], p[0], p[1], p[2], p[3], b[2], b[3]);
        }
        __syncwarp();                                      // (every lane has read the stage)
        if (issued < mine_n) fetch(issued++);
    }
    if (!ok) {                                             // copies in flight land before the CTA may leave
        for (int n = issued > STAGES ? issued - STAGES : 0; n < issued; ++n) mbar_wait(&bar[warp][n % STAGES], (n / STAGES) & 1, a.wait_limit);
        if (lane == 0) report_paged(a.hdr, 1);
        __syncwarp();
    }
    pdl_launch_dependents();
    if (bad) report_paged(a.hdr, 2);

    // ---- join: o[j][e]: row g + 8 (e / 2), channel 8 j + 2 c + e % 2 -----------------------------------------------------------
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        l[w] += __shfl_xor_sync(0xffffffffu, l[w], 1);
        l[w] += __shfl_xor_sync(0xffffffffu, l[w], 2);
        if (c == 0) { jn.m[warp][g + 8 * w] = m[w]; jn.l[warp][g + 8 * w] = l[w]; }
    }
    __syncthreads();                                       // (every warp is through with its ring)
    float* const so = reinterpret_cast<float*>(smem);
    if (tid == 0) jn.o = so;
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int j = 0; j < DP / 8; ++j)
            *reinterpret_cast<float2*>(so + (warp * kMmaRows + g + 8 * w) * JoinSpace<DP>::OP + 8 * j + 2 * c) = make_float2(o[j][2 * w], o[j][2 * w + 1]);
    __syncthreads();
    join_rows<DP>(a, jn, r, row0, nrow, hk, lsplit, rank);
}

// ---- host side ------------------------------------------------------------------------------------------------------
bool attend_few_takes(const AttendArgs& a, int dtype) {
    return a.cache.dim <= 128 && a.cache.page.d % kMmaSlots == 0 && attend_mma_takes(a, dtype) && cache_maps_fit(a);
}

template <int DP, int STAGES> static cudaError_t launch_few_t(const AttendArgs& a, int ls, long long ctas, cudaStream_t st) {
    using S = FewShape<DP, STAGES>;
    FewMaps maps;
    if (!make_cache_map(&maps.k, a, false, kMmaSlots) || !make_cache_map(&maps.v, a, true, kMmaSlots)) return cudaErrorInvalidValue;
    const void* fn = reinterpret_cast<const void*>(k_attend_few<DP, STAGES>);
    const size_t smem = S::SMEM + 1024;
    cudaError_t e = ensure_dynamic_smem(fn, smem);
    if (e != cudaSuccess) return e;
    if (ls > 3 && !large_cluster_fits(fn, kMmaThreads, smem)) ls = 3;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(ctas << ls)); cfg.blockDim = dim3(kMmaThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1u << ls; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = ls ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, k_attend_few<DP, STAGES>, maps, a, ls);
}
cudaError_t launch_attend_few(const AttendArgs& a, cudaStream_t st) {
    const long long ctas = most_tiles(a, kMmaRows, 0) * a.cache.heads;
    const int ls = few_split(a, ctas);
    if ((ctas << ls) > 0x7fffffffLL) return cudaErrorInvalidValue;
    if (a.cache.dim <= 64) return launch_few_t<64, 4>(a, ls, ctas, st);
    return launch_few_t<128, 2>(a, ls, ctas, st);
}

}  // namespace ttf

// What the two kernels for few new rows share: 16 packed rows per CTA, four warps that take the blocks of 16 slots in turn, and
// the join of their sums and of those of a cluster's CTAs.
#pragma once

#include "ttf_paged.cuh"
#include "ttf_cluster.cuh"
#include "ttf_async.cuh"

namespace ttf {

constexpr int kMmaWarps = 4, kMmaThreads = 32 * kMmaWarps, kMmaRows = 16, kMmaSlots = 16;

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 bytes into shared memory, zeros where `bytes` is 0 (the address is inside the cache all the same)
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int D> struct JoinSpace {
    static constexpr int OP = D + 4;                       // floats of a row
    float m[kMmaWarps][kMmaRows], l[kMmaWarps][kMmaRows];  // every warp's maxima and sums
    float* o;                                              // [warp][row][OP] their weighted values
    // what the ranks of a cluster send: rank p's sums of this rank's i-th row (row i * split + rank) are row i * split + p
    __align__(16) float in[kMmaRows][OP];
    float m_in[kMmaRows], l_in[kMmaRows];
};

// Adds up the warps' sums of the tile's `nrow` rows, then those of the ranks, and writes the rows.  Every thread of the CTA;
// jn.m, jn.l and jn.o are visible to all, and with a cluster every thread has arrived at its barrier once before.
template <int D, typename T = bf16_t>
__device__ __forceinline__ void join_rows(const AttendArgs& a, JoinSpace<D>& jn, const SeqRange& r, int row0, int nrow, int hk,
                                          int lsplit, int rank) {
    constexpr int OP = JoinSpace<D>::OP, Q4 = D / 4;
    const int tid = threadIdx.x, dim = a.cache.dim, split = 1 << lsplit;
    auto store = [&](int row, int d, float4 v, float sum) {
        const int token = (row0 + row) / a.group, head = hk * a.group + (row0 + row) - token * a.group;
        if (d >= dim || !in_bounds(a.hdr, 8, (long long)r.first + token, a.seq.rows)) return;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        float x[4] = {0.f, 0.f, 0.f, 0.f};                 // (no slot seen: zero)
        if (sum != 0.f) { x[0] = v.x * inv; x[1] = v.y * inv; x[2] = v.z * inv; x[3] = v.w * inv; }
        *reinterpret_cast<typename VecIO<T, 4>::Raw*>(reinterpret_cast<T*>(a.out.data) + (long long)(r.first + token) * a.out.row + (long long)head * a.out.head + d) = pack<4>(x, T{});
    };
    if (lsplit) { __syncwarp(); cluster_wait(); }          // every rank is running
    for (int e = tid; e < nrow * Q4; e += kMmaThreads) {
        const int row = e / Q4, d = (e - row * Q4) * 4;
        float mw[kMmaWarps], lw[kMmaWarps], mx = -INFINITY;
        float4 x[kMmaWarps];
#pragma unroll
        for (int w = 0; w < kMmaWarps; ++w) {
            mw[w] = jn.m[w][row]; lw[w] = jn.l[w][row];
            x[w] = *reinterpret_cast<const float4*>(jn.o + (w * kMmaRows + row) * OP + d);
            mx = fmaxf(mx, mw[w]);
        }
        const float ref = mx == -INFINITY ? 0.f : mx;
        float sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kMmaWarps; ++w) {
            if (lw[w] == 0.f) continue;                    // that warp saw nothing of the row
            const float f = exp2f(mw[w] - ref);
            sum = fmaf(f, lw[w], sum);
            v.x = fmaf(f, x[w].x, v.x); v.y = fmaf(f, x[w].y, v.y); v.z = fmaf(f, x[w].z, v.z); v.w = fmaf(f, x[w].w, v.w);
        }
        if (lsplit == 0) store(row, d, v, sum);
        else {
            const int to = row & (split - 1), slot = (row >> lsplit << lsplit) + rank;
            const uint32_t at = cluster_addr(smem_u32(&jn.in[slot][d]), to);
            asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
            if (d == 0) { st_cluster_f32(cluster_addr(smem_u32(&jn.m_in[slot]), to), mx); st_cluster_f32(cluster_addr(smem_u32(&jn.l_in[slot]), to), sum); }
        }
    }
    if (lsplit == 0) return;
    __syncwarp();
    cluster_arrive();
    cluster_wait();
    const int rows_mine = (nrow - rank + split - 1) >> lsplit;               // rows row % split == rank
    for (int e = tid; e < rows_mine * Q4; e += kMmaThreads) {
        const int i = e / Q4, row = rank + (i << lsplit), d = (e - i * Q4) * 4, slot = i << lsplit;
        float mx = -INFINITY;
        for (int p = 0; p < split; ++p) mx = fmaxf(mx, jn.m_in[slot + p]);
        const float ref = mx == -INFINITY ? 0.f : mx;
        float sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int p = 0; p < split; ++p) {
            const float lp = jn.l_in[slot + p], f = lp == 0.f ? 0.f : exp2f(jn.m_in[slot + p] - ref);
            const float4 x = *reinterpret_cast<const float4*>(&jn.in[slot + p][d]);
            if (lp == 0.f) continue;                       // that rank saw nothing of the row
            sum = fmaf(f, lp, sum);
            v.x = fmaf(f, x.x, v.x); v.y = fmaf(f, x.y, v.y); v.z = fmaf(f, x.z, v.z); v.w = fmaf(f, x.w, v.w);
        }
        store(row, d, v, sum);
    }
}

// CTAs (a power of two) that share the slots of a tile; `ctas` tiles at most.  The host knows how long a sequence may be, not
// how long it is.  Shares of long sequences stay above 2048 slots, so that the last CTAs to run are short against the call: 64
// sequences of 500 to 16000 slots, 8 heads of 128: 230 / 206 / 187 / 200 us with 1 / 2 / 4 / 8; 64 of 4400: 197 / 181 / 183 / 205;
// 64 of 500: 36 / 45 / 63 / 103 (what a CTA costs before its first and after its last block is not small against those).  Where
// the CTAs do not fill the GPU shares go down to 128 slots: one sequence of 2760 slots 32 / 19 / 12.3 / 9.2 us.  (What a sequence
// may be is the width of its table: 64 sequences of 500 slots take 35 us with a table of 500 slots, 62 with 8192, 101 with 16384.)
inline int few_split(const AttendArgs& a, long long ctas) {
    const long long slots = (long long)a.seq.table_pages * a.cache.page.d;
    const long long reach = (long long)a.window + a.seq.rows, longest = a.window > 0 && reach < slots ? reach : slots;
    const long long places = 3LL * sm_count();
    int ls = 0;
    while (ls < 3 && ((longest >> (ls + 1)) >= 2048 || ((ctas << (ls + 1)) <= places && (longest >> (ls + 1)) >= 128))) ++ls;
    if (ls == 3 && (ctas << 4) <= sm_count() && (longest >> 4) >= 256) ls = 4;
    return ls;
}

}  // namespace ttf

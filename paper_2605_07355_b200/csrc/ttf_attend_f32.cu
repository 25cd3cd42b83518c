// Attention of many new rows over a paged cache, fp32: chunks and whole prompts.
//
//   o = sum_s exp2(t_s - m) v_s / sum_s exp2(t_s - m),   t_s = scale log2(e) <q, k_s>,   m the running maximum
//
// One CTA takes 64 packed rows (tokens x query heads of a group, so that a group reads its keys and values once) of one sequence
// and key head, and walks the visible slots 32 at a time: 16 x 16 threads, four rows by two slots of scores each, then the same
// four rows by D / 16 channels of the sum.  A row belongs to the same 16 lanes in both products, so its maximum and its weights
// never leave them and one barrier per block is enough.  The next block is on its way (cp.async) meanwhile, its pages are looked
// up one block earlier.  Bound by shared memory: a read of 16 bytes takes a warp's four cycles whether lanes share addresses or
// not, and six of them feed 32 FMAs (eight cycles) of the scores, three as many of the sums.  8 heads of 128, 16 sequences of 128
// rows over 3000 slots: 976 us, 26 TFLOP/s (two rows by two slots a thread and 32 rows a CTA reached 15).
//
// Dot products run in four chains, and a block's products are summed apart and then added: over thousands of slots one chain
// would lose digits.  With few tiles the CTAs of a cluster share the slots and join their sums through distributed shared memory.
//
// A slot that a row does not see takes no part in that row's sum, whatever it holds.
#include <type_traits>

#include "ttf_attend_few.cuh"

namespace ttf {

constexpr int kF32Keys = 32, kF32Threads = 256, kF32TileRows = 64, kF32Weights = kF32Keys + 4;

template <int DCH> struct F32Shape {                       // DCH: 64-channel pieces of a head
    static constexpr int P = DCH * 64 + 4;                 // floats of a shared row (the pad spreads rows over the banks)
    static constexpr int KEYS = kF32Keys * P;
    static constexpr int FLOATS = kF32TileRows * P + 4 * KEYS + kF32TileRows * kF32Weights + 2 * kF32TileRows;
};

template <int DCH>
__global__ void __launch_bounds__(kF32Threads, DCH <= 2 ? 2 : 1)
k_attend_f32(const __grid_constant__ AttendArgs a, int lsplit)
{
    using S = F32Shape<DCH>;
    constexpr int P = S::P;
    extern __shared__ float4 f32_tile_smem[];
    float* const sq = reinterpret_cast<float*>(f32_tile_smem);
    float* const skv = sq + kF32TileRows * P;              // [2] keys and values of a block
    float* const sw = skv + 4 * S::KEYS;                   // weights
    float* const s_m = sw + kF32TileRows * kF32Weights;
    float* const s_l = s_m + kF32TileRows;
    const int tid = threadIdx.x, D = a.cache.dim;
    const int split = 1 << lsplit, rank = lsplit ? (int)cluster_rank() : 0;
    const int hk = blockIdx.y;

    pdl_wait();
    Tile t;
    // (every CTA of a cluster has the same tile, and so the same answer)
    if (!find_tile(a, Cut{Divisor{0, 0, 0}, 6}, blockIdx.x >> lsplit, blockIdx.x == 0 && blockIdx.y == 0, t)) return;
    const SeqRange r = t.r;
    const int* const table = a.seq.table + (long long)t.seq * a.seq.table_stride;
    const int row0 = t.tile * kF32TileRows;                // first packed row
    const long long packed = (long long)r.n * a.group;
    const int nrow = packed - row0 < kF32TileRows ? (int)(packed - row0) : kF32TileRows;

    // the slots that any row of the tile sees, in blocks of 32 from a multiple of 32 on, and this rank's share of the blocks
    const int tok_a = row0 / a.group, tok_z = (row0 + nrow - 1) / a.group;
    const int lo = seen_by(r, tok_a, a.causal, a.window).lo, hi = seen_by(r, tok_z, a.causal, a.window).hi;    // (both grow with the token)
    const int b_lo = lo / kF32Keys, b_hi = hi > lo ? (hi + kF32Keys - 1) / kF32Keys : b_lo;
    const int nb = b_hi - b_lo;
    const int my_a = b_lo + (int)((long long)nb * rank >> lsplit), my_z = b_lo + (int)((long long)nb * (rank + 1) >> lsplit);

    const int lr = tid >> 3, lc = tid & 7;                 // copies: slot lr of a block, every eighth piece of four channels
    const float* const kb = reinterpret_cast<const float*>(a.cache.k) + (long long)hk * a.cache.k_head;
    const float* const vb = reinterpret_cast<const float*>(a.cache.v) + (long long)hk * a.cache.v_head;
    bool bad = false, on = false;
    int pg = 0, in = 0;                                    // this thread's slot of the next block: page as the table has it, row
    auto look_up = [&](int blk) {
        const int s = blk * kF32Keys + lr;
        on = blk < my_z && s >= lo && s < hi;
        pg = 0; in = 0;
        if (on) {
            const int index = quotient(s, a.cache.page);
            pg = __ldcg(table + index);
            in = s - index * (int)a.cache.page.d;
        }
    };
    auto fetch = [&](int blk) {                            // zeros where no row looks and beyond the head
        if (blk < my_z) {
            if ((unsigned)pg >= (unsigned)a.cache.pages) { bad = true; pg = 0; }
            const float* const kp = kb + pg * a.cache.k_page + in * a.cache.k_row;
            const float* const vp = vb + pg * a.cache.v_page + in * a.cache.v_row;
            const uint32_t to = smem_u32(skv + (blk & 1) * 2 * S::KEYS + lr * P);
#pragma unroll
            for (int i = 0; i < 2 * DCH; ++i) {
                const int d = (lc + 8 * i) * 4;
                const bool read = on && d < D;
                cp_async16(to + d * 4, read ? kp + d : kb, read ? 16 : 0);
                cp_async16(to + (S::KEYS + d) * 4, read ? vp + d : vb, read ? 16 : 0);
            }
        }
        cp_async_commit();
    };
    look_up(my_a);
    fetch(my_a);
    look_up(my_a + 1);

    // queries, with the scale in them
    for (int e = tid; e < kF32TileRows * DCH * 16; e += kF32Threads) {
        const int row = e / (DCH * 16), d = (e - row * (DCH * 16)) * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row < nrow && d < D) {
            const int token = (row0 + row) / a.group, head = hk * a.group + (row0 + row) - token * a.group;
            v = __ldcg(reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.q.data) + (long long)(r.first + token) * a.q.row + (long long)head * a.q.head + d));
        }
        const float c = a.scale * 1.4426950408889634f;
        *reinterpret_cast<float4*>(sq + row * P + d) = make_float4(v.x * c, v.y * c, v.z * c, v.w * c);
    }

    const int ty = tid >> 4, tx = tid & 15;                // rows ty + 16 i, slots tx + 16 j, channels 64 c + 4 tx
    float acc[4][DCH][4], m[4], l[4];
    Seen mine[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = ty + 16 * i;
        mine[i] = row < nrow ? seen_by(r, (row0 + row) / a.group, a.causal, a.window) : Seen{0, 0};
        m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
        for (int c = 0; c < DCH; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][c][e] = 0.f;
    }

    for (int blk = my_a; blk < my_z; ++blk) {
        const int base = blk * kF32Keys;
        const float* const sk = skv + (blk & 1) * 2 * S::KEYS;
        const float* const sv = sk + S::KEYS;
        cp_async_wait<0>();
        __syncthreads();                                   // the block is here, and the one before has been read
        fetch(blk + 1);
        look_up(blk + 2);
        bool whole = true;                                 // all four rows see the whole block
#pragma unroll
        for (int i = 0; i < 4; ++i) whole = whole && mine[i].lo <= base && mine[i].hi >= base + kF32Keys;
        float f[4];
        {
            float4 sum[4][2];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) sum[i][j] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
            for (int d = 0; d < D; d += 4) {
                float4 q[4], k[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) k[j] = *reinterpret_cast<const float4*>(sk + (tx + 16 * j) * P + d);
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const float4*>(sq + (ty + 16 * i) * P + d);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        sum[i][j].x = fmaf(q[i].x, k[j].x, sum[i][j].x); sum[i][j].y = fmaf(q[i].y, k[j].y, sum[i][j].y);
                        sum[i][j].z = fmaf(q[i].z, k[j].z, sum[i][j].z); sum[i][j].w = fmaf(q[i].w, k[j].w, sum[i][j].w);
                    }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                bool see[2];
                float x[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int s = base + tx + 16 * j;
                    see[j] = s >= mine[i].lo && s < mine[i].hi;
                    x[j] = see[j] ? (sum[i][j].x + sum[i][j].y) + (sum[i][j].z + sum[i][j].w) : -INFINITY;
                }
                float top = fmaxf(x[0], x[1]);
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                top = fmaxf(top, m[i]);
                const float ref = top == -INFINITY ? 0.f : top;
                f[i] = m[i] == top ? 1.f : exp2f(m[i] - ref);
                m[i] = top;
                // (a score that is NaN where the row sees it stays NaN; one that it does not see is 0)
                const float p0 = see[0] ? exp2f(x[0] - ref) : 0.f, p1 = see[1] ? exp2f(x[1] - ref) : 0.f;
                l[i] = fmaf(l[i], f[i], p0 + p1);
                float* const w = sw + (ty + 16 * i) * kF32Weights + tx;
                w[0] = p0; w[16] = p1;
            }
        }
        __syncwarp();
        float part[4][DCH][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < DCH; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) part[i][c][e] = 0.f;
        auto weighted = [&](auto all) {
#pragma unroll 1
            for (int j = 0; j < kF32Keys; j += 4) {
                float w[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float4 x = *reinterpret_cast<const float4*>(sw + (ty + 16 * i) * kF32Weights + j);
                    w[i][0] = x.x; w[i][1] = x.y; w[i][2] = x.z; w[i][3] = x.w;
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int c = 0; c < DCH; ++c) {
                        const float4 v = *reinterpret_cast<const float4*>(sv + (j + u) * P + c * 64 + tx * 4);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            // (a slot outside a row's range is left out, not multiplied by zero: it may hold anything)
                            if (!decltype(all)::value && !(base + j + u >= mine[i].lo && base + j + u < mine[i].hi)) continue;
                            part[i][c][0] = fmaf(w[i][u], v.x, part[i][c][0]); part[i][c][1] = fmaf(w[i][u], v.y, part[i][c][1]);
                            part[i][c][2] = fmaf(w[i][u], v.z, part[i][c][2]); part[i][c][3] = fmaf(w[i][u], v.w, part[i][c][3]);
                        }
                    }
            }
        };
        if (__all_sync(0xffffffffu, whole)) weighted(std::true_type{}); else weighted(std::false_type{});
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < DCH; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][c][e] = fmaf(acc[i][c][e], f[i], part[i][c][e]);
    }
    pdl_launch_dependents();
    if (bad) report_paged(a.hdr, 2);

    auto store = [&](int row, int d, float4 o) {
        const int token = (row0 + row) / a.group, head = hk * a.group + (row0 + row) - token * a.group;
        if (d >= D || !in_bounds(a.hdr, 8, (long long)r.first + token, a.seq.rows)) return;
        *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out.data) + (long long)(r.first + token) * a.out.row + (long long)head * a.out.head + d) = o;
    };
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o);
    if (lsplit == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = ty + 16 * i;
            if (row >= nrow) continue;
            const float inv = 1.f / l[i];
#pragma unroll
            for (int c = 0; c < DCH; ++c)
                store(row, c * 64 + tx * 4, l[i] == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) :          // (no slot seen)
                      make_float4(acc[i][c][0] * inv, acc[i][c][1] * inv, acc[i][c][2] * inv, acc[i][c][3] * inv));
        }
        return;
    }
    // join: the sums go into shared memory (where the queries were), then every rank finishes the rows row % split == rank
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = ty + 16 * i;
        if (tx == 0) { s_m[row] = m[i]; s_l[row] = l[i]; }
#pragma unroll
        for (int c = 0; c < DCH; ++c)
            *reinterpret_cast<float4*>(sq + row * P + c * 64 + tx * 4) = make_float4(acc[i][c][0], acc[i][c][1], acc[i][c][2], acc[i][c][3]);
    }
    cluster_arrive();
    cluster_wait();
    const int rows_mine = (nrow - rank + split - 1) >> lsplit;               // (none when rank >= nrow)
    for (int e = tid; e < rows_mine * DCH * 16; e += kF32Threads) {
        const int row = rank + (e / (DCH * 16) << lsplit), d = (e % (DCH * 16)) * 4;
        float top = -INFINITY;
        for (int p = 0; p < split; ++p) top = fmaxf(top, ld_cluster_f32(cluster_addr(smem_u32(s_m + row), p)));
        const float ref = top == -INFINITY ? 0.f : top;
        float sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
        for (int p = 0; p < split; ++p) {
            const float lp = ld_cluster_f32(cluster_addr(smem_u32(s_l + row), p));
            if (lp == 0.f) continue;                       // that rank saw nothing of the row
            const float w = exp2f(ld_cluster_f32(cluster_addr(smem_u32(s_m + row), p)) - ref);
            sum = fmaf(w, lp, sum);
            const uint32_t at = cluster_addr(smem_u32(sq + row * P + d), p);
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] = fmaf(w, ld_cluster_f32(at + 4 * c), o[c]);
        }
        const float inv = 1.f / sum;
        store(row, d, sum == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv));
    }
    cluster_arrive();                                      // nobody leaves while its sums may be read
    cluster_wait();
}

bool attend_f32_takes(const AttendArgs& a, int dtype) {
    auto four = [](const void* p, long long s0, long long s1, long long s2) {
        return reinterpret_cast<uintptr_t>(p) % 16 == 0 && s0 % 4 == 0 && s1 % 4 == 0 && s2 % 4 == 0;
    };
    return dtype == TTF_DTYPE_F32 && a.cache.dim % 4 == 0 && four(a.q.data, a.q.row, a.q.head, 0) && four(a.out.data, a.out.row, a.out.head, 0) &&
           four(a.cache.k, a.cache.k_page, a.cache.k_row, a.cache.k_head) && four(a.cache.v, a.cache.v_page, a.cache.v_row, a.cache.v_head);
}
template <int DCH> static cudaError_t launch_f32_t(const AttendArgs& a, cudaStream_t st) {
    const void* fn = reinterpret_cast<const void*>(k_attend_f32<DCH>);
    const size_t smem = F32Shape<DCH>::FLOATS * sizeof(float);
    cudaError_t e = ensure_dynamic_smem(fn, smem);
    if (e != cudaSuccess) return e;
    const long long tiles = most_tiles(a, kF32TileRows, 0);
    // slots are shared until the CTAs fill their places twice (two an SM up to 128 channels, else one), as long as a rank has four
    // blocks of the longest sequence: 16 sequences of 64 new rows over 3000 slots, 8 heads of 128: 961 us without sharing, 492
    // shared by two, 513 by four; 4 heads of 256: 512 by two, 536 by four
    const long long slots = (long long)a.seq.table_pages * a.cache.page.d;
    const long long reach = (long long)a.window + a.seq.rows, longest = a.window > 0 && reach < slots ? reach : slots;
    int ls = 0;
    while (ls < 3 && (tiles * a.cache.heads << (ls + 1)) <= (DCH <= 2 ? 4 : 2) * sm_count() && (longest >> (ls + 1)) >= 4 * kF32Keys) ++ls;
    if ((tiles << ls) > 0x7fffffffLL) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles << ls), a.cache.heads); cfg.blockDim = dim3(kF32Threads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1u << ls; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = ls ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, k_attend_f32<DCH>, a, ls);
}
cudaError_t launch_attend_f32(const AttendArgs& a, cudaStream_t st) {
    switch ((a.cache.dim + 63) / 64) {
        case 1: return launch_f32_t<1>(a, st);
        case 2: return launch_f32_t<2>(a, st);
        case 3: return launch_f32_t<3>(a, st);
        default: return launch_f32_t<4>(a, st);
    }
}

}  // namespace ttf

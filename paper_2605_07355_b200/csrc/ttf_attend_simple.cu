// Attention of new rows over a paged cache in fp32 arithmetic, for heads that fit no 16-byte pieces: bf16 heads that the matrix
// instructions cannot take (channels not a multiple of 8, unaligned strides), fp32 heads in the same way.
//
//   o = sum_s exp2(t_s - m) v_s / sum_s exp2(t_s - m),   t_s = scale log2(e) <q, k_s>,   m the running maximum
//
// One CTA takes 32 packed rows (tokens x query heads of a group, so that a group reads its keys and values once) of one
// sequence and key head, and walks the visible slots 32 at a time: scores as 2 x 2 dot products per thread from shared
// memory, one softmax step with eight threads per row, then 2 rows x D / 16 channels of the sum per thread.  The next
// block is loaded into registers meanwhile, its pages are looked up one block earlier.  Bound by shared memory (four
// loads of 16 bytes feed sixteen FMAs) and, with few rows, by latency: the CTAs of a cluster then share the slots and
// join their sums through distributed shared memory.
//
// A slot that a row does not see takes no part in that row's sum, whatever it holds.
#include "ttf_paged.cuh"
#include "ttf_cluster.cuh"
#include "ttf_async.cuh"

namespace ttf {

constexpr int kSimpleRows = 32, kSimpleKeys = 32, kSimpleThreads = 256;

template <int DCH> struct SimpleShape {
    static constexpr int P = DCH * 64 + 4;                 // floats of a shared row (the pad spreads rows over the banks)
    static constexpr int FLOATS = 3 * 32 * P + 32 * 33 + 4 * 32;
};

template <typename T, int V, int DCH>
__global__ void __launch_bounds__(kSimpleThreads)
k_attend_simple(const __grid_constant__ AttendArgs a, int lsplit)
{
    using S = SimpleShape<DCH>;
    using Raw = typename VecIO<T, V>::Raw;
    constexpr int P = S::P;
    constexpr int NV = DCH * 64 / (8 * V);                 // vectors of a row per thread (eight threads per row)
    extern __shared__ float4 simple_smem[];
    float* const sq = reinterpret_cast<float*>(simple_smem);
    float* const sk = sq + 32 * P;
    float* const sv = sk + 32 * P;
    float* const ss = sv + 32 * P;                         // [32][33] scores, then weights
    float* const s_m = ss + 32 * 33;                       // [32] maximum, [32] sum, [32] factor of the step
    float* const s_l = s_m + 32;
    float* const s_f = s_l + 32;
    const int tid = threadIdx.x, D = a.cache.dim;
    const int split = 1 << lsplit, rank = lsplit ? (int)cluster_rank() : 0;
    const int hk = blockIdx.y;

    pdl_wait();
    Tile t;
    // (every CTA of a cluster has the same tile, and so the same answer)
    if (!find_tile(a, Cut{Divisor{0, 0, 0}, 5}, blockIdx.x >> lsplit, blockIdx.x == 0 && blockIdx.y == 0, t)) return;
    const SeqRange r = t.r;
    const int* const table = a.seq.table + (long long)t.seq * a.seq.table_stride;
    const int row0 = t.tile * kSimpleRows;                 // first packed row
    const long long packed = (long long)r.n * a.group;
    const int nrow = packed - row0 < kSimpleRows ? (int)(packed - row0) : kSimpleRows;

    // queries: row = tid / 8
    const int lr = tid >> 3, lc = tid & 7;
    {
        const bool on = lr < nrow;
        const int token = on ? (row0 + lr) / a.group : 0, g = on ? (row0 + lr) - token * a.group : 0;
        const T* src = reinterpret_cast<const T*>(a.q.data) + (long long)(r.first + token) * a.q.row + (long long)(hk * a.group + g) * a.q.head;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int d = (lc + 8 * i) * V;
            float x[V];
            Raw w = Raw{};
            if (on && d < D) w = load_cg(reinterpret_cast<const Raw*>(src + d));
            unpack<V>(w, x, T{});
#pragma unroll
            for (int c = 0; c < V; ++c) sq[lr * P + d + c] = x[c] * (a.scale * 1.4426950408889634f);
        }
    }
    if (tid < 32) { s_m[tid] = -INFINITY; s_l[tid] = 0.f; }

    // the slots that any row of the tile sees, in blocks of 32 from a multiple of 32 on, and this rank's share of the blocks
    const int tok_a = row0 / a.group, tok_z = (row0 + nrow - 1) / a.group;
    const Seen sa = seen_by(r, tok_a, a.causal, a.window), sz = seen_by(r, tok_z, a.causal, a.window);
    const int lo = sa.lo, hi = sz.hi;                      // (both grow with the token)
    const int b_lo = lo / kSimpleKeys, b_hi = hi > lo ? (hi + kSimpleKeys - 1) / kSimpleKeys : b_lo;
    const int nb = b_hi - b_lo;
    const int my_a = b_lo + (int)((long long)nb * rank >> lsplit), my_z = b_lo + (int)((long long)nb * (rank + 1) >> lsplit);

    bool bad = false;
    float rk[NV * V], rv[NV * V];
    long long k_at = 0, v_at = 0;                          // where this thread's key of the next block lies
    bool k_on = false;
    auto look_up = [&](int blk) {
        const int s = blk * kSimpleKeys + lr;
        k_on = blk < my_z && s >= lo && s < hi;
        if (k_on) {
            const int index = quotient(s, a.cache.page);
            const long long g = page_of(table, index, a.cache.pages, bad);
            const int in = s - index * (int)a.cache.page.d;
            k_at = g * a.cache.k_page + in * a.cache.k_row + (long long)hk * a.cache.k_head;
            v_at = g * a.cache.v_page + in * a.cache.v_row + (long long)hk * a.cache.v_head;
        }
    };
    auto load = [&]() {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int d = (lc + 8 * i) * V;
            Raw wk = Raw{}, wv = Raw{};
            if (k_on && d < D) {
                wk = load_cg(reinterpret_cast<const Raw*>(reinterpret_cast<const T*>(a.cache.k) + k_at + d));
                wv = load_cg(reinterpret_cast<const Raw*>(reinterpret_cast<const T*>(a.cache.v) + v_at + d));
            }
            float x[V];
            unpack<V>(wk, x, T{});
#pragma unroll
            for (int c = 0; c < V; ++c) rk[i * V + c] = x[c];
            unpack<V>(wv, x, T{});
#pragma unroll
            for (int c = 0; c < V; ++c) rv[i * V + c] = x[c];
        }
    };
    look_up(my_a);
    if (my_a < my_z) load();
    look_up(my_a + 1);

    const int ty = tid >> 4, tx = tid & 15;                // scores: rows ty, ty + 16, slots tx, tx + 16
    float acc[2][DCH][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < DCH; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][c][e] = 0.f;
    Seen mine[2];                                          // what this thread's two rows see
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = ty + 16 * i;
        mine[i] = row < nrow ? seen_by(r, (row0 + row) / a.group, a.causal, a.window) : Seen{0, 0};
    }
    const Seen soft = lr < nrow ? seen_by(r, (row0 + lr) / a.group, a.causal, a.window) : Seen{0, 0};

    for (int blk = my_a; blk < my_z; ++blk) {
        const int base = blk * kSimpleKeys;
        __syncthreads();                                   // the block before has been read
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int d = (lc + 8 * i) * V;
#pragma unroll
            for (int c = 0; c < V; ++c) { sk[lr * P + d + c] = rk[i * V + c]; sv[lr * P + d + c] = rv[i * V + c]; }
        }
        __syncthreads();
        if (blk + 1 < my_z) load();
        look_up(blk + 2);
        float4 sums[2][2];                                 // (four chains per dot product)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) sums[i][j] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int d = 0; d < D; d += 4) {                   // (channels from D to the next multiple of 4 are zeros in both)
            float4 q4[2], k4[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                q4[i] = *reinterpret_cast<const float4*>(sq + (ty + 16 * i) * P + d);
                k4[i] = *reinterpret_cast<const float4*>(sk + (tx + 16 * i) * P + d);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    sums[i][j].x = fmaf(q4[i].x, k4[j].x, sums[i][j].x); sums[i][j].y = fmaf(q4[i].y, k4[j].y, sums[i][j].y);
                    sums[i][j].z = fmaf(q4[i].z, k4[j].z, sums[i][j].z); sums[i][j].w = fmaf(q4[i].w, k4[j].w, sums[i][j].w);
                }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int s = base + tx + 16 * j;
                const float dot = (sums[i][j].x + sums[i][j].y) + (sums[i][j].z + sums[i][j].w);
                ss[(ty + 16 * i) * 33 + tx + 16 * j] = s >= mine[i].lo && s < mine[i].hi ? dot : -INFINITY;
            }
        __syncthreads();
        {                                                  // softmax step: row lr, slots lc, lc + 8, ...
            float x[4], mx = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = ss[lr * 33 + lc + 8 * i]; mx = fmaxf(mx, x[i]); }
#pragma unroll
            for (int o = 4; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float m0 = s_m[lr], m1 = fmaxf(m0, mx), ref = m1 == -INFINITY ? 0.f : m1;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int s = base + lc + 8 * i;
                // (a score that is NaN where the row sees it stays NaN; one that it does not see is 0)
                const float p = s >= soft.lo && s < soft.hi ? exp2f(x[i] - ref) : 0.f;
                sum += p;
                ss[lr * 33 + lc + 8 * i] = p;
            }
#pragma unroll
            for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            __syncwarp();
            if (lc == 0) {
                const float f = m0 == m1 ? 1.f : exp2f(m0 - ref);
                s_m[lr] = m1; s_l[lr] = s_l[lr] * f + sum; s_f[lr] = f;
            }
        }
        __syncthreads();
        // the block's products are summed apart and then added: over thousands of slots one chain would lose digits
        float part[2][DCH][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int c = 0; c < DCH; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) part[i][c][e] = 0.f;
        const int a0 = max(mine[0].lo - base, 0), z0 = min(mine[0].hi - base, kSimpleKeys);
        const int a1 = max(mine[1].lo - base, 0), z1 = min(mine[1].hi - base, kSimpleKeys);
        if (a0 == 0 && a1 == 0 && z0 == kSimpleKeys && z1 == kSimpleKeys) {
#pragma unroll 4
            for (int j = 0; j < kSimpleKeys; ++j) {
                const float p0 = ss[ty * 33 + j], p1 = ss[(ty + 16) * 33 + j];
#pragma unroll
                for (int c = 0; c < DCH; ++c) {
                    const float4 v = *reinterpret_cast<const float4*>(sv + j * P + c * 64 + tx * 4);
                    part[0][c][0] = fmaf(p0, v.x, part[0][c][0]); part[0][c][1] = fmaf(p0, v.y, part[0][c][1]);
                    part[0][c][2] = fmaf(p0, v.z, part[0][c][2]); part[0][c][3] = fmaf(p0, v.w, part[0][c][3]);
                    part[1][c][0] = fmaf(p1, v.x, part[1][c][0]); part[1][c][1] = fmaf(p1, v.y, part[1][c][1]);
                    part[1][c][2] = fmaf(p1, v.z, part[1][c][2]); part[1][c][3] = fmaf(p1, v.w, part[1][c][3]);
                }
            }
        } else {
            // (a slot outside a row's range is left out, not multiplied by zero: it may hold anything)
            const int jz = max(z0, z1);
#pragma unroll 4
            for (int j = min(a0, a1); j < jz; ++j) {
                const float p0 = ss[ty * 33 + j], p1 = ss[(ty + 16) * 33 + j];
                const bool in0 = j >= a0 && j < z0, in1 = j >= a1 && j < z1;
#pragma unroll
                for (int c = 0; c < DCH; ++c) {
                    const float4 v = *reinterpret_cast<const float4*>(sv + j * P + c * 64 + tx * 4);
                    if (in0) {
                        part[0][c][0] = fmaf(p0, v.x, part[0][c][0]); part[0][c][1] = fmaf(p0, v.y, part[0][c][1]);
                        part[0][c][2] = fmaf(p0, v.z, part[0][c][2]); part[0][c][3] = fmaf(p0, v.w, part[0][c][3]);
                    }
                    if (in1) {
                        part[1][c][0] = fmaf(p1, v.x, part[1][c][0]); part[1][c][1] = fmaf(p1, v.y, part[1][c][1]);
                        part[1][c][2] = fmaf(p1, v.z, part[1][c][2]); part[1][c][3] = fmaf(p1, v.w, part[1][c][3]);
                    }
                }
            }
        }
        const float f[2] = {s_f[ty], s_f[ty + 16]};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int c = 0; c < DCH; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][c][e] = fmaf(acc[i][c][e], f[i], part[i][c][e]);
    }
    if (bad) report_paged(a.hdr, 2);
    __syncthreads();

    auto store = [&](int row, int d, const float (&o)[4]) {
        const int token = (row0 + row) / a.group, g = (row0 + row) - token * a.group;
        if (!in_bounds(a.hdr, 8, (long long)r.first + token, a.seq.rows)) return;
        T* dst = reinterpret_cast<T*>(a.out.data) + (long long)(r.first + token) * a.out.row + (long long)(hk * a.group + g) * a.out.head + d;
        if constexpr (V >= 4) {
            float x[4] = {o[0], o[1], o[2], o[3]};
            if (d < D) *reinterpret_cast<typename VecIO<T, 4>::Raw*>(dst) = pack<4>(x, T{});
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x[1] = {o[e]};
                if (d + e < D) *reinterpret_cast<typename VecIO<T, 1>::Raw*>(dst + e) = pack<1>(x, T{});
            }
        }
    };
    if (lsplit == 0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = ty + 16 * i;
            if (row >= nrow) continue;
            const float l = s_l[row], inv = l == 0.f ? 0.f : 1.f / l;       // (no slot seen: the sums are zero)
#pragma unroll
            for (int c = 0; c < DCH; ++c) {
                float o[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = l == 0.f ? 0.f : acc[i][c][e] * inv;
                store(row, c * 64 + tx * 4, o);
            }
        }
        return;
    }
    // join: the sums go into shared memory (where the keys were), then every rank finishes the rows row % split == rank
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < DCH; ++c)
            *reinterpret_cast<float4*>(sk + (ty + 16 * i) * P + c * 64 + tx * 4) =
                make_float4(acc[i][c][0], acc[i][c][1], acc[i][c][2], acc[i][c][3]);
    cluster_arrive();
    cluster_wait();
    const int rows_mine = (nrow - rank + split - 1) >> lsplit;               // (none when rank >= nrow)
    for (int e = tid; e < rows_mine * DCH * 16; e += kSimpleThreads) {
        const int row = rank + (e / (DCH * 16) << lsplit), d = (e % (DCH * 16)) * 4;
        float m = -INFINITY;
        for (int p = 0; p < split; ++p) m = fmaxf(m, ld_cluster_f32(cluster_addr(smem_u32(s_m + row), p)));
        const float ref = m == -INFINITY ? 0.f : m;
        float l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
        for (int p = 0; p < split; ++p) {
            const float lp = ld_cluster_f32(cluster_addr(smem_u32(s_l + row), p));
            if (lp == 0.f) continue;                       // that rank saw nothing of the row
            const float f = exp2f(ld_cluster_f32(cluster_addr(smem_u32(s_m + row), p)) - ref);
            l = fmaf(f, lp, l);
            const uint32_t at = cluster_addr(smem_u32(sk + row * P + d), p);
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] = fmaf(f, ld_cluster_f32(at + 4 * c), o[c]);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] = l == 0.f ? 0.f : o[c] / l;
        store(row, d, o);
    }
    cluster_arrive();                                      // nobody leaves while its sums may be read
    cluster_wait();
}

template <typename T, int V, int DCH>
static cudaError_t launch_simple_t(const AttendArgs& a, cudaStream_t st) {
    const void* fn = reinterpret_cast<const void*>(k_attend_simple<T, V, DCH>);
    const size_t smem = SimpleShape<DCH>::FLOATS * sizeof(float);
    cudaError_t e = ensure_dynamic_smem(fn, smem);
    if (e != cudaSuccess) return e;
    const long long tiles = most_tiles(a, kSimpleRows, 0);
    // slots are shared until the CTAs fill the SMs twice, as long as a rank has four blocks of the longest sequence
    const long long slots = (long long)a.seq.table_pages * a.cache.page.d;
    const long long reach = (long long)a.window + a.seq.rows, longest = a.window > 0 && reach < slots ? reach : slots;
    int ls = 0;
    while (ls < 3 && (tiles * a.cache.heads << (ls + 1)) <= 2 * sm_count() && (longest >> (ls + 1)) >= 4 * kSimpleKeys) ++ls;
    if ((tiles << ls) > 0x7fffffffLL) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles << ls), a.cache.heads); cfg.blockDim = dim3(kSimpleThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1u << ls; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = ls ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, k_attend_simple<T, V, DCH>, a, ls);
}
template <typename T, int V> static cudaError_t launch_simple_v(const AttendArgs& a, cudaStream_t st) {
    switch ((a.cache.dim + 63) / 64) {
        case 1: return launch_simple_t<T, V, 1>(a, st);
        case 2: return launch_simple_t<T, V, 2>(a, st);
        case 3: return launch_simple_t<T, V, 3>(a, st);
        default: return launch_simple_t<T, V, 4>(a, st);
    }
}
static bool aligned_to(const void* p, long long s0, long long s1, long long s2, int V, size_t item) {
    return reinterpret_cast<uintptr_t>(p) % (V * item) == 0 && s0 % V == 0 && s1 % V == 0 && s2 % V == 0;
}
cudaError_t launch_attend_simple(const AttendArgs& a, int dtype, cudaStream_t st) {
    const size_t item = dtype == TTF_DTYPE_F32 ? 4 : 2;
    const bool four = a.cache.dim % 4 == 0 && aligned_to(a.q.data, a.q.row, a.q.head, 0, 4, item) &&
                      aligned_to(a.out.data, a.out.row, a.out.head, 0, 4, item) &&
                      aligned_to(a.cache.k, a.cache.k_page, a.cache.k_row, a.cache.k_head, 4, item) &&
                      aligned_to(a.cache.v, a.cache.v_page, a.cache.v_row, a.cache.v_head, 4, item);
    if (dtype == TTF_DTYPE_F32) return launch_simple_v<float, 1>(a, st);
    return four ? launch_simple_v<bf16_t, 4>(a, st) : launch_simple_v<bf16_t, 1>(a, st);
}

}  // namespace ttf

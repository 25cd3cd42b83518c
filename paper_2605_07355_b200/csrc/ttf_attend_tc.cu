// Attention of new rows over a paged cache on the fifth-generation tensor cores: bf16, heads of up to 128 channels.
//
//   S = Q K^T,  t = scale log2(e) S,  P = exp2(t - m),  O += P V,  l += sum P,  o = O / l
//
// The new tokens of a sequence times the query heads of a group are the rows of a tile (row = token * group + head), so that a
// group reads its keys and values once.  A CTA takes two tiles of up to 128 rows of one sequence and key head and walks their
// slots in blocks of (up to) 128:
//   warp 8       TMA: the pages of a block, keys then values, into a ring of [128 slots x DP channels] slots (128-byte swizzle;
//                channels beyond the head arrive as zeros)
//   warps 9, 10  tcgen05.mma, one thread per tile: S = Q K^T (both operands in shared memory), O += P V (P in tensor memory, V
//                read as the transposed operand)
//   warps 0 - 3  softmax of tile 0, one row per thread; warps 4 - 7 the same for tile 1
// While one tile's weights are formed the other tile's products run: O0 += P0 V(j), S0 = Q0 K(j+1)^T, O1 += P1 V(j),
// S1 = Q1 K(j+1)^T.  P takes the place of its scores in tensor memory, so the next scores of a tile are only asked for when the
// product before has completed; when scores arrive nobody touches O, and the softmax threads rescale it themselves.  They do so
// only where a maximum has grown by more than 8 (in powers of two: weights stay below 2^8, l and O carry the same factor, and
// nothing is lost, since bf16 and fp32 keep their relative precision), which after the first blocks is rare.
//
// Bound by the tensor pipe's operands and the chain of a tile together: half a block takes some 2090 cycles, of which a tile's
// softmax waits 600 for its scores and spends 40 on loading them, 290 on the maximum, 1000 on exponentials, sums and conversion;
// the thread that issues is held 1390 of them by its twelve products (those of the scores are 64 slots wide and so read Q from
// shared memory twice a block, 1.5 times what they multiply).  A CTA adds 6 us before its first scores and after its last.
// 4096 new rows over 16384 slots, 32 heads of 128: 1010 to 1025 us back to back, where the power cap holds the clock down (0.95
// PFLOP/s), 900 in bursts of 20 ms (1.07).  In such bursts slower were: scores handed over whole 1205, two threads a row 1022, one
// warp for both tiles' products 1330, an eighth of the exponentials on the fp32 pipe 917; scores and sums issued by two threads a
// tile made no difference.
//
// Rounded to fewer bits: the weights P, to bf16, since the second product takes its operands in 16 bits.  Each is off by half a step
// at most (2^-8 of its value), to either side; l adds up what they were before.  Against 64 bits the result is off by 0.0022 of its
// size, an fp32 evaluation rounded once by 0.0017.  ex2.approx is within 2 steps of fp32.
//
// Few tiles over many slots: the CTAs of a cluster share the blocks, and each finishes a part of the rows from what all of them
// send into its shared memory.
//
// Masks: only blocks that some row of the tile does not see whole are masked, by selection, whatever the keys hold.  Values of
// slots that no row of the CTA sees (stale rows of a page behind the length, slots before the window) are zeroed in shared memory.
//
// Every mbarrier wait is bounded; a wait that runs out is reported, the CTA's roles stop, wait (bounded) for their copies and
// products in flight, free the tensor memory and return.
#include <cuda.h>

#include "ttf_paged.cuh"
#include "ttf_async.cuh"
#include "ttf_cluster.cuh"
#include "ttf_tcgen05.cuh"
#include "ttf_tensormap.cuh"

namespace ttf {

constexpr int kAtRows = 128;                       // rows of a tile = tensor-memory lanes
constexpr int kAtSlots = 128;                      // slots of a block
constexpr int kAtHalf = 64;                        // slots whose scores and weights are handed over at a time
constexpr int kAtThreads = 352;

template <int DP> struct AttendShape {
    static constexpr int HALVES = DP / 64;                         // 128-byte columns of a row
    static constexpr int COL = 128 * 128;                          // bytes of one such column of 128 rows
    static constexpr int TILE = HALVES * COL;                      // a Q tile, a ring slot
    static constexpr int RING = DP == 128 ? 5 : 8;
    static constexpr int SMEM = 2 * TILE + RING * TILE;
    static constexpr int ML = 2 * kAtRows * DP;                    // what ranks send: [rank][tile][channel][row], then maxima, sums
    static constexpr uint32_t O_COL = 256;                         // tensor memory: S0 0, S1 128, O0, O1 from 256 on
    static_assert(SMEM + kMatchSmem > kSmShared && 2 * SMEM > kSmShared, "no other CTA with tensor memory fits beside this one");
};

struct AttendMaps { CUtensorMap q, k, v; };
struct AttendCut {
    Cut pair;                                      // the tokens of a CTA: two tiles
    Divisor block, group;                          // slots of a block, heads of a group
    int per_tile, box_rows, lsplit;                // tokens of a tile, rows of a TMA tile (a page or a part of one)
};

// D[tmem] (+)= A[tmem] . B[smem desc], issued by one thread
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
// operand whose rows (128 bytes: 64 elements along N, swizzled) run along K: 8-row groups 1024 bytes apart, the next 64
// elements of N `lead` bytes further
__device__ __forceinline__ uint64_t smem_desc_sw128_mn(uint32_t smem_addr, uint32_t lead) {
    return (smem_desc_sw128(smem_addr) & ~((uint64_t)0x3FFF << 16)) | ((uint64_t)(lead >> 4) << 16);
}
// bf16 x bf16 -> fp32, M = 128; b_mn: B runs along N
__host__ __device__ constexpr uint32_t idesc_attend(int n, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | (8u << 24);
}

__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int c0, int c1, int c2, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar))
        : "memory");
}

// 32 consecutive columns of this thread's tensor-memory lane
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
          "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
          "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
          "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
          "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
// the loads above have completed; the registers are operands of something behind the wait, so that nothing that reads them
// can be moved before it
template <int N> __device__ __forceinline__ void tmem_ld_wait(uint32_t (&r)[N]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; i += 8)
        asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]),
                          "+r"(r[i + 6]), "+r"(r[i + 7]) :: "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <int DP>
__global__ void __launch_bounds__(kAtThreads, 1)
k_attend_tc(const __grid_constant__ AttendMaps maps, const __grid_constant__ AttendArgs a, const __grid_constant__ AttendCut cut)
{
    using S = AttendShape<DP>;
    extern __shared__ unsigned char at_raw[];
    __shared__ uint64_t bar_q, bar_full[S::RING], bar_empty[S::RING], bar_raw, bar_s[2][2], bar_p[2][2], bar_pv[2], bar_o[2], bar_end;
    __shared__ uint32_t s_tmem;
    __shared__ int s_err;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int lsplit = cut.lsplit, per_tile = cut.per_tile, block = (int)cut.block.d, box_rows = cut.box_rows;
    const int split = 1 << lsplit, rank = lsplit ? (int)cluster_rank() : 0;
    const int work = blockIdx.x >> lsplit;
    const int hk = work % a.cache.heads;
    const int limit = a.wait_limit;

    // what does not depend on earlier work in the stream comes first
    const uint32_t base_addr = (smem_u32(at_raw) + 1023u) & ~1023u;
    unsigned char* const smem = at_raw + (base_addr - smem_u32(at_raw));
    if (warp == 8) {
        if (lane < S::RING) { mbar_init(&bar_full[lane], 1); mbar_init(&bar_empty[lane], 2); }
        if (lane == 0) {
            mbar_init(&bar_q, 1); mbar_init(&bar_raw, 1); mbar_init(&bar_end, 2);
            for (int x = 0; x < 2; ++x) {
                for (int b = 0; b < 2; ++b) { mbar_init(&bar_s[x][b], 1); mbar_init(&bar_p[x][b], 4); }
                mbar_init(&bar_pv[x], 1); mbar_init(&bar_o[x], 1);
            }
            s_err = 0;
            tensormap_prefetch(&maps.q); tensormap_prefetch(&maps.k); tensormap_prefetch(&maps.v);
        }
        mbar_init_fence();
    }
    // rows of the ring that no page fills (blocks of less than 128 slots): zero for good
    if (block < kAtSlots) {
        for (int col = 0; col < S::RING * S::HALVES; ++col)
            for (int o = block * 8 + tid; o < kAtSlots * 8; o += kAtThreads)
                *reinterpret_cast<uint4*>(smem + 2 * S::TILE + (size_t)col * S::COL + o * 16) = make_uint4(0, 0, 0, 0);
        fence_async_smem();
    }
    if (warp == 9) tmem_alloc(&s_tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;

    pdl_wait();
    Tile t;
    // (every CTA of a cluster has the same tile, and so the same answer)
    if (!find_tile(a, cut.pair, work / a.cache.heads, blockIdx.x == 0, t)) {
        if (warp == 9) tmem_dealloc(tmem, 512);
        return;
    }
    const SeqRange r = t.r;
    const int tok0 = t.tile * 2 * per_tile;                // first token of the CTA
    int ntok[2];
    ntok[0] = min(per_tile, r.n - tok0);
    ntok[1] = max(0, min(per_tile, r.n - tok0 - per_tile));

    // the blocks of this rank, and of each of its tiles
    const int tok_z = tok0 + ntok[0] + ntok[1] - 1;
    const int lo_u = seen_by(r, tok0, a.causal, a.window).lo, hi_u = seen_by(r, tok_z, a.causal, a.window).hi;
    const int b_lo = quotient(lo_u, cut.block), b_hi = hi_u > lo_u ? quotient(hi_u + block - 1, cut.block) : b_lo;
    const int j_lo = b_lo + (int)((long long)(b_hi - b_lo) * rank >> lsplit);
    const int j_hi = b_lo + (int)((long long)(b_hi - b_lo) * (rank + 1) >> lsplit);
    int jt_lo[2], jt_hi[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int ta = tok0 + x * per_tile;
        const int lo = seen_by(r, ta, a.causal, a.window).lo, hi = seen_by(r, ta + ntok[x] - 1, a.causal, a.window).hi;
        jt_lo[x] = max(j_lo, quotient(lo, cut.block));
        jt_hi[x] = ntok[x] > 0 && hi > lo ? min(j_hi, quotient(hi + block - 1, cut.block)) : 0;
        if (jt_hi[x] < jt_lo[x]) jt_hi[x] = jt_lo[x];
    }
    auto failed = [&]() { return *(volatile int*)&s_err != 0; };
    auto give_up = [&]() { atomicExch(&s_err, 1); };
    // (a role that gives up is noticed by the others, or their own waits run out)
    auto wait = [&](uint64_t* bar, int parity) {
        for (int i = 0; i < limit; ++i) {
            if (mbar_try_wait(bar, parity)) return true;
            if ((i & 63) == 63 && failed()) break;
        }
        give_up();
        return false;
    };

    int issued = 0, raw_at = -1;                           // warp 8: ring slots filled so far; phase of bar_raw that has not come
    if (warp == 8) {
        // ---- producer -------------------------------------------------------------------------------------------
        bool bad = false;
        if (lane == 0 && j_lo < j_hi) {
            const int tiles = ntok[1] > 0 ? 2 : 1;
            mbar_arrive_expect_tx(&bar_q, (uint32_t)(tiles * S::HALVES * per_tile * a.group * 128 + a.tx_extra));
            for (int x = 0; x < tiles; ++x)
                for (int h = 0; h < S::HALVES; ++h)
                    tma_load_3d(smem + x * S::TILE + h * S::COL, &maps.q, h * 64, hk * a.group, r.first + tok0 + x * per_tile, &bar_q);
        }
        const int* const table = a.seq.table + (long long)t.seq * a.seq.table_stride;
        const int page = (int)a.cache.page.d;
        int raw = 0;
        auto page_id = [&](int j) {                        // lane = page of the block (box_rows rows each)
            const int s0 = j * block + lane * box_rows;
            if (lane * box_rows >= block || j >= j_hi || s0 >= hi_u || s0 + box_rows <= lo_u) return -1;
            return page_of(table, quotient(s0, a.cache.page), a.cache.pages, bad);
        };
        int id = page_id(j_lo);
        for (int j = j_lo; j < j_hi; ++j) {
            const int next = page_id(j + 1);
            const uint32_t bytes = (uint32_t)(__popc(__ballot_sync(0xffffffffu, id >= 0)) * box_rows * 128 * S::HALVES);
            const int row = j * block + lane * box_rows - quotient(j * block + lane * box_rows, a.cache.page) * page;
            const int s0 = j * block;
            const bool edge = s0 < lo_u || s0 + block > hi_u;              // some slots are seen by no row of the CTA
            bool ok = true;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                const int idx = 2 * (j - j_lo) + kv, slot = idx % S::RING;
                ok = __all_sync(0xffffffffu, idx < S::RING || wait(&bar_empty[slot], ((idx / S::RING) & 1) ^ 1));
                if (!ok) break;
                uint64_t* const bar = kv && edge ? &bar_raw : &bar_full[slot];
                if (lane == 0) mbar_arrive_expect_tx(bar, bytes + (uint32_t)a.tx_extra);
                __syncwarp();
                unsigned char* const to = smem + 2 * S::TILE + slot * S::TILE;
                if (id >= 0) {
                    unsigned char* dst = to + lane * box_rows * 128;
                    const CUtensorMap* map = kv ? &maps.v : &maps.k;
#pragma unroll
                    for (int h = 0; h < S::HALVES; ++h) tma_load_4d(dst + h * S::COL, map, h * 64, row, hk, id, bar);
                }
                issued = idx + 1;
                if (kv && edge) {                          // their values: zeros, whatever the page (or an earlier block) holds
                    raw_at = raw & 1;
                    ok = __all_sync(0xffffffffu, wait(&bar_raw, raw_at));
                    if (!ok) break;
                    raw_at = -1;
                    ++raw;
                    const int head = max(0, lo_u - s0) * 8, tail = max(0, hi_u - s0) * 8;      // in 16-byte pieces
#pragma unroll
                    for (int h = 0; h < S::HALVES; ++h) {
                        for (int o = lane; o < head; o += 32) *reinterpret_cast<uint4*>(to + h * S::COL + o * 16) = make_uint4(0, 0, 0, 0);
                        for (int o = tail + lane; o < block * 8; o += 32) *reinterpret_cast<uint4*>(to + h * S::COL + o * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar_full + slot);
                }
            }
            if (!ok) break;
            id = next;
        }
        if (__any_sync(0xffffffffu, bad) && lane == 0) report_paged(a.hdr, 2);
    } else if (warp >= 9) {
        // ---- products: one thread per tile ------------------------------------------------------------------------
        if (lane == 0) {
            constexpr uint32_t id_s = idesc_attend(kAtHalf, false), id_o = idesc_attend(DP, true);
            const int x = warp - 9, t_lo = jt_lo[x], t_hi = jt_hi[x];
            const uint64_t dq = smem_desc_sw128(base_addr + x * S::TILE);
            const uint64_t dk0 = smem_desc_sw128(base_addr + 2 * S::TILE), dv0 = smem_desc_sw128_mn(base_addr + 2 * S::TILE, S::COL);
            // S = Q K^T of half a block's slots, keys in ring slot `at`
            auto scores = [&](int half, int at) {
                tc_fence_after();
                const uint64_t dk = dk0 + (uint64_t)((at * S::TILE + half * (kAtHalf * 128)) >> 4);
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    const uint64_t step = (uint64_t)(((k / 4) * S::COL + (k % 4) * 32) >> 4);
                    umma_bf16(tmem + x * 128 + half * kAtHalf, dq + step, dk + step, id_s, k > 0);
                }
                umma_commit(&bar_s[x][half]);
            };
            bool ok = j_lo < j_hi && wait(&bar_q, 0) && wait(&bar_full[0], 0);
            if (ok) {
                if (j_lo >= t_lo && j_lo < t_hi) { scores(0, 0); scores(1, 0); umma_commit(&bar_empty[0]); }
                else mbar_arrive(&bar_empty[0]);
            }
            int slot = 0, phase = 0;                       // keys of block j
            for (int j = j_lo; j < j_hi && ok; ++j) {
                int vs = slot + 1, vp = phase;             // its values
                if (vs == S::RING) { vs = 0; vp ^= 1; }
                slot = vs + 1; phase = vp;                 // the next block's keys
                if (slot == S::RING) { slot = 0; phase ^= 1; }
                const bool here = j >= t_lo && j < t_hi, next = j + 1 >= t_lo && j + 1 < t_hi;
                if (!(ok = wait(&bar_full[vs], vp))) break;
                if (!here) mbar_arrive(&bar_empty[vs]);
                const uint64_t dv = dv0 + (uint64_t)(vs * (S::TILE >> 4));
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (here) {                            // O += P V(j)
                        if (!(ok = wait(&bar_p[x][half], (j - t_lo) & 1))) break;
                        tc_fence_after();
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            umma_bf16_ts(tmem + S::O_COL + x * DP, tmem + x * 128 + half * kAtHalf + k * 8,
                                         dv + (uint64_t)((half * kAtHalf + k * 16) * 128 >> 4), id_o, k > 0 || half > 0 || j > t_lo);
                        umma_commit(&bar_pv[x]);
                        if (half) umma_commit(&bar_empty[vs]);
                    }
                    if (j + 1 < j_hi) {
                        if (half == 0 && !(ok = wait(&bar_full[slot], phase))) break;
                        // (P is in the place of S: the product has to be through before the next scores come there)
                        if (here && !(ok = wait(&bar_pv[x], half))) break;
                        if (next) scores(half, slot);
                        if (half) { if (next) umma_commit(&bar_empty[slot]); else mbar_arrive(&bar_empty[slot]); }
                    }
                }
            }
            umma_commit(&bar_o[x]);                        // (a barrier of its own: two phases of bar_pv may pass unseen)
            umma_commit(&bar_end);
        }
        __syncwarp();
    } else {
        // ---- softmax: one row per thread ----------------------------------------------------------------------------
        const int x = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t s_at = lanes + x * 128, o_at = lanes + S::O_COL + x * DP;
        const int nrow = ntok[x] * a.group;
        const Seen mine = row < nrow ? seen_by(r, tok0 + x * per_tile + quotient(row, cut.group), a.causal, a.window) : Seen{0, 0};
        // slots that every row of the tile sees
        const int all_lo = ntok[x] > 0 ? seen_by(r, tok0 + x * per_tile + ntok[x] - 1, a.causal, a.window).lo : 0;
        const int all_hi = ntok[x] > 0 ? seen_by(r, tok0 + x * per_tile, a.causal, a.window).hi : 0;
        const float c = a.scale * 1.4426950408889634f;
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        const int n = 2 * (jt_hi[x] - jt_lo[x]);           // halves of blocks
        for (int i = 0; i < n; ++i) {
            const int b = i & 1, parity = (i >> 1) & 1;
            if (!__all_sync(0xffffffffu, wait(&bar_s[x][b], parity))) { ok = false; break; }
            tc_fence_after();
            uint32_t s[kAtHalf];
            const uint32_t sb = s_at + b * kAtHalf;
            tmem_ld32(sb, s);
            tmem_ld32(sb + 32, s + 32);
            tmem_ld_wait(s);
            const int s0 = (jt_lo[x] + (i >> 1)) * block + b * kAtHalf;
            if (block < kAtSlots || s0 < all_lo || s0 + kAtHalf > all_hi) {
                const int lo = mine.lo - s0, hi = min(mine.hi - s0, block - b * kAtHalf);
#pragma unroll
                for (int e = 0; e < kAtHalf; ++e) s[e] = e >= lo && e < hi ? s[e] : 0xff800000u;
            }
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int e = 0; e < kAtHalf; e += 8)
#pragma unroll
                for (int y = 0; y < 4; ++y) mx[y] = max3(mx[y], __uint_as_float(s[e + 2 * y]), __uint_as_float(s[e + 2 * y + 1]));
            const float top = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]) * c;
            const bool grown = top > m + 8.f;              // (m = -inf: any number is)
            if (__any_sync(0xffffffffu, grown)) {
                const float m1 = grown ? top : m;
                const float f = m == m1 ? 1.f : exp2_approx(m - m1);
                m = m1;
                l *= f;
                if (i > 0) {                               // O, once the product of the half before has been added to it
                    if (!__all_sync(0xffffffffu, wait(&bar_pv[x], b ^ 1))) { ok = false; break; }
                    tc_fence_after();
#pragma unroll 1
                    for (int d = 0; d < DP; d += 32) {
                        uint32_t o[32];
                        tmem_ld32(o_at + d, o);
                        tmem_ld_wait(o);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                        tmem_st32(o_at + d, o);
                    }
                }
            }
            const float ref = m == -INFINITY ? 0.f : m;
            const Pair c2 = pair_of(c, c), ref2 = pair_of(-ref, -ref);
            Pair sum[2] = {0, 0};
            uint32_t p[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                const float2 t = both_of(fma2(pair_of(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])), c2, ref2));
                const float2 w = make_float2(exp2_approx(t.x), exp2_approx(t.y));
                sum[e & 1] = add2(sum[e & 1], pair_of(w.x, w.y));
                p[e] = bf16_pair(w.x, w.y);
            }
            tmem_st32(sb, p);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar_p[x][b]);
            const float2 both = both_of(add2(sum[0], sum[1]));
            l += both.x + both.y;
        }
        if (n > 0 && ok) wait(&bar_o[x], 0);               // O is complete
        if (n == 0 && j_lo < j_hi) wait(&bar_q, 0);        // (rows go out through the place of Q, which may still be on its way)
        __syncwarp();
        tc_fence_after();
        if (lsplit == 0) {
            // rows go out through the tile's own Q in shared memory (nobody reads it any more), so that a row leaves as a whole:
            // 16-byte piece q of row i lies at piece q ^ (i & 7)
            constexpr int PIECES = DP / 8;
            const float inv = l == 0.f ? 0.f : 1.f / l;
            unsigned char* const stage = smem + x * S::TILE + (warp & 3) * 32 * PIECES * 16;
#pragma unroll
            for (int i = 0; i < DP; i += 64) {
                uint32_t o[64];
                if (n > 0) { tmem_ld32(o_at + i, o); tmem_ld32(o_at + i + 32, o + 32); tmem_ld_wait(o); }
#pragma unroll
                for (int e = 0; e < 64; e += 8) {
                    uint4 w = make_uint4(0, 0, 0, 0);
                    if (n > 0 && l != 0.f) {
                        w.x = bf16_pair(__uint_as_float(o[e]) * inv, __uint_as_float(o[e + 1]) * inv);
                        w.y = bf16_pair(__uint_as_float(o[e + 2]) * inv, __uint_as_float(o[e + 3]) * inv);
                        w.z = bf16_pair(__uint_as_float(o[e + 4]) * inv, __uint_as_float(o[e + 5]) * inv);
                        w.w = bf16_pair(__uint_as_float(o[e + 6]) * inv, __uint_as_float(o[e + 7]) * inv);
                    }
                    *reinterpret_cast<uint4*>(stage + (lane * PIECES + (((i + e) / 8) ^ (lane & 7))) * 16) = w;
                }
            }
            __syncwarp();
            constexpr int ROWS = 32 / PIECES;              // rows at a time
            const int q = lane % PIECES;
            const bool on = q * 8 < a.cache.dim;
#pragma unroll 4
            for (int i = lane / PIECES; i < 32; i += ROWS) {
                const int at = (warp & 3) * 32 + i;
                const int token = quotient(at, cut.group), head = hk * a.group + at - token * a.group;
                const long long to = r.first + tok0 + x * per_tile + token;
                const uint4 w = *reinterpret_cast<const uint4*>(stage + (i * PIECES + (q ^ (i & 7))) * 16);
                if (on && at < nrow && in_bounds(a.hdr, 8, to, a.seq.rows))
                    *reinterpret_cast<uint4*>(reinterpret_cast<bf16_t*>(a.out.data) + to * a.out.row + (long long)head * a.out.head + q * 8) = w;
            }
        } else {
            // Every rank finishes 1 / split of the rows of both tiles: when all of them are through with their shared memory, rank p's
            // rows p * each .. + each - 1 are sent there from all ranks, channel by channel, so that the lanes of a warp write
            // consecutive words (16 bytes of a row per lane travel as 32 packets: 10000 cycles for 128 KB).
            const int each = kAtRows >> lsplit, to = row >> (7 - lsplit), col = row & (each - 1);
            __syncwarp();
            cluster_arrive();
            cluster_wait();
            const uint32_t ml = cluster_addr(base_addr + (uint32_t)(S::ML + (rank * 2 + x) * each + col) * 4, to);
            st_cluster_f32(ml, m);
            st_cluster_f32(ml + 2 * kAtRows * 4, l);
            if (n > 0) {
                const uint32_t at = cluster_addr(base_addr + (uint32_t)((rank * 2 + x) * DP * each + col) * 4, to);
#pragma unroll
                for (int i = 0; i < DP; i += 32) {
                    uint32_t o[32];
                    tmem_ld32(o_at + i, o);
                    tmem_ld_wait(o);
#pragma unroll
                    for (int e = 0; e < 32; ++e) st_cluster_u32(at + (uint32_t)((i + e) * each * 4), o[e]);
                }
            }
        }
    }
    pdl_launch_dependents();

    if (lsplit) {
        __syncwarp();
        if (warp >= 8) { cluster_arrive(); cluster_wait(); }               // (the softmax warps were there before they sent)
        cluster_arrive();
        cluster_wait();
        const int each = kAtRows >> lsplit, rows2 = 2 * each;
        const float* const f = reinterpret_cast<const float*>(smem);
        for (int e = tid; e < rows2 * (DP / 8); e += kAtThreads) {
            const int i = e & (rows2 - 1), d = (e >> (8 - lsplit)) * 8;   // row i of the rank's: tile i / each
            const int x = i >= each, col = i - x * each, row = rank * each + col;
            if (row >= ntok[x] * a.group || d >= a.cache.dim) continue;
            float mx = -INFINITY;
#pragma unroll 4
            for (int p = 0; p < split; ++p) mx = fmaxf(mx, f[S::ML + p * rows2 + i]);
            const float ref = mx == -INFINITY ? 0.f : mx;
            float l = 0.f, o[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) o[c] = 0.f;
#pragma unroll 2
            for (int p = 0; p < split; ++p) {
                const float lp = f[S::ML + 2 * kAtRows + p * rows2 + i], w = exp2_approx(f[S::ML + p * rows2 + i] - ref);
                if (lp == 0.f) continue;                   // that rank saw nothing of the row
                const float* const v = f + (p * 2 + x) * DP * each + d * each + col;
                l = fmaf(w, lp, l);
#pragma unroll
                for (int c = 0; c < 8; ++c) o[c] = fmaf(w, v[c * each], o[c]);
            }
            const float inv = l == 0.f ? 0.f : 1.f / l;
            const int in_tile = quotient(row, cut.group), token = tok0 + x * per_tile + in_tile, head = hk * a.group + row - in_tile * a.group;
            uint4 w = make_uint4(0, 0, 0, 0);
            if (l != 0.f)
                w = make_uint4(bf16_pair(o[0] * inv, o[1] * inv), bf16_pair(o[2] * inv, o[3] * inv), bf16_pair(o[4] * inv, o[5] * inv),
                               bf16_pair(o[6] * inv, o[7] * inv));
            if (in_bounds(a.hdr, 8, (long long)r.first + token, a.seq.rows))
                *reinterpret_cast<uint4*>(reinterpret_cast<bf16_t*>(a.out.data) + (long long)(r.first + token) * a.out.row + (long long)head * a.out.head + d) = w;
        }
    }
    tc_fence_before();
    __syncthreads();                                       // (from here on nobody gives up any more)
    if (warp == 8 && s_err) {                              // copies in flight land before the CTA may leave
        if (j_lo < j_hi) mbar_wait(&bar_q, 0, limit);
        if (raw_at >= 0) { mbar_wait(&bar_raw, raw_at, limit); --issued; }           // (that slot is never declared full)
        for (int i = issued > S::RING ? issued - S::RING : 0; i < issued; ++i)
            mbar_wait(&bar_full[i % S::RING], (i / S::RING) & 1, limit);
    }
    if (warp == 9) {
        tc_fence_after();
        if (s_err) mbar_wait(&bar_end, 0, limit);          // products in flight end before their accumulators are given back
        __syncwarp();
        tmem_dealloc(tmem, 512);
    }
    if (tid == 0 && s_err) report_paged(a.hdr, 1);
}

// ---- host side ------------------------------------------------------------------------------------------------------
// an axis of `n` elements, `s` elements apart, that a map can have: a broadcast axis (no step between its elements) it cannot
static bool axis_ok(long long n, long long s) { return (n == 1 || s > 0) && s >= 0 && s % 8 == 0 && s < (1LL << 38); }
static bool rows_fit(const HeadsView& h, int rows) {
    return reinterpret_cast<uintptr_t>(h.data) % 16 == 0 && axis_ok(rows, h.row) && axis_ok(h.heads, h.head);
}
bool cache_maps_fit(const AttendArgs& a) {
    const CacheView& c = a.cache;
    auto fit = [&](const void* p, long long page, long long row, long long head) {
        return reinterpret_cast<uintptr_t>(p) % 16 == 0 && axis_ok(c.pages, page) && axis_ok(c.page.d, row) && axis_ok(c.heads, head);
    };
    return fit(c.k, c.k_page, c.k_row, c.k_head) && fit(c.v, c.v_page, c.v_row, c.v_head) && encode_fn() != nullptr;
}

bool attend_tc_takes(const AttendArgs& a, int dtype) {
    const int page = (int)a.cache.page.d;
    return dtype == TTF_DTYPE_BF16 && a.cache.dim % 8 == 0 && a.cache.dim <= 128 && a.group <= kAtRows && a.scale > 0.f &&
           page % 8 == 0 && (page <= kAtSlots || page % kAtSlots == 0) &&
           rows_fit(a.q, a.seq.rows) && rows_fit(a.out, a.seq.rows) && cache_maps_fit(a);
}

// a map over axes of `n` elements with strides of `s` elements (0: an axis of one element, whose stride does not matter)
static bool encode(CUtensorMap* m, const void* data, int rank, const long long* n, const long long* s, const int* box) {
    cuuint64_t dims[4], strides[3];
    cuuint32_t bx[4], one[4] = {1, 1, 1, 1};
    for (int i = 0; i < rank; ++i) { dims[i] = (cuuint64_t)n[i]; bx[i] = (cuuint32_t)box[i]; }
    for (int i = 1; i < rank; ++i) strides[i - 1] = (cuuint64_t)(s[i] > 0 ? s[i] * 2 : 16);
    return encode_fn()(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(data), dims, strides, bx, one,
                       CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool make_cache_map(CUtensorMap* m, const AttendArgs& a, bool values, int rows) {
    const long long n[4] = {a.cache.dim, (int)a.cache.page.d, a.cache.heads, a.cache.pages};
    const long long s[4] = {1, values ? a.cache.v_row : a.cache.k_row, values ? a.cache.v_head : a.cache.k_head, values ? a.cache.v_page : a.cache.k_page};
    const int b[4] = {64, rows, 1, 1};
    return encode(m, values ? a.cache.v : a.cache.k, 4, n, s, b);
}

template <int DP> static cudaError_t launch_tc_t(const AttendArgs& a, cudaStream_t st) {
    using S = AttendShape<DP>;
    const int page = (int)a.cache.page.d, per = kAtRows / a.group;
    const int block = page < kAtSlots ? kAtSlots / page * page : kAtSlots, box = page < kAtSlots ? page : kAtSlots;
    AttendMaps maps;
    {
        const long long n[3] = {a.cache.dim, a.q.heads, a.seq.rows}, s[3] = {1, a.q.head, a.q.row};
        const int b[3] = {64, a.group, per};
        if (!encode(&maps.q, a.q.data, 3, n, s, b)) return cudaErrorInvalidValue;
    }
    if (!make_cache_map(&maps.k, a, false, box) || !make_cache_map(&maps.v, a, true, box)) return cudaErrorInvalidValue;
    const void* fn = reinterpret_cast<const void*>(k_attend_tc<DP>);
    const size_t smem = S::SMEM + 1024;
    cudaError_t e = ensure_dynamic_smem(fn, smem);
    if (e != cudaSuccess) return e;
    const long long ctas = most_tiles(a, 0, 2 * per) * a.cache.heads;
    const long long slots = (long long)a.seq.table_pages * page;
    const long long reach = (long long)a.window + a.seq.rows, longest = a.window > 0 && reach < slots ? reach : slots;
    // CTAs (a power of two) that share the slots of a pair of tiles.  A join costs 8 to 11 us (distributed shared memory takes in
    // some 14 bytes per clock, and the partial rows are 128 KB), a block of 128 slots 1.9 us.  Where the CTAs do not fill the SMs
    // shares go down to 512 slots (65 rows over 4000 slots, 8 key heads: 71 us alone, 49 / 33 shared by 2 / 8; over 1024 slots 23.2
    // and 25.4 / 21.8); where they do, two share sequences of more than 8192 slots, whose CTAs would be long against the call (6
    // sequences of 60 - 900 new rows over 400 - 12000, 2 key heads: 188 / 103 / 127 us with 1 / 2 / 4; 4096 new rows over 16384, 8 key
    // heads: 937 / 891 / 1108; 2760 new rows alone 84 / 133 / 227).
    int ls = 0;
    while (ls < 3 && (ctas << (ls + 1)) <= sm_count() && longest >= 2048 && (longest >> (ls + 1)) >= 512) ++ls;
    if (ls == 0 && longest >= 8192) ls = 1;
    if ((ctas << ls) > 0x7fffffffLL) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(ctas << ls)); cfg.blockDim = dim3(kAtThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1u << ls; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = ls ? 2 : 1;
    AttendCut cut = {cut_tokens(2 * per), make_divisor(block), make_divisor(a.group), per, box, ls};
    return cudaLaunchKernelEx(&cfg, k_attend_tc<DP>, maps, a, cut);
}
cudaError_t launch_attend_tc(const AttendArgs& a, cudaStream_t st) {
    return a.cache.dim <= 64 ? launch_tc_t<64>(a, st) : launch_tc_t<128>(a, st);
}

}  // namespace ttf

// Norms of queries and keys for each head, the rotation by the row's position, and the append of keys and values to the
// pages of a cache: one pass over the heads of a row.
//
//   y = x * w / sqrt(mean(x^2) + eps);   (u, v) -> factor * (u cos a - v sin a, v cos a + u sin a),   a = p[axis(j)] * freq[j]
//
// Bound by memory: every head is read once, kept in registers between the sum of squares and the rotation, and written
// once.  All heads of a row turn by the same angles, so a CTA takes whole rows: its first rot / 2 threads form the row's
// cosines and sines in shared memory (in turns, in 64 bits: an fp32 product loses the turn from positions of about 10^4
// on) while the heads' loads are in flight.  A head is an item of two V-channel vectors per lane (for the half layout the
// two halves of V pairs), the lanes of a head are the power of two that covers it, and a warp holds 32 / lanes heads.
// CTAs walk the rows with a stride, so that the worst-case capacity behind a count that only the device knows costs nothing;
// where there are fewer rows than places the heads of a row are spread over several CTAs.
#include "ttf_paged.cuh"

namespace ttf {

constexpr int kRotThreads = 256;

// NI items per lane (more than one only where a head has more items than a warp has lanes)
template <int V> struct Items { static constexpr int PER_LANE = kMaxDim / (2 * V) > 32 ? kMaxDim / (2 * V) / 32 : 1; };

// Where the two vectors of item `it` start.  Rotated items first (half layout: V pairs, so that the vectors are half a
// rotation apart; interleaved: consecutive), then consecutive channels.  Items are 2 V channels; the last one may reach
// beyond an odd head, which only V = 1 takes.
template <int V> __device__ __forceinline__ void item_at(int it, int rot, int interleaved, int& e0, int& e1) {
    const bool halves = !interleaved && it * 2 * V < rot;
    e0 = halves ? it * V : it * 2 * V;
    e1 = halves ? rot / 2 + it * V : e0 + V;
}

template <typename T, int V, bool APPEND>
__global__ void __launch_bounds__(kRotThreads)
k_rotate(const __grid_constant__ RotateArgs a, int lanes)
{
    using IO = VecIO<T, V>;
    using Raw = typename IO::Raw;
    constexpr int NI = Items<V>::PER_LANE;
    __shared__ float2 s_turn[2][kMaxDim / 2];
    const int tid = threadIdx.x, lane = tid & (lanes - 1);
    const int groups = kRotThreads / lanes, grp = tid / lanes;
    const int D = a.dim, rot = a.rot, pairs = rot >> 1;
    const int nitems = (D + 2 * V - 1) / (2 * V);
    const int Hq = a.q.heads, Hk = a.k.heads, heads = Hq + Hk + (APPEND ? a.v.heads : 0);
    // this CTA's heads
    const int h0 = (int)((long long)heads * blockIdx.y / gridDim.y), h1 = (int)((long long)heads * (blockIdx.y + 1) / gridDim.y);

    pdl_wait();
    int n = a.rows;
    if (APPEND) n = min(n, max(0, __ldcg(a.seq.start + a.seq.seqs)));
    else if (a.count) n = min(n, max(0, __ldcg(a.count)));

    // the coordinate that this thread's pair turns with
    int axis = 0;
    double freq = 0.0;
    if (tid < pairs) {
        freq = (double)__ldcg(a.freq + tid) * 0.15915494309189533577;          // turns per position
        if (a.axes > 1) {
            if (a.cyclic) {
                const int m = tid % a.axes;
                axis = m > 0 && tid / a.axes < (m == 1 ? a.sec1 : a.sec2) ? m : 0;
            } else axis = tid < a.sec0 ? 0 : (tid < a.sec0 + a.sec1 ? 1 : 2);
        }
    }

    int buf = 0;
    for (int row = blockIdx.x; row < n; row += gridDim.x, buf ^= 1) {
        // where the row's keys and values go
        long long k_at = 0, v_at = 0;
        bool stored = false, there = true;
        if (APPEND) {
            int b = 0;                                     // sequences that end at or before this row
            for (int s = (tid & 31); s - (tid & 31) < a.seq.seqs; s += 32)
                b += __popc(__ballot_sync(0xffffffffu, s < a.seq.seqs && __ldcg(a.seq.start + s + 1) <= row));
            SeqRange r = {0, 0, 0, false};
            if (b < a.seq.seqs) r = seq_range(a.seq, b, a.cache.page);
            const int i = row - r.first;
            there = r.ok && i >= 0 && i < r.n;
            bool bad = !there;
            const int slot = r.length - r.n + i;
            if (there && slot >= 0) {
                const int index = quotient(slot, a.cache.page);
                const int g = page_of(a.seq.table + (long long)b * a.seq.table_stride, index, a.cache.pages, bad);
                const int in_page = slot - index * (int)a.cache.page.d;
                k_at = g * a.cache.k_page + in_page * a.cache.k_row;
                v_at = g * a.cache.v_page + in_page * a.cache.v_row;
                stored = !bad && in_bounds(a.hdr, 7, (long long)g * a.cache.page.d + in_page, (long long)a.cache.pages * a.cache.page.d);
            }
            if (bad && tid == 0) report_paged(a.hdr, 2);
        }
        if (tid < pairs) {
            const double turn = (double)__ldcg(a.pos + (long long)row * a.axes + axis) * freq;
            float c, s;
            sincospif((float)(2.0 * (turn - rint(turn))), &s, &c);
            s_turn[buf][tid] = make_float2(c * a.factor, s * a.factor);
        }
        bool synced = false;                               // (the heads' loads are issued before the barrier)
        for (int hb = h0; hb < h1; hb += groups) {
            const int h = hb + grp;
            const bool on = h < h1 && there;
            const int kind = h < Hq ? 0 : (h < Hq + Hk ? 1 : 2);
            const HeadsView& in = kind == 0 ? a.q : (kind == 1 ? a.k : a.v);
            const int hh = h - (kind == 0 ? 0 : (kind == 1 ? Hq : Hq + Hk));
            const T* src = reinterpret_cast<const T*>(in.data) + (long long)row * in.row + (long long)hh * in.head;
            Raw ra[NI][2];
            int e[NI][2];
#pragma unroll
            for (int u = 0; u < NI; ++u) {
                const int it = lane + u * 32;
                item_at<V>(it, kind == 2 ? 0 : rot, a.interleaved, e[u][0], e[u][1]);
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    ra[u][w] = Raw{};
                    if (on && it < nitems && e[u][w] < D) ra[u][w] = load_cg(reinterpret_cast<const Raw*>(src + e[u][w]));
                }
            }
            if (!synced) { __syncthreads(); synced = true; }
            T* dst = nullptr;                              // NULL: nothing to store
            if (on && in_bounds(a.hdr, 6, (long long)row * heads + h, (long long)a.rows * heads)) {
                if (kind == 0) dst = reinterpret_cast<T*>(a.out_q.data) + (long long)row * a.out_q.row + (long long)hh * a.out_q.head;
                else if (!APPEND) dst = reinterpret_cast<T*>(a.out_k.data) + (long long)row * a.out_k.row + (long long)hh * a.out_k.head;
                else if (stored) dst = kind == 1 ? reinterpret_cast<T*>(a.cache.k) + k_at + (long long)hh * a.cache.k_head
                                                 : reinterpret_cast<T*>(a.cache.v) + v_at + (long long)hh * a.cache.v_head;
            }
            const void* weight = kind == 0 ? a.q_weight : (kind == 1 ? a.k_weight : nullptr);
            float x[NI][2][V];
            float ssq = 0.f;
#pragma unroll
            for (int u = 0; u < NI; ++u)
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    unpack<V>(ra[u][w], x[u][w], T{});
#pragma unroll
                    for (int c = 0; c < V; ++c) ssq = fmaf(x[u][w][c], x[u][w][c], ssq);
                }
            if (a.q_weight || a.k_weight) {                // (uniform over the warp: its heads may be of both kinds)
                for (int o = lanes >> 1; o > 0; o >>= 1) ssq += __shfl_xor_sync(0xffffffffu, ssq, o);
            }
            if (weight) {
                const float inv = 1.0f / sqrtf(ssq / (float)D + a.eps);
#pragma unroll
                for (int u = 0; u < NI; ++u)
#pragma unroll
                    for (int w = 0; w < 2; ++w)
                        if (lane + u * 32 < nitems && e[u][w] < D) {
                            float wt[V];
                            unpack<V>(load_cg(reinterpret_cast<const Raw*>(reinterpret_cast<const T*>(weight) + e[u][w])), wt, T{});
#pragma unroll
                            for (int c = 0; c < V; ++c) x[u][w][c] *= inv * wt[c];
                        }
            }
            if (kind != 2) {
#pragma unroll
                for (int u = 0; u < NI; ++u) {
                    if (a.interleaved) {
                        // flat channel c of the item's 2 V: pairs of neighbours
#pragma unroll
                        for (int c = 0; c < 2 * V; c += 2) {
                            if (e[u][0] + c >= rot) continue;
                            float& p0 = x[u][c / V][c % V];
                            float& p1 = x[u][(c + 1) / V][(c + 1) % V];
                            const float2 t = s_turn[buf][(e[u][0] + c) >> 1];
                            const float a0 = p0, a1 = p1;
                            p0 = a0 * t.x - a1 * t.y;
                            p1 = a1 * t.x + a0 * t.y;
                        }
                    } else if (e[u][0] < pairs && e[u][1] == pairs + e[u][0]) {
#pragma unroll
                        for (int c = 0; c < V; ++c) {
                            const float2 t = s_turn[buf][e[u][0] + c];
                            const float a0 = x[u][0][c], a1 = x[u][1][c];
                            x[u][0][c] = a0 * t.x - a1 * t.y;
                            x[u][1][c] = a1 * t.x + a0 * t.y;
                        }
                    }
                }
            }
            if (dst) {
#pragma unroll
                for (int u = 0; u < NI; ++u)
#pragma unroll
                    for (int w = 0; w < 2; ++w)
                        if (lane + u * 32 < nitems && e[u][w] < D)
                            *reinterpret_cast<Raw*>(dst + e[u][w]) = kind == 2 ? ra[u][w] : pack<V>(x[u][w], T{});
            }
        }
        if (!synced) __syncthreads();
    }
    pdl_launch_dependents();
}

// The widest vectors that heads, strides and the rotation's halves are made of.
static bool fits(const HeadsView& h, int V, size_t item) {
    return !h.data || (reinterpret_cast<uintptr_t>(h.data) % (V * item) == 0 && h.row % V == 0 && h.head % V == 0);
}
template <typename T, bool APPEND, int V>
static cudaError_t launch_rotate_v(const RotateArgs& a, cudaStream_t st) {
    const size_t item = sizeof(T);
    bool ok = a.dim % (2 * V) == 0 && (a.interleaved || (a.rot / 2) % V == 0);
    for (const HeadsView* h : {&a.q, &a.k, &a.v, &a.out_q, &a.out_k}) ok = ok && fits(*h, V, item);
    for (const void* w : {a.q_weight, a.k_weight}) ok = ok && reinterpret_cast<uintptr_t>(w) % (V * item) == 0;
    if (APPEND) {
        ok = ok && fits(HeadsView{a.cache.k, a.cache.k_row, a.cache.k_head, 0}, V, item) && a.cache.k_page % V == 0 &&
             fits(HeadsView{a.cache.v, a.cache.v_row, a.cache.v_head, 0}, V, item) && a.cache.v_page % V == 0;
    }
    if constexpr (V > 1) {
        if (!ok) return launch_rotate_v<T, APPEND, V / 2>(a, st);
    }
    int lanes = 1;
    while (lanes < 32 && lanes * 2 * V < a.dim) lanes *= 2;
    const int heads = a.q.heads + a.k.heads + (APPEND ? a.v.heads : 0), groups = kRotThreads / lanes;
    const int places = sm_count() * 6;
    const int most = (heads + groups - 1) / groups;        // CTAs that can share a row
    int split = places / a.rows;
    if (split > most) split = most;
    if (split < 1) split = 1;
    const int gx = a.rows < places ? a.rows : places;
    return launch_pdl(k_rotate<T, V, APPEND>, dim3(gx, split), dim3(kRotThreads), st, a, lanes);
}
cudaError_t launch_rotate(const RotateArgs& a, int dtype, bool append, cudaStream_t st) {
    if (a.rows < 1) return cudaSuccess;
    if (dtype == TTF_DTYPE_BF16)
        return append ? launch_rotate_v<bf16_t, true, 8>(a, st) : launch_rotate_v<bf16_t, false, 8>(a, st);
    return append ? launch_rotate_v<float, true, 4>(a, st) : launch_rotate_v<float, false, 4>(a, st);
}

}  // namespace ttf

// Norms of queries and keys for each head, the rotation by the row's position, and the append of keys and values to the
// pages of a cache: one pass over the heads of a row.
//
//   y = x * w / sqrt(mean(x^2) + eps);   (u, v) -> factor * (u cos a - v sin a, v cos a + u sin a),   a = p[axis(j)] * freq[j]
//
// Bound by memory: every head is read once, kept in registers between the sum of squares and the rotation, and written
// once.  All heads of a row turn by the same angles, so a warp takes a row (or, where there are fewer rows than warps, a
// part of a row's heads): its lanes form the row's cosines and sines once (in turns, in 64 bits: an fp32 product loses the
// turn from positions of about 10^4 on) and hand them round through shared memory; then each lane keeps the turns of its
// channels, multiplied with the norm's weight, in registers for all heads:
//   u' = inv (x_u (w_u c) - x_v (w_v s)),   v' = inv (x_v (w_v c) + x_u (w_u s)).
// (Turns and weights re-read from shared memory for every head cost as much as the rest: with CTAs that share rows the
// clip of 2703 rows, 32 + 8 heads of 128 took 21.7 us, 12.0 without norm and rotation; this form 14.5.)  A head is an item of
// two V-channel vectors per lane (for the half layout the two halves of V pairs), the lanes of a head are the power of two
// that covers it, and a warp holds 32 / lanes heads; the next heads are on their way while the present ones are worked on.
// Rows are dealt out to the warps by the number that only the device knows, so worst-case buffers cost nothing.
#include "ttf_paged.cuh"

#include <climits>
#include <type_traits>

namespace ttf {

constexpr int kRotThreads = 128;
constexpr int kRotCtas = 5;                        // per SM
constexpr int kRotParts = 64;                      // parts of a row's heads at most

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

// the sum over the lanes of a head
__device__ __forceinline__ float head_sum(float x, int lanes, int llanes) {
    if (llanes == 3) {                                     // (heads of 128 channels in bf16)
        x += __shfl_xor_sync(0xffffffffu, x, 4);
        x += __shfl_xor_sync(0xffffffffu, x, 2);
        x += __shfl_xor_sync(0xffffffffu, x, 1);
    } else
        for (int o = lanes >> 1; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// FULL: the lanes of a head hold exactly its channels
template <typename T, int V, bool APPEND, bool INTER, bool FULL>
__global__ void __launch_bounds__(kRotThreads, kRotCtas)
k_rotate(const __grid_constant__ RotateArgs a, int llanes)
{
    using Raw = typename VecIO<T, V>::Raw;
    constexpr int NI = Items<V>::PER_LANE;
    constexpr int AHEAD = 2;                               // heads of a lane on their way
    __shared__ float2 s_turn[kRotThreads / 32][kMaxDim / 2];
    const int ln = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int lanes = 1 << llanes, lane = ln & (lanes - 1), sub = ln >> llanes, per_warp = 32 >> llanes;
    const int D = a.dim, rot = a.rot, pairs = rot >> 1;
    const int nitems = (D + 2 * V - 1) / (2 * V);
    const int Hq = a.q.heads, Hk = a.k.heads, heads = Hq + Hk + (APPEND ? a.v.heads : 0);
    float2* const turn = s_turn[warp];

    int e[NI][2];                                          // this lane's channels
    bool in[NI][2], turned[NI];
#pragma unroll
    for (int u = 0; u < NI; ++u) {
        item_at<V>(lane + u * 32, rot, INTER, e[u][0], e[u][1]);
        in[u][0] = FULL ? u == 0 : lane + u * 32 < nitems && e[u][0] < D;
        in[u][1] = FULL ? u == 0 : lane + u * 32 < nitems && e[u][1] < D;
        turned[u] = in[u][0] && e[u][0] < rot;
    }
    pdl_wait();
    int n = a.rows, beyond = 0;
    // append: every step-th sequence's rows [first, end), one per lane
    [[maybe_unused]] const int step0 = (a.seq.seqs + 31) >> 5;
    [[maybe_unused]] int first0 = INT_MAX, end0 = 0;
    auto sequence_rows = [&](int s, int& first, int& end) { first = __ldcg(a.seq.start + s); end = __ldcg(a.seq.start + s + 1); };
    auto claims = [&](int first, int end, int row) { return first >= 0 && first <= row && row < end && end <= a.rows; };
    if (APPEND) {
        if (ln * step0 < a.seq.seqs) sequence_rows(ln * step0, first0, end0);
        // rows up to the last one that is claimed; of more than 32 sequences up to the last start, which is that where none goes back
        // (one more load than up to 32 need: append_streams 11.2 us so, 11.9 with the last start throughout)
        if (step0 == 1) n = __reduce_max_sync(0xffffffffu, claims(first0, end0, first0) ? end0 : 0);
        else n = min(n, max(0, __ldcg(a.seq.start + a.seq.seqs)));
        // The warp that has the least to do looks at all sequences, and reports what is wrong with any.  Rows beyond n that a sequence
        // claims all the same are its own.
        if (blockIdx.x == gridDim.x - 1 && warp == kRotThreads / 32 - 1) {
            bool bad = false;
            int last = 0;
            for (int s = ln; s < a.seq.seqs; s += 32) {
                int first, end;
                sequence_rows(s, first, end);
                bad |= !seq_range(a.seq, s, a.cache.page).ok;
                if (end > first && claims(first, end, first)) last = max(last, end);
            }
            if (bad) report_paged(a.hdr, 2);
            beyond = max(0, __reduce_max_sync(0xffffffffu, last) - n);
        }
    } else if (a.count) n = min(n, max(0, __ldcg(a.count)));

    const int warps = gridDim.x * (kRotThreads / 32);
    int parts = 1;                                         // of a row's heads
    if (n > 0 && n < warps) parts = min(min(warps / n, (heads + per_warp - 1) / per_warp), kRotParts);
    const int units = n * parts;
    // (without a sign: units may be as many as 2^31 - 1, and a warp counts one step beyond them)
    for (unsigned at = warp * gridDim.x + blockIdx.x; ; at += warps) {
        int row, h0 = 0, h1 = heads;
        if (at < (unsigned)units) {
            const int unit = (int)at;
            row = parts > 1 ? unit / parts : unit;
            if (parts > 1) {
                const int part = unit - row * parts;
                h0 = heads * part / parts; h1 = heads * (part + 1) / parts;
            }
        } else if (APPEND && beyond > 0) {
            row = n + --beyond;
            at -= warps;
        } else break;

        bool have = false;
        auto make_turns = [&]() {                          // cosine and sine of the row's pairs, for all lanes
            __syncwarp();
#pragma unroll 1
            for (int j = ln; j < pairs; j += 32) {
                int axis = 0;
                if (a.axes > 1) {
                    if (a.cyclic) {
                        const int of = a.axes == 2 ? j >> 1 : j / 3, m = j - of * a.axes;
                        axis = m > 0 && of < (m == 1 ? a.sec1 : a.sec2) ? m : 0;
                    } else axis = j < a.sec0 ? 0 : (j < a.sec0 + a.sec1 ? 1 : 2);
                }
                const double w = (double)__ldcg(a.pos + (long long)row * a.axes + axis) * ((double)__ldcg(a.freq + j) * 0.15915494309189533577);
                // (what is left of the turn, half a turn at most, is rounded to fp32: the angle is off by pi 2^-25 at most)
                float c, s;
                sincospif((float)(2.0 * (w - rint(w))), &s, &c);
                turn[j] = make_float2(c * a.factor, s * a.factor);
            }
            __syncwarp();
        };

        // where the row's keys and values go
        long long k_at = 0, v_at = 0;
        bool there = true, stored = false;
        auto find_place = [&]() {
            // the sequence that claims this row: 32 starts at a time, as long as they do not go back
            int lo = 0, step = step0, first = first0, end = end0;
            while (step > 1) {
                const unsigned upto = __ballot_sync(0xffffffffu, first <= row);
                lo += upto ? (31 - __clz(upto)) * step : 0;
                const int left = min(step, a.seq.seqs - lo);
                step = (left + 31) >> 5;
                first = INT_MAX;
                if (ln * step < left) sequence_rows(lo + ln * step, first, end);
            }
            unsigned found = __ballot_sync(0xffffffffu, claims(first, end, row));
            if (!found && step0 > 1)                       // a row of no sequence, or starts that go back somewhere: look at all
                for (lo = 0; lo < a.seq.seqs; lo += 32) {
                    first = INT_MAX;
                    if (lo + ln < a.seq.seqs) sequence_rows(lo + ln, first, end);
                    found = __ballot_sync(0xffffffffu, claims(first, end, row));
                    if (found) break;
                }
            const int src = __ffs(found) - 1, b = lo + src;
            there = found != 0;
            int slot = -1;
            if (there) {
                end = __shfl_sync(0xffffffffu, end, src);
                const int length = __ldcg(a.seq.length + b);
                there = length_fits(a.seq, length, a.cache.page);
                slot = length - end + row;
            }
            bool bad = false;
            if (there && slot >= 0) {
                const int index = quotient(slot, a.cache.page);
                const long long g = page_of(a.seq.table + (long long)b * a.seq.table_stride, index, a.cache.pages, bad);
                const int in_page = slot - index * (int)a.cache.page.d;
                k_at = g * a.cache.k_page + in_page * a.cache.k_row;
                v_at = g * a.cache.v_page + in_page * a.cache.v_row;
                stored = !bad && in_bounds(a.hdr, 7, g * a.cache.page.d + in_page, (long long)a.cache.pages * a.cache.page.d);
            }
            if (bad && ln == 0) report_paged(a.hdr, 2);
        };

        // kinds: 0 queries, 1 keys, 2 what is copied bit for bit: values, keys as they come
        auto pass = [&](auto kind_of, const HeadsView& src_of, int first, const void* weight, T* to, long long to_head, bool store) {
            constexpr int KIND = decltype(kind_of)::value;
            const int b = max(h0, first), z = min(h1, first + src_of.heads);
            if (b >= z) return;
            // lane group `sub` takes heads b + sub, b + sub + per_warp, ...; the last job of the warp may be short
            const int count = z - b, jobs = (count + per_warp - 1) >> (5 - llanes);
            const bool last_on = sub < count - (jobs - 1) * per_warp;
            const T* src = reinterpret_cast<const T*>(src_of.data) + (long long)row * src_of.row + (long long)(b - first + sub) * src_of.head;
            const long long step = src_of.head << (5 - llanes);
            Raw raw[AHEAD][NI][2];
            auto fetch = [&](int job, Raw (&x)[NI][2]) {
                const bool on = job + 1 < jobs || (job + 1 == jobs && last_on);
#pragma unroll
                for (int u = 0; u < NI; ++u)
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        x[u][w] = Raw{};
                        if (on && in[u][w]) x[u][w] = load_cg(reinterpret_cast<const Raw*>(src + e[u][w]));
                    }
                src += step;
            };
#pragma unroll
            for (int y = 0; y < AHEAD; ++y) fetch(y, raw[y]);
            if (APPEND && !have) find_place();
            // (with the first heads on their way)
            if (KIND != 2 && !have) make_turns();
            have = true;
            if (APPEND) {
                store = store && (KIND == 0 ? there : stored);
                to += KIND == 0 ? 0 : (KIND == 1 || first == Hq ? k_at : v_at);
            }
            to += (long long)(b - first + sub) * to_head;
            const long long to_step = to_head << (5 - llanes);
            // turn times weight: cu = w_u c, sv = - w_v s, cv = w_v c, su = w_u s
            float cu[NI][V], sv[NI][V], cv[NI][V], su[NI][V];
            if (KIND != 2) {
#pragma unroll
                for (int u = 0; u < NI; ++u) {
                    float w0[V], w1[V];
#pragma unroll
                    for (int c = 0; c < V; ++c) w0[c] = w1[c] = 1.f;
                    if (weight) {
                        if (in[u][0]) unpack<V>(load_cg(reinterpret_cast<const Raw*>(reinterpret_cast<const T*>(weight) + e[u][0])), w0, T{});
                        if (in[u][1]) unpack<V>(load_cg(reinterpret_cast<const Raw*>(reinterpret_cast<const T*>(weight) + e[u][1])), w1, T{});
                    }
#pragma unroll
                    for (int c = 0; c < V; ++c) {
                        // channels of pair c: the vectors' c, or 2c and 2c + 1 of the two vectors in a row
                        const float wu = INTER ? (2 * c < V ? w0[2 * c % V] : w1[2 * c % V]) : w0[c];
                        const float wv = INTER ? (2 * c + 1 < V ? w0[(2 * c + 1) % V] : w1[(2 * c + 1) % V]) : w1[c];
                        const int j = (INTER ? e[u][0] >> 1 : e[u][0]) + c;
                        const float2 t = turned[u] && j < pairs ? turn[j] : make_float2(1.f, 0.f);
                        cu[u][c] = wu * t.x; su[u][c] = wu * t.y;
                        cv[u][c] = wv * t.x; sv[u][c] = -wv * t.y;
                    }
                }
            }
            // as pairs: of neighbours in the half layout, else of (u, v)
            constexpr int NP = V == 1 ? 1 : (INTER ? V : V / 2);
            [[maybe_unused]] Pair cu2[NI][NP], sv2[NI][NP], cv2[NI][NP], su2[NI][NP];
            if constexpr (V > 1 && KIND != 2) {
#pragma unroll
                for (int u = 0; u < NI; ++u)
#pragma unroll
                    for (int c = 0; c < NP; ++c) {
                        cu2[u][c] = INTER ? pair_of(cu[u][c], cv[u][c]) : pair_of(cu[u][2 * c], cu[u][2 * c + 1]);
                        sv2[u][c] = INTER ? pair_of(sv[u][c], su[u][c]) : pair_of(sv[u][2 * c], sv[u][2 * c + 1]);
                        if constexpr (!INTER) {
                            cv2[u][c] = pair_of(cv[u][2 * c], cv[u][2 * c + 1]);
                            su2[u][c] = pair_of(su[u][2 * c], su[u][2 * c + 1]);
                        }
                    }
            }
            store = store && in_bounds(a.hdr, 6, (long long)(row + 1) * heads - 1, (long long)a.rows * heads);
            T* out[NI][2];
#pragma unroll
            for (int u = 0; u < NI; ++u) { out[u][0] = to + e[u][0]; out[u][1] = to + e[u][1]; }
#pragma unroll 1
            for (int j0 = 0; j0 < jobs; j0 += AHEAD) {
#pragma unroll
                for (int y = 0; y < AHEAD; ++y) {
                    const int job = j0 + y;
                    if (job >= jobs) break;                // (the same for the whole warp)
                    Raw res[NI][2];
                    if constexpr (KIND == 2) {
#pragma unroll
                        for (int u = 0; u < NI; ++u) { res[u][0] = raw[y][u][0]; res[u][1] = raw[y][u][1]; }
                        fetch(job + AHEAD, raw[y]);
                    } else if constexpr (V > 1) {
                        Pair x[NI][2][V / 2];
#pragma unroll
                        for (int u = 0; u < NI; ++u)
#pragma unroll
                            for (int w = 0; w < 2; ++w) unpack_pairs<V>(raw[y][u][w], x[u][w], T{});
                        fetch(job + AHEAD, raw[y]);
                        Pair inv = 0;
                        if (weight) {
                            Pair part[V / 2];
#pragma unroll
                            for (int c = 0; c < V / 2; ++c) {
                                part[c] = mul2(x[0][0][c], x[0][0][c]);
#pragma unroll
                                for (int u = 0; u < NI; ++u)
#pragma unroll
                                    for (int w = u == 0 ? 1 : 0; w < 2; ++w) part[c] = fma2(x[u][w][c], x[u][w][c], part[c]);
                            }
#pragma unroll
                            for (int c = V / 4; c > 0; c >>= 1)
#pragma unroll
                                for (int d = 0; d < c; ++d) part[d] = add2(part[d], part[d + c]);
                            const float2 two = both_of(part[0]);
                            const float root = rsqrtf(fmaf(head_sum(two.x + two.y, lanes, llanes), a.inv_dim, a.eps));
                            inv = pair_of(root, root);
                        }
#pragma unroll
                        for (int u = 0; u < NI; ++u) {
#pragma unroll
                            for (int c = 0; c < (INTER ? V : V / 2); ++c) {
                                // half layout: pairs of u and pairs of v; else (u, v) and (v, u)
                                Pair pu = INTER ? x[u][2 * c / V][c % (V / 2)] : x[u][0][c], pv = INTER ? 0 : x[u][1][c];
                                if (weight) { pu = mul2(pu, inv); if (!INTER) pv = mul2(pv, inv); }
                                Pair qu = pu, qv = pv;
                                if (INTER) { const float2 t = both_of(pu); qv = pair_of(t.y, t.x); }
                                // (channels that do not turn: their neighbour, whatever it holds, plays no part.  Without a norm
                                // sv is -0 there and su +0; with these signs both products are -0, and a negative zero stays one.)
                                if (rot < D) {
                                    const bool t = turned[u] && (!INTER || (e[u][0] >> 1) + c < pairs);
                                    qu = t ? qu : pair_of(-0.f, -0.f); qv = t ? qv : pair_of(0.f, INTER ? -0.f : 0.f);
                                }
                                const float2 y0 = both_of(fma2(pu, cu2[u][c], mul2(qv, sv2[u][c])));
                                const float2 y1 = INTER ? y0 : both_of(fma2(pv, cv2[u][c], mul2(qu, su2[u][c])));
                                auto put = [&](Raw& r, int i, float2 y) {
                                    uint32_t* const to = reinterpret_cast<uint32_t*>(&r);
                                    if constexpr (sizeof(T) == 2) to[i] = bf16_pair(y.x, y.y);
                                    else { to[2 * i] = __float_as_uint(y.x); to[2 * i + 1] = __float_as_uint(y.y); }
                                };
                                if (INTER) put(res[u][2 * c / V], c % (V / 2), y0);
                                else { put(res[u][0], c, y0); put(res[u][1], c, y1); }
                            }
                        }
                    } else {                               // single channels
                        float x[NI][2];
#pragma unroll
                        for (int u = 0; u < NI; ++u)
#pragma unroll
                            for (int w = 0; w < 2; ++w) {
                                float one[1];
                                unpack<1>(raw[y][u][w], one, T{});
                                x[u][w] = one[0];
                            }
                        fetch(job + AHEAD, raw[y]);
                        float inv = 1.f;
                        if (weight) {
                            float ssq = 0.f;
#pragma unroll
                            for (int u = 0; u < NI; ++u) ssq = fmaf(x[u][1], x[u][1], fmaf(x[u][0], x[u][0], ssq));
                            inv = rsqrtf(fmaf(head_sum(ssq, lanes, llanes), a.inv_dim, a.eps));
                        }
#pragma unroll
                        for (int u = 0; u < NI; ++u) {
                            const float pu = x[u][0] * inv, pv = x[u][1] * inv, qu = turned[u] ? pu : -0.f, qv = turned[u] ? pv : 0.f;
                            const float r0[1] = {fmaf(pu, cu[u][0], qv * sv[u][0])}, r1[1] = {fmaf(pv, cv[u][0], qu * su[u][0])};
                            res[u][0] = pack<1>(r0, T{}); res[u][1] = pack<1>(r1, T{});
                        }
                    }
                    if (store && (job + 1 < jobs || last_on)) {
#pragma unroll
                        for (int u = 0; u < NI; ++u)
#pragma unroll
                            for (int w = 0; w < 2; ++w)
                                if (in[u][w]) *reinterpret_cast<Raw*>(out[u][w]) = res[u][w];
                    }
#pragma unroll
                    for (int u = 0; u < NI; ++u) { out[u][0] += to_step; out[u][1] += to_step; }
                }
            }
        };
        pass(std::integral_constant<int, 0>{}, a.q, 0, a.q_weight, reinterpret_cast<T*>(a.out_q.data) + (long long)row * a.out_q.row, a.out_q.head, true);
        if (APPEND) {
            if (!a.as_they_come)
                pass(std::integral_constant<int, 1>{}, a.k, Hq, a.k_weight, reinterpret_cast<T*>(a.cache.k), a.cache.k_head, true);
#pragma unroll 1
            for (int v = a.as_they_come ? 0 : 1; v < 2; ++v)
                pass(std::integral_constant<int, 2>{}, v ? a.v : a.k, v ? Hq + Hk : Hq, nullptr, reinterpret_cast<T*>(v ? a.cache.v : a.cache.k),
                     v ? a.cache.v_head : a.cache.k_head, true);
        } else
            pass(std::integral_constant<int, 1>{}, a.k, Hq, a.k_weight, reinterpret_cast<T*>(a.out_k.data) + (long long)row * a.out_k.row, a.out_k.head, true);
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
    int ll = 0;
    while (ll < 5 && (2 * V << ll) < a.dim) ++ll;
    const int heads = a.q.heads + a.k.heads + (APPEND ? a.v.heads : 0), per_warp = 32 >> ll;
    // a warp per row, or per few heads of a row where that fills the SMs
    const long long most = (long long)a.rows * ((heads + per_warp - 1) / per_warp), warps = kRotThreads / 32;
    long long ctas = (most + warps - 1) / warps;
    if (ctas > sm_count() * kRotCtas) ctas = sm_count() * kRotCtas;
    const bool full = a.dim == 2 * V << ll;
    const dim3 grid((unsigned)ctas), block(kRotThreads);
    if (a.interleaved)
        return full ? launch_pdl(k_rotate<T, V, APPEND, true, true>, grid, block, st, a, ll) : launch_pdl(k_rotate<T, V, APPEND, true, false>, grid, block, st, a, ll);
    return full ? launch_pdl(k_rotate<T, V, APPEND, false, true>, grid, block, st, a, ll) : launch_pdl(k_rotate<T, V, APPEND, false, false>, grid, block, st, a, ll);
}
cudaError_t launch_rotate(const RotateArgs& a, int dtype, bool append, cudaStream_t st) {
    if (a.rows < 1) return cudaSuccess;
    if (dtype == TTF_DTYPE_BF16)
        return append ? launch_rotate_v<bf16_t, true, 8>(a, st) : launch_rotate_v<bf16_t, false, 8>(a, st);
    return append ? launch_rotate_v<float, true, 4>(a, st) : launch_rotate_v<float, false, 4>(a, st);
}

}  // namespace ttf

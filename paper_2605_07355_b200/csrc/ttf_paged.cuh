// Shared by the kernels behind the compressed clip (rotation, cache append, attention): the views of heads, cache and
// sequences that the kernels take, and the look-ups in them.
#pragma once

#include <cuda.h>

#include "../../include/ttf.h"
#include "ttf_internal.cuh"

namespace ttf {

constexpr int kMaxDim = 256;                       // channels of a head

// x / d for 0 <= x < 2^31 and a divisor that the host knows: one multiplication.  With l = ceil(log2 d) and
// m = ceil(2^(31 + l) / d) < 2^32 the error of m / 2^(31 + l) against 1 / d is below 2^-31 / d, so that the quotient is exact.
struct Divisor { unsigned d, m; int shift; };
inline Divisor make_divisor(int d) {
    int l = 0;
    while ((1LL << l) < d) ++l;
    Divisor v;
    v.d = (unsigned)d; v.shift = 31 + l;
    v.m = (unsigned)(((1ull << v.shift) + (unsigned)d - 1) / (unsigned)d);
    return v;
}
__host__ __device__ __forceinline__ int quotient(int x, const Divisor& v) {
    return (int)(((unsigned long long)(unsigned)x * v.m) >> v.shift);
}

struct HeadsView { void* data; long long row, head; int heads; };
// (the stride of an axis of one element is never used: zero, so that it spoils no alignment)
inline HeadsView view(const ttf_heads* h, int rows) {
    if (!h) return HeadsView{nullptr, 0, 0, 0};
    return HeadsView{h->data, rows > 1 ? h->row_stride : 0, h->heads > 1 ? h->head_stride : 0, h->heads};
}

struct CacheView {
    void *k, *v;
    long long k_page, k_row, k_head, v_page, v_row, v_head;
    int pages, heads, dim;
    Divisor page;                                  // rows of a page
};

struct SeqView {
    const int *start, *length, *table;
    long long table_stride;
    int table_pages, seqs, rows;
};

// (hdr: the words of HDR_* of a block that is part of the library image; what calls report stays there until it is asked for)
struct RotateArgs {
    HeadsView q, k, v, out_q, out_k;
    int dim, rows;
    const int* count;
    const int* pos;
    const float* freq;
    bool as_they_come;                             // append: keys are copied
    int rot, interleaved, axes, sec1, sec2, sec0, cyclic;
    float factor, eps, inv_dim;
    const void *q_weight, *k_weight;
    SeqView seq;                                   // append only
    CacheView cache;
    int* hdr;
};
cudaError_t launch_rotate(const RotateArgs& a, int dtype, bool append, cudaStream_t st);

struct AttendArgs {
    HeadsView q, out;
    SeqView seq;
    CacheView cache;
    float scale;
    int causal, window, group;
    int wait_limit, tx_extra;
    int* hdr;
};
cudaError_t launch_attend(const AttendArgs& a, int dtype, cudaStream_t st);
bool attend_tc_takes(const AttendArgs& a, int dtype);
cudaError_t launch_attend_tc(const AttendArgs& a, cudaStream_t st);
bool attend_f32_takes(const AttendArgs& a, int dtype);
cudaError_t launch_attend_f32(const AttendArgs& a, cudaStream_t st);
cudaError_t launch_attend_few32(const AttendArgs& a, cudaStream_t st);
bool attend_few_takes(const AttendArgs& a, int dtype);
cudaError_t launch_attend_few(const AttendArgs& a, cudaStream_t st);
// TMA tiles of the cache: 64 channels x `rows` slots of one head and page, 128-byte swizzle, zeros beyond the head
bool cache_maps_fit(const AttendArgs& a);
bool make_cache_map(CUtensorMap* m, const AttendArgs& a, bool values, int rows);
bool attend_mma_takes(const AttendArgs& a, int dtype);
cudaError_t launch_attend_mma(const AttendArgs& a, cudaStream_t st);
cudaError_t launch_attend_simple(const AttendArgs& a, int dtype, cudaStream_t st);

// Upper bound on the tiles of a call (the host does not know how the rows are spread over the sequences), and the CTAs of a
// cluster that share the slots of a tile.
inline long long most_tiles(const AttendArgs& a, int rows, int per) {
    return (per > 0 ? (long long)a.seq.rows / per : (long long)a.seq.rows * a.group / rows) + a.seq.seqs;
}

#ifdef __CUDACC__

// V consecutive channels as they lie in memory
template <typename T, int V> struct VecIO;
template <> struct VecIO<bf16_t, 8> { using Raw = uint4; };
template <> struct VecIO<bf16_t, 4> { using Raw = uint2; };
template <> struct VecIO<bf16_t, 2> { using Raw = uint32_t; };
template <> struct VecIO<bf16_t, 1> { using Raw = uint16_t; };
template <> struct VecIO<float, 4> { using Raw = uint4; };
template <> struct VecIO<float, 2> { using Raw = uint2; };
template <> struct VecIO<float, 1> { using Raw = uint32_t; };

__device__ __forceinline__ uint16_t load_cg(const uint16_t* p) { return __ldcg(reinterpret_cast<const unsigned short*>(p)); }
template <typename R> __device__ __forceinline__ R load_cg(const R* p) { return __ldcg(p); }

template <int V> __device__ __forceinline__ void unpack(const typename VecIO<bf16_t, V>::Raw& r, float (&x)[V], bf16_t) {
    if constexpr (V == 1) x[0] = __uint_as_float((uint32_t)r << 16);
    else {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
    }
}
template <int V> __device__ __forceinline__ void unpack(const typename VecIO<float, V>::Raw& r, float (&x)[V], float) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = __uint_as_float(w[i]);
}
// two fp32 -> bf16, round to nearest even (NaN stays NaN)
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <int V> __device__ __forceinline__ typename VecIO<bf16_t, V>::Raw pack(const float (&x)[V], bf16_t) {
    typename VecIO<bf16_t, V>::Raw r;
    if constexpr (V == 1) r = (uint16_t)(bf16_pair(x[0], x[0]) & 0xffffu);
    else {
        uint32_t* w = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) w[i] = bf16_pair(x[2 * i], x[2 * i + 1]);
    }
    return r;
}
template <int V> __device__ __forceinline__ typename VecIO<float, V>::Raw pack(const float (&x)[V], float) {
    typename VecIO<float, V>::Raw r;
    uint32_t* w = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = __float_as_uint(x[i]);
    return r;
}

// Two values in two registers side by side: a * b + c, a * b and a + b of both are one instruction of the fp32 pipe.  (With float2
// a pair may have to be moved together first: appending 2703 rows of 48 heads took 20.0 us, with pairs 18.0.)
typedef unsigned long long Pair;
__device__ __forceinline__ Pair pair_of(float x, float y) {
    Pair d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(x), "f"(y));
    return d;
}
__device__ __forceinline__ float2 both_of(Pair a) {
    float2 d;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(a));
    return d;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    Pair d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
    Pair d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
template <int V> __device__ __forceinline__ void unpack_pairs(const typename VecIO<bf16_t, V>::Raw& r, Pair (&x)[V / 2], bf16_t) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) x[i] = pair_of(bf16_lo(w[i]), bf16_hi(w[i]));
}
template <int V> __device__ __forceinline__ void unpack_pairs(const typename VecIO<float, V>::Raw& r, Pair (&x)[V / 2], float) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) x[i] = pair_of(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
}

// a call's outputs are not what was asked for: kind 1 a bounded wait gave up, 2 lengths or pages outside their arrays
__device__ __forceinline__ void report_paged(int* hdr, int kind) { atomicMax(hdr + HDR_ERROR, kind); }

__device__ __forceinline__ bool length_fits(const SeqView& s, int length, const Divisor& page) {
    return length >= 0 && length <= (1 << 30) && (long long)length <= (long long)s.table_pages * page.d;
}
// One sequence of a call, with nothing that could lead out of an array: n new rows from `first` on, `length` slots.
struct SeqRange { int first, n, length; bool ok; };
__device__ __forceinline__ SeqRange seq_range(const SeqView& s, int b, const Divisor& page) {
    SeqRange r;
    r.first = __ldcg(s.start + b);
    const int end = __ldcg(s.start + b + 1);
    r.length = __ldcg(s.length + b);
    r.ok = r.first >= 0 && end >= r.first && end <= s.rows && length_fits(s, r.length, page);
    r.n = r.ok ? end - r.first : 0;
    return r;
}

// Index of the page of slot `s`: always inside the cache; `bad` is raised where the table says otherwise.
__device__ __forceinline__ int page_of(const int* table_row, int index, int pages, bool& bad) {
    int g = __ldcg(table_row + index);
    if ((unsigned)g >= (unsigned)pages) { bad = true; g = 0; }
    return g;
}

// What row `token` of a sequence sees: slots [lo, hi).
struct Seen { int lo, hi; };
__device__ __forceinline__ Seen seen_by(const SeqRange& r, int token, int causal, int window) {
    const int c = r.length - r.n + token;          // its own slot
    Seen v;
    v.hi = c < 0 ? 0 : (causal ? c + 1 : r.length);
    v.lo = window > 0 && c >= window ? c - window + 1 : 0;
    return v;
}

// The tile of this CTA.  The new rows of a sequence times the query heads of a group are packed rows (row = token * group +
// head), cut into tiles of so many tokens or of so many packed rows; tiles are numbered over the sequences, and
// tile `index` from the end is looked up (with a causal mask the last tiles of a sequence take longest: they come first).
// Every warp does it for itself.  False: there is no such tile.
struct Tile { int seq, tile; SeqRange r; };
struct Cut { Divisor tokens; int lrows; };         // tiles of `tokens` tokens, or (tokens.d = 0) of 2^lrows packed rows
inline Cut cut_tokens(int per) { return Cut{make_divisor(per), 0}; }
inline Cut cut_rows(int lrows) { return Cut{Divisor{0, 0, 0}, lrows}; }
__device__ __forceinline__ int tiles_of(int n, int group, const Cut& cut) {
    return cut.tokens.d ? (n > 0 ? quotient(n - 1, cut.tokens) + 1 : 0)
                        : (int)(((long long)n * group + (1 << cut.lrows) - 1) >> cut.lrows);
}
__device__ __forceinline__ bool find_tile(const AttendArgs& a, const Cut& cut, int index, bool report, Tile& t) {
    const int lane = threadIdx.x & 31;
    int total = 0, c = 0;
    bool bad = false;
    SeqRange r = {0, 0, 0, false};
    for (int s0 = 0; s0 < a.seq.seqs; s0 += 32) {
        c = 0;
        if (s0 + lane < a.seq.seqs) {
            r = seq_range(a.seq, s0 + lane, a.cache.page);
            bad |= !r.ok;
            c = tiles_of(r.n, a.group, cut);
        }
        total += __reduce_add_sync(0xffffffffu, c);
    }
    if (report && __any_sync(0xffffffffu, bad) && threadIdx.x == 0) report_paged(a.hdr, 2);
    int want = total - 1 - index;
    if (want < 0) return false;
    for (int s0 = 0; s0 < a.seq.seqs; s0 += 32) {
        if (a.seq.seqs > 32) {                     // (up to 32 sequences are still in registers)
            c = 0;
            if (s0 + lane < a.seq.seqs) {
                r = seq_range(a.seq, s0 + lane, a.cache.page);
                c = tiles_of(r.n, a.group, cut);
            }
        }
        int upto = c;                              // inclusive scan
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const unsigned m = __ballot_sync(0xffffffffu, upto > want);
        if (m) {
            const int src = __ffs(m) - 1;
            t.seq = s0 + src;
            t.tile = want - __shfl_sync(0xffffffffu, upto - c, src);
            // (overlapping sequences, which are reported, may add up to more than 31 bits)
            if ((unsigned)t.tile >= (unsigned)__shfl_sync(0xffffffffu, c, src)) return false;
            t.r.first = __shfl_sync(0xffffffffu, r.first, src);
            t.r.n = __shfl_sync(0xffffffffu, r.n, src);
            t.r.length = __shfl_sync(0xffffffffu, r.length, src);
            t.r.ok = true;
            return true;
        }
        want -= __shfl_sync(0xffffffffu, upto, 31);
    }
    return false;
}

#endif  // __CUDACC__

}  // namespace ttf

// C ABI of what follows the compressed clip: argument validation of ttf_rotate, ttf_cache_append and ttf_attend, and the
// device status they share.  Declarations and contracts are in include/ttf.h.
#include "ttf_paged.cuh"

#include <nvtx3/nvToolsExt.h>

#include <cmath>
#include <mutex>

namespace ttf {

// What the calls report stays here until ttf_paged_status asks: one block per device, part of the library image, so that
// no call needs scratch and a captured graph none that could be given back.
static __device__ int g_paged_words[kHdrInts + 1];         // (the last word: what a query has taken)
constexpr int kMaxDevices = 64;
static int* g_paged_addr[kMaxDevices] = {};
static std::mutex g_paged_mu;

static int paged_words(int** out) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(e);
    if (dev < 0 || dev >= kMaxDevices) return TTF_ERR_UNSUPPORTED;
    std::lock_guard<std::mutex> lk(g_paged_mu);
    if (!g_paged_addr[dev]) {
        void* p = nullptr;
        e = cudaGetSymbolAddress(&p, g_paged_words);
        if (e != cudaSuccess) return cuda_fail(e);
        g_paged_addr[dev] = static_cast<int*>(p);
    }
    *out = g_paged_addr[dev];
    return TTF_OK;
}

// checked build: the slack of the index tests, set in stream order before a call
#ifdef TTF_DEBUG
__global__ void k_paged_slack(int* word, int value) { *word = value; }
static int begin_paged(int* hdr, cudaStream_t st) {
    k_paged_slack<<<1, 1, 0, st>>>(hdr + HDR_CHECK_SLACK, check_slack());
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? TTF_OK : cuda_fail(e);
}
#else
static int begin_paged(int*, cudaStream_t) { return TTF_OK; }
#endif

// reading and clearing is one step: a report of another stream comes before it, and is told now, or after it, and stays
__global__ void k_paged_take(int* words) { words[kHdrInts] = atomicExch(words + HDR_ERROR, 0); }
static std::mutex g_paged_query_mu;                        // one query at a time: they share the word

struct Range { Range(const char* name) { nvtxRangePushA(name); } ~Range() { nvtxRangePop(); } };

// the last element of a view must be addressable with 62 bits, whatever the signs of the strides
static bool reachable(long long n0, long long s0, long long n1, long long s1, long long n2, long long s2) {
    auto part = [](long long n, long long s) { return (double)(n > 0 ? n - 1 : 0) * std::fabs((double)s); };
    return part(n0, s0) + part(n1, s1) + part(n2, s2) < 4e18 / 4;
}
static int check_heads(const ttf_heads* h, int rows) {
    if (!h || !h->data || h->heads < 1) return TTF_ERR_INVALID_ARG;
    if (h->heads > 65535 || (long long)rows * h->heads >= (1LL << 31)) return TTF_ERR_UNSUPPORTED;
    return reachable(rows, h->row_stride, h->heads, h->head_stride, 0, 0) ? TTF_OK : TTF_ERR_UNSUPPORTED;
}
// no two elements of an output in one place
static bool apart(long long n0, long long s0, long long n1, long long s1, long long n2, long long s2) {
    return (n0 == 1 || s0) && (n1 == 1 || s1) && (n2 == 1 || s2);
}
static bool apart(const ttf_heads* h, int rows) { return !h || apart(rows, h->row_stride, h->heads, h->head_stride, 1, 0); }
static bool known_dtype(int dtype) { return dtype == TTF_DTYPE_F32 || dtype == TTF_DTYPE_BF16; }

static int check_rotation(const ttf_rotation* r, int head_dim, const int* positions) {
    if (!r || r->rot_dim < 0 || r->rot_dim % 2 || r->rot_dim > head_dim || r->axes < 1 || r->axes > 3) return TTF_ERR_INVALID_ARG;
    if (r->interleaved < 0 || r->interleaved > 1 || r->cyclic < 0 || r->cyclic > 1) return TTF_ERR_INVALID_ARG;
    if (!std::isfinite(r->factor) || !(r->eps >= 0.f) || !std::isfinite(r->eps)) return TTF_ERR_INVALID_ARG;
    if (r->rot_dim > 0 && (!r->freq || !positions)) return TTF_ERR_INVALID_ARG;
    if (r->axes > 1) {
        long long sum = 0;
        for (int a = 0; a < r->axes; ++a) {
            if (r->section[a] < 0) return TTF_ERR_INVALID_ARG;
            sum += r->section[a];
        }
        if (sum != r->rot_dim / 2) return TTF_ERR_INVALID_ARG;
        // cyclic: the pairs of axis a are a, a + axes, ...: there must be section[a] of them
        for (int a = 1; a < r->axes && r->cyclic; ++a)
            if (r->section[a] > 0 && (long long)(r->section[a] - 1) * r->axes + a >= r->rot_dim / 2) return TTF_ERR_INVALID_ARG;
    }
    return TTF_OK;
}
static void take_rotation(const ttf_rotation* r, const int* positions, RotateArgs* a) {
    a->pos = positions;
    a->freq = r ? r->freq : nullptr;
    a->rot = r ? r->rot_dim : 0;
    a->interleaved = r ? r->interleaved : 0;
    a->axes = r ? r->axes : 1;
    a->sec0 = r ? r->section[0] : 0; a->sec1 = r ? r->section[1] : 0; a->sec2 = r && r->axes > 2 ? r->section[2] : 0;
    a->cyclic = r ? r->cyclic : 0;
    a->factor = r ? r->factor : 1.f;
    a->eps = r ? r->eps : 0.f;
    a->q_weight = r ? r->q_weight : nullptr;
    a->k_weight = r ? r->k_weight : nullptr;
}

static int check_sequences(const ttf_sequences* s) {
    if (!s || s->seqs < 1 || s->rows < 1 || s->table_pages < 1) return TTF_ERR_INVALID_ARG;
    // (a stride of zero: all sequences have one list of pages)
    if (!s->start || !s->length || !s->table || (s->table_stride != 0 && s->table_stride < s->table_pages)) return TTF_ERR_INVALID_ARG;
    if (s->seqs > 1 << 30) return TTF_ERR_UNSUPPORTED;     // (the kernels count 32 beyond them)
    return reachable(s->seqs, s->table_stride, s->table_pages, 1, 0, 0) ? TTF_OK : TTF_ERR_UNSUPPORTED;
}
static int check_cache(const ttf_cache* c) {
    if (!c || !c->k || !c->v || c->pages < 1 || c->page_size < 1 || c->heads < 1 || c->head_dim < 1 || !known_dtype(c->dtype)) return TTF_ERR_INVALID_ARG;
    if (c->head_dim > kMaxDim || c->heads > 65535) return TTF_ERR_UNSUPPORTED;
    return reachable(c->pages, c->k_page, c->page_size, c->k_row, c->heads, c->k_head) &&
           reachable(c->pages, c->v_page, c->page_size, c->v_row, c->heads, c->v_head) ? TTF_OK : TTF_ERR_UNSUPPORTED;
}
static SeqView view(const ttf_sequences* s) {
    return SeqView{s->start, s->length, s->table, s->table_stride, s->table_pages, s->seqs, s->rows};
}
static CacheView view(const ttf_cache* c) {
    const bool p = c->pages > 1, r = c->page_size > 1, h = c->heads > 1;       // (as in view of heads)
    return CacheView{c->k, c->v, p ? c->k_page : 0, r ? c->k_row : 0, h ? c->k_head : 0, p ? c->v_page : 0, r ? c->v_row : 0,
                     h ? c->v_head : 0, c->pages, c->heads, c->head_dim, make_divisor(c->page_size)};
}

}  // namespace ttf

using namespace ttf;

#define TTF_CHECK(expr) do { const int rc_ = (expr); if (rc_ != TTF_OK) return rc_; } while (0)

extern "C" {

int ttf_rotate(const ttf_heads* q, const ttf_heads* k, int head_dim, int dtype, int rows, const int* count,
               const int* positions, const ttf_rotation* rotation, const ttf_heads* out_q, const ttf_heads* out_k,
               ttf_stream_t stream) {
    if ((!q && !k) || !q != !out_q || !k != !out_k || rows < 1 || head_dim < 1 || !known_dtype(dtype)) return TTF_ERR_INVALID_ARG;
    if (head_dim > kMaxDim) return TTF_ERR_UNSUPPORTED;
    TTF_CHECK(check_rotation(rotation, head_dim, positions));
    for (const ttf_heads* h : {q, k, out_q, out_k})
        if (h) TTF_CHECK(check_heads(h, rows));
    if ((q && q->heads != out_q->heads) || (k && k->heads != out_k->heads)) return TTF_ERR_INVALID_ARG;
    if (!apart(out_q, rows) || !apart(out_k, rows)) return TTF_ERR_INVALID_ARG;
    RotateArgs a = {};
    TTF_CHECK(paged_words(&a.hdr));
    a.q = ttf::view(q, rows); a.k = ttf::view(k, rows); a.out_q = ttf::view(out_q, rows); a.out_k = ttf::view(out_k, rows);
    a.dim = head_dim; a.inv_dim = 1.f / head_dim; a.rows = rows; a.count = count;
    take_rotation(rotation, positions, &a);
    a.cache.page = make_divisor(1);
    Range range("ttf rotate");
    TTF_CHECK(begin_paged(a.hdr, (cudaStream_t)stream));
    const cudaError_t e = launch_rotate(a, dtype, false, (cudaStream_t)stream);
    return e == cudaSuccess ? TTF_OK : cuda_fail(e);
}

int ttf_cache_append(const ttf_heads* k, const ttf_heads* v, const ttf_heads* q, const int* positions,
                     const ttf_rotation* rotation, const ttf_sequences* sequences, const ttf_cache* cache,
                     const ttf_heads* out_q, ttf_stream_t stream) {
    if (!k || !v || !q != !out_q || (q && !rotation)) return TTF_ERR_INVALID_ARG;
    TTF_CHECK(check_cache(cache));
    TTF_CHECK(check_sequences(sequences));
    if (rotation) TTF_CHECK(check_rotation(rotation, cache->head_dim, positions));
    for (const ttf_heads* h : {k, v, q, out_q})
        if (h) TTF_CHECK(check_heads(h, sequences->rows));
    if (k->heads != cache->heads || v->heads != cache->heads || (q && q->heads != out_q->heads)) return TTF_ERR_INVALID_ARG;
    if (!apart(out_q, sequences->rows) || !apart(cache->pages, cache->k_page, cache->page_size, cache->k_row, cache->heads, cache->k_head) ||
        !apart(cache->pages, cache->v_page, cache->page_size, cache->v_row, cache->heads, cache->v_head)) return TTF_ERR_INVALID_ARG;
    RotateArgs a = {};
    TTF_CHECK(paged_words(&a.hdr));
    const int rows = sequences->rows;
    a.q = ttf::view(q, rows); a.k = ttf::view(k, rows); a.v = ttf::view(v, rows); a.out_q = ttf::view(out_q, rows);
    a.dim = cache->head_dim; a.inv_dim = 1.f / cache->head_dim; a.rows = sequences->rows;
    take_rotation(rotation, positions, &a);
    a.as_they_come = !rotation || (!rotation->k_weight && rotation->rot_dim == 0);
    a.seq = ttf::view(sequences); a.cache = ttf::view(cache);
    Range range("ttf cache append");
    TTF_CHECK(begin_paged(a.hdr, (cudaStream_t)stream));
    const cudaError_t e = launch_rotate(a, cache->dtype, true, (cudaStream_t)stream);
    return e == cudaSuccess ? TTF_OK : cuda_fail(e);
}

int ttf_attend(const ttf_heads* q, const ttf_sequences* sequences, const ttf_cache* cache, float scale, int causal,
               int window, const ttf_heads* out, ttf_stream_t stream) {
    // (the kernels work in powers of two: scale log2(e) has to be a number as well)
    if (!q || !out || !std::isfinite(scale * 1.4426950408889634f) || causal < 0 || causal > 1 || window < 0) return TTF_ERR_INVALID_ARG;
    TTF_CHECK(check_cache(cache));
    TTF_CHECK(check_sequences(sequences));
    for (const ttf_heads* h : {q, out}) TTF_CHECK(check_heads(h, sequences->rows));
    if (q->heads != out->heads || q->heads % cache->heads || !apart(out, sequences->rows)) return TTF_ERR_INVALID_ARG;
    AttendArgs a = {};
    TTF_CHECK(paged_words(&a.hdr));
    a.q = ttf::view(q, sequences->rows); a.out = ttf::view(out, sequences->rows); a.seq = ttf::view(sequences); a.cache = ttf::view(cache);
    a.scale = scale; a.causal = causal; a.window = window; a.group = q->heads / cache->heads;
    a.wait_limit = wait_poll_limit(); a.tx_extra = wait_tx_extra();
    Range range("ttf attend");
    TTF_CHECK(begin_paged(a.hdr, (cudaStream_t)stream));
    const cudaError_t e = launch_attend(a, cache->dtype, (cudaStream_t)stream);
    return e == cudaSuccess ? TTF_OK : cuda_fail(e);
}

int ttf_paged_status(ttf_stream_t stream, int* host_status) {
    if (!host_status) return TTF_ERR_INVALID_ARG;
    int* words = nullptr;
    TTF_CHECK(paged_words(&words));
    const cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = cudaStreamSynchronize(st);             // (the caller's work, which may be long, without the lock)
    if (e != cudaSuccess) return cuda_fail(e);
    int v = 0;
    {
        std::lock_guard<std::mutex> lk(g_paged_query_mu);
        k_paged_take<<<1, 1, 0, st>>>(words);
        e = cudaGetLastError();
        if (e == cudaSuccess) e = cudaMemcpyAsync(&v, words + kHdrInts, sizeof(int), cudaMemcpyDeviceToHost, st);
        const cudaError_t w = cudaStreamSynchronize(st);   // (in any case: nothing may write v when it is gone)
        if (e == cudaSuccess) e = w;
    }
    if (e != cudaSuccess) return cuda_fail(e);
    *host_status = v == 0 ? TTF_OK : (v == 2 ? TTF_ERR_BOUNDS : TTF_ERR_TIMEOUT);
    return TTF_OK;
}

}  // extern "C"

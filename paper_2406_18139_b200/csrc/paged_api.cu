// Host side of the operators over a paged cache: argument checks, workspace, launches.  Nothing here
// synchronises with the device or allocates device memory.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "host.h"
#include "paged.h"

namespace lookm {
namespace {

constexpr int kMaxLen = 1 << 30;         // rows of a cache

bool aligned(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

int check_paged(const lookm_paged_layout* l) {
    if (!l) return LOOKM_ERR_INVALID_ARG;
    if (l->head_dim != kHeadDim) return LOOKM_ERR_UNSUPPORTED;
    if (l->n_kv_heads <= 0 || l->n_q_heads <= 0 || l->n_q_heads % l->n_kv_heads) return LOOKM_ERR_INVALID_ARG;
    if (l->n_q_heads > 65535 || l->n_q_heads / l->n_kv_heads > kTile) return LOOKM_ERR_UNSUPPORTED;
    if (l->page_rows < 16 || l->page_rows > 65536 || (l->page_rows & (l->page_rows - 1))) return LOOKM_ERR_UNSUPPORTED;
    if (l->n_pages <= 0 || l->table_stride <= 0) return LOOKM_ERR_INVALID_ARG;
    for (long long s : {l->page_stride, l->row_stride, l->head_stride}) {
        if (s < kHeadDim || s % 8) return LOOKM_ERR_INVALID_ARG;
        if (s >= (1ll << 38)) return LOOKM_ERR_UNSUPPORTED;          // (tensor maps keep 40 bits of bytes)
    }
    if (!(l->softmax_scale >= 0.f) || !std::isfinite(l->softmax_scale)) return LOOKM_ERR_INVALID_ARG;
    return LOOKM_OK;
}

int check_requests(const lookm_paged_layout* l, int n, const int* lens) {
    if (n <= 0 || !lens) return LOOKM_ERR_INVALID_ARG;
    if (n > 65535) return LOOKM_ERR_UNSUPPORTED;
    long long total = 0;
    for (int r = 0; r < n; ++r) {
        if (lens[r] < 0 || lens[r] > kMaxLen) return LOOKM_ERR_INVALID_ARG;
        if (((long long)lens[r] + l->page_rows - 1) / l->page_rows > l->table_stride) return LOOKM_ERR_INVALID_ARG;
        total += lens[r];
    }
    return total * l->n_q_heads >= (1ll << 40) ? LOOKM_ERR_UNSUPPORTED : LOOKM_OK;
}

// Token counts of a packed batch: ascending from 0, zero allowed.
int check_tokens(int n, const int* cu) {
    if (n <= 0 || !cu || cu[0] != 0) return LOOKM_ERR_INVALID_ARG;
    for (int r = 0; r < n; ++r)
        if (cu[r + 1] < cu[r]) return LOOKM_ERR_INVALID_ARG;
    return cu[n] > kMaxLen ? LOOKM_ERR_UNSUPPORTED : LOOKM_OK;
}

int check_pool(const void* k, const void* v, const int* table) {
    return k && v && table && aligned(k, 16) && aligned(v, 16) && aligned(table, 4) ? LOOKM_OK : LOOKM_ERR_INVALID_ARG;
}

int check_ws(const void* ws, size_t have, size_t need) {
    if (!ws || !aligned(ws, 256)) return LOOKM_ERR_INVALID_ARG;
    return have < need ? LOOKM_ERR_WORKSPACE_TOO_SMALL : LOOKM_OK;
}

Pages pages_of(const lookm_paged_layout* l, const int* table) {
    Pages p;
    p.table = table;
    p.table_stride = l->table_stride;
    p.n_pages = l->n_pages;
    p.page_shift = 0;
    while ((1 << p.page_shift) < l->page_rows) ++p.page_shift;
    p.n_q_heads = l->n_q_heads;
    p.n_kv_heads = l->n_kv_heads;
    p.page_stride = l->page_stride;
    p.row_stride = l->row_stride;
    p.head_stride = l->head_stride;
    return p;
}

// The workspace: the status word, and behind it what the call at hand needs.
constexpr size_t kStatusBytes = 256;

// A C entry lets no exception out.
template <class F>
int guarded(F f) {
    try {
        return f();
    } catch (...) {
        return LOOKM_ERR_CUDA;
    }
}

int append_rows(const void* q, const void* k, const void* v, const int* positions, const int* cu, const int* lens, int n,
                const lookm_layout* lay, const lookm_append_options* opt, void* q_out, void* cache_k, void* cache_v, float* mass,
                const int* table, const lookm_paged_layout* paged, void* ws, size_t ws_bytes, void* stream) {
    LOOKM_TRY(check_paged(paged));
    if (!lay || !k || !v || !q != !q_out) return LOOKM_ERR_INVALID_ARG;
    if (lay->head_dim != kHeadDim) return LOOKM_ERR_UNSUPPORTED;
    if (lay->n_kv_heads != paged->n_kv_heads || (q && lay->n_q_heads != paged->n_q_heads)) return LOOKM_ERR_INVALID_ARG;
    LOOKM_TRY(check_tokens(n, cu));
    LOOKM_TRY(check_requests(paged, n, lens));
    for (int r = 0; r < n; ++r) {
        const long long len = (long long)lens[r] + cu[r + 1] - cu[r];
        if (len > kMaxLen || (len + paged->page_rows - 1) / paged->page_rows > paged->table_stride) return LOOKM_ERR_INVALID_ARG;
    }
    LOOKM_TRY(check_pool(cache_k, cache_v, table));
    for (const void* p : {q, k, v, (const void*)q_out})
        if (!aligned(p, 16)) return LOOKM_ERR_INVALID_ARG;
    if (!aligned(mass, 4) || !aligned(positions, 4)) return LOOKM_ERR_INVALID_ARG;
    for (long long s : {lay->kv_stride_tok, lay->kv_stride_head})
        if (s <= 0 || s % 8) return LOOKM_ERR_INVALID_ARG;
    if (q)
        for (long long s : {lay->q_stride_tok, lay->q_stride_head, paged->q_stride_tok, paged->q_stride_head})
            if (s <= 0 || s % 8) return LOOKM_ERR_INVALID_ARG;
    AppendParams p;
    p.q_weight = opt ? opt->q_weight : nullptr;
    p.k_weight = opt ? opt->k_weight : nullptr;
    p.eps = opt ? opt->eps : 0.f;
    p.rotary_dim = opt ? opt->rotary_dim : 0;
    p.interleaved = opt ? opt->interleaved != 0 : 0;
    if (!aligned(p.q_weight, 16) || !aligned(p.k_weight, 16)) return LOOKM_ERR_INVALID_ARG;
    if ((p.q_weight || p.k_weight) && (!(p.eps >= 0.f) || !std::isfinite(p.eps))) return LOOKM_ERR_INVALID_ARG;
    if (p.rotary_dim < 0 || p.rotary_dim > kHeadDim) return LOOKM_ERR_INVALID_ARG;
    if (p.rotary_dim % 16) return LOOKM_ERR_UNSUPPORTED;
    if (p.rotary_dim && (!positions || !opt->inv_freq_host)) return LOOKM_ERR_INVALID_ARG;
    for (int i = 0; i < kMaxFreqs; ++i) {
        p.turns[i] = i < p.rotary_dim / 2 ? opt->inv_freq_host[i] / 6.283185307179586476925 : 0.;
        if (!std::isfinite(p.turns[i])) return LOOKM_ERR_INVALID_ARG;
    }
    LOOKM_TRY(check_ws(ws, ws_bytes, kStatusBytes));
    DeviceInfo di;
    LOOKM_TRY(device_info(di));
    g_launches = 0;
    p.pages = pages_of(paged, table);
    p.q = q;
    p.k = k;
    p.v = v;
    p.positions = positions;
    p.q_stride_tok = lay->q_stride_tok;
    p.q_stride_head = lay->q_stride_head;
    p.kv_stride_tok = lay->kv_stride_tok;
    p.kv_stride_head = lay->kv_stride_head;
    p.q_out = q_out;
    p.qo_stride_tok = paged->q_stride_tok;
    p.qo_stride_head = paged->q_stride_head;
    p.cache_k = cache_k;
    p.cache_v = cache_v;
    p.mass = mass;
    p.status = at<int>(ws, 0);
    for (int base = 0; base < n; base += kManyRequests) {
        Batch<AppendReq, kManyRequests> b;
        b.n = std::min(kManyRequests, n - base);
        b.pad = 0;
        for (int i = 0; i < b.n; ++i) b.r[i] = {cu[base + i], lens[base + i], base + i, 0};
        p.tok_begin = cu[base];
        p.tok_end = cu[base + b.n];
        if (p.tok_begin == p.tok_end) continue;
        LOOKM_CUDA(launch_append(p, b, di.sms, static_cast<cudaStream_t>(stream)));
        ++g_launches;
    }
    return LOOKM_OK;
}

int evict(const void* cache_k, const void* cache_v, const float* mass, const int* table, const int* lens, const int* budgets,
          const int* windows, int n, const lookm_paged_layout* paged, void* out_k, void* out_v, float* out_mass, const int* out_table,
          int* kept, void* ws, size_t ws_bytes, void* stream) {
    LOOKM_TRY(check_paged(paged));
    LOOKM_TRY(check_requests(paged, n, lens));
    LOOKM_TRY(check_pool(cache_k, cache_v, table));
    LOOKM_TRY(check_pool(out_k, out_v, out_table));
    if (!budgets || !windows || !mass || !out_mass || !aligned(mass, 4) || !aligned(out_mass, 4) || !aligned(kept, 4))
        return LOOKM_ERR_INVALID_ARG;
    long long total = 0;
    for (int r = 0; r < n; ++r) {
        if (budgets[r] <= 0 || windows[r] < 0) return LOOKM_ERR_INVALID_ARG;
        total += std::min(budgets[r], lens[r]);
    }
    if (total * paged->n_kv_heads >= (1ll << 40)) return LOOKM_ERR_UNSUPPORTED;
    LOOKM_TRY(check_ws(ws, ws_bytes, kStatusBytes + (kept ? 0 : 4 * (size_t)total * paged->n_kv_heads)));
    DeviceInfo di;
    LOOKM_TRY(device_info(di));
    g_launches = 0;
    EvictParams p;
    p.pages = pages_of(paged, table);
    p.out_table = out_table;
    p.cache_k = cache_k;
    p.cache_v = cache_v;
    p.mass = mass;
    p.out_k = out_k;
    p.out_v = out_v;
    p.out_mass = out_mass;
    p.kept = kept ? kept : at<int>(ws, kStatusBytes);
    p.status = at<int>(ws, 0);
    const bool in_place = cache_k == out_k || cache_v == out_v || mass == out_mass;
    Batch<EvictReq, kManyRequests> b;
    b.n = b.pad = 0;
    long long off = 0;
    for (int r = 0; r < n; ++r) {
        EvictReq q;
        q.len = lens[r];
        q.budget = std::min(budgets[r], lens[r]);
        q.window = std::min(windows[r], q.budget);
        q.index = r;
        q.kept_off = off;
        off += (long long)q.budget * paged->n_kv_heads;
        if (q.budget > 0) b.r[b.n++] = q;
        if (b.n == kManyRequests || (r == n - 1 && b.n)) {
            LOOKM_CUDA(launch_evict(p, b, in_place, di.sms, static_cast<cudaStream_t>(stream), &g_launches));
            b.n = 0;
        }
    }
    return LOOKM_OK;
}

}  // namespace
}  // namespace lookm

using namespace lookm;

extern "C" {

size_t lookm_paged_workspace_size(const lookm_paged_layout* paged, int n_requests, const int* new_lens_host,
                                  const int* cache_lens_host) {
    if (check_paged(paged) != LOOKM_OK || check_requests(paged, n_requests, cache_lens_host) != LOOKM_OK) return 0;
    size_t rows = 0;
    for (int r = 0; r < n_requests; ++r) rows += cache_lens_host[r];
    (void)new_lens_host;
    return align_up(kStatusBytes + 4 * rows * paged->n_kv_heads, 256);
}

int lookm_append_rows(const void* q, const void* k, const void* v, const int* positions, const int* cu_seqlens_host,
                      const int* cache_lens_host, int n_requests, const lookm_layout* layout, const lookm_append_options* options,
                      void* q_out, void* cache_k, void* cache_v, float* mass, const int* page_table, const lookm_paged_layout* paged,
                      void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return guarded([&] {
        return append_rows(q, k, v, positions, cu_seqlens_host, cache_lens_host, n_requests, layout, options, q_out, cache_k, cache_v, mass,
                           page_table, paged, workspace, workspace_bytes, cuda_stream);
    });
}

int lookm_evict(const void* cache_k, const void* cache_v, const float* mass, const int* page_table, const int* cache_lens_host,
                const int* budgets_host, const int* windows_host, int n_requests, const lookm_paged_layout* paged, void* out_k, void* out_v,
                float* out_mass, const int* out_page_table, int* kept_idx, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return guarded([&] {
        return evict(cache_k, cache_v, mass, page_table, cache_lens_host, budgets_host, windows_host, n_requests, paged, out_k, out_v,
                     out_mass, out_page_table, kept_idx, workspace, workspace_bytes, cuda_stream);
    });
}

}  // extern "C"

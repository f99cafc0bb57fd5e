// Host side of the operators over a paged cache: argument checks, workspace, launches.  Nothing here
// synchronises with the device or allocates device memory.
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <vector>

#include "host.h"
#include "paged.h"

namespace lookm {
namespace {

constexpr int kMaxLen = 1 << 25;         // rows of a cache, tokens of a call

bool aligned(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

float scale_log2(const lookm_paged_layout* l) {
    return (l->softmax_scale > 0.f ? l->softmax_scale : 1.0f / std::sqrt((float)kHeadDim)) * 1.4426950408889634f;
}

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
    if (!(l->softmax_scale >= 0.f) || !std::isfinite(scale_log2(l))) return LOOKM_ERR_INVALID_ARG;
    return LOOKM_OK;
}

int check_requests(const lookm_paged_layout* l, int n, const int* lens) {
    if (n <= 0 || !lens) return LOOKM_ERR_INVALID_ARG;
    if (n > 65535) return LOOKM_ERR_UNSUPPORTED;
    long long total = 0;
    for (int r = 0; r < n; ++r) {
        if (lens[r] < 0) return LOOKM_ERR_INVALID_ARG;
        if (lens[r] > kMaxLen) return LOOKM_ERR_UNSUPPORTED;
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
        if (len > kMaxLen) return LOOKM_ERR_UNSUPPORTED;
        if ((len + paged->page_rows - 1) / paged->page_rows > paged->table_stride) return LOOKM_ERR_INVALID_ARG;
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
    // in place, a row would otherwise be written where another one is still to be read
    if (q && q == q_out && ((cu[n] > 1 && lay->q_stride_tok != paged->q_stride_tok) ||
                            (paged->n_q_heads > 1 && lay->q_stride_head != paged->q_stride_head)))
        return LOOKM_ERR_INVALID_ARG;
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
    std::vector<EvictReq> reqs;
    long long off = 0;
    for (int r = 0; r < n; ++r) {
        EvictReq q;
        q.len = lens[r];
        q.budget = std::min(budgets[r], lens[r]);
        q.window = std::min(windows[r], q.budget);
        q.index = r;
        q.kept_off = off;
        off += (long long)q.budget * paged->n_kv_heads;
        if (q.budget > 0) reqs.push_back(q);
    }
    // the longest first, so that none of them is left for the end
    std::stable_sort(reqs.begin(), reqs.end(), [](const EvictReq& a, const EvictReq& b) { return a.budget > b.budget; });
    for (size_t base = 0; base < reqs.size(); base += kManyRequests) {
        Batch<EvictReq, kManyRequests> b;
        b.n = (int)std::min<size_t>(kManyRequests, reqs.size() - base);
        b.pad = 0;
        for (int i = 0; i < b.n; ++i) b.r[i] = reqs[base + i];
        LOOKM_CUDA(launch_evict(p, b, in_place, di.sms, static_cast<cudaStream_t>(stream), &g_launches));
    }
    return LOOKM_OK;
}

// ---- attention of the newest tokens -----------------------------------------------------------------
constexpr int kMaxCtas = 192;            // of a launch
constexpr int kMassInside = 2048;        // rows of a cache

// The workspace behind the status word: partial rows of the pieces (two a CTA), logits and log-sum-exps of a step.
struct ChunkSpace { size_t parts, part_lse, logits, lse, total; };
ChunkSpace chunk_space(size_t slot_rows, size_t logits, size_t lse) {
    size_t o = kStatusBytes;
    auto carve = [&](size_t bytes) { size_t at = o; o = align_up(o + bytes, 256); return at; };
    ChunkSpace w;
    w.parts = carve(4 * kHeadDim * 2 * kMaxCtas * slot_rows);
    w.part_lse = carve(4 * 2 * kMaxCtas * slot_rows);
    w.logits = carve(4 * logits);
    w.lse = carve(4 * lse);
    w.total = o;
    return w;
}
int slot_rows(const lookm_paged_layout* l, long long most_new) {
    const int group = l->n_q_heads / l->n_kv_heads;
    return (int)std::min<long long>(2ll * (kTile / group) * group, std::max<long long>(most_new, 1) * group);
}

// The steps of all units, and of the CTA that has most in the kernel's deal of whole units (0: so many units that they even out).
struct Deal { long long steps, most; };
Deal deal(const ChunkReq* reqs, int n, int tile_tokens, int heads, int sms) {
    long long units = 0;
    Deal d = {0, 0};
    for (int r = 0; r < n; ++r) units += (long long)reqs[r].n_sets * heads;
    if (units >= 4ll * sms) return d;
    long long load[kMaxCtas] = {};
    int i = 0, step = 1;
    for (int r = 0; r < n; ++r)
        for (int s = reqs[r].n_sets - 1; s >= 0; --s) {
            const int k = chunk_unit(reqs[r], s, tile_tokens).steps;
            d.steps += (long long)k * heads;
            for (int h = 0; h < heads; ++h) {
                d.most = std::max(d.most, load[i] += k);
                i += step;
                if (i == sms || i < 0) { i -= step; step = -step; }
            }
        }
    return d;
}

// Whether the CTAs of a launch take equal shares of all units' steps instead of whole units: where the SM with the most whole units
// would be busy for longer than a share, a second launch and what the pieces' partial rows cost.  A step takes about
// 1 us.  us, whole | shares: one prompt of 4096 tokens x 32 heads 131 | 163, 512 tokens over 32256, 32 heads on 8, 433 | 256, 8 x 256 over
// 9000, 8 heads, 132 | 100, 16 x 128 over 9000, 32 on 8, 284 | 310, 100 over 5000 x 40 49 | 34, one over 2000 x 32 21.6 | 18.3, four
// of one over 1000 to 3000 x 32 35.1 | 36.3.
long long in_shares(const Deal& d, int rows, int sms) { return (d.steps + sms - 1) / sms + 8 + rows / 8; }
bool takes_shares(const ChunkReq* reqs, int n, int tile_tokens, int heads, int rows, int sms, long long* total) {
    const Deal d = deal(reqs, n, tile_tokens, heads, sms);
    *total = d.steps;
    return d.most > 0 && d.steps < (1ll << 30) && d.most > in_shares(d, rows, sms);
}

// The entries of a call's requests in the order in which their units are dealt: longest units first.  Of several requests with few
// sets every set is an entry of its own, so that the order is that of the sets (sixteen of 11 to 195 tokens over 2000 to 15000 rows, 32 heads
// on 8: 338 | 276 steps on the SM that has most).
std::vector<ChunkReq> chunk_entries(const std::vector<ChunkReq>& reqs, int tile_tokens, int set_tiles) {
    std::vector<ChunkReq> all;
    long long sets = 0;
    for (const ChunkReq& q : reqs) sets += ((q.n_new + tile_tokens - 1) / tile_tokens + set_tiles - 1) / set_tiles;
    const bool each = reqs.size() > 1 && sets <= kManyRequests;
    all.reserve(each ? sets : reqs.size());
    for (ChunkReq q : reqs) {
        q.set_tiles = set_tiles;
        q.n_sets = ((q.n_new + tile_tokens - 1) / tile_tokens + set_tiles - 1) / set_tiles;
        if (!each || q.n_sets == 1) {
            all.push_back(q);
            continue;
        }
        const int n = q.n_sets;
        q.n_sets = 1;
        for (q.set_begin = 0; q.set_begin < n; ++q.set_begin) all.push_back(q);
    }
    std::stable_sort(all.begin(), all.end(), [&](const ChunkReq& a, const ChunkReq& b) {
        return chunk_unit(a, a.n_sets - 1, tile_tokens).steps > chunk_unit(b, b.n_sets - 1, tile_tokens).steps;
    });
    return all;
}

// bf16 [tokens, heads, 128]: boxes of the rows of a query tile
int make_map_q(CUtensorMap* map, const void* base, long long tokens, const lookm_paged_layout* l, int group, int tile_tokens) {
    auto enc = tensor_map_encoder();
    if (!enc) return LOOKM_ERR_CUDA;
    cuuint64_t dims[3] = {(cuuint64_t)kHeadDim, (cuuint64_t)l->n_q_heads, (cuuint64_t)tokens};
    cuuint64_t strides[2] = {(cuuint64_t)l->q_stride_head * 2, (cuuint64_t)l->q_stride_tok * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)group, (cuuint32_t)tile_tokens};
    cuuint32_t estr[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? LOOKM_OK : LOOKM_ERR_CUDA;
}
// A pool: boxes of (a part of) a page of one head
int make_map_pool(CUtensorMap* map, const void* base, const lookm_paged_layout* l) {
    auto enc = tensor_map_encoder();
    if (!enc) return LOOKM_ERR_CUDA;
    cuuint64_t dims[4] = {(cuuint64_t)kHeadDim, (cuuint64_t)l->page_rows, (cuuint64_t)l->n_kv_heads, (cuuint64_t)l->n_pages};
    cuuint64_t strides[3] = {(cuuint64_t)l->row_stride * 2, (cuuint64_t)l->head_stride * 2, (cuuint64_t)l->page_stride * 2};
    cuuint32_t box[4] = {64, (cuuint32_t)std::min(l->page_rows, kTile), 1, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? LOOKM_OK : LOOKM_ERR_CUDA;
}

// cu: NULL for a step (one token per request, weights accumulated into mass).
int chunk_attention(const void* q, const void* cache_k, const void* cache_v, float* mass, const int* table, const int* cu, const int* lens,
                    int n, const lookm_paged_layout* paged, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
    LOOKM_TRY(check_paged(paged));
    const bool step = cu == nullptr;
    if (!q || !out || !aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4)) return LOOKM_ERR_INVALID_ARG;
    if (step && (!mass || !aligned(mass, 4))) return LOOKM_ERR_INVALID_ARG;
    for (long long s : {paged->q_stride_tok, paged->q_stride_head}) {
        if (s <= 0 || s % 8) return LOOKM_ERR_INVALID_ARG;
        if (s >= (1ll << 38)) return LOOKM_ERR_UNSUPPORTED;
    }
    if (!step) LOOKM_TRY(check_tokens(n, cu));
    LOOKM_TRY(check_requests(paged, n, lens));
    LOOKM_TRY(check_pool(cache_k, cache_v, table));
    const int group = paged->n_q_heads / paged->n_kv_heads;
    const long long tokens = step ? n : cu[n];
    const int tile_tokens = kTile / group;
    std::vector<ChunkReq> reqs;
    long long logits = 0, most_new = 0, units = 0;
    for (int r = 0; r < n; ++r) {
        ChunkReq c;
        c.q_begin = step ? r : cu[r];
        c.n_new = step ? 1 : cu[r + 1] - cu[r];
        c.len = lens[r];
        c.index = r;
        c.n_sets = (c.n_new + tile_tokens - 1) / tile_tokens;
        c.unit_begin = c.set_begin = c.step_begin = c.head_steps = 0;
        c.set_tiles = 1;
        c.logits_begin = logits;
        if (c.len < c.n_new) return LOOKM_ERR_INVALID_ARG;
        logits += step ? logits_stride(c.len) * paged->n_q_heads : 0;
        if (c.n_new) reqs.push_back(c);
        most_new = std::max<long long>(most_new, c.n_new);
        units += (long long)c.n_sets * paged->n_kv_heads;
    }
    if (units + kMaxCtas >= (1ll << 31) || tokens * paged->n_q_heads >= (1ll << 40)) return LOOKM_ERR_UNSUPPORTED;
    const int rows = slot_rows(paged, most_new);
    const ChunkSpace space = chunk_space(rows, logits, step && !lse ? tokens * paged->n_q_heads : 0);
    LOOKM_TRY(check_ws(ws, ws_bytes, space.total));
    DeviceInfo di;
    LOOKM_TRY(device_info(di));
    g_launches = 0;
    if (reqs.empty()) return LOOKM_OK;
    // Sets of one query tile where sets of two would leave SMs idle.  A step of a single tile takes 1.3 times a pair's, with pages of 16
    // rows, whose loading is the bound, 1.65 times.  us, pairs | singles: one prompt of 2048 tokens x 8 heads 35 | 25, of 4096 x 8 65 | 42, of 2048 x 32
    // 45 | 55, four of 128 tokens over 3000, 32 heads on 8, 53 | 34, eight of 256 over 9000, 8 heads, 104 | 93; two of 60 over 4000, 32 on 8,
    // pages of 16, 37 | 56.
    const int sms = std::min(di.sms, kMaxCtas), heads = paged->n_kv_heads;
    std::vector<ChunkReq> entries = chunk_entries(reqs, tile_tokens, 2);
    if (most_new > tile_tokens && entries.size() <= (size_t)kManyRequests) {
        const Deal two = deal(entries.data(), (int)entries.size(), tile_tokens, heads, sms);
        if (two.most > 0) {
            std::vector<ChunkReq> singles = chunk_entries(reqs, tile_tokens, 1);
            if (singles.size() <= (size_t)kManyRequests) {
                const Deal one = deal(singles.data(), (int)singles.size(), tile_tokens, heads, sms);
                const long long in_ones = std::min(one.most, in_shares(one, std::min(rows, kTile), sms)),
                                in_twos = std::min(two.most, in_shares(two, rows, sms));
                if (one.most > 0 && (paged->page_rows == 16 ? 33 : 26) * in_ones < 20 * in_twos) entries.swap(singles);
            }
        }
    }
    reqs.swap(entries);
    CUtensorMap map_q, map_k, map_v;
    LOOKM_TRY(make_map_q(&map_q, q, tokens, paged, group, tile_tokens));
    LOOKM_TRY(make_map_pool(&map_k, cache_k, paged));
    LOOKM_TRY(make_map_pool(&map_v, cache_v, paged));
    ChunkParams p;
    p.pages = pages_of(paged, table);
    p.group = group;
    p.tile_tokens = tile_tokens;
    // Two warps load pages of 16 rows where every unit has one query tile and so memory is the bound (sixteen single tokens over 400 to 8192
    // rows, 32 heads on 8, us, one | two: 59.5 | 56.5); one of them is then missing where values are looked over (a prompt of 4096
    // x 32: 135 | 151).  Pages of 32 rows: 54.3 | 56.4.
    p.loaders = paged->page_rows == 16 && most_new <= tile_tokens ? 2 : 1;
    p.slot_rows = rows;
    p.n_tokens = (int)tokens;
    p.scale_log2 = scale_log2(paged);
    p.cache_v = cache_v;
    p.out = out;
    p.lse = lse ? lse : step ? at<float>(ws, space.lse) : nullptr;
    p.part_out = at<float>(ws, space.parts);
    p.part_lse = at<float>(ws, space.part_lse);
    p.logits = step ? at<float>(ws, space.logits) : nullptr;
    p.mass = mass;
    p.status = at<int>(ws, 0);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    for (size_t base = 0; base < reqs.size(); base += kManyRequests) {
        Batch<ChunkReq, kManyRequests> b;
        b.n = (int)std::min<size_t>(kManyRequests, reqs.size() - base);
        b.pad = 0;
        long long total = 0;
        const bool shares = takes_shares(&reqs[base], b.n, tile_tokens, heads, reqs[base].set_tiles == 1 ? std::min(rows, kTile) : rows, sms, &total);
        int ctas = sms;
        // Weights of short caches don't wait for a second launch.  (Of long ones half a CTA would take too long.)
        int longest = 0;
        for (int i = 0; i < b.n; ++i) longest = std::max(longest, reqs[base + i].len);
        p.mass_inside = step && longest <= kMassInside;
        p.n_units = p.share = p.total_steps = 0;
        if (shares) {
            p.total_steps = (int)total;
            p.share = (int)((total + sms - 1) / sms);
            ctas = (int)((total + p.share - 1) / p.share);
        }
        int at_step = 0;
        for (int i = 0; i < b.n; ++i) {
            ChunkReq& c = b.r[i] = reqs[base + i];
            c.unit_begin = p.n_units;
            p.n_units += c.n_sets * heads;
            if (!shares) continue;
            for (int s = 0; s < c.n_sets; ++s) c.head_steps += chunk_unit(c, s, tile_tokens).steps;
            c.step_begin = at_step;
            at_step += c.head_steps * heads;
        }
        LOOKM_CUDA(launch_chunk(map_q, map_k, map_v, p, b, std::min(ctas, shares ? ctas : p.n_units), st));
        ++g_launches;
        if (shares || (step && !p.mass_inside)) {
            LOOKM_CUDA(launch_chunk_finish(p, b, st));
            ++g_launches;
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
    size_t rows = 0, tokens = 0, logits = 0;
    for (int r = 0; r < n_requests; ++r) {
        if (new_lens_host && new_lens_host[r] < 0) return 0;
        rows += cache_lens_host[r];
        logits += logits_stride(cache_lens_host[r]) * paged->n_q_heads;
        tokens += new_lens_host ? new_lens_host[r] : 1;
    }
    long long most_new = 1;
    for (int r = 0; r < n_requests; ++r) most_new = std::max<long long>(most_new, new_lens_host ? new_lens_host[r] : 1);
    const size_t attention = chunk_space(slot_rows(paged, most_new), logits,
                                         std::max(tokens, (size_t)n_requests) * paged->n_q_heads).total;
    return std::max(align_up(kStatusBytes + 4 * rows * paged->n_kv_heads, 256), attention);
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

int lookm_chunk_attention(const void* q, const void* cache_k, const void* cache_v, const int* page_table, const int* cu_seqlens_host,
                          const int* cache_lens_host, int n_requests, const lookm_paged_layout* paged, void* out, float* lse,
                          void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!cu_seqlens_host) return LOOKM_ERR_INVALID_ARG;
    return guarded([&] {
        return chunk_attention(q, cache_k, cache_v, nullptr, page_table, cu_seqlens_host, cache_lens_host, n_requests, paged, out, lse,
                               workspace, workspace_bytes, cuda_stream);
    });
}

int lookm_step_attention(const void* q, const void* cache_k, const void* cache_v, float* mass, const int* page_table,
                         const int* cache_lens_host, int n_requests, const lookm_paged_layout* paged, void* out, float* lse,
                         void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return guarded([&] {
        return chunk_attention(q, cache_k, cache_v, mass, page_table, nullptr, cache_lens_host, n_requests, paged, out, lse, workspace,
                               workspace_bytes, cuda_stream);
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

// Eviction from a paged cache by accumulated attention weight: of the rows 0 .. len - 1 of a (request, KV head) the last
// `window` stay and the budget - window heaviest of the others, the lower row first among equals; what stays moves to rows
// 0 .. budget - 1 in its order.
//
// evict_select_kernel finds the rows (latency bound: four counting passes over keys that stay in registers), evict_copy_kernel and
// evict_in_place_kernel move their keys, values and masses (HBM bound: every kept row read and written once).
//   8192 rows x 8 heads down to 20 % 16 us (the launches' own cost is 6), 30000 x 8 29; sixteen caches of 1000 to 8192 rows x 32 heads down to
// 80 % in place 349 us = 5.4 TB/s, 0.83 of the copy rate, in a long row of calls 352 (rows, their pages and their numbers each waited for in turn: 752; two of the three asked
// for early 430; two or four rows a thread instead of three 350 and 429).
#include <algorithm>

#include "paged.h"
#include "ptx.cuh"

namespace lookm {
namespace {

constexpr int kSelThreads = 1024, kSelWarps = kSelThreads / 32;
constexpr int kHistCopies = 4;                   // warps that would count in the same word wait for one another

// Masses in an order that unsigned integers have: -0 as +0, NaN below everything.  Never 0: that is for rows beyond the candidates.
__device__ __forceinline__ uint32_t key_of(float x) {
    if (x != x) return 1u;
    const uint32_t b = __float_as_uint(x + 0.f);
    return (b & 0x80000000u) ? max(~b, 2u) : b | 0x80000000u;
}

// A cluster of CTAs per (request, KV head), each with consecutive candidates.  kKeys > 0: so many of them per thread, whose keys stay in
// registers; 0: any number, read again in every pass.
//   The threshold is the n_top-th largest key, found eight bits a step from counts of the digit among the keys that begin with what
// is known of it; the CTAs read one another's counts.  (Two bits a step by counting in registers took four times as long: three
// reductions per warp and step.)
template <int kKeys, int kRequests>
__global__ void __launch_bounds__(kSelThreads)
evict_select_kernel(const EvictParams p, const __grid_constant__ Batch<EvictReq, kRequests> batch, int cluster) {
    __shared__ int hist[kHistCopies][256];
    __shared__ int counts[2][256];               // of the CTA; two passes' in turn, so that one may still be read
    __shared__ int warp_total[8], found[2], above_equal[2];
    __shared__ int2 warp_count[kSelWarps];
    const EvictReq& rq = batch.r[blockIdx.y];
    const int h = blockIdx.x / cluster, rank = blockIdx.x % cluster, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n_cand = rq.len - rq.window, n_top = rq.budget - rq.window;
    const auto sync = [&] { if (cluster > 1) ptx::cluster_sync(); else __syncthreads(); };
    grid_dependency_wait();
    int* kept = p.kept + rq.kept_off + (long long)h * rq.budget;
    if (rank == 0)
        for (int i = threadIdx.x; i < rq.window; i += kSelThreads) kept[n_top + i] = n_cand + i;
    if (n_top == n_cand) {                       // nothing leaves
        for (int i = rank * kSelThreads + threadIdx.x; i < n_top; i += cluster * kSelThreads) kept[i] = i;
        return;
    }
    if (n_top == 0) return;
    // every warp has an even share of consecutive rows, one per lane and step
    const int steps = (n_cand + cluster * kSelThreads - 1) / (cluster * kSelThreads), w0 = (rank * kSelWarps + warp) * steps * 32;
    const auto read = [&](int s) {
        const int t = w0 + s * 32 + lane;
        if (s >= steps || t >= n_cand) return 0u;
        const int page = p.pages.page_of(rq.index, t, p.status);
        return page < 0 ? 1u : key_of(__ldg(p.mass + p.pages.mass_at(page, t, h)));
    };
    uint32_t key[kKeys > 0 ? kKeys : 1];
    if constexpr (kKeys > 0) {
#pragma unroll
        for (int s = 0; s < kKeys; ++s) key[s] = read(s);
    }
    const auto for_each = [&](auto&& f) {
        if constexpr (kKeys > 0) {
#pragma unroll
            for (int s = 0; s < kKeys; ++s) f(s, key[s]);
        } else {
            for (int s = 0; s < steps; ++s) f(s, read(s));
        }
    };
    uint32_t x = 0;
    int want = n_top, buf = 0;                   // rank of the threshold among the keys that begin with x
    for (int shift = 24; shift >= 0; shift -= 8, buf ^= 1) {
        for (int i = threadIdx.x; i < kHistCopies * 256; i += kSelThreads) (&hist[0][0])[i] = 0;
        __syncthreads();
        for_each([&](int, uint32_t k) {
            if (k != 0 && (shift == 24 || (k ^ x) >> (shift + 8) == 0)) atomicAdd(&hist[warp % kHistCopies][(k >> shift) & 255], 1);
        });
        __syncthreads();
        const int digit = 255 - threadIdx.x;
        if (threadIdx.x < 256) {
            int n = 0;
#pragma unroll
            for (int i = 0; i < kHistCopies; ++i) n += hist[i][digit];
            counts[buf][digit] = n;
        }
        sync();
        int n = 0, at_least = 0;                 // keys with this thread's digit, keys of the warp's with it or a larger one
        if (threadIdx.x < 256) {
            n = counts[buf][digit];
            for (int c = 1; c < cluster; ++c) n += ptx::ld_cluster_int(&counts[buf][digit], (rank + c) % cluster);
            at_least = n;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, at_least, d);
                if (lane >= d) at_least += y;
            }
            if (lane == 31) warp_total[warp] = at_least;
        }
        __syncthreads();
        if (threadIdx.x < 256) {
            for (int i = 0; i < warp; ++i) at_least += warp_total[i];
            if (at_least >= want && at_least - n < want) {
                found[0] = digit;
                found[1] = want - (at_least - n);
            }
        }
        __syncthreads();
        x |= (uint32_t)found[0] << shift;
        want = found[1];
    }
    // Rows above it all stay; of those equal to it the lowest that there is room for, `want`.
    int2 mine = {0, 0};                          // above, equal: of the warp
    for_each([&](int, uint32_t k) {
        mine.x += __popc(__ballot_sync(0xffffffffu, k > x));
        mine.y += __popc(__ballot_sync(0xffffffffu, k == x));
    });
    if (lane == 0) warp_count[warp] = mine;
    __syncthreads();
    int2 c = warp_count[lane];
    if (threadIdx.x < 32) {
        const int a = __reduce_add_sync(0xffffffffu, c.x), e = __reduce_add_sync(0xffffffffu, c.y);
        if (lane == 0) { above_equal[0] = a; above_equal[1] = e; }
    }
    sync();
    int at = 0, equal = 0;                       // above and equal before the warp's rows
    for (int r = 0; r < rank; ++r) {
        at += ptx::ld_cluster_int(&above_equal[0], r);
        equal += ptx::ld_cluster_int(&above_equal[1], r);
    }
    if (lane >= warp) c = make_int2(0, 0);
    at += __reduce_add_sync(0xffffffffu, c.x);
    equal += __reduce_add_sync(0xffffffffu, c.y);
    at += min(equal, want);
    for_each([&](int s, uint32_t k) {
        const unsigned lower = (1u << lane) - 1u;
        const unsigned eq = __ballot_sync(0xffffffffu, k == x);
        const bool stays = k > x || (k == x && equal + __popc(eq & lower) < want);
        const unsigned all = __ballot_sync(0xffffffffu, stays);
        if (stays) kept[at + __popc(all & lower)] = w0 + s * 32 + lane;
        at += __popc(all);
        equal += __popc(eq);
    });
    if (cluster > 1) ptx::cluster_sync();        // (no CTA leaves while another may read its counts)
}

constexpr int kMoveThreads = 256;
constexpr int kMoveRows = 4;                     // of a half-warp at a time

// To pages that share none with the cache's: half a warp per kept row, its key and its value together.
template <int kRequests>
__global__ void __launch_bounds__(kMoveThreads)
evict_copy_kernel(const EvictParams p, const __grid_constant__ Batch<EvictReq, kRequests> batch) {
    const EvictReq& rq = batch.r[blockIdx.z];
    const int h = blockIdx.y, l = threadIdx.x & 15;
    constexpr int kRows = kMoveThreads / 16 * kMoveRows;
    const int i0 = blockIdx.x * kRows + (threadIdx.x >> 4);
    grid_dependency_wait();
    if (blockIdx.x * kRows >= rq.budget) return;
    const int* kept = p.kept + rq.kept_off + (long long)h * rq.budget;
    Pages out = p.pages;
    out.table = p.out_table;
    uint4 k[kMoveRows], v[kMoveRows];
    float m[kMoveRows];
    long long to[kMoveRows], to_mass[kMoveRows];
    int from[kMoveRows];
#pragma unroll
    for (int j = 0; j < kMoveRows; ++j) {
        const int i = i0 + j * (kMoveThreads / 16);
        from[j] = i < rq.budget ? kept[i] : -1;
    }
#pragma unroll
    for (int j = 0; j < kMoveRows; ++j) {
        const int i = i0 + j * (kMoveThreads / 16);
        to[j] = -1;
        if (from[j] < 0) continue;
        const int src = p.pages.page_of(rq.index, from[j], p.status), dst = out.page_of(rq.index, i, p.status);
        if (src < 0 || dst < 0) continue;
        const long long at = 2 * p.pages.row_at(src, from[j], h) + l * 16;
        k[j] = __ldg(reinterpret_cast<const uint4*>(static_cast<const char*>(p.cache_k) + at));
        v[j] = __ldg(reinterpret_cast<const uint4*>(static_cast<const char*>(p.cache_v) + at));
        if (l == 0) m[j] = __ldg(p.mass + p.pages.mass_at(src, from[j], h));
        to[j] = 2 * out.row_at(dst, i, h) + l * 16;
        to_mass[j] = out.mass_at(dst, i, h);
    }
#pragma unroll
    for (int j = 0; j < kMoveRows; ++j) {
        if (to[j] < 0) continue;
        *reinterpret_cast<uint4*>(static_cast<char*>(p.out_k) + to[j]) = k[j];
        *reinterpret_cast<uint4*>(static_cast<char*>(p.out_v) + to[j]) = v[j];
        if (l == 0) p.out_mass[to_mass[j]] = m[j];
    }
}

// In place.  A cluster of CTAs takes a slice of 1 / kSlices of the features of all kept rows of one pool's head, in ascending order and
// a batch at a time: all loads of a batch, a barrier, its stores.  Row i comes from row kept[i] >= i, so a store never hits a row
// that a later batch still reads, and other clusters touch other bytes.  The rows of the next batch are asked for before this one's are
// stored, their pages a batch earlier and their numbers another.
constexpr int kPlaceRows = 3;                    // of a thread at a time
template <int kSlices, int kRequests>
__global__ void __launch_bounds__(kMoveThreads)
evict_in_place_kernel(const EvictParams p, const __grid_constant__ Batch<EvictReq, kRequests> batch, int cluster) {
    constexpr int kLanes = 16 / kSlices, kGroups = kMoveThreads / kLanes;        // lanes of a row, rows side by side
    const int unit = blockIdx.x / cluster, part = blockIdx.x % cluster, group = part * kGroups + threadIdx.x / kLanes;
    const int side = kGroups * cluster, step = side * kPlaceRows;
    const EvictReq& rq = batch.r[blockIdx.z];
    const int h = blockIdx.y, slice = unit >> 1;
    const bool is_v = unit & 1, has_mass = unit == 0 && threadIdx.x % kLanes == 0;
    grid_dependency_wait();
    const int* kept = p.kept + rq.kept_off + (long long)h * rq.budget;
    const char* in = static_cast<const char*>(is_v ? p.cache_v : p.cache_k) + (slice * kLanes + threadIdx.x % kLanes) * 16;
    char* to_pool = static_cast<char*>(is_v ? p.out_v : p.out_k) + (slice * kLanes + threadIdx.x % kLanes) * 16;
    // Nothing is waited for before it is needed, an iteration after it was asked for: row numbers, their pages, their rows.
    int after[kPlaceRows], from[kPlaceRows], src[kPlaceRows];
    const auto numbers = [&](int base) {
#pragma unroll
        for (int j = 0; j < kPlaceRows; ++j) {
            const int i = base + j * side + group;
            after[j] = i < rq.budget ? kept[i] : -1;
        }
    };
    const auto table_entry = [&](const int* table, int t) { return __ldg(table + (long long)rq.index * p.pages.table_stride + (t >> p.pages.page_shift)); };
    const auto pages = [&] {                     // of the numbers
#pragma unroll
        for (int j = 0; j < kPlaceRows; ++j) {
            from[j] = after[j];
            src[j] = from[j] < 0 ? 0 : table_entry(p.pages.table, from[j]);
        }
    };
    const auto is_page = [&](int page) {
        if (page >= 0 && page < p.pages.n_pages) return true;
        atomicMax(p.status, (int)LOOKM_ERR_DEVICE_BAD_INDEX);
        return false;
    };
    struct Rows {
        uint4 x[kPlaceRows];
        float m[kPlaceRows];
        int page[kPlaceRows];                    // where they go, if `live` has their bit
        unsigned live;
    } now, next;
    const auto rows = [&](int base, Rows& b) {
        b.live = 0;
#pragma unroll
        for (int j = 0; j < kPlaceRows; ++j) {
            if (from[j] < 0 || !is_page(src[j])) continue;
            b.live |= 1u << j;
            b.x[j] = *reinterpret_cast<const uint4*>(in + 2 * p.pages.row_at(src[j], from[j], h));
            if (has_mass) b.m[j] = p.mass[p.pages.mass_at(src[j], from[j], h)];
            b.page[j] = table_entry(p.out_table, base + j * side + group);
        }
    };
    numbers(0);
    pages();
    numbers(step);
    rows(0, now);
    pages();
    numbers(2 * step);
    for (int base = 0; base < rq.budget; base += step) {
        rows(base + step, next);
        pages();
        numbers(base + 3 * step);
        if (cluster > 1) ptx::cluster_sync(); else __syncthreads();
#pragma unroll
        for (int j = 0; j < kPlaceRows; ++j) {
            const int i = base + j * side + group;
            if (!(now.live >> j & 1) || !is_page(now.page[j])) continue;
            *reinterpret_cast<uint4*>(to_pool + 2 * p.pages.row_at(now.page[j], i, h)) = now.x[j];
            if (has_mass) p.out_mass[p.pages.mass_at(now.page[j], i, h)] = now.m[j];
        }
        now = next;
    }
}

template <int kRequests>
cudaError_t launch(const EvictParams& p, const Batch<EvictReq, kManyRequests>& batch, bool in_place, int num_sms, cudaStream_t stream,
                   int* launches) {
    Batch<EvictReq, kRequests> b;
    b.n = batch.n;
    b.pad = 0;
    int candidates = 0, budget = 0;
    for (int i = 0; i < kRequests; ++i) {
        b.r[i] = i < batch.n ? batch.r[i] : EvictReq{0, 0, 0, 0, 0};
        candidates = std::max(candidates, b.r[i].len - b.r[i].window);
        budget = std::max(budget, b.r[i].budget);
    }
    const int heads = p.pages.n_kv_heads;
    // Clusters down to two rows a thread, as long as all CTAs find room at once (two per SM).  us, one CTA a head | clusters: 30000 rows x 8
    // heads 52.5 | 29.4; too many CTAs: eight caches of 8000 x 32 90 | 122.
    int cluster = 1;
    while (cluster < 8 && candidates > cluster * 2 * kSelThreads && 2ll * cluster * heads * b.n <= 2 * num_sms) cluster *= 2;
    const int each = (candidates + cluster - 1) / cluster;
    const auto select = each <= 2 * kSelThreads    ? evict_select_kernel<2, kRequests>
                        : each <= 8 * kSelThreads  ? evict_select_kernel<8, kRequests>
                        : each <= 32 * kSelThreads ? evict_select_kernel<32, kRequests>
                                                   : evict_select_kernel<0, kRequests>;
    cudaError_t err = launch_chained_clusters(select, dim3(heads * cluster, b.n), dim3(kSelThreads), cluster, 0, stream, p, b, cluster);
    if (err != cudaSuccess) return err;
    ++*launches;
    if (in_place) {
        // Few units (pools x heads x requests): slices and clusters until every SM has some CTAs, as long as a batch does not exceed
        // the rows.
        const long long units = 2ll * heads * b.n, want = 4ll * num_sms;
        const int slices = units * 2 >= want ? 2 : 4;
        int cluster = 1;
        while (cluster < 8 && units * slices * cluster * 2 <= want + want / 4 &&
               cluster * 2 * kPlaceRows * kMoveThreads * slices / 16 <= budget)
            cluster *= 2;
        const auto move = slices == 2 ? evict_in_place_kernel<2, kRequests> : evict_in_place_kernel<4, kRequests>;
        err = launch_chained_clusters(move, dim3(2 * slices * cluster, heads, b.n), dim3(kMoveThreads), cluster, 0, stream, p, b, cluster);
    } else {
        constexpr int kRows = kMoveThreads / 16 * kMoveRows;
        err = launch_chained(evict_copy_kernel<kRequests>, dim3((budget + kRows - 1) / kRows, heads, b.n), dim3(kMoveThreads), 0, stream,
                             p, b);
    }
    if (err == cudaSuccess) ++*launches;
    return err;
}

}  // namespace

cudaError_t launch_evict(const EvictParams& p, const Batch<EvictReq, kManyRequests>& batch, bool in_place, int num_sms,
                         cudaStream_t stream, int* launches) {
    return batch.n <= kFewRequests ? launch<kFewRequests>(p, batch, in_place, num_sms, stream, launches)
                                   : launch<kManyRequests>(p, batch, in_place, num_sms, stream, launches);
}

}  // namespace lookm

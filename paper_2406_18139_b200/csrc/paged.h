// Internal declarations of the operators over a paged cache: paged_api.cu (host), append_kernel.cu,
// chunk_kernel.cu, evict_kernels.cu.
#pragma once
#include "internal.h"

namespace lookm {

// A paged cache as the kernels see it.  Row t of KV head h of request r is row t % page_rows of page
// table[r * table_stride + t / page_rows].
struct Pages {
    const int* table;
    int table_stride, n_pages;
    int page_shift;              // page_rows = 1 << page_shift
    int n_q_heads, n_kv_heads;
    long long page_stride, row_stride, head_stride;      // elements of the K and V pools
#ifdef __CUDACC__
    // The page of row t of request r; -1 (and *status) if the table names none.
    __device__ __forceinline__ int page_of(int r, int t, int* status) const {
        const int p = __ldg(table + (long long)r * table_stride + (t >> page_shift));
        if (p >= 0 && p < n_pages) return p;
        atomicMax(status, (int)LOOKM_ERR_DEVICE_BAD_INDEX);
        return -1;
    }
    __device__ __forceinline__ long long row_at(int page, int t, int h) const {
        return page * page_stride + (t & ((1 << page_shift) - 1)) * row_stride + h * head_stride;
    }
    __device__ __forceinline__ long long mass_at(int page, int t, int h) const {
        return (((long long)page * n_kv_heads + h) << page_shift) + (t & ((1 << page_shift) - 1));
    }
#endif
};

// The requests of a launch, by value (no table in device memory, no copy that would synchronise the host).  A launch takes
// kFewRequests (kFewChunks) or kManyRequests of them; longer batches take several launches.
constexpr int kFewRequests = 16, kManyRequests = 128, kFewChunks = 32;
template <class R, int kRequests>
struct Batch {
    int n;
    int pad;
    R r[kRequests];
};

// ---- append_kernel.cu ----------------------------------------------------------------------------
struct AppendReq {
    int tok_begin;               // first token on the packed token axis (ascending; the next one's ends it)
    int row_begin;               // cache row of that token
    int index;                   // of the request in the page table
    int pad;
};
constexpr int kMaxFreqs = kHeadDim / 2;
struct AppendParams {
    Pages pages;
    const void *q, *k, *v;       // q may be NULL
    const int* positions;
    long long q_stride_tok, q_stride_head, kv_stride_tok, kv_stride_head;
    const void *q_weight, *k_weight;     // [128] bf16 or NULL
    float eps;
    int rotary_dim, interleaved;
    void* q_out;
    long long qo_stride_tok, qo_stride_head;
    void *cache_k, *cache_v;
    float* mass;                 // or NULL
    int tok_begin, tok_end;      // tokens of this launch
    int* status;
    double turns[kMaxFreqs];     // frequencies in turns per position: inv_freq / (2 pi)
};
cudaError_t launch_append(const AppendParams& p, const Batch<AppendReq, kManyRequests>& batch, int num_sms, cudaStream_t stream);

// ---- chunk_kernel.cu -----------------------------------------------------------------------------
// Attention of the newest tokens of each request; a request may have several entries, one per set of query tiles.  The query rows
// of a KV head are (token, query head of the group) pairs, the heads of a token side by side; a tile has the rows of kTile / group
// tokens.
struct ChunkReq {
    int q_begin, n_new;          // its tokens on the packed axis
    int len;                     // cached rows, the new ones included
    int index;                   // of the request in the page table
    int unit_begin;              // units of the launch before its own
    int set_begin, n_sets;       // sets of query tiles that this entry has
    int step_begin;              // shares: steps of the launch before its own
    int head_steps;              // shares: steps of one of its KV heads
    int set_tiles;               // query tiles of a set: 2 (the request's last set perhaps 1), or 1
    long long logits_begin;      // steps with weights: first logit of its [query head][row] block
};
// Floats between two query heads' logits of a step: whole fours, for wide stores.
#ifdef __CUDACC__
__host__ __device__
#endif
inline long long logits_stride(int len) { return (len + 3) & ~3; }
// A unit of work: a set of query tiles of a KV head.
struct ChunkUnit {
    int tok0;                    // first token
    bool pair;                   // two query tiles
    int tiles0, tiles;           // tiles of cached rows that its first query tile sees, that it sees
    int steps;                   // its share of the work: so many for itself, and one per tile and query tile
};
constexpr int kUnitSteps = 2;
#ifdef __CUDACC__
__host__ __device__
#endif
inline ChunkUnit chunk_unit(const ChunkReq& q, int set, int tile_tokens) {
    ChunkUnit u;
    u.tok0 = (q.set_begin + set) * q.set_tiles * tile_tokens;
    u.pair = q.set_tiles == 2 && u.tok0 + tile_tokens < q.n_new;
    const int before = q.len - q.n_new, first = u.tok0 + tile_tokens, second = first + tile_tokens;
    u.tiles0 = (before + (first < q.n_new ? first : q.n_new) + kTile - 1) / kTile;
    u.tiles = u.pair ? (before + (second < q.n_new ? second : q.n_new) + kTile - 1) / kTile : u.tiles0;
    u.steps = kUnitSteps + (u.pair ? 2 : 1) * u.tiles;
    return u;
}
// The tile at which a cut after `local` of a unit's steps falls.
#ifdef __CUDACC__
__host__ __device__
#endif
inline int chunk_cut(const ChunkUnit& u, int local) {
    if (local >= u.steps) return u.tiles;
    const int t = (local - kUnitSteps) >> (u.pair ? 1 : 0);
    return t > 0 ? t : 0;
}
struct ChunkParams {
    Pages pages;
    int group, tile_tokens;      // query heads of a KV head, tokens of a query tile
    int n_units;
    int n_tokens;                // on the packed axis (= the row stride of lse)
    int share;                   // > 0: the CTAs take so many steps each of all units' ...
    int total_steps;             // ... which are so many; units that are cut leave partial rows
    int loaders;                 // warps that load the cached rows: 1 or 2
    int slot_rows;               // partial rows of a piece: two pieces per CTA, its first and its last
    float scale_log2;            // softmax scale * log2(e)
    const void* cache_v;
    void* out;                   // [tokens, n_q_heads, 128] bf16
    float* lse;                  // [n_q_heads, tokens] or NULL
    float* part_out;             // partial rows, normalised: [piece][row][128]
    float* part_lse;             // their log2-sum-exp2
    float* logits;               // steps with weights: q.k of every row (unscaled)
    float* mass;                 // steps with weights
    int mass_inside;             // ... of whole units are accumulated by the CTA that has the unit
    int* status;
};
cudaError_t launch_chunk(const CUtensorMap& map_q, const CUtensorMap& map_k, const CUtensorMap& map_v, const ChunkParams& p,
                         const Batch<ChunkReq, kManyRequests>& batch, int grid, cudaStream_t stream);
// Adds up the pieces of units that were cut, and with p.mass every row's weight to its mass.
cudaError_t launch_chunk_finish(const ChunkParams& p, const Batch<ChunkReq, kManyRequests>& batch, cudaStream_t stream);

// ---- evict_kernels.cu ------------------------------------------------------------------------------
struct EvictReq {
    int len, budget, window;     // window <= budget <= len
    int index;
    long long kept_off;          // start of its kept lists
};
struct EvictParams {
    Pages pages;
    const int* out_table;
    const void *cache_k, *cache_v;
    const float* mass;
    void *out_k, *out_v;
    float* out_mass;
    int* kept;
    int* status;
};
cudaError_t launch_evict(const EvictParams& p, const Batch<EvictReq, kManyRequests>& batch, bool in_place, int num_sms,
                         cudaStream_t stream, int* launches);

}  // namespace lookm

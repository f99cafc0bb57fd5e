// Attention of each request's newest tokens over its paged cache, causal among themselves:
//
//     s_ij = q_i . k_j * scale  for rows j <= len - n_new + i,   out_i = sum_j softmax(s_i)_j v_j
//
// chunk_kernel: persistent, one CTA per SM.  Two streams of work run side by side, each with a 128 x 128 fp32 block of logits
// and one of outputs in tensor memory (all 512 columns) and a warpgroup that turns logits into probabilities; while one
// warpgroup works, the tensor core multiplies for the other.  A unit of work is one KV head of one request with
//   two query tiles (128 rows each: tokens x query heads of the group): both streams meet every tile of 128 cached rows, or
//   one query tile: the streams take the cached rows' tiles alternately and are added up at the end.
// CTAs take whole units or, where these leave SMs idle, equal shares of all units' tiles (the pieces of units that are cut are
// added up by a second launch).
//   warps 0-3, 4-7  softmax of stream 0 and 1: a thread has a row of logits.  Probabilities become bf16 (the type of V, which
//                   the tensor core wants on both sides: an error of at most 2^-8 each that averages out over the row's sum, no
//                   larger than the output's own rounding) and lie where the logits lay, as the A operand of P V.  Sums stay
//                   fp32.  The reference that is subtracted follows the maximum only when that has grown by 2^8, so outputs are
//                   seldom rescaled
//   warp 8          query tiles and cached rows by TMA, page by page, into one ring of tiles for K and V alternately
//   warp 9          issues the MMAs: S = Q K^T, O += P V.  They run in the order they are issued in, so the next S may
//                   overwrite the P that the product before it reads
//   warps 10-11     V rows that not every row of the unit sees: what lies behind the cache's end becomes zero, and so do
//                   infinities and NaN (0 times which would be NaN in rows that don't see them); rows that do see them get
//                   them in the epilogue
//
// What bounds it.  Many query rows: the hand-overs from softmax to issuing warp to tensor core and back, some 1200 of 3600 clocks per
// two tiles; then the softmax (1900) and the products (2048), which overlap.  8192 tokens x 32 heads 468 us = 1.17 PFLOP/s, in a long
// row of calls 550 us at the board's power limit (tensor pipe half busy, special-function unit half).  Without exponentials 460,
// without any softmax arithmetic 417, with an eighth of P V 413, of Q K^T 397, of both 375.
// Slower: one issuing warp per stream (561: their products take turns and both streams wait longer), sixteen softmax warps with
// half a row each (582: 104 registers do not do), exponentials partly on the FMA pipe (+3 to 7 %), the reference from the tiles
// before so that exponentials need not wait for the maximum (500), polling instead of suspended waits (490).
// Few query rows: memory.  Sixteen single tokens over 400 to 8192 rows, 32 heads on 8, 57 us = 4.9 TB/s (58 in a long row of calls); with weights, over
// 400 to 16384, 107 us (110).
#include <algorithm>

#include <cuda_bf16.h>
#include <math.h>

#include "paged.h"
#include "ptx_paged.cuh"

namespace lookm {
namespace {

constexpr int kSoftmaxWarps = 8, kLoadWarp = 8, kMmaWarp = 9, kCleanWarp = 10;
constexpr int kThreads = 384;
constexpr int kHalfBytes = kTile * 64 * 2, kTileBytes = 2 * kHalfBytes;
constexpr int kRing = 5;
// Items between a flag's uses.  Values of item i + 4 may be looked over before stream 1 has written item i's outputs: of i + 1 to i + 4 it may
// have no tile, S of i + 2 needs nobody's outputs, and five tiles of the ring hold what comes after its K tile.  So five at least.
constexpr int kFlags = 8;
constexpr int kSoftmaxRegs = 216, kOtherRegs = 72;
static_assert(256 * kSoftmaxRegs + 128 * kOtherRegs <= 65536 / kThreads / 8 * 8 * kThreads, "register shares exceed the launch's");
constexpr float kRescaleAt = 8.f;                // log2 of the growth of a row's maximum at which its reference follows

struct __align__(1024) ChunkShared {
    uint8_t q[2][kTileBytes];
    uint8_t ring[kRing][kTileBytes];
    unsigned long long q_full[2], q_empty[2];
    unsigned long long full[kRing], empty[kRing];
    unsigned long long dirty[kRing];             // V tiles that warps 10 and 11 have to look at; they make them full
    unsigned long long s_full[2], p_part[2][2], pv_done[2], o_free[2];         // (p_part: halves of a tile's rows)
    unsigned long long merge_full, merge_free, lse_full, mma_done;
    float merge_m[kTile], merge_l[kTile];        // one query tile: stream 1's reference and sum
    float lse2[kTile];                           // steps: the rows' log2-sum-exp2
    int odd_values[kFlags];                      // V had infinities or NaN that were taken out
    uint32_t tmem_base;
    int abort_flag;
};
static_assert(sizeof(ChunkShared) <= 232448, "shared memory exceeds 227 KB");

struct Item {
    int q_begin, n_new, len, index, head;
    int tok0;                                    // of its first query tile
    bool pair;                                   // two query tiles
    bool partial;                                // a piece of a unit
    int piece;
    int t0;                                      // first tile of cached rows
    int nt, nt0, nt1;                            // tiles of cached rows: all (loaded; at least one), of stream 0, of stream 1
    int min_seen;                                // cached rows that its first token sees: every row of the item sees these
    long long logits_begin;
};

// The items of a CTA, which every role walks through by itself.  Either whole units, those of the longest requests and of
// these the sets that see most first, dealt in serpentine order; or equal shares of all units' steps, in which a
// CTA's first and last item may be a piece of a unit.
struct Walk {
    int round;
    int pos, begin;                              // shares: position, first step of the unit that it is in
    int r, head, set;                            // that unit

    template <int kRequests>
    __device__ __forceinline__ void start(const ChunkParams& p, const Batch<ChunkReq, kRequests>& batch) {
        round = 0;
        if (p.share > 0) find(blockIdx.x * p.share, p, batch);
    }
    // To step `at`.
    template <int kRequests>
    __device__ __forceinline__ void find(int at, const ChunkParams& p, const Batch<ChunkReq, kRequests>& batch) {
        pos = at;
        int lo = 0, hi = batch.n - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (batch.r[mid].step_begin <= pos) lo = mid; else hi = mid - 1;
        }
        r = lo;
        const ChunkReq& q = batch.r[r];
        head = (pos - q.step_begin) / q.head_steps;
        begin = q.step_begin + head * q.head_steps;
        set = 0;
        for (;;) {
            const int n = chunk_unit(q, set, p.tile_tokens).steps;
            if (begin + n > pos || set + 1 == q.n_sets) break;
            begin += n;
            ++set;
        }
    }
    // False: there is no further item.
    template <int kRequests>
    __device__ __forceinline__ bool next(const ChunkParams& p, const Batch<ChunkReq, kRequests>& batch, Item& it) {
        ChunkUnit u;
        int t0, t1, at_r;
        if (p.share == 0) {
            const int n = gridDim.x, i = round * n + ((round & 1) ? n - 1 - (int)blockIdx.x : (int)blockIdx.x);
            if (round * n >= p.n_units) return false;
            ++round;
            if (i >= p.n_units) return false;    // (only the last round is not full)
            int lo = 0, hi = batch.n - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (batch.r[mid].unit_begin <= i) lo = mid; else hi = mid - 1;
            }
            at_r = lo;
            const int k = i - batch.r[lo].unit_begin;
            it.head = k % p.pages.n_kv_heads;
            u = chunk_unit(batch.r[lo], batch.r[lo].n_sets - 1 - k / p.pages.n_kv_heads, p.tile_tokens);
            t0 = 0;
            t1 = u.tiles;
            it.piece = 0;
        } else {
            const int first = blockIdx.x * p.share, end = min(first + p.share, p.total_steps);
            do {
                if (pos >= end) return false;
                at_r = r;
                it.head = head;
                const ChunkReq& q = batch.r[r];
                u = chunk_unit(q, set, p.tile_tokens);
                t0 = chunk_cut(u, pos - begin);
                t1 = chunk_cut(u, end - begin);
                it.piece = 2 * blockIdx.x + (pos == first ? 0 : 1);
                pos = begin + u.steps;
                if (pos <= end) {                // on to the next unit
                    begin = pos;
                    if (++set == q.n_sets) {
                        set = 0;
                        if (++head == p.pages.n_kv_heads) { head = 0; ++r; }
                    }
                }
            } while (t0 == t1);
        }
        const ChunkReq& q = batch.r[at_r];
        it.q_begin = q.q_begin;
        it.n_new = q.n_new;
        it.len = q.len;
        it.index = q.index;
        it.logits_begin = q.logits_begin;
        it.tok0 = u.tok0;
        it.pair = u.pair;
        it.min_seen = q.len - q.n_new + u.tok0 + 1;
        it.t0 = t0;
        it.nt = t1 - t0;
        it.partial = it.nt != u.tiles;
        if (u.pair) {
            it.nt1 = it.nt;
            it.nt0 = min(max(u.tiles0 - t0, 0), it.nt);
        } else {
            it.nt0 = (it.nt + 1) >> 1;
            it.nt1 = it.nt >> 1;
        }
        return true;
    }
};
// Whether some row of the item does not see all 128 rows of tile t (or the cache ends in it).
__device__ __forceinline__ bool is_masked(const Item& it, int t) { return (it.t0 + t + 1) * kTile > it.min_seen; }

// The waits of a warp: all lanes wait, and all follow one verdict.
__device__ __forceinline__ bool warp_wait(unsigned long long* bar, uint32_t parity, volatile int* abort_flag) {
    return __all_sync(0xffffffffu, ptx::mbar_wait(ptx::smem_u32(bar), parity, abort_flag));
}

__device__ __forceinline__ bool odd_bf16(uint32_t x) { return (x & 0x7f80u) == 0x7f80u; }     // infinity or NaN

// ---- warp 8, and warp 11 where there are two loaders --------------------------------------------------
// A copy of half the features of a page's rows takes some 65 clocks to issue: 1000 per tile of pages of 16 rows, more than memory needs for the
// tile.  So two warps may take half of its pages each (p.loaders); warp 8 alone announces the bytes.
template <int kRequests>
__device__ __forceinline__ void load_tiles(const CUtensorMap& map_q, const CUtensorMap& map_k, const CUtensorMap& map_v,
                                           const ChunkParams& p, const Batch<ChunkReq, kRequests>& batch, ChunkShared& sh, int part) {
    const int lane = threadIdx.x & 31;
    volatile int* abort_flag = &sh.abort_flag;
    if (lane == 0) {
        ptx::prefetch_tensormap(&map_q);
        ptx::prefetch_tensormap(&map_k);
        ptx::prefetch_tensormap(&map_v);
    }
    const int box_rows = min(1 << p.pages.page_shift, kTile), boxes = kTile / box_rows / p.loaders, box = part * boxes + lane;
    const int q_bytes = p.tile_tokens * p.group * 256;
    uint32_t n = 0, nq = 0;                      // tiles and query tiles armed so far
    uint32_t dirty_phase = 0, last_dirty = 0;    // per stage: parity of its next use as a dirty one, whether its last use was one
    bool stop = false;
    Walk walk;
    Item it;
    walk.start(p, batch);
    while (!stop && walk.next(p, batch, it)) {
        for (int g = 0; part == 0 && g < (it.pair ? 2 : 1) && !stop; ++g, ++nq) {
            const int s = nq & 1;
            if (!warp_wait(&sh.q_empty[s], ((nq >> 1) & 1) ^ 1, abort_flag)) { stop = true; break; }
            if (lane == 0) {
                const uint32_t bar = ptx::smem_u32(&sh.q_full[s]), dst = ptx::smem_u32(&sh.q[s][0]);
                const int tok = it.q_begin + it.tok0 + g * p.tile_tokens;
                ptx::mbar_arrive_expect_tx(bar, q_bytes);
                ptx::tma_load_3d(dst, &map_q, 0, it.head * p.group, tok, bar);
                ptx::tma_load_3d(dst + kHalfBytes, &map_q, 64, it.head * p.group, tok, bar);
            }
        }
        // The table's entry for this lane's part of tile t, asked for a tile ahead and looked at when it is needed; where there is none, one
        // beyond the pool, which reads as zeros.
        const auto page_for = [&](int t) {
            const int row = (it.t0 + t) * kTile + box * box_rows;
            if (t >= it.nt || lane >= boxes || row >= it.len) return p.pages.n_pages;
            return __ldg(p.pages.table + (long long)it.index * p.pages.table_stride + (row >> p.pages.page_shift));
        };
        const auto load = [&](const CUtensorMap& map, int t, int page, bool dirty) {
            if (stop) return;
            const int s = n % kRing;
            if (!warp_wait(&sh.empty[s], ((n / kRing) & 1) ^ 1, abort_flag)) { stop = true; return; }
            const uint32_t bar = ptx::smem_u32(dirty ? &sh.dirty[s] : &sh.full[s]);
            if (part == 0 && lane == 0) {
                ptx::mbar_arrive_expect_tx(bar, kTileBytes);
                if (!dirty) ptx::mbar_arrive(bar);           // (a full tile takes two arrivals: the cleaning warps may be two)
            }
            last_dirty = (last_dirty & ~(1u << s)) | (dirty ? 1u << s : 0u);
            if (dirty) dirty_phase ^= 1u << s;
            __syncwarp();
            if (lane < boxes) {
                if (page < 0 || page > p.pages.n_pages ||
                    (page == p.pages.n_pages && (it.t0 + t) * kTile + box * box_rows < it.len)) {
                    atomicMax(p.status, (int)LOOKM_ERR_DEVICE_BAD_INDEX);
                    page = p.pages.n_pages;
                }
                const uint32_t dst = ptx::smem_u32(&sh.ring[s][0]) + box * box_rows * 128;
                const int in_page = ((it.t0 + t) * kTile + box * box_rows) & ((1 << p.pages.page_shift) - 1);
                ptx::tma_load_4d(dst, &map, 0, in_page, it.head, page, bar);
                ptx::tma_load_4d(dst + kHalfBytes, &map, 64, in_page, it.head, page, bar);
            }
            ++n;
        };
        // K runs ahead of V by one tile, with one query tile by two
        int page = page_for(0), page1 = page_for(1), page2 = 0;
        load(map_k, 0, page, false);
        if (!it.pair && it.nt > 1) load(map_k, 1, page1, false);
        for (int t = 0; t < it.nt && !stop; ++t) {
            page2 = page_for(t + 2);
            load(map_v, t, page, is_masked(it, t));
            if (it.pair && t + 1 < it.nt) load(map_k, t + 1, page1, false);
            if (!it.pair && t + 2 < it.nt) load(map_k, t + 2, page2, false);
            page = page1;
            page1 = page2;
        }
    }
    // After an abort: no copy may write shared memory once the CTA has left (bounded, the flag is ignored).
    if (*abort_flag && lane == 0) {
        int ignore = 0;
        for (uint32_t i = n > (uint32_t)kRing ? n - kRing : 0; i < n; ++i)
            if (last_dirty >> (i % kRing) & 1)
                ptx::mbar_wait(ptx::smem_u32(&sh.dirty[i % kRing]), (dirty_phase >> (i % kRing) & 1) ^ 1, &ignore, 200000000ull);
            else
                ptx::mbar_wait(ptx::smem_u32(&sh.full[i % kRing]), (i / kRing) & 1, &ignore, 200000000ull);
        for (uint32_t i = nq > 2u ? nq - 2 : 0; i < nq; ++i)
            ptx::mbar_wait(ptx::smem_u32(&sh.q_full[i & 1]), (i >> 1) & 1, &ignore, 200000000ull);
    }
    __syncwarp();
}

// ---- warp 9 ---------------------------------------------------------------------------------------
// The whole warp walks through the protocol and one lane issues: what the instructions take then lies in uniform registers.  (With
// one lane alone in the code, the eight MMAs of a product took 670 clocks to issue, more than their 512 to run.)
template <int kRequests>
__device__ __forceinline__ void issue_mmas(const ChunkParams& p, const Batch<ChunkReq, kRequests>& batch, ChunkShared& sh, uint32_t tmem) {
    volatile int* abort_flag = &sh.abort_flag;
    constexpr uint32_t idesc_s = ptx::umma_idesc_bf16(kTile, kTile), idesc_o = ptx::umma_idesc_bf16(kTile, kHeadDim) | ptx::kIdescBMnMajor;
    uint32_t n = 0, nq = 0;
    uint32_t p_phase = 0, o_phase = 3;           // a bit per stream: parity of the wait for its next probabilities, for its free outputs
    bool stop = false;
    const bool leader = ptx::elect_one();
    const auto commit = [&](unsigned long long* bar) { if (leader) ptx::umma_commit(ptx::smem_u32(bar)); };
    const auto wait = [&](unsigned long long* bar, uint32_t parity) {
        if (!stop && !warp_wait(bar, parity, abort_flag)) stop = true;
    };
    Walk walk;
    Item it;
    walk.start(p, batch);
    while (!stop && walk.next(p, batch, it)) {
        const int tiles = it.pair ? 2 : 1;
        for (int g = 0; g < tiles; ++g) wait(&sh.q_full[(nq + g) & 1], ((nq + g) >> 1) & 1);
        const auto qk = [&](int g, uint32_t stage) {             // S of stream g = its query tile x K^T
            if (stop) return;
            const uint64_t a = ptx::umma_desc_sw128(ptx::smem_u32(&sh.q[(nq + (it.pair ? g : 0)) & 1][0])),
                           b = ptx::umma_desc_sw128(ptx::smem_u32(&sh.ring[stage][0]));
            const uint32_t d = tmem + g * kTile;
            if (leader) {
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {             // (descriptors count in units of 16 bytes)
                    const uint32_t off = ((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4;
                    ptx::umma_bf16(d, a + off, b + off, idesc_s, kk > 0);
                }
            }
            commit(&sh.s_full[g]);
        };
        uint32_t begun = 0;                      // a bit per stream: its output block has something of this item
        const auto pv = [&](int g, uint32_t stage) {             // O of stream g += P x V
            wait(&sh.p_part[g][0], (p_phase >> g) & 1);
            if (stop) return;
            ptx::tc_fence_after_sync();
            const uint64_t b = ptx::umma_desc_sw128_mn(ptx::smem_u32(&sh.ring[stage][0]), kHalfBytes);
            const uint32_t d = tmem + 2 * kTile + g * kHeadDim, pr = tmem + g * kTile, more = begun >> g & 1;
            if (leader) {
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) ptx::umma_bf16_ts(d, pr + kk * 8, b + kk * (2048 >> 4), idesc_o, kk > 0 ? 1u : more);
            }
            wait(&sh.p_part[g][1], (p_phase >> g) & 1);
            if (stop) return;
            ptx::tc_fence_after_sync();
            if (leader) {
#pragma unroll
                for (int kk = 4; kk < 8; ++kk) ptx::umma_bf16_ts(d, pr + kk * 8, b + kk * (2048 >> 4), idesc_o, 1u);
            }
            p_phase ^= 1u << g;
            begun |= 1u << g;
            commit(&sh.pv_done[g]);
        };
        const auto arrived = [&] {               // the next tile of the ring
            const uint32_t s = n % kRing;
            wait(&sh.full[s], (n / kRing) & 1);
            ++n;
            if (!stop) ptx::tc_fence_after_sync();
            return s;
        };
        const auto release = [&](uint32_t s) { if (!stop) commit(&sh.empty[s]); };
        const auto queries_done = [&] {
            for (int g = 0; g < tiles && !stop; ++g) commit(&sh.q_empty[(nq + g) & 1]);
        };
        // the output blocks are free when the epilogue of the item before has read them
        const auto outputs_free = [&] {
            if (it.nt0 > 0) { wait(&sh.o_free[0], o_phase & 1); o_phase ^= 1; }
            if (it.nt1 > 0) { wait(&sh.o_free[1], o_phase >> 1); o_phase ^= 2; }
        };
        if (it.pair) {
            uint32_t k = arrived();
            if (it.nt0 > 0) qk(0, k);
            qk(1, k);
            release(k);
            if (it.nt == 1) queries_done();
            outputs_free();
            for (int t = 0; t < it.nt && !stop; ++t) {
                const uint32_t v = arrived();    // (both waits before those that matter: the tensor core's queue is short)
                if (t + 1 < it.nt) k = arrived();
                if (t < it.nt0) pv(0, v);
                if (t + 1 < it.nt0) qk(0, k);
                pv(1, v);
                release(v);
                if (t + 1 < it.nt) {
                    qk(1, k);
                    release(k);
                    if (t + 2 == it.nt) queries_done();
                }
            }
        } else {
            for (int t = 0; t < min(it.nt, 2); ++t) {
                const uint32_t k = arrived();
                qk(t, k);
                release(k);
            }
            if (it.nt <= 2) queries_done();
            outputs_free();
            for (int t = 0; t < it.nt && !stop; ++t) {
                const uint32_t v = arrived();
                uint32_t k = 0;
                if (t + 2 < it.nt) k = arrived();
                pv(t & 1, v);
                if (t + 2 < it.nt) qk(t & 1, k);
                release(v);
                if (t + 2 < it.nt) {
                    release(k);
                    if (t + 3 == it.nt) queries_done();
                }
            }
        }
        nq += tiles;
    }
    int ignore = 0;                              // no MMA may be running when TMEM is released
    commit(&sh.mma_done);
    ptx::mbar_wait(ptx::smem_u32(&sh.mma_done), 0, &ignore, 1000000000ull);
    __syncwarp();
}

// ---- warps 10 and 11 --------------------------------------------------------------------------------
template <int kRequests>
__device__ __forceinline__ void clean_values(const ChunkParams& p, const Batch<ChunkReq, kRequests>& batch, ChunkShared& sh) {
    const int lane = threadIdx.x & 31;
    const bool alone = p.loaders == 2;          // (else the two warps have half of the features each)
    const int half0 = alone ? 0 : (threadIdx.x >> 5) - kCleanWarp, half1 = alone ? 2 : half0 + 1;
    volatile int* abort_flag = &sh.abort_flag;
    uint32_t n = 0, n_items = 0, phase = 0;
    Walk walk;
    Item it;
    walk.start(p, batch);
    while (walk.next(p, batch, it)) {
        for (int t = 0; t < it.nt; ++t) {
            // the ring position of V tile t: K and V take turns, with one K tile ahead, or two with one query tile
            const uint32_t at = n + (it.pair ? 2 * t + 1 : t < it.nt - 1 ? 2 * t + 2 : 2 * t + 1);
            if (!is_masked(it, t)) continue;
            const uint32_t s = at % kRing;
            if (!warp_wait(&sh.dirty[s], (phase >> s) & 1, abort_flag)) return;
            phase ^= 1u << s;
            const int row0 = (it.t0 + t) * kTile;
            const int end = min(max(it.len - row0, 0), kTile), all_see = min(max(it.min_seen - row0, 0), kTile);
            bool odd = false;
            for (int half = half0; half < half1; ++half) {
                uint4* v = reinterpret_cast<uint4*>(&sh.ring[s][half * kHalfBytes]);  // [128 rows][8]; within a row any order
                for (int i = end * 8 + lane; i < kTile * 8; i += 32) v[i] = make_uint4(0, 0, 0, 0);
#pragma unroll 4
                for (int i = all_see * 8 + lane; i < end * 8; i += 32) {
                    uint4 x = v[i];
                    uint32_t* w = reinterpret_cast<uint32_t*>(&x);
                    bool here = false;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (odd_bf16(w[j])) { w[j] &= 0xffff0000u; here = true; }
                        if (odd_bf16(w[j] >> 16)) { w[j] &= 0xffffu; here = true; }
                    }
                    if (here) { v[i] = x; odd = true; }
                }
            }
            if (odd) sh.odd_values[n_items % kFlags] = (int)n_items + 1;
            ptx::fence_proxy_async_shared();
            __syncwarp();
            if (lane == 0) {
                ptx::mbar_arrive(ptx::smem_u32(&sh.full[s]));
                if (alone) ptx::mbar_arrive(ptx::smem_u32(&sh.full[s]));
            }
        }
        n += 2 * it.nt;
        ++n_items;
    }
}

// ---- warps 0 to 7 ------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 ab = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&ab);
}

// Steps: adds the weights of cached rows t, t + stride, ... < end to their mass, summed over the heads of the group; four rows at a time,
// pages and logits of two heads asked for together.  Requests may share pages (a prefix in common) and then add to the same masses: in one atomic
// operation each, so that nothing is lost.  A mass that one request adds to is that request's alone and doesn't depend on timing; the
// last bits of a shared one do, as the sharers come in any order.
__device__ __forceinline__ void add_weights(const ChunkParams& p, int index, int head, int len, const float* logits, const float* lse2, int t,
                                            int end, int stride) {
    const long long row = logits_stride(len);
    const int* table = p.pages.table + (long long)index * p.pages.table_stride;
    for (; t < end; t += 4 * stride) {
        int page[4];
        float w[4] = {0.f, 0.f, 0.f, 0.f}, x[2][4];
        const auto ask = [&](int g, float (&y)[4]) {
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = t + j * stride < end ? logits[g * row + t + j * stride] : 0.f;
        };
        const auto add = [&](int g, const float (&y)[4]) {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] += ptx::ex2(fmaf(y[j], p.scale_log2, -lse2[g]));
        };
#pragma unroll
        for (int j = 0; j < 4; ++j)
            page[j] = t + j * stride < end ? __ldg(table + ((t + j * stride) >> p.pages.page_shift)) : 0;
        ask(0, x[0]);
        if (p.group > 1) ask(1, x[1]);
        for (int g = 0; g < p.group; g += 2) {
            add(g, x[0]);
            if (g + 2 < p.group) ask(g + 2, x[0]);
            if (g + 1 < p.group) add(g + 1, x[1]);
            if (g + 3 < p.group) ask(g + 3, x[1]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (t + j * stride >= end) continue;
            if (page[j] >= 0 && page[j] < p.pages.n_pages)
                atomicAdd(p.mass + p.pages.mass_at(page[j], t + j * stride, head), w[j]);
            else
                atomicMax(p.status, (int)LOOKM_ERR_DEVICE_BAD_INDEX);
        }
    }
}

// 32 logits of a row as probabilities 2^(s * c + neg), in bf16 pairs; adds them up (before the rounding).
__device__ __forceinline__ void probabilities(const uint32_t (&s)[32], ptx::f32x2 c, ptx::f32x2 neg, ptx::f32x2 (&sum)[4], uint32_t (&pr)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float2 x = ptx::unpack2(ptx::fma2(ptx::pack2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), c, neg));
        const float a = ptx::ex2(x.x), b = ptx::ex2(x.y);
        sum[i & 3] = ptx::add2(sum[i & 3], ptx::pack2(a, b));
        pr[i] = pack_bf16(a, b);
    }
}

template <int kRequests, bool kStep>
__device__ __forceinline__ void softmax_rows(const ChunkParams& p, const Batch<ChunkReq, kRequests>& batch, ChunkShared& sh, uint32_t tmem) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = warp >> 2, row = (warp & 3) * 32 + lane;
    volatile int* abort_flag = &sh.abort_flag;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + g * kTile + lanes, to = tmem + 2 * kTile + g * kHeadDim + lanes;
    const float c = p.scale_log2;
    const int tok_in_tile = row / p.group, head_in_group = row - tok_in_tile * p.group;
    uint32_t n = 0, n_items = 0, n_merges = 0, n_masses = 0;
    Walk walk;
    Item it;
    walk.start(p, batch);
    while (walk.next(p, batch, it)) {
        const int tok = it.tok0 + (it.pair ? g * p.tile_tokens : 0) + tok_in_tile, q_head = it.head * p.group + head_in_group;
        const bool live = tok_in_tile < p.tile_tokens && tok < it.n_new;         // the row has a token
        const bool any_live = __any_sync(0xffffffffu, live);
        const int seen = live ? it.len - it.n_new + tok + 1 : 0x7fffffff;
        const int nt = g ? it.nt1 : it.nt0, t_first = it.t0 + (it.pair ? 0 : g), t_step = it.pair ? 1 : 2;
        float* to_logits = nullptr;
        if constexpr (kStep) to_logits = p.logits + it.logits_begin + (long long)q_head * logits_stride(it.len);
        float m = -INFINITY, l = 0.f;            // reference, sum
        for (int j = 0; j < nt; ++j, ++n) {
            const int t = t_first + j * t_step;
            if (!warp_wait(&sh.s_full[g], n & 1, abort_flag)) return;
            if (any_live) {
                uint32_t s[4][32];
                ptx::tc_fence_after_sync();
#pragma unroll
                for (int i = 0; i < 4; ++i) ptx::tmem_ld_32x32(ts + i * 32, s[i]);
                const int cols = seen - t * kTile;
                const bool masked = __any_sync(0xffffffffu, cols < kTile);
                ptx::tmem_ld_wait();
                if constexpr (kStep) {
                    if (live) {                  // (a step's rows see all that is cached; a row of logits has room for whole fours)
                        uint4* to_logits4 = reinterpret_cast<uint4*>(to_logits + t * kTile);
#pragma unroll
                        for (int i = 0; i < kTile / 4; ++i)
                            if (4 * i < cols)
                                to_logits4[i] = make_uint4(s[i >> 3][4 * i & 31], s[i >> 3][(4 * i & 31) + 1], s[i >> 3][(4 * i & 31) + 2],
                                                           s[i >> 3][(4 * i & 31) + 3]);
                    }
                    __syncwarp();
                }
                if (masked) {
#pragma unroll
                    for (int i = 0; i < kTile; ++i)
                        if (i >= cols) s[i >> 5][i & 31] = __float_as_uint(-INFINITY);
                }
                float mx[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    mx[i] = __uint_as_float(s[i][0]);
#pragma unroll
                    for (int k = 1; k < 31; k += 2) mx[i] = ptx::fmax3(mx[i], __uint_as_float(s[i][k]), __uint_as_float(s[i][k + 1]));
                    mx[i] = fmaxf(mx[i], __uint_as_float(s[i][31]));
                }
                const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                const bool grows = live && top > m && !((top - m) * c <= kRescaleAt);
                if (__any_sync(0xffffffffu, grows)) {
                    const float alpha = grows ? ptx::ex2((m - top) * c) : 1.f;
                    l *= alpha;
                    if (grows) m = top;
                    if (j > 0) {
                        if (!warp_wait(&sh.pv_done[g], (n - 1) & 1, abort_flag)) return;
                        ptx::tc_fence_after_sync();
#pragma unroll 1
                        for (int i = 0; i < kHeadDim; i += 16) {
                            uint32_t o[16];
                            ptx::tmem_ld_32x16(to + i, o);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                            ptx::tmem_st_32x16(to + i, o);
                        }
                    }
                }
                const float neg1 = m == -INFINITY ? 0.f : -m * c;
                const ptx::f32x2 c2 = ptx::pack2(c, c), neg = ptx::pack2(neg1, neg1);
                ptx::f32x2 sum[4] = {0, 0, 0, 0};
                uint32_t pr[16];
#pragma unroll
                for (int h = 0; h < 2; ++h) {    // the product with V begins with the first half of the rows
#pragma unroll
                    for (int i = 2 * h; i < 2 * h + 2; ++i) {
                        probabilities(s[i], c2, neg, sum, pr);
                        ptx::tmem_st_32x16(ts + i * 16, pr);
                    }
                    ptx::tmem_st_wait();
                    ptx::tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.p_part[g][h]));
                }
                const float2 v = ptx::unpack2(ptx::add2(ptx::add2(sum[0], sum[1]), ptx::add2(sum[2], sum[3])));
                l += v.x + v.y;
            } else if (lane == 0) {
                ptx::mbar_arrive(ptx::smem_u32(&sh.p_part[g][0]));
                ptx::mbar_arrive(ptx::smem_u32(&sh.p_part[g][1]));
            }
            __syncwarp();
        }
        // ---- the item's outputs ----
        if (nt > 0 && !warp_wait(&sh.pv_done[g], (n - 1) & 1, abort_flag)) return;
        ptx::tc_fence_after_sync();
        if (!it.pair && g == 1) {                // stream 0 adds both up
            if (!warp_wait(&sh.merge_free, (n_merges & 1) ^ 1, abort_flag)) return;
            sh.merge_m[row] = m;
            sh.merge_l[row] = l;
            ptx::tc_fence_before_sync();         // (stream 0 reads the output block that this one has waited for, and has rescaled)
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.merge_full));
            ++n_merges;
            ++n_items;
            continue;
        }
        float scale0 = 1.f, scale1 = 0.f, total = l, top = m;
        if (!it.pair) {
            if (!warp_wait(&sh.merge_full, n_merges & 1, abort_flag)) return;
            ptx::tc_fence_after_sync();          // (of stream 1's outputs only stream 1's warps know that they are there)
            ++n_merges;
            const float m1 = sh.merge_m[row], l1 = sh.merge_l[row];
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.merge_free));
            if (it.nt1 > 0) {
                top = fmaxf(m, m1);
                scale0 = m == top ? 1.f : ptx::ex2((m - top) * c);
                scale1 = m1 == top ? 1.f : ptx::ex2((m1 - top) * c);
                total = l * scale0 + l1 * scale1;
            }
        }
        const bool two = !it.pair && it.nt1 > 0;
        const float inv = 1.f / total;
        scale0 *= inv;
        scale1 *= inv;
        const float lse2 = (top == -INFINITY ? 0.f : top * c) + ptx::lg2(total);         // log2
        const bool nothing = it.partial && total == 0.f;         // a range of which the row sees none
        const bool odd = sh.odd_values[n_items % kFlags] == (int)n_items + 1;
        const long long part_row = (long long)it.piece * p.slot_rows + (tok - it.tok0) * p.group + head_in_group;
        const long long out_row = (long long)(it.q_begin + tok) * p.pages.n_q_heads + q_head;
        if (any_live) {
#pragma unroll 1
            for (int i = 0; i < kHeadDim; i += 16) {
                uint32_t o[16];
                if (nt > 0) {
                    ptx::tmem_ld_32x16(to + i, o);
                    ptx::tmem_ld_wait();
                }
#pragma unroll
                for (int k = 0; k < 16; ++k) o[k] = nothing || nt == 0 ? 0u : __float_as_uint(__uint_as_float(o[k]) * scale0);
                if (two) {
                    uint32_t o1[16];
                    ptx::tmem_ld_32x16(to + kHeadDim + i, o1);
                    ptx::tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (!nothing) o[k] = __float_as_uint(fmaf(__uint_as_float(o1[k]), scale1, __uint_as_float(o[k])));
                }
                if (odd && live) {               // infinities and NaN among the values that this row sees and others don't
                    for (int t = max(it.min_seen, it.t0 * kTile); t < min(seen, (it.t0 + it.nt) * kTile); ++t) {
                        const int page = p.pages.page_of(it.index, t, p.status);
                        if (page < 0) continue;
                        const uint32_t* v =
                            reinterpret_cast<const uint32_t*>(static_cast<const char*>(p.cache_v) + 2 * (p.pages.row_at(page, t, it.head) + i));
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const uint32_t x = v[k];
                            if (odd_bf16(x)) o[2 * k] = __float_as_uint(__uint_as_float(o[2 * k]) + __uint_as_float(x << 16));
                            if (odd_bf16(x >> 16)) o[2 * k + 1] = __float_as_uint(__uint_as_float(o[2 * k + 1]) + __uint_as_float(x & 0xffff0000u));
                        }
                    }
                }
                if (live && it.partial) {
                    uint4* dst = reinterpret_cast<uint4*>(p.part_out + part_row * kHeadDim + i);
#pragma unroll
                    for (int k = 0; k < 4; ++k) dst[k] = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
                } else if (live) {
                    uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + out_row * kHeadDim + i);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        uint32_t w[4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) w[x] = pack_bf16(__uint_as_float(o[8 * k + 2 * x]), __uint_as_float(o[8 * k + 2 * x + 1]));
                        dst[k] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
                __syncwarp();                    // (tensor memory is read by whole warps)
            }
            if (live) {
                if (it.partial) p.part_lse[part_row] = lse2;
                else if (p.lse) p.lse[(long long)q_head * p.n_tokens + it.q_begin + tok] = lse2 * 0.6931471805599453f;
            }
        }
        ptx::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) {
            if (nt > 0) ptx::mbar_arrive(ptx::smem_u32(&sh.o_free[g]));
            if (two) ptx::mbar_arrive(ptx::smem_u32(&sh.o_free[1]));
        }
        __syncwarp();
        if constexpr (kStep) {
            // The weights of a whole unit, by the warps of stream 0; the logits of both streams have been written (stream 1's before merge_full).
            if (p.mass_inside && !it.partial) {
                sh.lse2[row] = lse2;
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&sh.lse_full));
                if (!warp_wait(&sh.lse_full, n_masses & 1, abort_flag)) return;
                ++n_masses;
                add_weights(p, it.index, it.head, it.len, p.logits + it.logits_begin + (long long)it.head * p.group * logits_stride(it.len),
                            sh.lse2, row, it.len, kTile);
            }
        }
        ++n_items;
    }
}

template <int kRequests, bool kStep>
__global__ void __launch_bounds__(kThreads, 1)
chunk_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
             const __grid_constant__ ChunkParams p, const __grid_constant__ Batch<ChunkReq, kRequests> batch) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    ChunkShared& sh = *reinterpret_cast<ChunkShared*>(smem_raw);
    if (ptx::smem_u32(smem_raw) & 1023u) {       // (the swizzle needs it, and there is no room to round up in)
        grid_dependency_wait();
        if (threadIdx.x == 0) atomicMax(p.status, (int)LOOKM_ERR_UNSUPPORTED);
        return;
    }
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        const auto init = [](unsigned long long* bar, int count) { ptx::mbar_init(ptx::smem_u32(bar), count); };
        for (int i = 0; i < 2; ++i) {
            init(&sh.q_full[i], 1);
            init(&sh.q_empty[i], 1);
            init(&sh.s_full[i], 1);
            init(&sh.p_part[i][0], 4);
            init(&sh.p_part[i][1], 4);
            init(&sh.pv_done[i], 1);
            init(&sh.o_free[i], 4);
        }
        for (int i = 0; i < kRing; ++i) {
            init(&sh.full[i], 2);
            init(&sh.empty[i], 1);
            init(&sh.dirty[i], 1);
        }
        init(&sh.merge_full, 4);
        init(&sh.merge_free, 4);
        init(&sh.lse_full, 4);
        init(&sh.mma_done, 1);
        for (int i = 0; i < kFlags; ++i) sh.odd_values[i] = 0;
        sh.abort_flag = 0;
        ptx::fence_mbar_init();
    }
    if (warp == kMmaWarp) {
        ptx::tmem_alloc(ptx::smem_u32(&sh.tmem_base), 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    grid_dependency_wait();
    const uint32_t tmem = sh.tmem_base;
    if (warp < kSoftmaxWarps) {
        ptx::more_registers<kSoftmaxRegs>();
        softmax_rows<kRequests, kStep>(p, batch, sh, tmem);
    } else {
        ptx::fewer_registers<kOtherRegs>();
        if (warp == kLoadWarp) {
            load_tiles(map_q, map_k, map_v, p, batch, sh, 0);
        } else if (warp == kMmaWarp) {
            issue_mmas(p, batch, sh, tmem);
        } else if (warp == kCleanWarp + 1 && p.loaders == 2) {
            load_tiles(map_q, map_k, map_v, p, batch, sh, 1);
        } else {
            clean_values(p, batch, sh);
        }
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == kMmaWarp) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, 512);
    }
    if (threadIdx.x == 0 && sh.abort_flag) atomicMax(p.status, (int)LOOKM_ERR_DEVICE_TIMEOUT);
}

// ---- pieces added up, weights accumulated -----------------------------------------------------------
constexpr int kFinishThreads = 256, kFinishWarps = kFinishThreads / 32;
constexpr int kMassRows = 4 * kFinishThreads;    // cached rows of a CTA

// What a unit was cut into: CTAs first .. last, some of which may have none of its tiles.
struct Cuts {
    ChunkUnit u;
    int begin, first, last;
    __device__ __forceinline__ Cuts(const ChunkParams& p, const ChunkUnit& unit, int unit_begin) {
        u = unit;
        begin = unit_begin;
        first = last = 0;
        if (p.share == 0) return;
        first = begin / p.share;
        last = (begin + u.steps - 1) / p.share;
    }
    // The piece that CTA c has; -1: none
    __device__ __forceinline__ int piece_of(const ChunkParams& p, int c) const {
        const int from = c * p.share - begin, to = from + p.share;
        if (chunk_cut(u, max(from, 0)) == chunk_cut(u, to)) return -1;
        return 2 * c + (from >= 0 ? 0 : 1);
    }
    // Whether the unit has several pieces: a whole one has left none.
    __device__ __forceinline__ bool is_cut(const ChunkParams& p) const {
        if (first == last) return false;
        int pieces = 0;
        for (int c = first; c <= last && pieces < 2; ++c) pieces += piece_of(p, c) >= 0;
        return pieces > 1;
    }
};

// log2-sum-exp2 of a row of a unit that was cut; by kLanes lanes side by side, all of them of a warp together.
template <int kLanes>
__device__ __forceinline__ float row_lse2(const ChunkParams& p, const Cuts& cuts, int row) {
    const int lane = threadIdx.x & (kLanes - 1);
    float top = -INFINITY, sum = 0.f;
    for (int c = cuts.first + lane; c <= cuts.last; c += kLanes) {
        const int piece = cuts.piece_of(p, c);
        if (piece >= 0) top = fmaxf(top, p.part_lse[(long long)piece * p.slot_rows + row]);
    }
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    if (top == -INFINITY) top = 0.f;
    for (int c = cuts.first + lane; c <= cuts.last; c += kLanes) {
        const int piece = cuts.piece_of(p, c);
        if (piece >= 0) sum += ptx::ex2(p.part_lse[(long long)piece * p.slot_rows + row] - top);
    }
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    return top + ptx::lg2(sum);
}

// An output row of a unit that was cut, by half a warp: the pieces' rows in order, each times 2^(its log-sum-exp - the row's).  Both halves come
// here together, each with a row, which may be the same.
__device__ __forceinline__ void add_pieces(const ChunkParams& p, const ChunkReq& q, const Cuts& cuts, int head, int row) {
    const int lane = threadIdx.x & 15;
    const float lse2 = row_lse2<16>(p, cuts, row);
    float acc[8] = {};
    for (int c0 = cuts.first; c0 <= cuts.last; c0 += 16) {
        const int mine = c0 + lane <= cuts.last ? cuts.piece_of(p, c0 + lane) : -1;
        const float x = mine >= 0 ? p.part_lse[(long long)mine * p.slot_rows + row] : -INFINITY;
        const float w = x == -INFINITY ? 0.f : ptx::ex2(x - lse2);
        const int n = min(16, cuts.last - c0 + 1);
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
            const int piece = __shfl_sync(0xffffffffu, mine, i, 16);
            const float wi = __shfl_sync(0xffffffffu, w, i, 16), xi = __shfl_sync(0xffffffffu, x, i, 16);
            if (xi == -INFINITY) continue;
            const float4* o = reinterpret_cast<const float4*>(p.part_out + ((long long)piece * p.slot_rows + row) * kHeadDim + lane * 8);
            const float4 o0 = o[0], o1 = o[1];
            const float v[8] = {o0.x, o0.y, o0.z, o0.w, o1.x, o1.y, o1.z, o1.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) acc[k] = fmaf(v[k], wi, acc[k]);
        }
        __syncwarp();
    }
    const long long tok = q.q_begin + cuts.u.tok0 + row / p.group;
    const int q_head = head * p.group + row % p.group;
    if (lse2 == -INFINITY) {                     // no row has a weight
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[k] = NAN;
    }
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + (tok * p.pages.n_q_heads + q_head) * kHeadDim + lane * 8) =
        make_uint4(pack_bf16(acc[0], acc[1]), pack_bf16(acc[2], acc[3]), pack_bf16(acc[4], acc[5]), pack_bf16(acc[6], acc[7]));
    if (lane == 0 && p.lse) p.lse[(long long)q_head * p.n_tokens + tok] = lse2 * 0.6931471805599453f;
}
// ... all rows of the unit, `stride` half-warps from number `first` on
__device__ __forceinline__ void add_pieces_of_rows(const ChunkParams& p, const ChunkReq& q, const Cuts& cuts, int head, int first, int stride) {
    const int rows = min(q.n_new - cuts.u.tok0, q.set_tiles * p.tile_tokens) * p.group;
    const int half = (threadIdx.x >> 4) & 1;
    for (int row = first - half; row < rows; row += stride) add_pieces(p, q, cuts, head, min(row + half, rows - 1));
}

// blockIdx.x: a place between two CTAs' shares, and so a unit that may have been cut there (its first such place has it);
// blockIdx.y: rows in turn.
template <int kRequests>
__global__ void __launch_bounds__(kFinishThreads)
chunk_finish_kernel(const __grid_constant__ ChunkParams p, const __grid_constant__ Batch<ChunkReq, kRequests> batch) {
    Walk at;
    at.find((blockIdx.x + 1) * p.share, p, batch);
    const ChunkReq& q = batch.r[at.r];
    const Cuts cuts(p, chunk_unit(q, at.set, p.tile_tokens), at.begin);
    grid_dependency_wait();                      // (also by CTAs that leave: this grid's end has to mean the end of the one before it)
    if (cuts.first != (int)blockIdx.x || !cuts.is_cut(p)) return;
    add_pieces_of_rows(p, q, cuts, at.head, blockIdx.y * (2 * kFinishWarps) + (threadIdx.x >> 4), gridDim.y * 2 * kFinishWarps);
}

// Steps with weights.  blockIdx.x: unit; blockIdx.y: a block of its cached rows (the first also has the output rows).
template <int kRequests>
__global__ void __launch_bounds__(kFinishThreads, 4)
step_finish_kernel(const __grid_constant__ ChunkParams p, const __grid_constant__ Batch<ChunkReq, kRequests> batch) {
    __shared__ float lse2[kTile];
    int lo = 0, hi = batch.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (batch.r[mid].unit_begin <= (int)blockIdx.x) lo = mid; else hi = mid - 1;
    }
    const ChunkReq& q = batch.r[lo];
    const int head = blockIdx.x - q.unit_begin, warp = threadIdx.x >> 5;
    const Cuts cuts(p, chunk_unit(q, 0, p.tile_tokens), q.step_begin + head * q.head_steps);
    grid_dependency_wait();
    const bool is_cut = cuts.is_cut(p);
    if ((long long)blockIdx.y * kMassRows >= q.len || (p.mass_inside && !is_cut)) return;
    if (is_cut && blockIdx.y == 0) add_pieces_of_rows(p, q, cuts, head, threadIdx.x >> 4, 2 * kFinishWarps);
    for (int g = warp; g < p.group; g += kFinishWarps) {
        const float x = is_cut ? row_lse2<32>(p, cuts, g)
                               : p.lse[(long long)(head * p.group + g) * p.n_tokens + q.q_begin] * 1.4426950408889634f;
        if ((threadIdx.x & 31) == 0) lse2[g] = x;
    }
    __syncthreads();
    const int t0 = blockIdx.y * kMassRows;
    add_weights(p, q.index, head, q.len, p.logits + q.logits_begin + (long long)head * p.group * logits_stride(q.len), lse2, t0 + threadIdx.x,
                min(q.len, t0 + kMassRows), kFinishThreads);
}

template <int kRequests>
Batch<ChunkReq, kRequests> shorter(const Batch<ChunkReq, kManyRequests>& batch) {
    Batch<ChunkReq, kRequests> b;
    b.n = batch.n;
    b.pad = 0;
    for (int i = 0; i < kRequests; ++i) b.r[i] = i < batch.n ? batch.r[i] : ChunkReq{};
    return b;
}

template <int kRequests, bool kStep>
cudaError_t launch(const CUtensorMap& map_q, const CUtensorMap& map_k, const CUtensorMap& map_v, const ChunkParams& p,
                   const Batch<ChunkReq, kManyRequests>& batch, int grid, cudaStream_t stream) {
    constexpr size_t smem = sizeof(ChunkShared);
    static unsigned long long configured = 0;
    cudaError_t err = once_per_device(configured, [] {
        return cudaFuncSetAttribute(chunk_kernel<kRequests, kStep>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    });
    if (err != cudaSuccess) return err;
    return launch_chained(chunk_kernel<kRequests, kStep>, dim3(grid), dim3(kThreads), smem, stream, map_q, map_k, map_v, p,
                          shorter<kRequests>(batch));
}

template <int kRequests>
cudaError_t finish(const ChunkParams& p, const Batch<ChunkReq, kManyRequests>& batch, cudaStream_t stream) {
    if (p.mass) {
        int len = 0;
        for (int i = 0; i < batch.n; ++i) len = std::max(len, batch.r[i].len);
        return launch_chained(step_finish_kernel<kRequests>, dim3(p.n_units, (len + kMassRows - 1) / kMassRows), dim3(kFinishThreads), 0, stream,
                              p, shorter<kRequests>(batch));
    }
    const int places = (p.total_steps - 1) / p.share;
    if (places == 0) return cudaSuccess;
    return launch_chained(chunk_finish_kernel<kRequests>, dim3(places, (p.slot_rows + 2 * kFinishWarps - 1) / (2 * kFinishWarps)),
                          dim3(kFinishThreads), 0, stream, p, shorter<kRequests>(batch));
}

}  // namespace

cudaError_t launch_chunk(const CUtensorMap& map_q, const CUtensorMap& map_k, const CUtensorMap& map_v, const ChunkParams& p,
                         const Batch<ChunkReq, kManyRequests>& batch, int grid, cudaStream_t stream) {
    const bool few = batch.n <= kFewChunks;
    if (p.logits)
        return few ? launch<kFewChunks, true>(map_q, map_k, map_v, p, batch, grid, stream)
                   : launch<kManyRequests, true>(map_q, map_k, map_v, p, batch, grid, stream);
    return few ? launch<kFewChunks, false>(map_q, map_k, map_v, p, batch, grid, stream)
               : launch<kManyRequests, false>(map_q, map_k, map_v, p, batch, grid, stream);
}

cudaError_t launch_chunk_finish(const ChunkParams& p, const Batch<ChunkReq, kManyRequests>& batch, cudaStream_t stream) {
    return batch.n <= kFewChunks ? finish<kFewChunks>(p, batch, stream) : finish<kManyRequests>(p, batch, stream);
}

}  // namespace lookm

// New tokens on their way into a paged cache: per-head RMS norm of queries and keys, rotation to their positions,
// key and value rows written to the pages, the rows' mass set to zero.
//
//     y = x / sqrt(mean(x^2) + eps) * w        (a, b) -> (a cos - b sin, b cos + a sin)
//
// All in fp32 with one rounding to bf16 at the end.  The angle is position * frequency, taken in turns and in fp64 so
// that only its fraction is left before it becomes fp32: at position 2^20 an fp32 product would be off by 0.03 radians.
//
// Bound by HBM: every row is read once and written once.  Half a warp takes a row of 256 bytes.  Its lanes have eight features each:
// four and their partners in the rotation, so that no lane needs another's (eight consecutive ones of features that are not
// rotated, or whose partner is the next one).  A CTA takes a few tokens and some of their heads; its threads first work
// out these tokens' cosines and sines, which all heads share.
#include <algorithm>

#include <cuda_bf16.h>

#include "paged.h"
#include "ptx.cuh"

namespace lookm {
namespace {

constexpr int kThreads = 256, kHalfWarps = kThreads / 16;
constexpr int kTokens = 4;                       // of a CTA, at most
constexpr int kRows = 4;                         // of a half-warp at a time

struct TokenPlace { int index, row; };           // request and cache row

// Eight features of a lane: two groups of four, each two pairs.
struct Eight { ptx::f32x2 x[4]; };
__device__ __forceinline__ Eight unpack8(const uint2& a, const uint2& b) {
    const uint32_t w[4] = {a.x, a.y, b.x, b.y};
    Eight e;
#pragma unroll
    for (int i = 0; i < 4; ++i) e.x[i] = ptx::pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    return e;
}
__device__ __forceinline__ uint32_t pack_bf16(ptx::f32x2 x) {
    const float2 v = ptx::unpack2(x);
    const __nv_bfloat162 b = __floats2bfloat162_rn(v.x, v.y);
    return *reinterpret_cast<const uint32_t*>(&b);
}

// What a lane does to its features of every row of a token.
struct Rotation {
    bool turned, adjacent;       // whether its features are rotated; pairs are neighbours
    ptx::f32x2 cos[4], sin[4];   // adjacent: per pair, sin as (-sin, sin); else of the two pairs of the first group
};
__device__ __forceinline__ void norm_rotate(Eight& e, bool norm, const Eight& weight, float eps, const Rotation& r) {
    if (norm) {
        ptx::f32x2 sq = ptx::mul2(e.x[0], e.x[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) sq = ptx::fma2(e.x[i], e.x[i], sq);
        const float2 v = ptx::unpack2(sq);
        float sum = v.x + v.y;
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const float scale = rsqrtf(sum * (1.f / kHeadDim) + eps);
        const ptx::f32x2 scale2 = ptx::pack2(scale, scale);
#pragma unroll
        for (int i = 0; i < 4; ++i) e.x[i] = ptx::mul2(ptx::mul2(e.x[i], scale2), weight.x[i]);
    }
    if (!r.turned) return;
    if (r.adjacent) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 v = ptx::unpack2(e.x[i]);
            e.x[i] = ptx::fma2(e.x[i], r.cos[i], ptx::mul2(ptx::pack2(v.y, v.x), r.sin[i]));
        }
    } else {
        const ptx::f32x2 minus = ptx::pack2(-1.f, -1.f);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const ptx::f32x2 a = e.x[i], b = e.x[i + 2];
            e.x[i] = ptx::fma2(a, r.cos[i], ptx::mul2(ptx::mul2(b, r.sin[i]), minus));
            e.x[i + 2] = ptx::fma2(b, r.cos[i], ptx::mul2(a, r.sin[i]));
        }
    }
}

// Rows first .. last - 1 of a kind (queries, keys or values) of one token; all threads of the CTA.  kRows of a half-warp at a time, all
// asked for together.  Both halves of a warp run the same number of rounds: they shuffle together.
template <bool kWork>
__device__ __forceinline__ void token_rows(const char* from, long long from_stride, char* to, long long to_stride, int first, int last, int at_a,
                                           int at_b, bool norm, const Eight& weight, float eps, const Rotation& r) {
    const int half = (threadIdx.x >> 4) & 1;
    for (int i0 = first + (threadIdx.x >> 5) * 2; i0 < last; i0 += kHalfWarps * kRows) {
        uint2 a[kRows], b[kRows];
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
            const int i = i0 + j * kHalfWarps + half;
            a[j] = b[j] = make_uint2(0, 0);
            if (i < last) {
                a[j] = *reinterpret_cast<const uint2*>(from + i * from_stride + at_a);
                b[j] = *reinterpret_cast<const uint2*>(from + i * from_stride + at_b);
            }
        }
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
            const int i = i0 + j * kHalfWarps + half;
            if (i0 + j * kHalfWarps >= last) break;
            if (kWork && (norm || r.turned)) {
                Eight e = unpack8(a[j], b[j]);
                norm_rotate(e, norm, weight, eps, r);
                a[j] = make_uint2(pack_bf16(e.x[0]), pack_bf16(e.x[1]));
                b[j] = make_uint2(pack_bf16(e.x[2]), pack_bf16(e.x[3]));
            }
            if (kWork) __syncwarp();             // (lanes that are not rotated may have skipped)
            if (i < last) {
                *reinterpret_cast<uint2*>(to + i * to_stride + at_a) = a[j];
                *reinterpret_cast<uint2*>(to + i * to_stride + at_b) = b[j];
            }
        }
    }
}

template <int kRequests>
__global__ void __launch_bounds__(kThreads, 4)
append_kernel(const AppendParams p, const __grid_constant__ Batch<AppendReq, kRequests> batch, int tokens, int rows_per_cta) {
    __shared__ float2 turn[kTokens][kMaxFreqs];
    __shared__ TokenPlace place[kTokens];
    const int t0 = p.tok_begin + blockIdx.x * tokens, nt = min(tokens, p.tok_end - t0);
    if (threadIdx.x < nt) {
        const int t = t0 + threadIdx.x;
        int lo = 0, hi = batch.n - 1;            // last request that begins at t or before it: of empty ones at the same
        while (lo < hi) {                        // place the last, which is the one that has the token
            const int mid = (lo + hi + 1) >> 1;
            if (batch.r[mid].tok_begin <= t) lo = mid; else hi = mid - 1;
        }
        place[threadIdx.x] = {batch.r[lo].index, batch.r[lo].row_begin + t - batch.r[lo].tok_begin};
    }
    grid_dependency_wait();
    for (int i = threadIdx.x; i < nt * (p.rotary_dim >> 1); i += kThreads) {
        const int t = i / (p.rotary_dim >> 1), f = i - t * (p.rotary_dim >> 1);
        const double turns = (double)__ldg(p.positions + t0 + t) * p.turns[f];
        float2 v;
        sincospif(2.f * (float)(turns - rint(turns)), &v.y, &v.x);
        turn[t][f] = v;
    }
    __syncthreads();
    const int hq = p.q ? p.pages.n_q_heads : 0, hkv = p.pages.n_kv_heads;
    const int per_token = hq + 2 * hkv, first = blockIdx.y * rows_per_cta, last = min(first + rows_per_cta, per_token);
    const int l = threadIdx.x & 15;
    Rotation r;
    r.turned = l * 8 < p.rotary_dim;
    r.adjacent = p.interleaved;
    const bool split = r.turned && !p.interleaved;             // first group 4 l .. 4 l + 3, second group half a rotation further
    const int at_a = 2 * (split ? 4 * l : 8 * l), at_b = 2 * (split ? 4 * l + (p.rotary_dim >> 1) : 8 * l + 4);
    const auto weight_of = [&](const void* w) {
        const char* c = static_cast<const char*>(w);
        return c ? unpack8(__ldg(reinterpret_cast<const uint2*>(c + at_a)), __ldg(reinterpret_cast<const uint2*>(c + at_b))) : Eight{};
    };
    const Eight wq = weight_of(p.q_weight), wk = weight_of(p.k_weight);
    for (int t = 0; t < nt; ++t) {
        const TokenPlace at = place[t];
        const long long tok = t0 + t;
        if (r.turned) {
            const float2* angle = &turn[t][l * 4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (r.adjacent) {
                    r.cos[i] = ptx::pack2(angle[i].x, angle[i].x);
                    r.sin[i] = ptx::pack2(-angle[i].y, angle[i].y);
                } else if (i < 2) {
                    r.cos[i] = ptx::pack2(angle[2 * i].x, angle[2 * i + 1].x);
                    r.sin[i] = ptx::pack2(angle[2 * i].y, angle[2 * i + 1].y);
                }
            }
        }
        __syncwarp();
        if (first < hq)
            token_rows<true>(static_cast<const char*>(p.q) + 2 * tok * p.q_stride_tok, 2 * p.q_stride_head,
                             static_cast<char*>(p.q_out) + 2 * tok * p.qo_stride_tok, 2 * p.qo_stride_head, first, min(last, hq), at_a, at_b,
                             p.q_weight != nullptr, wq, p.eps, r);
        const int page = p.pages.page_of(at.index, at.row, p.status);
        if (page < 0) continue;
        const long long row = 2 * p.pages.row_at(page, at.row, 0), from = 2 * tok * p.kv_stride_tok;
        const int k0 = max(first - hq, 0), k1 = min(last - hq, hkv), v0 = max(first - hq - hkv, 0), v1 = last - hq - hkv;
        if (k0 < k1) {
            token_rows<true>(static_cast<const char*>(p.k) + from, 2 * p.kv_stride_head, static_cast<char*>(p.cache_k) + row,
                             2 * p.pages.head_stride, k0, k1, at_a, at_b, p.k_weight != nullptr, wk, p.eps, r);
            if (p.mass)
                for (int h = k0 + threadIdx.x; h < k1; h += kThreads) p.mass[p.pages.mass_at(page, at.row, h)] = 0.f;
        }
        if (v0 < v1)
            token_rows<false>(static_cast<const char*>(p.v) + from, 2 * p.kv_stride_head, static_cast<char*>(p.cache_v) + row,
                              2 * p.pages.head_stride, v0, v1, 16 * l, 16 * l + 8, false, wk, 0.f, r);
    }
}

template <int kRequests>
cudaError_t launch(const AppendParams& p, const Batch<AppendReq, kManyRequests>& batch, int num_sms, cudaStream_t stream) {
    Batch<AppendReq, kRequests> b;
    b.n = batch.n;
    b.pad = 0;
    for (int i = 0; i < kRequests; ++i) b.r[i] = i < batch.n ? batch.r[i] : AppendReq{0, 0, 0, 0};
    const int total = p.tok_end - p.tok_begin, per_token = (p.q ? p.pages.n_q_heads : 0) + 2 * p.pages.n_kv_heads;
    const int tokens = total >= kTokens * num_sms * 8 ? kTokens : 1, groups = (total + tokens - 1) / tokens;
    // few tokens: a token's rows are spread over CTAs, down to one row per half-warp
    const int parts = std::max(1, std::min((per_token + kHalfWarps - 1) / kHalfWarps, num_sms * 4 / groups));
    const int rows = ((per_token + parts - 1) / parts + 1) / 2 * 2;
    const dim3 grid(groups, (per_token + rows - 1) / rows);
    return launch_chained(append_kernel<kRequests>, grid, dim3(kThreads), 0, stream, p, b, tokens, rows);
}

}  // namespace

cudaError_t launch_append(const AppendParams& p, const Batch<AppendReq, kManyRequests>& batch, int num_sms, cudaStream_t stream) {
    return batch.n <= kFewRequests ? launch<kFewRequests>(p, batch, num_sms, stream) : launch<kManyRequests>(p, batch, num_sms, stream);
}

}  // namespace lookm

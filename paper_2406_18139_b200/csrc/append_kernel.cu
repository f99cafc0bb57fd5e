// New tokens on their way into a paged cache: per-head RMS norm of queries and keys, rotation to their positions,
// key and value rows written to the pages, the rows' mass set to zero.
//
//     y = x / sqrt(mean(x^2) + eps) * w        (a, b) -> (a cos - b sin, b cos + a sin)
//
// All in fp32 with one rounding to bf16 at the end.  The angle is position * frequency, taken in turns and in fp64 so
// that only its fraction is left before it becomes fp32: at position 2^20 an fp32 product would be off by 0.03 radians.
//
// Bound by HBM: every row is read once and written once.  Half a warp takes a row of 256 bytes, 16 bytes a lane; a
// CTA takes a few tokens and some of their heads, and its threads first work out these tokens' cosines and sines, which
// all heads share.
#include <algorithm>

#include <cuda_bf16.h>

#include "paged.h"
#include "ptx.cuh"

namespace lookm {
namespace {

constexpr int kThreads = 256, kHalfWarps = kThreads / 16;
constexpr int kTokens = 4;                       // of a CTA, at most

struct TokenPlace { int index, row; };           // request and cache row

__device__ __forceinline__ void unpack8(const uint4& raw, float (&x)[8]) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Features 8 * l .. 8 * l + 7 of a row, normed and rotated.  All 16 lanes of the half-warp come here together.
__device__ __forceinline__ uint4 norm_rotate(const uint4& raw, const uint4& weight, bool norm, const AppendParams& p, const float2* turn,
                                             int l) {
    float x[8];
    unpack8(raw, x);
    if (p.q_weight || p.k_weight) {              // (the same in both halves of the warp, which shuffle together)
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const float scale = rsqrtf(sum * (1.f / kHeadDim) + p.eps);
        float w[8];
        unpack8(weight, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = norm ? x[i] * scale * w[i] : x[i];
    }
    if (p.rotary_dim == 0) return norm ? pack8(x) : raw;
    float y[8];
    if (p.interleaved) {                         // pairs (2 i, 2 i + 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 t = turn[(l * 4 + i) & (kMaxFreqs - 1)];
            y[2 * i] = x[2 * i] * t.x - x[2 * i + 1] * t.y;
            y[2 * i + 1] = x[2 * i + 1] * t.x + x[2 * i] * t.y;
        }
    } else {                                     // pairs (i, i + rotary_dim / 2): rotary_dim / 16 lanes apart
        const int half = p.rotary_dim >> 4;
        const bool second = l >= half;
        const int other = (threadIdx.x & 16) | ((second ? l - half : l + half) & 15), f0 = (second ? l - half : l) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float z = __shfl_sync(0xffffffffu, x[i], other);
            const float2 t = turn[(f0 + i) & (kMaxFreqs - 1)];
            y[i] = second ? x[i] * t.x + z * t.y : x[i] * t.x - z * t.y;
        }
    }
    const bool turned = l * 8 < p.rotary_dim;
    if (!turned && !norm) return raw;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = turned ? y[i] : x[i];
    return pack8(x);
}

template <int kRequests>
__global__ void __launch_bounds__(kThreads)
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
    const int per_token = hq + 2 * hkv;
    const int l = threadIdx.x & 15, first = blockIdx.y * rows_per_cta, last = min(first + rows_per_cta, nt * per_token);
    uint4 wq = {0, 0, 0, 0}, wk = {0, 0, 0, 0};
    if (p.q_weight) wq = __ldg(static_cast<const uint4*>(p.q_weight) + l);
    if (p.k_weight) wk = __ldg(static_cast<const uint4*>(p.k_weight) + l);
    const char *q = static_cast<const char*>(p.q), *k = static_cast<const char*>(p.k), *v = static_cast<const char*>(p.v);
    // (both halves of a warp run the same number of rounds: they shuffle together)
    for (int i0 = first + (threadIdx.x >> 5) * 2; i0 < last; i0 += kHalfWarps) {
        const int i = i0 + ((threadIdx.x >> 4) & 1);
        const bool live = i < last;
        const int t = live ? i / per_token : 0, h = live ? i - t * per_token : 0;
        const bool is_q = h < hq, is_k = !is_q && h < hq + hkv;
        const int hh = is_q ? h : is_k ? h - hq : h - hq - hkv;
        const long long from = is_q ? (t0 + t) * p.q_stride_tok + hh * p.q_stride_head : (t0 + t) * p.kv_stride_tok + hh * p.kv_stride_head;
        uint4 raw = {0, 0, 0, 0};
        if (live) raw = *reinterpret_cast<const uint4*>((is_q ? q : is_k ? k : v) + 2 * from + l * 16);
        const TokenPlace at = place[t];
        char* to = nullptr;
        if (live && is_q) {
            to = static_cast<char*>(p.q_out) + 2 * ((t0 + t) * p.qo_stride_tok + hh * p.qo_stride_head);
        } else if (live) {
            const int page = p.pages.page_of(at.index, at.row, p.status);
            if (page >= 0) {
                to = static_cast<char*>(is_k ? p.cache_k : p.cache_v) + 2 * p.pages.row_at(page, at.row, hh);
                if (is_k && l == 0 && p.mass) p.mass[p.pages.mass_at(page, at.row, hh)] = 0.f;
            }
        }
        const uint4 y = norm_rotate(raw, is_q ? wq : wk, (is_q && p.q_weight) || (is_k && p.k_weight), p, turn[t], l);
        if (to) *reinterpret_cast<uint4*>(to + l * 16) = is_q || is_k ? y : raw;
    }
}

template <int kRequests>
cudaError_t launch(const AppendParams& p, const Batch<AppendReq, kManyRequests>& batch, int num_sms, cudaStream_t stream) {
    Batch<AppendReq, kRequests> b;
    b.n = batch.n;
    b.pad = 0;
    for (int i = 0; i < kRequests; ++i) b.r[i] = i < batch.n ? batch.r[i] : AppendReq{0, 0, 0, 0};
    const int total = p.tok_end - p.tok_begin, per_token = (p.q ? p.pages.n_q_heads : 0) + 2 * p.pages.n_kv_heads;
    const int tokens = total >= kTokens * num_sms * 4 ? kTokens : 1;
    const int groups = (total + tokens - 1) / tokens;
    // few tokens: their heads are spread over CTAs too, one row per half-warp
    int rows = tokens * per_token;
    if (groups < num_sms * 4) rows = std::max(kHalfWarps, (int)((long long)rows * groups / (num_sms * 4)));
    rows = (rows + kHalfWarps - 1) / kHalfWarps * kHalfWarps;
    const dim3 grid(groups, (tokens * per_token + rows - 1) / rows);
    return launch_chained(append_kernel<kRequests>, grid, dim3(kThreads), 0, stream, p, b, tokens, rows);
}

}  // namespace

cudaError_t launch_append(const AppendParams& p, const Batch<AppendReq, kManyRequests>& batch, int num_sms, cudaStream_t stream) {
    return batch.n <= kFewRequests ? launch<kFewRequests>(p, batch, num_sms, stream) : launch<kManyRequests>(p, batch, num_sms, stream);
}

}  // namespace lookm

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
// rotated, or whose partner is the next one).  A CTA takes a few tokens; its threads first work out these tokens' cosines and
// sines, which all heads share, then its warps take units of eight rows.
//   21100 tokens x 40 heads (1.3 GB) 226 us = 5.7 TB/s, 0.88 of the copy rate, in a long row of calls 241 us; x 32 heads on 8 106 us.  700 tokens x 32
// heads, inputs not in L2, 10.7 us; one token 3.3.  Earlier: a row per half-warp at a time, in order of heads, shuffles for the partners 370;
// four rows at a time, packed arithmetic 285.  Units of four rows 292, 3 CTAs per SM 245.
#include <algorithm>

#include <cuda_bf16.h>

#include "paged.h"
#include "ptx.cuh"

namespace lookm {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kTokens = 4;                       // of a CTA, at most
constexpr int kRows = 4, kUnitRows = 2 * kRows;  // of a half-warp at a time, of a warp

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
    ptx::f32x2 cos[4], sin[4], minus_sin[2];     // adjacent: per pair, sin as (-sin, sin); else of the two pairs of the first group
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
    if (r.turned) {
        if (r.adjacent) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 v = ptx::unpack2(e.x[i]);
                e.x[i] = ptx::fma2(e.x[i], r.cos[i], ptx::mul2(ptx::pack2(v.y, v.x), r.sin[i]));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const ptx::f32x2 a = e.x[i], b = e.x[i + 2];
                e.x[i] = ptx::fma2(a, r.cos[i], ptx::mul2(b, r.minus_sin[i]));
                e.x[i + 2] = ptx::fma2(b, r.cos[i], ptx::mul2(a, r.sin[i]));
            }
        }
    }
    __syncwarp();                                // (lanes that are not rotated have skipped that)
}

// A warp's unit of work: up to 2 * kRows rows of one kind (queries, keys or values) of one token, half a warp each and all asked for
// together.  `n` of them are there; src and dst are the lane's first group of four features in its half's first row.
// kSplit: a lane's second group of four features does not follow its first but lies `gap` bytes on.
template <bool kWork, bool kSplit>
__device__ __forceinline__ void unit_rows(const char* src, long long from_stride, char* dst, long long to_stride, int n, int gap, bool norm,
                                          const Eight& weight, float eps, const Rotation& r) {
    const int half = (threadIdx.x >> 4) & 1;
    uint2 a[kRows], b[kRows];
#pragma unroll
    for (int j = 0; j < kRows; ++j, src += from_stride) {
        a[j] = b[j] = make_uint2(0, 0);
        if (2 * j + half >= n) continue;
        if (kSplit) {
            a[j] = *reinterpret_cast<const uint2*>(src);
            b[j] = *reinterpret_cast<const uint2*>(src + gap);
        } else {
            const uint4 x = *reinterpret_cast<const uint4*>(src);
            a[j] = make_uint2(x.x, x.y);
            b[j] = make_uint2(x.z, x.w);
        }
    }
#pragma unroll
    for (int j = 0; j < kRows; ++j, dst += to_stride) {
        if (2 * j >= n) break;                   // (the same in both halves, which shuffle together)
        if (kWork) {
            Eight e = unpack8(a[j], b[j]);
            norm_rotate(e, norm, weight, eps, r);
            a[j] = make_uint2(pack_bf16(e.x[0]), pack_bf16(e.x[1]));
            b[j] = make_uint2(pack_bf16(e.x[2]), pack_bf16(e.x[3]));
        }
        if (2 * j + half >= n) continue;
        if (kSplit) {
            *reinterpret_cast<uint2*>(dst) = a[j];
            *reinterpret_cast<uint2*>(dst + gap) = b[j];
        } else {
            *reinterpret_cast<uint4*>(dst) = make_uint4(a[j].x, a[j].y, b[j].x, b[j].y);
        }
    }
}

template <int kRequests>
__global__ void __launch_bounds__(kThreads, 4)
append_kernel(const __grid_constant__ AppendParams p, const __grid_constant__ Batch<AppendReq, kRequests> batch, int tokens) {
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
    const int q_units = (hq + kUnitRows - 1) / kUnitRows, kv_units = (hkv + kUnitRows - 1) / kUnitRows, per_token = q_units + 2 * kv_units;
    const int l = threadIdx.x & 15, half = (threadIdx.x >> 4) & 1;
    Rotation r;
    r.turned = l * 8 < p.rotary_dim;
    r.adjacent = p.interleaved;
    // first group 4 l .. 4 l + 3, second group half a rotation further; else eight features in a row
    const bool split = r.turned && !p.interleaved;
    const int at = 2 * (split ? 4 * l : 8 * l), gap = split ? p.rotary_dim : 8;
    for (int u = blockIdx.y * kWarps + (threadIdx.x >> 5); u < nt * per_token; u += gridDim.y * kWarps) {
        const int t = u / per_token, k = u - t * per_token;
        const long long tok = t0 + t;
        const TokenPlace to = place[t];
        const bool is_q = k < q_units, is_k = !is_q && k < q_units + kv_units;
        const int first = (k - (is_q ? 0 : is_k ? q_units : q_units + kv_units)) * kUnitRows, n = min(kUnitRows, (is_q ? hq : hkv) - first);
        const long long from_stride = 2 * (is_q ? p.q_stride_head : p.kv_stride_head);
        const long long to_stride = 2 * (is_q ? p.qo_stride_head : p.pages.head_stride);
        const char* src = static_cast<const char*>(is_q ? p.q : is_k ? p.k : p.v) + 2 * tok * (is_q ? p.q_stride_tok : p.kv_stride_tok) +
                          (first + half) * from_stride;
        char* dst = static_cast<char*>(p.q_out) + 2 * tok * p.qo_stride_tok;
        if (!is_q) {
            const int page = p.pages.page_of(to.index, to.row, p.status);
            if (page < 0) continue;
            dst = static_cast<char*>(is_k ? p.cache_k : p.cache_v) + 2 * p.pages.row_at(page, to.row, 0);
            if (is_k && p.mass && (threadIdx.x & 31) < n) p.mass[p.pages.mass_at(page, to.row, first + (threadIdx.x & 31))] = 0.f;
        }
        dst += (first + half) * to_stride;
        const void* w = is_q ? p.q_weight : is_k ? p.k_weight : nullptr;
        Eight weight{};
        if (w) weight = unpack8(__ldg(reinterpret_cast<const uint2*>(static_cast<const char*>(w) + at)),
                                __ldg(reinterpret_cast<const uint2*>(static_cast<const char*>(w) + at + gap)));
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
                    r.minus_sin[i] = ptx::pack2(-angle[2 * i].y, -angle[2 * i + 1].y);
                }
            }
        }
        __syncwarp();
        if (!(is_q || is_k) || (!w && p.rotary_dim == 0))
            unit_rows<false, false>(src + 16 * l, 2 * from_stride, dst + 16 * l, 2 * to_stride, n, 8, false, weight, 0.f, r);
        else if (p.rotary_dim == 0 || p.interleaved)
            unit_rows<true, false>(src + at, 2 * from_stride, dst + at, 2 * to_stride, n, gap, w != nullptr, weight, p.eps, r);
        else
            unit_rows<true, true>(src + at, 2 * from_stride, dst + at, 2 * to_stride, n, gap, w != nullptr, weight, p.eps, r);
    }
}

template <int kRequests>
cudaError_t launch(const AppendParams& p, const Batch<AppendReq, kManyRequests>& batch, int num_sms, cudaStream_t stream) {
    Batch<AppendReq, kRequests> b;
    b.n = batch.n;
    b.pad = 0;
    for (int i = 0; i < kRequests; ++i) b.r[i] = i < batch.n ? batch.r[i] : AppendReq{0, 0, 0, 0};
    const int total = p.tok_end - p.tok_begin, hq = p.q ? p.pages.n_q_heads : 0;
    const int units = (hq + kUnitRows - 1) / kUnitRows + 2 * ((p.pages.n_kv_heads + kUnitRows - 1) / kUnitRows);
    const int tokens = total >= kTokens * num_sms * 8 ? kTokens : 1, groups = (total + tokens - 1) / tokens;
    // few tokens: a token's units are spread over CTAs, down to one per warp
    const int parts = std::max(1, std::min((units + kWarps - 1) / kWarps, num_sms * 4 / groups));
    return launch_chained(append_kernel<kRequests>, dim3(groups, parts), dim3(kThreads), 0, stream, p, b, tokens);
}

}  // namespace

cudaError_t launch_append(const AppendParams& p, const Batch<AppendReq, kManyRequests>& batch, int num_sms, cudaStream_t stream) {
    return batch.n <= kFewRequests ? launch<kFewRequests>(p, batch, num_sms, stream) : launch<kManyRequests>(p, batch, num_sms, stream);
}

}  // namespace lookm

// What the kernels for the new tokens of a step share: which keys a row sees, scores, values that are not finite, the merge of partials.
#pragma once

#include "decode_device.h"

namespace chess {

typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr float kLog2e = 1.44269504088896340736f;

// To nearest even.
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi)
{
    typedef __attribute__((ext_vector_type(2))) __bf16 pair;
    const pair p = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, p);
}

__device__ __forceinline__ int lanes_max(int v)
{
#pragma unroll
    for (int by = 32; by > 0; by /= 2) v = max(v, __shfl_xor(v, by));
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int lanes_min(int v)
{
#pragma unroll
    for (int by = 32; by > 0; by /= 2) v = min(v, __shfl_xor(v, by));
    return __builtin_amdgcn_readfirstlane(v);
}

// A sequence of the step: its length, pages, and new tokens (none where token_start names rows that are not there).
struct Span { int len, pages, start, n_new; };

__device__ __forceinline__ Span span_of(const AttendArgs& a, int b, int page_size)
{
    Span s;
    s.start = __builtin_amdgcn_readfirstlane(a.token_start[b]);
    s.n_new = __builtin_amdgcn_readfirstlane((int)((unsigned)a.token_start[b + 1] - (unsigned)a.token_start[b]));
    s.len = min(max(__builtin_amdgcn_readfirstlane(a.seq_lens[b]), 0), a.max_pages * page_size);
    s.pages = (s.len + page_size - 1) / page_size;
    if (s.n_new < 0 || s.start < 0 || s.start > a.n_rows - s.n_new) s.n_new = 0;
    s.n_new = min(s.n_new, a.max_new);
    return s;
}

// Query row r of a sequence and KV head: head r % G of its new token r / G.  A row that is not there is the last one again, and sees nothing.
struct RowView {
    int64_t at;              // row of q and out
    int p, lo, hi;           // its position, and the keys it sees
    float slope;             // in powers of two a position
    bool there;
};

__device__ __forceinline__ RowView view_of(const AttendArgs& a, const Span& s, int b, int h, int r)
{
    RowView v;
    const int G = a.group, last = s.n_new * G - 1;
    v.there = r <= last;
    r = min(r, last);
    const int i = (int)((unsigned)r / (unsigned)G), g = r - i * G;
    v.at = (int64_t)(s.start + i) * (a.n_kv_heads * G) + h * G + g;
    v.p = s.len - s.n_new + i;
    v.slope = a.slopes != nullptr ? a.slopes[h * G + g] * kLog2e : 0.f;
    v.lo = a.first_keys != nullptr ? max(a.first_keys[s.start + i], 0) : 0;
    if (a.window > 0) v.lo = max(v.lo, v.p - a.window + 1);
    v.hi = a.prefix_lens != nullptr ? max(v.p, a.prefix_lens[b] - 1) : v.p;
    v.hi = min(v.hi, s.len - 1);
    if (!v.there || v.p < 0) {
        v.lo = INT32_MAX;
        v.hi = -1;
    }
    return v;
}

// tanh to a few units in the last place: the odd series near 0, where 1 - 2 / (e^2x + 1) would lose what x has.
__device__ __forceinline__ float tanh_of(float x)
{
    const float x2 = x * x;
    const float near = x * fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 0x1.664f48p-6f, -0x1.ba1ba2p-5f), 0x1.111112p-3f), -0x1.555556p-2f), 1.f);
    const float e = __builtin_amdgcn_exp2f(fabsf(x) * (2.f * kLog2e));
    const float far = copysignf(1.f - 2.f * __builtin_amdgcn_rcpf(e + 1.f), x);
    return fabsf(x) < 0.3f ? near : far;
}

// A product of query and key as a power of two.
template <bool kCap>
__device__ __forceinline__ float score_of(const AttendArgs& a, float qk)
{
    if constexpr (kCap) return a.cap_out * tanh_of(qk * a.cap_in);
    return qk * a.scale_log2;
}

// Whether one of the wave's values is infinite or NaN: the largest of their magnitudes as bits, two at a time.
__device__ __forceinline__ bool not_finite(const uint4 (&v)[4][2])
{
    typedef __attribute__((ext_vector_type(2))) unsigned short pair;
    pair most = {0, 0};
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint32_t w[4] = {v[d][s].x, v[d][s].y, v[d][s].z, v[d][s].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(pair, w[i] & 0x7fff7fffu));
        }
    return __any(most.x >= 0x7f80 || most.y >= 0x7f80);
}

// Eight values: 1 (bf16) where one is +infinity (down: -infinity) or NaN, 0 elsewhere.
__device__ __forceinline__ uint4 not_finite_of(const uint4& v, bool down)
{
    const auto of = [&](uint32_t w) {
        uint32_t r = 0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t x = (w >> (16 * j)) & 0xffffu;
            if ((x & 0x7fffu) > 0x7f80u || x == (down ? 0xff80u : 0x7f80u)) r |= 0x3f80u << (16 * j);
        }
        return r;
    };
    return make_uint4(of(v.x), of(v.y), of(v.z), of(v.w));
}

// Eight values, 0 where one is not finite.
__device__ __forceinline__ uint4 finite_of(const uint4& v)
{
    const auto of = [&](uint32_t w) { return w & (((w & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u)); };
    return make_uint4(of(v.x), of(v.y), of(v.z), of(v.w));
}

// What the last split of a block of kRowsOf rows to arrive does: out = sum_s acc_s 2^(m_s - M) / sum_s l_s 2^(m_s - M), always in split order.
// A thread has four dims of a row; eight splits are asked for at a time.
template <int kRowsOf, int kThreads>
__device__ __forceinline__ void merge_parts(const AttendArgs& a, const Span& span, int h, int row0, int n_rows, int64_t part0, int n_splits)
{
    constexpr int kChunk = 8;
    const int G = a.group;
    for (int i = threadIdx.x; i < kRowsOf * 32; i += kThreads) {
        const int r = i >> 5, dim = 4 * (i & 31);
        if (row0 + r >= n_rows) break;
        float M = kNegBig, l = 0.f, x[4] = {};
        for (int s0 = 0; s0 < n_splits; s0 += kChunk) {
            uint64_t ml[kChunk], v[kChunk][2];
#pragma unroll
            for (int s = 0; s < kChunk; ++s) {
                const int64_t part = (part0 + min(s0 + s, n_splits - 1)) * kRowsOf + r;
                ml[s] = observe_u64(reinterpret_cast<const uint64_t*>(a.part_ml) + part);
                const uint64_t* at = reinterpret_cast<const uint64_t*>(a.part_acc + part * kHeadDim + dim);
                v[s][0] = observe_u64(at);
                v[s][1] = observe_u64(at + 1);
            }
            float top = M;
#pragma unroll
            for (int s = 0; s < kChunk; ++s) top = fmaxf(top, __builtin_bit_cast(float2, ml[s]).x);   // (the last one again changes nothing)
            const float keep = __builtin_amdgcn_exp2f(M - top);
            M = top;
            l *= keep;
#pragma unroll
            for (int d = 0; d < 4; ++d) x[d] *= keep;
#pragma unroll
            for (int s = 0; s < kChunk; ++s)
                if (s0 + s < n_splits) {
                    const float2 one = __builtin_bit_cast(float2, ml[s]), lo = __builtin_bit_cast(float2, v[s][0]), hi = __builtin_bit_cast(float2, v[s][1]);
                    const float by = __builtin_amdgcn_exp2f(one.x - M);
                    l += one.y * by;
                    x[0] += lo.x * by; x[1] += lo.y * by; x[2] += hi.x * by; x[3] += hi.y * by;
                }
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int rr = row0 + r, token = (int)((unsigned)rr / (unsigned)G), g = rr - token * G;
        const int64_t at = (int64_t)(span.start + token) * (a.n_kv_heads * G) + h * G + g;
        *reinterpret_cast<uint2*>(a.out + at * kHeadDim + dim) = make_uint2(two_bf16(x[0] * inv, x[1] * inv), two_bf16(x[2] * inv, x[3] * inv));
    }
}

}  // namespace chess

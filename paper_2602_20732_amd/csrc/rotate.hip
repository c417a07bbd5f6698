// Queries and keys of new tokens: each head normed by itself, turned by the token's position, and put where attention reads them.
//
//   y = x / sqrt(mean x^2 + eps) * w                               x: one head of one token, 128 bf16
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t) * scale       over pairs (a, b) of y's dims, t = position[axis of the pair] * frequency
//
// in fp32 from the projection's bf16 to the one rounding of the result.  A position times a frequency has up to 55 bits, and the angle matters to
// a 2^-9th of a turn at the least: the product and its reduction to a fraction of a turn are in fp64, sine and cosine are the hardware's,
// which take turns.
// A head is 16 lanes of 8 dims, so a load of 16 bytes a lane is four heads; a pair's other half is a lane away (or in the lane, where pairs
// lie side by side).  A workgroup has an entry of the write list (the new tokens of one page) and a run of heads; a wave takes a token
// at a time, works out its angles once and turns all heads of the run with them.  Values go into their pages (token-minor) as in quant_store.hip: a
// lane reads the same dims of 16 tokens, and has whole 32-byte rows to write.
// Bound: HBM, read and written alike; for single tokens the chain entry -> position -> angle -> store.
#include "attend_device.h"
#include "split_rule.h"

namespace chess {

constexpr int kRotateThreads = 256;

__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// Sum over the 16 lanes of a head, in every one of them.
__device__ __forceinline__ float head_sum(float v)
{
#define CHESS_ADD(ctrl) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, 0xf, 0xf, false));
    CHESS_ADD(0x128) CHESS_ADD(0x124) CHESS_ADD(0x122) CHESS_ADD(0x121)
#undef CHESS_ADD
    return v;
}

// The turn of a lane's eight dims: cosines, and sines with the sign that the pair's other half gets.
struct Turn {
    float c[8], s[8];
};

template <bool kBeside>
__device__ __forceinline__ Turn turn_of(const RotateArgs& a, int row, int ln)
{
    Turn t;
    const int half = a.pairs >> 3;                    // lanes of half a turned head
    const bool second = !kBeside && ln >= half;
    constexpr int kN = kBeside ? 4 : 8;
    // (lanes that are not turned work out the last one's angles and drop them)
    const int f0 = kBeside ? min(ln * 4, a.pairs - 4) : min(second ? ln - half : ln, half - 1) * 8;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        const int f = f0 + i, axis = (int)((f < 32 ? a.axis_lo : a.axis_hi) >> (2 * (f & 31))) & 3;
        const double revs = (double)a.positions[(int64_t)axis * a.position_stride + row] * (double)a.inv_freq[f] * 0.15915494309189533577;
        const float part = (float)(revs - __builtin_rint(revs));
        const float c = __builtin_amdgcn_cosf(part) * a.scale, s = __builtin_amdgcn_sinf(part) * a.scale;
        if constexpr (kBeside) {
            t.c[2 * i] = t.c[2 * i + 1] = c;
            t.s[2 * i] = -s;
            t.s[2 * i + 1] = s;
        } else {
            t.c[i] = c;
            t.s[i] = second ? s : -s;
        }
    }
    return t;
}

__device__ __forceinline__ void eight(float (&x)[8], const uint4& r)
{
    x[0] = low_half(r.x); x[1] = high_half(r.x); x[2] = low_half(r.y); x[3] = high_half(r.y);
    x[4] = low_half(r.z); x[5] = high_half(r.z); x[6] = low_half(r.w); x[7] = high_half(r.w);
}

// Up to kQuads times four heads of one token, from head `head0` on.
template <bool kBeside, int kQuads>
__device__ __forceinline__ void turn_heads(const RotateArgs& a, const uint16_t* src, uint16_t* dst, int64_t dst_head, int head0, int heads,
                                           const float* norm, const Turn& t, int lane)
{
    const int ln = lane & 15, half = a.pairs >> 3;
    const bool turned = kBeside ? ln * 4 < a.pairs : ln < 2 * half;
    const int other = kBeside ? ln : (ln < half ? ln + half : ln < 2 * half ? ln - half : ln);
    uint4 r[kQuads];
#pragma unroll
    for (int i = 0; i < kQuads; ++i)                  // (heads behind the last repeat it)
        r[i] = *(reinterpret_cast<const uint4*>(src + (int64_t)min(head0 + 4 * i + (lane >> 4), heads - 1) * kHeadDim) + ln);
    float w[8], w_other[8];
#pragma unroll
    for (int i = 0; i < kQuads; ++i) {
        const int h = head0 + 4 * i + (lane >> 4);
        if (head0 + 4 * i >= heads) break;
        float x[8], y[8];
        eight(x, r[i]);
        uint4 ro;
        if constexpr (!kBeside) {
            const int from = (lane & 48) | other;
            ro = make_uint4(__shfl(r[i].x, from), __shfl(r[i].y, from), __shfl(r[i].z, from), __shfl(r[i].w, from));
            eight(y, ro);
        }
        if (norm != nullptr) {
            if (i == 0 || a.norm_stride != 0) {
                const float* at = norm + (int64_t)min(h, heads - 1) * a.norm_stride;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    w[e] = at[ln * 8 + e];
                    if (!kBeside) w_other[e] = at[other * 8 + e];
                }
            }
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
            const float by = rsqrtf(head_sum(sum) * (1.f / kHeadDim) + a.eps);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] *= by * w[e];
                if (!kBeside) y[e] *= by * w_other[e];
            }
        }
        if constexpr (kBeside) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = x[e ^ 1];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = turned ? x[e] * t.c[e] + y[e] * t.s[e] : x[e];
        if (h < heads)
            *(reinterpret_cast<uint4*>(dst + h * dst_head) + ln) =
                make_uint4(two_bf16(x[0], x[1]), two_bf16(x[2], x[3]), two_bf16(x[4], x[5]), two_bf16(x[6], x[7]));
    }
}

// The new values of one page and head: [token][dim] -> [dim][token].
template <int B>
__device__ __forceinline__ void put_values(const RotateArgs& a, int64_t page_head, int h, int row0, int first, int count, int lane)
{
    constexpr int kWords = B / 16, kLanes = 64 / kWords;           // two dims a word
    const int ln = lane % kLanes, t0 = 16 * (lane / kLanes);
    const uint32_t* src = reinterpret_cast<const uint32_t*>(a.v + (int64_t)row0 * a.v_stride + h * kHeadDim) + ln * kWords;
    uint16_t* rows = a.v_pool + page_head * (B * kHeadDim) + (int64_t)ln * (2 * kWords) * B + t0;
    if (count < B) {                                  // what is not new stays as it is
        for (int t = max(t0, first); t < min(t0 + 16, first + count); ++t)
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
                const uint32_t v = src[(int64_t)(t - first) * (a.v_stride >> 1) + w];
                rows[(2 * w) * B + t - t0] = (uint16_t)v;
                rows[(2 * w + 1) * B + t - t0] = (uint16_t)(v >> 16);
            }
        return;
    }
    uint32_t r[16][kWords];
#pragma unroll
    for (int t = 0; t < 16; ++t)
#pragma unroll
        for (int w = 0; w < kWords; ++w) r[t][w] = src[(int64_t)(t0 + t) * (a.v_stride >> 1) + w];
#pragma unroll
    for (int w = 0; w < kWords; ++w)
#pragma unroll
        for (int odd = 0; odd < 2; ++odd) {
            uint32_t o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                o[i] = odd ? (r[2 * i][w] >> 16) | (r[2 * i + 1][w] & 0xffff0000u) : (r[2 * i][w] & 0xffffu) | (r[2 * i + 1][w] << 16);
            uint4* at = reinterpret_cast<uint4*>(rows + (2 * w + odd) * B);
            at[0] = make_uint4(o[0], o[1], o[2], o[3]);
            at[1] = make_uint4(o[4], o[5], o[6], o[7]);
        }
}

// Workgroup (part, entry): part = a run of query heads, then of key heads, then four value heads.  kPaged: entries of the write list; otherwise B
// rows each, keys to k_out.
template <int B, bool kPaged, bool kBeside, int kQuads>
__global__ __launch_bounds__(kRotateThreads) void rotate_kernel(RotateArgs a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int unit = blockIdx.x / (unsigned)a.parts, part = blockIdx.x - unit * a.parts;
    int phys = 0, row0, first = 0, count;
    if constexpr (kPaged) {
        if (unit >= min(a.counts[1], a.max_writes)) return;
        const int4 entry = a.writes[unit];
        phys = __builtin_amdgcn_readfirstlane(entry.x);
        row0 = __builtin_amdgcn_readfirstlane(entry.y);
        first = min(max(__builtin_amdgcn_readfirstlane(entry.z), 0), B - 1);
        count = min(__builtin_amdgcn_readfirstlane(entry.w), B - first);
        // rows or a page that are not there: nothing is stored
        if (count < 1 || row0 < 0 || row0 > a.n_rows - count || phys < 0 || phys >= a.n_pages) return;
    } else {
        row0 = unit * B;
        const int n = a.counts != nullptr ? min(a.counts[0], a.n_rows) : a.n_rows;
        count = min(B, n - row0);
        if (count < 1) return;
    }
    const int q_parts = a.q_parts, k_parts = a.k_parts;
    if (part >= q_parts + k_parts) {
        if constexpr (kPaged) {
            const int h = (part - q_parts - k_parts) * 4 + wave;
            if (h < a.kv_heads) put_values<B>(a, (int64_t)phys * a.kv_heads + h, h, row0, first, count, lane);
        }
        return;
    }
    const bool is_q = part < q_parts;
    const int heads = is_q ? a.q_heads : a.kv_heads, head0 = (is_q ? part : part - q_parts) * (4 * kQuads);
    for (int j = wave; j < count; j += kRotateThreads / 64) {
        const int row = row0 + j;
        const Turn t = turn_of<kBeside>(a, row, lane & 15);
        if (is_q)
            turn_heads<kBeside, kQuads>(a, a.q + row * a.q_stride, a.q_out + (int64_t)row * heads * kHeadDim, kHeadDim, head0, heads, a.q_norm, t, lane);
        else if (kPaged)
            turn_heads<kBeside, kQuads>(a, a.k + row * a.k_stride, a.k_out + ((int64_t)phys * heads * B + first + j) * kHeadDim, B * kHeadDim, head0, heads,
                                        a.k_norm, t, lane);
        else
            turn_heads<kBeside, kQuads>(a, a.k + row * a.k_stride, a.k_out + (int64_t)row * heads * kHeadDim, kHeadDim, head0, heads, a.k_norm, t, lane);
    }
}

template <int B, bool kPaged, int kQuads>
static hipError_t launch_of(const RotateArgs& a, int64_t units, bool beside, hipStream_t stream)
{
    const dim3 grid((unsigned)(units * a.parts));
    return beside ? launch(rotate_kernel<B, kPaged, true, kQuads>, grid, dim3(kRotateThreads), 0, stream, a)
                  : launch(rotate_kernel<B, kPaged, false, kQuads>, grid, dim3(kRotateThreads), 0, stream, a);
}

RotateShape rotate_shape(const chess_ctx* ctx, const RotateArgs& a, bool paged)
{
    RotateShape s;
    s.units = paged ? a.max_writes : cdiv(a.n_rows, 16);
    // a wave turns all heads that there are (up to 32) with the angles of a token, unless that leaves compute units idle
    s.quads = s.units >= 2 * (int64_t)ctx->n_cu ? 8 : 1;
    s.q_parts = a.q != nullptr ? (int)cdiv(a.q_heads, 4 * s.quads) : 0;
    s.k_parts = a.k != nullptr ? (int)cdiv(a.kv_heads, 4 * s.quads) : 0;
    s.parts = s.q_parts + s.k_parts + (paged ? (int)cdiv(a.kv_heads, 4) : 0);
    return s;
}

hipError_t launch_rotate(chess_ctx* ctx, RotateArgs a, bool paged, bool beside, hipStream_t stream)
{
    const RotateShape s = rotate_shape(ctx, a, paged);
    a.q_parts = s.q_parts; a.k_parts = s.k_parts; a.parts = s.parts;
    const bool many = s.quads == 8;
    if (!paged) return many ? launch_of<16, false, 8>(a, s.units, beside, stream) : launch_of<16, false, 1>(a, s.units, beside, stream);
    if (ctx->geom.page_size == 16) return many ? launch_of<16, true, 8>(a, s.units, beside, stream) : launch_of<16, true, 1>(a, s.units, beside, stream);
    return many ? launch_of<32, true, 8>(a, s.units, beside, stream) : launch_of<32, true, 1>(a, s.units, beside, stream);
}

}  // namespace chess

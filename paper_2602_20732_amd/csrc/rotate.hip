// Queries and keys of new tokens: each head normed by itself, turned by the token's position, and put where attention reads them.
//
//   y = x / sqrt(mean x^2 + eps) * w                               x: one head of one token, 128 bf16
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t) * scale       over pairs (a, b) of y's dims, t = position[axis of the pair] * frequency
//
// in fp32 from the projection's bf16 to the one rounding of the result.  A position times a frequency has up to 55 bits, and what matters is its
// fraction of a turn: product and fraction are in fp64, sine and cosine the hardware's, which take turns (2^-22.9 off at most, of 4 million measured).
// Weights are multiplied into a token's sines and cosines once, so that a head costs three products a dim: (a cw + b sw) / sqrt(..).
// A head is 16 lanes of 8 dims, so a load of 16 bytes a lane is four heads; a pair's other half is a lane away (or in the lane, where pairs
// lie side by side).  A workgroup has an entry of the write list (the new tokens of one page), a wave takes a token at a time, works out its
// angles once and turns all its heads with them; where there are few tokens, workgroups share their heads.  Values go into their pages (token-minor) as in
// quant_store.hip: a lane reads the same dims of 16 tokens, and has whole 32-byte rows to write.
// Bound: HBM, read and written alike; for single tokens the chain entry -> position -> angle -> store.  Measured: 65531 tokens of 28 + 2 x 4 heads into pages of
// 32 233 us, 24955 of 32 + 2 x 8 into pages of 16 121 us: 5.1 to 5.2 TB/s (a library copy of 0.3 to 2 GB 4.9 to 5.2); 32 sequences of 5 drafts 5.6 us, one token 3.5.
// Alone, without values: 65531 tokens of 28 + 4 heads 207 us (5.2 TB/s), 24955 of 32 + 8 110 (4.7), 160 6.0, one 3.0; weights a head, read anew for every token, 269
// and 144.
#include "attend_device.h"
#include "quant_device.h"
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

// What a lane's pairs turn by: fractions of a turn a position, and which row of the positions (two bits a pair).
template <bool kBeside>
struct Pairs {
    static constexpr int kN = kBeside ? 4 : 8;        // of a lane
    double turns[kN];
    uint32_t axes;
    bool turned, second;                              // whether the lane's dims turn; whether they are the pairs' second halves
    int other;                                        // the lane that has the other halves
    __device__ __forceinline__ Pairs(const RotateArgs& a, int ln)
    {
        const int half = a.pairs >> 3;                // lanes of half a turned head
        turned = kBeside ? ln * 4 < a.pairs : ln < 2 * half;
        second = !kBeside && ln >= half;
        other = kBeside || !turned ? ln : second ? ln - half : ln + half;
        // (lanes that do not turn work out the last ones' angles and drop them)
        const int f0 = kBeside ? min(ln * 4, a.pairs - 4) : min(second ? ln - half : ln, half - 1) * 8;
        axes = (uint32_t)((f0 < 32 ? a.axis_lo : a.axis_hi) >> (2 * (f0 & 31)));
#pragma unroll
        for (int i = 0; i < kN; ++i) turns[i] = (double)a.inv_freq[f0 + i] * 0.15915494309189533577;
    }
};

// A token's turn, with the weights of a kind of heads: y = x cw + (the pair's other half) sw.
struct Turn { float cw[8], sw[8]; };

// (cosine, sine) of each pair of the lane, times the scale.
template <bool kBeside>
__device__ __forceinline__ void angles_of(const RotateArgs& a, const Pairs<kBeside>& p, int row, float (&c)[Pairs<kBeside>::kN], float (&s)[Pairs<kBeside>::kN])
{
    int at[4];
    at[0] = load_same(a.positions, row);
    if (a.n_axes > 1)
#pragma unroll
        for (int y = 1; y < 4; ++y) at[y] = load_same(a.positions, (int64_t)min(y, a.n_axes - 1) * a.position_stride + row);
#pragma unroll
    for (int i = 0; i < Pairs<kBeside>::kN; ++i) {
        int x = at[0];
        if (a.n_axes > 1) {
            const uint32_t axis = p.axes >> (2 * i) & 3u;
            x = axis == 1 ? at[1] : axis == 2 ? at[2] : axis == 3 ? at[3] : x;
        }
        const float part = (float)__builtin_amdgcn_fract((double)x * p.turns[i]);
        c[i] = __builtin_amdgcn_cosf(part) * a.scale;
        s[i] = __builtin_amdgcn_sinf(part) * a.scale;
    }
}

// The weights of a lane's dims, and of those that their pairs' other halves are.
struct Weights { float own[8], other[8]; };

__device__ __forceinline__ void eight_at(float (&x)[8], const float* p)
{
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}

// norm: 128 weights, 16-byte aligned; not normed: all 1.
template <bool kBeside>
__device__ __forceinline__ Weights weights_of(const Pairs<kBeside>& p, bool normed, const float* norm, int ln)
{
    Weights w;
#pragma unroll
    for (int e = 0; e < 8; ++e) w.own[e] = w.other[e] = 1.f;
    if (normed) {
        eight_at(w.own, norm + ln * 8);
        if constexpr (!kBeside) eight_at(w.other, norm + p.other * 8);
    }
    if constexpr (kBeside)
#pragma unroll
        for (int e = 0; e < 8; ++e) w.other[e] = w.own[e ^ 1];
    return w;
}

template <bool kBeside>
__device__ __forceinline__ void weigh(Turn& t, const Pairs<kBeside>& p, const Weights& w, const float (&c)[Pairs<kBeside>::kN], const float (&s)[Pairs<kBeside>::kN])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int i = kBeside ? e / 2 : e;
        const bool plus = kBeside ? e & 1 : p.second;
        t.cw[e] = p.turned ? c[i] * w.own[e] : w.own[e];
        t.sw[e] = p.turned ? (plus ? s[i] : -s[i]) * w.other[e] : 0.f;
    }
}

__device__ __forceinline__ void eight(float (&x)[8], const uint4& r)
{
    x[0] = low_half(r.x); x[1] = high_half(r.x); x[2] = low_half(r.y); x[3] = high_half(r.y);
    x[4] = low_half(r.z); x[5] = high_half(r.z); x[6] = low_half(r.w); x[7] = high_half(r.w);
}

// Four heads, one every 16 lanes.
template <bool kBeside>
__device__ __forceinline__ uint4 turned_heads(const Pairs<kBeside>& p, const Turn& t, const uint4& r, bool norm, float eps, int lane)
{
    float x[8], y[8];
    eight(x, r);
    if constexpr (kBeside) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = p.turned ? x[e ^ 1] : 0.f;
    } else {
        const int from = (lane & 48) | p.other;
        const uint32_t keep = p.turned ? 0xffffffffu : 0u;       // (a dim that does not turn has no other: not even one that is not finite)
        eight(y, make_uint4(__shfl(r.x, from) & keep, __shfl(r.y, from) & keep, __shfl(r.z, from) & keep, __shfl(r.w, from) & keep));
    }
    float by = 1.f;
    if (norm) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
        by = rsqrtf(head_sum(sum) * (1.f / kHeadDim) + eps);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = fmaf(y[e], t.sw[e], x[e] * t.cw[e]) * by;
    return make_uint4(two_bf16(x[0], x[1]), two_bf16(x[2], x[3]), two_bf16(x[4], x[5]), two_bf16(x[6], x[7]));
}

// The new values of one page and head: [token][dim] -> [dim][token].
template <int B>
__device__ __forceinline__ void put_values(const RotateArgs& a, int64_t page_head, int h, int row0, int first, int count, int lane)
{
    constexpr int kWords = B / 16, kLanes = 64 / kWords;           // two dims a word
    const int ln = lane % kLanes, t0 = 16 * (lane / kLanes);
    const uint32_t* src = reinterpret_cast<const uint32_t*>(a.v + (int64_t)row0 * a.v_stride + h * kHeadDim) + ln * kWords;
    uint16_t* rows = a.v_pool + page_head * (B * kHeadDim) + (int64_t)ln * (2 * kWords) * B + t0;
    uint32_t r[16][kWords];
#pragma unroll
    for (int t = 0; t < 16; ++t)                      // (tokens that are not new repeat one that is)
#pragma unroll
        for (int w = 0; w < kWords; ++w) r[t][w] = __builtin_nontemporal_load((const __attribute__((address_space(1))) uint32_t*)src + (int64_t)min(max(t0 + t - first, 0), count - 1) * (a.v_stride >> 1) + w);
    uint32_t is_new[8];                               // halves of a row's eight words
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int t = t0 + 2 * i - first;
        is_new[i] = ((unsigned)t < (unsigned)count ? 0xffffu : 0u) | ((unsigned)(t + 1) < (unsigned)count ? 0xffff0000u : 0u);
    }
#pragma unroll
    for (int w = 0; w < kWords; ++w)
#pragma unroll
        for (int odd = 0; odd < 2; ++odd) {
            uint4* at = reinterpret_cast<uint4*>(rows + (2 * w + odd) * B);
            uint32_t o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                o[i] = odd ? (r[2 * i][w] >> 16) | (r[2 * i + 1][w] & 0xffff0000u) : (r[2 * i][w] & 0xffffu) | (r[2 * i + 1][w] << 16);
            if (count < B) {                          // what is not new stays as it is
                const uint4 was[2] = {at[0], at[1]};
                const uint32_t old[8] = {was[0].x, was[0].y, was[0].z, was[0].w, was[1].x, was[1].y, was[1].z, was[1].w};
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = (o[i] & is_new[i]) | (old[i] & ~is_new[i]);
            }
            at[0] = make_uint4(o[0], o[1], o[2], o[3]);
            at[1] = make_uint4(o[4], o[5], o[6], o[7]);
        }
}

// Workgroup (part, entry): the dies take workgroups in turn, and parts of unlike size side by side would be some dies' and not others' (keys and queries on
// even ones, values on odd ones: 65531 tokens in pages of 32 290 us instead of 260).  kPaged: entries of the write list, parts of four value heads behind those of queries and keys; otherwise B rows each, keys to
// k_out.  A part has every heads_parts-th run of 4 kQuads heads, queries' and then keys'.
template <int B, bool kPaged, bool kBeside, int kQuads>
__global__ __launch_bounds__(kRotateThreads) void rotate_kernel(RotateArgs a)
{
    ArgLines<0, sizeof(RotateArgs)> lines;
    lines.ask();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int part = blockIdx.x / (unsigned)a.units, unit = blockIdx.x - part * a.units;
    int phys = 0, row0, first = 0, count;
    if constexpr (kPaged) {
        const int4 entry = a.writes[unit];            // (there is room for as many as there are units: asked for with their number)
        if (unit >= a.counts[1]) return;
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
    lines.hold();
    if (part >= a.head_parts) {
        if constexpr (kPaged) {
            const int h = (part - a.head_parts) * 4 + wave;
            if (h < a.kv_heads) put_values<B>(a, (int64_t)phys * a.kv_heads + h, h, row0, first, count, lane);
        }
        return;
    }
    const int ln = lane & 15, runs = a.q_runs + a.k_runs;
    const Pairs<kBeside> pairs(a, ln);
    // weights that all heads share: a workgroup of one run has one kind's, in registers; one of all runs reads both kinds' again for every token
    Weights w;
    __shared__ __align__(16) float shared_norm[2][kHeadDim];
    if constexpr (kQuads > 1) {
        const float* norm = threadIdx.x < kHeadDim ? a.q_norm : a.k_norm;
        if (a.norm_stride == 0 && norm != nullptr) shared_norm[threadIdx.x / kHeadDim][threadIdx.x % kHeadDim] = norm[threadIdx.x % kHeadDim];
        __syncthreads();
    } else if (a.norm_stride == 0) {
        const float* norm = part < a.q_runs ? a.q_norm : a.k_norm;
        w = weights_of<kBeside>(pairs, norm != nullptr, norm, ln);
    }
    // (heads behind the last repeat it)
    const auto heads_of = [&](int j, int run, uint4 (&r)[kQuads]) {
        const bool is_q = run < a.q_runs;
        const int heads = is_q ? a.q_heads : a.kv_heads, head0 = (is_q ? run : run - a.q_runs) * (4 * kQuads) + (lane >> 4);
        const uint16_t* src = is_q ? a.q + (row0 + j) * a.q_stride : a.k + (row0 + j) * a.k_stride;
#pragma unroll
        for (int i = 0; i < kQuads; ++i) r[i] = load_16<true>(reinterpret_cast<const uint8_t*>(src + (int64_t)min(head0 + 4 * i, heads - 1) * kHeadDim + ln * 8));
    };
    // the next run's heads are asked for ahead of this one's work
    uint4 r[kQuads], r_next[kQuads];
    float c[Pairs<kBeside>::kN], s[Pairs<kBeside>::kN];
    Turn t;
    int j = wave, run = part, token = -1, kind = -1;
    if (j < count) heads_of(j, run, r);
    while (j < count) {
        const bool wraps = run + a.head_parts >= runs;
        const int j_next = wraps ? j + kRotateThreads / 64 : j, run_next = wraps ? part : run + a.head_parts;
        if (j_next < count) heads_of(j_next, run_next, r_next);
        const bool is_q = run < a.q_runs;
        const float* norm = is_q ? a.q_norm : a.k_norm;
        if (token != j) angles_of<kBeside>(a, pairs, row0 + j, c, s);
        if (a.norm_stride == 0 && (token != j || kind != (int)is_q)) {
            if constexpr (kQuads > 1) weigh<kBeside>(t, pairs, weights_of<kBeside>(pairs, norm != nullptr, shared_norm[is_q ? 0 : 1], ln), c, s);
            else weigh<kBeside>(t, pairs, w, c, s);
        }
        token = j;
        kind = is_q;
        const int heads = is_q ? a.q_heads : a.kv_heads, head0 = (is_q ? run : run - a.q_runs) * (4 * kQuads);
        uint16_t* dst = is_q ? a.q_out + (int64_t)(row0 + j) * heads * kHeadDim
                             : a.k_out + (kPaged ? ((int64_t)phys * heads * B + first + j) * kHeadDim : (int64_t)(row0 + j) * heads * kHeadDim);
        const int64_t dst_head = is_q || !kPaged ? kHeadDim : B * kHeadDim;
#pragma unroll
        for (int i = 0; i < kQuads; ++i) {
            const int h = head0 + 4 * i + (lane >> 4);
            if (head0 + 4 * i >= heads) break;
            if (a.norm_stride != 0) {
                const Weights of_head = weights_of<kBeside>(pairs, norm != nullptr, norm + (int64_t)min(h, heads - 1) * a.norm_stride, ln);
                weigh<kBeside>(t, pairs, of_head, c, s);
            }
            const uint4 y = turned_heads<kBeside>(pairs, t, r[i], norm != nullptr, a.eps, lane);
            if (h < heads) {
                uint4* at = reinterpret_cast<uint4*>(dst + h * dst_head) + ln;
                if constexpr (kQuads > 1) __builtin_nontemporal_store(u32x4{y.x, y.y, y.z, y.w}, (__attribute__((address_space(1))) u32x4*)at);
                else *at = y;
            }
        }
#pragma unroll
        for (int i = 0; i < kQuads; ++i) r[i] = r_next[i];
        j = j_next;
        run = run_next;
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
    // A wave turns all heads that there are with the angles of a token, unless that leaves compute units idle.  us, heads shared / all in one workgroup, 32 + 2 x 8
    // heads into pages of 16: 1 entry 4.7 / 6.3, 32 of 5 tokens 6.4 / 11.0, 128 full ones 19 / 23, 256 30 / 25, 511 55 / 41 (28 + 2 x 4, pages of 32: 128 25 / 36, 256
    // 42 / 41, 511 75 / 62).
    s.many = s.units >= 2 * (int64_t)ctx->n_cu;
    const int heads = s.many ? 16 : 4;
    s.q_runs = a.q != nullptr ? (int)cdiv(a.q_heads, heads) : 0;
    s.k_runs = a.k != nullptr ? (int)cdiv(a.kv_heads, heads) : 0;
    s.head_parts = s.many ? 1 : s.q_runs + s.k_runs;
    s.parts = s.head_parts + (paged ? (int)cdiv(a.kv_heads, 4) : 0);
    return s;
}

hipError_t launch_rotate(chess_ctx* ctx, RotateArgs a, bool paged, bool beside, hipStream_t stream)
{
    const RotateShape s = rotate_shape(ctx, a, paged);
    a.q_runs = s.q_runs; a.k_runs = s.k_runs; a.head_parts = s.head_parts; a.parts = s.parts; a.units = (int)s.units;
    if (!paged) return s.many ? launch_of<16, false, 4>(a, s.units, beside, stream) : launch_of<16, false, 1>(a, s.units, beside, stream);
    if (ctx->geom.page_size == 16) return s.many ? launch_of<16, true, 4>(a, s.units, beside, stream) : launch_of<16, true, 1>(a, s.units, beside, stream);
    return s.many ? launch_of<32, true, 4>(a, s.units, beside, stream) : launch_of<32, true, 1>(a, s.units, beside, stream);
}

}  // namespace chess

// New tokens' keys and values into 8-bit pages: one power-of-two scale for the tokens of a page and KV head.
//
// A wave owns the keys or the values of one touched page and head: it reads the new rows, takes a = max |x| and with it the smallest e with
// a 2^-e <= 448 (e4m3's largest), and stores e4m3(x 2^-e).  The scale being a power of two costs e4m3 nothing (its relative step
// does not depend on it), and all products with it are exact: the tokens that a page held before are moved to a larger scale by an exact
// product, rounded again only where they become subnormal.
// Values are token-minor in a page: a lane reads the same two (pages of 32: four) dims of 16 tokens and so has 16 bytes of each of the rows
// [dim][token] that it writes, without an exchange.
// Bound: HBM (2 bytes read, 1 written an element); for single tokens the chain entry -> rows -> store and the length of the code that runs once.
// us in a graph: 24K tokens, 8 KV heads, pages of 16 32.3 (4.75 TB/s; a copy of 2 GiB reaches 4.8 to 5.0), 64K, 4 heads, of 32 45.3 (4.45); a token of 32
// sequences, 8 heads, 4.4.  Rows not read as a stream: 36.3 and 50.8.  The values' conversion unrolled over dims: the tokens 4.7.
#include "chess_internal.h"
#include "quant_device.h"
#include "split_rule.h"

namespace chess {

// |x| of the larger of a word's two bf16 values as bits; a value that is not finite counts as 0.
__device__ __forceinline__ uint32_t larger_of(uint32_t w)
{
    const uint32_t lo = w & 0x7fffu, hi = (w >> 16) & 0x7fffu;
    return max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u);
}

__device__ __forceinline__ uint32_t wave_largest(uint32_t v)
{
#define CHESS_MAX(ctrl, rows) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xf, false));
    CHESS_MAX(0x111, 0xf) CHESS_MAX(0x112, 0xf) CHESS_MAX(0x114, 0xf) CHESS_MAX(0x118, 0xf) CHESS_MAX(0x142, 0xa) CHESS_MAX(0x143, 0xc)
#undef CHESS_MAX
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// The smallest e with a 2^-e <= 448 = 1.75 2^8, within what a scale can have (a: bits of a finite bf16 value >= 0; 0 and subnormals end at the
// smallest).
__device__ __forceinline__ int exponent_for(uint32_t a)
{
    const int e = (int)(a >> 7) - 127 - 8 + ((a & 0x7fu) > 0x60u ? 1 : 0);
    return min(max(e, kScaleMin), kScaleMax);
}

// A value as it is rounded: saturated (only the largest scale leaves something above 448); what is not finite becomes NaN, which the clamp
// alone would lose.
__device__ __forceinline__ float scaled(float x, float by)
{
    const float y = __builtin_amdgcn_fmed3f(x * by, -448.f, 448.f);
    return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? __uint_as_float(0x7fc00000u) : y;
}
__device__ __forceinline__ uint32_t four_bytes(float x0, float x1, float x2, float x3, float by)
{
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(x0, by), scaled(x1, by), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(scaled(x2, by), scaled(x3, by), lo, true);
}
// Of a word of two bf16 values.
__device__ __forceinline__ float first_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float second_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// The lowest n bytes of a word.
__device__ __forceinline__ uint32_t bytes_below(int n) { return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u; }

// Four stored bytes moved to a scale 1 / by times as large.
__device__ __forceinline__ uint32_t moved(uint32_t w, float by)
{
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(lo.x * by, lo.y * by, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(hi.x * by, hi.y * by, r, true);
}

// The larger of the exponent that the new values need and, where the page held tokens, its own; `by`: what old values are multiplied with.
__device__ __forceinline__ int grown(uint32_t largest, bool begun, float scale, float* by)
{
    const int need = exponent_for(largest);
    if (!begun) return need;
    const int e_old = (int)((__float_as_uint(scale) >> 23) & 255u) - 127, e = max(need, e_old);
    *by = power_of_two(max(e_old - e, -126));
    return e;
}

template <int B>
__global__ __launch_bounds__(256) void quant_store_kernel(StoreArgs a)
{
    const int lane = threadIdx.x & 63, unit = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
    const int H = a.heads, per = 2 * H, w = unit / per, part = unit - w * per, h = part >= H ? part - H : part;
    // (all three counts here: those that an entry is looked at with would be fetched behind counts[1] otherwise)
    if (((min(a.counts[1], a.max_writes) - 1 - w) | (a.n_rows - 1) | (a.n_pages - 1)) < 0) return;
    const int4 entry = a.writes[w];
    const int phys = __builtin_amdgcn_readfirstlane(entry.x), row0 = __builtin_amdgcn_readfirstlane(entry.y);
    const int first = min(max(__builtin_amdgcn_readfirstlane(entry.z), 0), B - 1), count = min(__builtin_amdgcn_readfirstlane(entry.w), B - first);
    // nothing new, or a row or page that is not there: one of these is negative (the differences wrap for negative rows and pages only, which say so themselves)
    const int rows_left = max((int)((unsigned)a.n_rows - (unsigned)row0), 0) - count, pages_left = (int)((unsigned)a.n_pages - 1u - (unsigned)phys);
    if (((count - 1) | row0 | rows_left | phys | pages_left) < 0) return;
    const size_t ph = (size_t)phys * H + h;
    float* scale_at = a.scales + 2 * ph + (part >= H ? 1 : 0);
    const float scale = first > 0 ? *scale_at : 0.f;
    float by = 1.f;
    if (part < H) {                                   // keys: 16 lanes a row, 8 dims a lane
        const int ln = lane & 15, tg = lane >> 4;
        const uint16_t* src = a.k_new + (int64_t)row0 * a.k_stride + h * kHeadDim + ln * 8;
        uint8_t* page = a.k_pool + ph * (B * kHeadDim);
        uint4 r[B / 4];
#pragma unroll
        for (int i = 0; i < B / 4; ++i)                   // (rows past the last repeat it)
            r[i] = load_16<true>(reinterpret_cast<const uint8_t*>(src + (int64_t)min(4 * i + tg, count - 1) * a.k_stride));
        uint32_t largest = 0;
#pragma unroll
        for (int i = 0; i < B / 4; ++i) largest = max(max(largest, max(larger_of(r[i].x), larger_of(r[i].y))), max(larger_of(r[i].z), larger_of(r[i].w)));
        const int e = grown(wave_largest(largest), first > 0, scale, &by);
        const float inv = power_of_two(-e);
        if (by != 1.f) {                              // tokens before: 8 lanes a row
            for (int t = lane >> 3; t < first; t += 8) {
                uint4* at = reinterpret_cast<uint4*>(page + t * kHeadDim) + (lane & 7);
                uint4 v = *at;
                v.x = moved(v.x, by); v.y = moved(v.y, by); v.z = moved(v.z, by); v.w = moved(v.w, by);
                *at = v;
            }
        }
#pragma unroll
        for (int i = 0; i < B / 4; ++i) {
            const int t = 4 * i + tg;
            if (t < count) {
                uint2 o;
                o.x = four_bytes(first_of(r[i].x), second_of(r[i].x), first_of(r[i].y), second_of(r[i].y), inv);
                o.y = four_bytes(first_of(r[i].z), second_of(r[i].z), first_of(r[i].w), second_of(r[i].w), inv);
                *reinterpret_cast<uint2*>(page + (first + t) * kHeadDim + ln * 8) = o;
            }
        }
        if (lane == 0) *scale_at = power_of_two(e);
    } else {                                          // values: 16 tokens of 2 kWords dims a lane
        constexpr int kWords = B / 16, kLanes = 64 / kWords;
        const int ln = lane % kLanes, t0 = 16 * (lane / kLanes);
        const uint32_t* src = reinterpret_cast<const uint32_t*>(a.v_new + (int64_t)row0 * a.v_stride + h * kHeadDim) + ln * kWords;
        uint8_t* rows = a.v_pool + ph * (B * kHeadDim) + ln * (2 * kWords * B) + t0;
        uint32_t r[16][kWords];
#pragma unroll
        for (int t = 0; t < 16; ++t)                  // (tokens that are not new repeat one that is)
#pragma unroll
            for (int w = 0; w < kWords; ++w)
                r[t][w] = __builtin_nontemporal_load((const __attribute__((address_space(1))) uint32_t*)src + (int64_t)min(max(t0 + t - first, 0), count - 1) * (a.v_stride >> 1) + w);
        uint32_t largest = 0;
#pragma unroll
        for (int t = 0; t < 16; ++t)
#pragma unroll
            for (int w = 0; w < kWords; ++w) largest = max(largest, larger_of(r[t][w]));
        const int e = grown(wave_largest(largest), first > 0, scale, &by);
        const float inv = power_of_two(-e);
        uint32_t is_new[4], is_old[4];                // bytes of a row's four words: written; moved to the new scale
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t below = bytes_below(first - t0 - 4 * i);
            is_new[i] = bytes_below(first + count - t0 - 4 * i) & ~below;
            is_old[i] = by != 1.f ? below : 0u;
        }
#pragma unroll
        for (int w = 0; w < kWords; ++w)
#pragma nounroll
            for (int odd = 0; odd < 2; ++odd) {       // (not unrolled: what runs once is as long as its code)
                uint4* at = reinterpret_cast<uint4*>(rows + (2 * w + odd) * B);
                const int up = odd ? 0 : 16;
                uint32_t o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x[4];
#pragma unroll
                    for (int y = 0; y < 4; ++y) x[y] = second_of(r[4 * i + y][w] << up);
                    o[i] = four_bytes(x[0], x[1], x[2], x[3], inv);
                }
                if (count < B) {                      // what is neither stays as it is
                    const uint4 was4 = *at;
                    const uint32_t was[4] = {was4.x, was4.y, was4.z, was4.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i] = (o[i] & is_new[i]) | (moved(was[i], by) & is_old[i]) | (was[i] & ~(is_new[i] | is_old[i]));
                }
                *at = make_uint4(o[0], o[1], o[2], o[3]);
            }
        if (lane == 0) *scale_at = power_of_two(e);
    }
}

hipError_t launch_quant_store(chess_ctx* ctx, const StoreArgs& a, hipStream_t stream)
{
    const int64_t waves = (int64_t)a.max_writes * 2 * a.heads;
    return launch(ctx->geom.page_size == 16 ? quant_store_kernel<16> : quant_store_kernel<32>, dim3((unsigned)cdiv(waves, 4)), dim3(256), 0, stream, a);
}

}  // namespace chess

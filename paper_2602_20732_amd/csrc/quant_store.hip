// New tokens' keys and values into 8-bit pages: one power-of-two scale for the tokens of a page and KV head.
//
// A wave owns the keys or the values of one touched page and head: it reads the new rows, takes a = max |x| and with it the smallest e with
// a 2^-e <= 448 (e4m3's largest), and stores e4m3(x 2^-e).  The scale being a power of two costs e4m3 nothing (its relative step
// does not depend on it), and all products with it are exact: the tokens that a page held before are moved to a larger scale by an exact
// product, rounded again only where they become subnormal.
// Values are token-minor in a page: a lane reads two dims of every token (256 bytes a wave and token) and so has the two rows
// [dim][token] that it writes, without an exchange.
// Bound: HBM (2 bytes read, 1 written an element); for single tokens the chain entry -> rows -> store.
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

// Two bf16 values as e4m3 bytes in the low half of the result.
__device__ __forceinline__ float scaled(float x, float by)
{
    // (saturated: only the largest scale leaves something above 448; what is not finite becomes NaN, which the clamp alone would lose)
    const float y = __builtin_amdgcn_fmed3f(x * by, -448.f, 448.f);
    return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? __uint_as_float(0x7fc00000u) : y;
}
template <bool kHigh>
__device__ __forceinline__ uint32_t to_bytes(uint32_t w, float by, uint32_t old)
{
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(scaled(__uint_as_float(w << 16), by), scaled(__uint_as_float(w & 0xffff0000u), by), (int)old, kHigh);
}

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
    if (w >= min(a.counts[1], a.max_writes)) return;
    const int4 entry = a.writes[w];
    const int phys = __builtin_amdgcn_readfirstlane(entry.x), row0 = __builtin_amdgcn_readfirstlane(entry.y);
    const int first = min(max(__builtin_amdgcn_readfirstlane(entry.z), 0), B - 1), count = min(__builtin_amdgcn_readfirstlane(entry.w), B - first);
    if (count <= 0) return;
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
        for (int i = 0; i < B / 4; ++i) r[i] = *reinterpret_cast<const uint4*>(src + (int64_t)min(4 * i + tg, count - 1) * a.k_stride);   // (repeats the last)
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
                o.x = to_bytes<true>(r[i].y, inv, to_bytes<false>(r[i].x, inv, 0));
                o.y = to_bytes<true>(r[i].w, inv, to_bytes<false>(r[i].z, inv, 0));
                *reinterpret_cast<uint2*>(page + (first + t) * kHeadDim + ln * 8) = o;
            }
        }
        if (lane == 0) *scale_at = power_of_two(e);
    } else {                                          // values: dims 2 lane and 2 lane + 1 of every token
        const uint16_t* src = a.v_new + (int64_t)row0 * a.v_stride + h * kHeadDim + lane * 2;
        uint4* rows = reinterpret_cast<uint4*>(a.v_pool + ph * (B * kHeadDim) + lane * (2 * B));
        uint32_t r[B];                                // token t of the page
#pragma unroll
        for (int t = 0; t < B; ++t) r[t] = *reinterpret_cast<const uint32_t*>(src + (int64_t)min(max(t - first, 0), count - 1) * a.v_stride);
        uint32_t largest = 0;
#pragma unroll
        for (int t = 0; t < B; ++t) largest = max(largest, larger_of(r[t]));
        const int e = grown(wave_largest(largest), first > 0, scale, &by);
        const float inv = power_of_two(-e);
        const bool whole = count == B;
#pragma unroll
        for (int t0 = 0; t0 < B; t0 += 16) {
            uint32_t even[4], odd[4];                 // 16 tokens of the two dims
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t x[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) x[y] = to_bytes<false>(r[t0 + 4 * i + y], inv, 0);
                even[i] = (x[0] & 255u) | (x[1] & 255u) << 8 | (x[2] & 255u) << 16 | x[3] << 24;
                odd[i] = (x[0] >> 8 & 255u) | (x[1] & 0xff00u) | (x[2] & 0xff00u) << 8 | (x[3] & 0xff00u) << 16;
            }
            uint4* at_even = rows + t0 / 16;
            uint4* at_odd = rows + B / 16 + t0 / 16;
            if (!whole) {                             // the bytes before `first` moved, those behind the new ones as they are
                const uint4 p = *at_even, q = *at_odd;
                const uint32_t was_even[4] = {p.x, p.y, p.z, p.w}, was_odd[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t is_new = 0, is_old = 0;
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const int t = t0 + 4 * i + y;
                        is_new |= t >= first && t < first + count ? 255u << (8 * y) : 0u;
                        is_old |= t < first && by != 1.f ? 255u << (8 * y) : 0u;
                    }
                    even[i] = (even[i] & is_new) | (moved(was_even[i], by) & is_old) | (was_even[i] & ~(is_new | is_old));
                    odd[i] = (odd[i] & is_new) | (moved(was_odd[i], by) & is_old) | (was_odd[i] & ~(is_new | is_old));
                }
            }
            *at_even = make_uint4(even[0], even[1], even[2], even[3]);
            *at_odd = make_uint4(odd[0], odd[1], odd[2], odd[3]);
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

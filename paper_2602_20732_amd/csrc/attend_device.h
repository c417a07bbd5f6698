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

// Over the lanes of a wave, by row shifts and row broadcasts; the same in every lane.
__device__ __forceinline__ int lanes_max(int v)
{
#define CHESS_MAX(ctrl, rows) v = max(v, __builtin_amdgcn_update_dpp(INT32_MIN, v, ctrl, rows, 0xf, false));
    CHESS_MAX(0x111, 0xf) CHESS_MAX(0x112, 0xf) CHESS_MAX(0x114, 0xf) CHESS_MAX(0x118, 0xf) CHESS_MAX(0x142, 0xa) CHESS_MAX(0x143, 0xc)
#undef CHESS_MAX
    return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ int lanes_min(int v) { return ~lanes_max(~v); }

// A sequence of the step: its length, pages, and new tokens (none where token_start names rows that are not there): how many of them are attended, and the
// position of the first (the last is at len - 1, whether it is attended or not).
struct Span { int len, pages, start, n_new, p0; };

__device__ __forceinline__ Span span_of(const AttendArgs& a, int b, int page_size)
{
    Span s;
    s.start = __builtin_amdgcn_readfirstlane(a.token_start[b]);
    s.n_new = __builtin_amdgcn_readfirstlane((int)((unsigned)a.token_start[b + 1] - (unsigned)a.token_start[b]));
    s.len = min(max(__builtin_amdgcn_readfirstlane(a.seq_lens[b]), 0), a.max_pages * page_size);
    s.pages = (s.len + page_size - 1) / page_size;
    if (s.n_new < 0 || s.start < 0 || s.start > a.n_rows - s.n_new) s.n_new = 0;
    s.p0 = s.len - s.n_new;
    s.n_new = min(s.n_new, a.max_new);
    return s;
}

// The same where each lane asks for a sequence of its own.
__device__ __forceinline__ Span span_by_lane(const AttendArgs& a, int b, int page_size)
{
    Span s;
    s.start = a.token_start[b];
    s.n_new = (int)((unsigned)a.token_start[b + 1] - (unsigned)s.start);
    s.len = min(max(a.seq_lens[b], 0), a.max_pages * page_size);
    s.pages = (s.len + page_size - 1) / page_size;
    if (s.n_new < 0 || s.start < 0 || s.start > a.n_rows - s.n_new) s.n_new = 0;
    s.p0 = s.len - s.n_new;
    s.n_new = min(s.n_new, a.max_new);
    return s;
}

// The first key of the window that ends at position p.  (p may be negative, the window as large as an int: no difference of the two.)
__device__ __forceinline__ int first_in_window(const AttendArgs& a, int p) { return a.window > 0 && p >= a.window ? p - a.window + 1 : 0; }

// Query row r of a sequence and KV head: head r % G of its new token r / G.  A row that is not there is the last one again, and sees nothing.
struct RowView {
    int64_t at;              // row of q and out
    int p, lo, hi;           // its position, and the keys it sees
    float slope;             // in powers of two a position
    bool there;
};

__device__ __forceinline__ int64_t row_at(const AttendArgs& a, const Span& s, int h, int r)
{
    const int G = a.group, i = (int)((unsigned)r / (unsigned)G);
    return (int64_t)(s.start + i) * (a.n_kv_heads * G) + h * G + (r - i * G);
}

__device__ __forceinline__ RowView view_of(const AttendArgs& a, const Span& s, int b, int h, int r)
{
    RowView v;
    const int G = a.group, last = s.n_new * G - 1;
    v.there = r <= last;
    r = min(r, last);
    const int i = (int)((unsigned)r / (unsigned)G), g = r - i * G;
    v.at = (int64_t)(s.start + i) * (a.n_kv_heads * G) + h * G + g;
    v.p = s.p0 + i;
    v.slope = a.slopes != nullptr ? a.slopes[h * G + g] * kLog2e : 0.f;
    v.lo = max(a.first_keys != nullptr ? a.first_keys[s.start + i] : 0, first_in_window(a, v.p));
    v.hi = a.prefix_lens != nullptr ? max(v.p, max(a.prefix_lens[b], 1) - 1) : v.p;
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

// A product that is rounded before anything is added to it.
__device__ __forceinline__ float product(float x, float y)
{
#pragma clang fp contract(off)
    return x * y;
}

// A product of query and key as a power of two.
template <bool kCap>
__device__ __forceinline__ float score_of(const AttendArgs& a, float qk)
{
    if constexpr (kCap) return product(a.cap_out, tanh_of(qk * a.cap_in));
    return product(qk, a.scale_log2);
}

// The larger magnitudes of two pairs of bf16 values and eight, as bits; whether one of them is infinite or NaN in any lane.
typedef __attribute__((ext_vector_type(2))) unsigned short Magnitudes;
__device__ __forceinline__ Magnitudes larger(Magnitudes most, const uint4& v)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(Magnitudes, w[i] & 0x7fff7fffu));
    return most;
}
__device__ __forceinline__ bool not_finite(Magnitudes most) { return __any(most.x >= 0x7f80 || most.y >= 0x7f80); }

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

// Which of a lane's 64 outputs of 32 rows (bit 16 d + i: element i of the product of dims 32 d ...) get an infinity, by values that are not finite.  In LDS,
// for each thread: this is rare, and registers are not free.
struct Odd { uint64_t up, down; };

// Where the piece of a dim lies that has the eight keys 16 s + 8 half .. of a tile.
template <int B>
__device__ __forceinline__ int value_piece(int dim, int half, int s)
{
    return B == 16 ? s * 256 + (dim >> 4) * 32 + half * 16 + (dim & 15) : (s >> 1) * 512 + (dim >> 4) * 64 + (2 * (s & 1) + half) * 16 + (dim & 15);
}

// Which of a lane's keys (bit 8 s + e of a 32 keys') its row sees, and which of those have a score of -infinity: these weigh nothing, and nothing times an
// infinity is NaN, where a weight that is only small times an infinity is one.
struct Seen { uint32_t any = 0, lowest = 0; };

// Eight bits as bf16 numbers.
__device__ __forceinline__ bf16x8 ones_of(uint32_t bits)
{
    const auto two = [&](int i) { return (bits >> i & 1u ? 0x3f80u : 0u) | (bits >> (i + 1) & 1u ? 0x3f800000u : 0u); };
    return as_bf16x8(make_uint4(two(0), two(2), two(4), two(6)));
}

// What values that are not finite do: those of 32 keys, of steps step0 and step0 + 1.
template <int B>
__device__ __forceinline__ void note_not_finite(Odd* odd, const uint4* values, int step0, int col, int half, const Seen& seen)
{
#pragma nounroll
    for (int i = 0; i < 8; ++i) {                     // (one at a time: this is rare, and registers are not free)
        const int d = i & 3, down = i >> 2;
        uint32_t any = seen.any, lowest = seen.lowest;
        asm volatile("" : "+v"(any), "+v"(lowest));   // (what follows from them is worked out anew)
        f32x16 n;
#pragma unroll
        for (int j = 0; j < 16; ++j) n[j] = 0.f;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint4 x = values[value_piece<B>(32 * d + col, half, step0 + s)];
            n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(not_finite_of(x, down)), ones_of(any >> (8 * s)), n, 0, 0, 0);
            n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(not_finite_of(x, !down)), ones_of(lowest >> (8 * s)), n, 0, 0, 0);
        }
        uint64_t bits = 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) bits |= n[j] > 0.f ? 1u << j : 0u;
        bits <<= 16 * d;
        if (down) odd->down |= bits;
        else odd->up |= bits;
    }
}

__device__ __forceinline__ void add_not_finite(f32x16 (&o)[4], const Odd& odd)
{
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (odd.up >> (16 * d + i) & 1) o[d][i] += INFINITY;
            if (odd.down >> (16 * d + i) & 1) o[d][i] -= INFINITY;
        }
}

// Where the first two of a partial's four sums of row r from dim on are, of a block's rows, and how many pairs of numbers further on the other two: 32 rows' in
// the order in which a wave's lanes have them (dims 32 d + 8 i + 4 half, row r % 32).  kLines: pairs of all lanes side by side, so that a store writes whole lines
// (a chunk of 1531 tokens, with 100 MB of partials: 815 -> 807 us); a lane's four together otherwise (16 sequences of drafts over every page 376 -> 368).
template <bool kLines>
constexpr int kOtherPair = kLines ? 64 : 1;
template <bool kLines>
__device__ __forceinline__ int64_t part_at(int64_t part, int n_rows, int r, int dim)
{
    return part * n_rows * kHeadDim + (int64_t)(r >> 5) * (32 * kHeadDim) + (dim >> 3) * 256 + ((dim >> 2 & 1) * 32 + (r & 31)) * (kLines ? 2 : 4);
}

// What the last of n_parts workgroups with partials of a block of kRowsOf rows to arrive does: out = sum_s acc_s 2^(m_s - M) / sum_s l_s 2^(m_s - M),
// always in the same order; number(s): which partial s is.  A thread has four dims of each of kPieces rows; kChunk partials of them are asked for at a time.
template <int kRowsOf, int kThreads, int kPieces, int kChunk, bool kLines, class Number>
__device__ __forceinline__ void merge_parts(const AttendArgs& a, const Span& span, int h, int row0, int n_rows, int n_parts, Number number)
{
    static_assert(kRowsOf * 32 % (kThreads * kPieces) == 0);
    for (int i = threadIdx.x; i < kRowsOf * 32; i += kThreads * kPieces) {
        int r[kPieces], dim[kPieces];
        float M[kPieces], l[kPieces], x[kPieces][4];
        bool any = false;
#pragma unroll
        for (int y = 0; y < kPieces; ++y) {
            const int piece = i + y * kThreads;       // a wave's: 32 rows, two fours of dims
            r[y] = (piece >> 10) * 32 + (piece & 31);
            dim[y] = 4 * (piece >> 5 & 31);
            any |= row0 + r[y] < n_rows;
            M[y] = kNegBig;
            l[y] = x[y][0] = x[y][1] = x[y][2] = x[y][3] = 0.f;
        }
        if (!any) continue;
        for (int s0 = 0; s0 < n_parts; s0 += kChunk) {
            uint64_t ml[kPieces][kChunk], v[kPieces][kChunk][2];
#pragma unroll
            for (int y = 0; y < kPieces; ++y)
#pragma unroll
                for (int s = 0; s < kChunk; ++s) {
                    const int64_t part = number(min(s0 + s, n_parts - 1));
                    ml[y][s] = observe_u64(reinterpret_cast<const uint64_t*>(a.part_ml) + part * kRowsOf + r[y]);
                    const uint64_t* at = reinterpret_cast<const uint64_t*>(a.part_acc + part_at<kLines>(part, kRowsOf, r[y], dim[y]));
                    v[y][s][0] = observe_u64(at);
                    v[y][s][1] = observe_u64(at + kOtherPair<kLines>);
                }
#pragma unroll
            for (int y = 0; y < kPieces; ++y) {
                float top = M[y];
#pragma unroll
                for (int s = 0; s < kChunk; ++s) top = fmaxf(top, __builtin_bit_cast(float2, ml[y][s]).x);   // (the last one again changes nothing)
                const float keep = __builtin_amdgcn_exp2f(M[y] - top);
                M[y] = top;
                l[y] *= keep;
#pragma unroll
                for (int d = 0; d < 4; ++d) x[y][d] *= keep;
#pragma unroll
                for (int s = 0; s < kChunk; ++s)
                    if (s0 + s < n_parts) {
                        const float2 one = __builtin_bit_cast(float2, ml[y][s]), lo = __builtin_bit_cast(float2, v[y][s][0]), hi = __builtin_bit_cast(float2, v[y][s][1]);
                        const float by = __builtin_amdgcn_exp2f(one.x - M[y]);
                        l[y] += one.y * by;
                        x[y][0] += lo.x * by; x[y][1] += lo.y * by; x[y][2] += hi.x * by; x[y][3] += hi.y * by;
                    }
            }
        }
#pragma unroll
        for (int y = 0; y < kPieces; ++y) {
            if (row0 + r[y] >= n_rows) continue;
            // A factor may come to 0 where the weights that it rescales do not: an infinite sum stays infinite.  (Looked for behind the sums: a choice a product
            // in code that runs once, cold, cost 1.5 to 2.7 us a launch.)
            const float any_nan = (x[y][0] + x[y][1]) + (x[y][2] + x[y][3]);
            if (__builtin_expect(any_nan != any_nan, 0)) {
                float again[4] = {0.f, 0.f, 0.f, 0.f};
#pragma nounroll
                for (int s = 0; s < n_parts; ++s) {
                    const int64_t part = number(s);
                    const float by = __builtin_amdgcn_exp2f(__builtin_bit_cast(float2, observe_u64(reinterpret_cast<const uint64_t*>(a.part_ml) + part * kRowsOf + r[y])).x - M[y]);
                    const uint64_t* at = reinterpret_cast<const uint64_t*>(a.part_acc + part_at<kLines>(part, kRowsOf, r[y], dim[y]));
                    const float2 lo = __builtin_bit_cast(float2, observe_u64(at)), hi = __builtin_bit_cast(float2, observe_u64(at + kOtherPair<kLines>));
                    const float v[4] = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
                    for (int d = 0; d < 4; ++d) again[d] += fabsf(v[d]) == INFINITY ? v[d] : v[d] * by;
                }
#pragma unroll
                for (int d = 0; d < 4; ++d) x[y][d] = x[y][d] != x[y][d] ? again[d] : x[y][d];
            }
            const float inv = l[y] == 0.f ? 0.f : 1.f / l[y];
            *reinterpret_cast<uint2*>(a.out + row_at(a, span, h, row0 + r[y]) * kHeadDim + dim[y]) =
                make_uint2(two_bf16(x[y][0] * inv, x[y][1] * inv), two_bf16(x[y][2] * inv, x[y][3] * inv));
        }
    }
}

// ---- pages into LDS -------------------------------------------------------------------------------------------------------------------------
// Loads that write LDS themselves: no registers hold what is on its way, so that tiles can be asked for far ahead.  One instruction moves 1 KB, a lane
// 16 bytes to the lane's place behind a common base; what a lane reads is its own choice, and that is how rows are swizzled.  The compiler does not
// know of these loads: whoever reads what they bring waits for them (loads_left) and whoever overwrites what was read waits for the reads (reads_done).
// A quarter of 4 KB from `base` (the same in every lane) + `at` and 1 KB each further on, to LDS bytes [lds, lds + 4096).  kOnce: what nobody reads again is
// not kept in the caches.
#define CHESS_LOAD_4K(hint)                                  \
    asm volatile("s_mov_b32 m0, %0\n\t"                      \
                 "s_nop 0\n\t"                               \
                 "global_load_lds_dwordx4 %2, %1" hint "\n\t" \
                 "global_load_lds_dwordx4 %3, %1 offset:0x400" hint "\n\t" \
                 "global_load_lds_dwordx4 %4, %1 offset:0x800" hint "\n\t" \
                 "global_load_lds_dwordx4 %5, %1 offset:0xc00" hint \
                 :                                           \
                 : "s"(lds), "s"(base), "v"(at0), "v"(at1), "v"(at2), "v"(at3) \
                 : "m0", "memory")
// (m0 is never the compiler's to allocate, of which it warns, but it may put a value there for instructions of its own and use it again later)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <bool kOnce>
__device__ __forceinline__ void load_4k(uint32_t lds, const void* base, uint32_t at0, uint32_t at1, uint32_t at2, uint32_t at3)
{
    if constexpr (kOnce) CHESS_LOAD_4K(" nt");
    else CHESS_LOAD_4K("");
}
#pragma clang diagnostic pop
#undef CHESS_LOAD_4K
template <int kLeft>
__device__ __forceinline__ void loads_left()
{
    static_assert(kLeft < 64);
    asm volatile("" : : : "memory");
    __builtin_amdgcn_s_waitcnt(0xf70 | (kLeft & 15) | (kLeft >> 4) << 14);       // vmcnt(kLeft), nothing else; the compiler counts its own loads with it
    asm volatile("" : : : "memory");
}
__device__ __forceinline__ void reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

template <class T>
__device__ __forceinline__ uint32_t lds_at(T* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) T*)p; }

// The same number in every lane, as a load of its own that does not count with the lanes' loads.
__device__ __forceinline__ int load_same(const int32_t* p, int64_t i) { return ((const __attribute__((address_space(4))) int32_t*)p)[i]; }

// What a lane reads of 16 keys (4 KB; of keys 16 .. 31 of a page the same) and of 4 KB of a page's values, so that sixteen lanes one behind the other, which read
// at once, find the pieces of 16 bytes that they want in different ones of the 16 that lie across all banks.
// Keys: row r has its piece c at c ^ turned(r), and lanes read rows in the order of turned(r).  Values: of sixteen dims, first every one's first piece, then every
// one's second and so on (two of a dim in pages of 16, four in pages of 32); as they lie in memory, a read of pages of 16 took 8 cycles where it takes 4.
__device__ __forceinline__ int turned(int r) { return (r & 19) + ((r & 4) << 1) + ((r & 8) >> 1); }     // bits 2 and 3 change places
struct PageLanes {
    uint32_t key[4], value;
    __device__ __forceinline__ PageLanes(int lane, int page_size)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) key[i] = (uint32_t)((lane >> 4) * 256 + ((lane & 15) ^ turned(4 * i + (lane >> 4))) * 16);
        value = (uint32_t)(page_size == 16 ? ((lane >> 5) * 16 + (lane & 15)) * 2 + ((lane >> 4) & 1) : (lane & 15) * 4 + (lane >> 4)) * 16;
    }
};

// Where 32 keys' operands lie in LDS, in 16-byte pieces from their page's (pages': of 16) beginning.  Row `col` of a product over keys is key
// 16 (col / 16) + 8 (bit 2) + 4 (bit 3) + (col % 4), and with it the 16 weights of a lane are keys 8 half .. + 7 and 16 + 8 half .. + 7.
__device__ __forceinline__ int key_of_col(int col) { return turned(col); }
__device__ __forceinline__ int key_piece(int key, int half, int step) { return key * 16 + ((2 * step + half) ^ turned(key & 15)); }

}  // namespace chess

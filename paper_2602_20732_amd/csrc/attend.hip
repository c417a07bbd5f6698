// Attention of the new tokens of a step, several of a sequence: every new token is a row of queries that sees an interval of the sequence's keys.
//
//   z = sm_scale q . k;   z = cap tanh(z / cap);   z -= slope |p - t|;   out = sum_t softmax(z)_t v_t   over the keys t in [lo, hi] of the row
//
// Causal order, a window, a prefix that all see and the start of the row's document are all of them an interval: lo and hi are worked out once
// a row, and a key is compared with two numbers.  A tile that every row sees whole is not compared at all.
#include "attend_device.h"

#include "deal.h"
#include "split_rule.h"

namespace chess {

// ---- few rows a sequence and KV head (drafted tokens): the keys are split ------------------------------------------------------
// A workgroup has up to 32 kRows query rows (token, head of the group) and every n-th tile of 32 keys, a wave every fourth of those; a wave
// reads K and V from the pages into the operands of 32 x 32 x 16 products:
//   S^T[key][row] = K[key][dim] Q^T[dim][row]             8 products a tile and 32 rows
//   O^T[dim][row] += V^T[dim][key] P^T[key][row]          8, twice: P as a bf16 number and a bf16 remainder (2^-17 of a weight)
// The key rows of the first are dealt so that the 16 weights a lane ends up with are the 2 x 8 that it has to supply to the second.
// The rows of the next tile are asked for as soon as the registers of this one's are free.
// Bound: HBM, for as long as a tile's products (1.3 us a wave of 64 rows) take less than its 16 KB do.
template <int B, int kRows, bool kList, bool kDealt, bool kCap>
__global__ __launch_bounds__(256, kRows == 1 ? 2 : 1) void attend_few_kernel(AttendArgs a)
{
    constexpr int PPT = 32 / B;
    __shared__ float comb[2][4][16][64];
    __shared__ float wave_m[4][32 * kRows], wave_l[4][32 * kRows];
    __shared__ int flag;
    __shared__ DealLds<4> deal;
    __shared__ uint4 queries[32 * kRows][16];         // 16-byte pieces of a row, piece i of row r at i ^ (r % 16): no two rows' on the same banks
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int col = lane & 31, half = lane >> 5;
    const int H = a.n_kv_heads, G = a.group;

    int b, h, split, n_splits;
    int64_t part0;
    if constexpr (kDealt) {
        h = blockIdx.x % H;
        const int slot = blockIdx.x / H;
        const SlotShare s = share_slots<B, 4, 32>(slot, a.n_slots, a.batch, a.n_splits, a.rows_most, a.seq_lens, a.max_pages, lane, wave, deal);
        if (s.b < 0) return;
        b = __builtin_amdgcn_readfirstlane(s.b);
        split = __builtin_amdgcn_readfirstlane(s.split);
        n_splits = __builtin_amdgcn_readfirstlane(s.n_splits);
        part0 = (int64_t)h * a.n_slots + __builtin_amdgcn_readfirstlane(s.first);
    } else {
        h = blockIdx.x % H;
        const int x = blockIdx.x / H;
        b = x % a.batch;
        split = x / a.batch;
        n_splits = a.n_splits;
        part0 = ((int64_t)blockIdx.y * a.batch * H + (int64_t)b * H + h) * n_splits;
    }
    const Span span = span_of(a, b, B);
    const int n_rows = span.n_new * G, row0 = blockIdx.y * (32 * kRows);
    if (row0 >= n_rows) return;

    // the rows: what each sees; their queries into LDS
    RowView row[kRows];
    int see_lo = INT32_MAX, see_hi = -1, all_lo = 0, all_hi = INT32_MAX;
#pragma unroll
    for (int y = 0; y < kRows; ++y) {
        row[y] = view_of(a, span, b, h, row0 + 32 * y + col);
        const uint4* src = reinterpret_cast<const uint4*>(a.q + row[y].at * kHeadDim) + 4 * wave + 2 * half;
#pragma unroll
        for (int s = 0; s < 2; ++s) queries[32 * y + col][(4 * wave + 2 * half + s) ^ (col & 15)] = src[s];
        if (row[y].there) {
            if (row[y].hi >= row[y].lo) {
                see_lo = min(see_lo, row[y].lo);
                see_hi = max(see_hi, row[y].hi);
            }
            all_lo = max(all_lo, row[y].lo);
            all_hi = min(all_hi, row[y].hi);
        }
    }
    see_lo = lanes_min(see_lo); see_hi = lanes_max(see_hi); all_lo = lanes_max(all_lo); all_hi = lanes_min(all_hi);

    __syncthreads();

    // its tiles
    const int P = span.pages;
    const int32_t* table = a.block_table + (int64_t)b * a.max_pages;
    const int32_t* ids = kList ? a.page_ids + ((int64_t)b * H + h) * a.max_sel : nullptr;
    const int n_list = kList ? min(max(a.n_selected[(int64_t)b * H + h], 0), a.max_sel) : P;
    int t_first = 0, t_end = P > 0 && see_hi >= see_lo ? (n_list + PPT - 1) / PPT : 0;
    if constexpr (!kList) {
        t_first = see_hi >= see_lo ? see_lo / 32 : 0;
        t_end = min(t_end, see_hi / 32 + 1);
    }
    const int stride = 4 * n_splits;
    int t = t_first + split * 4 + wave;

    float m[kRows], l[kRows];
    f32x16 o[kRows][4];
#pragma unroll
    for (int y = 0; y < kRows; ++y) {
        m[y] = kNegBig;
        l[y] = 0.f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[y][d][i] = 0.f;
    }

    int lp[PPT], lp_next[PPT], phys_next[PPT];
    uint4 k[8], v[4][2];
    const auto pages_of = [&](int tile, int (&page)[PPT]) {         // logical pages of a tile; a slot without one: -1
#pragma unroll
        for (int s = 0; s < PPT; ++s) {
            const int i = tile * PPT + s;
            int p = i;
            if constexpr (kList) p = ids[min(i, a.max_sel - 1)];
            page[s] = i < n_list && p >= 0 && p < P ? p : -1;
        }
    };
    const auto look_up = [&](const int (&page)[PPT], int (&phys)[PPT]) {
#pragma unroll
        for (int s = 0; s < PPT; ++s) phys[s] = table[max(page[s], 0)];
    };
    const auto load_k = [&](const int (&phys)[PPT]) {
        // row `col` of the product is key 16 (col / 16) + 8 (bit 2) + 4 (bit 3) + (col % 4) of the tile
        const int key = (col & 16) + ((col & 4) << 1) + ((col & 8) >> 1) + (col & 3);
        const int64_t pg = PPT == 1 || key < B ? phys[0] : phys[PPT - 1];
        const uint4* src = reinterpret_cast<const uint4*>(a.k_pool + ((pg * H + h) * B + key % B) * kHeadDim) + half;
#pragma unroll
        for (int s = 0; s < 8; ++s) k[s] = src[2 * s];
    };
    const auto load_v = [&](const int (&phys)[PPT]) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int64_t pg = phys[(16 * s) / B];
            const uint16_t* src = a.v_pool + ((pg * H + h) * kHeadDim + col) * B + (16 * s) % B + 8 * half;
#pragma unroll
            for (int d = 0; d < 4; ++d) v[d][s] = *reinterpret_cast<const uint4*>(src + d * 32 * B);
        }
    };
    const auto first_key = [&](const int (&page)[PPT], int s) {     // of the eight keys that a lane has of step s
        return page[(16 * s) / B] < 0 ? INT32_MIN / 2 : page[(16 * s) / B] * B + (16 * s) % B + 8 * half;
    };
    const auto scalar = [&](int (&x)[PPT]) {
#pragma unroll
        for (int s = 0; s < PPT; ++s) x[s] = __builtin_amdgcn_readfirstlane(x[s]);
    };

    if (t < t_end) {
        int phys[PPT];
        pages_of(t, lp);
        look_up(lp, phys);
        scalar(phys);
        load_k(phys);
        load_v(phys);
        pages_of(min(t + stride, t_end - 1), lp_next);
        look_up(lp_next, phys_next);
    }
    for (; t < t_end; t += stride) {
        // whether a row may see less than all of the tile
        bool part = false;
#pragma unroll
        for (int s = 0; s < PPT; ++s) part = part || lp[s] < 0 || lp[s] * B < all_lo || lp[s] * B + B - 1 > all_hi;
        part = __builtin_amdgcn_readfirstlane(part);
        f32x16 z[kRows];
#pragma unroll
        for (int y = 0; y < kRows; ++y) {
#pragma unroll
            for (int i = 0; i < 16; ++i) z[y][i] = 0.f;
#pragma unroll
            for (int s = 0; s < 8; ++s) z[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k[s]), as_bf16x8(queries[32 * y + col][(2 * s + half) ^ (col & 15)]), z[y], 0, 0, 0);
        }
        scalar(phys_next);
        int phys[PPT];
#pragma unroll
        for (int s = 0; s < PPT; ++s) phys[s] = phys_next[s];
        load_k(phys);                                 // (behind the last tile: that one's again)
        int lp_now[PPT];
#pragma unroll
        for (int s = 0; s < PPT; ++s) {
            lp_now[s] = lp[s];
            lp[s] = lp_next[s];
        }
        pages_of(min(t + 2 * stride, t_end - 1), lp_next);
        look_up(lp_next, phys_next);

        bf16x8 hi_part[kRows][2], lo_part[kRows][2];
#pragma unroll
        for (int y = 0; y < kRows; ++y) {
            // z[8 s + e] is key 16 s + 8 half + e of the tile
            float largest = kNegBig;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int key0 = first_key(lp_now, s);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float x = score_of<kCap>(a, z[y][8 * s + e]);
                    x = fmaf(-row[y].slope, fabsf((float)(row[y].p - key0 - e)), x);
                    const bool see = key0 + e >= row[y].lo && key0 + e <= row[y].hi;
                    if (part) x = see ? x : -INFINITY;
                    z[y][8 * s + e] = x;
                    largest = fmaxf(largest, x);
                }
            }
            largest = fmaxf(largest, __shfl_xor(largest, 32));
            const float m_new = fmaxf(m[y], largest);
            if (__any(m_new > m[y])) {
                const float alpha = __builtin_amdgcn_exp2f(m[y] - m_new);
                l[y] *= alpha;
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[y][d][i] *= alpha;
                m[y] = m_new;
            }
            float sum = 0.f;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float w = __builtin_amdgcn_exp2f(z[y][8 * s + e] - m[y]);
                    sum += w;
                    const __bf16 top = (__bf16)w;
                    hi_part[y][s][e] = top;
                    lo_part[y][s][e] = (__bf16)(w - (float)top);
                }
            l[y] += sum;
        }
        // keys that a row does not see weigh nothing, but nothing times a value that is not finite is NaN, and a remainder may be nothing or
        // negative: such values are taken out of the product, and what they do to the rows that see them is added by itself
        if (__builtin_expect(not_finite(v), 0)) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int y = 0; y < kRows; ++y) {
                bf16x8 seen[2], lowest[2];            // (a score of -infinity weighs nothing: that times an infinity is NaN, both of them here)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int key0 = first_key(lp_now, s);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const bool see = key0 + e >= row[y].lo && key0 + e <= row[y].hi;
                        seen[s][e] = (__bf16)(see ? 1.f : 0.f);
                        lowest[s][e] = (__bf16)(see && z[y][8 * s + e] == -INFINITY ? 1.f : 0.f);
                    }
                }
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int sign = 0; sign < 2; ++sign) {
                        f32x16 n;
#pragma unroll
                        for (int i = 0; i < 16; ++i) n[i] = 0.f;
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(not_finite_of(v[d][s], sign)), seen[s], n, 0, 0, 0);
                            n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(not_finite_of(v[d][s], !sign)), lowest[s], n, 0, 0, 0);
                        }
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[y][d][i] += n[i] > 0.f ? (sign ? -INFINITY : INFINITY) : 0.f;
                        __builtin_amdgcn_sched_barrier(0);          // (one after the other: this is rare, and registers are not)
                    }
            }
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int s = 0; s < 2; ++s) v[d][s] = finite_of(v[d][s]);
        }
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int y = 0; y < kRows; ++y)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    o[y][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v[d][s]), hi_part[y][s], o[y][d], 0, 0, 0);
                    o[y][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v[d][s]), lo_part[y][s], o[y][d], 0, 0, 0);
                }
        load_v(phys);
    }

    // the workgroup's waves: O^T[dim 32 d + 8 (i / 4) + 4 half + i % 4][row col]
#pragma unroll
    for (int y = 0; y < kRows; ++y) {
        l[y] += __shfl_xor(l[y], 32);
        if (half == 0) {
            wave_m[wave][32 * y + col] = m[y];
            wave_l[wave][32 * y + col] = l[y];
        }
    }
    __syncthreads();
    const bool whole = n_splits == 1;
#pragma unroll
    for (int y = 0; y < kRows; ++y) {
        float top = kNegBig, sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, wave_m[w][32 * y + col]);
#pragma unroll
        for (int w = 0; w < 4; ++w) sum += wave_l[w][32 * y + col] * __builtin_amdgcn_exp2f(wave_m[w][32 * y + col] - top);
        const float by = __builtin_amdgcn_exp2f(m[y] - top), inv = sum == 0.f ? 0.f : 1.f / sum;
        const int64_t part = (part0 + split) * (32 * kRows) + 32 * y + col;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            float(&buf)[4][16][64] = comb[d & 1];
#pragma unroll
            for (int i = 0; i < 16; ++i) buf[wave][i][lane] = o[y][d][i] * by;
            __syncthreads();
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = (buf[0][4 * wave + i][lane] + buf[1][4 * wave + i][lane]) + (buf[2][4 * wave + i][lane] + buf[3][4 * wave + i][lane]);
            const int dim = 32 * d + 8 * wave + 4 * half;
            if (whole) {
                if (row[y].there)
                    *reinterpret_cast<uint2*>(a.out + row[y].at * kHeadDim + dim) = make_uint2(two_bf16(x[0] * inv, x[1] * inv), two_bf16(x[2] * inv, x[3] * inv));
            } else {
                uint64_t* at = reinterpret_cast<uint64_t*>(a.part_acc + part * kHeadDim + dim);
                publish_u64(at, __builtin_bit_cast(uint64_t, make_float2(x[0], x[1])));
                publish_u64(at + 1, __builtin_bit_cast(uint64_t, make_float2(x[2], x[3])));
            }
        }
        if (!whole && wave == 0 && half == 0) publish_u64(reinterpret_cast<uint64_t*>(a.part_ml) + part, __builtin_bit_cast(uint64_t, make_float2(top, sum)));
    }
    if (whole) return;
    if (!arrive_last(a.arrivals + ((int64_t)b * H + h) * kArrivalStride + blockIdx.y, n_splits, &flag)) return;
    merge_parts<32 * kRows, 256>(a, span, h, row0, n_rows, part0, n_splits);
}

// ---- launch -----------------------------------------------------------------------------------------------------------------------------------
template <int B, int kRows, bool kCap>
static hipError_t launch_few(const AttendArgs& a, const AttendShape& s, bool list, hipStream_t stream)
{
    const dim3 grid((unsigned)(s.n_slots > 0 ? (int64_t)s.n_slots * a.n_kv_heads : (int64_t)a.batch * s.n_splits * a.n_kv_heads), (unsigned)s.blocks);
    if (list) return launch(attend_few_kernel<B, kRows, true, false, kCap>, grid, dim3(256), 0, stream, a);
    return s.n_slots > 0 ? launch(attend_few_kernel<B, kRows, false, true, kCap>, grid, dim3(256), 0, stream, a)
                         : launch(attend_few_kernel<B, kRows, false, false, kCap>, grid, dim3(256), 0, stream, a);
}

AttendShape attend_shape(const chess_ctx* ctx, int64_t max_new, int batch, bool list)
{
    const Geom& g = ctx->geom;
    const int ppt = kTileTokens / g.page_size;
    AttendShape s{};
    const int64_t rows = max_new * g.group, want = 2 * (int64_t)ctx->n_cu;
    s.rows = rows <= 32 ? 32 : 64;
    s.blocks = (int)cdiv(rows, s.rows);
    const int64_t pairs = (int64_t)batch * g.n_kv_heads * s.blocks, waves = cdiv(list ? g.max_sel : g.max_pages, 4 * ppt);
    // (an arrival counter for each block of a pair: 64)
    s.n_splits = s.blocks > kArrivalStride ? 1 : (int)clampi(want / pairs, 1, std::min<int64_t>(waves, 64));
    if (!list && s.blocks == 1 && batch > 1 && batch <= kDealMost && s.n_splits > 1) {
        s.n_slots = (int)(want / g.n_kv_heads);
        s.n_splits = (int)std::min<int64_t>(waves, 64);
    }
    s.parts = s.n_slots > 0 ? (int64_t)s.n_slots * g.n_kv_heads : s.n_splits > 1 ? pairs * s.n_splits : 0;
    return s;
}

hipError_t launch_attend(chess_ctx* ctx, AttendArgs a, const AttendShape& s, hipStream_t stream)
{
    a.n_slots = s.n_slots;
    a.n_splits = s.n_splits;
    const bool list = a.page_ids != nullptr, cap = a.cap_in != 0.f;
    if (ctx->geom.page_size == 16) {
        if (s.rows == 32) return cap ? launch_few<16, 1, true>(a, s, list, stream) : launch_few<16, 1, false>(a, s, list, stream);
        return cap ? launch_few<16, 2, true>(a, s, list, stream) : launch_few<16, 2, false>(a, s, list, stream);
    }
    if (s.rows == 32) return cap ? launch_few<32, 1, true>(a, s, list, stream) : launch_few<32, 1, false>(a, s, list, stream);
    return cap ? launch_few<32, 2, true>(a, s, list, stream) : launch_few<32, 2, false>(a, s, list, stream);
}

}  // namespace chess

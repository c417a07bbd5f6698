// Attention of the new tokens of a step, several of a sequence: every new token is a row of queries that sees an interval of the sequence's keys.
//
//   z = sm_scale q . k;   z = cap tanh(z / cap);   z -= slope |p - t|;   out = sum_t softmax(z)_t v_t   over the keys t in [lo, hi] of the row
//
// Causal order, a window, a prefix that all see and the start of the row's document are all of them an interval: lo and hi are worked out once
// a row, and a key is compared with two numbers.  A tile that every row sees whole is not compared at all.
#include <atomic>

#include "attend_device.h"
#include "deal.h"
#include "split_rule.h"

namespace chess {

// ---- few rows a sequence and KV head (drafted tokens): the keys are split ------------------------------------------------------
// A tile is 32 keys (16 KB).  The tiles of all sequences of a KV head lie in a line, in sequence order, and each of the head's workgroups (one a
// compute unit) takes an equal share of it: the segments of one or several sequences.  Within a segment a wave takes every fourth tile, all
// (token, head of the group) rows at once, up to 32 kRows of them:
//   S^T[key][row] = K[key][dim] Q^T[dim][row]             8 products of 32 x 32 x 16 a tile and 32 rows
//   O^T[dim][row] += V^T[dim][key] P^T[key][row]          8, twice: P as a bf16 number and a bf16 remainder (2^-17 of a weight)
// Each wave has two tiles of LDS of its own: one is worked on, the next is on its way (loads that write LDS, no barrier).  A sequence that lies in one share
// is written at once; partials of the others are merged by the last workgroup of the sequence to arrive.
// Bound: HBM, for as long as a tile's arithmetic (about 1 us a wave and 32 rows) takes less than the four waves' 64 KB do (2.7 us).  Measured, 32 query and 8 KV
// heads: 16 sequences of 5 drafts over every page of 8 to 64K keys (2.19 GB) 360 to 373 us, 5.9 to 6.1 TB/s, what a read reaches; 32 sequences of 2 to 8 over lists of 108 pages
// (229 MB) 46 us; one sequence's list of 21 pages 11.1.

// The first key that any of the tokens [from, to] sees for its document.
__device__ __forceinline__ int first_of_rows(const AttendArgs& a, int from, int to)
{
    int first = INT32_MAX;
    if (to - from < 3) {
        for (int i = from; i <= to; ++i) first = min(first, a.first_keys[i]);
        return first;
    }
    for (int i = from; i <= to; i += 32) {            // (fours of them, asked for together: one by one they were most of the plan's time)
        struct Four { int32_t first[4]; } four[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) __builtin_memcpy(&four[j], a.first_keys + min(i + 4 * j, to - 3), sizeof(Four));
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) first = min(first, four[j].first[e]);
    }
    return first;
}

// A lane's sequence as those that deal see it: the tiles of the keys that its rows can see at all, from `first` on, one at least if it has rows.
struct LineSpan { int start, n_new, p0, len, n_list, first, count; };

template <int B, bool kList>
__device__ __forceinline__ LineSpan line_span(const AttendArgs& a, int b, int h)
{
    constexpr int PPT = 32 / B;
    const bool there = b < a.batch;
    const int n_selected = kList ? a.n_selected[(int64_t)min(b, a.batch - 1) * a.n_kv_heads + h] : 0;
    const Span s = span_by_lane(a, min(b, a.batch - 1), B);
    LineSpan l{s.start, there ? s.n_new : 0, s.p0, s.len, kList ? min(max(n_selected, 0), a.max_sel) : s.pages, 0, 0};
    if constexpr (!kList) {
        l.first = first_in_window(a, s.p0) / 32;
        if (a.first_keys != nullptr && l.n_new > 0) l.first = max(l.first, max(first_of_rows(a, s.start, s.start + l.n_new - 1), 0) / 32);
    }
    if (l.n_new > 0) l.count = max((kList ? (l.n_list + PPT - 1) / PPT : (s.len + 31) / 32) - l.first, 1);
    return l;
}

constexpr int kFewRing = 4 * 2 * 1024;                // 16-byte pieces: two tiles a wave
constexpr size_t few_lds(int rows) { return (kFewRing + rows * 16) * 16; }

template <int B, int kRows, bool kList, bool kCap>
__global__ __launch_bounds__(256, 1) void attend_few_kernel(AttendArgs a)
{
    constexpr int PPT = 32 / B;
    extern __shared__ uint4 ring[];                   // [wave][stage][1024]: 512 pieces of keys, 512 of values; afterwards the waves' sums.  Then [row][16] the queries
    __shared__ float wave_m[4][32 * kRows], wave_l[4][32 * kRows];
    __shared__ int block_tiles[kDealMost / 64];
    __shared__ Odd odd[kRows][256];
    __shared__ int wave_odd[4], flag;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int col = lane & 31, half = lane >> 5;
    const int H = a.n_kv_heads, G = a.group, h = blockIdx.x % H, slot = blockIdx.x / H;

    // the line: its length, this workgroup's share, the sequence that it begins in
    LineSpan mine = line_span<B, kList>(a, lane, h);
    int before = 0, block = 0, upto = lanes_upto(mine.count), total = lane_of(upto, 63), of_block = 0, upto_block = 0;
    if (a.batch > 64) {
        for (int i = wave; i * 64 < a.batch; i += 4) {
            const int n = lane_of(lanes_upto(line_span<B, kList>(a, i * 64 + lane, h).count), 63);
            if (lane == 0) block_tiles[i] = n;
        }
        __syncthreads();
        of_block = lane * 64 < a.batch ? block_tiles[lane] : 0;
        upto_block = lanes_upto(of_block);
        total = lane_of(upto_block, 63);
    }
    // (a tile a wave at least)
    int share = max((int)(((int64_t)total + a.n_slots - 1) / a.n_slots), 4);
    // A change of sequence within a share costs what three rounds of the waves do.  If shares that are longer by no more than that suffice for sequences that
    // begin with a share of their own, they do, and no share has more than one (in a graph, 16 sequences of 500 to 4000 tokens 53.2 -> 48.3 us, 6 lists of 44 pages
    // 25.0 -> 21.5).
    int in_line = mine.count;                         // tiles of the line that the lane's sequence has
    bool alone = false;
    if (a.batch <= min(64, a.n_slots))
        for (int more = 0; more <= 12 && !alone; more += 4) {
            const int shares = (int)((unsigned)(mine.count + share + more - 1) / (unsigned)(share + more)), n = lanes_upto(shares);
            if (lane_of(n, 63) <= a.n_slots) {
                alone = true;
                share += more;
                in_line = shares * share;
                upto = n * share;
                total = lane_of(upto, 63);
            }
        }
    const int begin = slot * share, end = min(begin + share, total);
    if (begin >= end) return;
    if (a.batch > 64) {
        block = __builtin_ctzll(__ballot(upto_block > begin));
        before = lane_of(upto_block, block) - lane_of(of_block, block);
        mine = line_span<B, kList>(a, block * 64 + lane, h);
        upto = lanes_upto(mine.count);
    }
    const int at = __builtin_ctzll(__ballot(before + upto > begin));
    int b = __builtin_amdgcn_readfirstlane(block * 64 + at);
    int line = __builtin_amdgcn_readfirstlane(before + lane_of(upto, at) - (alone ? lane_of(in_line, at) : lane_of(mine.count, at)));     // where the sequence begins in the line

    const PageLanes from(lane, B);
    const uint32_t ring_lds = lds_at(ring) + (uint32_t)wave * (2 * 16384);
    const uint4* ring_own = ring + wave * 2048;
    uint4* queries = ring + kFewRing;

    for (; line < end && b < a.batch; ++b) {          // (b: should the lengths be changed meanwhile)
        if (b == block * 64 + 64) {
            ++block;
            mine = line_span<B, kList>(a, block * 64 + lane, h);
        }
        const int in_block = b - block * 64, count = lane_of(mine.count, in_block);
        if (count == 0) continue;
        const Span span{lane_of(mine.len, in_block), (lane_of(mine.len, in_block) + B - 1) / B, lane_of(mine.start, in_block), lane_of(mine.n_new, in_block),
                        lane_of(mine.p0, in_block)};
        const int first = lane_of(mine.first, in_block), n_list = lane_of(mine.n_list, in_block), line_end = line + count;
        // this segment, in tiles of the sequence
        int t = max(begin - line, 0) + first + wave;
        int t_end = min(end - line, count) + first;
        const int P = span.pages;
        const int32_t* table = a.block_table + (int64_t)b * a.max_pages;
        const int32_t* ids = kList ? a.page_ids + ((int64_t)b * H + h) * a.max_sel : nullptr;
        if (P == 0 || n_list == 0) t_end = 0;         // (a tile was dealt all the same, so that the rows are written)

        // Logical pages (one that is none of the sequence's: -1) and physical ones of the wave's next tiles, 64 at a time, one a lane: a window of the table (or
        // list) is asked for a window ahead, and what a tile needs of it is read from a lane.  (A scalar load a tile would be waited for with the LDS reads,
        // which count with it.)
        constexpr int kWindow = 64 / PPT;             // tiles of the wave
        const int t0 = t;
        struct Window { int page, phys; };
        const auto window_at = [&](int number) {
            const int i = (t0 + 4 * (number * kWindow + lane / PPT)) * PPT + lane % PPT;
            int p = i;
            if constexpr (kList) p = ids[min(i, a.max_sel - 1)];
            const int page = i < n_list && p >= 0 && p < P ? p : -1;
            return Window{page, table[max(page, 0)]};
        };
        // (Read once, so not kept in the caches: in a graph 32 sequences' lists 57.5 -> 51.6 us, every page of 16 sequences 409 -> 376.)
        const auto fetch = [&](const int (&phys)[PPT], int stage) {
            const uint32_t to = ring_lds + (uint32_t)stage * 16384;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int64_t at = ((int64_t)__builtin_amdgcn_readfirstlane(phys[s * PPT / 2]) * H + h) * (B * kHeadDim) + (PPT == 1 ? s * 2048 : 0);
                load_4k<true>(to + s * 4096, a.k_pool + at, from.key[0], from.key[1], from.key[2], from.key[3]);
                load_4k<true>(to + 8192 + s * 4096, a.v_pool + at, from.value, from.value, from.value, from.value);
            }
        };

        Window window{-1, 0}, window_next{-1, 0};     // the one that tile n + 2 of the wave is in, and the next
        const auto pages_of = [&](int n, int (&page)[PPT], int (&phys)[PPT]) {
#pragma unroll
            for (int s = 0; s < PPT; ++s) {
                page[s] = __builtin_amdgcn_readlane(window.page, n % kWindow * PPT + s);
                phys[s] = __builtin_amdgcn_readlane(window.phys, n % kWindow * PPT + s);
            }
        };
        int lp[PPT], lp_next[PPT], phys[PPT];
        if (t < t_end) {
            window = window_at(0);
            window_next = window_at(1);
            pages_of(0, lp, phys);
            fetch(phys, 0);
            pages_of(1, lp_next, phys);
            if (t + 4 < t_end) fetch(phys, 1);
        }
        // the rows: their queries (Q^T operands), what each sees
        const int n_rows = span.n_new * G;
        RowView row[kRows];
        int all_lo = 0, all_hi = INT32_MAX;
#pragma unroll
        for (int y = 0; y < kRows; ++y) {
            row[y] = view_of(a, span, b, h, 32 * y + col);
            // (piece i of row r at i ^ (r % 16): no two rows' on the same banks)
            const uint4* src = reinterpret_cast<const uint4*>(a.q + row[y].at * kHeadDim) + 4 * wave + 2 * half;
#pragma unroll
            for (int s = 0; s < 2; ++s) queries[(32 * y + col) * 16 + ((4 * wave + 2 * half + s) ^ (col & 15))] = src[s];
            if (row[y].there) {
                all_lo = max(all_lo, row[y].lo);
                all_hi = min(all_hi, row[y].hi);
            }
        }
        all_lo = lanes_max(all_lo);
        all_hi = lanes_min(all_hi);

        float m[kRows], l[kRows];
        f32x16 o[kRows][4];
        bool any_odd = false;
#pragma unroll
        for (int y = 0; y < kRows; ++y) odd[y][threadIdx.x] = Odd{0, 0};
#pragma unroll
        for (int y = 0; y < kRows; ++y) {
            m[y] = kNegBig;
            l[y] = 0.f;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[y][d][i] = 0.f;
        }

        __syncthreads();                              // the queries
        for (int n = 0, stage = 0; t < t_end; t += 4, ++n, stage ^= 1) {
            const uint4* keys = ring_own + stage * 1024;
            const uint4* values = keys + 512;
            if (t + 4 < t_end) loads_left<16>();
            else loads_left<0>();
            // whether a row may see less than all of the tile
            int less = 0;
#pragma unroll
            for (int s = 0; s < PPT; ++s) less |= lp[s] | (lp[s] * B - all_lo) | (all_hi - lp[s] * B - B + 1);
            const bool part = __builtin_amdgcn_readfirstlane(less) < 0;
            f32x16 z[kRows];
#pragma unroll
            for (int y = 0; y < kRows; ++y)
#pragma unroll
                for (int i = 0; i < 16; ++i) z[y][i] = 0.f;
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const bf16x8 k = as_bf16x8(keys[key_piece(key_of_col(col), half, s)]);
#pragma unroll
                for (int y = 0; y < kRows; ++y) z[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, as_bf16x8(queries[(32 * y + col) * 16 + ((2 * s + half) ^ (col & 15))]), z[y], 0, 0, 0);
            }
            uint4 v[4][2];
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int s = 0; s < 2; ++s) v[d][s] = values[value_piece<B>(32 * d + col, half, s)];

            const auto first_key = [&](int s) {       // of the eight keys that a lane has of step s
                const int page = lp[s * PPT / 2];
                return page < 0 ? INT32_MIN / 2 : page * B + (16 * s) % B + 8 * half;
            };
            bf16x8 hi_part[kRows][2], lo_part[kRows][2];
            Seen seen[kRows];
#pragma unroll
            for (int y = 0; y < kRows; ++y) {
                // z[8 s + e] is key 16 s + 8 half + e of the tile
                float largest = kNegBig;
                seen[y].any = part ? 0u : 0xffffu;
                seen[y].lowest = 0;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int key0 = first_key(s);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float x = score_of<kCap>(a, z[y][8 * s + e]);
                        x = fmaf(-row[y].slope, fabsf((float)(row[y].p - key0 - e)), x);
                        if (part) {
                            const bool see = key0 + e >= row[y].lo && key0 + e <= row[y].hi;
                            seen[y].any |= see ? 1u << (8 * s + e) : 0u;
                            x = see ? x : -INFINITY;
                        }
                        seen[y].lowest |= x == -INFINITY ? 1u << (8 * s + e) : 0u;
                        z[y][8 * s + e] = x;
                        largest = fmaxf(largest, x);
                    }
                }
                seen[y].lowest &= seen[y].any;
                largest = fmaxf(largest, __shfl_xor(largest, 32));
                const float m_new = fmaxf(m[y], largest);
                if (__any(m_new > m[y])) {
                    const float alpha = __builtin_amdgcn_exp2f(m[y] - m_new);
                    l[y] *= alpha;
#pragma unroll
                    for (int d = 0; d < 4; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[y][d][i] *= alpha;
                    __builtin_amdgcn_sched_barrier(0);
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
            // negative: such values are taken out of the product, and what they do to the rows that see them is noted by itself
            Magnitudes most = {0, 0};
#pragma unroll
            for (int d = 0; d < 4; ++d) most = larger(larger(most, v[d][0]), v[d][1]);
            if (__builtin_expect(not_finite(most), 0)) {
#pragma unroll
                for (int y = 0; y < kRows; ++y) note_not_finite<B>(&odd[y][threadIdx.x], values, 0, col, half, seen[y]);
                any_odd = true;
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int s = 0; s < 2; ++s) v[d][s] = finite_of(v[d][s]);
            }
            // the tile's LDS is free: the one after the next into it
            if ((n + 2) % kWindow == 0) {
                window = window_next;
                window_next = window_at((n + 2) / kWindow + 1);
            }
#pragma unroll
            for (int s = 0; s < PPT; ++s) lp[s] = lp_next[s];
            pages_of(n + 2, lp_next, phys);
            if (t + 8 < t_end) {
                reads_done();
                fetch(phys, stage);
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
        }

        // the workgroup's waves: O^T[dim 32 d + 8 (i / 4) + 4 half + i % 4][row col]
        if (lane == 0) wave_odd[wave] = any_odd;
#pragma unroll
        for (int y = 0; y < kRows; ++y) {
            l[y] += __shfl_xor(l[y], 32);
            if (half == 0) {
                wave_m[wave][32 * y + col] = m[y];
                wave_l[wave][32 * y + col] = l[y];
            }
        }
        __syncthreads();                              // (and no wave's tiles are read or written any more)
        float(*comb)[4][16][64] = reinterpret_cast<float(*)[4][16][64]>(ring);
        const int w0 = line / share, n_parts = (line_end - 1) / share - w0 + 1;
        const bool whole = n_parts == 1, some_odd = __builtin_amdgcn_readfirstlane(wave_odd[0] | wave_odd[1] | wave_odd[2] | wave_odd[3]) != 0;
        const int64_t part0 = 2 * ((int64_t)h * a.n_slots + w0);
        const int64_t part_own = 2 * ((int64_t)h * a.n_slots + slot) + (slot == w0 ? 1 : 0);
#pragma unroll
        for (int y = 0; y < kRows; ++y) {
            float top = kNegBig, sum = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) top = fmaxf(top, wave_m[w][32 * y + col]);
#pragma unroll
            for (int w = 0; w < 4; ++w) sum += wave_l[w][32 * y + col] * __builtin_amdgcn_exp2f(wave_m[w][32 * y + col] - top);
            const float by = __builtin_amdgcn_exp2f(m[y] - top), inv = sum == 0.f ? 0.f : 1.f / sum;
            const int64_t part = part_own * (32 * kRows) + 32 * y + col;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                float(&buf)[4][16][64] = comb[d];
#pragma unroll
                for (int i = 0; i < 16; ++i) buf[wave][i][lane] = o[y][d][i] * by;
            }
            __syncthreads();
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                float(&buf)[4][16][64] = comb[d];
                float x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = (buf[0][4 * wave + i][lane] + buf[1][4 * wave + i][lane]) + (buf[2][4 * wave + i][lane] + buf[3][4 * wave + i][lane]);
                // (infinities behind the sums: a wave's factor may come to 0 where the weights that it rescales do not)
                if (__builtin_expect(some_odd, 0)) {
                    uint64_t up = 0, down = 0;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        up |= odd[y][64 * w + lane].up;
                        down |= odd[y][64 * w + lane].down;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (up >> (16 * d + 4 * wave + i) & 1) x[i] += INFINITY;
                        if (down >> (16 * d + 4 * wave + i) & 1) x[i] -= INFINITY;
                    }
                }
                const int dim = 32 * d + 8 * wave + 4 * half;
                if (whole) {
                    if (row[y].there)
                        *reinterpret_cast<uint2*>(a.out + row[y].at * kHeadDim + dim) = make_uint2(two_bf16(x[0] * inv, x[1] * inv), two_bf16(x[2] * inv, x[3] * inv));
                } else {
                    uint64_t* to = reinterpret_cast<uint64_t*>(a.part_acc + part_at<false>(part_own, 32 * kRows, 32 * y + col, dim));
                    publish_u64(to, __builtin_bit_cast(uint64_t, make_float2(x[0], x[1])));
                    publish_u64(to + kOtherPair<false>, __builtin_bit_cast(uint64_t, make_float2(x[2], x[3])));
                }
            }
            if (!whole && wave == 0 && half == 0) publish_u64(reinterpret_cast<uint64_t*>(a.part_ml) + part, __builtin_bit_cast(uint64_t, make_float2(top, sum)));
            __syncthreads();
        }
        if (!whole && arrive_last(a.arrivals + ((int64_t)b * H + h) * kArrivalStride, n_parts, &flag))
            merge_parts<32 * kRows, 256, 2, 4, false>(a, span, h, 0, n_rows, n_parts, [&](int s) { return part0 + 2 * s + (s == 0 ? 1 : 0); });
        line = alone ? end : line_end;
    }
}

// ---- many rows (prompts): the rows are split ----------------------------------------------------------------------------------------------
// A unit is 128 rows (token, head of the group) of a sequence and KV head, 32 a wave, and a run of tiles of 64 keys (32 KB) that its workgroup brings to
// LDS for all of them, the next while one is worked on; the next tile's products of queries and keys are formed while this one's exponentials are.  The same
// products as above, twice as many keys at a time, but the weights are bf16: an output is rounded to bf16 all the same, and its weights' roundings come
// to less than that (the sum of the weights is of the unrounded ones).
// A plan says which units there are (plan_kernel): tiles that no row of a block sees are left out, and long blocks are cut where there are too
// few to fill the card; partials are merged by the last unit of a block to arrive.
// Bound: the matrix units and the exponentials beside them, 32 products of 32 cycles and 32 exponentials a lane for a tile and wave.  Measured, 32 query and 8 KV
// heads: 1531 tokens behind 31K 785 to 820 us by card, 980 to 1020 TFLOP/s (a large library product 1246); 12 prompts of 131 to 2051 tokens, documents of 1203 and a
// bias by distance 191 us, 515 TFLOP/s of the pairs that are seen: units of 8 tiles, each with 6.5 us of lookup, first tile and output around 22 us of tiles.

constexpr int kBlockRows = 128;
constexpr size_t kManyLds = 4 * 16384;                // two tiles' keys, two tiles' values
constexpr int kPlanThreads = 1024;

__device__ __forceinline__ int blocks_of(int n_new, int G) { return (int)(((int64_t)n_new * G + kBlockRows - 1) / kBlockRows); }

// The keys that a block's rows see at all: first and last (last < first: none).
struct Keys { int first, last; };
__device__ __forceinline__ Keys keys_of_block(const AttendArgs& a, const Span& s, int b, int block)
{
    const int G = a.group, row_end = min((block + 1) * kBlockRows, s.n_new * G) - 1;
    const int i0 = (int)((unsigned)(block * kBlockRows) / (unsigned)G), i1 = (int)((unsigned)row_end / (unsigned)G);
    const int p0 = s.p0 + i0, p1 = s.p0 + i1;
    Keys k{first_in_window(a, p0), min(a.prefix_lens != nullptr ? max(p1, max(a.prefix_lens[b], 1) - 1) : p1, s.len - 1)};
    if (a.first_keys != nullptr) {
        k.first = max(k.first, first_of_rows(a, s.start + i0, s.start + i1));
    }
    if (p1 < 0) k.last = -1;
    return k;
}

// One workgroup.  Blocks in sequence order: their tiles; how long a unit may be (by what the card would take for it, of sixteen lengths); the units, longest
// first as far as it is known (whole lengths, then the rest), and which partials they leave.
// Bound: the chain starts -> blocks -> sums -> units, and that its code runs once: 9 us for 48 blocks, 14 for 410 with documents' starts.
template <int B>
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(AttendArgs a)
{
    constexpr int kWaves = kPlanThreads / 64, kTry = 16, kEighths = 8;
    extern __shared__ int upto[];                     // [batch]: blocks of the sequences up to this one
    __shared__ int of_wave[3][kWaves], most_of_wave[kWaves], units_of_wave[kTry][kWaves], eighths_of_wave[kEighths * kWaves];
    __shared__ float tiles_of_wave[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // running sums over all threads' numbers, and the whole sums
    const auto sums_before = [&](int (&v)[3], int (&all)[3]) {
        int own[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) own[i] = lanes_upto(v[i]);
        __syncthreads();
        if (lane == 63)
#pragma unroll
            for (int i = 0; i < 3; ++i) of_wave[i][wave] = own[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const int upto_wave = lanes_upto(lane < kWaves ? of_wave[i][lane] : 0);
            all[i] = lane_of(upto_wave, kWaves - 1);
            v[i] = own[i] - v[i] + (wave > 0 ? lane_of(upto_wave, max(wave - 1, 0)) : 0);
        }
    };
    int n_blocks = 0;
    for (int b0 = 0; b0 < a.batch; b0 += kPlanThreads) {
        const int b = b0 + (int)threadIdx.x, n = b < a.batch ? blocks_of(span_by_lane(a, b, B).n_new, a.group) : 0;
        int v[3] = {n, 0, 0}, all[3];
        sums_before(v, all);
        if (b < a.batch) upto[b] = n_blocks + v[0] + n;
        n_blocks += all[0];
    }
    __syncthreads();
    n_blocks = min(n_blocks, a.blocks_most);
    int most = 1;
    float tiles = 0.f;                                // (estimates only)
    int4 own_block = make_int4(0, 0, 0, 0);           // of the first kPlanThreads: not read again
    for (int i = threadIdx.x; i < n_blocks; i += kPlanThreads) {
        int lo = 0, hi = a.batch - 1;                 // the first sequence whose blocks go beyond i
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (upto[mid] > i) hi = mid;
            else lo = mid + 1;
        }
        const int block = i - (lo > 0 ? upto[lo - 1] : 0);
        const Span s = span_by_lane(a, lo, B);
        const Keys k = keys_of_block(a, s, lo, block);
        const bool any = k.last >= k.first;
        int first = any ? k.first / 64 : 0, n = any ? k.last / 64 - first + 1 : 1;
        if (a.page_ids != nullptr) {                  // tiles of the longest list of its heads (those with shorter ones have units without tiles)
            int longest = 0;
#pragma unroll 8
            for (int h = 0; h < a.n_kv_heads; ++h) longest = max(longest, a.n_selected[(int64_t)lo * a.n_kv_heads + h]);
            first = 0;
            n = any ? max((min(longest, a.max_sel) + 64 / B - 1) / (64 / B), 1) : 1;
        }
        a.blocks[i] = make_int4(lo, block, first, n);
        if (i < kPlanThreads) own_block = make_int4(lo, block, first, n);
        most = max(most, n);
        tiles += (float)n;
        for (int h = 0; h < a.n_kv_heads; ++h) a.counters[(int64_t)i * a.n_kv_heads + h] = 0;
    }
    most = lanes_max(most);
    tiles = lane_of(lanes_upto(tiles), 63);
    if (lane == 0) {
        most_of_wave[wave] = most;
        tiles_of_wave[wave] = tiles;
    }
    __syncthreads();
    most = 1;
    tiles = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        most = max(most, most_of_wave[w]);
        tiles += tiles_of_wave[w];
    }
    const auto block_at = [&](int i) { return i < kPlanThreads ? own_block : a.blocks[i]; };      // (a thread's own)
    // units of each length tried
    const auto length = [&](int y) { return max((most + y) / (y + 1), 1); };
    int units[kTry] = {};
    for (int i = threadIdx.x; i < n_blocks; i += kPlanThreads) {
        const int n = block_at(i).w;
#pragma unroll
        for (int y = 0; y < kTry; ++y) units[y] += (n + length(y) - 1) / length(y);
    }
#pragma unroll
    for (int y = 0; y < kTry; ++y) {
        const int n = lanes_upto(units[y]);
        if (lane == 63) units_of_wave[y][wave] = n;
    }
    __syncthreads();
    // what each would take, in tiles: a unit costs some of its own, and a cut one the partials'.  Lane y: length y
    int n_units = 0;
    if (lane < kTry)
#pragma unroll
        for (int w = 0; w < kWaves; ++w) n_units += units_of_wave[lane][w];
    const int len_y = length(lane), extra = n_units - n_blocks;
    const float cut = extra > 0 ? 6.f : 0.f, slots = (float)a.n_slots, of_heads = (float)(n_units * a.n_kv_heads);
    // (a workgroup alone on its compute unit takes two thirds of the time for a tile: 32 sequences of 20 tokens over 27 tiles 80 us cut in halves, 68 whole)
    const float size = (2.f * of_heads <= slots ? 0.65f : 1.f) * (float)len_y + 5.f + cut;
    // units as long as each other go in rounds, others into the gaps
    const float in_rounds = ceilf(of_heads / slots) * size, in_gaps = ((float)a.n_kv_heads * tiles + of_heads * (5.f + cut)) / slots + 0.5f * size;
    float cost = fmaxf(fminf(in_rounds, in_gaps), size);
    if (lane > 0 && (lane >= kTry || len_y < 8 || extra > a.extra_most || min(n_units, 2 * extra) > a.parts_most)) cost = INFINITY;
    float least = cost;
#pragma unroll
    for (int by = 32; by > 0; by /= 2) least = fminf(least, __shfl_xor(least, by));
    const int len = lane_of(len_y, __builtin_ctzll(__ballot(cost <= 1.03f * least)));       // (the longest of those that are as good)
    // Whole lengths first, then what is left of the blocks by eighths of a length, the longest first, so that the last units to begin are short ones.  A wave
    // counts its blocks' by the lanes that have one; then where each wave's of each eighth begin.
    const auto eighth = [&](int i, int rest) { return i < n_blocks && rest > 0 ? 7 - min(8 * rest / len, 7) : kEighths; };
    int whole_before = 0, rest_before = 0, parts_before = 0, of_eighth = 0;               // (lane: eighth)
    for (int i0 = 0; i0 < n_blocks; i0 += kPlanThreads) {
        const int i = i0 + (int)threadIdx.x, n = i < n_blocks ? block_at(i).w : 0;
        int v[3] = {n / len, 0, 0}, all[3];
        sums_before(v, all);
        rest_before += all[0];
        const int own = eighth(i, n % len);
#pragma unroll
        for (int c = 0; c < kEighths; ++c) {
            const int n_own = __popcll(__ballot(own == c));
            if (lane == c) of_eighth += n_own;
        }
    }
    if (lane < kEighths) eighths_of_wave[lane * kWaves + wave] = of_eighth;
    __syncthreads();
    {
        const int e0 = eighths_of_wave[2 * lane], e1 = eighths_of_wave[2 * lane + 1], e = lanes_upto(e0 + e1);
        const int mine = min(lane, kEighths - 1) * kWaves + wave;      // where this wave's begin
        of_eighth = rest_before + __shfl(e - e0 - e1, mine >> 1) + ((mine & 1) != 0 ? __shfl(e0, mine >> 1) : 0);
        rest_before += lane_of(e, 63);
    }
    for (int i0 = 0; i0 < n_blocks; i0 += kPlanThreads) {
        const int i = i0 + (int)threadIdx.x;
        const int4 blk = i < n_blocks ? block_at(i) : make_int4(0, 0, 0, 0);
        const int whole = blk.w / len, rest = blk.w - whole * len, n = whole + (rest > 0 ? 1 : 0);
        int v[3] = {whole, n > 1 ? n : 0, 0}, all[3];
        sums_before(v, all);
        const int at = whole_before + v[0], part0 = parts_before + v[1], own = eighth(i, rest);
        whole_before += all[0];
        parts_before += all[1];
        int at_rest = 0;
#pragma unroll
        for (int c = 0; c < kEighths; ++c) {
            const unsigned long long those = __ballot(own == c);
            if (own == c) at_rest = lane_of(of_eighth, c) + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(those >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)those, 0));
            if (lane == c) of_eighth += __popcll(those);
        }
        for (int s = 0; s < n; ++s) {
            AttendUnit u;
            u.b = blk.x; u.block = blk.y;
            u.first = blk.z + s * len;
            u.end = blk.z + min((s + 1) * len, blk.w);
            u.n_parts = n; u.part = part0 + s; u.part0 = part0; u.counter = i;
            a.units[s < whole ? at + s : at_rest] = u;
        }
    }
    if (threadIdx.x == 0) *a.n_units = rest_before;
}

template <int B, bool kList, bool kGeneral>
__global__ __launch_bounds__(256, 2) void attend_many_kernel(AttendArgs a)
{
    constexpr int PPT = 64 / B;
    extern __shared__ uint4 stages[];                 // [2][1024] keys, [2][1024] values
    __shared__ Odd odd[256];
    __shared__ int wave_lo[4], wave_hi[4], wave_nan[4], flag;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int col = lane & 31, half = lane >> 5;
    const int H = a.n_kv_heads, G = a.group, h = blockIdx.x % H, unit = blockIdx.x / H;
    if (unit >= load_same(a.n_units, 0)) return;
    const auto of_unit = [&](int i) { return load_same(reinterpret_cast<const int32_t*>(a.units + unit), i); };
    const int b = of_unit(0), block = of_unit(1), n_parts = of_unit(4);
    int t = of_unit(2), t_end = of_unit(3);
    const Span span = span_of(a, b, B);
    const int P = span.pages, n_rows = span.n_new * G, row0 = block * kBlockRows + 32 * wave;
    const int32_t* table = a.block_table + (int64_t)b * a.max_pages;
    const int32_t* ids = kList ? a.page_ids + ((int64_t)b * H + h) * a.max_sel : nullptr;
    const int n_list = kList ? min(max(load_same(a.n_selected, (int64_t)b * H + h), 0), a.max_sel) : P;
    if constexpr (kList) t_end = min(t_end, (n_list + PPT - 1) / PPT);
    if (P == 0) t_end = 0;
    const int t_first = t;

    // a wave brings 16 keys, and 16 keys' values
    const PageLanes from(lane, B);
    const uint32_t to = lds_at(stages) + (uint32_t)wave * 4096;
    const auto page_at = [&](int i) {
        int p = i;
        if constexpr (kList) p = load_same(ids, min(i, a.max_sel - 1));
        return i < n_list && p >= 0 && p < P ? p : -1;
    };
    const auto place = [&](int phys) { return ((int64_t)__builtin_amdgcn_readfirstlane(phys) * H + h) * (B * kHeadDim) + (B == 32 ? (wave & 1) * 2048 : 0); };
    const auto fetch_keys = [&](int phys, int stage) {
        load_4k<false>(to + (uint32_t)stage * 16384, a.k_pool + place(phys), from.key[0], from.key[1], from.key[2], from.key[3]);
    };
    const auto fetch_values = [&](int phys, int stage) {
        load_4k<false>(to + 32768 + (uint32_t)stage * 16384, a.v_pool + place(phys), from.value, from.value, from.value, from.value);
    };
    // Physical pages by the 64, one a lane: a window of the table (or list) is asked for a window ahead, and what a tile needs of it is read from a lane.
    // (A scalar load a tile would be waited for with the LDS reads, which count with it.)
    constexpr int kWindow = 64 / PPT;                 // tiles
    const auto page_of_tile = [&](int tile) { return tile * PPT + (B == 32 ? wave >> 1 : wave); };
    const auto window_at = [&](int tile) {
        const int i = min(tile / kWindow * 64 + lane, kList ? a.max_sel - 1 : a.max_pages - 1);
        int p = i;
        if constexpr (kList) p = ids[i];
        return table[i < n_list && p >= 0 && p < P ? p : 0];
    };
    // keys of tile t and t + 1, values of t
    int phys = 0, window = 0, window_next = 0;        // phys: of tile t + 1; the window that tile t + 2 is in
    if (t < t_end) {
        const int first = load_same(table, max(page_at(page_of_tile(t)), 0));
        fetch_keys(first, 0);
        phys = load_same(table, max(page_at(page_of_tile(min(t + 1, t_end - 1))), 0));
        fetch_keys(phys, 1);
        fetch_values(first, 0);
        window = window_at(t + 2);
        window_next = window_at(t + 2 + kWindow);
    }

    RowView row = view_of(a, span, b, h, row0 + col);
    const bool works = row0 < n_rows;                 // a wave without rows only brings its keys
    uint4 q[8];
    {
        const uint4* src = reinterpret_cast<const uint4*>(a.q + row.at * kHeadDim) + half;
#pragma unroll
        for (int s = 0; s < 8; ++s) q[s] = src[2 * s];
    }
    // what all rows of the block see
    int all_lo = lanes_max(row.there ? row.lo : 0), all_hi = lanes_min(row.there ? row.hi : INT32_MAX);
    if (lane == 0) {
        wave_lo[wave] = all_lo;
        wave_hi[wave] = all_hi;
    }

    float m = kNegBig, l = 0.f;
    f32x16 o[4];
    bool any_odd = false;
    odd[threadIdx.x] = Odd{0, 0};
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

    loads_left<0>();
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        all_lo = max(all_lo, wave_lo[w]);
        all_hi = min(all_hi, wave_hi[w]);
    }
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    all_hi = __builtin_amdgcn_readfirstlane(all_hi);

    int stage = 0;                                    // of tile t
    // Keys of tile t + 1 and values of t are there, and nobody reads the keys of t and the values of t - 1 any more: those of t + 2 and t + 1 into their places.
    // (The first tile's are there already.)
    const auto begin_tile = [&] {
        loads_left<0>();
        if ((t + 2) % kWindow == 0 && t > t_first) {
            window = window_next;
            window_next = window_at(t + 2 + kWindow);
        }
        __syncthreads();
        const int phys_next = __builtin_amdgcn_readlane(window, page_of_tile(t + 2) & 63);
        if (t + 2 < t_end) fetch_keys(phys_next, stage);
        if (t + 1 < t_end) fetch_values(phys, stage ^ 1);
        phys = phys_next;
    };
    // whether every row of the block sees all of a tile (the same in every wave)
    const auto is_whole = [&](int tile) {
        if constexpr (!kList) return ((tile * 64 - all_lo) | (all_hi - tile * 64 - 63)) >= 0;
        int less = 0;
#pragma unroll
        for (int s = 0; s < PPT; ++s) {
            const int p = page_at(tile * PPT + s);
            less |= p | (p * B - all_lo) | (all_hi - p * B - B + 1);
        }
        return less >= 0;
    };
    const auto first_key = [&](int i) {               // of a lane's eight keys of step i
        const int p = page_at(t * PPT + 16 * i / B);
        return p < 0 ? INT32_MIN / 2 : p * B + (16 * i) % B + 8 * half;
    };
    // z[y][8 s + e] is key 32 y + 16 s + 8 half + e of a tile
    const auto products = [&](f32x16 (&z)[2], int of_stage) {
        const uint4* keys = stages + of_stage * 1024;
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int i = 0; i < 16; ++i) z[y][i] = 0.f;
#pragma unroll
        for (int s = 0; s < 8; ++s)
#pragma unroll
            for (int y = 0; y < 2; ++y)
                z[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(keys[key_piece(32 * y + key_of_col(col), half, s)]), as_bf16x8(q[s]), z[y], 0, 0, 0);
    };
    // values that are not finite, as above: what they do to the rows that see them is noted, then they are taken out of the tile, by all waves for all
    const auto clean = [&](const Seen (&seen)[2]) {
        uint4* values = stages + 2048 + stage * 1024;
        Magnitudes most = {0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i) most = larger(most, values[i * 64 + lane]);
        if (__builtin_expect(!not_finite(most), 1)) return;
        any_odd = true;
#pragma unroll
        for (int y = 0; y < 2; ++y) note_not_finite<B>(odd + threadIdx.x, values, 2 * y, col, half, seen[y]);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) values[i * 256 + threadIdx.x] = finite_of(values[i * 256 + threadIdx.x]);
        __syncthreads();
    };
    const float scale = kGeneral ? 1.f : a.scale_log2;
    // Tile t, whose products are in z; those of t + 1 into next while the exponentials of t are worked out.
    const auto work_on = [&](f32x16 (&z)[2], f32x16 (&next)[2]) {
        begin_tile();
        if constexpr (kGeneral) {
            if (a.cap_in != 0.f) {
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[y][i] = score_of<true>(a, z[y][i]);
            } else {
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[y][i] = score_of<false>(a, z[y][i]);
            }
            if (a.slopes != nullptr)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float d = (float)(row.p - first_key(i));
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[i >> 1][8 * (i & 1) + e] = fmaf(-row.slope, fabsf(d - (float)e), z[i >> 1][8 * (i & 1) + e]);
                }
        }
        if (!is_whole(t)) {
            Seen seen[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key0 = first_key(i);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool see = key0 + e >= row.lo && key0 + e <= row.hi;
                    const float x = z[i >> 1][8 * (i & 1) + e];
                    seen[i >> 1].any |= see ? 1u << (8 * (i & 1) + e) : 0u;
                    seen[i >> 1].lowest |= see && x == -INFINITY ? 1u << (8 * (i & 1) + e) : 0u;
                    z[i >> 1][8 * (i & 1) + e] = see ? x : -INFINITY;
                }
            }
            clean(seen);
        }
        float largest = z[0][0];
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int i = 0; i < 16; ++i) largest = fmaxf(largest, z[y][i]);
        // The running maximum (of scores times `scale`) and what was summed are moved to a new one where that is 2^8 times as large: until then weights above 1 do
        // no harm.
        const float m_new = fmaxf(m, product(fmaxf(largest, __shfl_xor(largest, 32)), scale));
        if (__any(m_new - m > 8.f)) {
            const float alpha = __builtin_amdgcn_exp2f(m - m_new);
            l *= alpha;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
            m = m_new;
        }
        // a score times `scale` this large is rounded before the difference, as the maximum was: what one rounding would keep could weigh more than 1
        float by = scale, top = m;
        if (!kGeneral && __builtin_expect(__any(fabsf(m_new) > 0x1p24f && m != kNegBig), 0)) {
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int i = 0; i < 16; ++i) z[y][i] = product(z[y][i], scale) - m;
            by = 1.f;
            top = 0.f;
        }
        __builtin_amdgcn_s_setprio(1);
        products(next, stage ^ 1);                    // (behind the last tile: of whatever is there)
        float sum = 0.f;
        bf16x8 w[2][2];
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = __builtin_amdgcn_exp2f(kGeneral ? z[y][8 * s + e] - top : fmaf(z[y][8 * s + e], by, -top));
                    sum += x;
                    w[y][s][e] = (__bf16)x;
                }
        l += sum;
        const uint4* values = stages + 2048 + stage * 1024;
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int d = 0; d < 4; ++d)
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(values[value_piece<B>(32 * d + col, half, s)]), w[s >> 1][s & 1], o[d], 0, 0, 0);
        __builtin_amdgcn_s_setprio(0);
        ++t;
        stage ^= 1;
    };
    if (works) {
        f32x16 z[2], z_next[2];
        if (t < t_end) products(z, 0);
        while (t < t_end) {
            work_on(z, z_next);
            if (t >= t_end) break;
            work_on(z_next, z);
        }
    } else {
        while (t < t_end) {
            begin_tile();
            const Seen none[2];
            if (!is_whole(t)) clean(none);
            ++t;
            stage ^= 1;
        }
    }
    // Tiles that all rows see whole are not looked through for values that are not finite.  Sums that come to NaN with one (a weight that is only small has become 0)
    // say so by themselves (as two do that are infinite either way), and then the values of those tiles are looked at: what they do is the same for every row.  (Units
    // whose values are finite pay the additions and a barrier: packed prompts 191.6 -> 193.3 us, a chunk 803 -> 805.)
    float of_dims[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int d = 0; d < 4; ++d) of_dims[d] += o[d][i];
    const float of_all = (of_dims[0] + of_dims[1]) + (of_dims[2] + of_dims[3]);
    const int some_nan = __any(of_all != of_all);
    if (lane == 0) wave_nan[wave] = some_nan;
    __syncthreads();                                  // (and nobody reads the last tile any more)
    if (__builtin_expect(__builtin_amdgcn_readfirstlane(wave_nan[0] | wave_nan[1] | wave_nan[2] | wave_nan[3]) != 0, 0)) {
        // A thread: half of a tile's values of a dim, eight at a time; bit 0: up, bit 1: down.  (A key that is not finite has a score of -infinity, if it has one that
        // is not a row's NaN: it weighs nothing.)
        const int dim = threadIdx.x % kHeadDim;
        uint32_t bits = 0;
#pragma nounroll
        for (int tile = t_first; tile < t_end && bits != 3; ++tile) {
            if (!is_whole(tile)) continue;
#pragma nounroll
            for (int i = 0; i < 4 && bits != 3; ++i) {
                const int token = (threadIdx.x / kHeadDim) * 32 + 8 * i;
                const int64_t at = ((int64_t)table[page_at(tile * PPT + token / B)] * H + h) * (B * kHeadDim);
                const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(a.v_pool + at + dim * B + token % B);
#pragma nounroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t x = (uint32_t)((e < 4 ? v.x : v.y) >> (16 * (e & 3))) & 0xffffu;
                    if ((x & 0x7f80u) != 0x7f80u) continue;
                    Magnitudes most = {(unsigned short)(x & 0x7fu ? 0x7f80 : 0), 0};
                    const uint4* key = reinterpret_cast<const uint4*>(a.k_pool + at + (token % B + e) * kHeadDim);
#pragma nounroll
                    for (int c = 0; c < kHeadDim / 8 && a.cap_in == 0.f && most.x < 0x7f80 && most.y < 0x7f80; ++c) most = larger(most, key[c]);
                    bits |= most.x >= 0x7f80 || most.y >= 0x7f80 ? 3u : x >> 15 != 0 ? 2u : 1u;
                }
            }
        }
        uint32_t* of_dim = reinterpret_cast<uint32_t*>(stages);
        of_dim[threadIdx.x] = bits;
        __syncthreads();
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int at = 32 * d + 8 * (i >> 2) + 4 * half + (i & 3);
                const uint32_t both = of_dim[at] | of_dim[kHeadDim + at];
                if (o[d][i] != o[d][i] && (both == 1 || both == 2)) o[d][i] = both == 1 ? INFINITY : -INFINITY;
            }
    }
    if (any_odd) add_not_finite(o, odd[threadIdx.x]);
    l += __shfl_xor(l, 32);
    if (n_parts == 1) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        int r = row0 + col;
        asm volatile("" : "+v"(r));                   // (worked out again, not kept: registers are not free)
        const int64_t at = row_at(a, span, h, r);
        if (r < n_rows)
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<uint2*>(a.out + at * kHeadDim + 32 * d + 2 * i + 4 * half) =
                        make_uint2(two_bf16(o[d][i] * inv, o[d][i + 1] * inv), two_bf16(o[d][i + 2] * inv, o[d][i + 3] * inv));
        return;
    }
    const int64_t part = (int64_t)of_unit(5) * H + h;
    if (works) {
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                uint64_t* at = reinterpret_cast<uint64_t*>(a.part_acc + part_at<true>(part, kBlockRows, 32 * wave + col, 32 * d + 2 * i + 4 * half));
                publish_u64(at, __builtin_bit_cast(uint64_t, make_float2(o[d][i], o[d][i + 1])));
                publish_u64(at + kOtherPair<true>, __builtin_bit_cast(uint64_t, make_float2(o[d][i + 2], o[d][i + 3])));
            }
        if (half == 0) publish_u64(reinterpret_cast<uint64_t*>(a.part_ml) + part * kBlockRows + 32 * wave + col, __builtin_bit_cast(uint64_t, make_float2(m, l)));
    }
    if (!arrive_last(a.counters + (int64_t)of_unit(7) * H + h, n_parts, &flag)) return;
    const int64_t part0 = (int64_t)of_unit(6) * H + h;
    merge_parts<kBlockRows, 256, 4, 4, true>(a, span, h, block * kBlockRows, n_rows, n_parts, [&](int s) { return part0 + (int64_t)s * H; });
}

// ---- launch -----------------------------------------------------------------------------------------------------------------------------------
// A kernel with more LDS than one may have unasked: asked for once a device (it costs the host more than a microsecond).
template <auto kKernel>
static hipError_t launch_lds(chess_ctx* ctx, dim3 grid, size_t lds, hipStream_t stream, const AttendArgs& a)
{
    static std::atomic<uint64_t> asked{0};
    const uint64_t bit = ctx->device < 64 ? (uint64_t)1 << ctx->device : 0;
    if ((asked.load(std::memory_order_relaxed) & bit) == 0) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kKernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
        asked.fetch_or(bit, std::memory_order_relaxed);
    }
    return launch(kKernel, grid, dim3(256), lds, stream, a);
}

template <int B, int kRows, bool kCap>
static hipError_t launch_few(chess_ctx* ctx, const AttendArgs& a, bool list, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.n_slots * a.n_kv_heads));
    return list ? launch_lds<attend_few_kernel<B, kRows, true, kCap>>(ctx, grid, few_lds(32 * kRows), stream, a)
                : launch_lds<attend_few_kernel<B, kRows, false, kCap>>(ctx, grid, few_lds(32 * kRows), stream, a);
}

template <int B, bool kList>
static hipError_t launch_many(chess_ctx* ctx, const AttendArgs& a, const AttendShape& s, bool general, hipStream_t stream)
{
    const dim3 grid((unsigned)((s.blocks + s.extra) * a.n_kv_heads));
    return general ? launch_lds<attend_many_kernel<B, kList, true>>(ctx, grid, kManyLds, stream, a) : launch_lds<attend_many_kernel<B, kList, false>>(ctx, grid, kManyLds, stream, a);
}

// Few rows: a line a KV head.  Many: units; `most` blocks and cut units that there can be, whatever the sequences are.
// The line has room for 64 rows.  us, as few / as many rows, in a graph, 8 KV heads, pages of 16, one sequence of 500, 4K, 32K, 130K keys, then 16 of 500, 4K, 32K:
//   32 rows  11 / 22    23 / 27    43 / 58    106 / 171      17 / 24    55 / 58    342 / 370
//   64 rows  20 / 26    38 / 32    66 / 65    146 / 180      27 / 27    77 / 63    439 / 378
// One KV head, 64 rows, one sequence of 32K: 191 / 66 (250 partials that one workgroup merges).  From 65 rows on there is no choice, and a block is cut into 16 units at
// most: 17 tokens of 4 heads a group behind 130K take 194 us (the keys alone 87 at 6.1 TB/s).
AttendShape attend_shape(const chess_ctx* ctx, int64_t n_rows, int64_t max_new, int64_t batch, bool list)
{
    const Geom& g = ctx->geom;
    AttendShape s{};
    max_new = std::min(max_new, n_rows);
    const int64_t cu = std::max(ctx->n_cu / g.n_kv_heads, 1);
    if (few_rows(max_new * g.group, batch, cdiv(list ? g.max_sel : g.max_pages, 32 / g.page_size), cu)) {
        s.rows = max_new * g.group <= 32 ? 32 : 64;
        s.n_slots = cu;
        s.parts = 2 * cu * g.n_kv_heads;
        return s;
    }
    s.rows = kBlockRows;
    s.n_slots = 2 * (int64_t)ctx->n_cu;               // workgroups that are on the card at once
    s.blocks = n_rows * g.group / kBlockRows + std::min(batch, n_rows);
    s.extra = 6 * cu;
    s.parts = 8 * cu * g.n_kv_heads;                  // (a block of n units has n partials, and n - 1 units more than one)
    return s;
}

hipError_t launch_attend(chess_ctx* ctx, AttendArgs a, const AttendShape& s, hipStream_t stream)
{
    a.n_slots = (int)s.n_slots;
    const bool list = a.page_ids != nullptr, cap = a.cap_in != 0.f, b16 = ctx->geom.page_size == 16;
    if (s.rows < kBlockRows) {
        if (b16) {
            if (s.rows == 32) return cap ? launch_few<16, 1, true>(ctx, a, list, stream) : launch_few<16, 1, false>(ctx, a, list, stream);
            return cap ? launch_few<16, 2, true>(ctx, a, list, stream) : launch_few<16, 2, false>(ctx, a, list, stream);
        }
        if (s.rows == 32) return cap ? launch_few<32, 1, true>(ctx, a, list, stream) : launch_few<32, 1, false>(ctx, a, list, stream);
        return cap ? launch_few<32, 2, true>(ctx, a, list, stream) : launch_few<32, 2, false>(ctx, a, list, stream);
    }
    a.blocks_most = (int)s.blocks;
    a.extra_most = (int)s.extra;
    a.parts_most = (int)(s.parts / a.n_kv_heads);
    const hipError_t e = launch(b16 ? plan_kernel<16> : plan_kernel<32>, dim3(1), dim3(kPlanThreads), (size_t)a.batch * sizeof(int), stream, a);
    if (e != hipSuccess) return e;
    const bool general = cap || a.slopes != nullptr;
    if (b16) return list ? launch_many<16, true>(ctx, a, s, general, stream) : launch_many<16, false>(ctx, a, s, general, stream);
    return list ? launch_many<32, true>(ctx, a, s, general, stream) : launch_many<32, false>(ctx, a, s, general, stream);
}

}  // namespace chess

// Attention over every page of a ragged batch: which sequence, and which of its splits, a workgroup takes.
#pragma once

#include "decode_device.h"
#include "split_rule.h"

namespace chess {

// Workgroups dealt by length (attention over every page of a ragged batch).  A KV head has n_slots workgroups for all
// the sequences together; a sequence of t tiles takes ceil(t / u) of them, with the smallest tile count u per workgroup, of
// 64 tried, for which the slots suffice.  Lane i holds the i-th of 63 steps from "all slots equally full" to a count that
// certainly fits; the last lane's is one workgroup per sequence (the host calls with n_slots >= batch).  Every workgroup
// computes the same numbers from the lengths in device memory, so a captured launch follows them.
// A workgroup gets at least a tile per wave (u >= NW), and a sequence at most 1.5 x the count at which its own tiles and
// its merge balance (choose_splits knows the longest possible length only): split finer, 16 workgroups' partials of a
// short sequence cost more than its tiles.
// With the same number of workgroups for every sequence the longest one set the time (the waves of the others idle,
// and HBM with them): 64 sequences of 1-8192 tokens, 8 KV heads, 235 us -> 195 us dealt.
// The dealing is a chain before the first request, so it is kept short: equal lengths need no search, a search looks at
// three candidates a step (the slots needed never grow with u), and beyond 64 sequences the waves share them.  Counting all
// 64 candidates sequence by sequence in every wave took 18 us of 512 sequences' launch.  us, fixed splits / every candidate
// counted / as here:
//   8 KV heads,  16 sequences of 1024 tokens   16.4 / 18.0 / 16.3    room for 64K, 8 sequences of 1-1024   11.1 / 14.0 /  8.7
//               64 sequences of 8192 tokens   371.6 / 380.8 / 370.3
//   1 KV head,  512 sequences of 1-1024 tokens 27.4 / 52.7 / 29.7    512 sequences of 1-8192   244.7 / 240.8 / 215.9
// What remains of its cost shows where there is nothing to gain: 0.3 us with equal lengths, 0.5-1.5 us with ragged ones of
// a few tiles, 3-5 us with 512-700 of those.
struct SlotShare { int b, split, n_splits, first, len; };
struct Share { int tiles, most; };                    // of one sequence; 0, 0: a lane without one

__device__ __forceinline__ int slots_of(const Share& q, float inv_u) { return min(1 + (int)((float)(q.tiles - 1) * inv_u), q.most); }

// Inclusive sum over the lanes (row shifts and row broadcasts, no LDS); lane 63 has the total.
template <class T>
__device__ __forceinline__ T lanes_upto(T v)
{
    static_assert(sizeof(T) == 4);
#define CHESS_UPTO(ctrl, rows) v += __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), ctrl, rows, 0xf, false));
    CHESS_UPTO(0x111, 0xf) CHESS_UPTO(0x112, 0xf) CHESS_UPTO(0x114, 0xf) CHESS_UPTO(0x118, 0xf) CHESS_UPTO(0x142, 0xa) CHESS_UPTO(0x143, 0xc)
#undef CHESS_UPTO
    return v;
}

template <class T>
__device__ __forceinline__ T lane_of(T v, int lane)
{
    static_assert(sizeof(T) == 4);
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

// What the waves of a workgroup tell each other where a batch has more than 64 sequences.
template <int NW>
struct DealLds {
    float total[NW];
    int other[NW], c12[3][NW], c3[3][NW];
    int block[kDealMost / 64];                        // workgroups of each 64 sequences
};

// kTokens: of a tile.
template <int B, int NW, int kTokens = kTileTokens>
__device__ __forceinline__ SlotShare share_slots(int slot, int n_slots, int batch, int most, int G, const int32_t* __restrict__ seq_lens,
                                                 int max_pages, int lane, int wave, DealLds<NW>& lds)
{
    const auto len_of = [&](int b) { return min(max(seq_lens[min(b, batch - 1)], 0), max_pages * B); };
    const float per_tile = 18.f / (float)G;           // (1.5 x sqrt(8 tiles / G))
    const auto share_of = [&](int b, int L) {
        const int n = max((L + kTokens - 1) / kTokens, 1);
        const int balanced = max((int)__builtin_amdgcn_sqrtf((float)n * per_tile), 1);
        return b < batch ? Share{n, min(balanced, most)} : Share{0, 0};
    };
    // up to 64 sequences: every wave has them all, one a lane.  More: a wave takes every NW-th block of 64 (the first of
    // them stays in registers, those beyond are read again for every pass, from the cache), and the sums meet in LDS.
    const bool wide = batch > 64;
    const int b00 = wide ? 64 * wave : 0, b_next = wide ? b00 + 64 * NW : batch;
    const int len0 = len_of(b00 + lane);
    const int len_first = len_of(0);
    const Share mine = share_of(b00 + lane, len0);
    const Share some = share_of(0, len_first);
    float total = (float)mine.tiles;                  // (an estimate that orders the candidates: fp32 is enough)
    int other = __ballot(mine.tiles != some.tiles && b00 + lane < batch) != 0;
    for (int b0 = b_next; b0 < batch; b0 += 64 * NW) {
        const int n = share_of(b0 + lane, len_of(b0 + lane)).tiles;
        total += (float)n;
        other |= __ballot(n != some.tiles && b0 + lane < batch) != 0;
    }
    total = lane_of(lanes_upto(total), 63);
    if (wide) {
        if (lane == 0) {
            lds.total[wave] = total;
            lds.other[wave] = other;
        }
        __syncthreads();
        total = 0.f;
        other = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            total += lds.total[w];
            other |= lds.other[w];
        }
    }
    SlotShare s = {-1, 0, 1, 0, 0};
    if (__builtin_amdgcn_readfirstlane(other) == 0) { // all as long: no search (quotients of small whole numbers: exact)
        s.n_splits = min(min((int)((float)n_slots / (float)batch), some.most), (some.tiles + NW - 1) / NW);
        const int b = (int)((float)slot / (float)s.n_splits);
        if (b < batch) {
            s.b = b;
            s.first = b * s.n_splits;
            s.split = slot - s.first;
            s.len = seq_lens[b];
        }
        return s;
    }
    const float lo = fmaxf(total / (float)n_slots, (float)NW), hi = fmaxf(total / fmaxf((float)(n_slots - batch), 1.f), lo);
    const float inv_u = lane == 63 ? 0.f : 1.f / (lo + (hi - lo) * (float)lane * (1.f / 62.f));
    int at = 0;
#pragma unroll
    for (int step = 16, i = 0; step > 0; step >>= 2, ++i) {   // the slots needed never grow with the candidate: 64 -> 16 -> 4 -> 1
        const float i1 = lane_of(inv_u, at + step - 1), i2 = lane_of(inv_u, at + 2 * step - 1), i3 = lane_of(inv_u, at + 3 * step - 1);
        // (two counts in one register: at most n_slots + batch each)
        int c12 = slots_of(mine, i1) | slots_of(mine, i2) << 16, c3 = slots_of(mine, i3);
        for (int b0 = b_next; b0 < batch; b0 += 64 * NW) {
            const Share q = share_of(b0 + lane, len_of(b0 + lane));
            c12 += slots_of(q, i1) | slots_of(q, i2) << 16;
            c3 += slots_of(q, i3);
        }
        c12 = lane_of(lanes_upto(c12), 63);
        c3 = lane_of(lanes_upto(c3), 63);
        if (wide) {
            if (lane == 0) {
                lds.c12[i][wave] = c12;
                lds.c3[i][wave] = c3;
            }
            __syncthreads();
            c12 = c3 = 0;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                c12 += lds.c12[i][w];
                c3 += lds.c3[i][w];
            }
        }
        at += (c12 & 0xffff) <= n_slots ? 0 : (c12 >> 16) <= n_slots ? step : c3 <= n_slots ? 2 * step : 3 * step;
        at = __builtin_amdgcn_readfirstlane(at);
    }
    const float inv = lane_of(inv_u, at);             // (the last candidate always fits)
    int b0 = 0, first = 0, len = len0;
    Share own = mine;
    if (wide) {                                       // the block of 64 the slot falls in
        for (b0 = b00; b0 < batch; b0 += 64 * NW) {
            const int n = lane_of(lanes_upto(slots_of(share_of(b0 + lane, len_of(b0 + lane)), inv)), 63);
            if (lane == 0) lds.block[b0 / 64] = n;
        }
        __syncthreads();
        const int n = 64 * lane < batch ? lds.block[lane] : 0, upto = lanes_upto(n);
        const unsigned long long past = __ballot(upto > slot);
        if (past == 0) return s;
        const int j = __builtin_ctzll(past);
        b0 = 64 * j;
        first = lane_of(upto, j) - lane_of(n, j);
        len = len_of(b0 + lane);
        own = share_of(b0 + lane, len);
    }
    const int n = slots_of(own, inv), upto = first + lanes_upto(n);
    const unsigned long long past = __ballot(upto > slot);
    if (past != 0) {
        const int j = __builtin_ctzll(past);
        s.b = b0 + j;
        s.n_splits = lane_of(n, j);
        s.first = lane_of(upto, j) - s.n_splits;
        s.split = slot - s.first;
        s.len = lane_of(len, j);
    }
    return s;
}

}  // namespace chess

// Paged decode attention over 8-bit pages, a list of them or every page: split-K with an online-softmax merge, as decode.hip does it for bf16.
//
// Work unit: one wave, one tile of 64 tokens (16 KB of keys and values, what 32 tokens are in bf16), all G <= 16 query heads of a KV head.
// Both products run on 16 x 16 x 32 bf16 MFMA tiles with fp32 accumulation: e4m3 bytes times a power of two are bf16 values exactly, so
// the queries stay bf16 and nothing is rounded that the cache has not rounded already.  A lane of group g = lane / 16:
//   S^T[token][head] = K[token][d] . Q^T[d][head]   four products of 16 tokens; its two 16-byte loads of a key row are d = 16 g .. + 15 and
//                                                   64 + 16 g .. + 15, and the contraction runs over d in that order for both operands
//   O^T[d][head]    += V^T[d][token] . P[token][head]   a 16-byte load is tokens 16 g .. + 15 of one d: two contraction steps of 32 tokens
// Row i of product c is token 16 (i / 4) + 4 c + i % 4, so the 16 weights a lane ends up with are those of its own 16 tokens, which lie in
// one page: no weight moves between lanes, and the page's two scales are one number each a lane (the keys' times the softmax scale, the
// values' inside the conversion).  The weights are split into three bf16 parts (24 bits; two parts were the largest error there was).
// Bound: HBM.
#include "deal.h"
#include "quant_device.h"

namespace chess {

constexpr int kQuantTokens = 64;     // of a tile
// The weighted sums and the sums of weights are both kept in units of 2^32: weights reach 1 and there are fewer than 2^31 of them, so that no sum of
// finite values leaves fp32 before it is divided (values reach 448 2^119; the smallest, 2^-73, are normal numbers either way).
constexpr float kSumUnit = 0x1p-32f;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// Eight stored bytes, times a power of two, as a MFMA operand.
__device__ __forceinline__ bf16x8 operand_of(uint32_t lo, uint32_t hi, float scale)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// Where a lane finds its parts of a tile: the physical page its key rows lie in (tokens 16 (m16 / 4) ..), that of its own 16 tokens (16 grp ..), and
// the logical page of these.
struct QuantRef {
    int pk, pv, lv;
};

template <int B>
struct QuantTile {
    uint4 k[4][2];      // [product][half row]
    uint4 v[8];         // [16-row block of d]
    float2 scale;       // of the lane's own page: keys, values
    int nt;             // how many of the lane's own tokens exist (<= 0: none)
};

// A lane's two page slots of tile t: indexes into the list, or logical pages.
template <int B>
struct QuantSlots {
    int k, v;
    __device__ __forceinline__ QuantSlots(int t, int m16, int grp) : k(t * (kQuantTokens / B) + (m16 >> 2) * 16 / B), v(t * (kQuantTokens / B) + grp * 16 / B) {}
};

// Listed pages of tile t at the lane's two places, as stored (an index beyond the list's row is its last entry; which entries count is decided later).
template <int B>
__device__ __forceinline__ int2 quant_ids(int t, const int32_t* ids, int max_sel, int m16, int grp)
{
    const QuantSlots<B> at(t, m16, grp);
    return make_int2(ids[min(at.k, max_sel - 1)], ids[min(at.v, max_sel - 1)]);
}

// Their physical pages.  A list: a bad id, or one behind the list's last, must not become a bad address.  Every page: the entry is read before
// the length is known, and quant_rows replaces those that are beyond it.
template <int B, bool kList>
__device__ __forceinline__ QuantRef quant_pages(int t, const int2& raw, const int32_t* bt_row, int P, int max_pages, int m16, int grp)
{
    const QuantSlots<B> at(t, m16, grp);
    const int lk = kList ? min(max(raw.x, 0), P - 1) : min(at.k, max_pages - 1), lv = kList ? min(max(raw.y, 0), P - 1) : min(at.v, max_pages - 1);
    return QuantRef{bt_row[lk], bt_row[lv], lv};
}

template <int B, bool kList, bool kOnce>
__device__ __forceinline__ void quant_rows(QuantTile<B>& tl, const QuantRef& r, int t, int n_pages, int L, int P, const uint8_t* k_pool,
                                           const uint8_t* v_pool, const float* scales, int H, int h, int m16, int grp)
{
    const QuantSlots<B> at(t, m16, grp);
    int pk = r.pk, pv = r.pv;
    if constexpr (!kList) {                           // (lane 0 has the tile's first page, which exists)
        const int first = __builtin_amdgcn_readfirstlane(r.pk);
        pk = at.k < P ? pk : first;
        pv = at.v < P ? pv : first;
    }
    const int64_t at_k = ((int64_t)pk * H + h) * (B * kHeadDim), at_v = (int64_t)pv * H + h;
    const uint8_t* k_row = k_pool + at_k + ((16 * (m16 >> 2)) % B + (m16 & 3)) * kHeadDim + 16 * grp;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int half = 0; half < 2; ++half) tl.k[c][half] = load_16<kOnce>(k_row + 4 * c * kHeadDim + 64 * half);
    tl.scale = *reinterpret_cast<const float2*>(scales + 2 * at_v);
    const uint8_t* v_row = v_pool + at_v * (B * kHeadDim) + m16 * B + 16 * grp % B;
#pragma unroll
    for (int blk = 0; blk < 8; ++blk) tl.v[blk] = load_16<kOnce>(v_row + blk * 16 * B);
    tl.nt = at.v < n_pages ? (r.lv == P - 1 ? L - r.lv * B : B) - 16 * grp % B : 0;
}

// 2^(score - largest), at most 1.  The score is the rounded product that the largest was chosen by, never one rounded together with the difference: a
// score of 1e9 is rounded by 64 and more, and the largest one's weight would be 2 to the power of its rounding, 0 or infinite instead of 1.
// (Rounded together, errors against 64 bits are a tenth smaller at ordinary scores: 16 sequences of 8-64K 6.7-7.4e-7 where 7.9-8.4e-7.)
__device__ __forceinline__ float weight_of(float score, float largest)
{
#pragma clang fp contract(off)
    return __builtin_amdgcn_exp2f(score - largest);
}

// Online-softmax state of one wave: all G heads of one KV head.
struct QuantAcc {
    bf16x8 qop[4];      // head m16: d = 64 j + 16 grp + 8 i .. + 7 is step 2 j + i; heads >= G are zero columns
    float m_run, l_run;
    f32x4 o[8];

    __device__ __forceinline__ void request(const uint16_t* __restrict__ q_rows, int G, int m16, int grp)
    {
        const uint4* src = reinterpret_cast<const uint4*>(q_rows + (size_t)(m16 < G ? m16 : 0) * kHeadDim) + 2 * grp;
#pragma unroll
        for (int st = 0; st < 4; ++st) qop[st] = as_bf16x8(src[8 * (st >> 1) + (st & 1)]);
    }
    __device__ __forceinline__ void start(int G, int m16)
    {
        const uint32_t keep = m16 < G ? 0xffffffffu : 0u;
#pragma unroll
        for (int st = 0; st < 4; ++st) {
            uint4 v = __builtin_bit_cast(uint4, qop[st]);
            v.x &= keep; v.y &= keep; v.z &= keep; v.w &= keep;
            qop[st] = as_bf16x8(v);
        }
        m_run = kNegBig;
        l_run = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    template <int B>
    __device__ __forceinline__ void process(QuantTile<B>& tl, float scale_log2)
    {
        f32x4 s[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            s[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint4 w = tl.k[c][half];
                s[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand_of(w.x, w.y, 1.f), qop[2 * half], s[c], 0, 0, 0);
                s[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand_of(w.z, w.w, 1.f), qop[2 * half + 1], s[c], 0, 0, 0);
            }
        }
        const float by = tl.scale.x * scale_log2, v_scale = tl.scale.y * kSumUnit;
        float x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = e < tl.nt ? s[e >> 2][e & 3] * by : -INFINITY;
        float tmax = x[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) tmax = fmaxf(tmax, x[e]);
        tmax = fmaxf(tmax, __shfl_xor(tmax, 16));
        tmax = fmaxf(tmax, __shfl_xor(tmax, 32));
        const float m_new = fmaxf(m_run, tmax);
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        m_run = m_new;
        float psum = 0.f;
        bf16x8 p[2][3];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float w = weight_of(x[e], m_new);
            psum += w;
            const __bf16 hi = (__bf16)w;
            const float rest = w - (float)hi;
            const __bf16 mid = (__bf16)rest;
            p[e >> 3][0][e & 7] = hi;
            p[e >> 3][1][e & 7] = mid;
            p[e >> 3][2][e & 7] = (__bf16)(rest - (float)mid);
        }
        l_run = l_run * alpha + psum;
        if (tl.nt < 16) {                             // bytes behind the last token may be anything (NaN among them)
            uint32_t keep[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int n = tl.nt - 4 * i;
                keep[i] = n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
            }
#pragma unroll
            for (int blk = 0; blk < 8; ++blk) {
                tl.v[blk].x &= keep[0]; tl.v[blk].y &= keep[1]; tl.v[blk].z &= keep[2]; tl.v[blk].w &= keep[3];
            }
        }
#pragma unroll
        for (int blk = 0; blk < 8; ++blk) {
            f32x4 acc = o[blk] * alpha;
            const uint4 w = tl.v[blk];
            const bf16x8 v0 = operand_of(w.x, w.y, v_scale), v1 = operand_of(w.z, w.w, v_scale);
#pragma unroll
            for (int part = 0; part < 3; ++part) {
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, p[0][part], acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, p[1][part], acc, 0, 0, 0);
            }
            o[blk] = acc;
        }
    }
};

struct QuantArgs {
    const uint8_t* k_pool;
    const uint8_t* v_pool;
    const float* scales;
    float* out;
    float* ws_acc;
    float* ws_ml;
    int32_t* arrivals;
    float scale_log2;
    int batch;
};
using QuantKernel = void (*)(uint64_t, uint64_t, uint64_t, uint64_t, uint64_t, int, int, int, int, QuantArgs);
using QuantLines = ArgLinesOf<QuantKernel, QuantArgs>;

// Attention over tiles t0, t0 + stride, ... < t_end of one row by one wave.
template <int B, bool kList, bool kOnce>
struct QuantWalk {
    int2 raw_cur, raw_nxt, raw_nn;
    QuantRef rc, rn;
    // what does not wait for lengths
    __device__ __forceinline__ void ask(int t, int stride, const int32_t* ids, int max_sel, const int32_t* bt_row, int max_pages, int m16, int grp)
    {
        if constexpr (kList) {
            raw_cur = quant_ids<B>(t, ids, max_sel, m16, grp);
            raw_nxt = quant_ids<B>(t + stride, ids, max_sel, m16, grp);
        } else {
            rc = quant_pages<B, false>(t, raw_cur, bt_row, 0, max_pages, m16, grp);
            rn = quant_pages<B, false>(t + stride, raw_nxt, bt_row, 0, max_pages, m16, grp);
        }
    }
    __device__ __forceinline__ void run(QuantAcc& acc, int t, int t_end, int stride, int n_pages, int L, int P, const int32_t* ids, int max_sel,
                                        const int32_t* bt_row, int max_pages, const QuantArgs& a, int H, int h, int m16, int grp)
    {
        if (t < t_end) {
            // block-table entries run one tile ahead of the rows, a list's page numbers one tile ahead of those
            if constexpr (kList) {
                rc = quant_pages<B, true>(t, raw_cur, bt_row, P, max_pages, m16, grp);
                rn = quant_pages<B, true>(t + stride, raw_nxt, bt_row, P, max_pages, m16, grp);
                raw_nn = quant_ids<B>(t + 2 * stride, ids, max_sel, m16, grp);
            }
            QuantTile<B> tl;
            for (; t < t_end; t += stride) {
                quant_rows<B, kList, kOnce>(tl, rc, t, n_pages, L, P, a.k_pool, a.v_pool, a.scales, H, h, m16, grp);
                const QuantRef rnn = quant_pages<B, kList>(t + 2 * stride, raw_nn, bt_row, P, max_pages, m16, grp);
                if constexpr (kList) raw_nn = quant_ids<B>(t + 3 * stride, ids, max_sel, m16, grp);
                acc.process(tl, a.scale_log2);
                rc = rn;
                rn = rnn;
            }
        }
        acc.l_run += __shfl_xor(acc.l_run, 16);
        acc.l_run += __shfl_xor(acc.l_run, 32);
        acc.l_run *= kSumUnit;
    }
};

// grid: (n_splits, H_kv, batch), or dealt by length (H_kv, n_slots).  heads: KV heads << 8 | group.
template <int B, int NW, bool kList, bool kDealt = false, bool kOnce = false>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(kList && NW == 4 ? 3 : 2))) void quant_decode_kernel(
    uint64_t seq_lens_at, uint64_t block_table_at, uint64_t q_at, uint64_t page_ids_at, uint64_t n_selected_at, int heads, int max_sel, int max_pages,
    int n_splits, QuantArgs a)
{
    constexpr int PPT = kQuantTokens / B;
    extern __shared__ float lds_f[];                  // DecodeLds<NW>::floats(G)
    __shared__ int lds_last;
    const int G = heads & 255, H = heads >> 8, h = kDealt ? blockIdx.x : blockIdx.y;
    QuantLines lines;
    lines.ask();
    DecodeLds<NW> lds(lds_f, G);
    const int32_t* seq_lens = device_pointer<const int32_t>(seq_lens_at);

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int m16 = lane & 15, grp = lane >> 4;
    int split = blockIdx.x, b = blockIdx.z, ns = n_splits, L_raw;
    size_t part0 = ((size_t)b * H + h) * n_splits;
    if constexpr (kDealt) {
        __shared__ DealLds<NW> deal_lds;
        const SlotShare sh = share_slots<B, NW, kQuantTokens>(blockIdx.y, gridDim.y, a.batch, n_splits, G, seq_lens, max_pages, lane, wave, deal_lds);
        if (sh.b < 0) return;                         // (uniform: nobody waits for a slot without work)
        split = sh.split;
        b = sh.b;
        ns = sh.n_splits;
        L_raw = sh.len;
        part0 = (size_t)h * gridDim.y + sh.first;
    }
    const size_t row = (size_t)b * H + h;
    const int32_t* ids = kList ? device_pointer<const int32_t>(page_ids_at) + row * max_sel : nullptr;
    const int32_t* bt_row = device_pointer<const int32_t>(block_table_at) + (size_t)b * max_pages;
    // tiles are dealt round-robin over splits and waves: the first of a wave is known before the list's length is
    const int stride = ns * NW, t = split + ns * wave;
    if constexpr (!kDealt) L_raw = load_by_lane(seq_lens + b);
    int n_raw = kList ? load_by_lane(device_pointer<const int32_t>(n_selected_at) + row) : 0;
    QuantWalk<B, kList, kOnce> walk;
    walk.ask(t, stride, ids, max_sel, bt_row, max_pages, m16, grp);
    QuantAcc acc;
    acc.request(device_pointer<const uint16_t>(q_at) + ((size_t)b * H * G + (size_t)h * G) * kHeadDim, G, m16, grp);
    requested_by_here();
    if constexpr (!kDealt) L_raw = __builtin_amdgcn_readfirstlane(L_raw);
    if (kList) n_raw = __builtin_amdgcn_readfirstlane(n_raw);
    const int L = min(max(L_raw, 0), max_pages * B);
    const int P = (L + B - 1) / B;
    const int n_pages = P == 0 ? 0 : (kList ? min(max(n_raw, 0), max_sel) : P);

    lines.hold();
    acc.start(G, m16);
    walk.run(acc, t, (n_pages + PPT - 1) / PPT, stride, n_pages, L, P, ids, max_sel, bt_row, max_pages, a, H, h, m16, grp);

    float* out_rows = a.out + ((size_t)b * H * G + (size_t)h * G) * kHeadDim;
    if (!combine_waves<NW>(acc.o, acc.m_run, acc.l_run, lds, G, ns, split, part0, out_rows, a.ws_acc, a.ws_ml)) return;
    if (!arrive_last(a.arrivals + row * kArrivalStride, ns, &lds_last)) return;
    if constexpr (kDealt) {                           // (the same in every lane, which the compiler cannot tell)
        ns = own_reg(__builtin_amdgcn_readfirstlane(ns));
        part0 = own_reg((unsigned)__builtin_amdgcn_readfirstlane((int)part0));
    }
    merge_splits<NW, kDealt ? kMergeDealt : kMergePlain>(G, ns, part0, out_rows, a.ws_acc, a.ws_ml);
}

// The tiles of a batch in a line, sequence after sequence (one without tokens counts for a tile), cut into shares that differ by at most one tile.
// Every wave works it out from the lengths in device memory, 64 sequences a round.
struct TileLine {
    int q, r;                        // a share is q tiles, the first r of them one more
    int b0;                          // the 64 sequences a lane has one of
    int len, tiles, upto;            // of the lane's sequence: tokens, tiles, the line's tiles up to its end

    template <int B>
    __device__ __forceinline__ void read(const int32_t* seq_lens, int batch, int max_pages, int lane)
    {
        len = min(max(seq_lens[min(b0 + lane, batch - 1)], 0), max_pages * B);
        tiles = b0 + lane < batch ? max((len + kQuantTokens - 1) / kQuantTokens, 1) : 0;
    }
    __device__ __forceinline__ int begin_of(int slot) const { return slot * q + min(slot, r); }
    __device__ __forceinline__ int slot_of(int tile) const
    {
        const int wide = r * (q + 1);
        return tile < wide ? tile / (q + 1) : r + (tile - wide) / q;
    }
};

// Attention over every page of a batch: grid (H_kv, slots), each workgroup a share of its KV head's tiles, which may end one sequence, hold several
// whole ones and begin another.  A sequence's parts are one a slot, in slot order, so the partials of sequence b start at the first of its slots
// plus b (its last slot may be the next one's first).
template <int B, int NW, bool kOnce>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2))) void quant_line_kernel(
    uint64_t seq_lens_at, uint64_t block_table_at, uint64_t q_at, uint64_t, uint64_t, int heads, int, int max_pages, int batch, QuantArgs a)
{
    extern __shared__ float lds_f[];                  // DecodeLds<NW>::floats(G)
    __shared__ int lds_last;
    const int G = heads & 255, H = heads >> 8, h = blockIdx.x, slot = blockIdx.y, slots = gridDim.y;
    QuantLines lines;
    lines.ask();
    DecodeLds<NW> lds(lds_f, G);
    const int32_t* seq_lens = device_pointer<const int32_t>(seq_lens_at);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int m16 = lane & 15, grp = lane >> 4;

    TileLine line;
    int total = 0;
    if (batch > 64) {
#pragma unroll 4
        for (line.b0 = 0; line.b0 < batch; line.b0 += 64) {
            line.read<B>(seq_lens, batch, max_pages, lane);
            total += line.tiles;
        }
    } else {
        line.b0 = 0;
        line.read<B>(seq_lens, batch, max_pages, lane);
        total = line.tiles;
    }
    line.upto = lanes_upto(total);
    total = lane_of(line.upto, 63);
    // (a share has a tile for every wave at least)
    const int used = min((int)gridDim.y, (total + NW - 1) / NW);
    if (slot >= used) return;
    line.q = total / used;
    line.r = total - line.q * used;
    int at = line.begin_of(slot);
    const int end = line.begin_of(slot + 1);
    if (at >= end) return;
    if (batch > 64) {                                 // the 64 sequences the share begins in
        total = 0;
        for (line.b0 = 0;; line.b0 += 64) {
            line.read<B>(seq_lens, batch, max_pages, lane);
            line.upto = total + lanes_upto(line.tiles);
            total = lane_of(line.upto, 63);
            if (total > at) break;
            if (line.b0 + 64 >= batch) return;        // (lengths that changed since they were summed end the walk, here and below)
        }
    }
    lines.hold();
    int i = __builtin_ctzll(__ballot(line.upto > at));
    while (line.b0 + i < batch) {
        const int b = line.b0 + i, L = lane_of(line.len, i), tiles = lane_of(line.tiles, i), upto = lane_of(line.upto, i), begin = upto - tiles;
        const int t0 = at - begin, t_end = min(end, upto) - begin;
        const int first = t0 == 0 && t_end == tiles ? slot : line.slot_of(begin), n_splits = t0 == 0 && t_end == tiles ? 1 : line.slot_of(upto - 1) - first + 1;
        const int32_t* bt_row = device_pointer<const int32_t>(block_table_at) + (size_t)b * max_pages;
        const int P = (L + B - 1) / B;
        QuantWalk<B, false, kOnce> walk;
        QuantAcc acc;
        walk.ask(t0 + wave, NW, nullptr, 0, bt_row, max_pages, m16, grp);
        acc.request(device_pointer<const uint16_t>(q_at) + ((size_t)b * H * G + (size_t)h * G) * kHeadDim, G, m16, grp);
        acc.start(G, m16);
        walk.run(acc, t0 + wave, min(t_end, P == 0 ? 0 : t_end), NW, P, L, P, nullptr, 0, bt_row, max_pages, a, H, h, m16, grp);

        float* out_rows = a.out + ((size_t)b * H * G + (size_t)h * G) * kHeadDim;
        const size_t part0 = own_reg((unsigned)(h * (slots + batch) + first + b));
        if (combine_waves<NW>(acc.o, acc.m_run, acc.l_run, lds, G, n_splits, slot - first, part0, out_rows, a.ws_acc, a.ws_ml) &&
            arrive_last(a.arrivals + ((size_t)b * H + h) * kArrivalStride, n_splits, &lds_last))
            merge_splits<NW, kMergeDealt>(G, n_splits, part0, out_rows, a.ws_acc, a.ws_ml);
        at = begin + t_end;
        if (at >= end) return;
        __syncthreads();                              // the next sequence's waves meet in the same LDS
        if (++i == 64) {
            i = 0;
            line.b0 += 64;
            const int before = upto;
            line.read<B>(seq_lens, batch, max_pages, lane);
            line.upto = before + lanes_upto(line.tiles);
        }
    }
}

static size_t quant_lds_bytes(int waves, int group) { return (size_t)(waves * group * kHeadDim + 2 * waves * group) * sizeof(float); }

hipError_t launch_quant_decode(chess_ctx* ctx, const uint16_t* q, const uint8_t* k_pool, const uint8_t* v_pool, const float* scales,
                               const int32_t* block_table, const int32_t* seq_lens, const int32_t* page_ids, const int32_t* n_selected, int batch,
                               int n_splits, int waves, int n_slots, float* out, float* ws_acc, float* ws_ml, int32_t* arrivals, hipStream_t stream)
{
    const Geom& g = ctx->geom;
    const bool dealt = n_slots > 0, line = dealt && waves == 4;   // (every page of a batch: see choose_quant_splits)
    const dim3 grid = dealt ? dim3(g.n_kv_heads, n_slots) : dim3(n_splits, g.n_kv_heads, batch), block(64 * waves);
    const size_t lds = quant_lds_bytes(waves, g.group);
    const int by_page = g.page_size == 16 ? 0 : 1, wide = waves == 8;
    // Pages as a stream where they are more than stays in the 256 MB behind the L2s from one step to the next: us, plain / so, one sequence of 32768
    // tokens, 8 KV heads (67 MB) 17.3 / 18.9, 65536 (134 MB) 30.0 / 28.6, 131072 54.6 / 51.9, 262139 of 4 heads, pages of 32, 56.8 / 53.4; 16 sequences
    // of 8-64K 224 / 218; lists, 96 of 60 pages of 16, 8 heads (188 MB) 40.4 / 37.7, 32 of 108 (113 MB; eight waves) 23.4 / 24.1.
    const bool once = (int64_t)batch * (page_ids ? g.max_sel : g.max_pages) * g.page_size * g.n_kv_heads * 2 * kHeadDim > 128LL << 20;
    // [page size 16 / 32]
    static const QuantKernel lists[2][2] = {{quant_decode_kernel<16, 4, true>, quant_decode_kernel<32, 4, true>},
                                            {quant_decode_kernel<16, 8, true>, quant_decode_kernel<32, 8, true>}};
    static const QuantKernel lists_streamed[2] = {quant_decode_kernel<16, 4, true, false, true>, quant_decode_kernel<32, 4, true, false, true>};
    static const QuantKernel every[2][2][2] = {{{quant_decode_kernel<16, 4, false>, quant_decode_kernel<32, 4, false>},
                                                {quant_decode_kernel<16, 8, false>, quant_decode_kernel<32, 8, false>}},
                                               {{quant_decode_kernel<16, 4, false, false, true>, quant_decode_kernel<32, 4, false, false, true>},
                                                {quant_decode_kernel<16, 8, false, false, true>, quant_decode_kernel<32, 8, false, false, true>}}};
    static const QuantKernel by_length[2][2] = {{quant_decode_kernel<16, 8, false, true>, quant_decode_kernel<32, 8, false, true>},
                                                {quant_decode_kernel<16, 8, false, true, true>, quant_decode_kernel<32, 8, false, true, true>}};
    static const QuantKernel in_line[2][2] = {{quant_line_kernel<16, 4, false>, quant_line_kernel<32, 4, false>},
                                              {quant_line_kernel<16, 4, true>, quant_line_kernel<32, 4, true>}};
    const QuantKernel kern = line ? in_line[once][by_page] : dealt ? by_length[once][by_page] : !page_ids ? every[once][wide][by_page]
                                  : once && !wide ? lists_streamed[by_page] : lists[wide][by_page];
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    return launch(kern, grid, block, lds, stream, (uint64_t)seq_lens, (uint64_t)block_table, (uint64_t)q, (uint64_t)page_ids, (uint64_t)n_selected,
                  g.n_kv_heads << 8 | g.group, g.max_sel, g.max_pages, line ? batch : n_splits,
                  QuantArgs{k_pool, v_pool, scales, out, ws_acc, ws_ml, arrivals, ctx->sm_scale * 1.4426950408889634f, batch});
}

// Four-wave workgroups of attention over every page of a batch that fit on a compute unit.
hipError_t quant_occupancy(int page_size, int group, int* blocks_per_cu)
{
    const QuantKernel kern = page_size == 16 ? quant_line_kernel<16, 4, false> : quant_line_kernel<32, 4, false>;
    return hipOccupancyMaxActiveBlocksPerMultiprocessor(blocks_per_cu, kern, 256, quant_lds_bytes(4, group));
}

}  // namespace chess

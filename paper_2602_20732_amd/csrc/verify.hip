// Drafted tokens against the target's probabilities, with given random numbers.
//
// Draft j (token x_j, drawn from q_j) stands while u_j q_j(x_j) < p_j(x_j).  The token behind the last that stands is drawn from
//   w(v) = max(p(v) - q(v), 0)   where a draft was refused (p(v) without x_j where the draft came without probabilities),  p(v) otherwise,
// as the first v with w(0) + ... + w(v) > u W, W the sum of all (drafts beyond those that may be looked at are dropped, not refused: the draw is from p(v)).
// What a program decides by must not depend on how sums were cut:
// u q is exact in fp64, sums are fp64 over pieces of 1024 that do not depend on the launch, so the same row gives the same token in every batch.
// Each workgroup finds the refused draft for itself (a gather a draft, a wave's ballot), then sums its pieces of the one row that counts;
// the last of a sequence to arrive looks through the pieces' sums, and through the one piece that the token is in.
// Bound: HBM (8 bytes a word of the vocabulary, of one row a sequence) behind the chain start -> token -> probabilities -> row.  Measured, 151936 words: 128
// sequences of 3 drafts 31.5 us, 4.9 TB/s; 32 sequences 13.5; one of 4 drafts 8.2.
#include "chess_internal.h"
#include "split_rule.h"

namespace chess {

constexpr int kVerThreads = 256;
constexpr int kVerStep = 4 * kVerThreads;             // words that a workgroup looks at at a time

// Inclusive sum over the workgroup, in thread order; *all: the whole sum.
__device__ __forceinline__ double sum_upto(double v, double* all)
{
    __shared__ double of_wave[kVerThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int by = 1; by < 64; by *= 2) {
        const double before = __shfl_up(v, by);
        if (lane >= by) v += before;
    }
    __syncthreads();                                  // (the last call's sums have been read)
    if (lane == 63) of_wave[wave] = v;
    __syncthreads();
    double base = 0., sum = 0.;
#pragma unroll
    for (int w = 0; w < kVerThreads / 64; ++w) {
        if (w == wave) base = sum;
        sum += of_wave[w];
    }
    *all = sum;
    return base + v;
}

// The first thread for which `here` holds; kVerThreads if none.
__device__ __forceinline__ int first_thread(bool here)
{
    __shared__ int of_wave[kVerThreads / 64];
    const uint64_t mask = __ballot(here);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = mask ? (int)(threadIdx.x & ~63u) + __builtin_ctzll(mask) : kVerThreads;
    __syncthreads();
    int first = kVerThreads;
#pragma unroll
    for (int w = kVerThreads / 64 - 1; w >= 0; --w) first = of_wave[w] < kVerThreads ? of_wave[w] : first;
    return first;
}
__device__ __forceinline__ int last_thread(bool here)
{
    __shared__ int of_wave[kVerThreads / 64];
    const uint64_t mask = __ballot(here);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = mask ? (int)(threadIdx.x & ~63u) + 63 - __builtin_clzll(mask) : -1;
    __syncthreads();
    int last = -1;
#pragma unroll
    for (int w = 0; w < kVerThreads / 64; ++w) last = max(last, of_wave[w]);
    return last;
}

// The row that the next token is drawn from.
struct DrawRow {
    const float* p;
    const float* q;          // or null
    int without;             // a word that does not count, or -1
    int vocab;
    bool wide;               // 16-byte loads
};

// Weights of words v0 .. v0 + 3; behind the vocabulary 0.  What is no weight (NaN, negative) is 0.
__device__ __forceinline__ void weights(double (&w)[4], const DrawRow& r, int64_t v0)
{
    float p[4] = {}, q[4] = {};
    if (r.wide && v0 + 4 <= r.vocab) {
        const float4 a = *reinterpret_cast<const float4*>(r.p + v0);
        p[0] = a.x; p[1] = a.y; p[2] = a.z; p[3] = a.w;
        if (r.q != nullptr) {
            const float4 b = *reinterpret_cast<const float4*>(r.q + v0);
            q[0] = b.x; q[1] = b.y; q[2] = b.z; q[3] = b.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (v0 + e < r.vocab) {
                p[e] = r.p[v0 + e];
                if (r.q != nullptr) q[e] = r.q[v0 + e];
            }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const double d = (double)p[e] - (double)q[e];
        w[e] = d > 0. && v0 + e != r.without ? d : 0.;
    }
}

// The sum of the weights of [begin, end), by one wave; begin and end (but for the vocabulary's) are multiples of kVerStep.  The order depends on nothing else.
__device__ __forceinline__ double wave_weights(const DrawRow& r, int64_t begin, int64_t end)
{
    const int lane = threadIdx.x & 63;
    double sum = 0.;
    for (int64_t at = begin; at < end; at += kVerStep) {
        double w[kVerStep / 256][4];
#pragma unroll
        for (int i = 0; i < kVerStep / 256; ++i) weights(w[i], r, at + i * 256 + 4 * lane);
#pragma unroll
        for (int i = 0; i < kVerStep / 256; ++i) sum += (w[i][0] + w[i][1]) + (w[i][2] + w[i][3]);
    }
#pragma unroll
    for (int by = 32; by > 0; by /= 2) sum += __shfl_xor(sum, by);
    return sum;
}

// The first word of [begin, end) with a weight at which `before` plus the weights up to it is above `level`; the last with a weight if none is
// (a level next to the whole sum, which was rounded otherwise), -1 if none has one.
__device__ __forceinline__ int find_word(const DrawRow& r, int64_t begin, int64_t end, double before, double level)
{
    __shared__ int found;
    int last = -1;
    for (int64_t at = begin; at < end; at += kVerStep) {
        const int64_t v0 = at + 4 * (int64_t)threadIdx.x;
        double w[4], all;
        weights(w, r, v0);
        const double mine = (w[0] + w[1]) + (w[2] + w[3]), upto = before + sum_upto(mine, &all);
        const int first = first_thread(mine > 0. && upto > level), some = last_thread(mine > 0.);
        if (some >= 0) {
            const int who = first < kVerThreads ? first : some;
            if ((int)threadIdx.x == who) {
                double sum = upto - mine;
                int v = -1, v_last = -1;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    sum += w[e];
                    if (w[e] > 0.) {
                        v_last = (int)v0 + e;
                        if (v < 0 && sum > level) v = v_last;
                    }
                }
                found = first < kVerThreads && v >= 0 ? v : v_last;
            }
            __syncthreads();
            last = found;
        }
        if (first < kVerThreads) break;
        before += all;
    }
    return last;
}

__global__ __launch_bounds__(kVerThreads) void verify_kernel(VerifyArgs a)
{
    __shared__ int flag;
    const int b = blockIdx.y, split = blockIdx.x, lane = threadIdx.x & 63;
    const int start = a.token_start[b], n_new = (int)((unsigned)a.token_start[b + 1] - (unsigned)start);
    const bool any = n_new > 0 && start >= 0 && start <= a.n_rows - n_new;
    const int n = any ? min(n_new - 1, a.most) : 0;
    const float* u = a.uniforms + (int64_t)b * (a.most + 1);
    // the first draft that does not stand
    int stand = n, refused_word = -1;
    for (int j0 = 0; j0 < n; j0 += 64) {
        const int j = j0 + lane;
        bool stands = true;
        int x = -1;
        if (j < n) {
            x = a.tokens[start + 1 + j];
            const bool word = x >= 0 && x < a.vocab;
            const float p = word ? a.target[(int64_t)(start + j) * a.target_stride + x] : 0.f;
            const float q = a.draft == nullptr ? 1.f : word ? a.draft[b * a.draft_seq + j * a.draft_row + x] : 0.f;
            stands = (double)u[j] * (double)q < (double)p;
        }
        const uint64_t mask = __ballot(!stands);
        if (mask != 0) {
            const int at = __builtin_ctzll(mask);
            stand = j0 + at;
            refused_word = __builtin_amdgcn_readlane(x, at);
            break;
        }
    }
    DrawRow r;
    r.p = a.target + (int64_t)(start + stand) * a.target_stride;
    r.q = stand < n && a.draft != nullptr ? a.draft + b * a.draft_seq + stand * a.draft_row : nullptr;
    r.without = stand < n && a.draft == nullptr ? refused_word : -1;
    r.vocab = a.vocab;
    r.wide = ((reinterpret_cast<uintptr_t>(r.p) | reinterpret_cast<uintptr_t>(r.q)) & 15) == 0;

    double* parts = a.parts + (int64_t)b * kVerPieces;
    if (any)
        for (int piece = split * a.per_split + (threadIdx.x >> 6); piece < min((split + 1) * a.per_split, a.n_pieces); piece += kVerThreads / 64) {
            const int64_t begin = (int64_t)piece * a.piece;
            const double sum = wave_weights(r, begin, min(begin + a.piece, (int64_t)a.vocab));
            if (lane == 0) publish_u64(reinterpret_cast<uint64_t*>(parts + piece), (uint64_t)__double_as_longlong(sum));
        }
    if (!arrive_last(a.arrivals + (int64_t)b * kArrivalStride, gridDim.x, &flag)) return;

    int token = -1;
    if (any) {
        __shared__ double base;
        const bool held = (int)threadIdx.x < a.n_pieces;
        const double mine = held ? __longlong_as_double((long long)observe_u64(reinterpret_cast<const uint64_t*>(parts + threadIdx.x))) : 0.;
        double all, upto = sum_upto(mine, &all);
        if (all > 0. && all < INFINITY) {
            const double level = (double)u[a.most] * all;
            const int first = first_thread(mine > 0. && upto > level), some = last_thread(mine > 0.), piece = first < kVerThreads ? first : some;
            if ((int)threadIdx.x == piece) base = upto - mine;
            __syncthreads();
            const int64_t begin = (int64_t)piece * a.piece;
            token = find_word(r, begin, min(begin + a.piece, (int64_t)a.vocab), base, level);
        } else if (stand < n) {                       // a refused draft, and nothing that the target has more of: from the target's own row
            r.q = nullptr;
            r.without = -1;
            double sum = 0.;
            for (int64_t at = 0; at < a.vocab; at += kVerStep) {
                double w[4];
                weights(w, r, at + 4 * (int64_t)threadIdx.x);
                sum += (w[0] + w[1]) + (w[2] + w[3]);
            }
            sum_upto(sum, &all);
            if (all > 0. && all < INFINITY) token = find_word(r, 0, a.vocab, 0., (double)u[a.most] * all);
        }
    }
    for (int j = threadIdx.x; j <= a.most; j += kVerThreads)
        a.out_tokens[(int64_t)b * (a.most + 1) + j] = !any ? -1 : j < stand ? a.tokens[start + 1 + j] : j == stand ? token : -1;
    if (threadIdx.x == 0) {
        a.n_accepted[b] = any ? stand : 0;
        a.lens_after[b] = a.seq_lens[b] - (any ? n_new - 1 - stand : 0);
    }
}

hipError_t launch_verify(chess_ctx* ctx, VerifyArgs a, hipStream_t stream)
{
    // pieces by the vocabulary alone; workgroups of a sequence: as many as fill the card, no more than there are pieces
    a.piece = (int)(cdiv(cdiv(a.vocab, kVerPieces), kVerStep) * kVerStep);
    a.n_pieces = (int)cdiv(a.vocab, a.piece);
    const int64_t want = clampi(4 * (int64_t)ctx->n_cu / a.batch, 1, a.n_pieces);
    a.per_split = (int)cdiv(a.n_pieces, want);
    return launch(verify_kernel, dim3((unsigned)cdiv(a.n_pieces, a.per_split), (unsigned)a.batch), dim3(kVerThreads), 0, stream, a);
}

}  // namespace chess

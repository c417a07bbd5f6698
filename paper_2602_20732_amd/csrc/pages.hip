// The pages of a batch, handed out and taken back on the device: free list -> block tables, token starts, slot map, write list.
//
// map_kernel: with w_b the tokens that sequence b takes, p_b the pages it gains and t_b the pages its tokens lie in, everything follows
// from the inclusive sums over b of the three.  Every workgroup forms them for itself (one load a sequence, sums by lane shifts and LDS),
// so there is no pass between counting and writing; then a group of B lanes takes an entry of the write list: finds its sequence in the
// sums, its page in the free list or the block table, and writes the B slots, the entry and the table.  What is written once a sequence
// (lengths, starts, counts) is one workgroup's; where the lengths or the free count are updated in place, the last one's to arrive.  Sums are capped at kSumCap, above every bound they are compared with: they cannot wrap, and stay ordered.
// Bound: the chain length -> sums -> search -> page -> slots; 8 bytes a token are little.
#include "chess_internal.h"
#include "split_rule.h"

namespace chess {

constexpr int kPageThreads = 256;
constexpr int kSumCap = 0x3fffffff;
constexpr int kFly = 4;              // entries of the write list a group has in hand at a time

__device__ __forceinline__ int capped(int a, int b) { return min(a + b, kSumCap); }

// Inclusive capped sum over the lanes of a wave.
__device__ __forceinline__ int wave_upto(int v)
{
#define CHESS_UPTO(ctrl, rows) v = capped(v, __builtin_amdgcn_update_dpp(0, v, ctrl, rows, 0xf, false));
    CHESS_UPTO(0x111, 0xf) CHESS_UPTO(0x112, 0xf) CHESS_UPTO(0x114, 0xf) CHESS_UPTO(0x118, 0xf) CHESS_UPTO(0x142, 0xa) CHESS_UPTO(0x143, 0xc)
#undef CHESS_UPTO
    return v;
}

// Inclusive capped sums of kSums values a sequence, for the sequences in order: value(b, v) gives them, upto[s][b] takes them.  Every thread
// of the workgroup; the sums can be read afterwards.
template <int kSums, class Value>
__device__ __forceinline__ void sums_upto(int batch, int* upto, Value value)
{
    constexpr int kWaves = kPageThreads / 64;
    __shared__ int of_wave[kSums][kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int before[kSums] = {};
    for (int b0 = 0; b0 < batch; b0 += kPageThreads) {
        const int b = b0 + (int)threadIdx.x;
        int v[kSums] = {};
        if (b < batch) value(b, v);
#pragma unroll
        for (int s = 0; s < kSums; ++s) {
            v[s] = wave_upto(v[s]);
            if (lane == 63) of_wave[s][wave] = v[s];
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < kSums; ++s) {
            int own = before[s];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                if (w < wave) own = capped(own, of_wave[s][w]);
                before[s] = capped(before[s], of_wave[s][w]);
            }
            if (b < batch) upto[s * batch + b] = capped(own, v[s]);
        }
        __syncthreads();
    }
}

// For each of kN numbers i the first of n sums that is above it (the last one is), in lockstep: log2 n dependent LDS reads for all of them.
template <int kN>
__device__ __forceinline__ void first_above(int (&at)[kN], const int* upto, int n, const int (&i)[kN])
{
#pragma unroll
    for (int x = 0; x < kN; ++x) at[x] = 0;
    for (int step = 1 << (31 - __builtin_clz(n)); step > 0; step >>= 1)
#pragma unroll
        for (int x = 0; x < kN; ++x) {
            const int to = at[x] + step;
            if (upto[min(to, n) - 1] <= i[x] && to < n) at[x] = to;
        }
}

// How many sequences come before the first that does not fit (fits() never holds again behind that one).
template <class Fits>
__device__ __forceinline__ int served(int batch, Fits fits)
{
    __shared__ int cut;
    if (threadIdx.x == 0) cut = batch;
    __syncthreads();
    for (int b = threadIdx.x; b < batch; b += kPageThreads)
        if (!fits(b)) {
            atomicMin(&cut, b);
            break;
        }
    __syncthreads();
    return cut;
}

// Whether this workgroup writes what is written once a sequence: where lengths or the free count are updated in place, the last to arrive, when
// nobody reads them any more; otherwise any will do.
__device__ __forceinline__ bool writes_rows(bool in_place, int32_t* arrivals)
{
    __shared__ int flag;
    if (in_place && gridDim.x > 1) return arrive_last(arrivals, gridDim.x, &flag);
    __syncthreads();
    return blockIdx.x == 0;
}

template <int B>
__global__ __launch_bounds__(kPageThreads) void map_kernel(MapArgs a)
{
    extern __shared__ int upto[];                     // [3][batch]: tokens, pages gained, pages touched; then [batch] lengths
    __shared__ int n_refused;
    const int batch = a.batch, n_free = max(*a.n_free, 0);
    if (threadIdx.x == 0) n_refused = 0;
    const int *tokens = upto, *gained = upto + batch, *touched = upto + 2 * batch;
    int* held = upto + 3 * batch;
    sums_upto<3>(batch, upto, [&](int b, int (&v)[3]) {
        const int64_t L = a.seq_lens[b], n = a.new_lens[b];
        held[b] = (int)L;
        if (L < 0 || n <= 0 || L + n > min((int64_t)a.max_pages * B, (int64_t)INT32_MAX - B)) return;
        v[0] = (int)min(n, (int64_t)kSumCap);
        v[1] = (int)((L + n + B - 1) / B - (L + B - 1) / B);
        v[2] = (int)((L + n - 1) / B - L / B + 1);
    });
    const int cut = served(batch, [&](int b) { return tokens[b] <= a.max_tokens && gained[b] <= n_free; });
    const int n_writes = cut > 0 ? touched[cut - 1] : 0;

    const int j = threadIdx.x % B, step = gridDim.x * (kPageThreads / B);
    for (int i0 = (blockIdx.x * kPageThreads + threadIdx.x) / B; i0 < n_writes; i0 += step * kFly) {
        // (kFly entries at once: each is a search and two round trips)
        int4 entry[kFly];
        int32_t* table_at[kFly];
        bool is_new[kFly];
        int i_of[kFly], b_of[kFly];
#pragma unroll
        for (int x = 0; x < kFly; ++x) i_of[x] = min(i0 + x * step, n_writes - 1);
        first_above(b_of, touched, cut, i_of);
#pragma unroll
        for (int x = 0; x < kFly; ++x) {
            const int i = i_of[x], b = b_of[x];
            const int token0 = b > 0 ? tokens[b - 1] : 0, gained0 = b > 0 ? gained[b - 1] : 0, touched0 = b > 0 ? touched[b - 1] : 0;
            const int L = held[b], after = L + tokens[b] - token0, had = (L + B - 1) / B;
            const int page = L / B + i - touched0, begin = max(L, page * B);
            table_at[x] = a.block_table + (size_t)b * a.max_pages + page;
            is_new[x] = page >= had;
            const int32_t* from = is_new[x] ? a.free_pages + (n_free - 1 - (gained0 + page - had)) : table_at[x];
            entry[x] = make_int4(*from, token0 + begin - L, begin % B, min(after, page * B + B) - begin);
        }
#pragma unroll
        for (int x = 0; x < kFly; ++x) {
            const int i = i0 + x * step;
            if (i >= n_writes) break;
            if (a.slots != nullptr && j < entry[x].w) a.slots[entry[x].y + j] = (int64_t)entry[x].x * B + entry[x].z + j;
            if (j == 0) {
                a.writes[i] = entry[x];
                if (is_new[x]) *table_at[x] = entry[x].x;
            }
        }
    }

    if (!writes_rows(a.in_place, a.arrivals)) return;
    for (int b = threadIdx.x; b < batch; b += kPageThreads) {
        const int upto_b = cut > 0 ? tokens[min(b, cut - 1)] : 0;
        const int got = b < cut ? upto_b - (b > 0 ? tokens[b - 1] : 0) : 0;
        if (a.new_lens[b] > 0 && got == 0) atomicAdd(&n_refused, 1);
        a.lens_after[b] = held[b] + got;
        a.token_start[b + 1] = upto_b;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        const int taken = cut > 0 ? gained[cut - 1] : 0;
        a.token_start[0] = 0;
        a.counts[0] = cut > 0 ? tokens[cut - 1] : 0;
        a.counts[1] = n_writes;
        a.counts[2] = taken;
        a.counts[3] = n_refused;
        *a.n_left = n_free - taken;
    }
}

// The pages of the sequences that ended, behind what the free list holds.  One thread an entry; lengths and the count by one workgroup, as above.
template <int B>
__global__ __launch_bounds__(kPageThreads) void release_kernel(ReleaseArgs a)
{
    extern __shared__ int upto[];                     // [batch]: pages pushed
    const int batch = a.batch, n_free = max(*a.n_free, 0);
    sums_upto<1>(batch, upto, [&](int b, int (&v)[1]) {
        if (a.done[b] != 0) v[0] = (int)min(((int64_t)max(a.seq_lens[b], 0) + B - 1) / B, (int64_t)a.max_pages);
    });
    const int cut = served(batch, [&](int b) { return upto[b] <= a.capacity - n_free; });
    const int total = cut > 0 ? upto[cut - 1] : 0;
    for (int i = blockIdx.x * kPageThreads + threadIdx.x; i < total; i += gridDim.x * kPageThreads) {
        int b[1];
        first_above(b, upto, cut, {i});
        a.free_pages[n_free + i] = a.block_table[(size_t)b[0] * a.max_pages + i - (b[0] > 0 ? upto[b[0] - 1] : 0)];
    }
    if (!writes_rows(a.in_place, a.arrivals)) return;
    for (int b = threadIdx.x; b < batch; b += kPageThreads) a.lens_after[b] = b < cut && a.done[b] != 0 ? 0 : a.seq_lens[b];
    if (threadIdx.x == 0) *a.n_left = n_free + total;
}

hipError_t launch_map(chess_ctx* ctx, const MapArgs& a, hipStream_t stream)
{
    const int B = ctx->geom.page_size;
    const unsigned n = (unsigned)clampi(cdiv(most_writes(a.max_tokens, a.batch, B), kFly * (kPageThreads / B)), 1, a.in_place ? 128 : 1024);
    const size_t lds = (size_t)a.batch * 4 * sizeof(int);
    const auto kern = B == 16 ? map_kernel<16> : map_kernel<32>;
    if (lds > 48 * 1024) {                            // (with what is static, 64 KB are not enough)
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    return launch(kern, dim3(n), dim3(kPageThreads), lds, stream, a);
}

hipError_t launch_release(chess_ctx* ctx, const ReleaseArgs& a, hipStream_t stream)
{
    const int B = ctx->geom.page_size;
    const unsigned n = (unsigned)clampi(cdiv((int64_t)a.batch * a.max_pages, 16 * kPageThreads), 1, 64);
    const size_t lds = (size_t)a.batch * sizeof(int);
    return launch(B == 16 ? release_kernel<16> : release_kernel<32>, dim3(n), dim3(kPageThreads), lds, stream, a);
}

}  // namespace chess

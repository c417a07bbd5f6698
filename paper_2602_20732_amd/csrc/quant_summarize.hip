// Key summaries (Sec. 3.1, Eq. 1-2) of 8-bit pages: page vector = scale / n times the sum of the page's e4m3 rows.
//
// e4m3 values are multiples of 2^-9 up to 448, so the sum of up to 32 of them has 23 bits: it is exact in fp32, in whatever order it is
// formed, and times a power of two still is.  A full page's mean is that number times scale / B; a partial one's is divided in fp64 and
// rounded once, as the summaries of bf16 pages are.
// quant_summarize_kernel: one workgroup owns one (sequence, KV head, grid); 8 lanes stream a page, 16 dims a lane (a row is 128 bytes).  Chunk
// and grid vectors as there.
// Bound: HBM, read and written (a fp32 vector is a quarter of a page of 16).  us, 8 sequences of 30-131K, 8 KV heads, pages of 16, fp32 vectors / 2
// of 196-222K, 4 heads, pages of 32, bf16 / 3 of 700-2161, 8 heads, of 32, bf16:
//   256 threads, 16 rows in flight   182 / 56 / 14.9      512 threads, 8 / 16 rows   180 / 53 / 10.1    182 / 56 / 9.9
//   1024 threads, 8 rows             197 / 61 / 9.9       512, 8, rows as a stream   180 / 49 / 11.1 (hence kOnce: see launch_all)
// The first is 4.8 to 5.2 TB/s, read and written, from card to card (a copy of 2 GiB: 4.8).  Vectors stored as a stream: 240 where 169 without.
#include "quant_device.h"
#include "split_rule.h"
#include "summary_device.h"

namespace chess {

// Eight dims of a row added to their sums.
__device__ __forceinline__ void add_bytes(float (&acc)[8], uint32_t a, uint32_t b)
{
    const f32x2 v[4] = {__builtin_amdgcn_cvt_pk_f32_fp8((int)a, false), __builtin_amdgcn_cvt_pk_f32_fp8((int)a, true),
                        __builtin_amdgcn_cvt_pk_f32_fp8((int)b, false), __builtin_amdgcn_cvt_pk_f32_fp8((int)b, true)};
#pragma unroll
    for (int i = 0; i < 4; ++i) { acc[2 * i] += v[i].x; acc[2 * i + 1] += v[i].y; }
}

// The mean of n of a page's rows from their sum, as a vector stores it: eight dims.
template <int B, class T>
__device__ __forceinline__ Row8<T> mean_of_rows(const float (&sum)[8], float scale, int n)
{
    double mean[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) mean[i] = n == B ? (double)(sum[i] * (scale * (1.f / B))) : (double)sum[i] * (double)scale / (double)n;
    Row8<T> r;
    r.set(mean);
    return r;
}

constexpr int kSumThreads = 512;
constexpr int kSumRows = 8;                           // rows of a page in flight
template <int B, class T, bool kOnce>
__global__ __launch_bounds__(kSumThreads) void quant_summarize_kernel(const uint8_t* __restrict__ k_pool, const float* __restrict__ scales,
                                                              const int32_t* __restrict__ block_table, const int32_t* __restrict__ seq_lens,
                                                              const int32_t* __restrict__ from_page, int recent, Geom g, T* __restrict__ pages,
                                                              T* __restrict__ chunks, T* __restrict__ grids)
{
    extern __shared__ float lds_f[];                  // [n_c * n_g][128] page vectors, then [n_g][128] chunk vectors, as stored
    T* lds = reinterpret_cast<T*>(lds_f);
    const int b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x;
    const int L = min(seq_lens[b], g.max_pages * B);
    if (L <= 0) return;
    const int P = (L + B - 1) / B;
    const int nc = (P + g.n_c - 1) / g.n_c, ng = (nc + g.n_g - 1) / g.n_g;
    // recent > 0: only the last `recent` pages are new; the grid's workgroups count back from the last grid
    const int gk = recent > 0 ? ng - 1 - (int)blockIdx.x : (int)blockIdx.x;
    if (gk >= ng || gk < 0) return;
    const int fp = max(recent > 0 ? P - recent : from_page != nullptr ? from_page[b] : 0, 0);
    const int ppg = g.n_c * g.n_g;
    if (gk < fp / ppg) return;                        // every unit of this grid is older
    const int fc = fp / g.n_c;
    const int p_lo = gk * ppg, p_hi = min(P, p_lo + ppg);
    const int c_lo = gk * g.n_g, c_hi = min(nc, c_lo + g.n_g);
    const size_t row = (size_t)b * g.n_kv_heads + h;
    T* pg = pages + row * g.max_pages * kHeadDim;
    T* cg = chunks + row * g.max_chunks * kHeadDim;
    T* gg = grids + row * g.max_grids * kHeadDim;
    T* lds_chunk = lds + (size_t)ppg * kHeadDim;

    const int grp = tid >> 3, ln = tid & 7;
    for (int j = p_lo + grp; j < p_hi; j += kSumThreads / 8) {
        T* dst = lds + (size_t)(j - p_lo) * kHeadDim + ln * 16;
        T* own = pg + (size_t)j * kHeadDim + ln * 16;
        Row8<T> mean[2];
        if (j >= fp) {
            const int64_t ph = (int64_t)block_table[(size_t)b * g.max_pages + j] * g.n_kv_heads + h;
            const int n = j == P - 1 ? L - j * B : B;
            const uint8_t* src = k_pool + ph * (B * kHeadDim) + ln * 16;
            const float scale = scales[2 * ph];
            float lo[8] = {}, hi[8] = {};
#pragma unroll
            for (int t0 = 0; t0 < B; t0 += kSumRows) {
                uint4 r[kSumRows];
#pragma unroll
                for (int t = 0; t < kSumRows; ++t) r[t] = load_16<kOnce>(src + min(t0 + t, n - 1) * kHeadDim);   // (rows past the last token repeat it and are not added)
#pragma unroll
                for (int t = 0; t < kSumRows; ++t)
                    if (t0 + t < n) {
                        add_bytes(lo, r[t].x, r[t].y);
                        add_bytes(hi, r[t].z, r[t].w);
                    }
            }
            mean[0] = mean_of_rows<B, T>(lo, scale, n);
            mean[1] = mean_of_rows<B, T>(hi, scale, n);
            mean[0].store(own);
            mean[1].store(own + 8);
        } else if (j / g.n_c >= fc) {                 // unchanged page whose chunk is being refreshed
            mean[0].load(own);
            mean[1].load(own + 8);
        } else {
            continue;
        }
        mean[0].store(dst);
        mean[1].store(dst + 8);
    }
    __syncthreads();
    units_above<T, kSumThreads>(lds, lds_chunk, g, gk, P, p_lo, c_lo, c_hi, fc, cg, gg, tid);
}

// The last pages of every sequence, as summarize_recent_kernel does it for bf16: 16 lanes a page, 8 dims a lane.
// shape: recent | n_c << 5 | n_g << 10 | KV heads << 15.
template <int B, class T>
__global__ __launch_bounds__(256) void quant_recent_kernel(uint64_t seq_lens_at, uint64_t block_table_at, uint64_t k_pool_at, uint64_t pages_at,
                                                           int max_pages, int shape, int rows, int max_chunks, uint32_t inv_nc, uint32_t inv_ng,
                                                           int max_grids, uint64_t scales_at)
{
    refresh_recent<B, T>(seq_lens_at, block_table_at, pages_at, max_pages, shape, rows, max_chunks, inv_nc, inv_ng, max_grids,
                         [&](int64_t block, int n, int ln) {
        const uint2* src = reinterpret_cast<const uint2*>(device_pointer<const uint8_t>(k_pool_at) + block * (B * kHeadDim)) + ln;
        const float scale = device_pointer<const float>(scales_at)[2 * block];
        uint2 r[B];
        float sum[8] = {};
#pragma unroll
        for (int t = 0; t < B; ++t) r[t] = src[min(t, n - 1) * 16];                  // (rows past the last token repeat it and are not added)
#pragma unroll
        for (int t = 0; t < B; ++t)
            if (t < n) add_bytes(sum, r[t].x, r[t].y);
        return mean_of_rows<B, T>(sum, scale, n);
    });
}

template <int B, class T>
static hipError_t launch_all(chess_ctx* ctx, const uint8_t* k_pool, const float* scales, const int32_t* block_table, const int32_t* seq_lens,
                             int batch, const int32_t* from_page, int recent, void* pages, void* chunks, void* grids, hipStream_t stream)
{
    const Geom& g = ctx->geom;
    if (recent > 0 && fits_recent(g, recent))
        return launch(quant_recent_kernel<B, T>, dim3(g.n_kv_heads, batch), dim3(256), recent_lds_bytes(g, recent, sizeof(T)), stream, (uint64_t)seq_lens,
                      (uint64_t)block_table, (uint64_t)k_pool, (uint64_t)pages, g.max_pages, recent | g.n_c << 5 | g.n_g << 10 | g.n_kv_heads << 15,
                      ctx->cfg.max_batch * g.n_kv_heads, g.max_chunks, g.inv_nc, g.inv_ng, g.max_grids, (uint64_t)scales);
    const int ppg = g.n_c * g.n_g;
    const size_t lds = (size_t)(ppg + g.n_g) * kHeadDim * sizeof(T);
    const int span = recent > 0 ? (int)recent_grids(recent, ppg, g.max_grids) : g.max_grids;
    // rows as a stream once they are more than the L2s hold (8 x 4 MB); fewer may still be there from the store that wrote them
    const bool once = (int64_t)batch * g.max_pages * g.n_kv_heads * B * kHeadDim > 32LL << 20;
    const auto kern = once ? quant_summarize_kernel<B, T, true> : quant_summarize_kernel<B, T, false>;
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    return launch(kern, dim3(span, g.n_kv_heads, batch), dim3(kSumThreads), lds, stream, k_pool, scales, block_table, seq_lens, from_page, recent, g,
                  static_cast<T*>(pages), static_cast<T*>(chunks), static_cast<T*>(grids));
}

hipError_t launch_quant_summarize(chess_ctx* ctx, const uint8_t* k_pool, const float* scales, const int32_t* block_table,
                                  const int32_t* seq_lens, int batch, const int32_t* from_page, int recent, void* pages, void* chunks,
                                  void* grids, hipStream_t stream)
{
    const bool bf16 = ctx->cfg.summary_dtype == CHESS_SUMMARY_BF16;
    const auto go = ctx->geom.page_size == 16 ? (bf16 ? launch_all<16, uint16_t> : launch_all<16, float>)
                                              : (bf16 ? launch_all<32, uint16_t> : launch_all<32, float>);
    return go(ctx, k_pool, scales, block_table, seq_lens, batch, from_page, recent, pages, chunks, grids, stream);
}

}  // namespace chess

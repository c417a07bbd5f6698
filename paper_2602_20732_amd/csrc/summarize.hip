// Hierarchical key summaries (Sec. 3.1): page vector = mean of the page's key rows (Eq. 1),
// chunk / grid vector = mean of the child vectors that exist (Eq. 2).
//
// One workgroup owns one (sequence, KV head, grid).  A 16-lane group streams one page: every lane
// issues 128-bit loads of 8 consecutive dims of one token row, so one wave instruction covers four
// 256-byte rows.  Each lane adds its 8 columns over the tokens in token order in fp64, so the sum
// is the same number whatever the launch shape; the mean is rounded to fp32 once.  Page vectors of
// the grid stay in LDS, chunk and grid means are formed from them without re-reading HBM.
#include "split_rule.h"
#include "summary_device.h"

namespace chess {

// T = storage type of the summaries (float, or bf16 bits: each stored mean is the fp32 mean rounded to nearest-even
// bf16, and a parent averages its children as they are stored)
template <int B, class T>
__global__ __launch_bounds__(256) void summarize_kernel(const uint16_t* __restrict__ k_pool,
                                                        const int32_t* __restrict__ block_table,
                                                        const int32_t* __restrict__ seq_lens,
                                                        const int32_t* __restrict__ from_page, int recent, Geom g,
                                                        T* __restrict__ pages, T* __restrict__ chunks,
                                                        T* __restrict__ grids)
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
    int fp = recent > 0 ? P - recent : (from_page ? from_page[b] : 0);
    fp = fp < 0 ? 0 : fp;
    const int ppg = g.n_c * g.n_g;
    if (gk < fp / ppg) return;                        // every unit of this grid is older than from_page
    const int fc = fp / g.n_c;
    const int p_lo = gk * ppg, p_hi = min(P, p_lo + ppg);
    const int c_lo = gk * g.n_g, c_hi = min(nc, c_lo + g.n_g);
    const size_t row = (size_t)b * g.n_kv_heads + h;
    T* pg = pages + row * g.max_pages * kHeadDim;
    T* cg = chunks + row * g.max_chunks * kHeadDim;
    T* gg = grids + row * g.max_grids * kHeadDim;
    T* lds_chunk = lds + (size_t)ppg * kHeadDim;

    const int grp = tid >> 4, ln = tid & 15;
    for (int j = p_lo + grp; j < p_hi; j += 16) {
        T* dst = lds + (size_t)(j - p_lo) * kHeadDim + ln * 8;
        Row8<T> r8;
        if (j >= fp) {
            const int64_t phys = block_table[(size_t)b * g.max_pages + j];
            const int n = (j == P - 1) ? L - j * B : B;
            const uint4* src = reinterpret_cast<const uint4*>(k_pool + ((phys * g.n_kv_heads + h) * B) * kHeadDim) + ln;
            double acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (n == B) {
#pragma unroll
                for (int t0 = 0; t0 < B; t0 += 16) {
                    uint4 r[16];
#pragma unroll
                    for (int t = 0; t < 16; ++t) r[t] = src[(t0 + t) * 16];
#pragma unroll
                    for (int t = 0; t < 16; ++t) add_row(acc, r[t]);
                }
            } else {
                for (int t = 0; t < n; ++t) add_row(acc, src[t * 16]);
            }
            const double dn = (double)n;
            double mean[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) mean[i] = acc[i] / dn;
            r8.set(mean);
            r8.store(pg + (size_t)j * kHeadDim + ln * 8);
        } else if (j / g.n_c >= fc) {                 // unchanged page whose chunk is being refreshed
            r8.load(pg + (size_t)j * kHeadDim + ln * 8);
        } else {
            continue;
        }
        r8.store(dst);
    }
    __syncthreads();

    units_above<T>(lds, lds_chunk, g, gk, P, p_lo, c_lo, c_hi, fc, cg, gg, tid);
}

// The same for the last few pages of every sequence (the per-step refresh, the catch-up before a reselection): one workgroup per
// (sequence, KV head), a 16-lane group per page and per unchanged page or chunk that a refreshed chunk or grid still averages, so
// everything is requested in two round trips behind the length (block-table entries, siblings; key rows) and the sums meet in LDS
// once a level.  The kernel above walks a grid's pages sixteen at a time and asks for an unchanged chunk when it comes to it.
// Bound: that chain.  us, 8 KV heads, sixteen draws of lengths of 8-16K, the kernel above / this one, 1 page, 10 and 16: 96 sequences 13.6 /
// 6.6, 23.9 / 12.4, 29.3 / 15.6; 32 11.0 / 5.3, 12.0 / 6.8, 15.3 / 8.3; one 5.5 / 4.2, 6.2 / 4.7, 7.4 / 5.1; pages of 32, 96 sequences 20.9 / 8.2,
// 38.6 / 18.8, 49.6 / 24.5 (all rows of a page at once: 12.0, 20.4, 26.8); 32 18.3 / 6.9, 20.5 / 9.3, 26.9 / 11.9; one 7.1 / 5.3, 8.7 / 6.0,
// 10.2 / 6.8.  With every last page full, where the kernel above is at its best: 96 11.6 / 8.5 (13.6 at once), 24.2 / 19.2, 35.1 / 25.0.
// shape: recent | n_c << 5 | n_g << 10 | KV heads << 15.  The arguments up to inv_ng are preloaded (see build.py).
template <int B, class T>
__global__ __launch_bounds__(256) void summarize_recent_kernel(uint64_t seq_lens_at, uint64_t block_table_at, uint64_t k_pool_at, uint64_t pages_at,
                                                               int max_pages, int shape, int rows, int max_chunks, uint32_t inv_nc,
                                                               uint32_t inv_ng, int max_grids)
{
    refresh_recent<B, T>(seq_lens_at, block_table_at, pages_at, max_pages, shape, rows, max_chunks, inv_nc, inv_ng, max_grids,
                         [&](int64_t block, int n, int ln) {
        const uint4* src = reinterpret_cast<const uint4*>(device_pointer<const uint16_t>(k_pool_at) + (block * B) * kHeadDim) + ln;
        double acc[8] = {0, 0, 0, 0, 0, 0, 0, 0}, mean[8];
        // (sixteen at a time: 32 rows of a page at once are 172 registers, two workgroups to a compute unit)
#pragma unroll
        for (int t0 = 0; t0 < B; t0 += 16) {
            uint4 r[16];
#pragma unroll
            for (int t = 0; t < 16; ++t) r[t] = src[min(t0 + t, n - 1) * 16];      // (rows past the last token repeat it and are not added)
#pragma unroll
            for (int t = 0; t < 16; ++t)
                if (t0 + t < n) add_row(acc, r[t]);
        }
        const double dn = (double)n;
#pragma unroll
        for (int i = 0; i < 8; ++i) mean[i] = acc[i] / dn;
        Row8<T> mean8;
        mean8.set(mean);
        return mean8;
    });
}

static hipError_t launch_recent(chess_ctx* ctx, const uint16_t* k_pool, const int32_t* block_table, const int32_t* seq_lens, int batch, int recent,
                                void* pages, hipStream_t stream)
{
    const Geom& g = ctx->geom;
    const bool bf16 = ctx->cfg.summary_dtype == CHESS_SUMMARY_BF16;
    const size_t lds = recent_lds_bytes(g, recent, bf16 ? sizeof(uint16_t) : sizeof(float));
    const auto kern = bf16 ? (g.page_size == 16 ? summarize_recent_kernel<16, uint16_t> : summarize_recent_kernel<32, uint16_t>)
                           : (g.page_size == 16 ? summarize_recent_kernel<16, float> : summarize_recent_kernel<32, float>);
    return launch(kern, dim3(g.n_kv_heads, batch), dim3(256), lds, stream, (uint64_t)seq_lens, (uint64_t)block_table, (uint64_t)k_pool, (uint64_t)pages,
                  g.max_pages, recent | g.n_c << 5 | g.n_g << 10 | g.n_kv_heads << 15, ctx->cfg.max_batch * g.n_kv_heads, g.max_chunks, g.inv_nc,
                  g.inv_ng, g.max_grids);
}

hipError_t launch_summarize(chess_ctx* ctx, const uint16_t* k_pool, const int32_t* block_table,
                            const int32_t* seq_lens, int batch, const int32_t* from_page, int recent,
                            void* pages, void* chunks, void* grids, hipStream_t stream)
{
    const Geom& g = ctx->geom;
    // (at its least favourable, one sequence whose last page is full, the kernel above and this one, 16 pages: of 32 8.0 / 6.8 us, of 16 6.0 / 5.1;
    // hierarchies of 4 x 4, where a grid is one trip for it, 5.9 / 7.1 and 4.7 / 5.3, but 8.4 / 7.1 and 5.4 / 5.4 over all lengths)
    if (recent > 0 && fits_recent(g, recent))
        return launch_recent(ctx, k_pool, block_table, seq_lens, batch, recent, pages, stream);
    const bool bf16 = ctx->cfg.summary_dtype == CHESS_SUMMARY_BF16;
    const size_t lds = (size_t)(g.n_c * g.n_g + g.n_g) * kHeadDim * (bf16 ? sizeof(uint16_t) : sizeof(float));
    const int ppg = g.n_c * g.n_g;
    const int span = recent > 0 ? (int)recent_grids(recent, ppg, g.max_grids) : g.max_grids;
    const dim3 grid(span, g.n_kv_heads, batch), block(256);
    const void* kern = bf16 ? (g.page_size == 16 ? reinterpret_cast<const void*>(summarize_kernel<16, uint16_t>)
                                                 : reinterpret_cast<const void*>(summarize_kernel<32, uint16_t>))
                            : (g.page_size == 16 ? reinterpret_cast<const void*>(summarize_kernel<16, float>)
                                                 : reinterpret_cast<const void*>(summarize_kernel<32, float>));
    if (lds > 64 * 1024) {
        hipError_t e = hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    if (bf16) {
        auto k = g.page_size == 16 ? summarize_kernel<16, uint16_t> : summarize_kernel<32, uint16_t>;
        return launch(k, grid, block, lds, stream, k_pool, block_table, seq_lens, from_page, recent, g,
                      static_cast<uint16_t*>(pages), static_cast<uint16_t*>(chunks), static_cast<uint16_t*>(grids));
    }
    auto k = g.page_size == 16 ? summarize_kernel<16, float> : summarize_kernel<32, float>;
    return launch(k, grid, block, lds, stream, k_pool, block_table, seq_lens, from_page, recent, g,
                  static_cast<float*>(pages), static_cast<float*>(chunks), static_cast<float*>(grids));
}

}  // namespace chess

// Key summaries (Sec. 3.1, Eq. 1-2) of 8-bit pages: page vector = scale / n times the sum of the page's e4m3 rows.
//
// e4m3 values are multiples of 2^-9 up to 448, so the sum of up to 32 of them has 23 bits: it is exact in fp32, in whatever order it is
// formed, and times a power of two still is.  A full page's mean is that number times scale / B; a partial one's is divided in fp64 and
// rounded once, as the summaries of bf16 pages are.
// One workgroup owns one (sequence, KV head, grid); 8 lanes stream a page, 16 dims a lane (a row is 128 bytes).  Chunk and grid vectors as there.
// Bound: HBM (one byte an element).
#include <algorithm>

#include "quant_device.h"
#include "summary_device.h"

namespace chess {

// 16 dims of a row added to their sums.
__device__ __forceinline__ void add_bytes(float (&acc)[16], const uint4& r)
{
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
        acc[4 * i] += lo.x; acc[4 * i + 1] += lo.y; acc[4 * i + 2] += hi.x; acc[4 * i + 3] += hi.y;
    }
}

// The mean of n of a page's rows from their sum, as a vector stores it: 16 dims.
template <int B, class T>
__device__ __forceinline__ void put_means(Row8<T> (&to)[2], const float (&sum)[16], float scale, int n)
{
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        double mean[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = sum[8 * half + i];
            mean[i] = n == B ? (double)(s * (scale * (1.f / B))) : (double)s * (double)scale / (double)n;
        }
        to[half].set(mean);
    }
}

template <int B, class T>
__global__ __launch_bounds__(256) void quant_summarize_kernel(const uint8_t* __restrict__ k_pool, const float* __restrict__ scales,
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
    for (int j = p_lo + grp; j < p_hi; j += 32) {
        T* dst = lds + (size_t)(j - p_lo) * kHeadDim + ln * 16;
        T* own = pg + (size_t)j * kHeadDim + ln * 16;
        Row8<T> mean[2];
        if (j >= fp) {
            const int64_t ph = (int64_t)block_table[(size_t)b * g.max_pages + j] * g.n_kv_heads + h;
            const int n = j == P - 1 ? L - j * B : B;
            const uint4* src = reinterpret_cast<const uint4*>(k_pool + ph * (B * kHeadDim)) + ln;
            const float scale = scales[2 * ph];
            float acc[16] = {};
#pragma unroll
            for (int t0 = 0; t0 < B; t0 += 16) {
                uint4 r[16];
#pragma unroll
                for (int t = 0; t < 16; ++t) r[t] = src[min(t0 + t, n - 1) * 8];     // (rows past the last token repeat it and are not added)
#pragma unroll
                for (int t = 0; t < 16; ++t)
                    if (t0 + t < n) add_bytes(acc, r[t]);
            }
            put_means<B>(mean, acc, scale, n);
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
    units_above<T>(lds, lds_chunk, g, gk, P, p_lo, c_lo, c_hi, fc, cg, gg, tid);
}

template <int B, class T>
static hipError_t launch_all(chess_ctx* ctx, const uint8_t* k_pool, const float* scales, const int32_t* block_table, const int32_t* seq_lens,
                             int batch, const int32_t* from_page, int recent, void* pages, void* chunks, void* grids, hipStream_t stream)
{
    const Geom& g = ctx->geom;
    const int ppg = g.n_c * g.n_g;
    const size_t lds = (size_t)(ppg + g.n_g) * kHeadDim * sizeof(T);
    const int span = recent > 0 ? std::min(g.max_grids, (recent + ppg - 2) / ppg + 1) : g.max_grids;   // grids `recent` pages can touch
    const auto kern = quant_summarize_kernel<B, T>;
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    return launch(kern, dim3(span, g.n_kv_heads, batch), dim3(256), lds, stream, k_pool, scales, block_table, seq_lens, from_page, recent, g,
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

// What the summaries of bf16 and of 8-bit pages share: stored vectors, and the chunks and the grid above a grid's pages.
#pragma once

#include "select_device.h"

namespace chess {

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

__device__ __forceinline__ void add_row(double (&acc)[8], const uint4& r)
{
    acc[0] += (double)bf16_lo(r.x); acc[1] += (double)bf16_hi(r.x);
    acc[2] += (double)bf16_lo(r.y); acc[3] += (double)bf16_hi(r.y);
    acc[4] += (double)bf16_lo(r.z); acc[5] += (double)bf16_hi(r.z);
    acc[6] += (double)bf16_lo(r.w); acc[7] += (double)bf16_hi(r.w);
}

// Eight consecutive elements of a stored vector (dims 8 ln .. 8 ln + 7), to and from memory (global or LDS).
template <class T>
struct Row8;
template <>
struct Row8<float> {
    float4 lo, hi;
    __device__ __forceinline__ void set(const double (&m)[8])
    {
        lo = make_float4((float)m[0], (float)m[1], (float)m[2], (float)m[3]);
        hi = make_float4((float)m[4], (float)m[5], (float)m[6], (float)m[7]);
    }
    __device__ __forceinline__ void load(const float* p) { lo = reinterpret_cast<const float4*>(p)[0]; hi = reinterpret_cast<const float4*>(p)[1]; }
    __device__ __forceinline__ void store(float* p) const { reinterpret_cast<float4*>(p)[0] = lo; reinterpret_cast<float4*>(p)[1] = hi; }
};
template <>
struct Row8<uint16_t> {
    uint4 v;
    // fp64 mean -> fp32 -> nearest-even bf16 (finite inputs), two per word
    static __device__ __forceinline__ uint32_t bf(double m)
    {
        const uint32_t u = __float_as_uint((float)m);
        return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
    }
    __device__ __forceinline__ void set(const double (&m)[8])
    {
        v = make_uint4(bf(m[0]) | (bf(m[1]) << 16), bf(m[2]) | (bf(m[3]) << 16), bf(m[4]) | (bf(m[5]) << 16), bf(m[6]) | (bf(m[7]) << 16));
    }
    __device__ __forceinline__ void load(const uint16_t* p) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<uint4*>(p) = v; }
};

__device__ __forceinline__ double as_f64(float v) { return (double)v; }
__device__ __forceinline__ double as_f64(uint16_t v) { return (double)__uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ void put_mean(float* p, double m) { *p = (float)m; }
__device__ __forceinline__ void put_mean(uint16_t* p, double m) { *p = (uint16_t)Row8<uint16_t>::bf(m); }

// The chunk vectors [c_lo, c_hi) of grid gk, those from fc on formed from the grid's page vectors in LDS (the first is page p_lo's) and
// the others read, then the grid's own.  kThreads threads; the page vectors are in place.
template <class T, int kThreads = 256>
__device__ __forceinline__ void units_above(const T* lds, T* lds_chunk, const Geom& g, int gk, int P, int p_lo, int c_lo, int c_hi, int fc,
                                            T* __restrict__ cg, T* __restrict__ gg, int tid)
{
    for (int idx = tid; idx < (c_hi - c_lo) * kHeadDim; idx += kThreads) {
        const int c = c_lo + idx / kHeadDim, dim = idx % kHeadDim;
        T v;
        if (c >= fc) {
            const int lo = c * g.n_c, hi = min(P, lo + g.n_c);
            double acc = 0.0;
            for (int j = lo; j < hi; ++j) acc += as_f64(lds[(size_t)(j - p_lo) * kHeadDim + dim]);
            put_mean(&v, acc / (double)(hi - lo));
            cg[(size_t)c * kHeadDim + dim] = v;
        } else {
            v = cg[(size_t)c * kHeadDim + dim];
        }
        lds_chunk[idx] = v;
    }
    __syncthreads();

    if (tid < kHeadDim) {
        double acc = 0.0;
        for (int c = 0; c < c_hi - c_lo; ++c) acc += as_f64(lds_chunk[c * kHeadDim + tid]);
        T v;
        put_mean(&v, acc / (double)(c_hi - c_lo));
        gg[(size_t)gk * kHeadDim + tid] = v;
    }
}

constexpr int kRecentMost = 16;                       // pages, and children of a unit: one per group
// The last few pages of every sequence and what is above them (one workgroup of 256 threads per KV head and sequence: summarize_recent_kernel).
// page_mean(block, n, ln): dims 8 ln .. 8 ln + 7 of the mean of the first n rows of block = physical page * KV heads + KV head.
template <int B, class T, class PageMean>
__device__ __forceinline__ void refresh_recent(uint64_t seq_lens_at, uint64_t block_table_at, uint64_t pages_at, int max_pages, int shape, int rows,
                                               int max_chunks, uint32_t inv_nc, uint32_t inv_ng, int max_grids, PageMean page_mean)
{
    extern __shared__ float lds_f[];                  // page vectors from the first refreshed chunk's first page on, then chunk vectors
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, grp = tid >> 4, ln = tid & 15;
    const int recent = shape & 31, n_c = (shape >> 5) & 31, n_g = (shape >> 10) & 31, H = shape >> 15;
    T* lds_page = reinterpret_cast<T*>(lds_f);
    T* lds_chunk = lds_page + (n_c - 1 + recent) * kHeadDim;
    const int L = min(__builtin_amdgcn_readfirstlane(load_by_lane(device_pointer<const int32_t>(seq_lens_at) + b)), max_pages * B);
    if (L <= 0) return;
    const int P = (L + B - 1) / B, fp = max(P - recent, 0), n_new = P - fp;
    const int fc = div_by(fp, inv_nc), lc = div_by(P - 1, inv_nc), fg = div_by(fc, inv_ng), lg = div_by(lc, inv_ng);
    const int p0 = fc * n_c, c0 = fg * n_g;
    const int j = fp + min(grp, n_new - 1);           // this group's page
    const int64_t phys = device_pointer<const int32_t>(block_table_at)[(size_t)b * max_pages + j];
    const int row = b * H + h;
    const VecBases at = bases_of(rows, row, max_pages, max_chunks, max_grids);
    T* pg = device_pointer<T>(pages_at) + (size_t)row * max_pages * kHeadDim;
    T* cg = pg + (int64_t)at.chunks * kHeadDim;
    T* gg = pg + (int64_t)at.grids * kHeadDim;
    // (as words, not as Row8 and not as arrays: those went through scratch memory)
    constexpr int kHi = sizeof(T) == 4 ? 1 : 0;       // eight elements are two 16-byte words, or one
    const uint4* from_page = reinterpret_cast<const uint4*>(pg + (size_t)min(p0 + grp, P - 1) * kHeadDim + ln * 8);
    const uint4* from_chunk = reinterpret_cast<const uint4*>(cg + (size_t)min(c0 + grp, lc) * kHeadDim + ln * 8);
    const uint4 page_lo = from_page[0], page_hi = from_page[kHi], chunk_lo = from_chunk[0], chunk_hi = from_chunk[kHi];
    asm volatile("" : : : "memory");                  // (requested here, not where they are stored)
    if (grp < n_new) {                                // (a wave whose groups have no page skips the rows)
        const int n = j == P - 1 ? L - j * B : B;
        const Row8<T> mean8 = page_mean(phys * H + h, n, ln);
        mean8.store(lds_page + (j - p0) * kHeadDim + ln * 8);
        mean8.store(pg + (size_t)j * kHeadDim + ln * 8);
    }
    if (p0 + grp < fp) {
        uint4* to = reinterpret_cast<uint4*>(lds_page + grp * kHeadDim + ln * 8);
        to[0] = page_lo;
        if (kHi) to[kHi] = page_hi;
    }
    if (c0 + grp < fc) {
        uint4* to = reinterpret_cast<uint4*>(lds_chunk + grp * kHeadDim + ln * 8);
        to[0] = chunk_lo;
        if (kHi) to[kHi] = chunk_hi;
    }
    __syncthreads();

    // a unit's mean, one dim a thread: its children [lo, hi), in order, eight read at a time
    const int dim = tid % kHeadDim;
    const auto mean_of = [&](const T* children, int lo, int hi, int from) {
        double sum = 0.0;
        for (int k0 = lo; k0 < hi; k0 += 8) {
            T v[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) v[x] = children[(min(k0 + x, hi - 1) - from) * kHeadDim + dim];
#pragma unroll
            for (int x = 0; x < 8; ++x)
                if (k0 + x < hi) sum += as_f64(v[x]);
        }
        T m;
        put_mean(&m, sum / (double)(hi - lo));
        return m;
    };
    for (int c = fc + tid / kHeadDim; c <= lc; c += 2) {
        const T v = mean_of(lds_page, c * n_c, min(P, c * n_c + n_c), p0);
        cg[(size_t)c * kHeadDim + dim] = v;
        lds_chunk[(c - c0) * kHeadDim + dim] = v;
    }
    __syncthreads();
    for (int k = fg + tid / kHeadDim; k <= lg; k += 2) gg[(size_t)k * kHeadDim + dim] = mean_of(lds_chunk, k * n_g, min(lc + 1, k * n_g + n_g), c0);
}

// Whether the kernels of the last pages can serve so many: a group a page, a child and a chunk.
inline bool fits_recent(const Geom& g, int recent)
{
    return recent <= kRecentMost && g.n_c <= kRecentMost && g.n_g <= kRecentMost && g.n_kv_heads < 1 << 16;
}
// Pages of the first refreshed chunk and the new ones, chunks of the first refreshed grid and the new ones.
inline size_t recent_lds_bytes(const Geom& g, int recent, size_t element)
{
    const int new_chunks = (recent + g.n_c - 2) / g.n_c + 1;
    return (size_t)(g.n_c - 1 + recent + g.n_g - 1 + new_chunks) * kHeadDim * element;
}

}  // namespace chess

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
// the others read, then the grid's own.  256 threads; the page vectors are in place.
template <class T>
__device__ __forceinline__ void units_above(const T* lds, T* lds_chunk, const Geom& g, int gk, int P, int p_lo, int c_lo, int c_hi, int fc,
                                            T* __restrict__ cg, T* __restrict__ gg, int tid)
{
    for (int idx = tid; idx < (c_hi - c_lo) * kHeadDim; idx += 256) {
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

}  // namespace chess

// What the two directions of the root-mean-square norm (gf_block.h) share: how a row is dealt to threads.
//
// A row is taken as octets that start on multiples of eight elements of the TENSOR, so that every load and store is a
// whole 16-byte vector wherever a row starts; the first and last octet of a row may hold neighbours' elements, which are masked.
// A team of threads (part of a warp, or a block) has a row; thread g of T has octets g, g + T, ..  Teams walk over the
// rows in steps of a multiple of eight rows, so that all rows of a team start at the same place of an octet: a
// thread has the same columns in all of them.
#pragma once

#include "gf_block.h"
#include "gf_octet.cuh"

namespace gf {

constexpr int kRmsThreads = 256;       // of a block whose rows have a warp or less
constexpr int kRmsMostThreads = 512;   // of a block that has one row at a time

struct RmsArgs {
    const void *x, *residual, *gamma;
    const void *gy, *gh;
    const float *rstd_in, *dots;       // dots (backward): sums of q xh / cols from a pass of their own, or NULL
    void *h, *y, *gres;                // y: y, or g_x
    uint8_t* codes;
    float *scales, *rstd, *part;
    long long rows, total, scale_pitch;
    int cols, pitch, log_tpr, gamma_bf16;
    int col_tile;                      // backward: columns of a block row of the grid
    float eps, inv_c;
    Drop drop;
};

__device__ __forceinline__ float rms_gamma(const RmsArgs& a, int c) {
    if (!a.gamma) return 1.f;
    return a.gamma_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(a.gamma)[c]) : static_cast<const float*>(a.gamma)[c];
}

// gamma of the eight columns from c on; those outside the row get 0
__device__ __forceinline__ void rms_gamma8(const RmsArgs& a, int c, Eight& p) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i >= 0 && c + i < a.cols ? rms_gamma(a, c + i) : 0.f;
    to_eight(v, p);
}

// The sum over a team; `red`: 32 floats that are not in use since the last sum but one.
template <bool WARP> __device__ __forceinline__ float rms_sum(float v, int log_tpr, float* red) {
    if constexpr (WARP) {
        for (int o = (1 << log_tpr) >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    } else {
        v = warp_sum(v);
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        const int n = (int)blockDim.x >> 5;
        float s = 0.f;
        for (int k = 0; k < n; k += 4) {               // places past the last warp hold zeros
            const float4 p = *reinterpret_cast<const float4*>(red + k);
            s += (p.x + p.y) + (p.z + p.w);
        }
        return s;
    }
}

static inline bool rms_off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
gf_status rms_validate(const gf_rms_desc* d);

// Octets of a row, wherever it starts
static inline int rms_octets(int cols) { return cols % 8 == 0 ? cols / 8 : (cols + 14) / 8; }

// Threads for rows of n octets.  WARP: 1 << log_tpr threads per row, of a whole warp up to `most` octets each; else a block, one or
// two octets per thread.  In every form only a thread's last octet may lie past the row.
struct RmsShape {
    bool warp;
    int log_tpr, threads, per_thread;
};
static inline RmsShape rms_shape(int n, int most, int least_log) {
    RmsShape s = {};
    s.warp = n <= 32 * most;
    if (s.warp) {
        s.log_tpr = least_log;
        while (s.log_tpr < 5 && (1 << s.log_tpr) < n) ++s.log_tpr;
        s.per_thread = (n + (1 << s.log_tpr) - 1) >> s.log_tpr;
        s.threads = kRmsThreads;
    } else {
        s.per_thread = n > 128 ? 2 : 1;
        s.threads = ((n + s.per_thread - 1) / s.per_thread + 31) / 32 * 32;
    }
    return s;
}

// Blocks of `kernel` that an SM holds; the query is made once per kernel, number of threads and device.  (The shared memory of some forms
// grows with the columns, but never so far that it, and not the registers, decides.)
template <typename Kern> static inline int rms_resident(Kern kernel, int threads, size_t smem, int (&cached)[kMaxDevices]) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 1;
    if (cached[dev] == 0) {
        int n = 0;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem) != cudaSuccess || n < 1) n = 1;
        cached[dev] = n;
    }
    return cached[dev];
}

}  // namespace gf

// Layer normalisation over the channels, forward and backward (gf_train.h).
#include <type_traits>

#include "gf_common.cuh"
#include "gf_train.h"

namespace gf {
namespace {

// ---- element access ----------------------------------------------------------------------
// V consecutive elements at p (V * sizeof(T) <= 16, p aligned to that) as floats.
template <typename T, int V> __device__ __forceinline__ void load_vec(const T* p, float (&v)[V]) {
    if constexpr (V == 1) v[0] = to_f32(p[0]);
    else if constexpr (std::is_same<T, float>::value) {
        if constexpr (V == 2) { const float2 a = *reinterpret_cast<const float2*>(p); v[0] = a.x; v[1] = a.y; }
        else { const float4 a = *reinterpret_cast<const float4*>(p); v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; }
    } else {
        uint32_t w[V / 2];
        if constexpr (V == 2) w[0] = *reinterpret_cast<const uint32_t*>(p);
        else if constexpr (V == 4) { const uint2 a = *reinterpret_cast<const uint2*>(p); w[0] = a.x; w[1] = a.y; }
        else { const uint4 a = *reinterpret_cast<const uint4*>(p); w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; }
#pragma unroll
        for (int i = 0; i < V / 2; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
}
template <typename T, int V> __device__ __forceinline__ void store_vec(T* p, const float (&v)[V]) {
    if constexpr (V == 1) p[0] = from_f32<T>(v[0]);
    else if constexpr (std::is_same<T, float>::value) {
        if constexpr (V == 2) *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
        else *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
        uint32_t w[V / 2];
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
        if constexpr (V == 2) *reinterpret_cast<uint32_t*>(p) = w[0];
        else if constexpr (V == 4) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// gamma or beta: fp32 or bf16, absent = `none`
struct Param {
    const void* p;
    int bf16;
    __device__ __forceinline__ float at(int c, float none) const {
        if (!p) return none;
        return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[c]) : static_cast<const float*>(p)[c];
    }
};

struct NormArgs {
    const void *x, *gy;
    void* out;                 // y, or g_x (NULL: not wanted)
    Param gamma, beta;
    const float *mean_in, *rstd_in;
    float *mean, *rstd;        // NULL: not wanted
    float* part;               // [blocks][2][C] sums of g_gamma and g_beta (NULL: not wanted)
    long long R;               // pixels
    int C;
    int HW;                    // pixels of a plane (channels-first)
    FastDiv div_hw;
    float eps, inv_c;
    int log_tpr;               // rows: log2 of the threads that share a row
};

// Sum over the threads that share a row.  One warp or less: shuffles.  Whole block: one more step
// through `red` (32 floats; the caller alternates two of them so that one barrier per sum is enough).
template <bool WHOLE_BLOCK> __device__ __forceinline__ float row_sum(float v, int log_tpr, float* red) {
    if constexpr (!WHOLE_BLOCK) {
        for (int o = (1 << log_tpr) >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    } else {
        v = warp_sum(v);
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        const int n = blockDim.x >> 5;
        return warp_sum((int)(threadIdx.x & 31) < n ? red[threadIdx.x & 31] : 0.f);
    }
}

constexpr int kRowThreads = 256;      // block size when a row has a warp or less

// ---- rows ------------------------------------------------------------------------------------
// One row stays in the registers of the threads that share it: x is read once, the variance is
// taken about the mean.
template <typename T, int V, int NV, bool WHOLE_BLOCK>
__global__ void __launch_bounds__(1024) ln_rows_fwd_kernel(const __grid_constant__ NormArgs a) {
    __shared__ float red[2][32];
    const int tpr = 1 << a.log_tpr;
    const int g = threadIdx.x & (tpr - 1);
    const long long row = (long long)blockIdx.x * (blockDim.x >> a.log_tpr) + (threadIdx.x >> a.log_tpr);
    const bool live = row < a.R;
    const T* x = static_cast<const T*>(a.x) + row * a.C;
    float v[NV][V];
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * tpr + g) * V;
        if (live && c < a.C) load_vec<T, V>(x + c, v[k]);
        else {
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) s += v[k][i];
    }
    const float mean = row_sum<WHOLE_BLOCK>(s, a.log_tpr, red[0]) / (float)a.C;
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if ((k * tpr + g) * V < a.C) {
#pragma unroll
            for (int i = 0; i < V; ++i) { const float d = v[k][i] - mean; q += d * d; }
        }
    }
    const float rstd = rsqrtf(row_sum<WHOLE_BLOCK>(q, a.log_tpr, red[1]) * a.inv_c + a.eps);
    if (!live) return;
    T* y = static_cast<T*>(a.out) + row * a.C;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * tpr + g) * V;
        if (c < a.C) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] = (v[k][i] - mean) * rstd * a.gamma.at(c + i, 1.f) + a.beta.at(c + i, 0.f);
            store_vec<T, V>(y + c, v[k]);
        }
    }
    if (a.mean && g == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
}

// Rows longer than the registers of a block: the row is read again from L2 for each pass.
template <typename T> __global__ void __launch_bounds__(1024) ln_rows_fwd_long_kernel(const __grid_constant__ NormArgs a) {
    __shared__ float red[2][32];
    const long long row = blockIdx.x;
    const T* x = static_cast<const T*>(a.x) + row * a.C;
    T* y = static_cast<T*>(a.out) + row * a.C;
    float s = 0.f;
    for (int c = threadIdx.x; c < a.C; c += blockDim.x) s += to_f32(x[c]);
    const float mean = row_sum<true>(s, 0, red[0]) / (float)a.C;
    float q = 0.f;
    for (int c = threadIdx.x; c < a.C; c += blockDim.x) { const float d = to_f32(x[c]) - mean; q += d * d; }
    const float rstd = rsqrtf(row_sum<true>(q, 0, red[1]) * a.inv_c + a.eps);
    for (int c = threadIdx.x; c < a.C; c += blockDim.x)
        y[c] = from_f32<T>((to_f32(x[c]) - mean) * rstd * a.gamma.at(c, 1.f) + a.beta.at(c, 0.f));
    if (a.mean && threadIdx.x == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
}

// Backward: every thread keeps the same columns for all rows of its block, so that g_gamma and
// g_beta are sums in registers until the block has no more rows; one [2][C] line per block is
// left for the finishing kernel.
template <typename T, int V, int NV, bool WHOLE_BLOCK>
__global__ void __launch_bounds__(WHOLE_BLOCK ? 512 : kRowThreads) ln_rows_bwd_kernel(const __grid_constant__ NormArgs a) {
    __shared__ float red[4][32];
    extern __shared__ float cols[];                       // !WHOLE_BLOCK: [2][C]
    const int tpr = 1 << a.log_tpr;
    const int g = threadIdx.x & (tpr - 1);
    const int rows_pb = blockDim.x >> a.log_tpr;
    float gam[NV][V], ag[NV][V], ab[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (k * tpr + g) * V + i;
            gam[k][i] = c < a.C ? a.gamma.at(c, 1.f) : 0.f;
            ag[k][i] = ab[k][i] = 0.f;
        }
    int turn = 0;
    for (long long r0 = (long long)blockIdx.x * rows_pb; r0 < a.R; r0 += (long long)gridDim.x * rows_pb, turn ^= 2) {
        const long long row = r0 + (threadIdx.x >> a.log_tpr);
        const bool live = row < a.R;
        const T* x = static_cast<const T*>(a.x) + row * a.C;
        const T* gy = static_cast<const T*>(a.gy) + row * a.C;
        const float mean = live ? a.mean_in[row] : 0.f, rstd = live ? a.rstd_in[row] : 0.f;
        float xh[NV][V], gv[NV][V];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * tpr + g) * V;
            if (live && c < a.C) {
                load_vec<T, V>(x + c, xh[k]);
                load_vec<T, V>(gy + c, gv[k]);
#pragma unroll
                for (int i = 0; i < V; ++i) xh[k][i] = (xh[k][i] - mean) * rstd;
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) xh[k][i] = gv[k][i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                ag[k][i] += gv[k][i] * xh[k][i];
                ab[k][i] += gv[k][i];
                const float h = gv[k][i] * gam[k][i];
                s1 += h;
                s2 += h * xh[k][i];
            }
        }
        if (a.out) {
            s1 = row_sum<WHOLE_BLOCK>(s1, a.log_tpr, red[turn]) * a.inv_c;
            s2 = row_sum<WHOLE_BLOCK>(s2, a.log_tpr, red[turn + 1]) * a.inv_c;
            if (live) {
                T* gx = static_cast<T*>(a.out) + row * a.C;
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    const int c = (k * tpr + g) * V;
                    if (c < a.C) {
#pragma unroll
                        for (int i = 0; i < V; ++i) xh[k][i] = rstd * (gv[k][i] * gam[k][i] - s1 - xh[k][i] * s2);
                        store_vec<T, V>(gx + c, xh[k]);
                    }
                }
            }
        }
    }
    if (!a.part) return;
    float* part = a.part + (size_t)blockIdx.x * 2 * a.C;
    if constexpr (WHOLE_BLOCK) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (k * tpr + g) * V + i;
                if (c < a.C) { part[c] = ag[k][i]; part[a.C + c] = ab[k][i]; }
            }
    } else {
        // lanes of a warp that hold the same columns, then the warps of the block in order
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i)
                for (int o = tpr; o < 32; o <<= 1) {
                    ag[k][i] += __shfl_xor_sync(0xffffffffu, ag[k][i], o);
                    ab[k][i] += __shfl_xor_sync(0xffffffffu, ab[k][i], o);
                }
        for (int w = 0; w < (int)(blockDim.x >> 5); ++w) {
            if ((int)(threadIdx.x >> 5) == w && (int)(threadIdx.x & 31) < tpr) {
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int c = (k * tpr + g) * V + i;
                        if (c < a.C) {
                            cols[c] = w == 0 ? ag[k][i] : cols[c] + ag[k][i];
                            cols[a.C + c] = w == 0 ? ab[k][i] : cols[a.C + c] + ab[k][i];
                        }
                    }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < 2 * a.C; c += blockDim.x) part[c] = cols[c];
    }
}

// Rows longer than the registers of a block: two passes over the row (the second from L2); the
// column sums are kept in the block's line of the workspace, each by the thread that owns the column.
template <typename T> __global__ void __launch_bounds__(1024) ln_rows_bwd_long_kernel(const __grid_constant__ NormArgs a) {
    __shared__ float red[4][32];
    float* part = a.part ? a.part + (size_t)blockIdx.x * 2 * a.C : nullptr;
    bool first = true;
    int turn = 0;
    for (long long row = blockIdx.x; row < a.R; row += gridDim.x, first = false, turn ^= 2) {
        const T* x = static_cast<const T*>(a.x) + row * a.C;
        const T* gy = static_cast<const T*>(a.gy) + row * a.C;
        const float mean = a.mean_in[row], rstd = a.rstd_in[row];
        float s1 = 0.f, s2 = 0.f;
        for (int c = threadIdx.x; c < a.C; c += blockDim.x) {
            const float xh = (to_f32(x[c]) - mean) * rstd, gv = to_f32(gy[c]);
            const float h = gv * a.gamma.at(c, 1.f);
            s1 += h;
            s2 += h * xh;
            if (part) {
                part[c] = first ? gv * xh : part[c] + gv * xh;
                part[a.C + c] = first ? gv : part[a.C + c] + gv;
            }
        }
        if (!a.out) continue;
        s1 = row_sum<true>(s1, 0, red[turn]) * a.inv_c;
        s2 = row_sum<true>(s2, 0, red[turn + 1]) * a.inv_c;
        T* gx = static_cast<T*>(a.out) + row * a.C;
        for (int c = threadIdx.x; c < a.C; c += blockDim.x) {
            const float xh = (to_f32(x[c]) - mean) * rstd;
            gx[c] = from_f32<T>(rstd * (to_f32(gy[c]) * a.gamma.at(c, 1.f) - s1 - xh * s2));
        }
    }
}

// ---- channels first --------------------------------------------------------------------------
// A block takes 32 V consecutive pixels (lane = pixel, V per lane) and all channels; warp w of CG
// has channels w, w + CG, ...  Pixels are numbered through all images, so that small planes fill
// the lanes; V divides the plane, so that a vector stays in it.
__device__ __forceinline__ long long pixel_offset(const NormArgs& a, long long q) {
    // R < 2^31: 32-bit division
    uint32_t n, p;
    a.div_hw.divmod((uint32_t)q, n, p);
    return (long long)n * a.C * a.HW + p;
}

// Sum over the warps of a block of one value per (lane, i); `red` is [32 warps][32 lanes * V].
template <int V> __device__ __forceinline__ void warps_sum(float (&v)[V], float* red) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, n = blockDim.x >> 5;
#pragma unroll
    for (int i = 0; i < V; ++i) red[(w * V + i) * 32 + lane] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = 0.f;
    for (int k = 0; k < n; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += red[(k * V + i) * 32 + lane];
}

// NCH: channels per warp held in registers; 0: the planes are read again (from L2) for each pass.
template <typename T, int V, int NCH>
__global__ void __launch_bounds__(1024) ln_planes_fwd_kernel(const __grid_constant__ NormArgs a) {
    extern __shared__ float red[];                        // [2][warps][32 V]
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, CG = blockDim.x >> 5;
    const long long q = ((long long)blockIdx.x * 32 + lane) * V;
    const bool live = q < a.R;
    const long long off = live ? pixel_offset(a, q) : 0;
    const T* x = static_cast<const T*>(a.x) + off;
    T* y = static_cast<T*>(a.out) + off;
    float mean[V], rstd[V];
#pragma unroll
    for (int i = 0; i < V; ++i) mean[i] = rstd[i] = 0.f;
    float* red2 = red + CG * 32 * V;
    if constexpr (NCH > 0) {
        float v[NCH][V];
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int c = j * CG + w;
            if (live && c < a.C) load_vec<T, V>(x + (long long)c * a.HW, v[j]);
            else {
#pragma unroll
                for (int i = 0; i < V; ++i) v[j][i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) mean[i] += v[j][i];
        }
        warps_sum<V>(mean, red);
#pragma unroll
        for (int i = 0; i < V; ++i) mean[i] /= (float)a.C;
#pragma unroll
        for (int j = 0; j < NCH; ++j)
            if (j * CG + w < a.C) {
#pragma unroll
                for (int i = 0; i < V; ++i) { const float d = v[j][i] - mean[i]; rstd[i] += d * d; }
            }
        warps_sum<V>(rstd, red2);
#pragma unroll
        for (int i = 0; i < V; ++i) rstd[i] = rsqrtf(rstd[i] * a.inv_c + a.eps);
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int c = j * CG + w;
            if (live && c < a.C) {
                const float gm = a.gamma.at(c, 1.f), bt = a.beta.at(c, 0.f);
#pragma unroll
                for (int i = 0; i < V; ++i) v[j][i] = (v[j][i] - mean[i]) * rstd[i] * gm + bt;
                store_vec<T, V>(y + (long long)c * a.HW, v[j]);
            }
        }
    } else {
        float v[V];
        for (int c = w; live && c < a.C; c += CG) {
            load_vec<T, V>(x + (long long)c * a.HW, v);
#pragma unroll
            for (int i = 0; i < V; ++i) mean[i] += v[i];
        }
        warps_sum<V>(mean, red);
#pragma unroll
        for (int i = 0; i < V; ++i) mean[i] /= (float)a.C;
        for (int c = w; live && c < a.C; c += CG) {
            load_vec<T, V>(x + (long long)c * a.HW, v);
#pragma unroll
            for (int i = 0; i < V; ++i) { const float d = v[i] - mean[i]; rstd[i] += d * d; }
        }
        warps_sum<V>(rstd, red2);
#pragma unroll
        for (int i = 0; i < V; ++i) rstd[i] = rsqrtf(rstd[i] * a.inv_c + a.eps);
        for (int c = w; live && c < a.C; c += CG) {
            load_vec<T, V>(x + (long long)c * a.HW, v);
            const float gm = a.gamma.at(c, 1.f), bt = a.beta.at(c, 0.f);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = (v[i] - mean[i]) * rstd[i] * gm + bt;
            store_vec<T, V>(y + (long long)c * a.HW, v);
        }
    }
    if (a.mean && live && w == 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) { a.mean[q + i] = mean[i]; a.rstd[q + i] = rstd[i]; }
    }
}

// v[j] of every lane -> the sum over the 32 lanes of v[j], for all j at once: each exchange halves
// the values a lane is responsible for (NCH - 1 shuffles and not 5 NCH).  N = NCH / 32 values (at
// least one) are left in a lane: those of j = lane * N + i, for NCH < 32 j = lane * NCH / 32.
template <int NCH> __device__ __forceinline__ void lanes_sum(float (&v)[NCH]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int step = 0; step < 5; ++step) {
        const int o = 16 >> step;
        const int n = NCH >> step;               // values held before this step (0: one, already shared out)
        if (n > 1) {
            const bool up = (lane & o) != 0;
#pragma unroll
            for (int k = 0; k < NCH / 2; ++k)
                if (k < n / 2) {
                    const float lo = v[k], hi = v[k + n / 2];
                    const float send = up ? lo : hi;
                    v[k] = (up ? hi : lo) + __shfl_xor_sync(0xffffffffu, send, o);
                }
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
        }
    }
}

template <typename T, int V, int NCH>
__global__ void __launch_bounds__(512) ln_planes_bwd_kernel(const __grid_constant__ NormArgs a, long long tiles) {
    extern __shared__ float red[];                        // [2 turns][2][warps][32 V]
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, CG = blockDim.x >> 5;
    constexpr int NA = NCH >= 32 ? NCH / 32 : 1;
    float ag[NA], ab[NA];
#pragma unroll
    for (int i = 0; i < NA; ++i) ag[i] = ab[i] = 0.f;
    const int red_n = CG * 32 * V;
    int turn = 0;
    for (long long t = blockIdx.x; t < tiles; t += gridDim.x, turn ^= 1) {
        const long long q = (t * 32 + lane) * V;
        const bool live = q < a.R;
        const long long off = live ? pixel_offset(a, q) : 0;
        const T* x = static_cast<const T*>(a.x) + off;
        const T* gy = static_cast<const T*>(a.gy) + off;
        float mean[V], rstd[V], s1[V], s2[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            mean[i] = live ? a.mean_in[q + i] : 0.f;
            rstd[i] = live ? a.rstd_in[q + i] : 0.f;
            s1[i] = s2[i] = 0.f;
        }
        float xh[NCH][V], gv[NCH][V];
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int c = j * CG + w;
            if (live && c < a.C) {
                load_vec<T, V>(x + (long long)c * a.HW, xh[j]);
                load_vec<T, V>(gy + (long long)c * a.HW, gv[j]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) { xh[j][i] = mean[i]; gv[j][i] = 0.f; }
            }
        }
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int c = j * CG + w;
            const float gm = c < a.C ? a.gamma.at(c, 1.f) : 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                xh[j][i] = (xh[j][i] - mean[i]) * rstd[i];
                const float h = gv[j][i] * gm;
                s1[i] += h;
                s2[i] += h * xh[j][i];
            }
        }
        if (a.part) {
            float p[NCH], b[NCH];
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                p[j] = b[j] = 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) { p[j] += gv[j][i] * xh[j][i]; b[j] += gv[j][i]; }
            }
            lanes_sum<NCH>(p);
            lanes_sum<NCH>(b);
#pragma unroll
            for (int i = 0; i < NA; ++i) { ag[i] += p[i]; ab[i] += b[i]; }
        }
        if (a.out) {
            warps_sum<V>(s1, red + turn * 2 * red_n);
            warps_sum<V>(s2, red + (turn * 2 + 1) * red_n);
#pragma unroll
            for (int i = 0; i < V; ++i) { s1[i] *= a.inv_c; s2[i] *= a.inv_c; }
            T* gx = static_cast<T*>(a.out) + off;
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                const int c = j * CG + w;
                if (live && c < a.C) {
                    const float gm = a.gamma.at(c, 1.f);
#pragma unroll
                    for (int i = 0; i < V; ++i) xh[j][i] = rstd[i] * (gv[j][i] * gm - s1[i] - xh[j][i] * s2[i]);
                    store_vec<T, V>(gx + (long long)c * a.HW, xh[j]);
                }
            }
        }
    }
    if (a.part) {
        float* part = a.part + (size_t)blockIdx.x * 2 * a.C;
        constexpr int share = NCH >= 32 ? 1 : 32 / NCH;   // lanes that hold the same sum
        if (lane % share == 0) {
#pragma unroll
            for (int i = 0; i < NA; ++i) {
                const int c = (lane / share * NA + i) * CG + w;
                if (c < a.C) { part[c] = ag[i]; part[a.C + c] = ab[i]; }
            }
        }
    }
}

// More channels than the registers of a block hold: two passes (the second from L2).
template <typename T, int V>
__global__ void __launch_bounds__(512) ln_planes_bwd_long_kernel(const __grid_constant__ NormArgs a, long long tiles) {
    extern __shared__ float red[];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, CG = blockDim.x >> 5;
    float* part = a.part ? a.part + (size_t)blockIdx.x * 2 * a.C : nullptr;
    const int red_n = CG * 32 * V;
    int turn = 0;
    bool first = true;
    for (long long t = blockIdx.x; t < tiles; t += gridDim.x, turn ^= 1, first = false) {
        const long long q = (t * 32 + lane) * V;
        const bool live = q < a.R;
        const long long off = live ? pixel_offset(a, q) : 0;
        const T* x = static_cast<const T*>(a.x) + off;
        const T* gy = static_cast<const T*>(a.gy) + off;
        float mean[V], rstd[V], s1[V], s2[V], xv[V], gv[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            mean[i] = live ? a.mean_in[q + i] : 0.f;
            rstd[i] = live ? a.rstd_in[q + i] : 0.f;
            s1[i] = s2[i] = xv[i] = gv[i] = 0.f;
        }
        for (int c = w; c < a.C; c += CG) {
            if (live) {
                load_vec<T, V>(x + (long long)c * a.HW, xv);
                load_vec<T, V>(gy + (long long)c * a.HW, gv);
            }
            const float gm = a.gamma.at(c, 1.f);
            float p = 0.f, b = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xh = (xv[i] - mean[i]) * rstd[i], h = gv[i] * gm;
                s1[i] += h;
                s2[i] += h * xh;
                p += gv[i] * xh;
                b += gv[i];
            }
            if (part) {
                p = warp_sum(p);
                b = warp_sum(b);
                if (lane == 0) { part[c] = first ? p : part[c] + p; part[a.C + c] = first ? b : part[a.C + c] + b; }
            }
        }
        if (!a.out) continue;
        warps_sum<V>(s1, red + turn * 2 * red_n);
        warps_sum<V>(s2, red + (turn * 2 + 1) * red_n);
        T* gx = static_cast<T*>(a.out) + off;
        for (int c = w; live && c < a.C; c += CG) {
            load_vec<T, V>(x + (long long)c * a.HW, xv);
            load_vec<T, V>(gy + (long long)c * a.HW, gv);
            const float gm = a.gamma.at(c, 1.f);
#pragma unroll
            for (int i = 0; i < V; ++i)
                xv[i] = rstd[i] * (gv[i] * gm - s1[i] * a.inv_c - (xv[i] - mean[i]) * rstd[i] * (s2[i] * a.inv_c));
            store_vec<T, V>(gx + (long long)c * a.HW, xv);
        }
    }
}

// ---- sums of the blocks' lines -------------------------------------------------------------------
// part [blocks][2 C] -> g_gamma, g_beta: the blocks in a fixed order.
constexpr int kFinX = 32, kFinY = 16;
__global__ void __launch_bounds__(kFinX * kFinY) ln_finish_kernel(const float* part, int blocks, int C, float* g_gamma, float* g_beta) {
    __shared__ float red[kFinY][kFinX + 1];
    pdl_wait();
    const long long col = (long long)blockIdx.x * kFinX + threadIdx.x;
    float s = 0.f;
    if (col < 2LL * C) {
#pragma unroll 4
        for (int b = threadIdx.y; b < blocks; b += kFinY) s += part[(size_t)b * 2 * C + col];
    }
    red[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y == 0 && col < 2LL * C) {
        for (int k = 1; k < kFinY; ++k) s += red[k][threadIdx.x];
        if (col < C) { if (g_gamma) g_gamma[col] = s; }
        else if (g_beta) g_beta[col - C] = s;
    }
}

// ---- host side --------------------------------------------------------------------------------------
gf_status norm_validate(const gf_norm_desc* d) {
    if (!d) return GF_ERR_NULL;
    if (d->N < 0 || d->C < 1 || d->H < 1 || d->W < 1 || !(d->eps >= 0.f)) return GF_ERR_BAD_DESC;
    if ((d->dtype != GF_F32 && d->dtype != GF_BF16) || (d->param_dtype != GF_F32 && d->param_dtype != GF_BF16)) return GF_ERR_BAD_DESC;
    if (d->layout != GF_NCHW && d->layout != GF_NHWC) return GF_ERR_BAD_DESC;
    // pixels are counted in 32 bits, and one channel index and plane offset fits 32 bits
    const long long hw = (long long)d->H * d->W;
    if (hw > 0x7fffffffLL || d->C > (1 << 24) || (d->N > 0 && hw > 0x7fffffffLL / d->N)) return GF_ERR_UNSUPPORTED;
    return GF_OK;
}

bool misaligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

struct NormPlan {
    bool planes;          // channels first with more than one pixel per plane
    int V;                // elements per load
    int log_tpr, NV;      // rows: threads per row; loads per thread (0: long rows)
    int CG, NCH;          // planes: warps, channels per warp (0: read again)
    int threads;
    long long work;       // blocks of work (row groups, or pixel tiles)
    int grid;             // backward: persistent blocks
};

// Widest load that keeps every row (plane) on its boundary.
int vec_for(long long n, int esize) {
    int v = 16 / esize;
    while (n % v != 0) v >>= 1;
    return v;
}

NormPlan norm_plan(const gf_norm_desc& d, bool backward) {
    NormPlan p = {};
    const int e = d.dtype == GF_F32 ? 4 : 2;
    const long long R = (long long)d.N * d.H * d.W;
    p.planes = d.layout == GF_NCHW && (long long)d.H * d.W > 1;
    if (!p.planes) {
        p.V = vec_for(d.C, e);
        const int most = backward ? 16 : 32;             // elements a thread holds
        const int max_log = backward ? 9 : 10;
        const long long vecs = (d.C + p.V - 1) / p.V;
        // few elements per thread while a warp is enough for the row, then more threads, then more elements
        int per = 8;
        auto fits = [&](int lt, int el) { return vecs <= (long long)(el / p.V) << lt; };
        p.log_tpr = 0;
        while (p.log_tpr < 5 && !fits(p.log_tpr, per)) ++p.log_tpr;
        if (!fits(p.log_tpr, per)) {
            per = most;
            while (p.log_tpr < max_log && !fits(p.log_tpr, per)) ++p.log_tpr;
        }
        p.NV = fits(p.log_tpr, per) ? per / p.V : 0;
        if (p.NV == 0) p.log_tpr = 10;
        p.threads = p.log_tpr > 5 ? 1 << p.log_tpr : kRowThreads;
        const int rows_pb = p.threads >> p.log_tpr;
        p.work = (R + rows_pb - 1) / rows_pb;
        const int per_sm = p.threads > 512 ? 1 : 1024 / p.threads;
        p.grid = (int)(p.work < (long long)sm_count() * per_sm ? p.work : (long long)sm_count() * per_sm);
    } else {
        p.V = vec_for((long long)d.H * d.W, e);
        if (p.V > 4) p.V = 4;
        const int max_cg = 16;
        p.CG = 4;
        while (p.CG < max_cg && (long long)p.CG * 8 < d.C) p.CG *= 2;
        const int most = 32;                             // values per thread (of each tensor)
        while (p.V > 1 && (long long)p.CG * (most / p.V) < d.C) p.V >>= 1;
        p.NCH = 8;
        while (p.NCH * p.V < most && (long long)p.CG * p.NCH < d.C) p.NCH *= 2;
        if ((long long)p.CG * p.NCH < d.C) { p.NCH = 0; p.V = vec_for((long long)d.H * d.W, e) >= 2 ? 2 : 1; }
        p.threads = 32 * p.CG;
        p.work = (R + 32LL * p.V - 1) / (32LL * p.V);
        const int per_sm = 1024 / p.threads;
        p.grid = (int)(p.work < (long long)sm_count() * per_sm ? p.work : (long long)sm_count() * per_sm);
    }
    return p;
}

template <typename T, int V, int NV> gf_status launch_rows(const NormArgs& a, const NormPlan& p, bool backward, cudaStream_t s) {
    if (!backward) {
        if (p.log_tpr > 5) ln_rows_fwd_kernel<T, V, NV, true><<<(unsigned)p.work, p.threads, 0, s>>>(a);
        else ln_rows_fwd_kernel<T, V, NV, false><<<(unsigned)p.work, p.threads, 0, s>>>(a);
    } else {
        if constexpr (V * NV <= 16) {
            if (p.log_tpr > 5) ln_rows_bwd_kernel<T, V, NV, true><<<p.grid, p.threads, 0, s>>>(a);
            else ln_rows_bwd_kernel<T, V, NV, false><<<p.grid, p.threads, (size_t)2 * a.C * 4, s>>>(a);
        } else return GF_ERR_UNSUPPORTED;
    }
    return after_launch();
}
template <typename T, int V> gf_status launch_rows_v(const NormArgs& a, const NormPlan& p, bool backward, cudaStream_t s) {
    switch (p.NV * V) {
        case 8: return launch_rows<T, V, 8 / V>(a, p, backward, s);
        case 16: return launch_rows<T, V, 16 / V>(a, p, backward, s);
        default: return launch_rows<T, V, 32 / V>(a, p, backward, s);
    }
}
template <typename T, int V> gf_status launch_planes_v(const NormArgs& a, const NormPlan& p, bool backward, cudaStream_t s) {
    const size_t smem = (size_t)(backward ? 4 : 2) * p.CG * 32 * V * 4;
    if (!backward) {
        const unsigned grid = (unsigned)p.work;
        switch (p.NCH) {
            case 8: ln_planes_fwd_kernel<T, V, 8><<<grid, p.threads, smem, s>>>(a); break;
            case 16: if constexpr (V <= 2) { ln_planes_fwd_kernel<T, V, 16><<<grid, p.threads, smem, s>>>(a); break; }
            case 32: if constexpr (V == 1) { ln_planes_fwd_kernel<T, V, 32><<<grid, p.threads, smem, s>>>(a); break; }
            default: ln_planes_fwd_kernel<T, V, 0><<<grid, p.threads, smem, s>>>(a);
        }
    } else {
        switch (p.NCH) {
            case 8: ln_planes_bwd_kernel<T, V, 8><<<p.grid, p.threads, smem, s>>>(a, p.work); break;
            case 16: if constexpr (V <= 2) { ln_planes_bwd_kernel<T, V, 16><<<p.grid, p.threads, smem, s>>>(a, p.work); break; }
            case 32: if constexpr (V == 1) { ln_planes_bwd_kernel<T, V, 32><<<p.grid, p.threads, smem, s>>>(a, p.work); break; }
            default: ln_planes_bwd_long_kernel<T, V><<<p.grid, p.threads, smem, s>>>(a, p.work);
        }
    }
    return after_launch();
}
template <typename T> gf_status launch_norm(const NormArgs& a, const NormPlan& p, bool backward, cudaStream_t s) {
    if (p.planes) {
        switch (p.V) {
            case 4: return launch_planes_v<T, 4>(a, p, backward, s);
            case 2: return launch_planes_v<T, 2>(a, p, backward, s);
            default: return launch_planes_v<T, 1>(a, p, backward, s);
        }
    }
    if (p.NV == 0) {
        if (!backward) ln_rows_fwd_long_kernel<T><<<(unsigned)a.R, 1024, 0, s>>>(a);
        else ln_rows_bwd_long_kernel<T><<<p.grid, 1024, 0, s>>>(a);
        return after_launch();
    }
    switch (p.V) {
        case 8: if constexpr (sizeof(T) == 2) return launch_rows_v<T, 8>(a, p, backward, s);
        case 4: return launch_rows_v<T, 4>(a, p, backward, s);
        case 2: return launch_rows_v<T, 2>(a, p, backward, s);
        default: return launch_rows_v<T, 1>(a, p, backward, s);
    }
}

NormArgs norm_args(const gf_norm_desc& d) {
    NormArgs a = {};
    a.R = (long long)d.N * d.H * d.W;
    a.C = d.C;
    a.HW = d.H * d.W;
    a.div_hw = FastDiv((uint32_t)a.HW);
    a.eps = d.eps;
    a.inv_c = 1.0f / (float)d.C;
    return a;
}

}  // namespace
}  // namespace gf

using namespace gf;

extern "C" {

gf_status gf_layer_norm_forward(const gf_norm_desc* desc, const void* x, const void* gamma, const void* beta, void* y, float* mean,
                                float* rstd, void* stream) {
    gf_status st = norm_validate(desc);
    if (st != GF_OK) return st;
    if (desc->N == 0) return GF_OK;
    if (!x || !y || (mean == nullptr) != (rstd == nullptr)) return GF_ERR_NULL;
    if (misaligned16(x) || misaligned16(y) || misaligned16(gamma) || misaligned16(beta) || misaligned16(mean) || misaligned16(rstd))
        return GF_ERR_ALIGN;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const NormPlan p = norm_plan(*desc, false);
    NormArgs a = norm_args(*desc);
    a.x = x; a.out = y; a.mean = mean; a.rstd = rstd; a.log_tpr = p.log_tpr;
    a.gamma = {gamma, desc->param_dtype == GF_BF16};
    a.beta = {beta, desc->param_dtype == GF_BF16};
    ProfScope prof(K_NORM_FWD, s);
    return desc->dtype == GF_F32 ? launch_norm<float>(a, p, false, s) : launch_norm<__nv_bfloat16>(a, p, false, s);
}

gf_status gf_layer_norm_backward_workspace_bytes(const gf_norm_desc* desc, size_t* bytes) {
    if (!bytes) return GF_ERR_NULL;
    gf_status st = norm_validate(desc);
    if (st != GF_OK) return st;
    const NormPlan p = norm_plan(*desc, true);
    *bytes = (size_t)(p.grid > 0 ? p.grid : 1) * 2 * desc->C * 4;
    return GF_OK;
}

gf_status gf_layer_norm_backward(const gf_norm_desc* desc, const void* g_y, const void* x, const void* gamma, const float* mean,
                                 const float* rstd, void* g_x, float* g_gamma, float* g_beta, void* workspace,
                                 size_t workspace_bytes, void* stream) {
    size_t need = 0;
    gf_status st = gf_layer_norm_backward_workspace_bytes(desc, &need);
    if (st != GF_OK) return st;
    const bool sums = g_gamma || g_beta;
    if (desc->N > 0 && (!g_y || !x || !mean || !rstd || (sums && !workspace))) return GF_ERR_NULL;
    const void* all[] = {g_y, x, gamma, mean, rstd, g_x, g_gamma, g_beta, workspace};
    for (const void* ptr : all)
        if (misaligned16(ptr)) return GF_ERR_ALIGN;
    if (sums && desc->N > 0 && workspace_bytes < need) return GF_ERR_WORKSPACE;
    if (!g_x && !sums) return GF_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const NormPlan p = norm_plan(*desc, true);
    if (desc->N > 0) {
        NormArgs a = norm_args(*desc);
        a.x = x; a.gy = g_y; a.out = g_x; a.mean_in = mean; a.rstd_in = rstd; a.log_tpr = p.log_tpr;
        a.gamma = {gamma, desc->param_dtype == GF_BF16};
        a.part = sums ? static_cast<float*>(workspace) : nullptr;
        ProfScope prof(K_NORM_BWD, s);
        st = desc->dtype == GF_F32 ? launch_norm<float>(a, p, true, s) : launch_norm<__nv_bfloat16>(a, p, true, s);
        if (st != GF_OK) return st;
    }
    if (!sums) return GF_OK;
    ProfScope prof(K_NORM_SUMS, s);
    const long long cols = 2LL * desc->C;
    return launch_pdl(ln_finish_kernel, dim3((unsigned)((cols + kFinX - 1) / kFinX)), dim3(kFinX, kFinY), 0, s,
                      (const float*)workspace, desc->N > 0 ? p.grid : 0, (int)desc->C, g_gamma, g_beta);
}

}  // extern "C"

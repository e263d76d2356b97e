// Layer normalisation over the channels, forward and backward (gf_train.h).
//
// All of it is bound by memory in principle: forward reads x and writes y, backward reads x and g_y and writes g_x, once
// each; the sums over pixels leave one line of 2 C floats per block.  Two ways through the tensor: rows (channels
// last) and tiles of planes (channels first), each with a form for few pixels that loads directly and one for many that
// keeps the copy engine ahead.  The variance is taken about the mean from values held on chip.
#include <type_traits>

#include "gf_common.cuh"
#include "gf_pipe.cuh"
#include "gf_tma.cuh"
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

// ---- pairs of fp32 --------------------------------------------------------------------------
// Two fp32 operations per instruction, each half rounded as the scalar operation is; the loops below are bound by instructions
// and their latency (8192 x 4096 bf16 backward 53 -> 51 us).
__device__ __forceinline__ void fma2(float (&d)[2], float a0, float a1, float b0, float b1, float c0, float c1) {
    asm("{\n\t.reg .b64 a, b, c;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 c, a, b, c;\n\t"
        "mov.b64 {%0, %1}, c;\n\t}"
        : "=f"(d[0]), "=f"(d[1])
        : "f"(a0), "f"(a1), "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}
__device__ __forceinline__ void mul2(float (&d)[2], float a0, float a1, float b0, float b1) {
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(d[0]), "=f"(d[1])
        : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}
__device__ __forceinline__ void add2(float (&d)[2], float a0, float a1, float b0, float b1) {
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(d[0]), "=f"(d[1])
        : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}
// d = a b + c, a b, a + b over V values; S: a scalar in b's (c's) place.
template <int V> __device__ __forceinline__ void v_fma(float (&d)[V], const float (&a)[V], const float (&b)[V], const float (&c)[V]) {
    if constexpr (V == 1) d[0] = a[0] * b[0] + c[0];
    else {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            float r[2];
            fma2(r, a[i], a[i + 1], b[i], b[i + 1], c[i], c[i + 1]);
            d[i] = r[0]; d[i + 1] = r[1];
        }
    }
}
template <int V> __device__ __forceinline__ void v_fma(float (&d)[V], const float (&a)[V], float b, const float (&c)[V]) {
    float bb[V];
#pragma unroll
    for (int i = 0; i < V; ++i) bb[i] = b;
    v_fma<V>(d, a, bb, c);
}
template <int V> __device__ __forceinline__ void v_mul(float (&d)[V], const float (&a)[V], const float (&b)[V]) {
    if constexpr (V == 1) d[0] = a[0] * b[0];
    else {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            float r[2];
            mul2(r, a[i], a[i + 1], b[i], b[i + 1]);
            d[i] = r[0]; d[i + 1] = r[1];
        }
    }
}
template <int V> __device__ __forceinline__ void v_add(float (&d)[V], const float (&a)[V], const float (&b)[V]) {
    if constexpr (V == 1) d[0] = a[0] + b[0];
    else {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            float r[2];
            add2(r, a[i], a[i + 1], b[i], b[i + 1]);
            d[i] = r[0]; d[i + 1] = r[1];
        }
    }
}
template <int V> __device__ __forceinline__ void v_fill(float (&d)[V], float x) {
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] = x;
}
template <int V> __device__ __forceinline__ float v_sum(const float (&a)[V]) {
    float s = a[0];
#pragma unroll
    for (int i = 1; i < V; ++i) s += a[i];
    return s;
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
// taken about the mean.  For few rows, all of them in flight at once: 8 x 768 bf16 takes 4 us, of which the launch is
// most; the ring kernel below has its barriers to set up first and measured no faster until every team had two rows.
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

// Rows longer than the registers of a block (16384): the row is read again from L2 for each pass, an element at a time.
// 1024 x 20000 fp32: 80 us, a third of the copy bandwidth.
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
    extern __shared__ float cols[];                       // !WHOLE_BLOCK: [warps][2][C], at most 32 KB
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
        float* mine = cols + (size_t)(threadIdx.x >> 5) * 2 * a.C;
        if ((int)(threadIdx.x & 31) < tpr) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int c = (k * tpr + g) * V + i;
                    if (c < a.C) { mine[c] = ag[k][i]; mine[a.C + c] = ab[k][i]; }
                }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * a.C; c += blockDim.x) {
            float p = cols[c];
            for (int w = 1; w < (int)(blockDim.x >> 5); ++w) p += cols[(size_t)w * 2 * a.C + c];
            part[c] = p;
        }
    }
}

// Rows longer than the registers of a block (8192): two passes over the row (the second from L2); the
// column sums are kept in the block's line of the workspace, each by the thread that owns the column: read and written
// for every row, which is most of the time (2048 x 12288 fp32: 222 us for 46 of bytes; 4096 x 8192, in registers: 77 for 61).
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

// ---- rows through shared memory ---------------------------------------------------------------------
// For more rows than there are teams of threads: a team (part of a block that shares a row) has its own ring of batches
// of whole rows, which the copy engine fills some batches ahead, so that the loads of the next rows run under
// the sums and stores of the present one.  A batch is one contiguous piece of memory, copied from the 16-byte
// boundary before it to the one after it.  The last bytes of a tensor whose size is no multiple of 16 are fetched with
// plain loads.
// Measured: 100352 x 576 fp32 forward 83 to 88 us, 5.3 to 5.6 TB/s (0.80 to 0.85 of the copy bandwidth), bf16 78 us
// (0.45); 8192 x 4096 bf16 backward 47 us and 4 us
// for the lines of sums, 4.3 TB/s: 8 warps per SM (the sums take their registers), about 7 us of it start and
// end; two rows at once with one exchange measured the same, 16 elements per thread and 16 warps measured 56 us in all.
//   SHIFT: rows whose length is no multiple of 16 bytes, one to a batch.  The number of teams is a multiple of the period (at most
//   8) with which the rows' offsets from a 16-byte boundary repeat, so that all rows of a team have the same
//   offset: its threads own whole aligned vectors, the first and last of which are partly the neighbouring rows'.
//   (4099 x 1001 fp32 backward: 16 us; element by element 23 us.)
struct RingArgs {
    int warps;                 // per team
    int stages, rows;          // batches in flight per team; rows per batch
    int stage_bytes;           // of one tensor's batch
    long long batches;
    uint32_t* err_word;
};

template <bool TEAM> __device__ __forceinline__ void team_sync(int team, int warps) {
    if constexpr (TEAM) asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(warps * 32) : "memory");
    else __syncwarp();
}

// Sums of N values over the threads that share a row (part of a warp, or a team of warps through `red` [N][16]).
template <bool TEAM, int N> __device__ __forceinline__ void team_sum(float (&s)[N], int log_tpr, float* red, int team, int warps) {
    if constexpr (TEAM) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int n = 0; n < N; ++n) s[n] += __shfl_xor_sync(0xffffffffu, s[n], o);
        const int w = (threadIdx.x >> 5) - team * warps;
        if ((threadIdx.x & 31) == 0) {
#pragma unroll
            for (int n = 0; n < N; ++n) red[n * 16 + w] = s[n];
        }
        team_sync<TEAM>(team, warps);
#pragma unroll
        for (int n = 0; n < N; ++n) {                       // places past the team's warps hold zeros
            const float4 p = *reinterpret_cast<const float4*>(red + n * 16);
            s[n] = (p.x + p.y) + (p.z + p.w);
            for (int k = 4; k < warps; k += 4) {
                const float4 q = *reinterpret_cast<const float4*>(red + n * 16 + k);
                s[n] += (q.x + q.y) + (q.z + q.w);
            }
        }
    } else {
        for (int o = (1 << log_tpr) >> 1; o > 0; o >>= 1)
#pragma unroll
            for (int n = 0; n < N; ++n) s[n] += __shfl_xor_sync(0xffffffffu, s[n], o);
    }
}

template <typename T, int V, int E, bool TEAM, bool BWD, bool SHIFT>
__global__ void __launch_bounds__(BWD ? 256 : 512) ln_rows_ring_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ RingArgs r) {
    constexpr int NV = E / V, NT = BWD ? 2 : 1;
    extern __shared__ __align__(128) unsigned char dyn[];
    __shared__ uint64_t full[8 * 8];                       // [team][stage]
    __shared__ __align__(16) float red[8][2][2 * 16];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int team = warp / r.warps, teams = (int)(blockDim.x >> 5) / r.warps;
    const int tid = threadIdx.x - team * r.warps * 32;      // within the team
    const int tpr = 1 << a.log_tpr, g = TEAM ? tid : tid & (tpr - 1);
    const int rows_at_once = TEAM ? 1 : 32 >> a.log_tpr;
    const int step = tpr * V;                               // columns between a thread's vectors
    const long long teams_all = (long long)gridDim.x * teams, first = (long long)blockIdx.x * teams + team;
    const int row_bytes = a.C * (int)sizeof(T);
    const long long total16 = (a.R * row_bytes) & ~15LL;    // whole 16-byte pieces of the tensor
    unsigned char* ring = dyn + (size_t)team * r.stages * NT * r.stage_bytes;
    if (threadIdx.x == 0) {
        for (int k = 0; k < teams * r.stages; ++k) mbar_init(&full[k], 1);
        mbar_fence_init();
    }
    if (TEAM)
        for (int k = threadIdx.x; k < 8 * 2 * 2 * 16; k += blockDim.x) (&red[0][0][0])[k] = 0.f;
    __syncthreads();
    const int shift = SHIFT ? (int)((first * row_bytes) & 15) / (int)sizeof(T) : 0;      // elements before the row in its first vector
    const int C = a.C + shift;                              // end of the row, counted from there
    // element i of the thread's vector k is in the row
    auto inside = [&](int k, int i) { const int c = k * step + g * V + i; return c >= shift && c < C; };
    // the vector is wholly in the row (for all vectors but a row's first and last one)
    auto whole = [&](int k) { return !SHIFT || ((k > 0 || g > 0 || shift == 0) && k * step + g * V + V <= C); };
    auto load = [&](long long b, int s) {                   // by one thread
        const long long lo = (b * r.rows * row_bytes) & ~15LL;
        long long hi = ((b + 1) * r.rows < a.R ? (b + 1) * r.rows : a.R) * row_bytes;
        hi = (hi + 15) & ~15LL;
        if (hi > total16) hi = total16;
        const uint32_t bytes = hi > lo ? (uint32_t)(hi - lo) : 0u;
        uint64_t* bar = &full[team * r.stages + s];
        mbar_expect_tx(bar, bytes * NT);
        if (bytes == 0) return;
        unsigned char* dst = ring + (size_t)s * NT * r.stage_bytes;
        bulk_g2s(dst, static_cast<const unsigned char*>(a.x) + lo, bytes, bar);
        if constexpr (BWD) bulk_g2s(dst + r.stage_bytes, static_cast<const unsigned char*>(a.gy) + lo, bytes, bar);
    };
    if (tid == 0)
        for (int s = 0; s < r.stages; ++s)
            if (first + s * teams_all < r.batches) load(first + s * teams_all, s);

    float gam[NV][V], bet[BWD ? 1 : NV][V], ag[BWD ? NV : 1][V], ab[BWD ? NV : 1][V];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = k * step + g * V + i - shift;
            gam[k][i] = inside(k, i) ? a.gamma.at(c, 1.f) : 0.f;
            if constexpr (!BWD) bet[k][i] = inside(k, i) ? a.beta.at(c, 0.f) : 0.f;
            else ag[k][i] = ab[k][i] = 0.f;
        }
    float mean_n = 0.f, rstd_n = 0.f;                       // of row `lane` of the next batch
    auto stats = [&](long long b) {
        const long long row = b * r.rows + lane;
        const bool there = b < r.batches && lane < r.rows && row < a.R;
        mean_n = there ? a.mean_in[row] : 0.f;
        rstd_n = there ? a.rstd_in[row] : 0.f;
    };
    if constexpr (BWD) stats(first);

    bool ok = true;
    int s = 0, slot = 0;
    uint32_t parity = 0;
    for (long long b = first; b < r.batches; b += teams_all) {
        // once a wait has run out nothing is waited for any more: the results are void, which the error word says
        if (ok) ok = mbar_wait_bounded(&full[team * r.stages + s], parity);
        const long long r0 = b * r.rows, lo = (r0 * row_bytes) & ~15LL;
        const int nr = (int)(a.R - r0 < r.rows ? a.R - r0 : r.rows);
        unsigned char* sx = ring + (size_t)s * NT * r.stage_bytes;
        if ((r0 + nr) * row_bytes > total16) {              // the tensor's last bytes
            const long long from = lo > total16 ? lo : total16;
            const int n = (int)(((r0 + nr) * row_bytes - from) / (long long)sizeof(T));
            if (tid < n) {
                reinterpret_cast<T*>(sx + (from - lo))[tid] = reinterpret_cast<const T*>(static_cast<const unsigned char*>(a.x) + from)[tid];
                if constexpr (BWD)
                    reinterpret_cast<T*>(sx + r.stage_bytes + (from - lo))[tid] =
                        reinterpret_cast<const T*>(static_cast<const unsigned char*>(a.gy) + from)[tid];
            }
            team_sync<TEAM>(team, r.warps);
        }
        const float mean_b = mean_n, rstd_b = rstd_n;
        if constexpr (BWD) stats(b + teams_all);
        const int row_in = TEAM ? 0 : lane >> a.log_tpr;    // of the rows that the warp has at once
        const T* x = reinterpret_cast<const T*>(sx + (SHIFT ? 0 : (int)(r0 * row_bytes - lo)) + row_in * row_bytes) + g * V;
        T* out = static_cast<T*>(a.out) + ((r0 + row_in) * a.C - shift) + g * V;
        for (int q = 0; q < nr; q += rows_at_once, slot ^= 1, x += rows_at_once * a.C, out += rows_at_once * a.C) {
            const int k_row = q + row_in;
            const int width = TEAM || k_row < nr ? C - g * V : 0;        // columns from this thread's first on
            float v[NV][V];
            auto put = [&](int k) {
                if (whole(k)) store_vec<T, V>(out + k * step, v[k]);
                else {
#pragma unroll
                    for (int i = 0; i < V; ++i) if (inside(k, i)) out[k * step + i] = from_f32<T>(v[k][i]);
                }
            };
            if constexpr (!BWD) {
                float sum[1], var[1], s1[V], minus_mean[V], rstd_v[V];
                v_fill<V>(s1, 0.f);
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    if (k * step >= C) break;               // the same for all threads
                    if (k * step < width) {
                        load_vec<T, V>(x + k * step, v[k]);
                        if (!whole(k)) {
#pragma unroll
                            for (int i = 0; i < V; ++i) if (!inside(k, i)) v[k][i] = 0.f;
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < V; ++i) v[k][i] = 0.f;
                    }
                    v_add<V>(s1, s1, v[k]);
                }
                sum[0] = v_sum<V>(s1);
                team_sum<TEAM, 1>(sum, a.log_tpr, red[team][0], team, r.warps);
                const float mean = sum[0] / (float)a.C;
                v_fill<V>(minus_mean, -mean);
                v_fill<V>(s1, 0.f);
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    if (k * step >= C) break;
                    if (k * step < width) {
                        v_add<V>(v[k], v[k], minus_mean);
                        if (!whole(k)) {
#pragma unroll
                            for (int i = 0; i < V; ++i) if (!inside(k, i)) v[k][i] = 0.f;
                        }
                        v_fma<V>(s1, v[k], v[k], s1);
                    }
                }
                var[0] = v_sum<V>(s1);
                team_sum<TEAM, 1>(var, a.log_tpr, red[team][1], team, r.warps);
                const float rstd = rsqrtf(var[0] * a.inv_c + a.eps);
                v_fill<V>(rstd_v, rstd);
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    if (k * step >= C) break;
                    if (k * step < width) {
                        v_mul<V>(v[k], v[k], rstd_v);
                        v_fma<V>(v[k], v[k], gam[k], bet[k]);
                        put(k);
                    }
                }
                if (a.mean && g == 0 && width > 0) { a.mean[r0 + k_row] = mean; a.rstd[r0 + k_row] = rstd; }
            } else {
                const T* gy = reinterpret_cast<const T*>(reinterpret_cast<const unsigned char*>(x) + r.stage_bytes);
                const float mean = __shfl_sync(0xffffffffu, mean_b, k_row & 31), rstd = __shfl_sync(0xffffffffu, rstd_b, k_row & 31);
                float gv[NV][V], s1[V], s2[V], minus_mean[V], rstd_v[V];
                v_fill<V>(s1, 0.f);
                v_fill<V>(s2, 0.f);
                v_fill<V>(minus_mean, -mean);
                v_fill<V>(rstd_v, rstd);
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    if (k * step >= C) break;
                    if (k * step < width) {
                        load_vec<T, V>(x + k * step, v[k]);
                        load_vec<T, V>(gy + k * step, gv[k]);
                        if (!whole(k)) {
#pragma unroll
                            for (int i = 0; i < V; ++i) if (!inside(k, i)) { v[k][i] = mean; gv[k][i] = 0.f; }
                        }
                    } else {                                // xh = 0 and gy = 0: adds nothing
#pragma unroll
                        for (int i = 0; i < V; ++i) { v[k][i] = mean; gv[k][i] = 0.f; }
                    }
                    v_add<V>(v[k], v[k], minus_mean);
                    v_mul<V>(v[k], v[k], rstd_v);
                    v_fma<V>(ag[k], gv[k], v[k], ag[k]);
                    v_add<V>(ab[k], ab[k], gv[k]);
                    v_mul<V>(gv[k], gv[k], gam[k]);
                    v_add<V>(s1, s1, gv[k]);
                    v_fma<V>(s2, gv[k], v[k], s2);
                }
                float sum[2] = {v_sum<V>(s1), v_sum<V>(s2)};
                if (a.out) {
                    team_sum<TEAM, 2>(sum, a.log_tpr, red[team][slot], team, r.warps);
                    float minus_m1[V], minus_m2[V];
                    v_fill<V>(minus_m1, -(sum[0] * a.inv_c * rstd));
                    v_fill<V>(minus_m2, -(sum[1] * a.inv_c * rstd));
#pragma unroll
                    for (int k = 0; k < NV; ++k) {
                        if (k * step >= C) break;
                        if (k * step < width) {
                            v_fma<V>(gv[k], gv[k], rstd_v, minus_m1);
                            v_fma<V>(v[k], v[k], minus_m2, gv[k]);
                            put(k);
                        }
                    }
                }
            }
        }
        team_sync<TEAM>(team, r.warps);                     // the batch has been read
        // after a wait that ran out no copy is started: its barrier may still be in the phase before
        if (tid == 0 && ok && b + r.stages * teams_all < r.batches) load(b + r.stages * teams_all, s);
        if (++s == r.stages) { s = 0; parity ^= 1u; }
    }
    if (!ok) {
        atomicOr(r.err_word, 8192u);
        let_settle();
    }
    if constexpr (BWD) {
        if (!a.part) return;
        float* cols = reinterpret_cast<float*>(dyn);        // [teams][2][C]
        float* part = a.part + (size_t)blockIdx.x * 2 * a.C;
        if constexpr (!TEAM) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i)
                    for (int o = tpr; o < 32; o <<= 1) {    // lanes of a warp that hold the same columns
                        ag[k][i] += __shfl_xor_sync(0xffffffffu, ag[k][i], o);
                        ab[k][i] += __shfl_xor_sync(0xffffffffu, ab[k][i], o);
                    }
        }
        __syncthreads();
        // every team leaves its sums over the rings; then a thread per column adds them in the teams' order
        if (tid < tpr) {
            float* mine = cols + (size_t)team * 2 * a.C;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int c = k * step + g * V + i - shift;
                    if (inside(k, i)) { mine[c] = ag[k][i]; mine[a.C + c] = ab[k][i]; }
                }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * a.C; c += blockDim.x) {
            float p = cols[c];
            for (int w = 1; w < teams; ++w) p += cols[(size_t)w * 2 * a.C + c];
            part[c] = p;
        }
    }
}

// ---- channels first --------------------------------------------------------------------------
// For small planes of odd size, and more channels than the tiles below hold (128 x 768 x 7 x 7 fp32: forward 48 us, backward 58,
// for 6 and 9 us of bytes; bf16 128 x 768 x 14 x 14: 60 and 157 for 12 and 18): a block takes 32 V consecutive pixels (lane = pixel, V
// per lane) and all channels; warp w of CG
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

// ---- channels first, through shared memory ------------------------------------------------------------
// A block takes the same few consecutive pixels of all channels of an image at a time: a tile of C short rows, of
// which several are on their way while one is worked on.  LP lanes lie along the pixels, 32 / LP along the
// channels, so that the sums over channels (per pixel) are sums in registers and a few exchanges per tile,
// and the sums over pixels (per channel) stay in a thread's registers for the whole kernel.  The tile is read
// from shared memory once per pass over it (two backward, three forward).
// Measured: 256 x 512 x 16 x 16 fp32 backward 77 us and 3 us for the lines of sums, 5.2 TB/s; 128 x 576 x 28 x 28 fp32, whose rows
// are 64 bytes long forward and 32 backward (longer ones of 576 channels do not fit three times), 129 and 177 us, 0.55 and 0.60 of the
// copy bandwidth; 64 x 96 x 55 x 55 bf16 forward 35 us,
// 2.2 TB/s: planes of odd size are read and written a pixel at a time, about 30 instructions per pixel and channel (tiles of
// 128 pixels 37 us, of 8 warps 53).
//   WHOLE: every row of a plane starts on a 16-byte boundary; tiles come as boxes of the copy engine, a lane has a
//          16-byte vector of pixels.
//   else : planes of odd size.  Each row is copied in 16-byte pieces from the boundary before it (its offset differs from
//          channel to channel); 32 lanes read and write single pixels, PX of them each.
struct PlaneArgs {
    CUtensorMap tm_x, tm_gy;   // WHOLE
    int boxes, box_rows;       // boxes of a tile (channels), rows of each
    int px, tiles_per_img;
    int pitch;                 // bytes of a channel's row in shared memory
    int stage_bytes;           // of one tensor's tile
    int stages;
    long long tiles;
    FastDiv div_tiles;
    int log_pieces;            // else: 16-byte pieces of a row, rounded up to a power of two
    uint32_t* err_word;
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// PX = 0: WHOLE, with 8 warps; 16 warps else (more instructions per byte)
constexpr int plane_warps(int PX) { return PX == 0 ? 8 : 16; }
template <typename T, int LP, int KC, int PX, bool BWD>
__global__ void __launch_bounds__((PX == 0 ? 8 : 16) * 32) ln_planes_tile_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ PlaneArgs t) {
    constexpr bool WHOLE = PX == 0;
    constexpr int kPlaneWarps = PX == 0 ? 8 : 16, kPlaneThreads = kPlaneWarps * 32;
    constexpr int NT = BWD ? 2 : 1, E = (int)sizeof(T);
    constexpr int V = WHOLE ? 16 / E : PX;                 // pixels of a thread
    constexpr int PT = LP * V;                              // pixels of a tile
    constexpr int CL = 32 / LP;                             // channels of a warp at once
    extern __shared__ __align__(128) unsigned char dyn[];
    __shared__ uint64_t full[8];
    __shared__ float red[kPlaneWarps * NT * PT];
    __shared__ float stat[NT * PT];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int cl = lane / LP, pl = lane % LP;
    auto pixel = [&](int i) { return WHOLE ? pl * V + i : pl + 32 * i; };
    auto place = [&](long long tile, uint32_t& n, int& p0) {
        uint32_t k;
        t.div_tiles.divmod((uint32_t)tile, n, k);
        p0 = (int)k * t.px;
    };
    auto load = [&](long long tile, int s) {
        unsigned char* dst = dyn + (size_t)s * NT * t.stage_bytes;
        if constexpr (WHOLE) {
            if (tid != 0 || tile >= t.tiles) return;
            uint32_t n;
            int p0;
            place(tile, n, p0);
            mbar_expect_tx(&full[s], (uint32_t)(t.boxes * t.box_rows * t.pitch * NT));
            for (int k = 0; k < t.boxes; ++k) {
                tma_load_3d(dst + k * t.box_rows * t.pitch, &t.tm_x, p0, k * t.box_rows, (int)n, &full[s]);
                if constexpr (BWD) tma_load_3d(dst + t.stage_bytes + k * t.box_rows * t.pitch, &t.tm_gy, p0, k * t.box_rows, (int)n, &full[s]);
            }
        } else {
            if (tile < t.tiles) {
                uint32_t n;
                int p0;
                place(tile, n, p0);
                const int np = min(t.px, a.HW - p0);
                const int piece = tid & ((1 << t.log_pieces) - 1), c0 = tid >> t.log_pieces, dc = kPlaneThreads >> t.log_pieces;
                const long long plane = (long long)a.HW * E, total = a.R * a.C * E, skip = plane * dc;
                long long row = (long long)n * a.C * plane + (long long)p0 * E + c0 * plane;
                uint32_t to = smem_u32(dst) + c0 * t.pitch + piece * 16;
                for (int c = c0; c < a.C; c += dc, row += skip, to += dc * t.pitch) {
                    const long long at = (row & ~15LL) + piece * 16;
                    if (at < row + np * E) {
                        const int bytes = total - at < 16 ? (int)(total - at) : 16;
                        cp_async16(to, static_cast<const unsigned char*>(a.x) + at, bytes);
                        if constexpr (BWD) cp_async16(to + t.stage_bytes, static_cast<const unsigned char*>(a.gy) + at, bytes);
                    }
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    if constexpr (WHOLE) {
        if (tid == 0) {
            for (int s = 0; s < t.stages; ++s) mbar_init(&full[s], 1);
            mbar_fence_init();
        }
        __syncthreads();
    }
    for (int s = 0; s < t.stages - (WHOLE ? 0 : 1); ++s) load(blockIdx.x + (long long)s * gridDim.x, s);

    constexpr bool kPar = KC <= 16;                         // gamma and beta in registers (else from L1)
    constexpr bool kHold = KC * V * NT <= 64;               // the tile in registers between the passes (else from shared memory)
    float gam[kPar ? KC : 1], bet[kPar && !BWD ? KC : 1], ag[BWD ? KC : 1], ab[BWD ? KC : 1];
#pragma unroll
    for (int k = 0; k < KC; ++k) {
        const int c = (k * kPlaneWarps + warp) * CL + cl;
        if constexpr (kPar) gam[k] = c < a.C ? a.gamma.at(c, 1.f) : 0.f;
        if constexpr (kPar && !BWD) bet[k] = c < a.C ? a.beta.at(c, 0.f) : 0.f;
        if constexpr (BWD) ag[k] = ab[k] = 0.f;
    }
    auto gamma_of = [&](int k, int c) { if constexpr (kPar) return gam[k]; else return a.gamma.at(c, 1.f); };
    auto beta_of = [&](int k, int c) { if constexpr (kPar && !BWD) return bet[k]; else return a.beta.at(c, 0.f); };
    // Sums over the channels of N values per pixel.  Over the CL lanes of a warp that hold the same pixels an exchange halves the
    // values a lane is responsible for, as long as there are two; then the warps through `red`; they end in stat[n * PT + pixel].
    auto over_channels = [&](auto& v) {
        constexpr int N = (int)(sizeof(v) / sizeof(float)) / V;
        constexpr int M = N * V;
        float w[M];
#pragma unroll
        for (int k = 0; k < M; ++k) w[k] = v[k / V][k % V];
        int at = 0;                                         // first of the values that this lane is left with
#pragma unroll
        for (int step = 0; (CL >> step) > 1; ++step) {
            const int o = 16 >> step, m = M >> step;
            if (m > 1) {
                const bool up_half = (lane & o) != 0;
                at += up_half ? m / 2 : 0;
#pragma unroll
                for (int k = 0; k < M / 2; ++k)
                    if (k < m / 2) {
                        const float send = up_half ? w[k] : w[k + m / 2];
                        w[k] = (up_half ? w[k + m / 2] : w[k]) + __shfl_xor_sync(0xffffffffu, send, o);
                    }
            } else w[0] += __shfl_xor_sync(0xffffffffu, w[0], o);
        }
        constexpr int left = M / CL > 0 ? M / CL : 1;
        // (lanes that share a value write it together)
#pragma unroll
        for (int k = 0; k < left; ++k) {
            const int q = at + k, n = q / V, i = q - n * V;
            red[warp * (NT * PT) + n * PT + pixel(i)] = w[k];
        }
        __syncthreads();
        for (int k = tid; k < N * PT; k += kPlaneThreads) {
            float s = 0.f;
#pragma unroll
            for (int u = 0; u < kPlaneWarps; ++u) s += red[u * (NT * PT) + k];
            stat[k] = s;
        }
        __syncthreads();
    };
    bool ok = true;
    int s = 0;
    uint32_t parity = 0;
    for (long long tile = blockIdx.x; tile < t.tiles; tile += gridDim.x) {
        uint32_t n;
        int p0;
        place(tile, n, p0);
        const int np = min(t.px, a.HW - p0);
        const long long q0 = (long long)n * a.HW + p0;
        float mean[V], rstd[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            mean[i] = rstd[i] = 0.f;
            if constexpr (BWD) {
                if (pixel(i) < np) { mean[i] = a.mean_in[q0 + pixel(i)]; rstd[i] = a.rstd_in[q0 + pixel(i)]; }
            }
        }
        if constexpr (WHOLE) {
            // once a wait has run out nothing is waited for any more: the results are void, which the error word says
            if (ok) ok = mbar_wait_bounded(&full[s], parity);
        } else {
            if (t.stages == 3) asm volatile("cp.async.wait_group 1;" ::: "memory");
            else asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncthreads();                                // this tile is here; the one before it has been read
            load(tile + (long long)(t.stages - 1) * gridDim.x, s == 0 ? t.stages - 1 : s - 1);
        }
        const unsigned char* sx = dyn + (size_t)s * NT * t.stage_bytes;
        const long long base = ((long long)n * a.C * a.HW + p0);      // of channel 0, in elements
        // A thread's channels lie kPlaneWarps * CL apart: 16 with planes of odd size, so that all of them have the same offset
        // from a 16-byte boundary.
        const int c_first = warp * CL + cl;
        const uint32_t off16 = ((uint32_t)(base * E) + (uint32_t)c_first * (uint32_t)((long long)a.HW * E & 15)) & 15u;
        const uint32_t in_tile = WHOLE ? (uint32_t)(c_first * (PT * E) + pl * 16) : (uint32_t)(c_first * t.pitch + pl * E) + off16;
        const uint32_t in_step = (uint32_t)(kPlaneWarps * CL) * (WHOLE ? (uint32_t)(PT * E) : (uint32_t)t.pitch);
        T* const out0 = static_cast<T*>(a.out) + base + (long long)c_first * a.HW + (WHOLE ? pl * V : pl);
        const long long out_step = (long long)(kPlaneWarps * CL) * a.HW;
        bool there[V];                                      // the thread's pixels are in the tile
#pragma unroll
        for (int i = 0; i < V; ++i) there[i] = pixel(i) < np;
        auto fetch = [&](const unsigned char* from, int k, float (&f)[V]) {
            const T* row = reinterpret_cast<const T*>(from + in_tile + (uint32_t)k * in_step);
            if constexpr (WHOLE) load_vec<T, V>(row, f);
            else {
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] = !BWD || there[i] ? to_f32(row[32 * i]) : 0.f;      // forward, a pixel is alone
            }
        };
        auto put = [&](int k, const float (&f)[V]) {
            T* dst = out0 + k * out_step;
            if constexpr (WHOLE) {
                if (there[0]) store_vec<T, V>(dst, f);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) if (there[i]) dst[32 * i] = from_f32<T>(f[i]);
            }
        };
        float xs[kHold ? KC : 1][V], gs[kHold && BWD ? KC : 1][V], minus_mean[V];
#pragma unroll
        for (int i = 0; i < V; ++i) minus_mean[i] = -mean[i];
        if constexpr (BWD) {
            float sum[2][V];
#pragma unroll
            for (int i = 0; i < V; ++i) sum[0][i] = sum[1][i] = 0.f;
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                const int c = (k * kPlaneWarps + warp) * CL + cl, at = kHold ? k : 0;
                if (c < a.C) {
                    fetch(sx, k, xs[at]);
                    fetch(sx + t.stage_bytes, k, gs[at]);
                    const float gm = gamma_of(k, c);
                    float w[V];
                    v_add<V>(xs[at], xs[at], minus_mean);
                    v_mul<V>(xs[at], xs[at], rstd);
                    v_mul<V>(w, gs[at], xs[at]);
                    ag[k] += v_sum<V>(w);
                    ab[k] += v_sum<V>(gs[at]);
                    v_fill<V>(w, gm);
                    v_mul<V>(gs[at], gs[at], w);
                    v_add<V>(sum[0], sum[0], gs[at]);
                    v_fma<V>(sum[1], gs[at], xs[at], sum[1]);
                }
            }
            if (a.out) {
                over_channels(sum);
                float m1[V], m2[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    m1[i] = -(stat[pixel(i)] * a.inv_c * rstd[i]);
                    m2[i] = -(stat[PT + pixel(i)] * a.inv_c * rstd[i]);
                }
#pragma unroll
                for (int k = 0; k < KC; ++k) {
                    const int c = (k * kPlaneWarps + warp) * CL + cl, at = kHold ? k : 0;
                    if (c < a.C) {
                        if constexpr (!kHold) {
                            fetch(sx, k, xs[at]);
                            fetch(sx + t.stage_bytes, k, gs[at]);
                            const float gm = gamma_of(k, c);
#pragma unroll
                            for (int i = 0; i < V; ++i) { xs[at][i] = (xs[at][i] - mean[i]) * rstd[i]; gs[at][i] *= gm; }
                        }
                        v_fma<V>(gs[at], gs[at], rstd, m1);
                        v_fma<V>(xs[at], xs[at], m2, gs[at]);
                        put(k, xs[at]);
                    }
                }
            }
        } else {
            float sum[1][V];
#pragma unroll
            for (int i = 0; i < V; ++i) sum[0][i] = 0.f;
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                const int c = (k * kPlaneWarps + warp) * CL + cl, at = kHold ? k : 0;
                if (c < a.C) {
                    fetch(sx, k, xs[at]);
#pragma unroll
                    for (int i = 0; i < V; ++i) sum[0][i] += xs[at][i];
                }
            }
            over_channels(sum);
#pragma unroll
            for (int i = 0; i < V; ++i) { mean[i] = stat[pixel(i)] / (float)a.C; sum[0][i] = 0.f; }
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                const int c = (k * kPlaneWarps + warp) * CL + cl, at = kHold ? k : 0;
                if (c < a.C) {
                    if constexpr (!kHold) fetch(sx, k, xs[at]);
#pragma unroll
                    for (int i = 0; i < V; ++i) { xs[at][i] -= mean[i]; sum[0][i] += xs[at][i] * xs[at][i]; }
                }
            }
            over_channels(sum);
#pragma unroll
            for (int i = 0; i < V; ++i) rstd[i] = rsqrtf(stat[pixel(i)] * a.inv_c + a.eps);
            if (a.mean && warp == 0 && cl == 0) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (pixel(i) < np) { a.mean[q0 + pixel(i)] = mean[i]; a.rstd[q0 + pixel(i)] = rstd[i]; }
            }
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                const int c = (k * kPlaneWarps + warp) * CL + cl, at = kHold ? k : 0;
                if (c < a.C) {
                    if constexpr (!kHold) {
                        fetch(sx, k, xs[at]);
#pragma unroll
                        for (int i = 0; i < V; ++i) xs[at][i] -= mean[i];
                    }
                    const float gm = gamma_of(k, c), bt = beta_of(k, c);
#pragma unroll
                    for (int i = 0; i < V; ++i) xs[at][i] = xs[at][i] * rstd[i] * gm + bt;
                    put(k, xs[at]);
                }
            }
        }
        if constexpr (WHOLE) {
            __syncthreads();                                // the tile has been read
            if (ok) load(tile + (long long)t.stages * gridDim.x, s);      // (none after a wait that ran out: its barrier may be in the phase before)
        }
        if (++s == t.stages) { s = 0; parity ^= 1u; }
    }
    if (!ok) {
        atomicOr(t.err_word, 8192u);
        let_settle();
    }
    if constexpr (BWD) {
        if (!a.part) return;
        float* part = a.part + (size_t)blockIdx.x * 2 * a.C;
#pragma unroll
        for (int k = 0; k < KC; ++k) {
#pragma unroll
            for (int o = LP >> 1; o > 0; o >>= 1) {
                ag[k] += __shfl_xor_sync(0xffffffffu, ag[k], o);
                ab[k] += __shfl_xor_sync(0xffffffffu, ab[k], o);
            }
            const int c = (k * kPlaneWarps + warp) * CL + cl;
            if (pl == 0 && c < a.C) { part[c] = ag[k]; part[a.C + c] = ab[k]; }
        }
    }
}

// ---- sums of the blocks' lines -------------------------------------------------------------------
// part [blocks][2 C] -> g_gamma, g_beta: the blocks in a fixed order.
constexpr int kFinX = 32, kFinY = 32;
__global__ void __launch_bounds__(kFinX * kFinY) ln_finish_kernel(const float* part, int blocks, int C, float* g_gamma, float* g_beta, uint32_t* status) {
    __shared__ float red[kFinY][kFinX + 1];
    pdl_wait();
    if (status && blockIdx.x == 0 && threadIdx.x == 0 && threadIdx.y == 0) *status = 0;
    const long long col = (long long)blockIdx.x * kFinX + threadIdx.x;
    float s = 0.f;
    if (col < 2LL * C) {
#pragma unroll 10
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

// Which kernel a call takes.
enum NormKind { ROWS_DIRECT, ROWS_LONG, ROWS_RING, PLANES_DIRECT, PLANES_LONG, PLANES_TILE };
struct NormPlan {
    NormKind kind;
    int V;                // elements per load
    int log_tpr, E;       // rows: threads per row; elements per thread
    bool shift;           // rows off 16-byte boundaries, taken as aligned vectors
    int CG, NCH;          // planes, direct: warps, channels per warp
    int threads;
    long long work;       // blocks of work (row groups, or pixel tiles)
    int grid;             // persistent blocks
    size_t smem;
    RingArgs ring;
    PlaneArgs tile;
    int KC, LP, PX;       // planes, tiles (PX = 0: whole 16-byte pieces)
};

// Widest load that keeps every row (plane) on its boundary.
int vec_for(long long n, int esize) {
    int v = 16 / esize;
    while (n % v != 0) v >>= 1;
    return v;
}

constexpr size_t kNormSmem = 220 * 1024;

void plan_rows(const gf_norm_desc& d, bool backward, long long R, NormPlan& p) {
    const int e = d.dtype == GF_F32 ? 4 : 2;
    const int max_log = backward ? 8 : 9;
    const long long row_bytes = (long long)d.C * e;
    // A thread holds up to 32 elements, so that the work per row (exchanges, statistics) is shared by many of them;
    // two lanes at least share a row of more than 8.
    auto share_out = [&](int V, long long vecs) {
        auto fits = [&](int lt, int el) { return vecs <= (long long)(el / V) << lt; };
        p.V = V;
        p.E = 8;
        p.log_tpr = 0;
        if (!fits(1, 8)) p.E = 16;
        if (!fits(2, 16)) p.E = 32;
        while (p.log_tpr < max_log && !fits(p.log_tpr, p.E)) ++p.log_tpr;
        return fits(p.log_tpr, p.E);
    };
    auto plain = [&] { const int V = vec_for(d.C, e); return share_out(V, d.C / V); };
    // Long rows off the 16-byte boundaries: aligned vectors, with a row of their own for each copy (short rows are
    // better copied many at a time, and read element by element).
    const int full = 16 / e;
    auto shifted = [&] {
        const long long vecs = (d.C + 2 * full - 2) / full;
        p.V = full;
        p.log_tpr = 5;                                   // a warp at least: the batch is one row
        for (p.E = 8; p.E < 32 && vecs > 32LL * (p.E / full); p.E *= 2) {}
        while (p.log_tpr < max_log && vecs > (long long)(p.E / full) << p.log_tpr) ++p.log_tpr;
        return vecs <= (long long)(p.E / full) << p.log_tpr;
    };
    p.shift = row_bytes % 16 != 0 && row_bytes >= 512;
    if (!(p.shift ? shifted() : plain())) {
        p.kind = ROWS_LONG;
        p.threads = 1024;
        p.work = R;
        p.grid = (int)(R < sm_count() ? R : sm_count());
        return;
    }
    p.threads = p.log_tpr > 8 ? 1 << p.log_tpr : kRowThreads;
    // The ring: per team of warps, batches of whole rows, three on their way.  Forward, two blocks per SM; backward a
    // thread's sums take the registers of one.
    const int nt = backward ? 2 : 1;
    const int warps = p.log_tpr > 5 ? 1 << (p.log_tpr - 5) : 1, teams = p.threads / 32 / warps;
    const int at_once = p.log_tpr > 5 ? 1 : 32 >> p.log_tpr;
    RingArgs& r = p.ring;
    r.warps = warps;
    int per_sm = backward ? 1 : 2;
    if (kNormSmem / per_sm / teams / nt < (size_t)(2 * (row_bytes + 160))) per_sm = 1;
    const long long all = (long long)per_sm * sm_count() * teams;
    const long long budget = (long long)(kNormSmem / per_sm / teams / nt);       // of one tensor's batches
    long long rows = (budget / 3 - 160) / row_bytes;
    const long long fair = R / (all * 3);                // at least three batches for every team
    if (rows > fair) rows = fair;
    if (rows > 32) rows = 32;
    rows = rows / at_once * at_once;
    if (rows < at_once) rows = at_once;
    if (p.shift) rows = 1;                               // at_once is 1 too
    r.rows = (int)rows;
    r.stage_bytes = (int)((rows * row_bytes + 32 + 127) / 128 * 128);
    r.stages = (int)(budget / r.stage_bytes > 4 ? 4 : budget / r.stage_bytes);
    r.batches = (R + rows - 1) / rows;
    // Fewer rows than two rounds of teams: every row is on its way at once in the direct kernel, and nothing is left to
    // prefetch
    if (r.stages < 2 || r.batches < 2 * (long long)sm_count() * teams) {
        p.kind = ROWS_DIRECT;
        if (p.shift && !plain()) p.kind = ROWS_LONG;
        p.shift = false;
        if (backward && p.E > 16) {                      // the direct kernel holds 16 elements per thread
            p.E = 16;
            ++p.log_tpr;
        }
        if (p.kind == ROWS_LONG) { p.threads = 1024; p.work = R; p.grid = (int)(R < sm_count() ? R : sm_count()); return; }
        p.threads = p.log_tpr > 5 ? 1 << p.log_tpr : kRowThreads;        // one row per block when a warp is not enough
        const int rows_pb = p.threads >> p.log_tpr;
        p.work = (R + rows_pb - 1) / rows_pb;
        const int resident = 1024 / p.threads;
        p.grid = (int)(p.work < (long long)sm_count() * resident ? p.work : (long long)sm_count() * resident);
        p.smem = backward && p.log_tpr <= 5 ? (size_t)p.threads / 32 * 2 * d.C * 4 : 0;
        return;
    }
    const long long grid = (r.batches + teams - 1) / teams;
    p.kind = ROWS_RING;
    p.grid = (int)(grid < (long long)per_sm * sm_count() ? grid : (long long)per_sm * sm_count());
    if (p.shift && teams < 8) p.grid = p.grid / (8 / teams) * (8 / teams);      // a multiple of 8 teams (there are 2 x 148 x teams rows at least)
    p.smem = (size_t)teams * r.stages * nt * r.stage_bytes;
    if (backward && p.smem < (size_t)teams * 8 * d.C) p.smem = (size_t)teams * 8 * d.C;
}

void plan_planes(const gf_norm_desc& d, bool backward, long long R, NormPlan& p) {
    const int e = d.dtype == GF_F32 ? 4 : 2, nt = backward ? 2 : 1;
    const long long HW = (long long)d.H * d.W;
    const bool whole = HW * e % 16 == 0;                 // every row of a plane starts on a 16-byte boundary
    auto tiles = [&](int px) {
        PlaneArgs& t = p.tile;
        t.px = px;
        t.tiles_per_img = (int)((HW + px - 1) / px);
        t.tiles = (long long)d.N * t.tiles_per_img;
        t.div_tiles = FastDiv((uint32_t)t.tiles_per_img);
        p.threads = plane_warps(p.PX) * 32;
        p.kind = PLANES_TILE;
    };
    if (whole) {
        // Rows of 128 bytes, of 64 or of 32, as long as three tiles are in flight (two of the shortest).
        for (int lp = 8; lp >= 2; lp >>= 1) {
            PlaneArgs& t = p.tile;
            t.boxes = (d.C + 255) / 256;
            t.box_rows = ((d.C + t.boxes - 1) / t.boxes + 3) / 4 * 4;       // boxes land on 128-byte boundaries
            t.pitch = lp * 16;
            const long long stage = ((long long)t.boxes * t.box_rows * t.pitch + 127) / 128 * 128;
            constexpr int kPlaneWarps = plane_warps(0);
            const long long fixed = kPlaneWarps * nt * lp * 16 / e * 4 + nt * lp * 16 / e * 4 + 2048;      // exchange, and what a block takes
            const long long fit = ((long long)kNormSmem - 2 * fixed) / (nt * stage);
            const int kc = (d.C + kPlaneWarps * (32 / lp) - 1) / (kPlaneWarps * (32 / lp));
            if (fit < (lp > 2 ? 3 : 2) || kc > 16) continue;
            const int px = lp * 16 / e;
            if (lp > 2 && HW <= px / 2) continue;        // shorter rows would do
            if ((long long)d.N * ((HW + px - 1) / px) > 0x7fffffffLL) continue;
            tiles(px);
            p.LP = lp;
            p.KC = kc <= 2 ? 2 : kc <= 4 ? 4 : kc <= 8 ? 8 : 16;
            t.stage_bytes = (int)stage;
            // two blocks per SM where both can have three tiles in flight
            const int per_sm = fit >= 6 ? 2 : 1;
            t.stages = (int)(fit / per_sm > 6 ? 6 : fit / per_sm);
            p.smem = (size_t)t.stages * nt * stage;
            p.grid = (int)(t.tiles < (long long)per_sm * sm_count() ? t.tiles : (long long)per_sm * sm_count());
            return;
        }
    } else if (HW * e >= 64) {
        // Rows of 256 pixels (bf16, few channels: the tile stays in registers), of 128, or of 32, as long as two tiles are in flight.
        constexpr int kPlaneWarps = plane_warps(1);
        const int kc = (d.C + kPlaneWarps - 1) / kPlaneWarps;
        for (int px = e == 2 && kc <= 8 ? 8 : 4; px >= 1 && kc <= 32; px = px == 8 ? 4 : px - 3) {
            PlaneArgs& t = p.tile;
            const int pieces = 32 * px * e / 16 + 1;
            t.log_pieces = 0;
            while ((1 << t.log_pieces) < pieces) ++t.log_pieces;
            t.pitch = pieces * 16;
            const long long stage = ((long long)d.C * t.pitch + 127) / 128 * 128;
            const long long fixed = (kPlaneWarps + 1) * nt * 32 * px * 4 + 2048;
            const long long fit = ((long long)kNormSmem - 2 * fixed) / (nt * stage);
            if (fit < 2 || (px > 1 && HW <= 32) || (px > 4 && HW <= 128)) continue;
            p.PX = px;
            tiles(32 * px);
            p.KC = kc <= 8 ? 8 : kc <= 16 ? 16 : 32;
            t.stage_bytes = (int)stage;
            const int per_sm = fit >= 4 && p.KC <= 8 ? 2 : 1;        // registers of 512 threads
            t.stages = fit / per_sm >= 3 ? 3 : 2;
            p.smem = (size_t)t.stages * nt * stage;
            p.grid = (int)(t.tiles < (long long)per_sm * sm_count() ? t.tiles : (long long)per_sm * sm_count());
            return;
        }
    }
    // Small planes (pixels are numbered through all images), and more channels than shared memory holds.
    p.V = vec_for(HW, e);
    if (p.V > 4) p.V = 4;
    p.CG = 4;
    while (p.CG < 16 && (long long)p.CG * 8 < d.C) p.CG *= 2;
    const int most = 32;                                 // values per thread (of each tensor)
    while (p.V > 1 && (long long)p.CG * (most / p.V) < d.C) p.V >>= 1;
    p.NCH = 8;
    while (p.NCH * p.V < most && (long long)p.CG * p.NCH < d.C) p.NCH *= 2;
    p.kind = PLANES_DIRECT;
    if ((long long)p.CG * p.NCH < d.C) { p.kind = PLANES_LONG; p.V = vec_for(HW, e) >= 2 ? 2 : 1; }
    p.threads = 32 * p.CG;
    p.work = (R + 32LL * p.V - 1) / (32LL * p.V);
    const int per_sm = 1024 / p.threads;
    p.grid = (int)(p.work < (long long)sm_count() * per_sm ? p.work : (long long)sm_count() * per_sm);
    p.smem = (size_t)(backward ? 4 : 2) * p.CG * 32 * p.V * 4;
}

NormPlan norm_plan(const gf_norm_desc& d, bool backward) {
    NormPlan p = {};
    const long long R = (long long)d.N * d.H * d.W;
    if (d.layout == GF_NCHW && (long long)d.H * d.W > 1) plan_planes(d, backward, R, p);
    else plan_rows(d, backward, R, p);
    return p;
}

template <typename T, int V, int E, bool TEAM, bool BWD, bool SHIFT> gf_status launch_ring(const NormArgs& a, const NormPlan& p, cudaStream_t s) {
    static size_t configured[kMaxDevices] = {};
    if (gf_status st = ensure_dyn_smem(ln_rows_ring_kernel<T, V, E, TEAM, BWD, SHIFT>, p.smem, configured); st != GF_OK) return st;
    RingArgs r = p.ring;
    r.err_word = global_err_word();
    if (!r.err_word) return GF_ERR_CUDA;
    ln_rows_ring_kernel<T, V, E, TEAM, BWD, SHIFT><<<p.grid, p.threads, p.smem, s>>>(a, r);
    return after_launch();
}
template <typename T, int V, int E> gf_status launch_rows(const NormArgs& a, const NormPlan& p, bool backward, cudaStream_t s) {
    constexpr int NV = E / V;
    const bool team = p.log_tpr > 5;
    if (p.kind == ROWS_RING) {
        // Several warps share a row only where 32 elements per thread are not enough; rows read element by element are short.
        if constexpr (V * (int)sizeof(T) == 16 && E == 32) {
            if (team && p.shift) return backward ? launch_ring<T, V, E, true, true, true>(a, p, s) : launch_ring<T, V, E, true, false, true>(a, p, s);
            if (team) return backward ? launch_ring<T, V, E, true, true, false>(a, p, s) : launch_ring<T, V, E, true, false, false>(a, p, s);
        }
        if constexpr (V * (int)sizeof(T) == 16) {
            if (p.shift) return backward ? launch_ring<T, V, E, false, true, true>(a, p, s) : launch_ring<T, V, E, false, false, true>(a, p, s);
        }
        return backward ? launch_ring<T, V, E, false, true, false>(a, p, s) : launch_ring<T, V, E, false, false, false>(a, p, s);
    }
    if (!backward) {
        bool done = false;
        if constexpr (E == 32) {
            if (team) { ln_rows_fwd_kernel<T, V, NV, true><<<(unsigned)p.work, p.threads, 0, s>>>(a); done = true; }
        }
        if (!done) ln_rows_fwd_kernel<T, V, NV, false><<<(unsigned)p.work, p.threads, 0, s>>>(a);
    } else if constexpr (E <= 16) {
        bool done = false;
        if constexpr (E == 16) {
            if (team) { ln_rows_bwd_kernel<T, V, NV, true><<<p.grid, p.threads, 0, s>>>(a); done = true; }
        }
        if (!done) ln_rows_bwd_kernel<T, V, NV, false><<<p.grid, p.threads, p.smem, s>>>(a);
    }
    return after_launch();
}
template <typename T, int V> gf_status launch_rows_v(const NormArgs& a, const NormPlan& p, bool backward, cudaStream_t s) {
    switch (p.E) {
        case 8: return launch_rows<T, V, 8>(a, p, backward, s);
        case 16: return launch_rows<T, V, 16>(a, p, backward, s);
        default: return launch_rows<T, V, 32>(a, p, backward, s);
    }
}
template <typename T, int V> gf_status launch_planes_v(const NormArgs& a, const NormPlan& p, bool backward, cudaStream_t s) {
    if (!backward) {
        const unsigned grid = (unsigned)p.work;
        switch (p.kind == PLANES_LONG ? 0 : p.NCH) {
            case 8: ln_planes_fwd_kernel<T, V, 8><<<grid, p.threads, p.smem, s>>>(a); break;
            case 16: if constexpr (V <= 2) { ln_planes_fwd_kernel<T, V, 16><<<grid, p.threads, p.smem, s>>>(a); break; }
            case 32: if constexpr (V == 1) { ln_planes_fwd_kernel<T, V, 32><<<grid, p.threads, p.smem, s>>>(a); break; }
            default: ln_planes_fwd_kernel<T, V, 0><<<grid, p.threads, p.smem, s>>>(a);
        }
    } else {
        switch (p.kind == PLANES_LONG ? 0 : p.NCH) {
            case 8: ln_planes_bwd_kernel<T, V, 8><<<p.grid, p.threads, p.smem, s>>>(a, p.work); break;
            case 16: if constexpr (V <= 2) { ln_planes_bwd_kernel<T, V, 16><<<p.grid, p.threads, p.smem, s>>>(a, p.work); break; }
            case 32: if constexpr (V == 1) { ln_planes_bwd_kernel<T, V, 32><<<p.grid, p.threads, p.smem, s>>>(a, p.work); break; }
            default: ln_planes_bwd_long_kernel<T, V><<<p.grid, p.threads, p.smem, s>>>(a, p.work);
        }
    }
    return after_launch();
}
template <typename T, int LP, int KC, int PX, bool BWD>
gf_status launch_tile_inst(const NormArgs& a, const gf_norm_desc& d, const NormPlan& p, cudaStream_t s) {
    static size_t configured[kMaxDevices] = {};
    if (gf_status st = ensure_dyn_smem(ln_planes_tile_kernel<T, LP, KC, PX, BWD>, p.smem, configured); st != GF_OK) return st;
    PlaneArgs t = p.tile;
    t.err_word = global_err_word();
    if (!t.err_word) return GF_ERR_CUDA;
    if constexpr (PX == 0) {
        const uint64_t hw = (uint64_t)a.HW, c = (uint64_t)a.C;
        if (!make_tmap_plain(&t.tm_x, a.x, sizeof(T), hw, c, (uint64_t)d.N, hw, hw * c, (uint32_t)t.px, (uint32_t)t.box_rows, 1) ||
            (BWD && !make_tmap_plain(&t.tm_gy, a.gy, sizeof(T), hw, c, (uint64_t)d.N, hw, hw * c, (uint32_t)t.px, (uint32_t)t.box_rows, 1)))
            return GF_ERR_CUDA;
    }
    ln_planes_tile_kernel<T, LP, KC, PX, BWD><<<p.grid, p.threads, p.smem, s>>>(a, t);
    return after_launch();
}
template <typename T, int LP, int KC, int PX>
gf_status launch_tile_way(const NormArgs& a, const gf_norm_desc& d, const NormPlan& p, bool backward, cudaStream_t s) {
    return backward ? launch_tile_inst<T, LP, KC, PX, true>(a, d, p, s) : launch_tile_inst<T, LP, KC, PX, false>(a, d, p, s);
}
template <typename T, int LP> gf_status launch_tile_whole(const NormArgs& a, const gf_norm_desc& d, const NormPlan& p, bool backward, cudaStream_t s) {
    switch (p.KC) {
        case 2: return launch_tile_way<T, LP, 2, 0>(a, d, p, backward, s);
        case 4: return launch_tile_way<T, LP, 4, 0>(a, d, p, backward, s);
        case 8: return launch_tile_way<T, LP, 8, 0>(a, d, p, backward, s);
        default: return launch_tile_way<T, LP, 16, 0>(a, d, p, backward, s);
    }
}
template <typename T, int PX> gf_status launch_tile_odd(const NormArgs& a, const gf_norm_desc& d, const NormPlan& p, bool backward, cudaStream_t s) {
    switch (p.KC) {
        case 8: return launch_tile_way<T, 32, 8, PX>(a, d, p, backward, s);
        case 16: return launch_tile_way<T, 32, 16, PX>(a, d, p, backward, s);
        default: return launch_tile_way<T, 32, 32, PX>(a, d, p, backward, s);
    }
}
template <typename T> gf_status launch_tile(const NormArgs& a, const gf_norm_desc& d, const NormPlan& p, bool backward, cudaStream_t s) {
    if constexpr (sizeof(T) == 2) {
        if (p.PX == 8) return launch_tile_way<T, 32, 8, 8>(a, d, p, backward, s);
    }
    if (p.PX == 4) return launch_tile_odd<T, 4>(a, d, p, backward, s);
    if (p.PX == 1) return launch_tile_odd<T, 1>(a, d, p, backward, s);
    if (p.LP == 8) return launch_tile_whole<T, 8>(a, d, p, backward, s);
    return p.LP == 4 ? launch_tile_whole<T, 4>(a, d, p, backward, s) : launch_tile_whole<T, 2>(a, d, p, backward, s);
}
template <typename T> gf_status launch_norm(const NormArgs& a, const gf_norm_desc& d, const NormPlan& p, bool backward, cudaStream_t s) {
    if (p.kind == PLANES_TILE) return launch_tile<T>(a, d, p, backward, s);
    if (p.kind == PLANES_DIRECT || p.kind == PLANES_LONG) {
        switch (p.V) {
            case 4: if constexpr (sizeof(T) == 2) return launch_planes_v<T, 4>(a, p, backward, s);      // (fp32: a whole piece, a tile)
            case 2: return launch_planes_v<T, 2>(a, p, backward, s);
            default: return launch_planes_v<T, 1>(a, p, backward, s);
        }
    }
    if (p.kind == ROWS_LONG) {
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
    return desc->dtype == GF_F32 ? launch_norm<float>(a, *desc, p, false, s) : launch_norm<__nv_bfloat16>(a, *desc, p, false, s);
}

gf_status gf_layer_norm_backward_workspace_bytes(const gf_norm_desc* desc, size_t* bytes) {
    if (!bytes) return GF_ERR_NULL;
    gf_status st = norm_validate(desc);
    if (st != GF_OK) return st;
    const NormPlan p = norm_plan(*desc, true);
    *bytes = 256 + (size_t)(p.grid > 0 ? p.grid : 1) * 2 * desc->C * 4;      // error word | lines of sums
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
    float* part = sums && desc->N > 0 ? reinterpret_cast<float*>(static_cast<char*>(workspace) + 256) : nullptr;
    if (desc->N > 0) {
        NormArgs a = norm_args(*desc);
        a.x = x; a.gy = g_y; a.out = g_x; a.mean_in = mean; a.rstd_in = rstd; a.log_tpr = p.log_tpr;
        a.gamma = {gamma, desc->param_dtype == GF_BF16};
        a.part = part;
        ProfScope prof(K_NORM_BWD, s);
        st = desc->dtype == GF_F32 ? launch_norm<float>(a, *desc, p, true, s) : launch_norm<__nv_bfloat16>(a, *desc, p, true, s);
        if (st != GF_OK) return st;
    }
    if (!sums) return GF_OK;
    ProfScope prof(K_NORM_SUMS, s);
    const long long cols = 2LL * desc->C;
    return launch_pdl(ln_finish_kernel, dim3((unsigned)((cols + kFinX - 1) / kFinX)), dim3(kFinX, kFinY), 0, s,
                      (const float*)part, desc->N > 0 ? p.grid : 0, (int)desc->C, g_gamma, g_beta,
                      desc->N > 0 ? static_cast<uint32_t*>(workspace) : nullptr);
}

}  // extern "C"

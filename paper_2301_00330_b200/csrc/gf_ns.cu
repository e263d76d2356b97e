// Newton-Schulz orthogonalisation and the Muon step (gf_train.h).
//
// X [m, n] with m <= n (the input is transposed on its way in when it is tall).  All operands of the
// products are fp16 times kScale = 2^10: X of a normalised matrix has entries of rms 1 / sqrt(m n) and
// magnitude at most about 1.3, so that the scaled values use the middle of fp16's range.  With
// GF_NS_F32 each operand is a pair hi + lo of fp16 and a product is hi hi + hi lo + lo hi (2^-22
// relative is dropped).  X is carried as a pair in either case: a X is added to the product in fp32.
// Accumulators are fp32 in tensor memory.
#include <cuda_fp16.h>

#include "gf_common.cuh"
#include "gf_tc.cuh"
#include "gf_tma.cuh"
#include "gf_train.h"

namespace gf {
namespace {

constexpr float kScale = 1024.f, kInvScale = 1.f / 1024.f;
constexpr int kMaxLayers = 48;              // layers whose pointers travel in one launch's arguments
constexpr int kNormBlocks = 128;            // partial sums per matrix, at most
constexpr int kNormThreads = 512;

inline size_t up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// ---- inputs: sum of squares, and the matrix as scaled fp16 ----------------------------------------
// Where a matrix's values come from: G itself, or the momentum update of a Muon step.
struct Source {
    const void* g[kMaxLayers];              // gradients (batched G: g[0] with the stride rows * cols)
    const float* mom[kMaxLayers];           // momentum before the step (NULL in g-only sources)
    float* mom_out[kMaxLayers];
    int batched, bf16, taps, nesterov;
    float momentum;
    int rows, cols;
};

__device__ __forceinline__ float source_grad(const Source& s, int b, long long e) {
    const long long at = (s.batched ? (long long)b * s.rows * s.cols : 0) + e * s.taps;
    const void* p = s.g[s.batched ? 0 : b];
    return s.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]) : static_cast<const float*>(p)[at];
}

// Sums of squares of the matrices to be orthogonalised, one partial per block; a Muon step also
// writes the new momentum here.  Squares are added in fp32 within a thread, in fp64 across threads.
template <bool MUON> __global__ void __launch_bounds__(kNormThreads) ns_norm_kernel(const __grid_constant__ Source s, double* part, uint32_t* err_word) {
    pdl_launch_dependents();
    pdl_wait();
    if (err_word && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) { err_word[0] = 0; err_word[32] = 0; }   // and the barrier
    const int b = blockIdx.y;
    const long long n = (long long)s.rows * s.cols;
    float q = 0.f;
    const long long stride = (long long)gridDim.x * kNormThreads;
    constexpr int kAtOnce = 8;                            // loads in flight per thread
    for (long long e0 = (long long)blockIdx.x * kNormThreads + threadIdx.x; e0 < n; e0 += kAtOnce * stride) {
        float g[kAtOnce], m[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const long long e = e0 + k * stride;
            g[k] = e < n ? source_grad(s, b, e) : 0.f;
            if constexpr (MUON) m[k] = e < n ? s.mom[b][e] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            float u = g[k];
            if constexpr (MUON) {
                const float mo = s.momentum * m[k] + (1.f - s.momentum) * u;
                if (e0 + k * stride < n) s.mom_out[b][e0 + k * stride] = mo;
                u = s.nesterov ? (1.f - s.momentum) * u + s.momentum * mo : mo;
            }
            q += u * u;
        }
    }
    double d = q;
    for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
    __shared__ double red[kNormThreads / 32];
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = d;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kNormThreads / 32; ++w) d += red[w];
        part[(size_t)b * gridDim.x + blockIdx.x] = d;
    }
}

// X[b][i][j] = kScale u / (norm + eps) as pairs of fp16, rows of `ld` elements; transposed when the
// matrix is tall.  A 64 x 64 tile per block, 16 elements per thread.
constexpr int kCast = 64;
template <bool MUON>
__global__ void __launch_bounds__(256) ns_cast_kernel(const __grid_constant__ Source s, const double* part, int parts, float eps, __half* X,
                                                      int m, int n, int ld, long long lo_off, int transposed) {
    __shared__ float tile[kCast][kCast + 1];
    __shared__ float scale_sh;
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.z, tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
    const int j0 = blockIdx.x * kCast, i0 = blockIdx.y * kCast;     // in the matrix as it was given
    float u[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const int i = i0 + ty + 4 * k, j = j0 + tx;
        u[k] = 0.f;
        if (i < s.rows && j < s.cols) {
            const long long e = (long long)i * s.cols + j;
            u[k] = source_grad(s, b, e);
            if constexpr (MUON) {
                const float mo = s.mom_out[b][e];
                u[k] = s.nesterov ? (1.f - s.momentum) * u[k] + s.momentum * mo : mo;
            }
        }
    }
    if (threadIdx.x < 32) {
        double q = 0;
        for (int k = threadIdx.x; k < parts; k += 32) q += part[(size_t)b * parts + k];
        for (int o = 16; o > 0; o >>= 1) q += __shfl_xor_sync(0xffffffffu, q, o);
        // 0 / (0 + 0): a matrix of zeros with eps = 0 gives zeros
        const float scale = kScale / ((float)sqrt(q) + eps);
        if (threadIdx.x == 0) scale_sh = isinf(scale) ? 0.f : scale;
    }
    __syncthreads();
    const float scale = scale_sh;
    if (transposed) {
#pragma unroll
        for (int k = 0; k < 16; ++k) tile[ty + 4 * k][tx] = u[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k) u[k] = tile[tx][ty + 4 * k];
    }
    const int x0 = transposed ? i0 : j0, y0 = transposed ? j0 : i0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const int i = y0 + ty + 4 * k, j = x0 + tx;
        if (i < m && j < n) {
            const float v = u[k] * scale;
            const __half hi = __float2half_rn(v);
            __half* dst = X + ((size_t)b * m + i) * ld + j;
            dst[0] = hi;
            dst[lo_off] = __float2half_rn(v - __half2float(hi));
        }
    }
}

// ---- products ------------------------------------------------------------------------------------------
enum Phase { PH_GRAM = 0, PH_POLY, PH_APPLY };

struct PhaseShape {
    int bn;                        // columns of a tile (128 rows)
    int stages, stage_bytes;       // operand ring
    int tiles, tiles_n;            // tiles per matrix; per row of tiles (not symmetric)
};
struct IterateArgs {
    CUtensorMap tm_x[2], tm_a, tm_b;      // boxes of 64 x 64; third dimension: part * batch + matrix
    PhaseShape shape[3];
    float coeff[GF_NS_MAX_STEPS][3];
    int batch, m, n, steps;
    __half *x[2], *a, *b;
    int ldx, lda;
    long long x_lo, a_lo;          // elements from the high to the low parts
    void* out;
    int out_bf16, transposed;
    uint32_t *err_word, *barrier;
};

constexpr int kBox = 8192;                 // bytes of a 64 x 64 box
constexpr int kMaxStages = 8;
constexpr int kRing = 196608;              // bytes of the operand ring
constexpr int kThreads = 320;              // copies, products, eight warps of results
// k chunks of 64 that one accumulator takes when results are wanted to 32 bits: the tensor core
// adds without rounding to nearest, so that long sums drift towards zero (K = 2048 in one accumulator: 2e-5
// of the result); 2 chunks are 24 additions, the rest are fp32 additions in registers.
constexpr int kSegment = 2;

// Row and column of tile t of the lower triangle (128-row tiles that reach the diagonal).
__device__ __forceinline__ void lower_tile(int t, int bn, int& ti, int& tj) {
    if (bn == 128) {
        int r = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
        while (r * (r + 1) / 2 > t) --r;
        while ((r + 1) * (r + 2) / 2 <= t) ++r;
        ti = r; tj = t - r * (r + 1) / 2;
    } else {
        // bn = 256: rows 2g and 2g + 1 have g + 1 tiles; bn = 64: row g has 2 (g + 1) tiles
        int g = (int)((sqrtf(4.f * (float)t + 1.f) - 1.f) * 0.5f);
        while (g * (g + 1) > t) --g;
        while ((g + 1) * (g + 2) <= t) ++g;
        const int r = t - g * (g + 1);
        if (bn == 256) { ti = 2 * g + r / (g + 1); tj = r % (g + 1); }
        else { ti = g; tj = r; }
    }
}
int lower_tiles(int M, int bn) {
    int n = 0;
    for (int ti = 0; ti * 128 < M; ++ti) {
        const int reach = ti * 128 + 127 < M - 1 ? ti * 128 + 127 : M - 1;
        n += reach / bn + 1;
    }
    return n;
}
__device__ __forceinline__ void tile_at(const PhaseShape& ps, bool symmetric, int tt, int& ti, int& tj) {
    if (symmetric) lower_tile(tt, ps.bn, ti, tj);
    else { ti = tt / ps.tiles_n; tj = tt - ti * ps.tiles_n; }
}

// 32 consecutive fp16 values, high and low parts.
struct Pairs { uint4 h[4], l[4]; };
__device__ __forceinline__ void fetch_pairs(const __half* p, long long lo, bool has_lo, Pairs& r) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        r.h[q] = *reinterpret_cast<const uint4*>(p + q * 8);
        if (has_lo) r.l[q] = *reinterpret_cast<const uint4*>(p + lo + q * 8);
    }
}
__device__ __forceinline__ void add_pairs(const Pairs& r, bool has_lo, float scale, float v_scale, float (&v)[32]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t h[4] = {r.h[q].x, r.h[q].y, r.h[q].z, r.h[q].w}, l[4] = {r.l[q].x, r.l[q].y, r.l[q].z, r.l[q].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[e]));
            if (has_lo) {
                const float2 g = __half22float2(*reinterpret_cast<const __half2*>(&l[e]));
                f.x += g.x; f.y += g.y;
            }
            const int k = q * 8 + 2 * e;
            v[k] = scale * f.x + v_scale * v[k];
            v[k + 1] = scale * f.y + v_scale * v[k + 1];
        }
    }
}
__device__ __forceinline__ void store_pairs(__half* p, long long lo, bool has_lo, const float (&f)[32]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t h[4], l[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = f[q * 8 + 2 * e], y = f[q * 8 + 2 * e + 1];
            const __half2 hv = __floats2half2_rn(x, y);
            const float2 back = __half22float2(hv);
            const __half2 lv = __floats2half2_rn(x - back.x, y - back.y);
            h[e] = *reinterpret_cast<const uint32_t*>(&hv);
            l[e] = *reinterpret_cast<const uint32_t*>(&lv);
        }
        *reinterpret_cast<uint4*>(p + q * 8) = make_uint4(h[0], h[1], h[2], h[3]);
        if (has_lo) *reinterpret_cast<uint4*>(p + lo + q * 8) = make_uint4(l[0], l[1], l[2], l[3]);
    }
}

// The values that the results of a block of 32 x 32 need besides the sums: A for the polynomial, X for the
// last product of a step.  Row i, columns j0 ... (within the padded rows; row i < m).
template <int SPLIT>
__device__ __forceinline__ void fetch(const IterateArgs& p, int phase, int step, int b, int i, int j0, Pairs& r) {
    if (i >= p.m) return;
    if (phase == PH_POLY) fetch_pairs(p.a + ((long long)b * p.m + i) * p.lda + j0, p.a_lo, SPLIT == 2, r);
    else if (phase == PH_APPLY) fetch_pairs(p.x[step & 1] + ((long long)b * p.m + i) * p.ldx + j0, p.x_lo, true, r);
}

// What becomes of 32 columns of a row of the product: row i (of the warp's 32 from i0), columns j0 ..; `v` are the raw sums.
// Symmetric products: blocks of 32 x 32 below the diagonal are written twice (once mirrored), blocks on it once,
// blocks above it not at all; a block is a warp's, so that nothing here diverges.
template <int SPLIT>
__device__ __forceinline__ void emit(const IterateArgs& p, int phase, int step, int b, int i, int j0, const Pairs& r, float (&v)[32]) {
    if (i >= p.m) return;
    if (phase != PH_APPLY) {
        if (phase == PH_POLY) add_pairs(r, SPLIT == 2, p.coeff[step][1], p.coeff[step][2] * kInvScale, v);
        else {
#pragma unroll
            for (int k = 0; k < 32; ++k) v[k] *= kInvScale;
        }
        __half* out = phase == PH_GRAM ? p.a : p.b;
        store_pairs(out + ((long long)b * p.m + i) * p.lda + j0, p.a_lo, SPLIT == 2, v);
        if (j0 < (i & ~31)) {                              // j0 + 31 < m
            __half* col = out + ((long long)b * p.m + j0) * p.lda + i;
#pragma unroll
            for (int k = 0; k < 32; ++k) {
                const __half h = __float2half_rn(v[k]);
                col[(long long)k * p.lda] = h;
                if constexpr (SPLIT == 2) col[(long long)k * p.lda + p.a_lo] = __float2half_rn(v[k] - __half2float(h));
            }
        }
        return;
    }
    // a X is added in fp32 from the pair, so that only the smaller part of the step sees rounded operands
    add_pairs(r, true, p.coeff[step][0], kInvScale, v);
    if (step + 1 < p.steps) {
        store_pairs(p.x[(step + 1) & 1] + ((long long)b * p.m + i) * p.ldx + j0, p.x_lo, true, v);
        return;
    }
    const int live = min(32, p.n - j0);
    const long long base = (long long)b * p.m * p.n;
#pragma unroll
    for (int k = 0; k < 32; ++k) v[k] *= kInvScale;
    if (p.transposed) {
#pragma unroll
        for (int k = 0; k < 32; ++k)
            if (k < live) {
                const long long o = base + (long long)(j0 + k) * p.m + i;
                if (p.out_bf16) static_cast<__nv_bfloat16*>(p.out)[o] = __float2bfloat16_rn(v[k]);
                else static_cast<float*>(p.out)[o] = v[k];
            }
        return;
    }
    const long long o = base + (long long)i * p.n + j0;
    if (p.out_bf16) {
        __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(p.out) + o;
        if (live == 32 && (p.n & 7) == 0) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(v[q * 8 + 2 * e], v[q * 8 + 2 * e + 1]);
                    w[e] = *reinterpret_cast<const uint32_t*>(&h);
                }
                *reinterpret_cast<uint4*>(dst + q * 8) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 32; ++k) if (k < live) dst[k] = __float2bfloat16_rn(v[k]);
        }
    } else {
        float* dst = static_cast<float*>(p.out) + o;
        if (live == 32 && (p.n & 3) == 0) {
#pragma unroll
            for (int q = 0; q < 8; ++q)
                *reinterpret_cast<float4*>(dst + q * 4) = make_float4(v[q * 4], v[q * 4 + 1], v[q * 4 + 2], v[q * 4 + 3]);
        } else {
#pragma unroll
            for (int k = 0; k < 32; ++k) if (k < live) dst[k] = v[k];
        }
    }
}

// Orders generic-proxy accesses to global memory with the copy engine's.
__device__ __forceinline__ void fence_proxy_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }

// All blocks of a cooperative launch meet.  `ok` false in any thread ends the kernel of every block: the error
// word tells the others.  The wait is bounded like every other.
__device__ __forceinline__ bool grid_meet(const IterateArgs& p, uint32_t target, bool ok, int* flag) {
    __threadfence();
    fence_proxy_async_all();
    const int bad = __syncthreads_or(!ok);
    if (threadIdx.x == 0) {
        int go = !bad;
        if (bad) atomicOr(p.err_word, 4096u);
        else {
            atomicAdd(p.barrier, 1u);
            const long long t0 = clock64();
            for (int spins = 0;; ++spins) {
                uint32_t seen;
                asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(p.barrier) : "memory");
                if (seen >= target) break;
                if ((spins & 255) == 255) {
                    uint32_t err;
                    asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(err) : "l"(p.err_word) : "memory");
                    if (err != 0) { go = 0; break; }
                    if (clock64() - t0 > 2 * kWaitCycles) { atomicOr(p.err_word, 4096u); go = 0; break; }
                }
            }
        }
        *flag = go;
        __threadfence();
    }
    __syncthreads();
    fence_proxy_async_all();
    return *flag != 0;
}

// The whole iteration in one launch: every phase deals its tiles (128 x bn, of all matrices) to the blocks in turn, and
// the blocks meet between phases.
template <int SPLIT> __global__ void __launch_bounds__(kThreads, 1) ns_iterate_kernel(const __grid_constant__ IterateArgs p) {
    extern __shared__ unsigned char dyn_raw[];
    unsigned char* dyn = align1024(dyn_raw);
    __shared__ uint64_t full[kMaxStages], empty[kMaxStages], done[2], drained[2];
    __shared__ uint32_t tmem_base;
    __shared__ int flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kMaxStages; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(&done[s], 1); mbar_init(&drained[s], 8); }
        mbar_fence_init();
    }
    if (warp == 1) { tmem_alloc(&tmem_base, 512); tmem_relinquish(); }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_base;
    fence_proxy_async_all();
    bool ok = true;
    uint32_t ring = 0;                 // one bit per stage: the parity of its next use
    uint32_t use = 0;                  // accumulators taken so far (products), emptied so far (results)

    for (int turn = 0; turn < 3 * p.steps; ++turn) {
        const int step = turn / 3, phase = turn - 3 * step;
        const PhaseShape ps = p.shape[phase];
        const bool symmetric = phase != PH_APPLY;
        const int K = phase == PH_GRAM ? p.n : p.m;
        const int chunks = (K + 63) / 64;
        const int segment = SPLIT == 2 ? kSegment : chunks;
        const int total = ps.tiles * p.batch;
        if (warp == 0) {
            if (lane == 0) {
                const CUtensorMap* ta = phase == PH_GRAM ? &p.tm_x[step & 1] : phase == PH_POLY ? &p.tm_a : &p.tm_b;
                const CUtensorMap* tb = phase == PH_POLY ? &p.tm_a : &p.tm_x[step & 1];
                const int a_bytes = 2 * kBox, b_bytes = ps.bn / 64 * kBox;
                int s = 0;
                for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
                    const int b = t / ps.tiles;
                    int ti, tj;
                    tile_at(ps, symmetric, t - b * ps.tiles, ti, tj);
                    for (int q = 0; q < chunks; ++q) {
                        ok = mbar_wait_bounded(&empty[s], ((ring >> s) & 1u) ^ 1u);
                        if (!ok) break;
                        unsigned char* st = dyn + (size_t)s * ps.stage_bytes;
                        mbar_expect_tx(&full[s], (uint32_t)ps.stage_bytes);
#pragma unroll
                        for (int h = 0; h < SPLIT; ++h) {
                            const int z = h * p.batch + b;
                            unsigned char* sa = st + h * a_bytes;
                            unsigned char* sb = st + SPLIT * a_bytes + h * b_bytes;
                            tma_load_3d(sa, ta, q * 64, ti * 128, z, &full[s]);
                            tma_load_3d(sa + kBox, ta, q * 64, ti * 128 + 64, z, &full[s]);
                            for (int c = 0; c * 64 < ps.bn; ++c) {
                                if (symmetric) tma_load_3d(sb + c * kBox, tb, q * 64, tj * ps.bn + c * 64, z, &full[s]);
                                else tma_load_3d(sb + c * kBox, tb, tj * ps.bn + c * 64, q * 64, z, &full[s]);
                            }
                        }
                        ring ^= 1u << s;
                        if (++s == ps.stages) s = 0;
                    }
                }
            }
        } else if (warp == 1) {
            if (lane == 0) {
                // fp16 x fp16 -> fp32; B is K-major in the symmetric products, MN-major otherwise
                const uint32_t idesc = (1u << 4) | ((symmetric ? 0u : 1u) << 16) | ((uint32_t)(ps.bn >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
                const uint32_t b_step = symmetric ? 32u : 2048u, b_lbo = symmetric ? 16u : 8192u;
                const uint32_t a_bytes = 2 * kBox, b_bytes = (uint32_t)(ps.bn / 64 * kBox);
                int s = 0;
                for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
                    for (int q = 0; q < chunks; ++q) {
                        const int buf = (int)(use & 1u);
                        const bool first = q % segment == 0, last = q % segment == segment - 1 || q == chunks - 1;
                        if (first && use >= 2) ok = mbar_wait_bounded(&drained[buf], ((use >> 1) - 1) & 1u);
                        if (ok) ok = mbar_wait_bounded(&full[s], (ring >> s) & 1u);
                        if (!ok) break;
                        tc_fence_after_sync();
                        const uint32_t d = tmem + (uint32_t)(buf * 256);
                        const uint32_t a_hi = smem_u32(dyn + (size_t)s * ps.stage_bytes), a_lo = a_hi + a_bytes;
                        const uint32_t b_hi = a_hi + SPLIT * a_bytes, b_lo = b_hi + b_bytes;
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks) {
                            const uint64_t ad = umma_smem_desc(a_hi + ks * 32, 16, 1024), bd = umma_smem_desc(b_hi + ks * b_step, b_lbo, 1024);
                            umma_bf16(d, ad, bd, idesc, !(first && ks == 0));
                            if constexpr (SPLIT == 2) {
                                umma_bf16(d, ad, umma_smem_desc(b_lo + ks * b_step, b_lbo, 1024), idesc, 1u);
                                umma_bf16(d, umma_smem_desc(a_lo + ks * 32, 16, 1024), bd, idesc, 1u);
                            }
                        }
                        umma_commit(&empty[s]);
                        ring ^= 1u << s;
                        if (++s == ps.stages) s = 0;
                        if (last) { umma_commit(&done[buf]); ++use; }
                    }
                }
            }
        } else {
            const int quarter = warp & 3, half = (warp - 2) >> 2;
            const int cols = ps.bn / 2;                       // of this warp
            for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
                const int b = t / ps.tiles;
                int ti, tj;
                tile_at(ps, symmetric, t - b * ps.tiles, ti, tj);
                const int i = ti * 128 + quarter * 32 + lane;
                const int j0 = tj * ps.bn + half * cols;
                // columns past the matrix, or past the diagonal of the warp's rows, are not read (the same for the whole warp)
                const int reach = symmetric ? min(p.m, ti * 128 + quarter * 32 + 32) : p.n;
                Pairs pr;
                if (j0 < reach) fetch<SPLIT>(p, phase, step, b, i, j0, pr);        // on its way while the product runs
                if constexpr (SPLIT == 1) {
                    const int buf = (int)(use & 1u);
                    ok = mbar_wait_bounded(&done[buf], (use >> 1) & 1u);
                    ++use;
                    if (!ok) break;
                    tc_fence_after_sync();
                    for (int c = 0; c < cols && j0 + c < reach; c += 32) {
                        uint32_t raw[32];
                        tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * 256 + half * cols + c), raw);
                        const Pairs now = pr;
                        if (c + 32 < cols && j0 + c + 32 < reach) fetch<SPLIT>(p, phase, step, b, i, j0 + c + 32, pr);
                        tmem_ld_wait();
                        float v[32];
#pragma unroll
                        for (int k = 0; k < 32; ++k) v[k] = __uint_as_float(raw[k]);
                        emit<SPLIT>(p, phase, step, b, i, j0 + c, now, v);
                        __syncwarp();                         // the next read of tensor memory is the whole warp's
                    }
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&drained[buf]);
                } else {
                    float acc[4][32];
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int k = 0; k < 32; ++k) acc[c][k] = 0.f;
                    for (int q = 0; q < chunks; q += kSegment) {
                        const int buf = (int)(use & 1u);
                        ok = mbar_wait_bounded(&done[buf], (use >> 1) & 1u);
                        ++use;
                        if (!ok) break;
                        tc_fence_after_sync();
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            if (c * 32 < cols && j0 + c * 32 < reach) {
                                uint32_t raw[32];
                                tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * 256 + half * cols + c * 32), raw);
                                tmem_ld_wait();
#pragma unroll
                                for (int k = 0; k < 32; ++k) acc[c][k] += __uint_as_float(raw[k]);
                            }
                        }
                        tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&drained[buf]);
                    }
                    if (!ok) break;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if (c * 32 < cols && j0 + c * 32 < reach) {
                            if (c > 0) fetch<SPLIT>(p, phase, step, b, i, j0 + c * 32, pr);
                            emit<SPLIT>(p, phase, step, b, i, j0 + c * 32, pr, acc[c]);
                        }
                        __syncwarp();
                    }
                }
            }
        }
        if (turn + 1 < 3 * p.steps) {
            ok = grid_meet(p, (uint32_t)(turn + 1) * gridDim.x, ok, &flag);
            if (!ok) break;
        }
    }
    if (!ok) {
        atomicOr(p.err_word, 4096u);
        const long long t0 = clock64();           // copies may still be on their way to this CTA's shared memory
        while (clock64() - t0 < 2000000LL) {}
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == 1) tmem_dealloc(tmem, 512);
}

// W' = (1 - lr wd) W - f O for the layers of a launch; O [rows, cols] fp32, one value for all taps.
struct UpdateArgs {
    const void* w[kMaxLayers];
    void* w_out[kMaxLayers];
    const float* O;
    long long n;                   // rows * cols
    int taps, bf16;
    float keep, f;
    FastDiv div_taps;
};
__global__ void __launch_bounds__(256) muon_update_kernel(const __grid_constant__ UpdateArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.y;
    const float* O = a.O + (size_t)b * a.n;
    const long long total = a.n * a.taps;
    for (long long e = (long long)blockIdx.x * blockDim.x + threadIdx.x; e < total; e += (long long)gridDim.x * blockDim.x) {
        const float o = O[a.taps == 1 ? e : e / a.taps];
        if (a.bf16)
            static_cast<__nv_bfloat16*>(a.w_out[b])[e] =
                __float2bfloat16_rn(a.keep * __bfloat162float(static_cast<const __nv_bfloat16*>(a.w[b])[e]) - a.f * o);
        else
            static_cast<float*>(a.w_out[b])[e] = a.keep * static_cast<const float*>(a.w[b])[e] - a.f * o;
    }
}

// ---- host side --------------------------------------------------------------------------------------------
struct NsPlan {
    int batch, rows, cols, m, n, ldx, lda, split, transposed;
    int norm_blocks;
    size_t off_part, off_x[2], off_a, off_b, off_o, total;
    long long x_lo, a_lo;          // elements from the high to the low parts
};

NsPlan ns_plan(int batch, int rows, int cols, int precision, bool muon) {
    NsPlan p = {};
    p.batch = batch; p.rows = rows; p.cols = cols;
    p.transposed = rows > cols;
    p.m = rows < cols ? rows : cols;
    p.n = rows < cols ? cols : rows;
    p.split = precision == GF_NS_F32 ? 2 : 1;
    p.ldx = (p.n + 31) / 32 * 32;            // results are written 32 columns at a time
    p.lda = (p.m + 31) / 32 * 32;
    const long long per = ((long long)rows * cols + 8 * kNormThreads - 1) / (8 * kNormThreads);
    p.norm_blocks = (int)(per < kNormBlocks ? per : kNormBlocks);
    p.x_lo = (long long)batch * p.m * p.ldx;
    p.a_lo = (long long)batch * p.m * p.lda;
    size_t off = 256;
    p.off_part = off; off += up((size_t)batch * p.norm_blocks * 8, 256);
    for (int k = 0; k < 2; ++k) { p.off_x[k] = off; off += up((size_t)p.x_lo * 4, 256); }
    p.off_a = off; off += up((size_t)p.a_lo * 2 * p.split, 256);
    p.off_b = off; off += up((size_t)p.a_lo * 2 * p.split, 256);
    p.off_o = off;
    if (muon) off += up((size_t)batch * rows * cols * 4, 256);
    p.total = off;
    return p;
}

const float kDefaultCoeffs[3] = {3.4445f, -4.7750f, 2.0315f};

// The tile width with the least estimated time: rounds of tiles over the SMs, times the width plus what a tile
// costs whatever its width (its 128 rows of A).
PhaseShape phase_shape(const NsPlan& p, bool symmetric) {
    PhaseShape best = {};
    double least = 0;
    for (int bn = 256; bn >= 64; bn >>= 1) {
        PhaseShape s;
        s.bn = bn;
        s.stage_bytes = p.split * (2 + bn / 64) * kBox;
        s.stages = kRing / s.stage_bytes < kMaxStages ? kRing / s.stage_bytes : kMaxStages;
        s.tiles_n = ((symmetric ? p.m : p.n) + bn - 1) / bn;
        s.tiles = symmetric ? lower_tiles(p.m, bn) : (p.m + 127) / 128 * s.tiles_n;
        const double cost = (double)cdiv64((long long)s.tiles * p.batch, sm_count()) * (bn + 64);
        if (least == 0 || cost < least) { least = cost; best = s; }
    }
    return best;
}

template <int SPLIT> gf_status launch_iterate(const IterateArgs& a, cudaStream_t s) {
    constexpr size_t smem = (size_t)kRing + 1024;
    static size_t configured[kMaxDevices] = {};
    if (gf_status st = ensure_dyn_smem(ns_iterate_kernel<SPLIT>, smem, configured); st != GF_OK) return st;
    long long most = 1;
    for (const PhaseShape& ps : a.shape) most = (long long)ps.tiles * a.batch > most ? (long long)ps.tiles * a.batch : most;
    const int grid = most < sm_count() ? (int)most : sm_count();
    ProfScope prof(K_NS_PRODUCT, s);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem; cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeCooperative;          // the blocks wait for one another between phases
    attr[0].val.cooperative = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, ns_iterate_kernel<SPLIT>, a);
    count_launch();
    return e == cudaSuccess ? GF_OK : GF_ERR_CUDA;
}

// The iteration from X in the workspace (written by ns_cast_kernel) to O.
gf_status ns_iterate(const NsPlan& p, char* base, int steps, const float* coeffs, void* O, int out_bf16, cudaStream_t s) {
    IterateArgs a = {};
    a.batch = p.batch; a.m = p.m; a.n = p.n; a.steps = steps;
    for (int k = 0; k < steps; ++k)
        for (int e = 0; e < 3; ++e) a.coeff[k][e] = coeffs ? coeffs[3 * k + e] : kDefaultCoeffs[e];
    a.x[0] = reinterpret_cast<__half*>(base + p.off_x[0]);
    a.x[1] = reinterpret_cast<__half*>(base + p.off_x[1]);
    a.a = reinterpret_cast<__half*>(base + p.off_a);
    a.b = reinterpret_cast<__half*>(base + p.off_b);
    a.ldx = p.ldx; a.lda = p.lda; a.x_lo = p.x_lo; a.a_lo = p.a_lo;
    a.out = O; a.out_bf16 = out_bf16; a.transposed = p.transposed;
    a.err_word = reinterpret_cast<uint32_t*>(base);
    a.barrier = reinterpret_cast<uint32_t*>(base + 128);
    a.shape[PH_GRAM] = a.shape[PH_POLY] = phase_shape(p, true);
    a.shape[PH_APPLY] = phase_shape(p, false);
    for (const PhaseShape& ps : a.shape)
        if ((long long)ps.tiles * p.batch > 0x3fffffffLL) return GF_ERR_UNSUPPORTED;
    const uint64_t m = (uint64_t)p.m, n = (uint64_t)p.n, lx = (uint64_t)p.ldx, la = (uint64_t)p.lda, b = (uint64_t)p.batch;
    // the maps move 16-bit elements; zeros beyond the matrices are the same in fp16
    if (!make_tmap_bf16(&a.tm_x[0], a.x[0], 3, n, m, 2 * b, lx, m * lx, 64) || !make_tmap_bf16(&a.tm_x[1], a.x[1], 3, n, m, 2 * b, lx, m * lx, 64) ||
        !make_tmap_bf16(&a.tm_a, a.a, 3, m, m, b * p.split, la, m * la, 64) || !make_tmap_bf16(&a.tm_b, a.b, 3, m, m, b * p.split, la, m * la, 64))
        return GF_ERR_CUDA;
    return p.split == 2 ? launch_iterate<2>(a, s) : launch_iterate<1>(a, s);
}

template <bool MUON> gf_status launch_prepare(const NsPlan& p, const Source& src, int first, int count, char* base, float eps, cudaStream_t s) {
    ProfScope prof(K_NS_PREPARE, s);
    double* part = reinterpret_cast<double*>(base + p.off_part) + (size_t)first * p.norm_blocks;
    gf_status st = launch_pdl(ns_norm_kernel<MUON>, dim3(p.norm_blocks, count), dim3(kNormThreads), 0, s, src, part,
                              first == 0 ? reinterpret_cast<uint32_t*>(base) : nullptr);
    if (st != GF_OK) return st;
    __half* X = reinterpret_cast<__half*>(base + p.off_x[0]) + (size_t)first * p.m * p.ldx;
    const dim3 grid((p.cols + kCast - 1) / kCast, (p.rows + kCast - 1) / kCast, count), block(256);
    return launch_pdl(ns_cast_kernel<MUON>, grid, block, 0, s, src, (const double*)part, p.norm_blocks, eps, X, p.m, p.n, p.ldx, p.x_lo, p.transposed);
}

bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
bool bad_dtype(int d) { return d != GF_F32 && d != GF_BF16; }

gf_status check_shape(int batch, int rows, int cols, int precision, int steps, float eps) {
    if (batch < 0 || rows < 1 || cols < 1 || steps < 1 || steps > GF_NS_MAX_STEPS || !(eps >= 0.f)) return GF_ERR_BAD_DESC;
    if (precision != GF_NS_F16 && precision != GF_NS_F32) return GF_ERR_BAD_DESC;
    if (rows > 16384 || cols > 16384 || batch > 32767) return GF_ERR_UNSUPPORTED;
    return GF_OK;
}

}  // namespace
}  // namespace gf

using namespace gf;

extern "C" {

gf_status gf_newton_schulz_workspace_bytes(const gf_ns_desc* d, size_t* bytes) {
    if (!d || !bytes) return GF_ERR_NULL;
    if (gf_status st = check_shape(d->batch, d->rows, d->cols, d->precision, d->steps, d->eps); st != GF_OK) return st;
    if (bad_dtype(d->in_dtype) || bad_dtype(d->out_dtype)) return GF_ERR_BAD_DESC;
    *bytes = ns_plan(d->batch, d->rows, d->cols, d->precision, false).total;
    return GF_OK;
}

gf_status gf_newton_schulz(const gf_ns_desc* d, const void* G, void* O, void* workspace, size_t workspace_bytes, const float* h_coeffs,
                           void* stream) {
    size_t need = 0;
    if (gf_status st = gf_newton_schulz_workspace_bytes(d, &need); st != GF_OK) return st;
    if (d->batch == 0) return GF_OK;
    if (!G || !O || !workspace) return GF_ERR_NULL;
    if (off16(G) || off16(O) || off16(workspace)) return GF_ERR_ALIGN;
    if (workspace_bytes < need) return GF_ERR_WORKSPACE;
    const NsPlan p = ns_plan(d->batch, d->rows, d->cols, d->precision, false);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char* base = static_cast<char*>(workspace);
    Source src = {};
    src.g[0] = G; src.batched = 1; src.bf16 = d->in_dtype == GF_BF16; src.taps = 1; src.rows = d->rows; src.cols = d->cols;
    if (gf_status st = launch_prepare<false>(p, src, 0, d->batch, base, d->eps, s); st != GF_OK) return st;
    return ns_iterate(p, base, d->steps, h_coeffs, O, d->out_dtype == GF_BF16, s);
}

gf_status gf_muon_workspace_bytes(const gf_muon_desc* d, size_t* bytes) {
    if (!d || !bytes) return GF_ERR_NULL;
    if (gf_status st = check_shape(d->count, d->rows, d->cols, d->precision, d->steps, d->eps); st != GF_OK) return st;
    if (bad_dtype(d->grad_dtype) || bad_dtype(d->weight_dtype) || d->taps < 1 || (d->nesterov != 0 && d->nesterov != 1)) return GF_ERR_BAD_DESC;
    if (d->taps > 4096) return GF_ERR_UNSUPPORTED;
    *bytes = ns_plan(d->count, d->rows, d->cols, d->precision, true).total;
    return GF_OK;
}

gf_status gf_muon_step(const gf_muon_desc* d, const void* const* h_grad, const float* const* h_momentum, const void* const* h_weight,
                       float* const* h_momentum_out, void* const* h_weight_out, void* workspace, size_t workspace_bytes,
                       const float* h_coeffs, void* stream) {
    size_t need = 0;
    if (gf_status st = gf_muon_workspace_bytes(d, &need); st != GF_OK) return st;
    if (d->count == 0) return GF_OK;
    if (!h_grad || !h_momentum || !h_weight || !h_momentum_out || !h_weight_out || !workspace) return GF_ERR_NULL;
    if (off16(workspace)) return GF_ERR_ALIGN;
    for (int k = 0; k < d->count; ++k) {
        const void* ptrs[] = {h_grad[k], h_momentum[k], h_weight[k], h_momentum_out[k], h_weight_out[k]};
        const int sizes[] = {d->grad_dtype == GF_F32 ? 4 : 2, 4, d->weight_dtype == GF_F32 ? 4 : 2, 4, d->weight_dtype == GF_F32 ? 4 : 2};
        for (int e = 0; e < 5; ++e) {
            if (!ptrs[e]) return GF_ERR_NULL;
            if (reinterpret_cast<uintptr_t>(ptrs[e]) % (uintptr_t)sizes[e] != 0) return GF_ERR_ALIGN;
        }
    }
    if (workspace_bytes < need) return GF_ERR_WORKSPACE;
    const NsPlan p = ns_plan(d->count, d->rows, d->cols, d->precision, true);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char* base = static_cast<char*>(workspace);
    const float root = sqrtf((float)d->taps);
    for (int first = 0; first < d->count; first += kMaxLayers) {
        const int n = d->count - first < kMaxLayers ? d->count - first : kMaxLayers;
        Source src = {};
        for (int k = 0; k < n; ++k) {
            src.g[k] = h_grad[first + k];
            src.mom[k] = h_momentum[first + k];
            src.mom_out[k] = h_momentum_out[first + k];
        }
        src.bf16 = d->grad_dtype == GF_BF16; src.taps = d->taps; src.nesterov = d->nesterov; src.momentum = d->momentum;
        src.rows = d->rows; src.cols = d->cols;
        // the flattened matrix is u (x) (1 .. 1): its norm is sqrt(taps) times that of u
        if (gf_status st = launch_prepare<true>(p, src, first, n, base, d->eps / root, s); st != GF_OK) return st;
    }
    float* O = reinterpret_cast<float*>(base + p.off_o);
    if (gf_status st = ns_iterate(p, base, d->steps, h_coeffs, O, 0, s); st != GF_OK) return st;
    for (int first = 0; first < d->count; first += kMaxLayers) {
        const int n = d->count - first < kMaxLayers ? d->count - first : kMaxLayers;
        UpdateArgs u = {};
        for (int k = 0; k < n; ++k) { u.w[k] = h_weight[first + k]; u.w_out[k] = h_weight_out[first + k]; }
        u.n = (long long)d->rows * d->cols;
        u.O = O + (size_t)first * u.n;
        u.taps = d->taps; u.bf16 = d->weight_dtype == GF_BF16;
        u.keep = 1.f - d->lr * d->weight_decay;
        u.f = d->lr * d->scale / root;
        const long long blocks = (u.n * u.taps + 1023) / 1024;
        const long long most = cdiv64(8LL * sm_count(), n);
        if (gf_status st = launch_pdl(muon_update_kernel, dim3((unsigned)(blocks < most ? blocks : most), n), dim3(256), 0, s, u); st != GF_OK) return st;
    }
    return GF_OK;
}

}  // extern "C"

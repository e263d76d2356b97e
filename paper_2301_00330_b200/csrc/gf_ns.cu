// Newton-Schulz orthogonalisation and the Muon step (gf_train.h).
//
// X [m, n] with m <= n (the input is transposed on its way in when it is tall).  All operands of the
// products are fp16 times kScale = 2^10: X of a normalised matrix has entries of rms 1 / sqrt(m n) and
// magnitude at most about 1.3, so that the scaled values use the middle of fp16's range.  With
// GF_NS_F32 each operand is a pair hi + lo of fp16, within max(2^-22 |v|, 2^-35) of its value v (below |v| = 2^-13 lo is
// subnormal), and a product is hi hi + hi lo + lo hi (2^-22 relative is dropped).  X is carried as a pair in either case: a X is added to the product in fp32.
// Accumulators are fp32 in tensor memory.
//
// Layout of X, A = X X^T and B = b A + c A A in the workspace: [part][matrix][column / 8][row][column % 8], 16
// bytes per (row, 8 columns).  A piece of 8 columns is the same thing to the tensor core whether its
// columns are the contracted index (K-major, X X^T) or the free one (MN-major, B X): core matrices of
// 8 rows of 16 bytes, unswizzled.  So one layout serves all products, the copy engine moves whole 1 or 2 KB lines of
// it, and a warp that holds 32 rows of a result (a row per lane) writes 512 consecutive bytes per
// instruction.  (Row-major operands in 128-byte-swizzled tiles measured 365 us per step of a 4096 x 4096 matrix:
// boxes of 8 KB fed 44 bytes per clock and SM, and results written row by row took 10 us a tile.)
#include <cuda_fp16.h>

#include <type_traits>

#include "gf_common.cuh"
#include "gf_tc.cuh"
#include "gf_tma.cuh"
#include "gf_train.h"

namespace gf {
namespace {

constexpr float kScale = 1024.f, kInvScale = 1.f / 1024.f;
constexpr int kMaxLayers = 48;              // layers whose pointers travel in one launch's arguments
constexpr int kArrived = 4096;              // counters of split tiles
constexpr int kNormBlocks = 256;            // partial sums per matrix, at most
constexpr int kNormThreads = 256;

inline size_t up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// ---- inputs: sum of squares, and the matrix as scaled fp16 ----------------------------------------
// Where a matrix's values come from: G itself, or the momentum update of a Muon step.
struct Source {
    const void* g[kMaxLayers];              // gradients (batched G: g[0] with the stride rows * cols)
    const float* mom[kMaxLayers];           // momentum before the step (NULL in g-only sources)
    float* mom_out[kMaxLayers];
    int batched, bf16, taps, nesterov;
    int vec;                                // four elements at a time: one value per 4 or 2 bytes, rows and pointers on boundaries of them
    float momentum;
    int rows, cols;
};

// Elements e .. e + 3 of matrix b's gradient; `live` of them exist (four where s.vec).
__device__ __forceinline__ void source_grad4(const Source& s, int b, long long e, int live, float (&g)[4]) {
    const long long at = (s.batched ? (long long)b * s.rows * s.cols : 0) + e * s.taps;
    const void* p = s.g[s.batched ? 0 : b];
    if (s.vec) {
        if (s.bf16) {
            const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(p) + at);
            g[0] = __uint_as_float(w.x << 16); g[1] = __uint_as_float(w.x & 0xffff0000u);
            g[2] = __uint_as_float(w.y << 16); g[3] = __uint_as_float(w.y & 0xffff0000u);
        } else {
            const float4 w = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
            g[0] = w.x; g[1] = w.y; g[2] = w.z; g[3] = w.w;
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        g[k] = 0.f;
        if (k < live) g[k] = s.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at + k * s.taps]) : static_cast<const float*>(p)[at + k * s.taps];
    }
}
// Four floats of a momentum buffer.
__device__ __forceinline__ void momentum4(const float* p, int vec, int live, float (&m)[4]) {
    if (vec) { const float4 w = *reinterpret_cast<const float4*>(p); m[0] = w.x; m[1] = w.y; m[2] = w.z; m[3] = w.w; return; }
#pragma unroll
    for (int k = 0; k < 4; ++k) { m[k] = 0.f; if (k < live) m[k] = p[k]; }
}

// (Bound by memory; with the cast and the last kernel about 40 us of the 1.3 ms of 4096 x 4096.)
// Sums of squares of the matrices to be orthogonalised, one partial per block; a Muon step also
// writes the new momentum here.  Squares are added in fp32 within a thread, in fp64 across threads.
template <bool MUON> __global__ void __launch_bounds__(kNormThreads) ns_norm_kernel(const __grid_constant__ Source s, double* part, uint32_t* err_word) {
    pdl_launch_dependents();
    pdl_wait();
    if (err_word && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) { err_word[0] = 0; err_word[32] = 0; }   // and the barrier
    if (err_word && blockIdx.x == 0 && blockIdx.y == 0)
        for (int k = threadIdx.x; k < kArrived; k += kNormThreads) err_word[64 + k] = 0;               // and the counters of split tiles
    const int b = blockIdx.y;
    const long long n = (long long)s.rows * s.cols;
    float q = 0.f;
    const long long stride = 4LL * gridDim.x * kNormThreads;
    constexpr int kAtOnce = 4;                            // groups of four in flight per thread
    for (long long e0 = 4LL * (blockIdx.x * kNormThreads + threadIdx.x); e0 < n; e0 += kAtOnce * stride) {
        float g[kAtOnce][4], m[kAtOnce][4];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const long long e = e0 + k * stride;
            const int live = e < n ? (n - e < 4 ? (int)(n - e) : 4) : 0;
            if (live > 0) {
                source_grad4(s, b, e, live, g[k]);
                if constexpr (MUON) momentum4(s.mom[b] + e, s.vec, live, m[k]);
            } else g[k][0] = g[k][1] = g[k][2] = g[k][3] = m[k][0] = m[k][1] = m[k][2] = m[k][3] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const long long e = e0 + k * stride;
            if constexpr (MUON) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    m[k][i] = s.momentum * m[k][i] + (1.f - s.momentum) * g[k][i];
                    g[k][i] = s.nesterov ? (1.f - s.momentum) * g[k][i] + s.momentum * m[k][i] : m[k][i];
                }
                if (s.vec) { if (e < n) *reinterpret_cast<float4*>(s.mom_out[b] + e) = make_float4(m[k][0], m[k][1], m[k][2], m[k][3]); }
                else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) if (e + i < n) s.mom_out[b][e + i] = m[k][i];
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) q += g[k][i] * g[k][i];
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

// X = kScale u / (norm + eps) as pairs of fp16 in the blocked layout; transposed when the matrix is tall.  A 64 x 64 tile per
// block through shared memory: read along the given rows, written 16 bytes (8 columns of a row) per thread.
// Columns past n in the last piece are zeros: they are contracted over.
constexpr int kCast = 64;
template <bool MUON>
__global__ void __launch_bounds__(256) ns_cast_kernel(const __grid_constant__ Source s, const double* part, int parts, float eps, __half* X,
                                                      int m, int n, int pieces, long long lo_off, int transposed) {
    __shared__ float tile[kCast][kCast + 1];
    __shared__ float scale_sh;
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.z, tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
    const int j0 = blockIdx.x * kCast, i0 = blockIdx.y * kCast;     // in the matrix as it was given
    const int cx = (threadIdx.x & 15) * 4, cy = threadIdx.x >> 4;   // four columns of every 16th row
    float u[4][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int i = i0 + cy + 16 * k, j = j0 + cx;
        u[k][0] = u[k][1] = u[k][2] = u[k][3] = 0.f;
        if (i < s.rows && j < s.cols) {
            const long long e = (long long)i * s.cols + j;
            const int live = min(4, s.cols - j);
            source_grad4(s, b, e, live, u[k]);
            if constexpr (MUON) {
                float mo[4];
                momentum4(s.mom_out[b] + e, s.vec, live, mo);
#pragma unroll
                for (int d = 0; d < 4; ++d) u[k][d] = s.nesterov ? (1.f - s.momentum) * u[k][d] + s.momentum * mo[d] : mo[d];
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
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int d = 0; d < 4; ++d) tile[cy + 16 * k][cx + d] = u[k][d];
    __syncthreads();
    const float scale = scale_sh;
    const int x0 = transposed ? i0 : j0, y0 = transposed ? j0 : i0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int row = tx, piece = ty + 4 * k;
        const int i = y0 + row, j = x0 + piece * 8;
        if (i >= m || j >= n) continue;
        uint32_t h[4], l[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float v[2];
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                const int c = piece * 8 + 2 * e + d;
                v[d] = j + 2 * e + d < n ? (transposed ? tile[c][row] : tile[row][c]) * scale : 0.f;
            }
            const __half2 hv = __floats2half2_rn(v[0], v[1]);
            const float2 back = __half22float2(hv);
            const __half2 lv = __floats2half2_rn(v[0] - back.x, v[1] - back.y);
            h[e] = *reinterpret_cast<const uint32_t*>(&hv);
            l[e] = *reinterpret_cast<const uint32_t*>(&lv);
        }
        __half* dst = X + (((long long)b * pieces + (j >> 3)) * m + i) * 8;
        *reinterpret_cast<uint4*>(dst) = make_uint4(h[0], h[1], h[2], h[3]);
        *reinterpret_cast<uint4*>(dst + lo_off) = make_uint4(l[0], l[1], l[2], l[3]);
    }
}

// The last iterate to where it is wanted: O (row-major, transposed back), or the weights of a Muon step,
// W' = keep W - f O with one value for all taps.
struct FinishArgs {
    const void* w[kMaxLayers];     // Muon: weights before and after
    void* w_out[kMaxLayers];
    void* out;                     // O of the whole batch
    const __half* x;
    int m, n, pieces, transposed, cols, rows;
    long long lo;
    int bf16, taps;
    float keep, f;
    FastDiv div_taps;
};
constexpr int kFinRows = 16;                       // rows of the result per block, 64 columns
template <bool MUON> __global__ void __launch_bounds__(256) ns_finish_kernel(const __grid_constant__ FinishArgs a) {
    __shared__ float tile[kFinRows][kCast + 1];    // [row][column] of the result as it is wanted
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.z;
    const int c0 = blockIdx.x * kCast, r0 = blockIdx.y * kFinRows;
    if (threadIdx.x < 128) {
        // a thread has 8 columns of a row of X: 16 rows x 8 pieces, or (transposed) 64 rows x 2 pieces
        const int row = a.transposed ? threadIdx.x & 63 : threadIdx.x & 15, piece = a.transposed ? threadIdx.x >> 6 : threadIdx.x >> 4;
        const int i = (a.transposed ? c0 : r0) + row, j = (a.transposed ? r0 : c0) + piece * 8;
        if (i < a.m && j < a.n) {
            const __half* src = a.x + (((long long)b * a.pieces + (j >> 3)) * a.m + i) * 8;
            const uint4 hv = *reinterpret_cast<const uint4*>(src), lv = *reinterpret_cast<const uint4*>(src + a.lo);
            const uint32_t h[4] = {hv.x, hv.y, hv.z, hv.w}, l[4] = {lv.x, lv.y, lv.z, lv.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&h[e])), q = __half22float2(*reinterpret_cast<const __half2*>(&l[e]));
                const float v[2] = {(p.x + q.x) * kInvScale, (p.y + q.y) * kInvScale};
#pragma unroll
                for (int d = 0; d < 2; ++d) {
                    const int c = piece * 8 + 2 * e + d;
                    if (a.transposed) tile[c][row] = v[d];
                    else tile[row][c] = v[d];
                }
            }
        }
    }
    __syncthreads();
    const int nr = min(kFinRows, a.rows - r0), nc = min(kCast, a.cols - c0);
    if constexpr (!MUON) {
        const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
        const long long base = (long long)b * a.rows * a.cols;
#pragma unroll
        for (int k = 0; k < kFinRows / 4; ++k) {
            const int r = ty + 4 * k;
            if (r < nr && tx < nc) {
                const long long o = base + (long long)(r0 + r) * a.cols + c0 + tx;
                if (a.bf16) static_cast<__nv_bfloat16*>(a.out)[o] = __float2bfloat16_rn(tile[r][tx]);
                else static_cast<float*>(a.out)[o] = tile[r][tx];
            }
        }
    } else {
        // a row of the tile is nc * taps consecutive weights; a warp takes two rows
        const int span = nc * a.taps, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        for (int r = warp; r < nr; r += 8) {
            const long long o = ((long long)(r0 + r) * a.cols + c0) * a.taps;
            if (a.bf16) {
                const __nv_bfloat16* w = static_cast<const __nv_bfloat16*>(a.w[b]) + o;
                __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.w_out[b]) + o;
                for (int e0 = lane; e0 < span; e0 += 32 * 8) {
                    float v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) if (e0 + 32 * k < span) v[k] = __bfloat162float(w[e0 + 32 * k]);
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (e0 + 32 * k < span) out[e0 + 32 * k] = __float2bfloat16_rn(a.keep * v[k] - a.f * tile[r][a.div_taps.div((uint32_t)(e0 + 32 * k))]);
                }
            } else {
                const float* w = static_cast<const float*>(a.w[b]) + o;
                float* out = static_cast<float*>(a.w_out[b]) + o;
                for (int e0 = lane; e0 < span; e0 += 32 * 8) {
                    float v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) if (e0 + 32 * k < span) v[k] = w[e0 + 32 * k];
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (e0 + 32 * k < span) out[e0 + 32 * k] = a.keep * v[k] - a.f * tile[r][a.div_taps.div((uint32_t)(e0 + 32 * k))];
                }
            }
        }
    }
}

// ---- products ------------------------------------------------------------------------------------------
enum Phase { PH_GRAM = 0, PH_POLY, PH_APPLY };

// One CTA works on 128 rows of a tile; a pair of CTAs (two SMs, one product of the tensor cores) on 256, each with half of the
// tile's columns as its share of the second operand.
struct PhaseShape {
    int bn;                        // columns of a tile
    int stages, stage_bytes;       // operand ring of a CTA
    int tiles, tiles_n;            // tiles per matrix; per row of tiles (not symmetric)
    int splits, per;               // parts of the contracted index that a tile is dealt out in; chunks of 64 of each
};
struct IterateArgs {
    CUtensorMap tm_a[4];           // first operands, 128 rows x 64 k: X[0], X[1], A, B
    CUtensorMap tm_g[3];           // second operands of the symmetric products, rows x 64 k: X[0], X[1], A
    CUtensorMap tm_n[2];           // second operand of B X, 64 k x columns: X[0], X[1]
    PhaseShape shape[3];
    float coeff[GF_NS_MAX_STEPS][3];
    int batch, m, n, steps;
    __half *x[2], *a, *b;
    float* trace;                  // [matrix][rows / 32]: sums of A's diagonal over 32 rows, times kScale
    int blocks;                    // of 32 rows
    int x_pieces, a_pieces;        // of 8 columns
    long long x_lo, a_lo;          // elements from the high to the low parts
    float* partial;                // sums of the parts of split tiles: [tile, CTA of a pair][part][warp][column][lane]
    uint32_t* arrived;             // [tile, CTA of a pair][warp]: parts that are there; zero between phases
    uint32_t *err_word, *barrier;
};

constexpr int kMaxStages = 8;
constexpr int kRing = 196608;              // bytes of the operand ring
constexpr int kMaxSplits = 8;
constexpr int kThreads = 320;              // copies, products, eight warps of results
// k chunks of 64 that one accumulator takes when results are wanted to 32 bits: the tensor core
// adds without rounding to nearest, so that long sums drift towards zero (K = 2048 in one accumulator: 2e-5
// of the result); 2 chunks are 24 additions, the rest are fp32 additions in registers.
constexpr int kSegment = 2;

// Tile t of the lower triangle: `rows` x bn tiles that reach the diagonal, rows = bn or 2 bn.
__device__ __forceinline__ void lower_tile(int t, bool square, int& ti, int& tj) {
    if (square) {
        int r = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
        while (r * (r + 1) / 2 > t) --r;
        while ((r + 1) * (r + 2) / 2 <= t) ++r;
        ti = r; tj = t - r * (r + 1) / 2;
    } else {                       // row g has 2 (g + 1) tiles
        int g = (int)((sqrtf(4.f * (float)t + 1.f) - 1.f) * 0.5f);
        while (g * (g + 1) > t) --g;
        while ((g + 1) * (g + 2) <= t) ++g;
        ti = g; tj = t - g * (g + 1);
    }
}
int lower_tiles(int M, int rows, int bn) {
    int n = 0;
    for (int i = 0; i < M; i += rows) n += (i + rows < M ? i + rows - 1 : M - 1) / bn + 1;
    return n;
}

// 32 consecutive columns (4 pieces) of one row in the blocked layout, high and low parts; `piece` elements lie
// between pieces.  Pieces from `live` on do not exist.
struct Pairs { uint4 h[4], l[4]; };
__device__ __forceinline__ void fetch_pairs(const __half* p, long long piece, long long lo, bool has_lo, int live, Pairs& r) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (q < live) {
            r.h[q] = *reinterpret_cast<const uint4*>(p + q * piece);
            if (has_lo) r.l[q] = *reinterpret_cast<const uint4*>(p + q * piece + lo);
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
// 32 values as packed fp16, and what is left of them.
__device__ __forceinline__ void pack_pairs(const float (&f)[32], bool has_lo, uint32_t (&h)[16], uint32_t (&l)[16]) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const __half2 hv = __floats2half2_rn(f[2 * e], f[2 * e + 1]);
        h[e] = *reinterpret_cast<const uint32_t*>(&hv);
        if (has_lo) {
            const float2 back = __half22float2(hv);
            const __half2 lv = __floats2half2_rn(f[2 * e] - back.x, f[2 * e + 1] - back.y);
            l[e] = *reinterpret_cast<const uint32_t*>(&lv);
        }
    }
}
__device__ __forceinline__ void store_row(__half* p, long long piece, int live, const uint32_t (&w)[16]) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (q < live) *reinterpret_cast<uint4*>(p + q * piece) = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
}
// The mirror image of a warp's 32 x 32 block (a row per lane): through shared memory in rows of 80 bytes (no bank conflicts), back as
// transposed 8 x 8 matrices, out as 128 consecutive bytes per instruction.  `out`: row j0 of piece i0 / 8; pieces from
// `live` on do not exist.
__device__ __forceinline__ void store_mirror(__half* out, long long piece, int live, unsigned char* buf, const uint32_t (&w)[16]) {
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int q = 0; q < 4; ++q)
        *reinterpret_cast<uint4*>(buf + lane * 80 + q * 16) = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
    __syncwarp();
#pragma unroll
    for (int o = 0; o < 4; ++o) {
        if (o >= live) break;
        uint32_t r[4];
        const uint32_t at = smem_u32(buf) + (uint32_t)((8 * o + (lane & 7)) * 80 + (lane >> 3) * 16);
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(at)
                     : "memory");
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<uint32_t*>(out + o * piece + (8 * q + (lane >> 2)) * 8 + (lane & 3) * 2) = r[q];
    }
}

// B = b A + c A A near convergence is close to a multiple of the identity, -2.7 I, against which a X = 3.4 X is then set: most of
// what rounding B and X to fp16 costs is lost on that multiple.  It is taken out: with s = b t + c t^2, t the mean
// eigenvalue of A (its trace / m), B - s I is what is rounded and multiplied, and (a + s) X is added in fp32.  Pairs do
// not need it.  (96 x 576
// in fp16 operands: error of O 1.8e-3 without, 1.1e-3 with it.)
__device__ __forceinline__ float shift_of(float mean, float cb, float cc) { return mean * (cb + cc * mean); }

// The values that the results of a block of 32 x 32 need besides the sums: A for the polynomial, X for the
// last product of a step.  Row i, columns j0 ...
template <int SPLIT>
__device__ __forceinline__ void fetch(const IterateArgs& p, int phase, int step, int b, int i, int j0, Pairs& r) {
    if (i >= p.m) return;
    if (phase == PH_POLY)
        fetch_pairs(p.a + (((long long)b * p.a_pieces + (j0 >> 3)) * p.m + i) * 8, 8LL * p.m, p.a_lo, SPLIT == 2, p.a_pieces - (j0 >> 3), r);
    else if (phase == PH_APPLY)
        fetch_pairs(p.x[step & 1] + (((long long)b * p.x_pieces + (j0 >> 3)) * p.m + i) * 8, 8LL * p.m, p.x_lo, true, p.x_pieces - (j0 >> 3), r);
}

// What becomes of 32 columns of a row of the product: row i (of the warp's 32), columns j0 ..; `v` are the raw sums.
// Symmetric products: blocks of 32 x 32 below the diagonal are written twice (once mirrored), blocks on it once,
// blocks above it not at all; a block is a warp's, so that nothing here diverges.  Columns past the matrix hold
// zeros: their sums are of zeros.
template <int SPLIT>
__device__ __forceinline__ void emit(const IterateArgs& p, int phase, int step, int b, int i, int j0, float shift, const Pairs& r, unsigned char* buf,
                                     float (&v)[32]) {
    uint32_t h[16], l[16];
    if (phase == PH_APPLY) {
        if (i >= p.m) return;
        // a X is added in fp32 from the pair, so that only the smaller part of the step sees rounded operands
        add_pairs(r, true, p.coeff[step][0] + shift, kInvScale, v);
        pack_pairs(v, true, h, l);
        __half* out = p.x[(step + 1) & 1] + (((long long)b * p.x_pieces + (j0 >> 3)) * p.m + i) * 8;
        const int live = p.x_pieces - (j0 >> 3);
        store_row(out, 8LL * p.m, live, h);
        store_row(out + p.x_lo, 8LL * p.m, live, l);
        return;
    }
    const bool on_diagonal = j0 == (i & ~31);                 // the same for the whole warp
    if (SPLIT == 1 && phase == PH_GRAM && on_diagonal) {
        float d = 0.f;
#pragma unroll
        for (int k = 0; k < 32; ++k) if (k == (i & 31) && i < p.m) d = v[k];
        d = warp_sum(d) * kInvScale;
        if ((i & 31) == 0) p.trace[b * p.blocks + (i >> 5)] = d;
    }
    if (phase == PH_POLY) {
        add_pairs(r, SPLIT == 2, p.coeff[step][1], p.coeff[step][2] * kInvScale, v);
        if (SPLIT == 1 && on_diagonal) {
#pragma unroll
            for (int k = 0; k < 32; ++k) if (k == (i & 31)) v[k] -= shift * kScale;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] *= kInvScale;
    }
    if (i >= p.m) {                                           // the columns that fill up the last piece of the mirror image
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = 0.f;
    }
    pack_pairs(v, SPLIT == 2, h, l);
    __half* out = (phase == PH_GRAM ? p.a : p.b) + (long long)b * p.a_pieces * p.m * 8;
    if (i < p.m) {
        __half* row = out + ((long long)(j0 >> 3) * p.m + i) * 8;
        store_row(row, 8LL * p.m, p.a_pieces - (j0 >> 3), h);
        if constexpr (SPLIT == 2) store_row(row + p.a_lo, 8LL * p.m, p.a_pieces - (j0 >> 3), l);
    }
    if (!on_diagonal) {                                       // below it: j0 + 31 < m
        const int piece = (i & ~31) >> 3;
        __half* col = out + ((long long)piece * p.m + j0) * 8;
        store_mirror(col, 8LL * p.m, p.a_pieces - piece, buf, h);
        if constexpr (SPLIT == 2) store_mirror(col + p.a_lo, 8LL * p.m, p.a_pieces - piece, buf, l);
    }
}

// Unswizzled operand tile: core matrices of 8 rows x 16 bytes.  lbo / sbo: bytes between core matrices along k / along the free
// index for a K-major tile, the other way round for an MN-major one.
__device__ __forceinline__ uint64_t plain_smem_desc(uint32_t saddr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)((lbo_bytes >> 4) & 0x3FFFu) << 16) |
           ((uint64_t)((sbo_bytes >> 4) & 0x3FFFu) << 32) | ((uint64_t)1 << 46);
}

// ---- pairs of CTAs ------------------------------------------------------------------------------------------
constexpr uint32_t kLeaderMask = 0xFEFFFFFFu;      // a shared address of either CTA -> the same place in the first one
template <bool PAIR> __device__ __forceinline__ void load_box(void* dst, const CUtensorMap* m, int x, int y, int z, uint64_t* bar) {
    if constexpr (!PAIR) tma_load_3d(dst, m, x, y, z, bar);
    else        // the bytes land here, their arrival is counted on the first CTA's barrier
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                smem_u32(dst)),
            "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar) & kLeaderMask)
            : "memory");
}
template <bool PAIR> __device__ __forceinline__ void mma_f16(uint32_t d, uint64_t ad, uint64_t bd, uint32_t idesc, uint32_t accumulate) {
    if constexpr (!PAIR) umma_bf16(d, ad, bd, idesc, accumulate);      // kind::f16: the descriptor says fp16
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(ad), "l"(bd), "r"(idesc), "r"(accumulate)
            : "memory");
}
template <bool PAIR> __device__ __forceinline__ void commit(uint64_t* bar) {
    if constexpr (!PAIR) umma_commit(bar);
    else asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                          smem_u32(bar)),
                      "h"((uint16_t)3)
                      : "memory");
}
__device__ __forceinline__ void arrive_leader(uint64_t* bar) {
    asm volatile(
        "{\n\t.reg .b32 a;\n\t"
        "mapa.shared::cluster.u32 a, %0, 0;\n\t"
        "mbarrier.arrive.release.cluster.shared::cluster.b64 _, [a];\n\t}" ::"r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void cluster_meet() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// One thread of a converged warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

// All blocks of a cooperative launch meet: the writes before it are visible to all after it.  `ok` false in any thread ends the
// kernel of every block: the error word tells the others.  The wait is bounded like every other.
__device__ __forceinline__ bool grid_meet(const IterateArgs& p, uint32_t target, bool ok, int* flag) {
    const int bad = __syncthreads_or(!ok);
    if (threadIdx.x == 0) {
        int go = !bad;
        if (bad) atomicOr(p.err_word, 4096u);
        else {
            __threadfence();
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
    }
    __syncthreads();
    // what the other blocks wrote through the generic proxy is read by this warp's copies through the asynchronous one
    if (threadIdx.x < 32) asm volatile("fence.proxy.async;" ::: "memory");
    return *flag != 0;
}

// Matrix, row and column of tile t of a phase.
template <int ROWS> __device__ __forceinline__ void tile_of(const PhaseShape& ps, bool symmetric, int t, int& b, int& ti, int& tj) {
    b = t / ps.tiles;
    const int tt = t - b * ps.tiles;
    if (symmetric) lower_tile(tt, ps.bn == ROWS, ti, tj);
    else { ti = tt / ps.tiles_n; tj = tt - ti * ps.tiles_n; }
}

// What a phase multiplies, and how.
struct PhaseView {
    int step, phase, chunks, segment, total, share, splits, per;
    bool symmetric;
    uint32_t a_bytes, b_bytes;
};
template <int SPLIT, bool PAIR> __device__ __forceinline__ PhaseView phase_view(const IterateArgs& p, int turn) {
    PhaseView v;
    v.step = turn / 3;
    v.phase = turn - 3 * v.step;
    v.symmetric = v.phase != PH_APPLY;
    v.chunks = ((v.phase == PH_GRAM ? p.n : p.m) + 63) / 64;
    v.segment = SPLIT == 2 ? kSegment : v.chunks;
    v.splits = p.shape[v.phase].splits;
    v.per = p.shape[v.phase].per;
    v.total = p.shape[v.phase].tiles * p.batch * v.splits;      // units of work: (tile, part), parts of a tile side by side
    v.share = PAIR ? p.shape[v.phase].bn / 2 : p.shape[v.phase].bn;         // columns of the second operand held here
    v.a_bytes = 128 * 128;
    v.b_bytes = (uint32_t)v.share * 128;
    return v;
}

// The whole iteration in one launch: every phase deals its tiles (of all matrices) to the CTAs or pairs in turn, and
// all meet between phases.  Each role has a loop over the phases of its own, so that its registers are its own.
// The two issuing warps run as whole warps and elect the thread that issues: descriptors and addresses then stay in
// uniform registers.  (With the loop under `lane == 0` every product took 110 clocks to issue, whatever its size.)
// Measured, five steps: 4096 x 4096 in fp16 operands, with the kernels around it, 1.32 to 1.39 ms back to back under the power
// cap (SM clock 1.43 to 1.53 GHz), 1.15 to 1.18 ms in runs of a few calls; a CTA pair's chunk of 64 in 528 clocks where the
// products alone take 512, and 8 rounds of tiles for 7.1 rounds of work; 4 x 2048 x 512 with pairs of fp16 244 us, bound by operands from L2 (58
// bytes per clock and SM), 3000 clocks per meeting and 2500 to 9000 per tile's results; 6 x 256 x 256 105 us, 12000 clocks per
// phase of which the products take 3600.
template <int SPLIT, bool PAIR> __global__ void __launch_bounds__(kThreads, 1) ns_iterate_kernel(const __grid_constant__ IterateArgs p) {
    extern __shared__ unsigned char dyn_raw[];
    unsigned char* dyn = align1024(dyn_raw);
    __shared__ uint64_t full[kMaxStages], empty[kMaxStages], done[2], drained[2];
    __shared__ uint32_t tmem_base;
    __shared__ int flag;
    __shared__ __align__(16) unsigned char mirrors[8][32 * 80];
    constexpr int kRows = PAIR ? 256 : 128;                 // of a tile
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;      // uniform
    const uint32_t rank = PAIR ? cluster_rank() : 0u;
    const int unit = PAIR ? blockIdx.x >> 1 : blockIdx.x, units = PAIR ? gridDim.x >> 1 : gridDim.x;
    const int turns = 3 * p.steps;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kMaxStages; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(&done[s], 1); mbar_init(&drained[s], PAIR ? 16 : 8); }
        mbar_fence_init();
    }
    if (warp == 1) {
        if constexpr (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "r"(512) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else { tmem_alloc(&tmem_base, 512); tmem_relinquish(); }
    }
    tc_fence_before_sync();
    __syncthreads();
    if constexpr (PAIR) cluster_meet();                     // the other CTA's barriers are ready
    tc_fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base, 0);
    asm volatile("fence.proxy.async;" ::: "memory");
    bool ok = true;
    auto meet = [&](int turn) {
        return end_of_turn(turn, turns, ok, [&](bool good) { return grid_meet(p, (uint32_t)(turn + 1) * gridDim.x, good, &flag); });
    };

    if (warp == 0) {
        uint32_t ring = 0;             // one bit per stage: the parity of its next use
        for (int turn = 0; turn < turns && ok; ++turn) {
            const PhaseView v = phase_view<SPLIT, PAIR>(p, turn);
            const PhaseShape ps = p.shape[v.phase];
            const CUtensorMap* ta = v.phase == PH_GRAM ? &p.tm_a[v.step & 1] : v.phase == PH_POLY ? &p.tm_a[2] : &p.tm_a[3];
            const CUtensorMap* tb = v.phase == PH_GRAM ? &p.tm_g[v.step & 1] : v.phase == PH_POLY ? &p.tm_g[2] : &p.tm_n[v.step & 1];
            int s = 0;
            for (int t = unit; t < v.total && ok; t += units) {
                int b, ti, tj;
                tile_of<kRows>(ps, v.symmetric, t / v.splits, b, ti, tj);
                const int row = ti * kRows + (int)rank * 128, col = tj * ps.bn + (int)rank * v.share;
                const int q0 = t % v.splits * v.per, q1 = min(q0 + v.per, v.chunks);
                for (int q = q0; q < q1; ++q) {
                    ok = mbar_wait_warp(&empty[s], ((ring >> s) & 1u) ^ 1u);
                    if (!ok) break;
                    if (elect_one()) {
                        unsigned char* st = dyn + (size_t)s * ps.stage_bytes;
                        if (rank == 0) mbar_expect_tx(&full[s], (uint32_t)ps.stage_bytes * (PAIR ? 2u : 1u));
#pragma unroll
                        for (int h = 0; h < SPLIT; ++h) {
                            const int z = h * p.batch + b;
                            unsigned char* sb = st + SPLIT * v.a_bytes + h * v.b_bytes;
                            load_box<PAIR>(st + h * v.a_bytes, ta, row * 2, q * 8, z, &full[s]);
                            if (v.symmetric) load_box<PAIR>(sb, tb, col * 2, q * 8, z, &full[s]);
                            else load_box<PAIR>(sb, tb, q * 128, col / 8, z, &full[s]);
                        }
                    }
                    __syncwarp();
                    ring ^= 1u << s;
                    if (++s == ps.stages) s = 0;
                }
            }
            ok = meet(turn);
        }
    } else if (warp == 1) {
        uint32_t ring = 0, use = 0;    // use: accumulators taken so far
        for (int turn = 0; turn < turns && ok; ++turn) {
            const PhaseView v = phase_view<SPLIT, PAIR>(p, turn);
            const PhaseShape ps = p.shape[v.phase];
            if (rank == 0) {
                // fp16 x fp16 -> fp32; B is K-major in the symmetric products, MN-major otherwise
                const uint32_t idesc = (1u << 4) | ((v.symmetric ? 0u : 1u) << 16) | ((uint32_t)(ps.bn >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24);
                const uint64_t a_form = plain_smem_desc(0, 2048, 128);
                const uint64_t b_form = v.symmetric ? plain_smem_desc(0, (uint32_t)v.share * 16u, 128) : plain_smem_desc(0, 128, 1024);
                const uint32_t b_step = (v.symmetric ? (uint32_t)v.share * 32u : 256u) >> 4;      // 16 k further, in 16 bytes
                const uint32_t ring0 = smem_u32(dyn) >> 4;      // (in the first CTA of a pair, whose addresses carry no rank)
                int s = 0;
                for (int t = unit; t < v.total && ok; t += units) {
                    const int n = min(v.per, v.chunks - t % v.splits * v.per);
                    int in = 0;                                 // chunks in the present accumulator
                    for (int q = 0; q < n; ++q) {
                        const int buf = (int)(use & 1u);
                        const bool first = in == 0, last = in == v.segment - 1 || q == n - 1;
                        in = last ? 0 : in + 1;
                        if (first && use >= 2) ok = mbar_wait_warp(&drained[buf], ((use >> 1) - 1) & 1u);
                        if (ok) ok = mbar_wait_warp(&full[s], (ring >> s) & 1u);
                        if (!ok) break;
                        tc_fence_after_sync();
                        if (elect_one()) {
                            const uint32_t d = tmem + (uint32_t)(buf * 256);
                            const uint32_t at = ring0 + (uint32_t)s * ((uint32_t)ps.stage_bytes >> 4);
                            const uint64_t a_hi = a_form + at, a_lo = a_hi + (v.a_bytes >> 4);
                            const uint64_t b_hi = b_form + at + SPLIT * (v.a_bytes >> 4), b_lo = b_hi + (v.b_bytes >> 4);
#pragma unroll
                            for (int ks = 0; ks < 4; ++ks) {
                                mma_f16<PAIR>(d, a_hi + ks * 256, b_hi + ks * b_step, idesc, !(first && ks == 0));
                                if constexpr (SPLIT == 2) {
                                    mma_f16<PAIR>(d, a_hi + ks * 256, b_lo + ks * b_step, idesc, 1u);
                                    mma_f16<PAIR>(d, a_lo + ks * 256, b_hi + ks * b_step, idesc, 1u);
                                }
                            }
                            commit<PAIR>(&empty[s]);
                            if (last) commit<PAIR>(&done[buf]);
                        }
                        __syncwarp();
                        ring ^= 1u << s;
                        if (++s == ps.stages) s = 0;
                        if (last) ++use;
                    }
                }
            }
            ok = meet(turn);
        }
    } else {
        uint32_t use = 0;              // accumulators emptied so far
        for (int turn = 0; turn < turns && ok; ++turn) {
            const PhaseView view = phase_view<SPLIT, PAIR>(p, turn);
            const PhaseShape ps = p.shape[view.phase];
            const int step = view.step, phase = view.phase, segment = view.segment, total = view.total;
            const bool symmetric = view.symmetric;
            unsigned char* const mirror = mirrors[warp - 2];
            const int quarter = warp & 3, half = (warp - 2) >> 2;
            const int cols = ps.bn / 2;                       // of this warp
            constexpr int kChunks = PAIR ? 4 : 2;             // of 32 columns, at most
            const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * cols);
            for (int t = unit; t < total && ok; t += units) {
                int b, ti, tj;
                tile_of<kRows>(ps, symmetric, t / view.splits, b, ti, tj);
                const int part = t % view.splits, chunks = min(view.per, view.chunks - part * view.per);
                const bool split = view.splits > 1;
                const int i0 = ti * kRows + (int)rank * 128 + quarter * 32, i = i0 + lane;
                const int j0 = tj * ps.bn + half * cols;
                // columns past the matrix, or past the diagonal of the warp's rows, are not read (the same for the whole warp)
                const int reach = i0 >= p.m ? 0 : symmetric ? min(p.m, i0 + 32) : p.n;
                // where this warp's sums go when the tile is split
                const int slot = (t / view.splits * (PAIR ? 2 : 1) + (int)rank) * 8 + warp - 2;
                const long long tile_floats = (long long)cols * 32, part_floats = 8 * tile_floats;
                float* const place = p.partial + ((long long)(slot >> 3) * view.splits * 8 + (slot & 7)) * tile_floats + lane;
                Pairs pr;
                if (!split && j0 < reach) fetch<SPLIT>(p, phase, step, b, i, j0, pr);        // on its way while the product runs
                float shift = 0.f;
                if (SPLIT == 1 && phase != PH_GRAM) {
                    float trace = 0.f;
                    for (int k = lane; k < p.blocks; k += 32) trace += p.trace[b * p.blocks + k];
                    shift = shift_of(warp_sum(trace) * kInvScale / (float)p.m, p.coeff[step][1], p.coeff[step][2]);
                }
                float acc[SPLIT == 2 ? kChunks : 1][32];
                if constexpr (SPLIT == 2) {
#pragma unroll
                    for (int c = 0; c < kChunks; ++c)
#pragma unroll
                        for (int k = 0; k < 32; ++k) acc[c][k] = 0.f;
                }
                for (int q = 0; q < chunks; q += segment) {
                    const int buf = (int)(use & 1u);
                    ok = mbar_wait_warp(&done[buf], (use >> 1) & 1u);
                    ++use;
                    if (!ok) break;
                    tc_fence_after_sync();
#pragma unroll
                    for (int c = 0; c < kChunks; ++c) {
                        const int j = j0 + c * 32;
                        if (c * 32 < cols && j < reach) {
                            uint32_t raw[32];
                            tmem_ld32(lanes + (uint32_t)(buf * 256 + c * 32), raw);
                            if constexpr (SPLIT == 1) {
                                const Pairs now = pr;
                                if (!split && c + 1 < kChunks && (c + 1) * 32 < cols && j + 32 < reach) fetch<SPLIT>(p, phase, step, b, i, j + 32, pr);
                                tmem_ld_wait();
#pragma unroll
                                for (int k = 0; k < 32; ++k) acc[0][k] = __uint_as_float(raw[k]);
                                if (split) {
#pragma unroll
                                    for (int k = 0; k < 32; ++k) place[part * part_floats + (c * 32 + k) * 32] = acc[0][k];
                                } else emit<SPLIT>(p, phase, step, b, i, j, shift, now, mirror, acc[0]);
                                __syncwarp();                 // the next read of tensor memory is the whole warp's
                            } else {
                                tmem_ld_wait();
#pragma unroll
                                for (int k = 0; k < 32; ++k) acc[c][k] += __uint_as_float(raw[k]);
                            }
                        }
                    }
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) {
                        if constexpr (PAIR) arrive_leader(&drained[buf]);
                        else mbar_arrive(&drained[buf]);
                    }
                }
                if (!ok) break;
                if (split) {
                    // The warp that brings a tile's last part adds all parts, in their order whoever it is, and goes on.
                    if constexpr (SPLIT == 2) {
#pragma unroll
                        for (int c = 0; c < kChunks; ++c)
                            if (c * 32 < cols && j0 + c * 32 < reach) {
#pragma unroll
                                for (int k = 0; k < 32; ++k) place[part * part_floats + (c * 32 + k) * 32] = acc[c][k];
                            }
                    }
                    __threadfence();
                    __syncwarp();
                    uint32_t before = 0;
                    if (lane == 0) before = atomicAdd(p.arrived + slot, 1u);
                    before = __shfl_sync(0xffffffffu, before, 0);
                    if (before != (uint32_t)view.splits - 1u) continue;
                    __threadfence();
                    if (lane == 0) p.arrived[slot] = 0;
#pragma unroll 1
                    for (int c = 0; c * 32 < cols && j0 + c * 32 < reach; ++c) {
                        fetch<SPLIT>(p, phase, step, b, i, j0 + c * 32, pr);
                        float sum[32];
#pragma unroll
                        for (int k = 0; k < 32; ++k) sum[k] = 0.f;
#pragma unroll 1
                        for (int r = 0; r < view.splits; r += 2) {          // two parts on their way at once, added in order
                            float x[32], y[32];
                            const bool two = r + 1 < view.splits;
#pragma unroll
                            for (int k = 0; k < 32; ++k) x[k] = __ldcg(place + r * part_floats + (c * 32 + k) * 32);
#pragma unroll
                            for (int k = 0; k < 32; ++k) y[k] = two ? __ldcg(place + (r + 1) * part_floats + (c * 32 + k) * 32) : 0.f;
#pragma unroll
                            for (int k = 0; k < 32; ++k) sum[k] = (sum[k] + x[k]) + y[k];
                        }
                        emit<SPLIT>(p, phase, step, b, i, j0 + c * 32, shift, pr, mirror, sum);
                        __syncwarp();
                    }
                } else if constexpr (SPLIT == 2) {
#pragma unroll
                    for (int c = 0; c < kChunks; ++c) {
                        if (c * 32 < cols && j0 + c * 32 < reach) {
                            if (c > 0) fetch<SPLIT>(p, phase, step, b, i, j0 + c * 32, pr);
                            emit<SPLIT>(p, phase, step, b, i, j0 + c * 32, shift, pr, mirror, acc[c]);
                        }
                        __syncwarp();
                    }
                }
            }
            ok = meet(turn);
        }
    }
    if (!ok) {
        atomicOr(p.err_word, 4096u);
        let_settle();
    }
    tc_fence_before_sync();
    __syncthreads();
    if constexpr (PAIR) cluster_meet();           // nothing of the other CTA refers to this one any more
    tc_fence_after_sync();
    if (warp == 1) {
        if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
        else tmem_dealloc(tmem, 512);
    }
}

// ---- small matrices ---------------------------------------------------------------------------------------
// m <= 128 and n <= 2048: a cluster of CTAs per matrix holds everything on chip for the whole call, in one launch.  A CTA has a slice
// of at most 256 columns of X: as fp32 in tensor memory and as fp16 (pairs) in shared memory.  Only X X^T needs the other
// slices: every CTA owns some of its columns, the others send it their partial sums of these (stores into its shared
// memory), it adds them in the order of the ranks and sends the result to all.  The polynomial is computed by every
// CTA, B X by each for its slice.  (The general kernel takes 4 to 5 us per product of this size, of which the product
// itself is a tenth: two passes through L2 and a meeting of the grid; 96 x 576 took 71 us there and takes 45 here, 11000
// clocks per step: 3000 the partial sums and A, 4000 meetings, 2000 products, 2000 results.  More rows do not fit one
// accumulator, more columns not a cluster of 8.  Reading the others' sums instead of being sent
// them took 4500 clocks per step, three times as long.)
constexpr int kSmallThreads = 256;
constexpr int kSmallCols = 256;            // columns of a slice, at most
constexpr int kSmallCluster = 8;
constexpr int kSmallPart = 86016;          // partial sums that a CTA is sent: at most 7 x 3 pieces of 4 KB; also tiles on their way in and out
// A or B: 32 KB, as pairs 64, then in the partial sums' place (all together would not fit)
constexpr int small_region(int split) { return split == 1 ? kSmallPart + 32768 : kSmallPart; }

struct SmallArgs {
    Source src;
    const void* w[kMaxLayers];             // Muon: weights
    void* w_out[kMaxLayers];
    void* out;                             // O
    int m, n, slice, cluster, transposed, steps;
    int out_bf16, taps;
    float keep, f, eps;
    float coeff[GF_NS_MAX_STEPS][3];
    FastDiv div_taps;
    uint32_t *err_word, *status;           // the library's word for waits that run out; the workspace's, cleared here
};

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
        "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
        "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, int rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void peer_store4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint32_t pack_half2(float x, float y) {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// (hi, lo) of a pair of values as fp16
__device__ __forceinline__ void split_half2(float x, float y, uint32_t& hi, uint32_t& lo) {
    const __half2 h = __floats2half2_rn(x, y);
    const float2 back = __half22float2(h);
    hi = *reinterpret_cast<const uint32_t*>(&h);
    lo = pack_half2(x - back.x, y - back.y);
}

template <int SPLIT, bool MUON> __global__ void __launch_bounds__(kSmallThreads, 1) ns_small_kernel(const __grid_constant__ SmallArgs p) {
    extern __shared__ unsigned char dyn_raw[];
    unsigned char* const region = align1024(dyn_raw);                     // partial sums, tiles
    unsigned char* const as = region + (SPLIT == 1 ? kSmallPart : 0);     // A / B: [part][16][128][8] fp16
    unsigned char* const xs = region + (SPLIT == 1 ? kSmallPart + 32768 : kSmallPart);      // X: [part][slice / 8][128][8] fp16
    __shared__ uint64_t bar;
    __shared__ uint32_t tmem_base;
    __shared__ double red[kSmallThreads / 32], total;
    __shared__ uint32_t send_to[16];                                      // where the partial sums of a piece of 8 columns go
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const int quarter = warp & 3, half = warp >> 2, row = quarter * 32 + lane;      // tensor memory: this thread's lane
    const int rank = p.cluster > 1 ? (int)cluster_rank() : 0, b = blockIdx.x / p.cluster;
    const int c0 = rank * p.slice, width = max(0, min(p.slice, p.n - c0));          // columns of X that this CTA has
    const uint32_t x_lo = (uint32_t)p.slice * 256u;                                 // bytes to the low parts
    const Source& s = p.src;
    auto all_meet = [&] { if (p.cluster > 1) cluster_meet(); else __syncthreads(); };
    if (tid == 0) {
        mbar_init(&bar, 1);
        mbar_fence_init();
        if (blockIdx.x == 0) *p.status = 0;
    }
    if (warp == 0) { tmem_alloc(&tmem_base, 512); tmem_relinquish(); }
    tc_fence_before_sync();
    all_meet();
    tc_fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base, 0);
    const uint32_t tx = tmem + ((uint32_t)(quarter * 32) << 16), td = tx + 256u;    // X; sums
    bool ok = true;
    uint32_t phase = 0;

    // ---- in: 64 columns of X at a time through a tile [column][row], raw into tensor memory
    float* tile = reinterpret_cast<float*>(region);                       // [64][129]
    // Pieces of 8 columns of A: rank r owns those from r P / cluster on.  Rows and pieces past the matrix stay out.
    const int P = (p.m + 7) / 8;
    auto first_of = [&](int r) { return (r * P + p.cluster - 1) / p.cluster; };
    const int mine = first_of(rank), count = first_of(rank + 1) - mine;   // at most 8
    if (p.cluster > 1 && tid < P) {
        const int owner = tid * p.cluster / P, first = first_of(owner), n = first_of(owner + 1) - first;
        send_to[tid] = peer_addr(smem_u32(region) + (uint32_t)((rank * n + tid - first) * 4096), owner);      // there: [rank][piece][column / 4][row][4]
    }
    float q = 0.f;
    for (int j0 = 0; j0 < p.slice; j0 += 64) {
        float u[32];
        // the type is asked for outside the loop, so that all 32 loads are on their way at once
        auto take = [&](const auto* g) {
            const int i = p.transposed ? tid & 127 : tid >> 6, j = j0 + (p.transposed ? tid >> 7 : tid & 63);
            const int di = p.transposed ? 0 : 4, dj = p.transposed ? 2 : 0;
            const long long e0 = p.transposed ? (long long)(c0 + j) * s.cols + i : (long long)i * s.cols + c0 + j;
            const long long de = p.transposed ? 2LL * s.cols : 4LL * s.cols;
            g += (s.batched ? (long long)b * s.rows * s.cols : 0) + e0 * s.taps;
#pragma unroll
            for (int k = 0; k < 32; ++k) u[k] = i + di * k < p.m && j + dj * k < width ? to_f32(g[de * s.taps * k]) : 0.f;
            if constexpr (MUON) {
                const float* from = s.mom[b] + e0;
                float* to = s.mom_out[b] + e0;
                float mo[32];
#pragma unroll
                for (int k = 0; k < 32; ++k) mo[k] = i + di * k < p.m && j + dj * k < width ? from[de * k] : 0.f;
#pragma unroll
                for (int k = 0; k < 32; ++k) {
                    mo[k] = s.momentum * mo[k] + (1.f - s.momentum) * u[k];
                    u[k] = s.nesterov ? (1.f - s.momentum) * u[k] + s.momentum * mo[k] : mo[k];
                    if (i + di * k < p.m && j + dj * k < width) to[de * k] = mo[k];
                }
            }
        };
        if (s.bf16) take(static_cast<const __nv_bfloat16*>(s.g[s.batched ? 0 : b]));
        else take(static_cast<const float*>(s.g[s.batched ? 0 : b]));
#pragma unroll
        for (int k = 0; k < 32; ++k) {
            const int i = p.transposed ? tid & 127 : (tid >> 6) + 4 * k, j = p.transposed ? (tid >> 7) + 2 * k : tid & 63;
            tile[j * 129 + i] = u[k];
            q += u[k] * u[k];
        }
        __syncthreads();
        if (j0 + half * 32 < p.slice) {
            uint32_t v[32];
#pragma unroll
            for (int k = 0; k < 32; ++k) v[k] = __float_as_uint(tile[(half * 32 + k) * 129 + row]);
            tmem_st32(tx + (uint32_t)(j0 + half * 32), v);
        }
        __syncthreads();
    }
    tmem_st_wait();
    // ---- norm of the whole matrix: the CTAs' sums in the order of their ranks
    {
        double d = q;
        for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
        if (lane == 0) red[warp] = d;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kSmallThreads / 32; ++w) d += red[w];
            total = d;
        }
        all_meet();
        d = 0;
        for (int k = 0; k < p.cluster; ++k) {
            double v = total;
            if (p.cluster > 1) asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(peer_addr(smem_u32(&total), k)) : "memory");
            d += v;
        }
        const float scale0 = kScale / ((float)sqrt(d) + p.eps);
        const float scale = isinf(scale0) ? 0.f : scale0;                 // a matrix of zeros with eps = 0 gives zeros
        for (int j = half * 32; j < p.slice; j += 64) {
            uint32_t v[32];
            tmem_ld32(tx + (uint32_t)j, v);
            tmem_ld_wait();
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                uint32_t h[4], l[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = __uint_as_float(v[8 * g + 2 * e]) * scale, y = __uint_as_float(v[8 * g + 2 * e + 1]) * scale;
                    v[8 * g + 2 * e] = __float_as_uint(x);
                    v[8 * g + 2 * e + 1] = __float_as_uint(y);
                    split_half2(x, y, h[e], l[e]);
                }
                if (j + 8 * g < p.slice) {
                    unsigned char* dst = xs + ((j >> 3) + g) * 2048 + row * 16;
                    *reinterpret_cast<uint4*>(dst) = make_uint4(h[0], h[1], h[2], h[3]);
                    if constexpr (SPLIT == 2) *reinterpret_cast<uint4*>(dst + x_lo) = make_uint4(l[0], l[1], l[2], l[3]);
                }
            }
            tmem_st32(tx + (uint32_t)j, v);
        }
        tmem_st_wait();
    }

    // One product, issued by one thread and waited for by all: D (columns from `col` on) = A B over `steps16` steps of 16.
    // K-major operands: 16-byte columns 2048 bytes apart; B of the last product MN-major.
    // (in a cluster the bits above a shared address' own 18 name the CTA: they are not the descriptor's)
    const uint32_t a_at = (smem_u32(as) >> 4) & 0x3FFFu, x_at = (smem_u32(xs) >> 4) & 0x3FFFu;
    const uint64_t k_major = plain_smem_desc(0, 2048, 128), mn_major = plain_smem_desc(0, 128, 2048);
    auto begin = [&] {                                       // operands were written through the generic proxy
        fence_proxy_async_smem();
        tc_fence_before_sync();
        all_meet();
        asm volatile("fence.proxy.async;" ::: "memory");     // those that other CTAs wrote
        tc_fence_after_sync();
    };
    auto finish = [&] {
        if (ok) ok = mbar_wait_bounded(&bar, phase);         // (after a wait that ran out nothing is waited for any more)
        phase ^= 1u;
        tc_fence_after_sync();
    };
    const uint32_t rows16 = (uint32_t)(p.m + 15) / 16u;

    for (int step = 0; step < p.steps; ++step) {
        // ---- partial X X^T: two accumulators of at most 8 steps each (24 additions with pairs)
        begin();
        const int k16 = p.slice / 16, first = (k16 + 1) / 2;
        if (warp == 0 && elect_one()) {
            const uint32_t idesc = (1u << 4) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
            for (int k = 0; k < k16; ++k) {
                const uint64_t hi = k_major + x_at + (uint32_t)k * 256u, lo = hi + (x_lo >> 4);
                const uint32_t d = tmem + 256u + (k >= first ? 128u : 0u);
                umma_bf16(d, hi, hi, idesc, k != 0 && k != first);
                if constexpr (SPLIT == 2) { umma_bf16(d, hi, lo, idesc, 1u); umma_bf16(d, lo, hi, idesc, 1u); }
            }
            umma_commit(&bar);
        }
        __syncwarp();
        finish();
        // this thread's row, 64 columns of half `half`; then to where they are added up
        const bool two = k16 > first;
        if (p.cluster == 1) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int j = half * 64 + c * 32;
                uint32_t v[32], w[32];
                tmem_ld32(td + (uint32_t)j, v);
                if (two) tmem_ld32(td + 128u + (uint32_t)j, w);
                tmem_ld_wait();
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    uint32_t h[4], l[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int k = 8 * g + 2 * e;
                        const float x = __uint_as_float(v[k]) + (two ? __uint_as_float(w[k]) : 0.f);
                        const float y = __uint_as_float(v[k + 1]) + (two ? __uint_as_float(w[k + 1]) : 0.f);
                        split_half2(x * kInvScale, y * kInvScale, h[e], l[e]);
                    }
                    unsigned char* dst = as + ((j >> 3) + g) * 2048 + row * 16;
                    *reinterpret_cast<uint4*>(dst) = make_uint4(h[0], h[1], h[2], h[3]);
                    if constexpr (SPLIT == 2) *reinterpret_cast<uint4*>(dst + 32768) = make_uint4(l[0], l[1], l[2], l[3]);
                }
            }
        } else {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int j = half * 64 + c * 32;
                if (j >= p.m || quarter * 32 >= p.m) continue;            // the same for the whole warp
                uint32_t v[32], w[32];
                tmem_ld32(td + (uint32_t)j, v);
                if (two) tmem_ld32(td + 128u + (uint32_t)j, w);
                tmem_ld_wait();
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int piece = (j >> 3) + g;
                    if (piece >= P) continue;
                    float f[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(v[8 * g + e]) + (two ? __uint_as_float(w[8 * g + e]) : 0.f);
                    const uint32_t to = send_to[piece] + (uint32_t)(row * 16);
                    peer_store4(to, __float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
                    peer_store4(to + 2048u, __float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
                }
            }
            cluster_meet();
            float sum[4][8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int piece = (tid >> 7) + 2 * k, i = tid & 127;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[k][e] = 0.f;
                if (piece < count && i < p.m)
                    for (int r = 0; r < p.cluster; ++r) {
                        const float4 x = *reinterpret_cast<const float4*>(region + (r * count + piece) * 4096 + i * 16);
                        const float4 y = *reinterpret_cast<const float4*>(region + (r * count + piece) * 4096 + 2048 + i * 16);
                        sum[k][0] += x.x; sum[k][1] += x.y; sum[k][2] += x.z; sum[k][3] += x.w;
                        sum[k][4] += y.x; sum[k][5] += y.y; sum[k][6] += y.z; sum[k][7] += y.w;
                    }
            }
            if constexpr (SPLIT == 2) cluster_meet();        // all have added: A may take the partial sums' place
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int piece = (tid >> 7) + 2 * k, i = tid & 127;
                if (piece < count) {
                    uint32_t h[4], l[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) split_half2(sum[k][2 * e] * kInvScale, sum[k][2 * e + 1] * kInvScale, h[e], l[e]);
                    const uint32_t at = smem_u32(as) + (uint32_t)((mine + piece) * 2048 + i * 16);
                    for (int r = 0; r < p.cluster; ++r) {
                        const uint32_t to = peer_addr(at, r);
                        peer_store4(to, h[0], h[1], h[2], h[3]);
                        if constexpr (SPLIT == 2) peer_store4(to + 32768u, l[0], l[1], l[2], l[3]);
                    }
                }
            }
            // the odd piece that fills up 16 contracted columns
            if (P & 1) {
                if (tid < 128) {
                    *reinterpret_cast<uint4*>(as + P * 2048 + tid * 16) = make_uint4(0u, 0u, 0u, 0u);
                    if constexpr (SPLIT == 2) *reinterpret_cast<uint4*>(as + 32768 + P * 2048 + tid * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
            }
        }
        // ---- A A, and B = b A + c A A in A's place
        begin();
        if (warp == 0 && elect_one()) {
            const uint32_t idesc = (1u << 4) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
            for (uint32_t k = 0; k < rows16; ++k) {
                const uint64_t hi = k_major + a_at + k * 256u, lo = hi + (32768u >> 4);
                umma_bf16(tmem + 256u, hi, hi, idesc, k != 0);
                if constexpr (SPLIT == 2) { umma_bf16(tmem + 256u, hi, lo, idesc, 1u); umma_bf16(tmem + 256u, lo, hi, idesc, 1u); }
            }
            umma_commit(&bar);
        }
        __syncwarp();
        finish();
        // the mean eigenvalue of A is taken out of B (see `shift_of`); every warp adds the diagonal itself
        float shift = 0.f;
        if constexpr (SPLIT == 1) {
            float trace = 0.f;
            for (int i = lane; i < p.m; i += 32) trace += __half2float(*reinterpret_cast<const __half*>(as + (i >> 3) * 2048 + i * 16 + (i & 7) * 2));
            shift = shift_of(warp_sum(trace) * kInvScale / (float)p.m, p.coeff[step][1], p.coeff[step][2]);
            __syncthreads();                                 // before B takes A's place
        }
        const float ca = p.coeff[step][0] + shift, cb = p.coeff[step][1], cc = p.coeff[step][2] * kInvScale;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int j = half * 64 + c * 32;
            uint32_t v[32];
            tmem_ld32(td + (uint32_t)j, v);
            tmem_ld_wait();
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                unsigned char* at = as + ((j >> 3) + g) * 2048 + row * 16;
                const uint4 hv = *reinterpret_cast<const uint4*>(at);
                uint4 lv = make_uint4(0u, 0u, 0u, 0u);
                if constexpr (SPLIT == 2) lv = *reinterpret_cast<const uint4*>(at + 32768);
                const uint32_t hw[4] = {hv.x, hv.y, hv.z, hv.w}, lw[4] = {lv.x, lv.y, lv.z, lv.w};
                uint32_t h[4], l[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int k = 8 * g + 2 * e;
                    float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hw[e]));
                    if constexpr (SPLIT == 2) {
                        const float2 o = __half22float2(*reinterpret_cast<const __half2*>(&lw[e]));
                        f.x += o.x; f.y += o.y;
                    }
                    split_half2(cb * f.x + cc * __uint_as_float(v[k]) - (j + k == row ? shift * kScale : 0.f),
                                cb * f.y + cc * __uint_as_float(v[k + 1]) - (j + k + 1 == row ? shift * kScale : 0.f), h[e], l[e]);
                }
                *reinterpret_cast<uint4*>(at) = make_uint4(h[0], h[1], h[2], h[3]);
                if constexpr (SPLIT == 2) *reinterpret_cast<uint4*>(at + 32768) = make_uint4(l[0], l[1], l[2], l[3]);
            }
        }
        // ---- B X for this slice, X = a X + B X
        fence_proxy_async_smem();
        tc_fence_before_sync();
        __syncthreads();
        tc_fence_after_sync();
        if (warp == 0 && elect_one()) {
            const uint32_t idesc = (1u << 4) | (1u << 16) | ((uint32_t)(p.slice >> 3) << 17) | ((128u >> 4) << 24);
            for (uint32_t k = 0; k < rows16; ++k) {
                const uint64_t hi = k_major + a_at + k * 256u, lo = hi + (32768u >> 4);
                const uint64_t xhi = mn_major + x_at + k * 16u, xlo = xhi + (x_lo >> 4);
                umma_bf16(tmem + 256u, hi, xhi, idesc, k != 0);
                if constexpr (SPLIT == 2) { umma_bf16(tmem + 256u, hi, xlo, idesc, 1u); umma_bf16(tmem + 256u, lo, xhi, idesc, 1u); }
            }
            umma_commit(&bar);
        }
        __syncwarp();
        finish();
        const bool last = step + 1 == p.steps;
        for (int j = half * 32; j < p.slice; j += 64) {
            uint32_t v[32], w[32];
            tmem_ld32(tx + (uint32_t)j, v);
            tmem_ld32(td + (uint32_t)j, w);
            tmem_ld_wait();
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                uint32_t h[4], l[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int k = 8 * g + 2 * e;
                    const float x = ca * __uint_as_float(v[k]) + kInvScale * __uint_as_float(w[k]);
                    const float y = ca * __uint_as_float(v[k + 1]) + kInvScale * __uint_as_float(w[k + 1]);
                    v[k] = __float_as_uint(x);
                    v[k + 1] = __float_as_uint(y);
                    split_half2(x, y, h[e], l[e]);
                }
                if (!last && j + 8 * g < p.slice) {
                    unsigned char* dst = xs + ((j >> 3) + g) * 2048 + row * 16;
                    *reinterpret_cast<uint4*>(dst) = make_uint4(h[0], h[1], h[2], h[3]);
                    if constexpr (SPLIT == 2) *reinterpret_cast<uint4*>(dst + x_lo) = make_uint4(l[0], l[1], l[2], l[3]);
                }
            }
            tmem_st32(tx + (uint32_t)j, v);
        }
        tmem_st_wait();
    }

    // ---- out, through the same tile
    for (int j0 = 0; j0 < width; j0 += 64) {
        __syncthreads();
        if (j0 + half * 32 < p.slice) {
            uint32_t v[32];
            tmem_ld32(tx + (uint32_t)(j0 + half * 32), v);
            tmem_ld_wait();
#pragma unroll
            for (int k = 0; k < 32; ++k) tile[(half * 32 + k) * 129 + row] = __uint_as_float(v[k]) * kInvScale;
        }
        __syncthreads();
        const int cols = min(64, width - j0);
        if constexpr (!MUON) {
            auto give = [&](auto* o) {
                const int i = p.transposed ? tid & 127 : tid >> 6, j = p.transposed ? tid >> 7 : tid & 63;
                const int di = p.transposed ? 0 : 4, dj = p.transposed ? 2 : 0;
                const long long de = p.transposed ? 2LL * s.cols : 4LL * s.cols;
                using Out = typename std::remove_pointer<decltype(o)>::type;
                o += (long long)b * s.rows * s.cols + (p.transposed ? (long long)(c0 + j0 + j) * s.cols + i : (long long)i * s.cols + c0 + j0 + j);
#pragma unroll
                for (int k = 0; k < 32; ++k)
                    if (i + di * k < p.m && j + dj * k < cols) o[de * k] = from_f32<Out>(tile[(j + dj * k) * 129 + i + di * k]);
            };
            if (p.out_bf16) give(static_cast<__nv_bfloat16*>(p.out));
            else give(static_cast<float*>(p.out));
        } else {
            // rows of W as they lie in memory: columns j of row i, or (transposed) all i of row j; taps values each.  All rows of the
            // tile in one sequence, 24 values on their way per thread (8: 13 us of the 59 for 576 x 96).
            const int nr = p.transposed ? cols : p.m, nc = p.transposed ? p.m : cols, span = nc * p.taps, all = nr * span;
            const long long base = (p.transposed ? (long long)(c0 + j0) * s.cols : (long long)(c0 + j0)) * p.taps, pitch = (long long)s.cols * p.taps;
            auto update = [&](const auto* w, auto* out) {
                using Weight = typename std::remove_pointer<decltype(out)>::type;
                constexpr int kAtOnce = 24;
                // place `at` = row r, value e of the row; the next of this thread lies kSmallThreads further
                const int dr = kSmallThreads / span, de = kSmallThreads - dr * span;
                int r = tid / span, e = tid - r * span;
                for (int at = tid; at < all; at += kSmallThreads * kAtOnce) {
                    float v[kAtOnce];
                    long long o[kAtOnce];
                    int from[kAtOnce];
#pragma unroll
                    for (int k = 0; k < kAtOnce; ++k) {
                        const int c = (int)p.div_taps.div((uint32_t)e);
                        o[k] = base + r * pitch + e;
                        from[k] = p.transposed ? r * 129 + c : c * 129 + r;
                        v[k] = at + kSmallThreads * k < all ? to_f32(w[o[k]]) : 0.f;
                        r += dr;
                        e += de;
                        if (e >= span) { e -= span; ++r; }
                    }
#pragma unroll
                    for (int k = 0; k < kAtOnce; ++k)
                        if (at + kSmallThreads * k < all) out[o[k]] = from_f32<Weight>(p.keep * v[k] - p.f * tile[from[k]]);
                }
            };
            if (p.out_bf16) update(static_cast<const __nv_bfloat16*>(p.w[b]), static_cast<__nv_bfloat16*>(p.w_out[b]));
            else update(static_cast<const float*>(p.w[b]), static_cast<float*>(p.w_out[b]));
        }
    }
    if (!ok) {
        atomicOr(p.err_word, 16384u);
        let_settle();
    }
    tc_fence_before_sync();
    all_meet();                                              // no CTA leaves while its memory may be read
    tc_fence_after_sync();
    if (warp == 0) tmem_dealloc(tmem, 512);
}

// ---- host side --------------------------------------------------------------------------------------------
struct Shapes {
    PhaseShape shape[3];
    bool pair;
    int units;                     // CTAs or pairs that run at once
    size_t partial_bytes;
};
struct NsPlan {
    int batch, rows, cols, m, n, x_pieces, a_pieces, split, transposed;
    int norm_blocks;
    size_t off_part, off_x[2], off_a, off_b, off_trace, off_partial, total;
    long long x_lo, a_lo;          // elements from the high to the low parts
    Shapes shapes;                 // (not of small matrices)
};

// Clocks that a phase takes, and its shape with the fewest.  A chunk of 64 of the contracted index costs what its bytes take
// to come from L2 (58 per clock and SM, measured) or its products take to run, whichever is more; a tile's results cost
// by their width, under the next tile's products except for the last; a split tile costs the way through L2.  (Splitting:
// 300 x 3000 219 -> 140 us, 1001 x 2048 264 -> 239, both with pairs of fp16.)
PhaseShape phase_shape(const NsPlan& p, int phase, bool pair, int units, double* clocks) {
    PhaseShape best = {};
    double least = 0;
    const int rows = pair ? 256 : 128;
    const bool symmetric = phase != PH_APPLY;
    const int chunks = ((phase == PH_GRAM ? p.n : p.m) + 63) / 64;
    for (int bn = rows; bn >= rows / 2; bn >>= 1) {
        PhaseShape s;
        s.bn = bn;
        s.stage_bytes = p.split * (128 + (pair ? bn / 2 : bn)) * 128;
        s.stages = kRing / s.stage_bytes < kMaxStages ? kRing / s.stage_bytes : kMaxStages;
        s.tiles_n = ((symmetric ? p.m : p.n) + bn - 1) / bn;
        s.tiles = symmetric ? lower_tiles(p.m, rows, bn) : (p.m + rows - 1) / rows * s.tiles_n;
        const double products = (p.split == 2 ? 12 : 4) * (double)(bn / 2 > 48 ? bn / 2 : 48);
        const double chunk = s.stage_bytes / 58.0 > products ? s.stage_bytes / 58.0 : products;
        const double results = 1000.0 + 32.0 * bn;
        const long long all = (long long)s.tiles * p.batch;
        for (s.splits = 1; s.splits <= kMaxSplits; ++s.splits) {
            s.per = (chunks + s.splits - 1) / s.splits;
            if (s.splits > 1 && (all * s.splits > units || s.per < 2 || (s.splits - 1) * s.per >= chunks)) continue;
            const double t = (double)cdiv64(all * s.splits, units) * s.per * chunk + results + (s.splits > 1 ? 2500.0 + 4.0 * s.splits * bn : 0.0);
            if (least == 0 || t < least) { least = t; best = s; }
        }
    }
    *clocks = least;
    return best;
}

int resident_pairs();
Shapes choose_shapes(const NsPlan& p) {
    Shapes best = {};
    double least = 0;
    // Pairs of fp16 always run on single CTAs: CTA pairs measured slower on every size (1536 x 1536 334 us single, 363 paired;
    // 2560 x 2560 1176 and 1326; 4096 x 4096 4350 and 4830; 8192 x 8192 36.8 and 38.2 ms, all back to back under the power cap).
    const int pairs = p.split == 1 ? resident_pairs() : 0;
    for (int pair = 0; pair <= (pairs > 0 ? 1 : 0); ++pair) {
        Shapes c = {};
        c.pair = pair != 0;
        c.units = pair ? pairs : sm_count();
        double sum = 0;
        for (int ph = 0; ph < 3; ++ph) {
            double t;
            PhaseShape& s = c.shape[ph];
            s = phase_shape(p, ph, c.pair, c.units, &t);
            sum += t;
            const size_t bytes = s.splits > 1 ? (size_t)s.tiles * p.batch * (pair ? 2 : 1) * s.splits * 8 * (s.bn / 2) * 128 : 0;
            if (bytes > c.partial_bytes) c.partial_bytes = bytes;
        }
        // CTA pairs take 1.25 times this estimate (measured on both sides of where it decides, us back to back, single CTAs and pairs: by the
        // estimate, single / pairs = 1.06: 1024 x 4096 217 and 250; 1.22: 1536 x 1536 191 and 194; 1.31: 1500 x 2100 239 and 227;
        // 1.36: 2048 x 2048 279 and 267; 1.47: 2560 x 2560 517 and 454; 1.76: 4096 x 4096 1750 and 1375).
        if (c.pair) sum *= 1.25;
        if (least == 0 || sum < least) { least = sum; best = c; }
    }
    return best;
}

bool use_small(const NsPlan& p) { return p.m <= 128 && p.n <= kSmallCols * kSmallCluster; }

NsPlan ns_plan(int batch, int rows, int cols, int precision) {
    NsPlan p = {};
    p.batch = batch; p.rows = rows; p.cols = cols;
    p.transposed = rows > cols;
    p.m = rows < cols ? rows : cols;
    p.n = rows < cols ? cols : rows;
    p.split = precision == GF_NS_F32 ? 2 : 1;
    p.x_pieces = (p.n + 7) / 8;
    p.a_pieces = (p.m + 7) / 8;
    const long long per = ((long long)rows * cols + 8 * kNormThreads - 1) / (8 * kNormThreads);      // two groups of four per thread
    p.norm_blocks = (int)(per < kNormBlocks ? per : kNormBlocks);
    p.x_lo = 8LL * batch * p.m * p.x_pieces;
    p.a_lo = 8LL * batch * p.m * p.a_pieces;
    size_t off = 256 + kArrived * 4;
    p.off_part = off; off += up((size_t)batch * p.norm_blocks * 8, 256);
    for (int k = 0; k < 2; ++k) { p.off_x[k] = off; off += up((size_t)p.x_lo * 4, 256); }
    p.off_a = off; off += up((size_t)p.a_lo * 2 * p.split, 256);
    p.off_b = off; off += up((size_t)p.a_lo * 2 * p.split, 256);
    p.off_trace = off; off += up((size_t)batch * ((p.m + 31) / 32) * 4, 256);
    if (use_small(p)) { p.total = 256; return p; }
    p.shapes = choose_shapes(p);
    p.off_partial = off; off += up(p.shapes.partial_bytes, 256);
    p.total = off;
    return p;
}

const float kDefaultCoeffs[3] = {3.4445f, -4.7750f, 2.0315f};

template <int SPLIT, bool PAIR> gf_status launch_iterate(const IterateArgs& a, int units, cudaStream_t s) {
    constexpr size_t smem = (size_t)kRing + 1024;
    static size_t configured[kMaxDevices] = {};
    if (gf_status st = ensure_dyn_smem(ns_iterate_kernel<SPLIT, PAIR>, smem, configured); st != GF_OK) return st;
    long long most = 1;
    for (const PhaseShape& ps : a.shape) {
        const long long all = (long long)ps.tiles * a.batch * ps.splits;
        if (all > most) most = all;
    }
    const int used = most < units ? (int)most : units;
    ProfScope prof(K_NS_PRODUCT, s);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(PAIR ? 2 * used : used); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem; cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeCooperative;          // the blocks wait for one another between phases
    attr[0].val.cooperative = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = PAIR ? 2 : 1; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = PAIR ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, ns_iterate_kernel<SPLIT, PAIR>, a);
    count_launch();
    return e == cudaSuccess ? GF_OK : GF_ERR_CUDA;
}

// Pairs of CTAs that are resident at once (0: none).
int resident_pairs() {
    static int cached[kMaxDevices] = {};                  // pairs + 1
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 0;
    if (cached[dev] == 0) {
        constexpr size_t smem = (size_t)kRing + 1024;
        static size_t configured[kMaxDevices] = {};
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(2); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr; cfg.numAttrs = 1;
        int n = 0;
        if (ensure_dyn_smem(ns_iterate_kernel<1, true>, smem, configured) != GF_OK ||
            cudaOccupancyMaxActiveClusters(&n, ns_iterate_kernel<1, true>, &cfg) != cudaSuccess)
            n = 0;
        cached[dev] = n + 1;
    }
    return cached[dev] - 1;
}

// The iteration from X in the workspace (written by ns_cast_kernel); the result is X[steps & 1].
gf_status ns_iterate(const NsPlan& p, char* base, int steps, const float* coeffs, cudaStream_t s) {
    IterateArgs a = {};
    a.batch = p.batch; a.m = p.m; a.n = p.n; a.steps = steps;
    for (int k = 0; k < steps; ++k)
        for (int e = 0; e < 3; ++e) a.coeff[k][e] = coeffs ? coeffs[3 * k + e] : kDefaultCoeffs[e];
    a.x[0] = reinterpret_cast<__half*>(base + p.off_x[0]);
    a.x[1] = reinterpret_cast<__half*>(base + p.off_x[1]);
    a.a = reinterpret_cast<__half*>(base + p.off_a);
    a.b = reinterpret_cast<__half*>(base + p.off_b);
    a.trace = reinterpret_cast<float*>(base + p.off_trace);
    a.blocks = (p.m + 31) / 32;
    a.x_pieces = p.x_pieces; a.a_pieces = p.a_pieces; a.x_lo = p.x_lo; a.a_lo = p.a_lo;
    a.err_word = reinterpret_cast<uint32_t*>(base);
    a.barrier = reinterpret_cast<uint32_t*>(base + 128);
    a.partial = reinterpret_cast<float*>(base + p.off_partial);
    a.arrived = reinterpret_cast<uint32_t*>(base + 256);
    const bool pair = p.shapes.pair;
    const int units = p.shapes.units;
    for (int k = 0; k < 3; ++k) a.shape[k] = p.shapes.shape[k];
    const uint64_t m = (uint64_t)p.m, b = (uint64_t)p.batch, xp = (uint64_t)p.x_pieces, ap = (uint64_t)p.a_pieces;
    auto share = [&](int phase) { return (uint32_t)(pair ? a.shape[phase].bn / 2 : a.shape[phase].bn); };
    // two 8-byte units are the 8 columns of a row
    auto map = [&](CUtensorMap* out, const __half* src, uint64_t pieces, uint64_t planes, uint32_t rows, uint32_t columns) {
        return make_tmap_u64(out, src, 2 * m, pieces, planes, 2 * m, 2 * m * pieces, 2 * rows, columns / 8);
    };
    bool good = map(&a.tm_a[2], a.a, ap, b * p.split, 128, 64) && map(&a.tm_a[3], a.b, ap, b * p.split, 128, 64) &&
                map(&a.tm_g[2], a.a, ap, b * p.split, share(PH_POLY), 64);
    for (int k = 0; k < 2 && good; ++k)
        good = map(&a.tm_a[k], a.x[k], xp, 2 * b, 128, 64) && map(&a.tm_g[k], a.x[k], xp, 2 * b, share(PH_GRAM), 64) &&
               map(&a.tm_n[k], a.x[k], xp, 2 * b, 64, share(PH_APPLY));
    if (!good) return GF_ERR_CUDA;
    if (pair) return launch_iterate<1, true>(a, units, s);        // (pairs of fp16: single CTAs, see choose_shapes)
    return p.split == 2 ? launch_iterate<2, false>(a, units, s) : launch_iterate<1, false>(a, units, s);
}

template <bool MUON> gf_status launch_finish(const NsPlan& p, const FinishArgs& f, int count, cudaStream_t s) {
    ProfScope prof(K_NS_FINISH, s);
    const dim3 grid((p.cols + kCast - 1) / kCast, (p.rows + kFinRows - 1) / kFinRows, count);
    return launch_pdl(ns_finish_kernel<MUON>, grid, dim3(256), 0, s, f);
}
FinishArgs finish_args(const NsPlan& p, char* base, int steps, int first) {
    FinishArgs f = {};
    f.x = reinterpret_cast<const __half*>(base + p.off_x[steps & 1]) + 8LL * first * p.x_pieces * p.m;
    f.m = p.m; f.n = p.n; f.pieces = p.x_pieces; f.lo = p.x_lo; f.transposed = p.transposed; f.rows = p.rows; f.cols = p.cols; f.taps = 1;
    return f;
}

template <bool MUON> gf_status launch_prepare(const NsPlan& p, const Source& src, int first, int count, char* base, float eps, cudaStream_t s) {
    ProfScope prof(K_NS_PREPARE, s);
    double* part = reinterpret_cast<double*>(base + p.off_part) + (size_t)first * p.norm_blocks;
    gf_status st = launch_pdl(ns_norm_kernel<MUON>, dim3(p.norm_blocks, count), dim3(kNormThreads), 0, s, src, part,
                              first == 0 ? reinterpret_cast<uint32_t*>(base) : nullptr);
    if (st != GF_OK) return st;
    __half* X = reinterpret_cast<__half*>(base + p.off_x[0]) + 8LL * first * p.m * p.x_pieces;
    const dim3 grid((p.cols + kCast - 1) / kCast, (p.rows + kCast - 1) / kCast, count), block(256);
    return launch_pdl(ns_cast_kernel<MUON>, grid, block, 0, s, src, (const double*)part, p.norm_blocks, eps, X, p.m, p.n, p.x_pieces, p.x_lo, p.transposed);
}

template <int SPLIT, bool MUON> gf_status launch_small_t(const SmallArgs& a, int count, cudaStream_t s) {
    const size_t smem = (size_t)small_region(SPLIT) + (size_t)a.slice * 256 * SPLIT + 1024;
    static size_t configured[kMaxDevices] = {};
    if (gf_status st = ensure_dyn_smem(ns_small_kernel<SPLIT, MUON>, smem, configured); st != GF_OK) return st;
    ProfScope prof(K_NS_PRODUCT, s);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(count * a.cluster)); cfg.blockDim = dim3(kSmallThreads); cfg.dynamicSmemBytes = smem; cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = a.cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, ns_small_kernel<SPLIT, MUON>, a);
    count_launch();
    return e == cudaSuccess ? GF_OK : GF_ERR_CUDA;
}
// `a` holds the source, the outputs and the update's factors; count matrices.
gf_status launch_small(const NsPlan& p, SmallArgs& a, bool muon, int count, int steps, const float* coeffs, float eps, char* base, cudaStream_t s) {
    a.m = p.m; a.n = p.n; a.transposed = p.transposed; a.steps = steps; a.eps = eps;
    a.cluster = (p.n + kSmallCols - 1) / kSmallCols;
    a.slice = ((p.n + a.cluster - 1) / a.cluster + 15) / 16 * 16;
    for (int k = 0; k < steps; ++k)
        for (int e = 0; e < 3; ++e) a.coeff[k][e] = coeffs ? coeffs[3 * k + e] : kDefaultCoeffs[e];
    a.err_word = global_err_word();
    if (!a.err_word) return GF_ERR_CUDA;
    a.status = reinterpret_cast<uint32_t*>(base);
    if (muon) return p.split == 2 ? launch_small_t<2, true>(a, count, s) : launch_small_t<1, true>(a, count, s);
    return p.split == 2 ? launch_small_t<2, false>(a, count, s) : launch_small_t<1, false>(a, count, s);
}

bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
bool bad_dtype(int d) { return d != GF_F32 && d != GF_BF16; }

gf_status check_shape(int batch, int rows, int cols, int precision, int steps, float eps) {
    if (batch < 0 || rows < 1 || cols < 1 || steps < 1 || steps > GF_NS_MAX_STEPS || !(eps >= 0.f)) return GF_ERR_BAD_DESC;
    if (precision != GF_NS_F16 && precision != GF_NS_F32) return GF_ERR_BAD_DESC;
    if (rows > 16384 || cols > 16384 || batch > 32767) return GF_ERR_UNSUPPORTED;      // at most 2^14 tiles of a matrix: units of work fit 32 bits
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
    *bytes = ns_plan(d->batch, d->rows, d->cols, d->precision).total;
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
    const NsPlan p = ns_plan(d->batch, d->rows, d->cols, d->precision);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char* base = static_cast<char*>(workspace);
    Source src = {};
    src.g[0] = G; src.batched = 1; src.bf16 = d->in_dtype == GF_BF16; src.taps = 1; src.rows = d->rows; src.cols = d->cols;
    src.vec = d->cols % 4 == 0;                 // G is on a 16-byte boundary, and so are its rows and matrices, or 8 in bf16
    if (use_small(p)) {
        SmallArgs a = {};
        a.src = src;
        a.out = O; a.out_bf16 = d->out_dtype == GF_BF16; a.taps = 1;
        return launch_small(p, a, false, d->batch, d->steps, h_coeffs, d->eps, base, s);
    }
    if (gf_status st = launch_prepare<false>(p, src, 0, d->batch, base, d->eps, s); st != GF_OK) return st;
    if (gf_status st = ns_iterate(p, base, d->steps, h_coeffs, s); st != GF_OK) return st;
    FinishArgs f = finish_args(p, base, d->steps, 0);
    f.out = O; f.bf16 = d->out_dtype == GF_BF16;
    return launch_finish<false>(p, f, d->batch, s);
}

gf_status gf_muon_workspace_bytes(const gf_muon_desc* d, size_t* bytes) {
    if (!d || !bytes) return GF_ERR_NULL;
    if (gf_status st = check_shape(d->count, d->rows, d->cols, d->precision, d->steps, d->eps); st != GF_OK) return st;
    if (bad_dtype(d->grad_dtype) || bad_dtype(d->weight_dtype) || d->taps < 1 || (d->nesterov != 0 && d->nesterov != 1)) return GF_ERR_BAD_DESC;
    if (d->taps > 4096) return GF_ERR_UNSUPPORTED;
    *bytes = ns_plan(d->count, d->rows, d->cols, d->precision).total;
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
    const NsPlan p = ns_plan(d->count, d->rows, d->cols, d->precision);
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
        src.vec = d->taps == 1 && d->cols % 4 == 0;
        for (int k = 0; k < n; ++k)
            if (off16(src.g[k]) || off16(src.mom[k]) || off16(src.mom_out[k])) src.vec = 0;
        // the flattened matrix is u (x) (1 .. 1): its norm is sqrt(taps) times that of u
        if (use_small(p)) {
            SmallArgs a = {};
            a.src = src;
            for (int k = 0; k < n; ++k) { a.w[k] = h_weight[first + k]; a.w_out[k] = h_weight_out[first + k]; }
            a.out_bf16 = d->weight_dtype == GF_BF16;
            a.taps = d->taps; a.div_taps = FastDiv((uint32_t)d->taps);
            a.keep = 1.f - d->lr * d->weight_decay;
            a.f = d->lr * d->scale / root;
            if (gf_status st = launch_small(p, a, true, n, d->steps, h_coeffs, d->eps / root, base, s); st != GF_OK) return st;
            continue;
        }
        if (gf_status st = launch_prepare<true>(p, src, first, n, base, d->eps / root, s); st != GF_OK) return st;
    }
    if (use_small(p)) return GF_OK;
    if (gf_status st = ns_iterate(p, base, d->steps, h_coeffs, s); st != GF_OK) return st;
    for (int first = 0; first < d->count; first += kMaxLayers) {
        const int n = d->count - first < kMaxLayers ? d->count - first : kMaxLayers;
        FinishArgs f = finish_args(p, base, d->steps, first);
        for (int k = 0; k < n; ++k) { f.w[k] = h_weight[first + k]; f.w_out[k] = h_weight_out[first + k]; }
        f.taps = d->taps; f.div_taps = FastDiv((uint32_t)d->taps); f.bf16 = d->weight_dtype == GF_BF16;
        f.keep = 1.f - d->lr * d->weight_decay;
        f.f = d->lr * d->scale / root;
        if (gf_status st = launch_finish<true>(p, f, n, s); st != GF_OK) return st;
    }
    return GF_OK;
}

}  // extern "C"

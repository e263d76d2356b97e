// Root-mean-square norm of a residual sum, backward (gf_block.h).
//
// Bound by memory: g_y, g_h and h are read and the gradients written once.  A thread keeps gamma and the sums of g_gamma for
// its columns in registers over all rows of its team; each block leaves a line of sums, which a second kernel adds in a fixed order.
// Measured: 65536 x 256 fp32 44 us (0.92 of the copy bandwidth), 16384 x 2048 bf16 with an fp32 residual 92 (0.89), 8192 x 4096 bf16 51
// (0.79: 28 rows per block, of which the first and the lines of sums take 6 us), 100352 x 576 bf16 with dropout 114 (0.77; without the
// next row brought to L2 136), 4099 x 1001 fp32 19 to 20 (0.63: 7 rows per block), in tiles of columns 2000 x 16384 bf16 112 (0.36), fp32 150 (0.53).
#include "gf_rms.cuh"

namespace gf {
namespace {

// Rows longer than the registers of a block come with their dots: the grid's second dimension then deals out column tiles.
// With one or two octets a thread the team's next row is on its way while one is computed; with three there are no registers
// for that, and more rows per block instead.
template <typename TX, typename TR, int NO, bool WARP, bool ALIGNED, bool DOTS>
__global__ void __launch_bounds__(WARP ? kRmsThreads : kRmsMostThreads, WARP && NO > 2 ? 2 : 1) rms_bwd_kernel(const __grid_constant__ RmsArgs a) {
    __shared__ __align__(16) float red[2][32];
    extern __shared__ float lines[];                     // WARP: [teams][cols] sums
    pdl_launch_dependents();
    constexpr bool kAhead = NO <= 2;
    const int tpr = !WARP ? (int)blockDim.x : NO > 1 ? 32 : 1 << a.log_tpr;
    const int g = WARP ? (int)threadIdx.x & (tpr - 1) : (int)threadIdx.x;
    const int log_tpr = NO > 1 ? 5 : a.log_tpr;
    const int teams_pb = WARP ? kRmsThreads >> log_tpr : 1, team = WARP ? (int)threadIdx.x >> log_tpr : 0;
    const int first_of_warp = WARP ? ((int)threadIdx.x & ~31) >> log_tpr : 0;
    const long long step = (long long)gridDim.x * teams_pb;
    long long row = (long long)blockIdx.x * teams_pb + team;
    const int phase = ALIGNED ? 0 : (int)((row * a.cols) & 7);
    const int tile0 = DOTS ? (int)blockIdx.y * (a.col_tile >> 3) : 0;        // first octet of the tile
    if (!WARP && threadIdx.x < 64) (&red[0][0])[threadIdx.x] = 0.f;
    pdl_wait();
    if (!WARP) __syncthreads();

    // octet k of this thread: columns c0(k) .. c0(k) + 7; only its last may lie past the row
    auto c0 = [&](int k) { return 8 * (tile0 + k * tpr + g) - phase; };
    const bool last = c0(NO - 1) < a.cols;
    auto there = [&](int k) { return k + 1 < NO || last; };
    Eight gam[NO], sum[NO];
#pragma unroll
    for (int k = 0; k < NO; ++k) {
        rms_gamma8(a, c0(k), gam[k]);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[k][i] = 0;
    }
    uint64_t key, offset;
    load_seed(a.drop, key, offset);

    const TX* const gy = static_cast<const TX*>(a.gy);
    const TR* const h = static_cast<const TR*>(a.h);
    const TR* const gh = a.gres || a.y ? static_cast<const TR*>(a.gh) : nullptr;
    Octet<TX> ngy[NO];
    Octet<TR> nh[NO], ngh[NO];
    float nrstd = 0.f, ndot = 0.f;
#pragma unroll
    for (int k = 0; k < NO; ++k) {
        ngy[k].clear();
        nh[k].clear();
        ngh[k].clear();
    }
    // e: the place of this thread's first octet in a row, in elements; e + 8 k tpr: of octet k
    const long long e_step = step * a.cols;
    long long e = ((row * a.cols >> 3) + tile0 + g) * 8;
    auto fetch = [&](long long r, long long at) {
        if (r >= a.rows) {                               // a row of zeros: it leaves the sums as they are
            nrstd = 0.f;
#pragma unroll
            for (int k = 0; k < NO; ++k) {
                ngy[k].clear();
                nh[k].clear();
            }
            return;
        }
        nrstd = a.rstd_in[r];
        if (DOTS) ndot = a.dots[r];
        const bool inside = at + 8 * (NO - 1) * tpr + 8 <= a.total;          // whole vectors (the tensor's last octet may not be one)
#pragma unroll
        for (int k = 0; k < NO; ++k) {
            if (there(k)) {
                const long long p = at + 8 * k * tpr;
                if (ALIGNED || inside) {
                    ngy[k].load(gy + p);
                    nh[k].load(h + p);
                    if (gh) ngh[k].load(gh + p);
                } else {
                    load_octet(ngy[k], gy, p >> 3, a.total);
                    load_octet(nh[k], h, p >> 3, a.total);
                    if (gh) load_octet(ngh[k], gh, p >> 3, a.total);
                }
            }
        }
    };
    if (kAhead) fetch(row, e);
    int turn = 0;
    for (long long warp_row = (long long)blockIdx.x * teams_pb + first_of_warp; warp_row < a.rows; warp_row += step, row += step, e += e_step, turn ^= 1) {
        if constexpr (!kAhead) {
            fetch(row, e);
            if (row + step < a.rows) {                   // the next row, from memory to L2 meanwhile
#pragma unroll
                for (int k = 0; k < NO; ++k) {
                    if (there(k)) {
                        const long long p = e + e_step + 8 * k * tpr;
                        asm volatile("prefetch.global.L2 [%0];" ::"l"(gy + p));
                        asm volatile("prefetch.global.L2 [%0];" ::"l"(h + p));
                        if (gh) asm volatile("prefetch.global.L2 [%0];" ::"l"(gh + p));
                    }
                }
            }
        }
        const bool live = row < a.rows;
        const float rstd = nrstd, dot = ndot;
        const uint64_t rstd2 = pair_of(rstd, rstd);
        // g_y and h rstd of octet k
        auto take = [&](int k, Eight& q, Eight& xh) {
            ngy[k].get(q);
            nh[k].get(xh);
            if (!ALIGNED && (c0(k) < 0 || c0(k) + 8 > a.cols)) {
                float f[8], x[8];
                from_eight(q, f);
                from_eight(xh, x);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c0(k) + i < 0 || c0(k) + i >= a.cols) f[i] = x[i] = 0.f;
                to_eight(f, q);
                to_eight(x, xh);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) xh[i] = mul_pair(xh[i], rstd2);
        };
        Eight q[kAhead ? NO : 1], xh[kAhead ? NO : 1];
        Octet<TR> add[kAhead ? NO : 1];                  // g_h, which makes room for the next row's
        uint64_t dots = 0;
        if (kAhead) {
#pragma unroll
            for (int k = 0; k < NO; ++k) {
                take(k, q[kAhead ? k : 0], xh[kAhead ? k : 0]);
                add[kAhead ? k : 0] = ngh[k];
            }
            fetch(row + step, e + e_step);
        }
#pragma unroll
        for (int k = 0; k < NO; ++k) {
            const int s = kAhead ? k : 0;
            if (!kAhead) take(k, q[0], xh[0]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[k][i] = fma_pair(q[s][i], xh[s][i], sum[k][i]);
                q[s][i] = mul_pair(q[s][i], gam[k][i]);
                dots = fma_pair(q[s][i], xh[s][i], dots);
            }
        }
        if (!a.gres && !a.y) continue;
        const float mean = DOTS ? dot : rms_sum<WARP>(sum_of(dots), log_tpr, red[turn]) * a.inv_c;
        const uint64_t minus = pair_of(-mean, -mean);
#pragma unroll
        for (int k = 0; k < NO; ++k) {
            const int c = c0(k), s = kAhead ? k : 0;
            if (!live || !there(k)) continue;
            Eight v;
            if (kAhead) add[s].get(v);
            else {
                ngh[k].get(v);
                take(k, q[0], xh[0]);
#pragma unroll
                for (int i = 0; i < 4; ++i) q[0][i] = mul_pair(q[0][i], gam[k][i]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = fma_pair(rstd2, fma_pair(xh[s][i], minus, q[s][i]), v[i]);
            const bool whole = ALIGNED || (c >= 0 && c + 8 <= a.cols);
            if (a.gres) {
                TR* const p = static_cast<TR*>(a.gres) + e + 8 * k * tpr;
                if (whole) {
                    Octet<TR> o;
                    o.set(v);
                    o.store(p);
                } else {
                    float f[8];
                    from_eight(v, f);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (c + i >= 0 && c + i < a.cols) p[i] = from_f32<TR>(f[i]);
                }
            }
            if (a.y) {
                if (a.drop.threshold) drop_octet(v, (uint64_t)(e >> 3) + (uint64_t)(k * tpr), key, offset, a.drop);
                TX* const p = static_cast<TX*>(a.y) + e + 8 * k * tpr;
                if (whole) {
                    Octet<TX> o;
                    o.set(v);
                    o.store(p);
                } else {
                    float f[8];
                    from_eight(v, f);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (c + i >= 0 && c + i < a.cols) p[i] = from_f32<TX>(f[i]);
                }
            }
        }
    }
    if (!a.part) return;
    float* const part = a.part + (size_t)blockIdx.x * a.cols;
    if constexpr (WARP) {
        float* const line = lines + (size_t)team * a.cols;
#pragma unroll
        for (int k = 0; k < NO; ++k) {
            float f[8];
            from_eight(sum[k], f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = c0(k) + i;
                if (c >= 0 && c < a.cols) line[c] = f[i];
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.cols; c += kRmsThreads) {
            float t = lines[c];
            for (int w = 1; w < teams_pb; ++w) t += lines[(size_t)w * a.cols + c];
            part[c] = t;
        }
    } else {
#pragma unroll
        for (int k = 0; k < NO; ++k) {
            float f[8];
            from_eight(sum[k], f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = c0(k) + i;
                if (c >= 0 && c < a.cols) part[c] = f[i];
            }
        }
    }
}

// dots[row] = sum over the row of g_y gamma xh / cols, for rows longer than a block's registers
template <typename TX, typename TR> __global__ void __launch_bounds__(1024) rms_dots_kernel(const __grid_constant__ RmsArgs a, float* dots) {
    __shared__ __align__(16) float red[2][32];
    pdl_launch_dependents();
    pdl_wait();
    int turn = 0;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const long long e0 = row * a.cols, e1 = e0 + a.cols;
        float s = 0.f;
        const float rstd = a.rstd_in[row];
        for (long long f = (e0 >> 3) + threadIdx.x; f * 8 < e1; f += 1024) {
            Octet<TX> gy;
            Octet<TR> h;
            load_octet(gy, static_cast<const TX*>(a.gy), f, a.total);
            load_octet(h, static_cast<const TR*>(a.h), f, a.total);
            float v[8], w[8];
            gy.get(v);
            h.get(w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const long long c = f * 8 + i - e0;
                if (c >= 0 && c < a.cols) s = fmaf(v[i] * rms_gamma(a, (int)c), w[i] * rstd, s);
            }
        }
        s = rms_sum<false>(s, 0, red[turn]);
        if (threadIdx.x == 0) dots[row] = s * a.inv_c;
    }
}

// g_gamma from the blocks' lines: thread (x, y) adds lines y, y + 32, .. of a column, then the 32 sums are added in order.
__global__ void __launch_bounds__(1024) rms_sums_kernel(const float* part, int lines, int cols, float* g_gamma) {
    __shared__ float sums[32][33];
    pdl_launch_dependents();
    pdl_wait();
    const int c = blockIdx.x * 32 + threadIdx.x;
    float s = 0.f;
    if (c < cols) {
#pragma unroll 8
        for (int b = threadIdx.y; b < lines; b += 32) s += part[(size_t)b * cols + c];
    }
    sums[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    s = warp_sum(sums[threadIdx.x][threadIdx.y]);        // a warp per column
    const int out = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x == 0 && out < cols) g_gamma[out] = s;
}

struct BwdPlan {
    RmsShape shape;
    bool tiles;                 // rows longer than a block's registers
    long long blocks;           // along the rows
    size_t off_part, bytes;
};
constexpr int kMostBlocks = 8;  // per SM
constexpr int kTileCols = 8 * kRmsMostThreads;

BwdPlan plan(const gf_rms_desc* d) {
    BwdPlan p = {};
    const int n = rms_octets(d->cols);
    // octets that a thread's registers hold of a row: of 32-bit rows, and of rows that start anywhere, fewer
    const int each = d->cols % 8 != 0 || d->residual_dtype == GF_F32 ? 2 : 3;
    p.tiles = n > 2 * kRmsMostThreads;
    p.shape = rms_shape(n, each, 1);
    if (p.tiles) p.shape = RmsShape{false, 0, kRmsMostThreads, 1};
    const int teams = p.shape.warp ? kRmsThreads >> p.shape.log_tpr : 1;
    const long long tiles = p.tiles ? cdiv64((long long)n * 8, kTileCols) : 1;
    long long most = (long long)sm_count() * 2048 / p.shape.threads;
    if (most > (long long)sm_count() * kMostBlocks) most = (long long)sm_count() * kMostBlocks;
    most = cdiv64(most, tiles);
    p.blocks = cdiv64(d->rows, teams);
    if (p.blocks > most) p.blocks = most;
    p.blocks = cdiv64(p.blocks, 8) * 8;
    p.off_part = p.tiles ? (size_t)cdiv64(d->rows, 64) * 256 : 0;
    p.bytes = p.off_part + (size_t)p.blocks * d->cols * 4;
    return p;
}

gf_status launch_sums(const float* part, int lines, int cols, float* g_gamma, cudaStream_t s) {
    return launch_pdl(rms_sums_kernel, dim3((unsigned)((cols + 31) / 32)), dim3(32, 32), 0, s, part, lines, cols, g_gamma);
}

template <typename TX, typename TR, int NO, bool WARP, bool ALIGNED, bool DOTS>
gf_status launch(const RmsArgs& a, const BwdPlan& p, float* g_gamma, cudaStream_t s) {
    auto kernel = rms_bwd_kernel<TX, TR, NO, WARP, ALIGNED, DOTS>;
    const int teams = WARP ? kRmsThreads >> p.shape.log_tpr : 1;
    const size_t smem = WARP && a.part ? (size_t)teams * a.cols * 4 : 0;
    static int cached[WARP ? 6 : kRmsMostThreads / 32 + 1][kMaxDevices] = {};
    const int resident = rms_resident(kernel, p.shape.threads, smem, cached[WARP ? p.shape.log_tpr : p.shape.threads / 32]);
    const unsigned tiles = DOTS ? (unsigned)cdiv64((long long)rms_octets(a.cols) * 8, kTileCols) : 1u;
    long long grid = cdiv64((long long)sm_count() * resident / 8 * 8, tiles) / 8 * 8;
    if (grid < 8) grid = 8;
    if (grid > p.blocks) grid = p.blocks;
    const gf_status st = launch_pdl(kernel, dim3((unsigned)grid, tiles), dim3(p.shape.threads), smem, s, a);
    return st == GF_OK && g_gamma ? launch_sums(a.part, (int)grid, a.cols, g_gamma, s) : st;
}

template <typename TX, typename TR, bool ALIGNED> gf_status dispatch(RmsArgs a, const BwdPlan& p, float* g_gamma, cudaStream_t s) {
    gf_status st;
    a.log_tpr = p.shape.log_tpr;
    if (p.tiles) {
        if (a.gres || a.y) {
            const long long most = sm_count() * 2;
            float* const dots = const_cast<float*>(a.dots);
            st = launch_pdl(rms_dots_kernel<TX, TR>, dim3((unsigned)(a.rows < most ? a.rows : most)), dim3(1024), 0, s, a, dots);
            if (st != GF_OK) return st;
        }
        a.col_tile = kTileCols;
        return launch<TX, TR, 1, false, ALIGNED, true>(a, p, g_gamma, s);
    }
    if (p.shape.warp) {
        if (p.shape.per_thread == 1) return launch<TX, TR, 1, true, ALIGNED, false>(a, p, g_gamma, s);
        if (p.shape.per_thread == 2) return launch<TX, TR, 2, true, ALIGNED, false>(a, p, g_gamma, s);
        if constexpr (ALIGNED) {
            if constexpr (sizeof(TR) == 2) return launch<TX, TR, 3, true, ALIGNED, false>(a, p, g_gamma, s);
        }
        return GF_ERR_UNSUPPORTED;                        // (no plan asks for it)
    }
    if (p.shape.per_thread == 1) return launch<TX, TR, 1, false, ALIGNED, false>(a, p, g_gamma, s);
    return launch<TX, TR, 2, false, ALIGNED, false>(a, p, g_gamma, s);
}

}  // namespace
}  // namespace gf

using namespace gf;

extern "C" {

gf_status gf_rms_norm_backward_workspace_bytes(const gf_rms_desc* desc, size_t* bytes) {
    if (!bytes) return GF_ERR_NULL;
    const gf_status st = rms_validate(desc);
    if (st != GF_OK) return st;
    *bytes = plan(desc).bytes;
    return GF_OK;
}

gf_status gf_rms_norm_backward(const gf_rms_desc* desc, const void* g_y, const void* g_h, const void* h, const float* rstd, const void* gamma,
                               const uint64_t* seed, void* g_residual, void* g_x, float* g_gamma, void* workspace, size_t workspace_bytes,
                               void* stream) {
    const gf_status st = rms_validate(desc);
    if (st != GF_OK) return st;
    if (!g_residual && !g_x && !g_gamma) return GF_OK;
    RmsArgs a = {};
    a.drop = make_drop(desc->p, seed);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (rms_off16(g_gamma)) return GF_ERR_ALIGN;
    ProfScope prof(K_RMS_BWD, s);
    if (desc->rows == 0) return g_gamma ? launch_sums(nullptr, 0, desc->cols, g_gamma, s) : GF_OK;
    const BwdPlan p = plan(desc);
    if (!g_y || !h || !rstd || (!workspace && p.bytes > 0 && (g_gamma || p.tiles)) || (g_x && a.drop.threshold && !seed)) return GF_ERR_NULL;
    if (rms_off16(g_y) || rms_off16(g_h) || rms_off16(h) || rms_off16(rstd) || rms_off16(gamma) || rms_off16(g_residual) || rms_off16(g_x) ||
        rms_off16(workspace) || (reinterpret_cast<uintptr_t>(seed) & 7u) != 0)
        return GF_ERR_ALIGN;
    if (desc->dtype != desc->residual_dtype && g_residual == g_y) return GF_ERR_UNSUPPORTED;      // an element's place is not its gradient's
    if ((g_gamma || p.tiles) && workspace_bytes < p.bytes) return GF_ERR_WORKSPACE;
    a.gy = g_y; a.gh = g_h; a.h = const_cast<void*>(h); a.rstd_in = rstd; a.gamma = gamma; a.gamma_bf16 = desc->param_dtype == GF_BF16;
    a.gres = g_residual; a.y = g_x;
    if (!g_x) a.drop.threshold = 0;
    a.dots = static_cast<const float*>(workspace);
    a.part = g_gamma ? reinterpret_cast<float*>(static_cast<char*>(workspace) + p.off_part) : nullptr;
    a.rows = desc->rows; a.cols = desc->cols; a.total = desc->rows * desc->cols;
    a.inv_c = 1.f / (float)desc->cols;
    const bool aligned = desc->cols % 8 == 0;
    auto go = [&](auto tx, auto tr) {
        using TX = decltype(tx);
        using TR = decltype(tr);
        return aligned ? dispatch<TX, TR, true>(a, p, g_gamma, s) : dispatch<TX, TR, false>(a, p, g_gamma, s);
    };
    if (desc->dtype == GF_F32) return go(float(), float());
    if (desc->residual_dtype == GF_F32) return go(__nv_bfloat16(), float());
    return go(__nv_bfloat16(), __nv_bfloat16());
}

}  // extern "C"

// Root-mean-square norm of a residual sum, backward (gf_block.h).
//
// Bound by memory: g_y, g_h and h are read and the gradients written once.  A thread keeps gamma and the sums of g_gamma for
// its columns in registers over all rows of its team; each block leaves a line of sums, which a second kernel adds in a fixed order.
#include "gf_rms.cuh"

namespace gf {
namespace {

// Rows longer than the registers of a block come with their dots: the grid's second dimension then deals out column tiles.
template <typename TX, typename TR, int NO, bool WARP, bool ALIGNED, bool DOTS>
__global__ void __launch_bounds__(WARP ? kRmsThreads : kRmsMostThreads) rms_bwd_kernel(const __grid_constant__ RmsArgs a) {
    __shared__ __align__(16) float red[2][32];
    extern __shared__ float lines[];                     // WARP: [teams][cols] sums
    pdl_launch_dependents();
    const int tpr = WARP ? 1 << a.log_tpr : (int)blockDim.x;
    const int g = WARP ? (int)threadIdx.x & (tpr - 1) : (int)threadIdx.x;
    const int teams_pb = WARP ? kRmsThreads >> a.log_tpr : 1, team = WARP ? (int)threadIdx.x >> a.log_tpr : 0;
    const int first_of_warp = WARP ? ((int)threadIdx.x & ~31) >> a.log_tpr : 0;
    const long long step = (long long)gridDim.x * teams_pb;
    long long row = (long long)blockIdx.x * teams_pb + team;
    const int phase = ALIGNED ? 0 : (int)((row * a.cols) & 7);
    const int tile0 = DOTS ? (int)blockIdx.y * (a.col_tile >> 3) : 0;        // first octet of the tile
    if (!WARP && threadIdx.x < 64) (&red[0][0])[threadIdx.x] = 0.f;
    pdl_wait();
    if (!WARP) __syncthreads();

    // octet k of this thread: columns c0(k) .. c0(k) + 7; a tile's last octet belongs to the next tile unless it is the row's last
    auto octet = [&](int k) { return tile0 + k * tpr + g; };
    auto c0 = [&](int k) { return 8 * octet(k) - phase; };
    auto mine = [&](int k) { return c0(k) < a.cols && (!DOTS || k * tpr + g < (a.col_tile >> 3)); };
    float gam[NO][8], sum[NO][8];
#pragma unroll
    for (int k = 0; k < NO; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = c0(k) + i;
            gam[k][i] = c >= 0 && c < a.cols ? rms_gamma(a, c) : 0.f;
            sum[k][i] = 0.f;
        }
    uint64_t key = 0, offset = 0;
    if (a.drop.threshold) { key = a.drop.seed[0]; offset = a.drop.seed[1]; }

    Octet<TX> ngy[NO];
    Octet<TR> nh[NO], ngh[NO];
    float nrstd = 0.f, ndot = 0.f;
    const TR* const gh = a.gres ? static_cast<const TR*>(a.gh) : a.y ? static_cast<const TR*>(a.gh) : nullptr;
    auto fetch = [&](long long r) {
        const long long base = r * a.cols >> 3;
        if (r < a.rows) {
            nrstd = a.rstd_in[r];
            if (DOTS) ndot = a.dots[r];
        }
#pragma unroll
        for (int k = 0; k < NO; ++k) {
            ngy[k].clear();
            nh[k].clear();
            ngh[k].clear();
            if (r < a.rows && mine(k)) {
                const long long f = base + octet(k);
                if (ALIGNED) {
                    ngy[k].load(static_cast<const TX*>(a.gy) + f * 8);
                    nh[k].load(static_cast<const TR*>(a.h) + f * 8);
                    if (gh) ngh[k].load(gh + f * 8);
                } else {
                    load_octet(ngy[k], static_cast<const TX*>(a.gy), f, a.total);
                    load_octet(nh[k], static_cast<const TR*>(a.h), f, a.total);
                    if (gh) load_octet(ngh[k], gh, f, a.total);
                }
            }
        }
    };
    fetch(row);
    int turn = 0;
    for (long long warp_row = (long long)blockIdx.x * teams_pb + first_of_warp; warp_row < a.rows; warp_row += step, row += step, turn ^= 1) {
        const bool live = row < a.rows;
        const long long base = row * a.cols >> 3;
        const float rstd = live ? nrstd : 0.f;
        float q[NO][8], xh[NO][8];
        Octet<TR> add[NO];
        float s = 0.f;
        const float dot = ndot;
#pragma unroll
        for (int k = 0; k < NO; ++k) {
            ngy[k].get(q[k]);
            nh[k].get(xh[k]);
            add[k] = ngh[k];
        }
        fetch(row + step);
#pragma unroll
        for (int k = 0; k < NO; ++k) {
            const int c = c0(k);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (!ALIGNED && (c + i < 0 || c + i >= a.cols)) q[k][i] = xh[k][i] = 0.f;
                xh[k][i] *= rstd;
                sum[k][i] = fmaf(q[k][i], xh[k][i], sum[k][i]);
                q[k][i] *= gam[k][i];
                s = fmaf(q[k][i], xh[k][i], s);
            }
        }
        if (!a.gres && !a.y) continue;
        if (DOTS) s = dot;
        else s = rms_sum<WARP>(s, a.log_tpr, red[turn]) * a.inv_c;
#pragma unroll
        for (int k = 0; k < NO; ++k) {
            const int c = c0(k);
            if (!live || !mine(k)) continue;
            const long long e = (base + octet(k)) * 8;
            float v[8];
            add[k].get(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = fmaf(rstd, q[k][i] - xh[k][i] * s, v[i]);
            const bool whole = ALIGNED || (c >= 0 && c + 8 <= a.cols);
            if (a.gres) {
                TR* const p = static_cast<TR*>(a.gres) + e;
                if (whole) {
                    Octet<TR> o;
                    o.set(v);
                    o.store(p);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (c + i >= 0 && c + i < a.cols) p[i] = from_f32<TR>(v[i]);
                }
            }
            if (a.y) {
                if (a.drop.threshold) drop_octet(v, (uint64_t)(base + octet(k)), key, offset, a.drop.threshold, a.drop.scale);
                TX* const p = static_cast<TX*>(a.y) + e;
                if (whole) {
                    Octet<TX> o;
                    o.set(v);
                    o.store(p);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (c + i >= 0 && c + i < a.cols) p[i] = from_f32<TX>(v[i]);
                }
            }
        }
    }
    if (!a.part) return;
    float* const part = a.part + (size_t)blockIdx.x * a.cols;
    if constexpr (WARP) {
        float* const line = lines + (size_t)team * a.cols;
#pragma unroll
        for (int k = 0; k < NO; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = c0(k) + i;
                if (c >= 0 && c < a.cols) line[c] = sum[k][i];
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
            if (!mine(k)) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = c0(k) + i;
                if (c >= 0 && c < a.cols) part[c] = sum[k][i];
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
    p.tiles = n > 2 * kRmsMostThreads;
    p.shape = rms_shape(n, 2, 1);
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
        return launch<TX, TR, 2, true, ALIGNED, false>(a, p, g_gamma, s);
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

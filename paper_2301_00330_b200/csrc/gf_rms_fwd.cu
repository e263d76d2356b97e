// Root-mean-square norm of a residual sum, forward (gf_block.h), with results in 16, 32 or 8 bits.
//
// Bound by memory: x and residual are read and h and y (or codes) written once; a row stays in the registers of its team between
// the sum and the results, and the team's next row is on its way meanwhile.  Rows of three octets a thread are bound by instructions
// as well: 106 a thread and octet, with dropout's random bits 228, with rounding to 8 bits 184 (of 96 octets that the lanes have for
// 576 columns' 72).
// Measured: 16384 x 2048 bf16 with an fp32 residual to 8 bits 59 to 64 us (0.88 to 0.95 of the copy bandwidth), 100352 x 576 bf16 75 to 77 (0.91
// to 0.94), with dropout 92 to 98, to 8 bits 76 to 82, 65536 x 256 fp32 43 (0.95); rows in parts, 2000 x 16384 bf16 88 (0.45), fp32 120 (0.67).
#include "gf_rms.cuh"

namespace gf {

gf_status rms_validate(const gf_rms_desc* d) {
    if (!d) return GF_ERR_NULL;
    auto known = [](int t) { return t == GF_F32 || t == GF_BF16; };
    if (d->rows < 0 || d->cols < 1 || !known(d->dtype) || !known(d->residual_dtype) || !known(d->param_dtype) || !(d->eps >= 0.f) || !valid_p(d->p))
        return GF_ERR_BAD_DESC;
    if (d->dtype == GF_F32 && d->residual_dtype == GF_BF16) return GF_ERR_UNSUPPORTED;
    if (d->cols > 1 << 24 || d->rows > ((int64_t)1 << 60) / d->cols) return GF_ERR_UNSUPPORTED;
    return GF_OK;
}

namespace {

// A value's place in a row of floats in shared memory: threads that write (or read) elements 8 apart meet 32 different banks.
__device__ __forceinline__ int skewed(int c) { return c + (c >> 5); }

// ALIGNED: rows are whole octets.  OUT8: codes and scales in y's place; 16 threads that follow one another have the 128
// columns of a scale.  Rows that are not whole octets change places for that through shared memory.
// (Registers: with a bound of one block per SM the compiler orders 32-bit rows of one octet a thread so that 65536 x 256 takes 43.5 us
// instead of 51; the other forms are as fast or faster without: 100352 x 576 bf16 77, with it 100.)
template <typename TX, typename TR, int NO, bool WARP, bool ALIGNED, bool OUT8>
__global__ void __launch_bounds__(WARP ? kRmsThreads : kRmsMostThreads, WARP && NO == 1 && sizeof(TX) == 4 ? 1 : 0) rms_fwd_kernel(const __grid_constant__ RmsArgs a) {
    __shared__ __align__(16) float red[2][32];
    extern __shared__ float rows_smem[];
    pdl_launch_dependents();
    const int tpr = !WARP ? (int)blockDim.x : NO > 1 ? 32 : 1 << a.log_tpr;
    const int g = WARP ? (int)threadIdx.x & (tpr - 1) : (int)threadIdx.x;
    const int log_tpr = NO > 1 ? 5 : a.log_tpr;
    const int teams_pb = WARP ? kRmsThreads >> log_tpr : 1, team = WARP ? (int)threadIdx.x >> log_tpr : 0;
    const int first_of_warp = WARP ? ((int)threadIdx.x & ~31) >> log_tpr : 0;
    const long long step = (long long)gridDim.x * teams_pb;
    long long row = (long long)blockIdx.x * teams_pb + team;
    const int phase = ALIGNED ? 0 : (int)((row * a.cols) & 7);
    float* const line = rows_smem + (size_t)team * skewed(a.cols + 7);
    if (!WARP && threadIdx.x < 64) (&red[0][0])[threadIdx.x] = 0.f;
    pdl_wait();
    if (!WARP) __syncthreads();

    const TX* const x = static_cast<const TX*>(a.x);
    const TR* const res = static_cast<const TR*>(a.residual);
    // octet k of this thread: columns c0(k) .. c0(k) + 7, of an ALIGNED row all of them or none
    auto c0 = [&](int k) { return 8 * (k * tpr + g) - phase; };
    const bool last = c0(NO - 1) < a.cols;
    auto there = [&](int k) { return k + 1 < NO || last; };
    Eight gam[NO];
#pragma unroll
    for (int k = 0; k < NO; ++k) rms_gamma8(a, c0(k), gam[k]);
    uint64_t key, offset;
    load_seed(a.drop, key, offset);

    Octet<TX> nx[NO];
    Octet<TR> nr[NO];
#pragma unroll
    for (int k = 0; k < NO; ++k) {
        nx[k].clear();
        nr[k].clear();
    }
    // e: the place of this thread's first octet in a row, in elements; e + 8 k tpr: of octet k
    const long long e_step = step * a.cols;
    long long e = ((row * a.cols >> 3) + g) * 8;
    auto fetch = [&](long long at) {
        const bool inside = at + 8 * (NO - 1) * tpr + 8 <= a.total;          // whole vectors (the tensor's last octet may not be one)
#pragma unroll
        for (int k = 0; k < NO; ++k) {
            if (there(k)) {
                if (ALIGNED || inside) {
                    nx[k].load(x + at + 8 * k * tpr);
                    if (res) nr[k].load(res + at + 8 * k * tpr);
                } else {
                    load_octet(nx[k], x, (at >> 3) + k * tpr, a.total);
                    if (res) load_octet(nr[k], res, (at >> 3) + k * tpr, a.total);
                }
            }
        }
    };
    if (row < a.rows) fetch(e);
    int turn = 0;
    // (the lanes of a warp go round together, as long as any of its rows is left)
    for (long long warp_row = (long long)blockIdx.x * teams_pb + first_of_warp; warp_row < a.rows; warp_row += step, row += step, e += e_step, turn ^= 1) {
        const bool live = row < a.rows;
        Eight v[NO], w[NO];
#pragma unroll
        for (int k = 0; k < NO; ++k) {
            nx[k].get(v[k]);
            nr[k].get(w[k]);                             // (zeros without a residual)
        }
        if (row + step < a.rows) fetch(e + e_step);
        uint64_t squares = 0;
#pragma unroll
        for (int k = 0; k < NO; ++k) {
            const int c = c0(k);
            if (a.drop.threshold) drop_octet(v[k], w[k], (uint64_t)(e >> 3) + (uint64_t)(k * tpr), key, offset, a.drop);
            else {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[k][i] = add_pair(v[k][i], w[k][i]);
            }
            if (a.h) {
                Octet<TR> o;
                o.set(v[k]);
                o.get(v[k]);                             // the norm is that of h as it is kept
                if (live && there(k)) {
                    TR* const h = static_cast<TR*>(a.h) + e + 8 * k * tpr;
                    if (ALIGNED || (c >= 0 && c + 8 <= a.cols)) o.store(h);
                    else {
                        float f[8];
                        from_eight(v[k], f);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (c + i >= 0 && c + i < a.cols) h[i] = from_f32<TR>(f[i]);
                    }
                }
            }
            if ((!ALIGNED && (c < 0 || c + 8 > a.cols)) || (OUT8 && k + 1 == NO && !last)) {     // what is not the row's counts as zero
                float f[8];
                from_eight(v[k], f);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i < 0 || c + i >= a.cols) f[i] = 0.f;
                to_eight(f, v[k]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) squares = fma_pair(v[k][i], v[k][i], squares);
        }
        const float s = rms_sum<WARP>(sum_of(squares), log_tpr, red[turn]);
        const float rstd = __frcp_rn(__fsqrt_rn(fmaf(s, a.inv_c, a.eps)));
        if (a.rstd && live && g == 0) a.rstd[row] = rstd;
        const uint64_t rstd2 = pair_of(rstd, rstd);
#pragma unroll
        for (int k = 0; k < NO; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[k][i] = mul_pair(mul_pair(v[k][i], rstd2), gam[k][i]);
        if constexpr (!OUT8) {
#pragma unroll
            for (int k = 0; k < NO; ++k) {
                const int c = c0(k);
                if (!live || !there(k)) continue;
                TX* const y = static_cast<TX*>(a.y) + e + 8 * k * tpr;
                if (ALIGNED || (c >= 0 && c + 8 <= a.cols)) {
                    Octet<TX> o;
                    o.set(v[k]);
                    o.store(y);
                } else {
                    float f[8];
                    from_eight(v[k], f);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (c + i >= 0 && c + i < a.cols) y[i] = from_f32<TX>(f[i]);
                }
            }
        } else {
            float f[NO][8];
#pragma unroll
            for (int k = 0; k < NO; ++k) from_eight(v[k], f[k]);
            if constexpr (!ALIGNED) {                    // from the tensor's octets to the row's own
#pragma unroll
                for (int k = 0; k < NO; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int c = c0(k) + i;
                        if (c >= 0 && c < a.cols) line[skewed(c)] = f[k][i];
                    }
                if (WARP) __syncwarp();
                else __syncthreads();
#pragma unroll
                for (int k = 0; k < NO; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int c = 8 * (k * tpr + g) + i;
                        f[k][i] = c < a.cols ? line[skewed(c)] : 0.f;
                    }
                if (WARP) __syncwarp();
            }
            float scale[NO], by[NO], least = INFINITY;
#pragma unroll
            for (int k = 0; k < NO; ++k) {
                uint32_t m = magnitude(f[k]);
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
                scale[k] = by[k] = scale_of(m);
                least = fminf(least, scale[k]);
            }
            if (is_small_scale(least)) {                 // (once a row: 100352 x 576 bf16 78.5 us, asked by octets 79.8, never 77.2)
#pragma unroll
                for (int k = 0; k < NO; ++k)
                    if (is_small_scale(scale[k])) {      // larger numbers with the same quotients
                        by[k] *= kFp8Up;
#pragma unroll
                        for (int i = 0; i < 8; ++i) f[k][i] *= kFp8Up;
                    }
            }
#pragma unroll
            for (int k = 0; k < NO; ++k) {
                const int c = 8 * (k * tpr + g);
                if (live && c < a.pitch) {
                    *reinterpret_cast<uint2*>(a.codes + row * a.pitch + c) = codes8(f[k], by[k], __frcp_rn(by[k]), a.cols - c);
                    if ((g & 15) == 0 && c < a.cols) a.scales[(long long)(c >> 7) * a.scale_pitch + row] = scale[k];
                }
            }
        }
    }
}

// Rows longer than the registers of a block: h is written on the way to the sum and read again (from L2) for the results.
constexpr int kLongThreads = 1024;
template <typename TX, typename TR, bool OUT8> __global__ void __launch_bounds__(kLongThreads) rms_fwd_long_kernel(const __grid_constant__ RmsArgs a) {
    __shared__ __align__(16) float red[2][32];
    pdl_launch_dependents();
    pdl_wait();
    const TX* const x = static_cast<const TX*>(a.x);
    const TR* const res = static_cast<const TR*>(a.residual);
    TR* const h = static_cast<TR*>(a.h);
    uint64_t key, offset;
    load_seed(a.drop, key, offset);
    int turn = 0;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const long long e0 = row * a.cols, e1 = e0 + a.cols;
        float s = 0.f;
        for (long long f = (e0 >> 3) + threadIdx.x; f * 8 < e1; f += kLongThreads) {
            Octet<TX> ox;
            load_octet(ox, x, f, a.total);
            Octet<TR> r;
            r.clear();
            if (res) load_octet(r, res, f, a.total);
            float v[8], w[8];
            ox.get(v);
            r.get(w);
            if (a.drop.threshold) drop_octet(v, w, (uint64_t)f, key, offset, a.drop);
            else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += w[i];
            }
            if (h) {
                Octet<TR> o;
                o.set(v);
                o.get(v);
                if (f * 8 >= e0 && f * 8 + 8 <= e1) o.store(h + f * 8);
                else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (f * 8 + i >= e0 && f * 8 + i < e1) h[f * 8 + i] = from_f32<TR>(v[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (f * 8 + i >= e0 && f * 8 + i < e1) s = fmaf(v[i], v[i], s);
        }
        s = rms_sum<false>(s, 0, red[turn]);              // (also: h of the whole row is visible to the block)
        const float rstd = __frcp_rn(__fsqrt_rn(fmaf(s, a.inv_c, a.eps)));
        if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
        const TR* const from = h ? h : reinterpret_cast<const TR*>(a.x);      // without h: x, of the same type
        if constexpr (OUT8) {
            for (int c = 8 * (int)threadIdx.x; c < (a.pitch + 127) / 128 * 128; c += 8 * kLongThreads) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = c + i < a.cols ? to_f32(from[e0 + c + i]) * rstd * rms_gamma(a, c + i) : 0.f;
                uint32_t m = magnitude(v);
                const uint32_t half = 0xffffu << ((threadIdx.x & 16));
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(half, m, o));
                const float scale = scale_of(m);
                if (c < a.pitch) {
                    uint8_t* const to = a.codes + row * a.pitch + c;
                    *reinterpret_cast<uint2*>(to) = codes8(v, scale, __frcp_rn(scale), a.cols - c);
                    divide_codes(to, scale, min(8, a.cols - c), [&](int i) { return to_f32(from[e0 + c + i]) * rstd * rms_gamma(a, c + i); });
                    if ((threadIdx.x & 15) == 0 && c < a.cols) a.scales[(long long)(c >> 7) * a.scale_pitch + row] = scale;
                }
            }
        } else {
            TX* const y = static_cast<TX*>(a.y);
            for (long long f = (e0 >> 3) + threadIdx.x; f * 8 < e1; f += kLongThreads) {
                const int c = (int)(f * 8 - e0);
                if (c >= 0 && c + 8 <= a.cols) {
                    Octet<TR> o;
                    o.load(from + f * 8);
                    float v[8];
                    o.get(v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = v[i] * rstd * rms_gamma(a, c + i);
                    Octet<TX> t;
                    t.set(v);
                    t.store(y + f * 8);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (c + i >= 0 && c + i < a.cols) y[f * 8 + i] = from_f32<TX>(to_f32(from[f * 8 + i]) * rstd * rms_gamma(a, c + i));
                }
            }
        }
    }
}

template <typename TX, typename TR, int NO, bool WARP, bool ALIGNED, bool OUT8> gf_status launch(const RmsArgs& a, const RmsShape& sh, cudaStream_t s) {
    auto kernel = rms_fwd_kernel<TX, TR, NO, WARP, ALIGNED, OUT8>;
    const int teams = WARP ? kRmsThreads >> sh.log_tpr : 1;
    const int width = a.cols + 7;
    const size_t smem = OUT8 && !ALIGNED ? (size_t)teams * (width + (width >> 5)) * 4 : 0;
    static int cached[WARP ? 6 : kRmsMostThreads / 32 + 1][kMaxDevices] = {};
    const int resident = rms_resident(kernel, sh.threads, smem, cached[WARP ? sh.log_tpr : sh.threads / 32]);
    const long long want = cdiv64(a.rows, teams), most = (long long)sm_count() * resident / 8 * 8;
    long long grid = want < most ? want : most;
    if (!ALIGNED) grid = cdiv64(grid, 8) * 8;             // steps of a multiple of eight rows
    return launch_pdl(kernel, dim3((unsigned)grid), dim3(sh.threads), smem, s, a);
}

template <typename TX, typename TR, bool ALIGNED, bool OUT8> gf_status dispatch(const RmsArgs& a, cudaStream_t s) {
    int n = rms_octets(a.cols);
    if (OUT8 && a.pitch / 8 > n) n = a.pitch / 8;
    if (n > 2 * kRmsMostThreads) {
        const long long most = sm_count() * 2;
        return launch_pdl(rms_fwd_long_kernel<TX, TR, OUT8>, dim3((unsigned)(a.rows < most ? a.rows : most)), dim3(kLongThreads), 0, s, a);
    }
    const RmsShape sh = rms_shape(n, 3, OUT8 ? 4 : 1);
    RmsArgs b = a;
    b.log_tpr = sh.log_tpr;
    if (sh.warp) {
        if (sh.per_thread == 1) return launch<TX, TR, 1, true, ALIGNED, OUT8>(b, sh, s);
        if (sh.per_thread == 2) return launch<TX, TR, 2, true, ALIGNED, OUT8>(b, sh, s);
        return launch<TX, TR, 3, true, ALIGNED, OUT8>(b, sh, s);
    }
    if (sh.per_thread == 1) return launch<TX, TR, 1, false, ALIGNED, OUT8>(b, sh, s);
    return launch<TX, TR, 2, false, ALIGNED, OUT8>(b, sh, s);
}

template <bool OUT8> gf_status run(const gf_rms_desc* d, const void* x, const void* residual, const uint64_t* seed, const void* gamma, void* h, void* y,
                                   void* codes, float* scales, float* rstd, void* stream) {
    const gf_status st = rms_validate(d);
    if (st != GF_OK) return st;
    RmsArgs a = {};
    a.drop = make_drop(d->p, seed);
    const bool h_is_x = !residual && a.drop.threshold == 0;
    if (h_is_x && (h || d->dtype != d->residual_dtype)) return GF_ERR_BAD_DESC;
    if (d->rows == 0) return GF_OK;
    if (!x || (OUT8 ? !codes || !scales : !y) || (a.drop.threshold && !seed) || (!h && !h_is_x)) return GF_ERR_NULL;
    if (rms_off16(x) || rms_off16(residual) || rms_off16(gamma) || rms_off16(h) || rms_off16(y) || rms_off16(codes) || rms_off16(scales) ||
        rms_off16(rstd) || (reinterpret_cast<uintptr_t>(seed) & 7u) != 0)
        return GF_ERR_ALIGN;
    if (d->dtype != d->residual_dtype && h == x) return GF_ERR_UNSUPPORTED;       // an element's place is not its sum's
    a.x = x; a.residual = residual; a.gamma = gamma; a.gamma_bf16 = d->param_dtype == GF_BF16;
    a.h = h;
    a.y = y; a.codes = static_cast<uint8_t*>(codes); a.scales = scales; a.rstd = rstd;
    a.rows = d->rows; a.cols = d->cols; a.total = d->rows * d->cols;
    a.pitch = GF_FP8_PITCH(d->cols); a.scale_pitch = GF_FP8_SCALE_PITCH(d->rows);
    a.eps = d->eps; a.inv_c = 1.f / (float)d->cols;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    ProfScope prof(K_RMS_FWD, s);
    const bool aligned = d->cols % 8 == 0;
    auto go = [&](auto tx, auto tr) {
        using TX = decltype(tx);
        using TR = decltype(tr);
        return aligned ? dispatch<TX, TR, true, OUT8>(a, s) : dispatch<TX, TR, false, OUT8>(a, s);
    };
    if (d->dtype == GF_F32) return go(float(), float());
    if (d->residual_dtype == GF_F32) return go(__nv_bfloat16(), float());
    return go(__nv_bfloat16(), __nv_bfloat16());
}

}  // namespace
}  // namespace gf

using namespace gf;

extern "C" {

gf_status gf_rms_norm_forward(const gf_rms_desc* desc, const void* x, const void* residual, const uint64_t* seed, const void* gamma, void* h,
                              void* y, float* rstd, void* stream) {
    return run<false>(desc, x, residual, seed, gamma, h, y, nullptr, nullptr, rstd, stream);
}

gf_status gf_rms_norm_forward_fp8(const gf_rms_desc* desc, const void* x, const void* residual, const uint64_t* seed, const void* gamma, void* h,
                                  void* codes, float* scales, float* rstd, void* stream) {
    if (desc && desc->rows > 0x7fffffffLL) return GF_ERR_UNSUPPORTED;
    return run<true>(desc, x, residual, seed, gamma, h, nullptr, codes, scales, rstd, stream);
}

}  // extern "C"

// Dropout from a counter, with the residual's addition (gf_block.h).
//
// Bound by memory: x (and the residual) read once, y written once.  An octet is the unit: its 128 random bits are one Philox
// block of some 80 integer instructions, with the choices 120, which the memory's time covers (16 bits per element; 32 would take twice
// the blocks).  Two octets a thread and a block for every 512: 100352 x 576 bf16 with a residual 50 us in a captured run of
// calls, 53 from a cold cache, 57 as a program calls it (its bytes ask for 53; a quarter of those it writes are still in L2 when it ends).
// One octet a thread in blocks that stay: 68.
#include "gf_block.h"
#include "gf_octet.cuh"

namespace gf {

Drop make_drop(float p, const uint64_t* seed) {
    Drop d;
    d.threshold = (uint32_t)__builtin_rint((double)p * 65536.0);
    d.scale = d.threshold < 65536u ? (float)(65536.0 / (65536.0 - d.threshold)) : 0.f;
    d.seed = seed;
    return d;
}

namespace {

constexpr int kThreads = 256, kEach = 2;
constexpr int64_t kMostCount = 0x7fffffffLL * (kThreads * kEach * 8);      // blocks of a grid

// kEach octets a thread, the loads of all on their way before the first is computed
template <typename TX, typename TY, bool RESIDUAL>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const TX* x, const TY* residual, TY* y, long long count, const __grid_constant__ Drop d) {
    pdl_launch_dependents();
    const long long octets = (count + 7) / 8, first = (long long)blockIdx.x * (kThreads * kEach) + threadIdx.x;
    pdl_wait();
    uint64_t key, offset;
    load_seed(d, key, offset);
    Octet<TX> a[kEach];
    Octet<TY> r[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const long long f = first + k * kThreads;
        if (f < octets) {
            load_octet(a[k], x, f, count);
            if constexpr (RESIDUAL) load_octet(r[k], residual, f, count);
        }
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const long long f = first + k * kThreads;
        if (f >= octets) break;
        float v[8], w[8];
        a[k].get(v);
        if constexpr (RESIDUAL) r[k].get(w);
        if (d.threshold) {
            if constexpr (RESIDUAL) drop_octet(v, w, (uint64_t)f, key, offset, d);
            else drop_octet(v, (uint64_t)f, key, offset, d);
        } else if constexpr (RESIDUAL) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += w[i];
        }
        if (f * 8 + 8 <= count) {
            r[k].set(v);
            r[k].store(y + f * 8);
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (f * 8 + i < count) y[f * 8 + i] = from_f32<TY>(v[i]);
        }
    }
}

template <typename TX, typename TY> gf_status launch(const void* x, const void* residual, void* y, long long count, const Drop& d, cudaStream_t s) {
    const long long blocks = cdiv64((count + 7) / 8, kThreads * kEach);
    const dim3 grid((unsigned)blocks);
    ProfScope prof(K_DROPOUT, s);
    if (residual)
        return launch_pdl(dropout_kernel<TX, TY, true>, grid, dim3(kThreads), 0, s, static_cast<const TX*>(x), static_cast<const TY*>(residual),
                          static_cast<TY*>(y), count, d);
    return launch_pdl(dropout_kernel<TX, TY, false>, grid, dim3(kThreads), 0, s, static_cast<const TX*>(x), static_cast<const TY*>(residual),
                      static_cast<TY*>(y), count, d);
}

bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
bool is_dtype(int d) { return d == GF_F32 || d == GF_BF16; }

gf_status run(const gf_dropout_desc* desc, const void* x, int x_dtype, const void* residual, const uint64_t* seed, void* y, int y_dtype,
              cudaStream_t s) {
    if (desc->count == 0) return GF_OK;
    const Drop d = make_drop(desc->p, seed);
    if (!x || !y || (d.threshold && !seed)) return GF_ERR_NULL;
    if (off16(x) || off16(y) || off16(residual) || (reinterpret_cast<uintptr_t>(seed) & 7u) != 0) return GF_ERR_ALIGN;
    if (x_dtype != y_dtype && y == x) return GF_ERR_UNSUPPORTED;          // an element's place is not its result's
    if (x_dtype == GF_F32) {
        if (y_dtype == GF_F32) return launch<float, float>(x, residual, y, desc->count, d, s);
        return launch<float, __nv_bfloat16>(x, residual, y, desc->count, d, s);
    }
    if (y_dtype == GF_F32) return launch<__nv_bfloat16, float>(x, residual, y, desc->count, d, s);
    return launch<__nv_bfloat16, __nv_bfloat16>(x, residual, y, desc->count, d, s);
}

gf_status validate(const gf_dropout_desc* d) {
    if (!d) return GF_ERR_NULL;
    if (d->count < 0 || !valid_p(d->p) || !is_dtype(d->dtype) || !is_dtype(d->out_dtype)) return GF_ERR_BAD_DESC;
    return d->count > kMostCount ? GF_ERR_UNSUPPORTED : GF_OK;
}

}  // namespace
}  // namespace gf

using namespace gf;

extern "C" {

gf_status gf_dropout_forward(const gf_dropout_desc* desc, const void* x, const void* residual, const uint64_t* seed, void* y, void* stream) {
    const gf_status st = validate(desc);
    if (st != GF_OK) return st;
    return run(desc, x, desc->dtype, residual, seed, y, desc->out_dtype, static_cast<cudaStream_t>(stream));
}

gf_status gf_dropout_backward(const gf_dropout_desc* desc, const void* g_y, const uint64_t* seed, void* g_x, void* stream) {
    const gf_status st = validate(desc);
    if (st != GF_OK) return st;
    return run(desc, g_y, desc->out_dtype, nullptr, seed, g_x, desc->dtype, static_cast<cudaStream_t>(stream));
}

}  // extern "C"

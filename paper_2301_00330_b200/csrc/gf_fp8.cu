// Matrices in 8 bits with scales for groups of 128 (gf_block.h): quantisers, and the product of 8-bit rows with an 8-bit weight.
#include "gf_block.h"
#include "gf_octet.cuh"
#include "gf_pipe.cuh"
#include "gf_tc.cuh"
#include "gf_tma.cuh"

namespace gf {
namespace {

bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
bool is_dtype(int d) { return d == GF_F32 || d == GF_BF16; }

// ---- quantisers ------------------------------------------------------------------------------------------------------
// Rows: sixteen threads have the 128 columns of a scale, a block 16 rows by 4 scales, so that the loads of four octets are on their
// way at once and the scales of 16 rows make whole sectors.  Bound by memory.
constexpr int kQuantThreads = 256, kQuantRows = 16, kQuantGroups = 4;

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kQuantThreads) quantize_rows_kernel(const T* x, uint8_t* codes, float* scales, long long rows, int cols, int pitch,
                                                                      long long scale_pitch, int chunks, long long blocks) {
    pdl_launch_dependents();
    pdl_wait();
    const int part = threadIdx.x & 15;
    const long long total = rows * cols;
    for (long long b = blockIdx.x; b < blocks; b += gridDim.x) {
        const long long row = b / chunks * kQuantRows + (threadIdx.x >> 4);
        const int c0 = (int)(b % chunks) * (128 * kQuantGroups) + part * 8;
        Octet<T> o[kQuantGroups];
#pragma unroll
        for (int k = 0; k < kQuantGroups; ++k) {
            const int c = c0 + 128 * k;
            if (row < rows && c < cols) {
                if (ALIGNED) o[k].load(x + row * cols + c);
                else load_anywhere(o[k], x, row * cols + c, total);
            } else o[k].clear();
        }
#pragma unroll
        for (int k = 0; k < kQuantGroups; ++k) {
            const int c = c0 + 128 * k;
            float v[8];
            o[k].get(v);
            if (!ALIGNED) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i >= cols) v[i] = 0.f;
            }
            uint32_t m = magnitude(v);
#pragma unroll
            for (int s = 8; s > 0; s >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, s));
            const float scale = scale_of(m);
            if (row < rows && c < pitch) {
                *reinterpret_cast<uint2*>(codes + row * pitch + c) = codes8(v, scale, __frcp_rn(scale), cols - c);
                if (part == 0 && c < cols) scales[(long long)(c >> 7) * scale_pitch + row] = scale;
            }
        }
    }
}

// Blocks: one 128 x 128 block at a time, held in registers between its maximum and its codes.  Run once per frozen weight.
template <typename T> __global__ void __launch_bounds__(kQuantThreads) quantize_blocks_kernel(const T* x, uint8_t* codes, float* scales, long long rows, int cols, int pitch,
                                                                                         int col_blocks, long long blocks) {
    __shared__ uint32_t red[kQuantThreads / 32];
    pdl_launch_dependents();
    pdl_wait();
    const long long total = rows * cols;
    for (long long b = blockIdx.x; b < blocks; b += gridDim.x) {
        const long long row0 = b / col_blocks * 128 + (threadIdx.x >> 4);
        const int c = (int)(b % col_blocks) * 128 + (threadIdx.x & 15) * 8;
        Octet<T> o[8];
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const long long row = row0 + 16 * k;
            if (row < rows && c < cols) load_anywhere(o[k], x, row * cols + c, total);
            else o[k].clear();
            float v[8];
            o[k].get(v);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i >= cols) v[i] = 0.f;
            m = max(m, magnitude(v));
        }
        m = __reduce_max_sync(0xffffffffu, m);
        __syncthreads();                             // the sums of the block before are read
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kQuantThreads / 32; ++k) m = max(m, red[k]);
        const float scale = scale_of(m), inv = __frcp_rn(scale);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const long long row = row0 + 16 * k;
            float v[8];
            o[k].get(v);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i >= cols) v[i] = 0.f;
            if (row < rows && c < pitch)
                *reinterpret_cast<uint2*>(codes + row * pitch + c) = codes8(v, scale, inv, cols - c);
        }
        if (threadIdx.x == 0) scales[b] = scale;
    }
}

// ---- product ---------------------------------------------------------------------------------------------------------
// out[m, j] = sum over chunks q of 128 terms of  sa[m, q] sw[j / 128, q] (sum over the chunk of A[m, l] W'[l, j]),
// W' = W^T (the layer) or W (the gradient of its input).  The tensor cores add a chunk into one of two accumulators in tensor
// memory; warps that wait for it scale it and add it to fp32 registers while the next chunk is multiplied into the other.
struct ProductArgs {
    CUtensorMap tm_w, tm_a;
    const float *sa, *sw;
    const void* bias;
    void* out;
    uint32_t* err_word;
    long long sa_pitch, sw_j, sw_q;      // strides of the scales: rows of sa; blocks of columns and chunks of sw
    int M, J, chunks, per, split;        // per: chunks of a CTA of a cluster of `split`
    int tiles_m, bias_bf16;
    int mn_major;                        // W is read with the contracted index as its rows
};

__host__ __device__ constexpr uint32_t fp8_idesc(int M, int N, uint32_t a_mn, uint32_t b_mn) {     // e4m3 x e4m3 -> fp32
    return (1u << 4) | (a_mn << 15) | (b_mn << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
__device__ __forceinline__ void umma_fp8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ void cluster_meet() { asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ float peer_load(uint32_t addr, int rank) {
    float v;
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.f32 %0, [a];\n\t}" : "=f"(v) : "r"(addr), "r"(rank) : "memory");
    return v;
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ float bias_at(const ProductArgs& p, int j) {
    if (!p.bias) return 0.f;
    return p.bias_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.bias)[j]) : static_cast<const float*>(p.bias)[j];
}

// A tile is 128 columns of the result (rows of the accumulator) by T of its rows, so that the weight is the operand of
// 128 and few rows of A cost no more than they are.  The chunks of a tile are split over a cluster of CTAs where there
// are few tiles, and the parts are added through distributed shared memory, in the order of the CTAs.
//   warp 0: copies; warp 1: products; warps 2 to 5: scaling, a quarter of the accumulator's rows each.
// Blocks of a cluster wait for one another and hold tensor memory: the ring is sized so that the blocks an SM can hold never
// want more than its 512 columns, or two clusters could each hold what the other waits for.
constexpr int kFewThreads = 192;
__host__ __device__ constexpr int few_stages(int T) { return T <= 32 ? 4 : 3; }
constexpr size_t few_smem(int T) { return (size_t)few_stages(T) * (16384 + T * 128) + 1024; }
static_assert(227 * 1024 / few_smem(16) * 32 <= 512 && 227 * 1024 / few_smem(32) * 64 <= 512 && 227 * 1024 / few_smem(64) * 128 <= 512 &&
                  227 * 1024 / few_smem(128) * 256 <= 512 && 227 * 1024 / few_smem(64) <= 3,
              "tensor memory of the blocks of an SM");

template <int T, typename TO> __global__ void __launch_bounds__(kFewThreads) fp8_few_kernel(const __grid_constant__ ProductArgs p) {
    extern __shared__ unsigned char dyn_raw[];
    unsigned char* const dyn = align1024(dyn_raw);
    constexpr int kStages = few_stages(T), kStageBytes = 16384 + T * 128, kCols = 2 * T;
    __shared__ uint64_t full[kStages], empty[kStages], done[2], drained[2];
    __shared__ uint32_t tmem_base;
    __shared__ __align__(16) float scale[2][T];
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int rank = (int)blockIdx.x % p.split, tile = (int)blockIdx.x / p.split;
    const int m0 = tile % p.tiles_m * T, j0 = tile / p.tiles_m * 128;
    const int q0 = rank * p.per, n = min(p.per, p.chunks - q0);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(&done[s], 1); mbar_init(&drained[s], 4); }
        mbar_fence_init();
    }
    pdl_wait();
    if (warp == 1) { tmem_alloc(&tmem_base, kCols); tmem_relinquish(); }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    pdl_launch_dependents();      // (tensor memory is taken: a kernel that is scheduled from here on cannot hold it while it waits for this one)
    const uint32_t tmem = tmem_base;
    bool ok = true;

    if (warp == 0) {
        for (int q = 0; q < n; ++q) {
            const int s = q % kStages;
            ok = mbar_wait_warp(&empty[s], ((uint32_t)(q / kStages) & 1u) ^ 1u);
            if (!ok) break;
            if (elect_one()) {
                unsigned char* st = dyn + (size_t)s * kStageBytes;
                mbar_expect_tx(&full[s], kStageBytes);
                const int l = (q0 + q) * 128;
                if (p.mn_major) tma_load_2d(st, &p.tm_w, j0, l, &full[s]);
                else tma_load_2d(st, &p.tm_w, l, j0, &full[s]);
                tma_load_2d(st + 16384, &p.tm_a, l, m0, &full[s]);
            }
            __syncwarp();
        }
    } else if (warp == 1) {
        const uint32_t idesc = fp8_idesc(128, T, p.mn_major ? 1u : 0u, 0u);
        const uint32_t a_step = p.mn_major ? 4096u : 32u;
        for (int q = 0; q < n; ++q) {
            const int s = q % kStages, buf = q & 1;
            if (q >= 2) ok = mbar_wait_warp(&drained[buf], ((uint32_t)(q >> 1) - 1u) & 1u);
            if (ok) ok = mbar_wait_warp(&full[s], (uint32_t)(q / kStages) & 1u);
            if (!ok) break;
            tc_fence_after_sync();
            if (elect_one()) {
                const uint32_t a = smem_u32(dyn) + (uint32_t)s * kStageBytes, b = a + 16384u;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    umma_fp8(tmem + (uint32_t)(buf * T), umma_smem_desc(a + k * a_step, 16384, 1024), umma_smem_desc(b + k * 32, 16, 1024), idesc, k > 0);
                umma_commit(&empty[s]);
                umma_commit(&done[buf]);
            }
            __syncwarp();
        }
    } else {
        const int t = (int)threadIdx.x - 64, quarter = warp & 3;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
        const float* const sa = p.sa + m0 + t;
        const float* const sw = p.sw + (long long)(j0 >> 7) * p.sw_j;
        const bool has = t < T && m0 + t < p.M;
        auto scale_at = [&](int q) { return has ? sa[(long long)(q0 + q) * p.sa_pitch] * sw[(long long)(q0 + q) * p.sw_q] : 0.f; };
        float acc[T];
#pragma unroll
        for (int i = 0; i < T; ++i) acc[i] = 0.f;
        if (t < T) scale[0][t] = scale_at(0);
        asm volatile("bar.sync 1, 128;" ::: "memory");
        for (int q = 0; q < n; ++q) {
            const int buf = q & 1;
            const float next = q + 1 < n ? scale_at(q + 1) : 0.f;
            ok = mbar_wait_warp(&done[buf], (uint32_t)(q >> 1) & 1u);
            if (bar_any(1, 128, !ok)) { ok = false; break; }
            tc_fence_after_sync();
#pragma unroll
            for (int c = 0; c < T; c += 16) {
                uint32_t raw[16];
                tmem_ld16(lanes + (uint32_t)(buf * T + c), raw);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[c + i] = fmaf(__uint_as_float(raw[i]), scale[buf][c + i], acc[c + i]);
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&drained[buf]);
            if (t < T) scale[buf ^ 1][t] = next;
            asm volatile("bar.sync 1, 128;" ::: "memory");
        }
        const int r = quarter * 32 + lane, j = j0 + r;
        TO* const out = static_cast<TO*>(p.out) + (long long)m0 * p.J + j;
        if (p.split == 1) {
            const float b = j < p.J ? bias_at(p, j) : 0.f;
#pragma unroll
            for (int i = 0; i < T; ++i)
                if (j < p.J && m0 + i < p.M) out[(long long)i * p.J] = from_f32<TO>(acc[i] + b);
        } else {
            float* const part = reinterpret_cast<float*>(dyn) + r;      // every copy and product of this CTA is done with the ring
            if (ok) {
#pragma unroll
                for (int i = 0; i < T; ++i) part[i * 128] = acc[i];
            }
        }
    }
    if (!ok) {
        atomicOr(p.err_word, 8192u);
        let_settle();
    }
    if (p.split > 1) {
        cluster_meet();
        if (warp >= 2) {
            const int r = (warp & 3) * 32 + lane, j = j0 + r;
            const int first = T * rank / p.split, end = T * (rank + 1) / p.split;
            const uint32_t part = smem_u32(dyn) + (uint32_t)r * 4u;
            const float b = j < p.J ? bias_at(p, j) : 0.f;
            TO* const out = static_cast<TO*>(p.out) + (long long)m0 * p.J + j;
            for (int i = first; i < end; ++i) {
                if (m0 + i >= p.M) break;
                float v = 0.f;
                for (int k = 0; k < p.split; ++k) v += peer_load(part + (uint32_t)i * 512u, k);
                if (j < p.J) out[(long long)i * p.J] = from_f32<TO>(v + b);
            }
        }
        cluster_meet();                                  // nothing of another CTA is read any more
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == 1) tmem_dealloc(tmem, kCols);
}

template <int T, typename TO> gf_status launch_few(ProductArgs& a, const void* codes, int L, long long a_pitch, cudaStream_t s) {
    static size_t configured[kMaxDevices] = {};
    auto kernel = fp8_few_kernel<T, TO>;
    const gf_status st = ensure_dyn_smem(kernel, few_smem(T), configured);
    if (st != GF_OK) return st;
    if (!make_tmap_u8_2d(&a.tm_a, codes, (uint64_t)L, (uint64_t)a.M, (uint64_t)a_pitch, T)) return GF_ERR_CUDA;
    a.tiles_m = (a.M + T - 1) / T;
    const long long tiles = (long long)a.tiles_m * ((a.J + 127) / 128);
    int split = (int)(2LL * sm_count() / tiles);
    split = split < 1 ? 1 : split > 8 ? 8 : split;
    if (split > a.chunks) split = a.chunks;
    a.per = (a.chunks + split - 1) / split;
    a.split = (a.chunks + a.per - 1) / a.per;
    if (tiles * a.split > 0x7fffffffLL) return GF_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * a.split)); cfg.blockDim = dim3(kFewThreads); cfg.dynamicSmemBytes = few_smem(T); cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.split; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a);
    count_launch();
    return e == cudaSuccess ? GF_OK : GF_ERR_CUDA;
}

template <typename TO> gf_status product(ProductArgs& a, const void* codes, int L, long long a_pitch, cudaStream_t s) {
    if (a.M <= 16) return launch_few<16, TO>(a, codes, L, a_pitch, s);
    if (a.M <= 32) return launch_few<32, TO>(a, codes, L, a_pitch, s);
    if (a.M <= 64) return launch_few<64, TO>(a, codes, L, a_pitch, s);
    return launch_few<128, TO>(a, codes, L, a_pitch, s);
}

constexpr int kMostDim = 1 << 24;

gf_status validate(const gf_fp8_desc* d) {
    if (!d) return GF_ERR_NULL;
    if (d->rows < 0 || d->cols < 1 || !is_dtype(d->dtype)) return GF_ERR_BAD_DESC;
    return d->cols > kMostDim ? GF_ERR_UNSUPPORTED : GF_OK;
}

gf_status check(const gf_fp8_desc* d, const void* x, const void* codes, const void* scales) {
    const gf_status st = validate(d);
    if (st != GF_OK || d->rows == 0) return st;
    if (!x || !codes || !scales) return GF_ERR_NULL;
    return off16(x) || off16(codes) || off16(scales) ? GF_ERR_ALIGN : GF_OK;
}

}  // namespace
}  // namespace gf

using namespace gf;

extern "C" {

gf_status gf_fp8_quantize_rows(const gf_fp8_desc* desc, const void* x, void* codes, float* scales, void* stream) {
    const gf_status st = check(desc, x, codes, scales);
    if (st != GF_OK || desc->rows == 0) return st;
    const int chunks = (desc->cols + 128 * kQuantGroups - 1) / (128 * kQuantGroups);
    const long long blocks = cdiv64(desc->rows, kQuantRows) * chunks, most = (long long)sm_count() * 8;
    const dim3 grid((unsigned)(blocks < most ? blocks : most));
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    ProfScope prof(K_FP8_QUANTIZE, s);
    auto go = [&](auto t, auto kernel) {
        using T = decltype(t);
        return launch_pdl(kernel, grid, dim3(kQuantThreads), 0, s, static_cast<const T*>(x), static_cast<uint8_t*>(codes), scales, (long long)desc->rows,
                          desc->cols, GF_FP8_PITCH(desc->cols), (long long)GF_FP8_SCALE_PITCH((long long)desc->rows), chunks, blocks);
    };
    const bool aligned = desc->cols % 8 == 0;
    if (desc->dtype == GF_F32) return aligned ? go(float(), quantize_rows_kernel<float, true>) : go(float(), quantize_rows_kernel<float, false>);
    return aligned ? go(__nv_bfloat16(), quantize_rows_kernel<__nv_bfloat16, true>) : go(__nv_bfloat16(), quantize_rows_kernel<__nv_bfloat16, false>);
}

gf_status gf_fp8_quantize_blocks(const gf_fp8_desc* desc, const void* w, void* codes, float* scales, void* stream) {
    const gf_status st = check(desc, w, codes, scales);
    if (st != GF_OK || desc->rows == 0) return st;
    const int col_blocks = (desc->cols + 127) / 128;
    const long long blocks = cdiv64(desc->rows, 128) * col_blocks, most = (long long)sm_count() * 8;
    const dim3 grid((unsigned)(blocks < most ? blocks : most));
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    ProfScope prof(K_FP8_QUANTIZE, s);
    auto go = [&](auto t, auto kernel) {
        using T = decltype(t);
        return launch_pdl(kernel, grid, dim3(kQuantThreads), 0, s, static_cast<const T*>(w), static_cast<uint8_t*>(codes), scales, (long long)desc->rows,
                          desc->cols, GF_FP8_PITCH(desc->cols), col_blocks, blocks);
    };
    return desc->dtype == GF_F32 ? go(float(), quantize_blocks_kernel<float>) : go(__nv_bfloat16(), quantize_blocks_kernel<__nv_bfloat16>);
}

gf_status gf_fp8_matmul(const gf_fp8_matmul_desc* desc, const void* a, const float* a_scales, const void* w, const float* w_scales, const void* bias,
                        void* out, void* stream) {
    if (!desc) return GF_ERR_NULL;
    const gf_fp8_matmul_desc& d = *desc;
    if (d.M < 0 || d.N < 1 || d.K < 1 || d.transposed < 0 || d.transposed > 1 || !is_dtype(d.out_dtype) || !is_dtype(d.bias_dtype)) return GF_ERR_BAD_DESC;
    if (d.N > kMostDim || d.K > kMostDim) return GF_ERR_UNSUPPORTED;
    if (d.M == 0) return GF_OK;
    if (!a || !a_scales || !w || !w_scales || !out) return GF_ERR_NULL;
    if (off16(a) || off16(a_scales) || off16(w) || off16(w_scales) || off16(bias) || off16(out)) return GF_ERR_ALIGN;
    const int L = d.transposed ? d.N : d.K;                 // contracted
    const long long col_blocks = (d.K + 127) / 128;
    ProductArgs p = {};
    p.sa = a_scales; p.sw = w_scales; p.bias = bias; p.bias_bf16 = d.bias_dtype == GF_BF16; p.out = out;
    p.M = d.M; p.J = d.transposed ? d.K : d.N; p.chunks = (L + 127) / 128;
    p.sa_pitch = GF_FP8_SCALE_PITCH((long long)d.M);
    p.sw_j = d.transposed ? 1 : col_blocks;
    p.sw_q = d.transposed ? col_blocks : 1;
    p.mn_major = d.transposed;
    p.err_word = global_err_word();
    if (!p.err_word) return GF_ERR_CUDA;
    // (in either form a box is 128 bytes of 128 rows of W)
    if (!make_tmap_u8_2d(&p.tm_w, w, (uint64_t)d.K, (uint64_t)d.N, (uint64_t)GF_FP8_PITCH(d.K), 128)) return GF_ERR_CUDA;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    ProfScope prof(K_FP8_PRODUCT, s);
    const long long a_pitch = GF_FP8_PITCH((long long)L);
    return d.out_dtype == GF_F32 ? product<float>(p, a, L, a_pitch, s) : product<__nv_bfloat16>(p, a, L, a_pitch, s);
}

}  // extern "C"

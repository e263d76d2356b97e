// Matrices in 8 bits with scales for groups of 128 (gf_block.h): quantisers, and the product of 8-bit rows with an 8-bit weight.
#include "gf_bench.h"
#include "gf_block.h"
#include "gf_octet.cuh"
#include "gf_pipe.cuh"
#include "gf_tc.cuh"
#include "gf_tma.cuh"

#include <type_traits>

namespace gf {
namespace {

bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
bool is_dtype(int d) { return d == GF_F32 || d == GF_BF16; }

// ---- quantisers ------------------------------------------------------------------------------------------------------
// Rows: sixteen threads (eight, with two octets each, of 16-bit values) have the 128 columns of a scale; a block has 16 (32) rows by 4
// scales, so that the loads of four octets are on their way at once and the scales of its rows make whole sectors.
// Bound by memory, for 16-bit values by instructions too (65536 x 512: 17.5 us, 0.88 of the copy bandwidth; 32 bits 26.6, 0.97; with one
// octet a thread 16 bits took 20.7).  Rows that are not whole octets are put together from two vectors each: 20000 x 1001 bf16 21 us.
constexpr int kQuantThreads = 256, kQuantGroups = 4;
template <typename T> constexpr int kQuantEach = sizeof(T) == 2 ? 2 : 1;
template <typename T> constexpr int kQuantRows = kQuantThreads / (16 / kQuantEach<T>);

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kQuantThreads) quantize_rows_kernel(const T* x, uint8_t* codes, float* scales, long long rows, int cols, int pitch,
                                                                      long long scale_pitch, int chunks, long long blocks) {
    pdl_launch_dependents();
    pdl_wait();
    constexpr int E = kQuantEach<T>, kParts = 16 / E, G = kQuantGroups / E;      // loads at once: G groups
    const int part = threadIdx.x % kParts;
    const long long total = rows * cols;
    uint32_t least = 0xffffffffu;                    // of the scales' orders
    for (long long b = blockIdx.x; b < blocks; b += gridDim.x) {
        const long long row = b / chunks * kQuantRows<T> + threadIdx.x / kParts;
        const int first = (int)(b % chunks) * (128 * kQuantGroups), end = min(pitch, first + 128 * kQuantGroups);
        for (int base = first; base < end; base += 128 * G) {                       // (the same for the block)
            const int c0 = base + part * 8 * E;
            Octet<T> o[G][E];
#pragma unroll
            for (int k = 0; k < G; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int c = c0 + 128 * k + 8 * e;
                    if (row < rows && c < cols) {
                        if (ALIGNED) o[k][e].load(x + row * cols + c);
                        else load_anywhere(o[k][e], x, row * cols + c, total);
                    } else o[k][e].clear();
                }
#pragma unroll
            for (int k = 0; k < G; ++k) {
                const int c = c0 + 128 * k;
                float v[E][8];
                uint32_t m = 0;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    o[k][e].get(v[e]);
                    if (!ALIGNED) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (c + 8 * e + i >= cols) v[e][i] = 0.f;
                    }
                    m = max(m, magnitude(v[e]));
                }
#pragma unroll
                for (int s = kParts / 2; s > 0; s >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, s));
                const float scale = scale_of(m), inv = __frcp_rn(scale);
                least = min(least, scale_order(scale));
                if (row < rows && c < pitch) {
                    uint2 w[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) w[e] = codes8(v[e], scale, inv, cols - c - 8 * e);
                    uint8_t* const to = codes + row * pitch + c;
                    if constexpr (E == 2) *reinterpret_cast<uint4*>(to) = make_uint4(w[0].x, w[0].y, w[1].x, w[1].y);      // (the pitch is one of 16)
                    else *reinterpret_cast<uint2*>(to) = w[0];
                    if (part == 0 && c < cols) scales[(long long)(c >> 7) * scale_pitch + row] = scale;
                }
            }
        }
    }
    if (!__any_sync(0xffffffffu, is_small_order(least))) return;
    __syncwarp();
    for (long long b = blockIdx.x; b < blocks; b += gridDim.x) {      // once more: scales and values lie in memory
        const long long row = b / chunks * kQuantRows<T> + threadIdx.x / kParts;
        const int first = (int)(b % chunks) * (128 * kQuantGroups), end = min(cols, first + 128 * kQuantGroups);
        if (row < rows)
            for (int c = first + part * 8 * E; c < end; c += 128)
                divide_codes(codes + row * pitch + c, scales[(long long)(c >> 7) * scale_pitch + row], min(8 * E, cols - c),
                             [&](int i) { return to_f32(x[row * cols + c + i]); });
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
            if (row < rows && c < pitch) {
                uint8_t* const to = codes + row * pitch + c;
                *reinterpret_cast<uint2*>(to) = codes8(v, scale, inv, cols - c);
                divide_codes(to, scale, min(8, cols - c), [&](int i) { return to_f32(x[row * cols + c + i]); });
            }
        }
        if (threadIdx.x == 0) scales[b] = scale;
    }
}

// ---- product ---------------------------------------------------------------------------------------------------------
// out[m, j] = sum over chunks q of 128 terms of  sa[m, q] sw[j / 128, q] (sum over the chunk of A[m, l] W'[l, j]),
// W' = W^T (the layer) or W (the gradient of its input).  The tensor cores add a chunk into one of two accumulators in tensor
// memory; warps that wait for it scale it and add it to fp32 registers while the next chunk is multiplied into the other.
struct ProductArgs {
    CUtensorMap tm_w, tm_a, tm_out;
    const float *sa, *sw;
    const void* bias;
    void* out;
    uint32_t* err_word;
    long long sa_pitch, sw_j, sw_q;      // strides of the scales: rows of sa; blocks of columns and chunks of sw
    int M, J, chunks, split;
    int share, longer;                   // few: of the `split` CTAs of a cluster the first `longer` have share + 1 chunks, the others share
    int tiles_m, bias_bf16;
    int bn;                              // wide: columns of a tile
    int out_map;                         // wide: results leave by the copy engine (their rows are whole 16-byte pieces)
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
__device__ __forceinline__ float4 peer_load4(uint32_t addr, int rank) {
    float4 v;
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n\t}"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(addr), "r"(rank)
                 : "memory");
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
// Waits for the loads before, and says so of their registers: nothing that uses them comes earlier.
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]),
                   "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}
__device__ __forceinline__ float bias_at(const ProductArgs& p, int j) {
    if (!p.bias) return 0.f;
    return p.bias_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.bias)[j]) : static_cast<const float*>(p.bias)[j];
}

// A row's scale times a block's, where that product is no normal number of fp32 (rows of zeros have the smallest scale, 2^-126): the sum
// of a chunk, zero or a multiple of 2^-18 below 2^25, is taken `first` times, which is exact, and then `then` times.  That way of adding
// stands apart, so that sums under normal products are not held up (for many rows the warp that has waited asks with the vote that ends
// its wait: the gradient of 4096 x 8192 x 4096 takes 155.6 us, 154.3 without the question, with a row of zeros in a hundred 183.8 and 150.8;
// 65536 x 2048 x 512 112.6 and 112.4, 115.3 and 112.1).
constexpr float kFirst = 0x1p100f;
struct TwoFactors {
    float first, then;
};
__device__ __forceinline__ bool is_normal(float s) { return fabsf(s) >= 0x1p-126f && fabsf(s) < INFINITY; }
__device__ __forceinline__ TwoFactors two_factors(float a, float w) {
    const float s = a * w, most = fmaxf(fabsf(a), fabsf(w)), least = fminf(fabsf(a), fabsf(w));
    if (fabsf(s) < 0x1p-126f) return {1.f / kFirst, copysignf(least * kFirst * most, s)};       // (below 2^-226 nothing is left either way)
    if (isinf(s) && most < INFINITY) return {kFirst, copysignf(fminf(most * (1.f / kFirst) * least, 0x1.fffffep127f), s)};      // finite: zero stays zero
    return {1.f, s};
}

// A tile is 128 columns of the result (rows of the accumulator) by T of its rows, so that the weight is the operand of
// 128 and few rows of A cost no more than they are.  The chunks of a tile are split over a cluster of CTAs where there
// are few tiles, and the parts are added through distributed shared memory, in the order of the CTAs.
//   warp 0: copies; warp 1: products; warps 2 to 5: scaling, a quarter of the accumulator's rows each.
// Bound by latency: 8 x 4096 x 4096 6.2 to 6.9 us, of which its bytes take 2.6 (16.8 MB from memory; a launch, one round of copies, four chunks,
// two meetings of the cluster); 8 x 768 x 768 3.4 to 3.8.
constexpr int kFewThreads = 192;
__host__ __device__ constexpr int few_stages(int T) { return T <= 32 ? 4 : 3; }
__host__ __device__ constexpr int few_buffers(int T) { return T <= 32 ? 4 : 2; }      // accumulators
constexpr int kFewScales = 16;                                                        // chunks whose scales are held at once
constexpr size_t few_smem(int T) { return (size_t)few_stages(T) * (16384 + T * 128) + 1024; }

template <int T, typename TO> __global__ void __launch_bounds__(kFewThreads) fp8_few_kernel(const __grid_constant__ ProductArgs p) {
    extern __shared__ unsigned char dyn_raw[];
    unsigned char* const dyn = align1024(dyn_raw);
    constexpr int kStages = few_stages(T), kStageBytes = 16384 + T * 128, kBuffers = few_buffers(T), kCols = kBuffers * T;
    __shared__ uint64_t full[kStages], empty[kStages], done[kBuffers], drained[kBuffers];
    __shared__ uint32_t tmem_base;
    __shared__ __align__(16) float scale[kFewScales][T];
    __shared__ __align__(16) __nv_bfloat16 first[kFewScales][T];      // and factors before them (two_factors), powers of two
    __shared__ int any_first;                            // other than 1 so far; written and read on either side of the scales' barriers
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int rank = (int)(blockIdx.x % (unsigned)p.split), tile = (int)(blockIdx.x / (unsigned)p.split);
    const int m0 = tile % p.tiles_m * T, j0 = tile / p.tiles_m * 128;
    const int q0 = rank * p.share + min(rank, p.longer), n = p.share + (rank < p.longer);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int s = 0; s < kBuffers; ++s) { mbar_init(&done[s], 1); mbar_init(&drained[s], 4); }
        any_first = 0;
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
            const int s = q % kStages, buf = q % kBuffers;
            if (q >= kBuffers) ok = mbar_wait_warp(&drained[buf], ((uint32_t)(q / kBuffers) - 1u) & 1u);
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
        const float* const sw = p.sw + (long long)(j0 >> 7) * p.sw_j;
        uint64_t acc[T / 2];
#pragma unroll
        for (int i = 0; i < T / 2; ++i) acc[i] = 0;
        // adds the accumulators of chunks from .. to - 1, whose scales are held
        auto add = [&](auto with_first, int from, int to) {
            for (int q = from; q < to && ok; ++q) {
                const int buf = q % kBuffers, held = q % kFewScales;
                ok = mbar_wait_warp(&done[buf], (uint32_t)(q / kBuffers) & 1u);
                if (!ok) break;
                tc_fence_after_sync();
#pragma unroll
                for (int c = 0; c < T; c += 16) {
                    uint32_t raw[16];
                    tmem_ld16(lanes + (uint32_t)(buf * T + c), raw);
                    tmem_ld_wait_for(raw);
                    if constexpr (decltype(with_first)::value) {
#pragma unroll
                        for (int h = 0; h < 16; h += 8) {
                            Octet<__nv_bfloat16> o;
                            float f[8];
                            o.load(&first[held][c + h]);
                            o.get(f);
#pragma unroll
                            for (int i = 0; i < 8; ++i) raw[h + i] = __float_as_uint(__uint_as_float(raw[h + i]) * f[i]);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const ulonglong2 s = *reinterpret_cast<const ulonglong2*>(&scale[held][c + i]);
                        uint64_t* const a = acc + (c + i) / 2;
                        a[0] = fma_pair(pair_of(__uint_as_float(raw[i]), __uint_as_float(raw[i + 1])), s.x, a[0]);
                        a[1] = fma_pair(pair_of(__uint_as_float(raw[i + 2]), __uint_as_float(raw[i + 3])), s.y, a[1]);
                    }
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&drained[buf]);
            }
        };
        // (after a wait that ran out a warp has part in the barriers still, and in nothing else)
        for (int q = 0; q < n; q += kFewScales) {
            if (q > 0) asm volatile("bar.sync 1, 128;" ::: "memory");
            const int end = min(n, q + kFewScales);      // the scales of the chunks up to there: by all four warps, for all
            bool odd = false;
            for (int i = t; i < (end - q) * T; i += 128) {
                const int m = m0 + i % T;
                const long long at = q0 + q + i / T;
                const float s = m < p.M ? p.sa[at * p.sa_pitch + m] * sw[at * p.sw_q] : 0.f;
                scale[i / T][i % T] = s;
                first[i / T][i % T] = __float2bfloat16_rn(1.f);
                odd |= m < p.M && !is_normal(s);
            }
            if (odd) {
                any_first = 1;
#pragma unroll 1
                for (int i = t; i < (end - q) * T; i += 128) {
                    const int m = m0 + i % T;
                    const long long at = q0 + q + i / T;
                    if (m < p.M) {
                        const TwoFactors f = two_factors(p.sa[at * p.sa_pitch + m], sw[at * p.sw_q]);
                        scale[i / T][i % T] = f.then;
                        first[i / T][i % T] = __float2bfloat16_rn(f.first);
                    }
                }
            }
            asm volatile("bar.sync 1, 128;" ::: "memory");
            if (any_first) add(std::true_type(), q, end);
            else add(std::false_type(), q, end);
        }
        const int r = quarter * 32 + lane, j = j0 + r;
        if (p.split == 1) {
            TO* const out = static_cast<TO*>(p.out) + (long long)m0 * p.J + j;
            const float b = j < p.J ? bias_at(p, j) : 0.f;
#pragma unroll
            for (int i = 0; i < T; ++i) {
                const float2 f = unpair(acc[i / 2]);
                if (j < p.J && m0 + i < p.M) out[(long long)i * p.J] = from_f32<TO>((i & 1 ? f.y : f.x) + b);
            }
        } else {
            float* const part = reinterpret_cast<float*>(dyn) + r;      // every copy and product of this CTA is done with the ring
            if (ok) {
#pragma unroll
                for (int i = 0; i < T; i += 2) {
                    const float2 f = unpair(acc[i / 2]);
                    part[i * 128] = f.x;
                    part[i * 128 + 128] = f.y;
                }
            }
        }
    }
    if (!ok) {
        atomicOr(p.err_word, 8192u);
        let_settle();
    }
    // Tensor memory goes back before this CTA waits for the others of its cluster: a CTA that holds it waits for nothing but its own
    // copies and products, so that no two clusters (of this or another kernel) can each hold what the other waits for.
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == 1) tmem_dealloc(tmem, kCols);
    if (p.split > 1) {
        // A CTA adds its share of the tile's rows, four columns a thread, with the loads of all parts on their way at once.
        constexpr int kCells = T * 32 / 128;                            // of a thread, for the whole tile
        cluster_meet();
        const int i0 = (int)threadIdx.x - 64, first = T * rank / p.split, cells = (T * (rank + 1) / p.split - first) * 32;
        float4 sum[kCells / 2];                                         // (split >= 2)
        if (warp >= 2) {
#pragma unroll
            for (int c = 0; c < kCells / 2; ++c) {
                const int cell = i0 + c * 128;
                if (cell < cells) {
                    const uint32_t at = smem_u32(dyn) + (uint32_t)((first + (cell >> 5)) * 512 + (cell & 31) * 16);
                    float4 v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = k < p.split ? peer_load4(at, k) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int k = 1; k < 8; ++k) { v[0].x += v[k].x; v[0].y += v[k].y; v[0].z += v[k].z; v[0].w += v[k].w; }
                    sum[c] = v[0];
                }
            }
        }
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");   // what this CTA needs of the others is read
        if (warp >= 2) {
#pragma unroll
            for (int c = 0; c < kCells / 2; ++c) {
                const int cell = i0 + c * 128, m = m0 + first + (cell >> 5), j = j0 + (cell & 31) * 4;
                if (cell < cells && m < p.M && j < p.J) {
                    const float v[4] = {sum[c].x, sum[c].y, sum[c].z, sum[c].w};
                    TO* const out = static_cast<TO*>(p.out) + (long long)m * p.J + j;
                    __align__(16) TO o[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i] = from_f32<TO>(v[i] + (j + i < p.J ? bias_at(p, j + i) : 0.f));
                    if ((p.J & 3) == 0) {
                        if constexpr (sizeof(TO) == 4) *reinterpret_cast<uint4*>(out) = *reinterpret_cast<const uint4*>(o);
                        else *reinterpret_cast<uint2*>(out) = *reinterpret_cast<const uint2*>(o);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (j + i < p.J) out[i] = o[i];
                    }
                }
            }
        }
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");      // nothing of another CTA is read any more
    }
}

// CTAs that share the chunks of a tile, up to two per SM in all, by what that takes in microseconds: 0.6 a chunk, 1.5 for the cluster
// and its joining and 0.15 more for each of its CTAs.  Halves, quarters and eighths are considered, each with as many CTAs as it has
// shares: 6 of 3 chunks for 17 and 18 (8 x 2304 x 2304 4.9 us; dealt to 8 it takes 5.4).  Only 3 are 4 instead (8 x 768 x 768 3.4 us for 3.7,
// 100 x 768 x 768 5.2 for 5.7).
int few_ctas(int chunks, int split) {
    const int share = (chunks + split - 1) / split, ctas = (chunks + share - 1) / share;
    return ctas == 3 ? 4 : ctas;
}
double few_time(int chunks, int ctas) { return 0.6 * ((chunks + ctas - 1) / ctas) + (ctas > 1 ? 1.5 + 0.15 * ctas : 0.0); }
int few_cluster(long long tiles, int chunks) {
    int best = 1;
    for (int split = 2; split <= 8 && split <= chunks && split * tiles <= 2LL * sm_count(); split *= 2) {
        const int ctas = few_ctas(chunks, split);
        if (few_time(chunks, ctas) < few_time(chunks, best)) best = ctas;
    }
    return best;
}

// Rows of A of a tile
int few_rows(int M) { return M <= 16 ? 16 : M <= 32 ? 32 : 64; }
int few_cluster(const ProductArgs& a, int rows) { return few_cluster(cdiv64(a.M, rows) * ((a.J + 127) / 128), a.chunks); }

template <int T, typename TO>
gf_status launch_few(ProductArgs& a, const void* w, const void* codes, int N, int K, int L, long long a_pitch, cudaStream_t s) {
    static size_t configured[kMaxDevices] = {};
    auto kernel = fp8_few_kernel<T, TO>;
    const gf_status st = ensure_dyn_smem(kernel, few_smem(T), configured);
    if (st != GF_OK) return st;
    // (in either form a box is 128 bytes of 128 rows of W)
    if (!make_tmap_u8_2d(&a.tm_w, w, (uint64_t)K, (uint64_t)N, (uint64_t)GF_FP8_PITCH(K), 128)) return GF_ERR_CUDA;
    if (!make_tmap_u8_2d(&a.tm_a, codes, (uint64_t)L, (uint64_t)a.M, (uint64_t)a_pitch, T)) return GF_ERR_CUDA;
    a.tiles_m = (int)cdiv64(a.M, T);
    const long long tiles = (long long)a.tiles_m * ((a.J + 127) / 128);
    a.split = few_cluster(a, T);
    a.share = a.chunks / a.split;
    a.longer = a.chunks % a.split;
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

// Many rows: pairs of CTAs walk over tiles of 256 rows by 128 or 256 columns.  Each CTA of a pair has 128 rows of the result, and
// brings its 128 rows of A and half of the tile's columns of W; the products of a pair (cta_group::2) read both halves, so that a
// chunk of 128 terms costs each SM 32 KB from L2 for 512 clocks of products.
//   warp 0: copies; warp 1 (of the first CTA): products; warps 4 to 19: scaling, a quarter of the rows by a quarter of
//   the columns each, in registers, which the first four warps give up for them; the next tile's first two chunks are
//   multiplied while they write their results, by the copy engine where rows are whole 16-byte pieces (65536 x 2048 x 512: 97 to 113 us;
//   stored by the warps 143; 14672 x 4241 x 64, whose rows are not, 59 in bf16 and 102 in fp32, 4240 columns 24 and 47).
// What bounds it is the accumulators' way out of tensor memory, once for every 128 terms, which the scales ask for: reading one
// takes the port that the products accumulate through for 260 clocks of a chunk's 512, and between a chunk's product and the next
// product into its accumulator lie 1700 clocks of signals, reads and sums, with two accumulators: about 1100 clocks a chunk.  4096 x
// 8192 x 4096 runs at 1.75 to 1.9 PFLOP/s either way (the power that its data take decides; 1.6 under the power cap, which runs of some
// milliseconds meet); with the reads and sums left out the products take 2.97.  Measured and not taken: four accumulators of half the columns (A is read
// twice: 159 us for 147), 8 scaling warps of 128 columns (157), scales through a ring in shared memory (147 for 140).
constexpr int kWideThreads = 640, kWideStages = 5, kWideStage = 32768, kWidePiece = 32 * 128;
constexpr int kWideWarps = 16;                     // that scale
constexpr size_t kWideSmem = (size_t)kWideStages * kWideStage + kWideWarps * kWidePiece + 1024;
static_assert(kWideSmem + 256 <= 232448, "shared memory of a block");
static_assert(128 * 32 + 512 * 112 <= kWideThreads * 96, "registers of the launch");
constexpr uint32_t kLeaderMask = 0xFEFFFFFFu;      // a shared address of either CTA -> the same place in the first one

__device__ __forceinline__ void load_box_pair(void* dst, const CUtensorMap* m, int x, int y, uint64_t* bar) {
    // the bytes land here, their arrival is counted on the first CTA's barrier
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(smem_u32(bar) & kLeaderMask)
        : "memory");
}
// As umma_smem_desc, for tiles of 64-byte rows under the 64-byte swizzle
__device__ __forceinline__ uint64_t umma_smem_desc64(uint32_t saddr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
    return (umma_smem_desc(saddr, lbo_bytes, sbo_bytes) & ~((uint64_t)7 << 61)) | ((uint64_t)4 << 61);
}
__device__ __forceinline__ void umma_fp8_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void commit_pair(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
                 "h"((uint16_t)3)
                 : "memory");
}
// (What the arrival orders are reads of tensor memory, for which the fence of tcgen05 stands.  Releasing ordinary memory to the cluster
// as well took about 1500 clocks an arrival: 3.0 -> 1.2 PFLOP/s of products.)
__device__ __forceinline__ void arrive_leader(uint64_t* bar) {
    asm volatile(
        "{\n\t.reg .b32 a;\n\t"
        "mapa.shared::cluster.u32 a, %0, 0;\n\t"
        "mbarrier.arrive.shared::cluster.b64 _, [a];\n\t}" ::"r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]),
                   "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]),
                   "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]),
                   "+r"(r[31])::"memory");
}

// NC columns of a warp's 32 rows into `buf`: a thread has a row, whose 16-byte pieces lie as the copy engine's
// swizzle has them (rows of 128 or 64 bytes), so that neither these writes nor the copy's reads meet in a bank.
template <typename TO, int NC> __device__ __forceinline__ void stage_piece(unsigned char* buf, const uint64_t* acc, int lane) {
    constexpr int kVec = 16 / (int)sizeof(TO), kBytes = NC * (int)sizeof(TO);
    static_assert(kBytes == 128 || kBytes == 64, "rows of a swizzle's width");
    const int flip = kBytes == 128 ? lane & 7 : (lane >> 1) & 3;
#pragma unroll
    for (int c = 0; c < NC; c += kVec) {
        float v[kVec];
#pragma unroll
        for (int i = 0; i < kVec; i += 2) {
            const float2 f = unpair(acc[(c + i) / 2]);
            v[i] = f.x; v[i + 1] = f.y;
        }
        uint4 w;
        if constexpr (sizeof(TO) == 4) w = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        else {
            uint32_t* const q = &w.x;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                q[i] = *reinterpret_cast<const uint32_t*>(&b);
            }
        }
        *reinterpret_cast<uint4*>(buf + lane * kBytes + ((c / kVec) ^ flip) * 16) = w;
    }
}
// The same piece to memory by the warp itself, where the result's rows are not whole 16-byte pieces.
// 32 bits: a row at a time, an element a lane.
__device__ __forceinline__ void store_elements(float* out, int pitch, const unsigned char* buf, int rows, int live) {
    const int lane = (int)threadIdx.x & 31;
#pragma unroll 1
    for (int r0 = 0; r0 < rows; r0 += 8) {
        float w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = *reinterpret_cast<const float*>(buf + (r0 + k) * 128 + (((lane >> 2) ^ k) & 7) * 16 + (lane & 3) * 4);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (r0 + k < rows && lane < live) out[(long long)(r0 + k) * pitch + lane] = w[k];
    }
}
// 16 bits: eight (four) lanes have a row and write what lies between its 16-byte boundaries in whole pieces, two of the buffer's
// shifted, and the elements before and behind one by one (14672 x 4241 x 64: 97 us an element a lane, 59 so).
template <int kBytes> __device__ __forceinline__ void store_shifted(__nv_bfloat16* out, int pitch, const unsigned char* buf, int rows, int live) {
    using TO = __nv_bfloat16;
    constexpr int kVec = 8, kLanes = kBytes / 16, kRows = 32 / kLanes;
    const int lane = (int)threadIdx.x & 31, v = lane % kLanes;
#pragma unroll 2
    for (int r = lane / kLanes; r < 32; r += kRows) {
        TO* const row = out + (long long)r * pitch;
        const unsigned char* const from = buf + r * kBytes;
        const int turn = kBytes == 128 ? r & 7 : (r >> 1) & 3;
        const int head = (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / 2;      // elements before the first boundary
        const uint4 a = *reinterpret_cast<const uint4*>(from + (v ^ turn) * 16), b = *reinterpret_cast<const uint4*>(from + (min(v + 1, kLanes - 1) ^ turn) * 16);
        if (r < rows) {
            if (head + (v + 1) * kVec <= live) {
                uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                const int words = head / 2;                                                // 0 .. 3
                if (words & 2) {
#pragma unroll
                    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
                }
                if (words & 1) {
#pragma unroll
                    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
                }
                if (head & 1) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
                }
                *reinterpret_cast<uint4*>(row + head + v * kVec) = make_uint4(w[0], w[1], w[2], w[3]);
            }
            auto at = [&](int c) { return *reinterpret_cast<const TO*>(from + ((c / kVec) ^ turn) * 16 + c % kVec * 2); };
            const int tail = live > head ? head + (live - head) / kVec * kVec : head;
#pragma unroll
            for (int e = v; e < kVec - 1; e += kLanes) {
                if (e < min(head, live)) row[e] = at(e);
                if (tail + e < live) row[tail + e] = at(tail + e);
            }
        }
    }
}
// (A call of its own, so that its registers are not taken from the loop that scales: with them 64 bytes went to memory there, a
// quarter of the time of 4096 x 8192 x 4096.)
template <typename TO> __device__ __noinline__ void store_piece(TO* out, int pitch, const unsigned char* buf, int rows, int live, int bytes) {
    __syncwarp();
    if constexpr (sizeof(TO) == 4) store_elements(out, pitch, buf, rows, live);
    else if (bytes == 128) store_shifted<128>(out, pitch, buf, rows, live);
    else store_shifted<64>(out, pitch, buf, rows, live);
    __syncwarp();
}

// Adds the bias of a warp's columns, one (and for 64 columns another) of which each lane brings, by way of `buf`.
__device__ __forceinline__ void add_bias(uint64_t (&acc)[32], float* buf, float b0, float b1, int cols, int lane) {
    buf[lane] = b0;
    buf[32 + lane] = b1;
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 64; c += 4) {
        if (c < cols) {
            const float4 v = *reinterpret_cast<const float4*>(buf + c);
            const float2 x = unpair(acc[c / 2]), y = unpair(acc[c / 2 + 1]);
            acc[c / 2] = pair_of(x.x + v.x, x.y + v.y);
            acc[c / 2 + 1] = pair_of(y.x + v.z, y.y + v.w);
        }
    }
    __syncwarp();
}

template <typename TO> __global__ void __launch_bounds__(kWideThreads, 1) fp8_wide_kernel(const __grid_constant__ ProductArgs p) {
    extern __shared__ unsigned char dyn_raw[];
    unsigned char* const dyn = align1024(dyn_raw);
    __shared__ uint64_t full[kWideStages], empty[kWideStages], done[4], drained[4];
    __shared__ uint32_t tmem_base;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int rank = (int)blockIdx.x & 1, unit = (int)blockIdx.x >> 1, units = (int)gridDim.x >> 1;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kWideStages; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int s = 0; s < 4; ++s) { mbar_init(&done[s], 1); mbar_init(&drained[s], 2 * kWideWarps); }
        mbar_fence_init();
    }
    pdl_wait();
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before_sync();
    __syncthreads();
    cluster_meet();                                      // the other CTA's barriers are ready
    tc_fence_after_sync();
    pdl_launch_dependents();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base, 0);
    const int share = p.bn / 2;                          // columns whose W a CTA brings
    const int tiles_j = (p.J + p.bn - 1) / p.bn;
    const int tiles = p.tiles_m * tiles_j;
    const uint32_t shift = p.bn == 256 ? 1u : 2u, buffers = 1u << shift;      // accumulators in tensor memory
    // tiles unit, unit + units, ..: rows and columns of tiles are counted on, not divided
    const int step_m = units / tiles_j, step_j = units % tiles_j;
    auto advance = [&](int& tm, int& tj) {
        tm += step_m;
        tj += step_j;
        if (tj >= tiles_j) { tj -= tiles_j; ++tm; }
    };
    unsigned char* const pieces = dyn + kWideStages * kWideStage;
    constexpr int kPieceCols = sizeof(TO) == 2 ? 64 : 32;                      // columns that are staged at once, at most
    bool ok = true;

    if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
    if (warp == 0) {
        uint32_t ring = 0;                               // one bit per stage: the parity of its next use
        int s = 0;
        const uint32_t bytes = 16384u + (uint32_t)share * 128u;
        int tm = unit / tiles_j, tj = unit % tiles_j;
        for (int t = unit; t < tiles && ok; t += units, advance(tm, tj)) {
            const int m = tm * 256 + rank * 128, j = tj * p.bn + rank * share;
            for (int q = 0; q < p.chunks; ++q) {
                ok = mbar_wait_warp(&empty[s], ((ring >> s) & 1u) ^ 1u);
                if (!ok) break;
                if (elect_one()) {
                    unsigned char* const st = dyn + (size_t)s * kWideStage;
                    if (rank == 0) mbar_expect_tx(&full[s], 2u * bytes);
                    load_box_pair(st, &p.tm_a, q * 128, m, &full[s]);
                    if (p.mn_major) load_box_pair(st + 16384, &p.tm_w, j, q * 128, &full[s]);
                    else load_box_pair(st + 16384, &p.tm_w, q * 128, j, &full[s]);
                }
                __syncwarp();
                ring ^= 1u << s;
                if (++s == kWideStages) s = 0;
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            const uint32_t idesc = fp8_idesc(256, p.bn, 0u, p.mn_major ? 1u : 0u);
            // W: rows of 128 terms, or 128 rows of a CTA's 128 or 64 columns
            const uint64_t a_form = umma_smem_desc(0, 16, 1024);
            const uint64_t b_form = p.mn_major && share == 64 ? umma_smem_desc64(0, 8192, 512) : umma_smem_desc(0, 16384, 1024);
            const uint32_t b_step = p.mn_major ? (uint32_t)share * 2u : 2u;  // 32 terms further, in 16 bytes
            const uint32_t ring0 = smem_u32(dyn) >> 4;
            uint32_t ring = 0, use = 0;
            int s = 0;
            for (int t = unit; t < tiles && ok; t += units) {
                for (int q = 0; q < p.chunks; ++q, ++use) {
                    const uint32_t buf = use & (buffers - 1u);
                    ok = mbar_wait_warp(&full[s], (ring >> s) & 1u);         // (long there: the accumulator is what is waited for)
                    if (ok && use >= buffers) ok = mbar_wait_warp(&drained[buf], ((use >> shift) - 1u) & 1u);
                    if (!ok) break;
                    tc_fence_after_sync();
                    if (elect_one()) {
                        const uint32_t at = ring0 + (uint32_t)s * (kWideStage >> 4);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            umma_fp8_pair(tmem + buf * (uint32_t)p.bn, a_form + at + k * 2, b_form + at + 1024u + k * b_step, idesc, k > 0);
                        commit_pair(&done[buf]);
                        commit_pair(&empty[s]);
                    }
                    __syncwarp();
                    ring ^= 1u << s;
                    if (++s == kWideStages) s = 0;
                }
            }
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 112;");
        const int quarter = warp & 3, cols = p.bn / 4, col = ((warp - 4) >> 2) * cols;      // this warp's columns: 32 or 64, and where
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)col;
        unsigned char* const piece = pieces + (warp - 4) * kWidePiece;
        // The scales of the next chunk, this tile's or the next one's, are fetched while one is added.
        uint32_t n = 0;                                  // chunks so far
        int ft = unit, fm = unit / tiles_j, fj = unit % tiles_j, fq = 0;
        int tm = fm, tj = fj;
        const float *fa = nullptr, *fw = nullptr;
        auto fetch_from = [&] {
            fa = p.sa + min((long long)fm * 256 + rank * 128 + quarter * 32 + lane, (long long)p.M - 1);
            fw = p.sw + (long long)min((fj * p.bn + col) >> 7, (p.J - 1) >> 7) * p.sw_j;
        };
        fetch_from();
        float a_next = __ldg(fa), w_next = __ldg(fw);
        auto fetch = [&] {
            if (++fq == p.chunks) {
                fq = 0;
                ft += units;
                advance(fm, fj);
                if (ft < tiles) fetch_from();            // (else: once more what is there)
            } else {
                fa += p.sa_pitch;
                fw += p.sw_q;
            }
            a_next = __ldg(fa);
            w_next = __ldg(fw);
        };
        for (int t = unit; t < tiles && ok; t += units, advance(tm, tj)) {
            const long long row0 = (long long)tm * 256 + rank * 128 + quarter * 32;
            const int j0 = tj * p.bn + col;
            uint64_t acc[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[i] = 0;
            float bias0 = 0.f, bias1 = 0.f;              // of this lane's columns; on their way while the tile is computed
            if (p.bias) {
                if (j0 + lane < p.J) bias0 = bias_at(p, j0 + lane);
                if (cols == 64 && j0 + 32 + lane < p.J) bias1 = bias_at(p, j0 + 32 + lane);
            }
            // adds a chunk's accumulator
            auto add = [&](auto with_first, uint32_t buf, TwoFactors f) {
                const uint64_t scale = pair_of(f.then, f.then);
                tc_fence_after_sync();
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if (c * 32 < cols) {
                        uint32_t raw[32];
                        tmem_ld32(lanes + buf * (uint32_t)p.bn + (uint32_t)(c * 32), raw);
                        tmem_ld_wait_for(raw);
                        if ((c + 1) * 32 >= cols) {      // the accumulator is read
                            tc_fence_before_sync();
                            __syncwarp();
                            if (lane == 0) arrive_leader(&drained[buf]);
                        }
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            uint64_t v = pair_of(__uint_as_float(raw[2 * i]), __uint_as_float(raw[2 * i + 1]));
                            if constexpr (decltype(with_first)::value) v = mul_pair(v, pair_of(f.first, f.first));
                            acc[c * 16 + i] = fma_pair(v, scale, acc[c * 16 + i]);
                        }
                    }
                }
            };
            for (int q = 0; q < p.chunks && ok; ++q, ++n) {
                const uint32_t buf = n & (buffers - 1u);
                const float a_now = a_next, w_now = w_next, now = a_now * w_now;
                fetch();
                const bool normal = is_normal(now), there = mbar_wait_bounded(&done[buf], (n >> shift) & 1u);
                if (__all_sync(0xffffffffu, there && normal)) add(std::false_type(), buf, TwoFactors{1.f, now});
                else {
                    ok = __all_sync(0xffffffffu, there);
                    if (!ok) break;
                    add(std::true_type(), buf, two_factors(a_now, w_now));
                }
            }
            if (!ok) break;
            if (row0 >= p.M || j0 >= p.J) continue;
            for (int c = 0; c < cols && j0 + c < p.J; c += kPieceCols) {
                bulk_wait_read<0>();                     // the copy before has read the buffer (for the thread that started it)
                __syncwarp();
                if (c == 0 && p.bias) add_bias(acc, reinterpret_cast<float*>(piece), bias0, bias1, cols, lane);
                if (cols >= kPieceCols) {
                    if (c == 0) stage_piece<TO, kPieceCols>(piece, acc, lane);
                    else stage_piece<TO, kPieceCols>(piece, acc + kPieceCols / 2 % 32, lane);
                } else stage_piece<TO, 32>(piece, acc, lane);
                if (p.out_map) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(reinterpret_cast<uint64_t>(&p.tm_out)),
                                     "r"(j0 + c), "r"((int)row0), "r"(smem_u32(piece))
                                     : "memory");
                        bulk_commit();
                    }
                } else {
                    store_piece(static_cast<TO*>(p.out) + row0 * p.J + j0 + c, p.J, piece, (int)min(32LL, p.M - row0), min(p.J - j0 - c, min(cols, kPieceCols)),
                                min(cols, kPieceCols) * (int)sizeof(TO));
                }
            }
        }
        bulk_wait_all();
    }
    if (!ok) {
        atomicOr(p.err_word, 8192u);
        let_settle();
    }
    tc_fence_before_sync();
    __syncthreads();
    cluster_meet();                                      // nothing of the other CTA refers to this one any more
    tc_fence_after_sync();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

int wide_columns(int J) { return J <= 128 ? 128 : 256; }
template <typename TO> bool whole_pieces(int J) { return (long long)J * sizeof(TO) % 16 == 0; }

template <typename TO> gf_status launch_wide(ProductArgs& a, const void* w, const void* codes, int N, int K, int L, long long a_pitch, cudaStream_t s) {
    static size_t configured[kMaxDevices] = {};
    auto kernel = fp8_wide_kernel<TO>;
    const gf_status st = ensure_dyn_smem(kernel, kWideSmem, configured);
    if (st != GF_OK) return st;
    a.tiles_m = (int)cdiv64(a.M, 256);
    a.bn = wide_columns(a.J);
    if (!make_tmap_u8_2d(&a.tm_a, codes, (uint64_t)L, (uint64_t)a.M, (uint64_t)a_pitch, 128)) return GF_ERR_CUDA;
    if (a.mn_major ? !make_tmap_u8_2d(&a.tm_w, w, (uint64_t)K, (uint64_t)N, (uint64_t)GF_FP8_PITCH(K), 128, (uint32_t)a.bn / 2)
                   : !make_tmap_u8_2d(&a.tm_w, w, (uint64_t)K, (uint64_t)N, (uint64_t)GF_FP8_PITCH(K), (uint32_t)a.bn / 2))
        return GF_ERR_CUDA;
    // (a tile's last columns and rows are cut off by the map)
    a.out_map = whole_pieces<TO>(a.J);
    if (a.out_map && !make_tmap_swizzled(&a.tm_out, a.out, (int)sizeof(TO), (uint64_t)a.J, (uint64_t)a.M, sizeof(TO) == 2 && a.bn == 256 ? 64u : 32u, 32u)) return GF_ERR_CUDA;
    const long long tiles = (long long)a.tiles_m * ((a.J + a.bn - 1) / a.bn);
    if (tiles > 0x7fffffffLL) return GF_ERR_UNSUPPORTED;
    const long long pairs = sm_count() / 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * (tiles < pairs ? tiles : pairs))); cfg.blockDim = dim3(kWideThreads); cfg.dynamicSmemBytes = kWideSmem; cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a);
    count_launch();
    return e == cudaSuccess ? GF_OK : GF_ERR_CUDA;
}

// Which kernel: estimates in microseconds, fitted to both on 1 to 10000 rows by 96 to 8192 columns and terms.  Wide: a chunk of a
// tile of 256 columns takes 0.55 (128: 0.3), results 1.3, and 2.7 (32 bits: 3.5) more where rows are not
// whole 16-byte pieces.  Few: as above, or of an SM's time, where there are more tiles than SMs, 0.46 a chunk and 1.8 a tile at least.  (300 x 4096 x 4096: 20.3 wide, 25.2 few; 200 rows:
// 19.9, 17.4; 2048 x 512 x 4096: 20.0, 16.3; 1024 x 2048 x 2048: 13.8, 15.8; 2000 x 1000 x 576: 7.9, 6.7; 4099 rows: 8.2, 12.0.)
template <typename TO> bool wide_is_faster(const ProductArgs& a) {
    if (a.M <= 32) return false;
    const int bn = wide_columns(a.J);
    const double by_hand = whole_pieces<TO>(a.J) ? 0.0 : sizeof(TO) == 4 ? 3.5 : 2.7;
    const double tiles = (double)cdiv64(a.M, 256) * ((a.J + bn - 1) / bn), rounds = (double)(long long)((tiles + sm_count() / 2 - 1) / (sm_count() / 2));
    const double wide = 3.2 + rounds * ((bn == 256 ? 0.55 : 0.3) * a.chunks + 1.3 + by_hand);
    const long long few_tiles = cdiv64(a.M, 64) * ((a.J + 127) / 128);
    const double alone = few_time(a.chunks, few_cluster(a, 64)), each = 0.46 * a.chunks;
    const double all = (each > 1.8 ? each : 1.8) * (double)few_tiles / sm_count();
    return wide < 3.5 + (alone > all ? alone : all);
}

template <typename TO> gf_status product(ProductArgs& a, const void* w, const void* codes, int N, int K, int L, long long a_pitch, cudaStream_t s) {
    if (wide_is_faster<TO>(a)) return launch_wide<TO>(a, w, codes, N, K, L, a_pitch, s);
    switch (few_rows(a.M)) {
        case 16: return launch_few<16, TO>(a, w, codes, N, K, L, a_pitch, s);
        case 32: return launch_few<32, TO>(a, w, codes, N, K, L, a_pitch, s);
        default: return launch_few<64, TO>(a, w, codes, N, K, L, a_pitch, s);
    }
}

template <typename TO> int32_t form(const ProductArgs& a) {
    if (wide_is_faster<TO>(a)) return 1 | (wide_columns(a.J) == 128 ? 2 : 0) | (whole_pieces<TO>(a.J) ? 0 : 4);
    return few_cluster(a, few_rows(a.M)) << 8;
}

constexpr int kMostDim = 1 << 24;

gf_status validate(const gf_fp8_desc* d) {
    if (!d) return GF_ERR_NULL;
    if (d->rows < 0 || d->cols < 1 || !is_dtype(d->dtype)) return GF_ERR_BAD_DESC;
    return d->cols > kMostDim ? GF_ERR_UNSUPPORTED : GF_OK;
}

gf_status validate(const gf_fp8_matmul_desc& d) {
    if (d.M < 0 || d.N < 1 || d.K < 1 || d.transposed < 0 || d.transposed > 1 || !is_dtype(d.out_dtype) || !is_dtype(d.bias_dtype)) return GF_ERR_BAD_DESC;
    return d.N > kMostDim || d.K > kMostDim ? GF_ERR_UNSUPPORTED : GF_OK;
}

void set_sizes(ProductArgs& p, const gf_fp8_matmul_desc& d) {
    p.M = d.M; p.J = d.transposed ? d.K : d.N; p.chunks = ((d.transposed ? d.N : d.K) + 127) / 128;
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
    const long long blocks = cdiv64(desc->rows, desc->dtype == GF_F32 ? kQuantRows<float> : kQuantRows<__nv_bfloat16>) * chunks, most = 1 << 30;
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
    const gf_status st = validate(d);
    if (st != GF_OK || d.M == 0) return st;
    if (!a || !a_scales || !w || !w_scales || !out) return GF_ERR_NULL;
    if (off16(a) || off16(a_scales) || off16(w) || off16(w_scales) || off16(bias) || off16(out)) return GF_ERR_ALIGN;
    const int L = d.transposed ? d.N : d.K;                 // contracted
    const long long col_blocks = (d.K + 127) / 128;
    ProductArgs p = {};
    p.sa = a_scales; p.sw = w_scales; p.bias = bias; p.bias_bf16 = d.bias_dtype == GF_BF16; p.out = out;
    set_sizes(p, d);
    p.sa_pitch = GF_FP8_SCALE_PITCH((long long)d.M);
    p.sw_j = d.transposed ? 1 : col_blocks;
    p.sw_q = d.transposed ? col_blocks : 1;
    p.mn_major = d.transposed;
    p.err_word = global_err_word();
    if (!p.err_word) return GF_ERR_CUDA;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    ProfScope prof(K_FP8_PRODUCT, s);
    const long long a_pitch = GF_FP8_PITCH((long long)L);
    return d.out_dtype == GF_F32 ? product<float>(p, w, a, d.N, d.K, L, a_pitch, s) : product<__nv_bfloat16>(p, w, a, d.N, d.K, L, a_pitch, s);
}

int32_t gf_selftest_fp8_form(const gf_fp8_matmul_desc* desc) {
    if (!desc || validate(*desc) != GF_OK || desc->M == 0) return -1;
    ProductArgs p = {};
    set_sizes(p, *desc);
    return desc->out_dtype == GF_F32 ? form<float>(p) : form<__nv_bfloat16>(p);
}

}  // extern "C"

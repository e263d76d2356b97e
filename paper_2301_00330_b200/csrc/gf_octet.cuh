// Rows taken as octets: eight consecutive elements, as the elementwise operators and row norms of gf_block.h read, compute and
// write them, with the counter-based random bits of an octet and its rounding to 8 bits.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "gf_common.cuh"

namespace gf {

// ---- pairs of fp32 ---------------------------------------------------------------------------------------
// Two operations per instruction, each half rounded as the scalar one is: the loops over rows are bound by instructions.
__device__ __forceinline__ uint64_t pair_of(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 unpair(uint64_t v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float sum_of(uint64_t v) {
    const float2 f = unpair(v);
    return f.x + f.y;
}
// Eight values as four pairs
typedef uint64_t Eight[4];
__device__ __forceinline__ void to_eight(const float (&v)[8], Eight& p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = pair_of(v[2 * i], v[2 * i + 1]);
}
__device__ __forceinline__ void from_eight(const Eight& p, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpair(p[i]);
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
}

// ---- eight elements as they lie in memory ------------------------------------------------------------------
template <typename T> struct Octet {
    static constexpr int kWords = 2 * (int)sizeof(T);      // 32-bit words
    uint32_t w[kWords];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0u;
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&b);
            }
        }
    }
    __device__ __forceinline__ void get(Eight& p) const {
        float v[8];
        get(v);
        to_eight(v, p);
    }
    __device__ __forceinline__ void set(const Eight& p) {
        float v[8];
        from_eight(p, v);
        set(v);
    }
    // p: 16-byte aligned
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < kWords; i += 4) {
            const uint4 a = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint32_t*>(p) + i);
            w[i] = a.x; w[i + 1] = a.y; w[i + 2] = a.z; w[i + 3] = a.w;
        }
    }
    __device__ __forceinline__ void store(T* p) const {
#pragma unroll
        for (int i = 0; i < kWords; i += 4)
            *reinterpret_cast<uint4*>(reinterpret_cast<uint32_t*>(p) + i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
    }
    // element i from memory (i is a constant where this is called)
    __device__ __forceinline__ void put(int i, T v) {
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v);
        else {
            const uint32_t b = __bfloat16_as_ushort(v);
            w[i >> 1] = i & 1 ? (w[i >> 1] & 0xffffu) | (b << 16) : (w[i >> 1] & 0xffff0000u) | b;
        }
    }
};

// The aligned octet number f of a tensor of `total` elements; what lies past its end reads as zeros.
template <typename T> __device__ __forceinline__ void load_octet(Octet<T>& o, const T* base, long long f, long long total) {
    const long long e = f * 8;
    if (e + 8 <= total) { o.load(base + e); return; }
    o.clear();
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (e + i < total) o.put(i, base[e + i]);
}

// Eight elements from element e on, wherever that lies; those past the tensor's end read as zeros.  Two aligned octets, shifted.
template <typename T> __device__ __forceinline__ void load_anywhere(Octet<T>& o, const T* base, long long e, long long total) {
    const int shift = (int)(e & 7);
    Octet<T> a, b;
    load_octet(a, base, e >> 3, total);
    if (shift == 0) { o = a; return; }
    b.clear();
    if ((e >> 3) * 8 + 8 < total) load_octet(b, base, (e >> 3) + 1, total);
    constexpr int n = Octet<T>::kWords;
    uint32_t w[2 * n];
#pragma unroll
    for (int i = 0; i < n; ++i) { w[i] = a.w[i]; w[n + i] = b.w[i]; }
    constexpr int four = n / 2, two = n / 4;
    if (shift & 4) {
#pragma unroll
        for (int i = 0; i + four < 2 * n; ++i) w[i] = w[i + four];
    }
    if (shift & 2) {
#pragma unroll
        for (int i = 0; i + two < 2 * n; ++i) w[i] = w[i + two];
    }
    if (shift & 1) {
#pragma unroll
        for (int i = 0; i < n; ++i) w[i] = sizeof(T) == 4 ? w[i + 1] : __funnelshift_r(w[i], w[i + 1], 16);
    }
#pragma unroll
    for (int i = 0; i < n; ++i) o.w[i] = w[i];
}

// ---- random bits of an octet ------------------------------------------------------------------------------------
// Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", SC 2011).
__device__ __forceinline__ uint4 philox(uint64_t block, uint64_t offset, uint64_t key) {
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)p1;
        c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// Dropout as the kernels take it.  threshold 0: nothing is dropped.
struct Drop {
    const uint64_t* seed;
    uint32_t threshold;        // of 65536
    float scale;               // 65536 / (65536 - threshold); 0 when all is dropped
};
Drop make_drop(float p, const uint64_t* seed);
static inline bool valid_p(float p) { return p >= 0.f && p <= 1.f; }

// The two words of a seed.
__device__ __forceinline__ void load_seed(const Drop& d, uint64_t& key, uint64_t& offset) {
    key = offset = 0;
    if (d.threshold) {
        key = d.seed[0];
        offset = d.seed[1];
    }
}

// The 16 bits of element i of an octet decide at the top of a word: (w >> 16) >= t is w >= t << 16, and for all to be dropped
// (t = 65536) no word passes.
__device__ __forceinline__ bool is_kept(const uint32_t (&w)[4], int i, const Drop& d) {
    const uint32_t bits = i & 1 ? w[i >> 1] : w[i >> 1] << 16;          // (what lies below the half does not matter)
    return bits >= d.threshold << 16 && d.threshold != 65536u;
}

// v[i] <- kept ? v[i] scale : 0 for the elements of octet number f.
__device__ __forceinline__ void drop_octet(float (&v)[8], uint64_t f, uint64_t key, uint64_t offset, const Drop& d) {
    const uint4 r = philox(f, offset, key);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = is_kept(w, i, d) ? v[i] * d.scale : 0.f;
}

__device__ __forceinline__ void drop_octet(Eight& v, uint64_t f, uint64_t key, uint64_t offset, const Drop& d) {
    float x[8];
    from_eight(v, x);
    drop_octet(x, f, key, offset, d);
    to_eight(x, v);
}

// v[i] <- kept ? v[i] scale + add[i] : add[i].
// The product is rounded before the sum, so that the sum is that of the dropped branch as it is without a residual.  Left unrounded
// inside a fused operation it carries the scale's own error into sums that cancel: with 4/3 for p = 1/4 exact ties of a bf16 sum
// went the wrong way, one element in 600.  (One value at a time: a product and a sum of pairs are fused by the compiler.)
__device__ __forceinline__ void drop_octet(Eight& v, const Eight& add, uint64_t f, uint64_t key, uint64_t offset, const Drop& d) {
    const uint4 r = philox(f, offset, key);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
    float kept[8], dropped[8];
    from_eight(v, kept);
#pragma unroll
    for (int i = 0; i < 8; ++i) kept[i] = __fmul_rn(kept[i], d.scale);
    Eight sum;
    to_eight(kept, sum);
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = add_pair(sum[i], add[i]);
    from_eight(sum, kept);
    from_eight(add, dropped);
#pragma unroll
    for (int i = 0; i < 8; ++i) kept[i] = is_kept(w, i, d) ? kept[i] : dropped[i];
    to_eight(kept, v);
}

__device__ __forceinline__ void drop_octet(float (&v)[8], const float (&add)[8], uint64_t f, uint64_t key, uint64_t offset, const Drop& d) {
    Eight x, w;
    to_eight(v, x);
    to_eight(add, w);
    drop_octet(x, w, f, key, offset, d);
    from_eight(x, v);
}

// ---- 8 bits ---------------------------------------------------------------------------------------------------------
constexpr float kFp8Top = 448.f, kFp8Tiny = 1.17549435e-38f;

// Largest magnitude as bits: ordered like unsigned numbers, NaN above all.
__device__ __forceinline__ uint32_t magnitude(const float (&v)[8]) {
    float m;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(v[0]), "f"(v[1]), "f"(v[2]));
#pragma unroll
    for (int i = 3; i < 8; i += 2) asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(v[i]), "f"(v[i + 1 < 8 ? i + 1 : i]));
    return __float_as_uint(m) & 0x7fffffffu;
}
__device__ __forceinline__ float scale_of(uint32_t magnitude_bits) {
    return magnitude_bits >= 0x7f800000u ? __uint_as_float(magnitude_bits) : fmaxf(__uint_as_float(magnitude_bits) * (1.f / kFp8Top), kFp8Tiny);
}
// Two values to codes, the first in the low byte; values of magnitude above 448 give 448, NaN gives NaN.
__device__ __forceinline__ uint32_t codes2(float a, float b) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
    return r;
}
// Codes of eight values, of which `valid` are the row's (the others get 0), under `scale`, inv its rounded reciprocal.  The quotient
// is the product with inv and one correction by the remainder (Markstein 1990: the correctly rounded quotient), so that codes
// are those of a division.  It is formed of -v, and the codes' signs turned at the end: in that order of signs a remainder of
// zero leaves the sign of a zero.  A scale that is not finite leaves NaN.
// The remainder has to be exact.  Its last place is that of the quotient, 2^-34 just below the lowest border (2^-10), times that of the
// scale, and may not lie below 2^-149, as it does with scales below 2^-92: who calls this sees to small scales (below).
__device__ __forceinline__ uint2 codes8(const float (&v)[8], float scale, float inv, int valid) {
    uint32_t c[4];
    const uint64_t minus_inv = pair_of(-inv, -inv), scale2 = pair_of(scale, scale);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t x = pair_of(v[2 * i], v[2 * i + 1]), y = mul_pair(x, minus_inv);
        const float2 q = unpair(fma_pair(fma_pair(y, scale2, x), minus_inv, y));
        c[i] = codes2(q.x, q.y);
    }
    uint2 r = make_uint2((c[0] | (c[1] << 16)) ^ 0x80808080u, (c[2] | (c[3] << 16)) ^ 0x80808080u);
    if (valid < 8) {
        r.x = valid >= 4 ? r.x : valid <= 0 ? 0u : r.x & (0xffffffffu >> (32 - 8 * valid));
        r.y = valid <= 4 ? 0u : r.y & (0xffffffffu >> (64 - 8 * valid));
    }
    return r;
}

// Scales that are too small for codes8.  The quotients are those of values and scale taken kFp8Up times, or of a division.
constexpr float kFp8Small = 0x1p-90f, kFp8Up = 0x1p64f;
__device__ __forceinline__ bool is_small_scale(float scale) { return scale < kFp8Small; }
// For the search of a tensor's small scales: numbers in their order, the smallest scale of all being the largest.  That is a power of two,
// whose quotients need no correction, and zeros have it, which are not to be looked for.
__device__ __forceinline__ uint32_t scale_order(float scale) { return __float_as_uint(scale) - (__float_as_uint(kFp8Tiny) + 1u); }
__device__ __forceinline__ bool is_small_order(uint32_t order) { return order < scale_order(kFp8Small); }

// Codes of n values by division, if the scale is too small for codes8.  value(i): where they can be had again, so that this may stand
// behind the loop that calls codes8 (with a choice of factors within, rows of 65536 x 512 bf16 take 19.6 us, with this 17.3).
template <typename Value> __device__ __forceinline__ void divide_codes(uint8_t* codes, float scale, int n, Value&& value) {
    if (!is_small_order(scale_order(scale))) return;
#pragma unroll 1
    for (int i = 0; i < n; ++i) codes[i] = (uint8_t)codes2(__fdiv_rn(value(i), scale), 0.f);
}

}  // namespace gf

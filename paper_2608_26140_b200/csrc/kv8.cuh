// Device helpers of the 8-bit cache: what a code and an exponent byte stand for, and conversions both ways.
//
// A (request, KV head, block of tokens) has one exponent byte e; its code c stands for c * 2^(e - 127).  e = 0: the block
// holds nothing and reads as zero whatever its codes.  Powers of two cost int8 at most one of its 8 bits against a free
// scale (e4m3 none: a floating-point code is as exact at any scale) and make everything else exact: x * 2^(127 - e) before
// the rounding, code * 2^(e - 127) in bf16, a code by itself in f16.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"

namespace acache {

constexpr int kKv8E4m3 = 0, kKv8Int8 = 1;
constexpr int kKv8MinExp = 16;      // lowest exponent of a block that holds something: its smallest code is a normal number in bf16
// A block's largest value lands in [2^top, 2^(top + 1)) scales.  int8: 64 to 127 (127.5 saturates, half a step like any
// other rounding).  e4m3: 128 to 256, so that nothing saturates; the codes above, up to 448, would give no bit.
template <int FMT>
__host__ __device__ constexpr int kv8_top() { return FMT == kKv8Int8 ? 6 : 7; }

// 2^(e - 127) for e in 1 .. 254, 0 for e = 0 (and below: a factor too small to matter)
__device__ __forceinline__ float kv8_scale(int e) { return e > 0 ? __int_as_float(e << 23) : 0.f; }

// ---- codes to f16 (exact) ---------------------------------------------------------------
// 4 codes -> (codes 0, 1), (codes 2, 3)
template <int FMT>
__device__ __forceinline__ void kv8_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    if constexpr (FMT == kKv8Int8) {
        // the byte as the low bits of 1024 + (code + 128), then minus 1152
        const uint32_t u = w ^ 0x80808080u;
        const uint32_t l = __byte_perm(u, 0x64646464u, 0x4140), h = __byte_perm(u, 0x64646464u, 0x4342);
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(l), "r"(0x64806480u));
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(h), "r"(0x64806480u));
    } else {
        asm("{\n\t.reg .b16 a, b;\n\t"
            "mov.b32 {a, b}, %2;\n\t"
            "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
            "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
            : "=r"(lo), "=r"(hi)
            : "r"(w));
    }
}

__device__ __forceinline__ float2 f16x2_to_f32(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }

// ---- values (in scales) to codes --------------------------------------------------------
// 4 finite values -> 4 codes; int8 saturates, e4m3 values stay below 256
template <int FMT>
__device__ __forceinline__ uint32_t kv8_round(float a, float b, float c, float d) {
    if constexpr (FMT == kKv8Int8) {
        // clamped, then rounded to the nearest even whole number by the addition of 1.5 * 2^23: the low byte is the code
        auto r = [](float x) { return __float_as_uint(fminf(fmaxf(x, -127.f), 127.f) + 12582912.f); };
        return __byte_perm(__byte_perm(r(a), r(b), 0x0040), __byte_perm(r(c), r(d), 0x0040), 0x5410);
    } else {
        uint32_t w;
        asm("{\n\t.reg .b16 a, b;\n\t"
            "cvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\t"
            "cvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n\t"
            "mov.b32 %0, {a, b};\n\t}"
            : "=r"(w)
            : "f"(a), "f"(b), "f"(c), "f"(d));
        return w;
    }
}
// 4 bf16 values times a power of two; int8: multiplied (exactly, but for values too small to matter) and clamped in pairs
template <int FMT>
__device__ __forceinline__ uint32_t kv8_round_bf16(uint32_t ab, uint32_t cd, float pow2) {
    if constexpr (FMT == kKv8Int8) {
        auto pair = [](uint32_t x, uint32_t s) {
            uint32_t y;
            asm("{\n\t.reg .b32 t;\n\t"
                "mul.rn.bf16x2 t, %1, %2;\n\t"
                "min.bf16x2 t, t, %3;\n\t"
                "max.bf16x2 %0, t, %4;\n\t}"
                : "=r"(y) : "r"(x), "r"(s), "r"(0x42FE42FEu), "r"(0xC2FEC2FEu));          // 127, -127
            return y;
        };
        auto r = [](float x) { return __float_as_uint(x + 12582912.f); };
        const uint32_t half = __float_as_uint(pow2) >> 16, s = half | half << 16, y = pair(ab, s), z = pair(cd, s);
        return __byte_perm(__byte_perm(r(bf16_lo(y)), r(bf16_hi(y)), 0x0040), __byte_perm(r(bf16_lo(z)), r(bf16_hi(z)), 0x0040), 0x5410);
    } else {
        return kv8_round<FMT>(bf16_lo(ab) * pow2, bf16_hi(ab) * pow2, bf16_lo(cd) * pow2, bf16_hi(cd) * pow2);
    }
}
// The same for values that need care: not finite (int8: NaN is 0, an infinity the largest code; e4m3: both are NaN), or of
// the block at the top of bf16's range, whose largest values would round past it (limit: the largest code to be used).
template <int FMT>
__device__ __forceinline__ uint32_t kv8_round_careful(float a, float b, float c, float d, float limit) {
    auto mend = [limit](float x) {
        if constexpr (FMT == kKv8Int8) return x != x ? 0.f : x;
        if (!(fabsf(x) < INFINITY)) return __int_as_float(0x7FC00000);
        return fminf(fmaxf(x, -limit), limit);
    };
    return kv8_round<FMT>(mend(a), mend(b), mend(c), mend(d));
}

// 32 bytes at a time: whole sectors of rows that lie apart.  whole: p is a multiple of 32 (callers guarantee 16)
__device__ __forceinline__ bool on_sector(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31u) == 0; }
__device__ __forceinline__ void st_global32(void* p, const uint32_t (&v)[8], bool whole) {
    if (!whole) {
        static_cast<uint4*>(p)[0] = make_uint4(v[0], v[1], v[2], v[3]);
        static_cast<uint4*>(p)[1] = make_uint4(v[4], v[5], v[6], v[7]);
        return;
    }
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]),
                 "r"(v[6]), "r"(v[7])
                 : "memory");
}

// ---- what the attention kernels share ----------------------------------------------------
// log2 units.  p is f16, normal from 2^-14 to 2^16: a new reference lies kStart below the largest logit, whose p is then 2^kStart, and moves
// when one passes it by kRaise.  So the largest p of a row is between 2^8 and 2^16, keys 2^-22 below it keep 11 bits and what is lost of any
// other is at most 2^-33 of the largest: thousands of keys 16 nats below a first one that says little still give their sum to 2^-10.
// (Logits here are y, which hold the scales of the values: p is what softmax and scale make together.)
// The price is that references move: one 4 above the largest logit moved 0.04 to 0.14 times a warp, this one 2.3 to 3 times.
constexpr float kRaise = 15.9f, kStart = 8.f;
constexpr int kFarApart = 100;                       // most by which E0 is above an ev
// A key's weight in the denominator, 2^(E0 - ev), times 2^-kWeightBias: 2^20 keys of the largest p and the largest weight come to 2^104
// (without it 2^136, past fp32), one key of p = 2^8 and the smallest weight to 2^-24.
constexpr int kWeightBias = 32;
__device__ __forceinline__ float kv8_weight(int behind) { return kv8_scale(127 - kWeightBias + min(behind, kFarApart)); }
// 2^(E0 - 127 - kWeightBias), exact down to the lowest exponent (2^-143, not a normal number): what sums over denominators are multiplied by.
// By itself, after the division: 1 / l times it may be smaller than any number, or larger.
__device__ __forceinline__ float kv8_unbias(int e0) { return kv8_scale(e0) * (1.f / 4294967296.f); }

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// of another CTA of the cluster
__device__ __forceinline__ float ld_peer(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_peer4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
// Results over several sets of keys, each with the log2 of its denominator, put together.
struct Sum {
    float mx = -INFINITY, den = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    __device__ __forceinline__ void add(float x, const float4& w) {
        if (x == -INFINITY) return;                              // no keys
        const float m = fmaxf(mx, x);                            // (a NaN comes through by fp)
        const float fo = mx == -INFINITY ? 0.f : ex2(mx - m), fp = ex2(x - m);
        mx = m;
        den = fmaf(den, fo, fp);
        v.x = fmaf(v.x, fo, fp * w.x); v.y = fmaf(v.y, fo, fp * w.y); v.z = fmaf(v.z, fo, fp * w.z); v.w = fmaf(v.w, fo, fp * w.w);
    }
    __device__ __forceinline__ float4 mean() const {
        const float i = den == 0.f ? 0.f : 1.f / den;
        return make_float4(v.x * i, v.y * i, v.z * i, v.w * i);
    }
    __device__ __forceinline__ float lse2() const { return den == 0.f ? -INFINITY : mx + log2f(den); }
};

}  // namespace acache

// Rows of logits as lm_score.hip and lm_sample.hip read them: the order of classes, a lane's classes of a chunk, values that so many lanes reach.
#pragma once
#include "lm_device.h"

namespace mt {
namespace {

constexpr float kNone = -__builtin_inff();

// Order of classes: larger logit first, then lower number; as one integer, larger in front.  0 is no class.
__device__ __forceinline__ uint64_t order_key(float x, uint32_t c)
{
    uint32_t b = __builtin_bit_cast(uint32_t, x == 0.0f ? 0.0f : x);      // (both zeros are equal)
    b = b & 0x80000000u ? ~b : b | 0x80000000u;
    return (uint64_t)b << 32 | (0xffffffffu - c);
}
__device__ __forceinline__ float key_logit(uint64_t key)
{
    const uint32_t b = (uint32_t)(key >> 32);
    return __builtin_bit_cast(float, b & 0x80000000u ? b ^ 0x80000000u : ~b);
}
__device__ __forceinline__ int32_t key_class(uint64_t key) { return (int32_t)(0xffffffffu - (uint32_t)key); }

// A value that at least n of the lanes' values reach, and not many more; -infinity if there are not so many.
__device__ __forceinline__ float bar_of(float v, uint32_t n)
{
    // between the smallest and the largest, over values ordered as integers, an eighth at a time: three rounds of seven comparisons that wait for nothing
    // between them (bit by bit, sixteen that each wait for a count, took three times as long)
    uint32_t b = __builtin_bit_cast(uint32_t, v);
    b = v > kNone ? (b & 0x80000000u ? ~b : b | 0x80000000u) : 0;
    if ((uint32_t)__popcll(__ballot(b != 0)) < n) return kNone;
    uint32_t lo = ~wave_fold(b ? ~b : 0u, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
    uint32_t span = wave_fold(b, [](uint32_t p, uint32_t q) { return p > q ? p : q; }) - lo;
#pragma nounroll
    for (int round = 0; round < 3; ++round) {
        const uint32_t step = span / 8 + 1;
        uint32_t eighths = 0;
#pragma unroll
        for (uint32_t i = 1; i < 8; ++i) eighths += (uint32_t)__popcll(__ballot(b >= lo + i * step)) >= n;
        lo += eighths * step;
        span = step;
    }
    return __builtin_bit_cast(float, lo & 0x80000000u ? lo ^ 0x80000000u : ~lo);
}

// A lane's classes of a chunk as they come from memory: vectors of 16 bytes, 64 of them side by side.
template <typename T, uint32_t VECS> struct Raw {
    static constexpr uint32_t kVec = 16 / sizeof(T), kVecs = VECS, kPer = kVec * kVecs, kChunk = 64 * kPer;      // ... a lane's and a wave's classes at a time
    u32x4 v[kVecs];
    uint32_t bits[kVecs];

    static __device__ __forceinline__ uint32_t first(uint32_t base, uint32_t i, uint32_t lane) { return base + (i * 64 + lane) * kVec; }

    template <bool MASK>
    __device__ __forceinline__ void load(const T* x, const uint32_t* allowed, uint32_t base, uint32_t lane, uint32_t classes)
    {
        if (base + kChunk <= classes) {
#pragma unroll
            for (uint32_t i = 0; i < kVecs; ++i) v[i] = *(const typename Any<T>::vec16*)(x + first(base, i, lane));
        } else {
#pragma unroll
            for (uint32_t i = 0; i < kVecs; ++i) {
                const uint32_t c = first(base, i, lane);
                u32x4 w{0, 0, 0, 0};
                if (c + kVec <= classes) w = *(const typename Any<T>::vec16*)(x + c);
                else if (c < classes) {
#pragma unroll
                    for (uint32_t e = 0; e < kVec; ++e)
                        if (c + e < classes) {
                            if constexpr (sizeof(T) == 2) w[e / 2] |= (uint32_t)((const uint16_t*)x)[c + e] << (16 * (e % 2));
                            else w[e] = ((const uint32_t*)x)[c + e];
                        }
                }
                v[i] = w;
            }
        }
        if constexpr (MASK) {
#pragma unroll
            for (uint32_t i = 0; i < kVecs; ++i) {
                const uint32_t c = first(base, i, lane);
                bits[i] = c < classes ? allowed[c >> 5] >> (c & 31) : 0;
            }
        }
    }

    template <bool MASK>
    __device__ __forceinline__ void logits(float (&x)[kPer], uint32_t base, uint32_t lane, uint32_t n) const
    {
#pragma unroll
        for (uint32_t i = 0; i < kVecs; ++i) {
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) { x[8 * i + 2 * e] = bf16_lo(v[i][e]); x[8 * i + 2 * e + 1] = bf16_hi(v[i][e]); }
            } else {
                const f32x4 f = __builtin_bit_cast(f32x4, v[i]);
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) x[4 * i + e] = f[e];
            }
            if constexpr (MASK) {
#pragma unroll
                for (uint32_t e = 0; e < kVec; ++e) if (!((bits[i] >> e) & 1)) x[kVec * i + e] = kNone;
            }
        }
        if (base + kChunk > n) {
#pragma unroll
            for (uint32_t i = 0; i < kVecs; ++i)
#pragma unroll
                for (uint32_t e = 0; e < kVec; ++e) if (first(base, i, lane) + e >= n) x[kVec * i + e] = kNone;
        }
    }
};

}  // namespace
}  // namespace mt

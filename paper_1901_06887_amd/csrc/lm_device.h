// Device helpers shared by the operators behind language models' answers (lm_*.hip).
#pragma once
#include "lm_internal.h"
#include "mt_device.h"

namespace mt {

// A grid holds fewer than 2^32 threads: rows, of 1024 threads at most, that one launch takes.
constexpr uint32_t kRowsAtOnce = 1u << 21;
template <typename V> void move_rows(V*& p, uint64_t elements) { if (p) p += elements; }

// Loads and stores of 16 or 8 bytes at any element's address.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
template <typename T> struct Any;
template <> struct Any<uint8_t> { typedef u32x4 vec16 __attribute__((aligned(1))); typedef u32x2 vec8 __attribute__((aligned(1))); };
template <> struct Any<__bf16> { typedef u32x4 vec16 __attribute__((aligned(2))); typedef u32x2 vec8 __attribute__((aligned(2))); };
template <> struct Any<float> { typedef u32x4 vec16 __attribute__((aligned(4))); typedef u32x2 vec8 __attribute__((aligned(4))); };

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
// two fp32 to bf16 (nearest even), packed
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
}

// Eight consecutive elements as fp32, from any element's address.
__device__ __forceinline__ void load8(const __bf16* p, float (&v)[8])
{
    const u32x4 w = *(const Any<__bf16>::vec16*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_lo(w[i]); v[2 * i + 1] = bf16_hi(w[i]); }
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8])
{
    // (whole vectors: the compiler takes element 0 for every element of one that is cast by elements)
    const f32x4 a = __builtin_bit_cast(f32x4, *(const Any<float>::vec16*)p), b = __builtin_bit_cast(f32x4, *(const Any<float>::vec16*)(p + 4));
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
// ... and back, STREAM: past the caches (nothing reads them before they are full of later rows).
template <bool STREAM> __device__ __forceinline__ void store8(__bf16* p, const float (&v)[8])
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    if constexpr (STREAM) __builtin_nontemporal_store(w, (Any<__bf16>::vec16*)p); else *(Any<__bf16>::vec16*)p = w;
}
template <bool STREAM> __device__ __forceinline__ void store8(float* p, const float (&v)[8])
{
    const f32x4 a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
    const u32x4 wa = __builtin_bit_cast(u32x4, a), wb = __builtin_bit_cast(u32x4, b);
    Any<float>::vec16 *qa = (Any<float>::vec16*)p, *qb = (Any<float>::vec16*)(p + 4);
    if constexpr (STREAM) { __builtin_nontemporal_store(wa, qa); __builtin_nontemporal_store(wb, qb); }
    else { *qa = wa; *qb = wb; }
}
// The first n (0 .. 8) of them, element by element; zeros behind.
template <typename T> __device__ __forceinline__ void load_some(const T* p, uint32_t n, float (&v)[8])
{
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) v[i] = i < n ? (float)p[i] : 0.0f;
}
template <typename T> __device__ __forceinline__ void store_some(T* p, uint32_t n, const float (&v)[8])
{
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) if (i < n) p[i] = (T)v[i];
}

// Between writes and reads of LDS by lanes of one wave.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
    __builtin_amdgcn_wave_barrier();
}

// Over the wave, in every lane, by data-parallel-primitive moves (no LDS traffic): shifts by 1, 2, 4, 8 inside rows of 16 lanes, lane 15
// of a row to the next, lane 31 to the upper half; the last lane has it all.
template <typename F> __device__ __forceinline__ uint32_t wave_fold(uint32_t v, F f)
{
#define MT_FOLD(ctrl, rows) v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xf, false))
    MT_FOLD(0x111, 0xf); MT_FOLD(0x112, 0xf); MT_FOLD(0x114, 0xf); MT_FOLD(0x118, 0xf); MT_FOLD(0x142, 0xa); MT_FOLD(0x143, 0xc);
#undef MT_FOLD
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
// (lanes without a source get 0, which adds nothing)
__device__ __forceinline__ float wave_total(float v)
{
    return __builtin_bit_cast(float, wave_fold(__builtin_bit_cast(uint32_t, v), [](uint32_t a, uint32_t b) {
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b)); }));
}
__device__ __forceinline__ uint32_t wave_total(uint32_t v) { return wave_fold(v, [](uint32_t a, uint32_t b) { return a + b; }); }
// The largest; NaN only if all are.  (As integers in the order of the values, above 0.)
__device__ __forceinline__ float wave_max(float v)
{
    uint32_t b = __builtin_bit_cast(uint32_t, v);
    b = v == v ? (b & 0x80000000u ? ~b : b | 0x80000000u) : 0;
    b = wave_fold(b, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
    return b == 0 ? __builtin_nanf("") : __builtin_bit_cast(float, b & 0x80000000u ? b ^ 0x80000000u : ~b);
}

}  // namespace mt

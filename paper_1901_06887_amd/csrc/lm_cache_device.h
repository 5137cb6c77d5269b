// Device helpers of the kernels on language models' caches: whose rows, where tokens lie.
#pragma once
#include "lm_cache.h"
#include "lm_device.h"

namespace mt {

inline uint32_t value_bytes(uint32_t dtype) { return dtype == MT_F32 ? 4 : dtype == MT_BF16 ? 2 : 1; }

// Batch entry b: its sequence, and rows first .. last - 1 of the call's; row r is token length - (after - r).  (Rows are below 2^31, so nothing here leaves 32 bits.)
struct SeqRows {
    int32_t seq;                 // -1: none
    int32_t length, first, last, after;
    // tokens up to row `first + j` and with it; 0 or less: it stands in front of the sequence
    __device__ __forceinline__ int32_t upto(int32_t j) const { return length - (after - (first + j)) + 1; }
};
__device__ __forceinline__ SeqRows seq_rows(const mt_kv_cache& c, const mt_kv_batch& b, uint32_t i)
{
    SeqRows r;
    const int32_t seq = b.seqs ? b.seqs[i] : (int32_t)i;
    const int32_t f0 = b.first_row ? b.first_row[i] : (int32_t)i;
    r.after = b.first_row ? b.first_row[i + 1] : (int32_t)i + 1;
    const bool there = (uint32_t)seq < c.seqs;
    r.seq = there ? seq : -1;
    r.length = there ? max(c.lengths[seq], 0) : 0;
    r.first = max(f0, 0);
    r.last = max(min(r.after, (int32_t)b.rows), r.first);         // (whatever first_row holds: last - first fits)
    return r;
}

// Page of a token of sequence `seq`; -1 where it has none.
__device__ __forceinline__ int32_t page_of(const mt_kv_cache& c, int32_t seq, int32_t token)
{
    const uint32_t i = (uint32_t)token / c.page_tokens;
    if (token < 0 || i >= c.table_width) return -1;
    const int32_t p = c.table[(uint64_t)seq * c.table_stride + i];
    return (uint32_t)p < c.n_pages ? p : -1;
}

// The scale of elements of which `most` is the largest magnitude, as e8m0: the least power of two at which it is no more than 448.  (448 is 1.75 * 2^8.)
__device__ __forceinline__ uint32_t scale_for(float most)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, most);
    if (!(most < __builtin_inff())) return 255;
    if (b == 0) return 127;
    const int e = (int)(b >> 23) - 135 + ((b & 0x7fffffu) > 0x600000u);
    return (uint32_t)(max(e, -126) + 127);
}
// The factor that brings elements to it: 2^-e; NaN for 255.
__device__ __forceinline__ float to_scale(uint32_t e8m0) { return e8m0 == 255 ? __builtin_nanf("") : __builtin_bit_cast(float, (254 - e8m0) << 23); }
__device__ __forceinline__ float of_scale(uint32_t e8m0)      // (0 is 2^-127, below the normal range)
{
    return e8m0 == 255 ? __builtin_nanf("") : e8m0 == 0 ? 5.877471754e-39f : __builtin_bit_cast(float, e8m0 << 23);
}
__device__ __forceinline__ uint32_t two_e4m3(float a, float b) { return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffffu; }
__device__ __forceinline__ float of_e4m3(uint32_t v) { return __builtin_amdgcn_cvt_f32_fp8(v, 0); }

}  // namespace mt

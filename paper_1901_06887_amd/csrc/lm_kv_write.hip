// mt_kv_write: new tokens' keys and values into their pages.
//
// A token's keys lie side by side, its values page_tokens apart.  In 8 bits a token and head share the power of two that its largest magnitude takes.
#include "lm_cache_device.h"

namespace mt {
namespace {

// A wave to a token and head.
template <typename T, typename C>
__global__ void __launch_bounds__(256) kv_write_kernel(KvWriteArgs w)
{
    const mt_kv_cache& c = w.c;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = c.head_dim;
    const SeqRows s = seq_rows(c, w.b, blockIdx.x);
    if (s.seq < 0) return;
    for (uint32_t j = blockIdx.y; (int32_t)j < s.last - s.first; j += gridDim.y) {
        const int32_t token = s.upto((int32_t)j) - 1;
        const int64_t r = s.first + (int32_t)j;
        const int32_t page = page_of(c, s.seq, token);
        if (page < 0) continue;
        const uint32_t slot = (uint32_t)token % c.page_tokens;
        for (uint32_t h = wave; h < c.heads; h += 4) {
            const T* k = (const T*)w.a.k + r * w.a.k_stride + h * D;
            const T* v = (const T*)w.a.v + r * w.a.v_stride + h * D;
            const uint64_t at = w.a.layer * c.layer_stride + page * c.page_stride + (uint64_t)h * c.page_tokens * D;
            C *ko = (C*)c.k + at + slot * D, *vo = (C*)c.v + at + slot;
            if constexpr (sizeof(C) == 1) {
                float km = 0, vm = 0;
                bool odd_k = false, odd_v = false;
                for (uint32_t d = lane; d < D; d += 64) {
                    const float kd = (float)k[d], vd = (float)v[d];
                    odd_k |= kd != kd; odd_v |= vd != vd;
                    km = fmaxf(km, fabsf(kd)); vm = fmaxf(vm, fabsf(vd));
                }
                const uint32_t ke = __ballot(odd_k) ? 255 : scale_for(wave_max(km)), ve = __ballot(odd_v) ? 255 : scale_for(wave_max(vm));
                const float kf = to_scale(ke), vf = to_scale(ve);
                for (uint32_t d = lane; d < D; d += 64) {
                    const uint32_t both = two_e4m3((float)k[d] * kf, (float)v[d] * vf);
                    ko[d] = (uint8_t)both;
                    vo[(uint64_t)d * c.page_tokens] = (uint8_t)(both >> 8);
                }
                const uint64_t to = w.a.layer * c.scales_layer_stride + page * c.scales_page_stride + h * c.page_tokens + slot;
                if (lane == 0) { c.k_scales[to] = (uint8_t)ke; c.v_scales[to] = (uint8_t)ve; }
            } else {
                for (uint32_t d = lane; d < D; d += 64) {
                    ko[d] = k[d];
                    vo[(uint64_t)d * c.page_tokens] = v[d];
                }
            }
        }
    }
}

}  // namespace

hipError_t launch_kv_write(const KvWriteArgs& w, hipStream_t s)
{
    const dim3 grid(w.b.n_seqs, std::min(w.b.max_new, 4096u));
    const bool narrow = w.c.dtype == MT_KV8;
    if (w.a.dtype == MT_BF16) return launch(narrow ? kv_write_kernel<__bf16, uint8_t> : kv_write_kernel<__bf16, __bf16>, grid, 256, 0, s, w);
    return launch(narrow ? kv_write_kernel<float, uint8_t> : kv_write_kernel<float, float>, grid, 256, 0, s, w);
}

}  // namespace mt

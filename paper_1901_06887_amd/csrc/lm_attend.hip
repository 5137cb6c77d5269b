// mt_attend: new tokens attend to all of their sequence's tokens in a paged cache.
#include "lm_cache_device.h"

namespace mt {
namespace {

template <typename T> __device__ __forceinline__ float value_of(T x) { return (float)x; }
template <> __device__ __forceinline__ float value_of(uint8_t x) { return of_e4m3(x); }

// A workgroup to a row and query head; 256 tokens at a time, a thread to each, then a thread to each element of the output.
template <typename T, typename C>
__global__ void __launch_bounds__(256) attend_kernel(AttendArgs g)
{
    const mt_kv_cache& c = g.c;
    const mt_attend_args& a = g.a;
    __shared__ float p[256], folds[8], q[MT_KV_MAX_DIM];
    __shared__ int32_t pages[256];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, D = c.head_dim, PT = c.page_tokens;
    const uint32_t qh = blockIdx.y, h = qh / (a.q_heads / c.heads);
    const SeqRows s = seq_rows(c, g.b, blockIdx.x);
    for (int64_t r = s.first + blockIdx.z; r < s.last; r += gridDim.z) {
        const int64_t upto = s.length - (s.after - r) + 1;
        const int64_t begin = a.window ? max(upto - (int64_t)a.window, (int64_t)0) : 0, end = min(upto, (int64_t)c.table_width * PT);
        __syncthreads();
        if (tid < D) q[tid] = (float)((const T*)a.q)[r * a.q_stride + qh * D + tid];
        float m = -3e38f, l = 0, o = 0;
        for (int64_t t0 = begin; t0 < end; t0 += 256) {
            __syncthreads();
            const int64_t t = t0 + tid;
            const int32_t page = t < end ? page_of(c, s.seq, t) : -1;
            float x = -__builtin_inff();
            const uint64_t at = a.layer * c.layer_stride + page * c.page_stride + (uint64_t)h * PT * D, sc = a.layer * c.scales_layer_stride + page * c.scales_page_stride + h * PT;
            if (page >= 0) {
                const C* k = (const C*)c.k + at + (uint32_t)(t % PT) * D;
                float dot = 0;
                for (uint32_t d = 0; d < D; ++d) dot = fmaf(q[d], value_of(k[d]), dot);
                if constexpr (sizeof(C) == 1) dot *= of_scale(c.k_scales[sc + t % PT]);
                x = dot * a.scale;
            }
            pages[tid] = page;
            // (a NaN makes the sum NaN, not the maximum)
            const float most = wave_max(x == x ? x : -__builtin_inff());
            if (lane == 0) folds[wave] = most;
            __syncthreads();
            const float to = fmaxf(fmaxf(fmaxf(folds[0], folds[1]), fmaxf(folds[2], folds[3])), m), f = expf(m - to);
            const float e = page < 0 ? 0.0f : expf(x - to);
            p[tid] = e;
            const float total = wave_total(e);
            if (lane == 0) folds[4 + wave] = total;
            __syncthreads();
            l = l * f + (folds[4] + folds[5]) + (folds[6] + folds[7]);
            o *= f;
            m = to;
            if (tid < D)
                for (uint32_t i = 0; i < 256; ++i) {
                    if (pages[i] < 0) continue;
                    const uint32_t slot = (uint32_t)((t0 + i) % PT);
                    float v = value_of(((const C*)c.v)[a.layer * c.layer_stride + pages[i] * c.page_stride + ((uint64_t)h * D + tid) * PT + slot]);
                    if constexpr (sizeof(C) == 1) v *= of_scale(c.v_scales[a.layer * c.scales_layer_stride + pages[i] * c.scales_page_stride + h * PT + slot]);
                    o = fmaf(p[i], v, o);
                }
        }
        const bool none = l == 0.0f;
        if (tid < D) ((T*)a.out)[r * a.out_stride + qh * D + tid] = (T)(none ? 0.0f : o / l);
        if (tid == 0 && a.lse) a.lse[(uint64_t)r * a.q_heads + qh] = none ? -__builtin_inff() : m + logf(l);
    }
}

}  // namespace

uint64_t attend_scratch_bytes(const mt_kv_cache&, const mt_kv_batch&, uint32_t, uint32_t) { return 0; }

hipError_t launch_attend(const AttendArgs& g, hipStream_t s)
{
    const dim3 grid(g.b.n_seqs, g.a.q_heads, std::min(g.b.max_new, 64u));
    const bool narrow = g.c.dtype == MT_KV8;
    if (g.a.dtype == MT_BF16) return launch(narrow ? attend_kernel<__bf16, uint8_t> : attend_kernel<__bf16, __bf16>, grid, 256, 0, s, g);
    return launch(narrow ? attend_kernel<float, uint8_t> : attend_kernel<float, float>, grid, 256, 0, s, g);
}

}  // namespace mt

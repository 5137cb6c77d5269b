// mt_score: log probabilities and ranks of given classes, entropy and the best alternatives of rows of logits.
//
// With m the largest allowed logit, z = (x - m) / T, S = sum e^z and U = sum z e^z: log p = z - log S and the entropy is log S - U / S, a sum of two
// terms that are not negative.  (x - m) / 2 is what is worked with: x - m itself can leave fp32's range.
#include "lm_device.h"

namespace mt {
namespace {

constexpr float kNone = -__builtin_inff();

// A class's logit, -infinity where it is not allowed.
template <typename T>
__device__ __forceinline__ float logit(const T* x, const uint32_t* allowed, uint32_t c, uint32_t n)
{
    if (c >= n || (allowed && !((allowed[c >> 5] >> (c & 31)) & 1))) return kNone;
    return (float)x[c];
}

// Order of classes: larger logit first, then lower number; as one integer, larger in front.  0: no class.
__device__ __forceinline__ uint64_t order_key(float x, uint32_t c)
{
    if (x == kNone) return 0;
    uint32_t b = __builtin_bit_cast(uint32_t, x == 0.0f ? 0.0f : x);      // (both zeros are equal)
    b = b & 0x80000000u ? ~b : b | 0x80000000u;
    return (uint64_t)b << 32 | (0xffffffffu - c);
}

// Half of x - m: with finite x and m this is never out of range.
__device__ __forceinline__ float half_below(float x, float m) { return fmaf(0.5f, x, -0.5f * m); }
__device__ __forceinline__ float log_prob(float x, float m, float inv_t, float log_s) { return half_below(x, m) * inv_t * 2.0f - log_s; }

template <typename V, typename F>
__device__ __forceinline__ V over_workgroup(V v, V* lds, F f)
{
    for (int d = 1; d < 64; d *= 2) v = f(v, __shfl_xor(v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (uint32_t w = 1; w < blockDim.x / 64; ++w) v = f(v, lds[w]);
    return v;
}

// One workgroup to a row: its maximum, its sums, ranks, and the alternatives one after the other.
template <typename T>
__global__ void __launch_bounds__(256) score_kernel(ScoreArgs s)
{
    __shared__ float fl[4];
    __shared__ uint64_t kl[4];
    const mt_score_args& a = s.a;
    const uint64_t row = blockIdx.x;
    const T* x = (const T*)a.logits + row * a.row_stride;
    const uint32_t* allowed = a.allowed ? a.allowed + row * a.allowed_stride : nullptr;
    const uint32_t n = a.n_classes ? (uint32_t)min(max(a.n_classes[row], 0), (int32_t)a.classes) : a.classes;
    const auto larger = [](float p, float q) { return fmaxf(p, q); };
    const auto sum = [](float p, float q) { return p + q; };
    float m = kNone;
    uint32_t count = 0;
    for (uint32_t c = threadIdx.x; c < n; c += 256) { const float v = logit(x, allowed, c, n); m = fmaxf(m, v); count |= v != kNone; }
    m = over_workgroup(m, fl, larger);
    const bool some = over_workgroup(count, (uint32_t*)fl, [](uint32_t p, uint32_t q) { return p | q; }) != 0;      // (a NaN is no maximum)
    float S = 0.0f, U = 0.0f;
    if (some)
        for (uint32_t c = threadIdx.x; c < n; c += 256) {
            const float h = half_below(logit(x, allowed, c, n), m);
            const float e = __builtin_amdgcn_exp2f(h * s.exp2_scale);
            S += e; U = fmaf(fmaxf(h, -1e30f), e, U);
        }
    S = over_workgroup(S, fl, sum);
    U = over_workgroup(U, fl, sum);
    const bool lost = some && !(S < __builtin_inff());         // NaN or +infinity among the allowed
    const float log_s = logf(S);
    const float nan = __builtin_nanf("");
    if (threadIdx.x == 0 && a.entropy) a.entropy[row] = lost ? nan : some ? log_s - 2.0f * s.inv_t * (U / S) : 0.0f;
    for (uint32_t g = 0; g < a.n_given; ++g) {
        const int32_t c = a.given[row * a.n_given + g];
        const float at = c >= 0 ? logit(x, allowed, (uint32_t)c, n) : kNone;
        const bool there = at != kNone;
        if (a.given_ranks) {
            uint32_t in_front = 0;
            if (there && !lost)
                for (uint32_t d = threadIdx.x; d < n; d += 256) {
                    const float v = logit(x, allowed, d, n);
                    in_front += v > at || (v == at && d < (uint32_t)c);
                }
            in_front = over_workgroup(in_front, (uint32_t*)fl, [](uint32_t p, uint32_t q) { return p + q; });
            if (threadIdx.x == 0) a.given_ranks[row * a.n_given + g] = there && !lost ? (int32_t)in_front : -1;
        }
        if (threadIdx.x == 0 && a.given_logprobs) a.given_logprobs[row * a.n_given + g] = !there ? kNone : lost ? nan : log_prob(at, m, s.inv_t, log_s);
    }
    uint64_t below = ~0ull;
    for (uint32_t k = 0; k < a.top; ++k) {
        uint64_t best = 0;
        if (some && !lost)
            for (uint32_t c = threadIdx.x; c < n; c += 256) {
                const uint64_t key = order_key(logit(x, allowed, c, n), c);
                if (key < below && key > best) best = key;
            }
        best = over_workgroup(best, kl, [](uint64_t p, uint64_t q) { return p > q ? p : q; });
        below = best;
        if (threadIdx.x == 0) {
            const uint32_t c = 0xffffffffu - (uint32_t)best;
            if (a.top_ids) a.top_ids[row * a.top + k] = best ? (int32_t)c : -1;
            if (a.top_logprobs) a.top_logprobs[row * a.top + k] = best ? log_prob((float)x[c], m, s.inv_t, log_s) : lost ? nan : kNone;
        }
    }
}

}  // namespace

void score_split(uint32_t, uint32_t classes, uint32_t* parts, uint32_t* part_len) { *parts = 1; *part_len = classes; }
uint64_t score_scratch_bytes(uint32_t, uint32_t, uint32_t, uint32_t) { return 0; }

hipError_t launch_score(const ScoreArgs& a, hipStream_t s)
{
    if (a.a.dtype == MT_BF16) hipLaunchKernelGGL((score_kernel<__bf16>), dim3(a.a.rows), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((score_kernel<float>), dim3(a.a.rows), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace mt

// mt_sample: one class for every row of logits, drawn with the row's own settings.
//
// Weights are whole numbers, e^((x - max) / T) times a power of two, from exponentials in 64 bits; all sums of them are exact, whatever their order. What a row keeps is a front part of its classes in their
// order (falling logits, lower numbers first among equals): the last one kept is found digit by digit of the order's key, by counts for top_k and by weights for top_p.
#include "lm_cache_device.h"

namespace mt {
namespace {

constexpr float kNone = -__builtin_inff();
constexpr uint32_t kThreads = 1024, kWaves = kThreads / 64;

// Order of classes as one integer, larger in front; 0 is no class.
__device__ __forceinline__ uint64_t order_key(float x, uint32_t c)
{
    uint32_t b = __builtin_bit_cast(uint32_t, x == 0.0f ? 0.0f : x);      // (both zeros are equal)
    b = b & 0x80000000u ? ~b : b | 0x80000000u;
    return (uint64_t)b << 32 | (0xffffffffu - c);
}

// A row as its settings see it.
template <typename T> struct Row {
    const T* x;
    const uint32_t* allowed;
    uint32_t n;              // classes that there are
    double most, inv_t, unit;

    __device__ __forceinline__ float logit(uint32_t c) const
    {
        if (c >= n || (allowed && !((allowed[c >> 5] >> (c & 31)) & 1))) return kNone;
        return (float)x[c];
    }
    __device__ __forceinline__ double share(float v) const { return exp(((double)v - most) * inv_t); }
    __device__ __forceinline__ uint64_t weight(double share) const { return (uint64_t)rint(share * unit); }
};

struct Lds {
    uint64_t words[kWaves];
    uint64_t bins[256];
    uint64_t chosen, above;
};

template <typename V, typename F> __device__ __forceinline__ V fold_all(V v, uint64_t* lds, F f)
{
    for (int d = 32; d; d >>= 1) v = f(v, (V)__shfl_xor(v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = __builtin_bit_cast(uint64_t, v);
    __syncthreads();
    v = __builtin_bit_cast(V, lds[0]);
    for (uint32_t w = 1; w < kWaves; ++w) v = f(v, __builtin_bit_cast(V, lds[w]));
    __syncthreads();
    return v;
}
__device__ __forceinline__ uint64_t sum_all(uint64_t v, uint64_t* lds) { return fold_all<uint64_t>(v, lds, [](uint64_t a, uint64_t b) { return a + b; }); }

// The key at which the values of the classes in front of it and its own first reach `target`; amount(c, key) is a class's value.
template <typename F> __device__ uint64_t reach(uint32_t n, uint64_t target, Lds& t, F amount)
{
    uint64_t prefix = 0, before = 0;
    for (int shift = 56; shift >= 0; shift -= 8) {
        __syncthreads();
        if (threadIdx.x < 256) t.bins[threadIdx.x] = 0;
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < n; c += kThreads) {
            uint64_t key;
            const uint64_t v = amount(c, &key);
            if (v && (shift == 56 || key >> (shift + 8) == prefix)) atomicAdd((unsigned long long*)&t.bins[key >> shift & 255], (unsigned long long)v);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            int b = 255;
            uint64_t sum = before;
            while (b > 0 && sum + t.bins[b] < target) sum += t.bins[b--];
            t.chosen = (uint64_t)b; t.above = sum;
        }
        __syncthreads();
        prefix = prefix << 8 | t.chosen;
        before = t.above;
    }
    return prefix;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_kernel(SampleArgs s)
{
    __shared__ Lds t;
    const mt_sample_args& a = s.a;
    const uint32_t row = blockIdx.x, tid = threadIdx.x;
    const float temperature = a.temperature ? a.temperature[row] : 1.0f, uniform = a.uniform[row], top_p = a.top_p ? a.top_p[row] : 1.0f, min_p = a.min_p ? fminf(a.min_p[row], 1.0f) : 0.0f;
    const bool greedy = temperature < 1.17549435e-38f;
    const int32_t top_k = greedy ? 1 : a.top_k ? a.top_k[row] : 0;
    Row<T> x;
    x.x = (const T*)a.logits + row * a.row_stride;
    x.allowed = a.allowed ? a.allowed + row * a.allowed_stride : nullptr;
    x.n = a.n_classes ? (uint32_t)min(max(a.n_classes[row], 0), (int32_t)a.classes) : a.classes;
    x.inv_t = greedy ? 1.0 : 1.0 / (double)temperature;
    x.unit = (double)(1ull << s.bits);

    bool lost = !(temperature >= 0.0f) || uniform != uniform || top_p != top_p || (a.min_p && a.min_p[row] != a.min_p[row]);
    uint64_t best = 0;
    uint32_t odd = 0;
    for (uint32_t c = tid; c < x.n; c += kThreads) {
        const float v = x.logit(c);
        odd |= v != v || v == __builtin_inff();
        if (v > kNone) best = max(best, order_key(v, c));
    }
    best = fold_all<uint64_t>(best, t.words, [](uint64_t p, uint64_t q) { return p > q ? p : q; });
    odd = __syncthreads_or(odd);
    int32_t id = -1, kept = lost || odd ? -1 : 0;
    float logprob = lost || odd ? __builtin_nanf("") : kNone;
    if (best && !lost && !odd) {
        x.most = (double)(float)x.x[0xffffffffu - (uint32_t)best];
        uint64_t bar = 1;
        if (top_k > 0 && (uint32_t)top_k < x.n)
            bar = max(bar, reach(x.n, (uint64_t)top_k, t, [&](uint32_t c, uint64_t* key) -> uint64_t { const float v = x.logit(c); *key = order_key(v, c); return v > kNone; }));
        // (a class's weight and whether it is kept, so far)
        const auto weigh = [&](uint32_t c, uint64_t* key, uint64_t* weight) {
            const float v = x.logit(c);
            *key = order_key(v, c);
            if (!(v > kNone) || *key < bar) return false;
            const double share = x.share(v);
            *weight = x.weight(share);
            return share >= (double)min_p;
        };
        const auto amount = [&](uint32_t c, uint64_t* key) -> uint64_t { uint64_t w; return weigh(c, key, &w) ? w : 0; };
        if (top_p < 1.0f) {
            uint64_t sum = 0, key;
            for (uint32_t c = tid; c < x.n; c += kThreads) sum += amount(c, &key);
            sum = sum_all(sum, t.words);
            bar = max(bar, reach(x.n, (uint64_t)fmax(ceil((double)top_p * (double)sum), 1.0), t, amount));
        }
        uint64_t sum = 0, count = 0;
        int32_t last = -1;
        for (uint32_t c = tid; c < x.n; c += kThreads) {
            uint64_t key, w;
            if (weigh(c, &key, &w)) { sum += w; ++count; if (w) last = (int32_t)c; }
        }
        sum = sum_all(sum, t.words);
        kept = (int32_t)sum_all(count, t.words);
        last = (int32_t)fold_all<int64_t>(last, t.words, [](int64_t p, int64_t q) { return p > q ? p : q; });
        // the first class up to which there is more than `target`
        const double at = (double)uniform * (double)sum;
        const uint64_t target = at <= 0 ? 0 : at >= (double)sum ? sum : (uint64_t)at;
        uint64_t before = 0;
        id = last;
        for (uint32_t base = 0; base < x.n; base += kThreads) {
            uint64_t key;
            const uint64_t w = base + tid < x.n ? amount(base + tid, &key) : 0;
            uint64_t upto = w;
            for (int d = 1; d < 64; d <<= 1) { const uint64_t o = __shfl_up(upto, d); if ((tid & 63) >= (uint32_t)d) upto += o; }
            __syncthreads();
            if ((tid & 63) == 63) t.words[tid >> 6] = upto;
            if (tid == 0) t.chosen = ~0ull;
            __syncthreads();
            uint64_t all = 0;
            for (uint32_t v = 0; v < kWaves; ++v) { if (v < tid >> 6) upto += t.words[v]; all += t.words[v]; }
            if (w && before + upto > target && before + upto - w <= target) t.chosen = base + tid;
            __syncthreads();
            if (t.chosen != ~0ull) { id = (int32_t)t.chosen; break; }
            before += all;
            __syncthreads();
        }
        logprob = (float)(((double)(float)x.x[id] - x.most) * x.inv_t - log((double)sum / x.unit));
    }
    if (tid == 0) {
        if (a.ids) a.ids[row] = id;
        if (a.logprobs) a.logprobs[row] = logprob;
        if (a.kept) a.kept[row] = kept;
    }
}

}  // namespace

uint64_t sample_scratch_bytes(uint32_t, uint32_t) { return 0; }

hipError_t launch_sample(const SampleArgs& s, hipStream_t st)
{
    return launch(s.a.dtype == MT_BF16 ? sample_kernel<__bf16> : sample_kernel<float>, dim3(s.a.rows), kThreads, 0, st, s);
}

}  // namespace mt

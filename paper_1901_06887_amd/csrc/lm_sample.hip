// mt_sample: one class for every row of logits, drawn with the row's own settings.
//
// What a row keeps is a front part of its classes in their order (falling logits, lower numbers first among equals), so a row is settled by the last class that it keeps, its `bar`, and by how much weight
// stands in front of the class that a random number picks. Weights are 2^(c (x - x0)) in 64 bits (a polynomial of degree 8, 1.1e-12 of itself); sums are 64-bit ones in an order that does not depend on timing.
//
// A workgroup to a row, an equal share of its classes to every wave. The bar is found by what the settings ask for:
//   the first class alone (temperature 0, top_k 1, top_p 0): the largest logit, one pass
//   top_k: the lanes' largest first classes give a value that at least top_k classes reach; what reaches it goes into a list in LDS in the same pass. Where those are too many, or top_k is
//     large, numbers of classes per bin (of logits) say in a pass before which classes to list. The list is put in order and settles everything
//   top_p: weight per bin and wave in LDS in the first pass; a second one lists the bin that holds the bar. The weights of what is kept are then known for every wave's share
//   neither: sums for every wave's share
// The class is then looked for in the share that holds it, a few classes to a thread. Bins are laid by the lanes' largest first classes, so that neither a few very
// large logits nor many very small ones (masks of the type's lowest value) spoil them. A row for which a list does not suffice (thousands of classes in
// one bin, top_k of thousands) is settled digit by digit of the order's key: right, but sixteen and more passes.
//
// What bounds it, as measured: 1024 rows of 32768 fp32 classes with top_p take 88 us, 52 without (2.6 TB/s). The second is the 64-bit weights (some 45 vector instructions to a lane and class);
// with top_p the weights' pass with its bins is about half, the pass that lists, from the caches and memory, a quarter, and bins, list and shares the rest. One row is a chain of
// dependent steps: 15 us for 32768 classes with top_k, 37 for 64 masked bf16 rows of 65001 with top_k and top_p, where the list's pass is 10 and its order and sums the rest.
#include "lm_cache_device.h"
#include "lm_logits.h"

namespace mt {
namespace {

constexpr uint32_t kBins = 640;                   // (40 KiB of LDS to eight waves: three workgroups to a compute unit)
constexpr uint32_t kNobody = 0xffffffffu;

// A constant in scalar registers (the compiler would give every one a pair of vector registers).
__device__ __forceinline__ double scalar(double v) { asm("" : "+s"(v)); return v; }

// A row's weights: 2^(c (x - one)), 1 at `one`. (c x + b with a rounded b would be one instruction less; where logits are large that rounding alone is thousands.)
struct Weigh {
    double c, one;
    __device__ __forceinline__ Weigh(double per, float at) : c(per), one((double)at) {}
    __device__ __forceinline__ double exponent(float x) const { return ((double)x - one) * c; }
    __device__ __forceinline__ double operator()(float x) const
    {
        // 2^y = 2^n 2^f, n the nearest whole number (the low bits of y + 1.5 2^52), 2^f a polynomial; y of less than -1000, -infinity too, count as -1000
        const double y = fmax(exponent(x), -1000.0), t = y + 6755399441055744.0, f = y - (t - 6755399441055744.0);
        double p = fma(scalar(1.3344183484134179e-06), f, scalar(1.5314209223349525e-05));
        p = fma(p, f, scalar(0.0001540309828656179));
        p = fma(p, f, scalar(0.0013333434157560176));
        p = fma(p, f, scalar(0.009618129558838935));
        p = fma(p, f, scalar(0.05550410959228811));
        p = fma(p, f, scalar(0.2402265069474259));
        p = fma(p, f, scalar(0.6931471805412327));
        p = fma(p, f, 1.0);
        const uint64_t bits = __builtin_bit_cast(uint64_t, p);
        return __builtin_bit_cast(double, (uint64_t)((uint32_t)(bits >> 32) + ((uint32_t)__builtin_bit_cast(uint64_t, t) << 20)) << 32 | (uint32_t)bits);
    }
};

// What a workgroup of WAVES waves shares.
template <uint32_t WAVES> struct Lds {
    static constexpr uint32_t kWaves = WAVES, kThreads = 64 * WAVES;
    static constexpr uint32_t kCap = 500 * WAVES;                 // entries of the list
    static constexpr uint32_t kNotes = 500 * WAVES;               // lanes' classes of a chunk, by number
    union {
        double mass[kWaves][kBins];
        uint32_t count[kWaves][kBins];
        struct {
            uint64_t keys[kCap];
            union { uint16_t notes[kNotes]; double weights[kThreads]; uint32_t counts[kBins > kThreads ? kBins : kThreads]; };      // (weights of the first kThreads entries, once the notes have been read)
        } list;
        uint64_t digits[256];
    };
    uint64_t words[kWaves];
    double share[kWaves];                         // kept weight of every wave's eighth
    float bars[kWaves], spreads[kWaves];
    uint32_t noted, listed, found;
    uint64_t chosen, above;
};

// Inclusive sums over the wave's lanes by data-parallel-primitive moves; the last lane has the total.
template <typename V> __device__ __forceinline__ V wave_scan(V v)
{
    static_assert(sizeof(V) == 8, "");
    // (lanes without a source get 0)
#define MT_ADD(ctrl, rows)                                                                                                                                   \
    {                                                                                                                                                        \
        const uint64_t b = __builtin_bit_cast(uint64_t, v);                                                                                                  \
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, ctrl, rows, 0xf, false), hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), ctrl, rows, 0xf, false); \
        v += __builtin_bit_cast(V, (uint64_t)hi << 32 | lo);                                                                                                 \
    }
    MT_ADD(0x111, 0xf) MT_ADD(0x112, 0xf) MT_ADD(0x114, 0xf) MT_ADD(0x118, 0xf) MT_ADD(0x142, 0xa) MT_ADD(0x143, 0xc)
#undef MT_ADD
    return v;
}
template <typename V> __device__ __forceinline__ V wave_sum(V v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, wave_scan(v));
    return __builtin_bit_cast(V, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, 63) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63) << 32);
}
// Over the workgroup, the same in every thread.
template <typename V, typename L, typename F> __device__ __forceinline__ V fold_all(V v, L& t, F f)
{
    static_assert(sizeof(V) == 8, "");
#pragma unroll
    for (uint32_t d = 32; d; d >>= 1) v = f(v, (V)__shfl_xor(v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) t.words[threadIdx.x >> 6] = __builtin_bit_cast(uint64_t, v);
    __syncthreads();
    v = __builtin_bit_cast(V, t.words[0]);
#pragma unroll
    for (uint32_t w = 1; w < L::kWaves; ++w) v = f(v, __builtin_bit_cast(V, t.words[w]));
    return v;
}
template <typename V, typename L> __device__ __forceinline__ V sum_all(V v, L& t)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) t.words[threadIdx.x >> 6] = __builtin_bit_cast(uint64_t, v);
    __syncthreads();
    v = __builtin_bit_cast(V, t.words[0]);
#pragma unroll
    for (uint32_t w = 1; w < L::kWaves; ++w) v += __builtin_bit_cast(V, t.words[w]);
    return v;
}
// Exclusive sums over the workgroup's threads.
template <typename V, typename L> __device__ __forceinline__ V scan_all(V v, L& t, V* total)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const V upto = wave_scan(v);
    __syncthreads();
    if (lane == 63) t.words[wave] = __builtin_bit_cast(uint64_t, upto);
    __syncthreads();
    V before = 0, all = 0;
#pragma unroll
    for (uint32_t w = 0; w < L::kWaves; ++w) { const V o = __builtin_bit_cast(V, t.words[w]); if (w < wave) before += o; all += o; }
    *total = all;
    return before + (upto - v);
}

// Bins of logits, 0 in front; what is in none has kBins or more.
struct Bins {
    float top, per;
    __device__ __forceinline__ float place(float x) const { return (top - x) * per; }
};

// The least logit whose place is in front of `limit`. (Places fall as logits rise, roundings included: 64 candidates at a time, in the order of the values as integers.)
__device__ __forceinline__ float first_logit(const Bins& bins, float limit, uint32_t lane)
{
    uint32_t lo = 0x00800000u, span = 0xff800000u - lo;           // from the lowest finite value to infinity, which is in front of every limit
#pragma nounroll
    for (int round = 0; round < 6; ++round) {
        const uint32_t step = span / 64 + 1, b = lo + min((lane + 1) * step, span);
        const float x = __builtin_bit_cast(float, b & 0x80000000u ? b ^ 0x80000000u : ~b);
        const uint32_t behind = (uint32_t)__popcll(__ballot(!(bins.place(x) < limit)));
        lo += min(behind * step, span);
        span = min(step, span - min(behind * step, span));
    }
    const uint32_t b = lo + (bins.place(__builtin_bit_cast(float, lo & 0x80000000u ? lo ^ 0x80000000u : ~lo)) < limit ? 0 : 1);
    return __builtin_bit_cast(float, b & 0x80000000u ? b ^ 0x80000000u : ~b);
}

// The last class that is kept; everything in front of it is kept too.
struct Bar {
    float x;
    uint32_t c;
    __device__ __forceinline__ bool keeps(float v, uint32_t at) const { return v > x || (v == x && at <= c && v > kNone); }
};

// The least logit of a weight of `least` (0 .. 1) of that of `top`: where it should be, and its neighbours.
__device__ __forceinline__ float least_logit(float top, double c, double least, uint32_t lane)
{
    if (!(least > 0)) return kNone;
    const float near = (float)((double)top + log2(least) / c);
    if (!(near > -3.4e38f)) return kNone;         // (temperatures at which every logit weighs enough)
    uint32_t b = __builtin_bit_cast(uint32_t, near == 0.0f ? 0.0f : near);
    b = (b & 0x80000000u ? ~b : b | 0x80000000u) + lane - 32;
    const float x = __builtin_bit_cast(float, b & 0x80000000u ? b ^ 0x80000000u : ~b);
    const uint64_t enough = __ballot(x <= top && exp2(((double)x - (double)top) * c) >= least);
    return enough ? __builtin_bit_cast(float, __builtin_amdgcn_readlane((int)__builtin_bit_cast(uint32_t, x), __builtin_ctzll(enough))) : top;
}

template <typename T, bool MASK> struct Row {
    static constexpr uint32_t kVecs = sizeof(T) == 4 ? 4 : 2;
    using R = Raw<T, kVecs>;
    static constexpr uint32_t kPer = R::kPer, kChunk = R::kChunk;
    static constexpr bool kMask = MASK;
    const T* x;
    const uint32_t* allowed;
    uint32_t n, share;           // classes that there are; classes of a wave

    __device__ __forceinline__ float at(uint32_t c) const
    {
        if (c >= n || (MASK && !((allowed[c >> 5] >> (c & 31)) & 1))) return kNone;
        return (float)x[c];
    }
    static __device__ __forceinline__ uint32_t number(uint32_t base, int i, uint32_t lane) { return R::first(base, i / R::kVec, lane) + i % R::kVec; }
    // f(logits of a chunk, its first class) for a wave's chunks of classes base .. end - 1. DEEP: two chunks on their way, at twice the code
    template <bool DEEP, typename F> __device__ __forceinline__ void walk(uint32_t base, uint32_t end, uint32_t lane, F f) const
    {
        base = __builtin_amdgcn_readfirstlane(base);
        if (base >= end) return;
        asm volatile("" : "+s"(base));            // (or the addresses of every pass's first chunk wait in registers)
        constexpr uint32_t ahead = DEEP ? 2 * kChunk : kChunk;
        R one{}, two{};
        one.template load<MASK>(x, allowed, base, lane, end);
        if (DEEP && base + kChunk < end) two.template load<MASK>(x, allowed, base + kChunk, lane, end);
        while (true) {
            float v[kPer];
            one.template logits<MASK>(v, base, lane, end);
            if (base + ahead < end) one.template load<MASK>(x, allowed, base + ahead, lane, end);
            f(v, base);
            base += kChunk;
            if (base >= end) break;
            if constexpr (DEEP) {
                float u[kPer];
                two.template logits<MASK>(u, base, lane, end);
                if (base + ahead < end) two.template load<MASK>(x, allowed, base + ahead, lane, end);
                f(u, base);
                base += kChunk;
                if (base >= end) break;
            }
        }
    }
};

// The largest of a lane's logits; NaN if one is.
template <uint32_t PER> __device__ __forceinline__ float largest_of(const float (&v)[PER])
{
    float m = v[0];
#pragma unroll
    for (uint32_t i = 1; i < PER; ++i) m = __builtin_elementwise_maximum(m, v[i]);
    return m;
}

// What a pass sees of the largest logit: a lane's largest, and the first class of the chunk that it is in.
struct Most {
    float x = kNone;
    uint32_t base = 0;
    bool odd = false;            // a NaN
    __device__ __forceinline__ void look(float m, uint32_t at)
    {
        odd |= m != m;
        if (m > x) { x = m; base = at; }
    }
};

// The key at which the values of the classes in front of it and its own first reach `target`; amount(c, key) is a class's value. (Digit by digit: every digit is a pass over the row.)
template <typename L, typename F> __device__ __forceinline__ uint64_t reach(uint32_t n, uint64_t target, L& t, F amount)
{
    constexpr uint32_t kThreads = L::kThreads;
    uint64_t prefix = 0, before = 0;
#pragma nounroll
    for (int shift = 56; shift >= 0; shift -= 8) {
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < 256; i += kThreads) t.digits[i] = 0;
        __syncthreads();
#pragma nounroll
        for (uint32_t c = threadIdx.x; c < n; c += kThreads) {
            uint64_t key;
            const uint64_t v = amount(c, &key);
            if (v && (shift == 56 || key >> (shift + 8) == prefix)) atomicAdd((unsigned long long*)&t.digits[key >> shift & 255], (unsigned long long)v);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            int b = 255;
            uint64_t sum = before;
            while (b > 0 && sum + t.digits[b] < target) sum += t.digits[b--];
            t.chosen = (uint64_t)b; t.above = sum;
        }
        __syncthreads();
        prefix = prefix << 8 | t.chosen;
        before = t.above;
    }
    return prefix;
}

// The list's keys in falling order. Up to kThreads of them: what is in front of an entry is counted, an entry to one thread or more; more: a bitonic network whose comparisons all go one way, so that what lies behind the last
// entry can be taken for the smallest and never moves.
template <typename L> __device__ __forceinline__ void put_in_order(L& t, uint32_t n)
{
    constexpr uint32_t kThreads = L::kThreads;
    uint64_t* keys = t.list.keys;
    const uint32_t tid = threadIdx.x;
    if (n <= kThreads) {
        uint32_t* before = t.list.counts;
        const uint32_t wide = (n + 63) / 64 * 64, parts = kThreads / wide, each = ((n + parts - 1) / parts + 7) / 8 * 8, part = tid / wide, e = tid % wide;
        const uint64_t own = e < n ? keys[e] : 0;
        before[tid] = 0;
        if (tid < 8) keys[n + tid] = 0;           // (behind the last: there is room for kThreads and 8 more)
        __syncthreads();
        if (part < parts) {
            uint32_t some = 0;
            const uint32_t stop = min((part + 1) * each, n);
            for (uint32_t i = part * each; i < stop; i += 8)
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) some += keys[i + j] > own;
            if (e < n && some) atomicAdd(&before[e], some);
        }
        __syncthreads();
        const uint32_t to = before[tid];
        __syncthreads();
        if (tid < n) keys[to] = own;
        __syncthreads();
        return;
    }
    uint32_t all = 2 * kThreads;
    while (all < n) all *= 2;
    for (uint32_t k = 2; k <= all; k *= 2)
        for (uint32_t j = k / 2; j; j /= 2) {
            for (uint32_t p = tid; p < all / 2; p += kThreads) {
                const uint32_t lo = p / j * 2 * j + p % j, hi = j == k / 2 ? lo / k * k + (k - 1 - lo % k) : lo + j;
                if (hi < n) {
                    const uint64_t a = keys[lo], b = keys[hi];
                    if (a < b) { keys[lo] = b; keys[hi] = a; }
                }
            }
            __syncthreads();
        }
}

// A thread's entries of the list, side by side.
template <typename L> struct Own {
    uint32_t first, end;
    __device__ __forceinline__ explicit Own(uint32_t n)
    {
        const uint32_t each = ceil_div(n, L::kThreads);
        first = min(threadIdx.x * each, n);
        end = min(first + each, n);
    }
    // Their weights (0 for logits below `least`), which stay in the list as far as it has room for them, and the sum.
    __device__ __forceinline__ double weights(L& t, const Weigh& weigh, float least) const
    {
        double sum = 0;
#pragma nounroll
        for (uint32_t i = first; i < end; ++i) {
            const float x = key_logit(t.list.keys[i]);
            const double w = x >= least ? weigh(x) : 0.0;
            if (i < L::kThreads) t.list.weights[i] = w;
            sum += w;
        }
        return sum;
    }
    // How many of them are kept: those of weight in front of which there is less than `target` (the list's first always).
    __device__ __forceinline__ uint64_t kept(const L& t, const Weigh& weigh, float least, double at, double target) const
    {
        uint64_t n = 0;
#pragma nounroll
        for (uint32_t i = first; i < end; ++i) {
            const float x = key_logit(t.list.keys[i]);
            if (x < least || (i && !(at < target))) break;
            ++n;
            at += weigh(x);
        }
        return n;
    }
};

// A pass notes lanes that hold something for the list: the number of a lane's classes of a chunk among all such (at most 2^16, as there are 16 classes each). What doesn't fit is counted alone.
template <typename L> __device__ __forceinline__ void note(L& t, bool holds, uint32_t number, uint32_t lane)
{
    const uint64_t lanes = __ballot(holds);
    if (lanes == 0) return;
    uint32_t at = 0;
    if (lane == 0) at = atomicAdd(&t.noted, (uint32_t)__popcll(lanes));
    at = (uint32_t)__builtin_amdgcn_readfirstlane((int)at) + __builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0));
    if (holds && at < L::kNotes) t.list.notes[at] = (uint16_t)number;
}
// Behind it, those of the noted classes whose logits lie in from .. behind, `behind` left out, go into the list, a lane's classes to a thread. Their number stays in t.listed, also where they don't fit.
template <typename L, typename W> __device__ __forceinline__ void list_noted(L& t, const W& x, float from, float behind)
{
    constexpr uint32_t kPer = W::kPer;
    const uint32_t lane = threadIdx.x & 63, n = min(t.noted, L::kNotes);
    const bool all = t.noted <= L::kNotes;
    if (threadIdx.x == 0) t.listed = all ? 0 : L::kCap + 1;
    __syncthreads();
    for (uint32_t i = threadIdx.x; all && i < (n + 63) / 64 * 64; i += L::kThreads) {
        float v[kPer];
        const uint32_t number = i < n ? t.list.notes[i] : 0, first = i < n ? number / 64 * W::kChunk + number % 64 * W::R::kVec : x.n;
        typename W::R raw;
        raw.template load<W::kMask>(x.x, x.allowed, first, 0, x.n);
        raw.template logits<W::kMask>(v, first, 0, x.n);
        uint32_t mine = 0;
#pragma unroll
        for (uint32_t e = 0; e < kPer; ++e) mine |= v[e] >= from && v[e] < behind ? 1u << e : 0;
        const uint32_t own = (uint32_t)__popc(mine), upto = wave_inclusive_scan(own);
        uint32_t at = 0;
        if (lane == 63) at = atomicAdd(&t.listed, upto);
        at = (uint32_t)__builtin_amdgcn_readlane((int)at, 63) + upto - own;
#pragma unroll
        for (uint32_t e = 0; e < kPer; ++e)
            if (mine >> e & 1) {
                if (at < L::kCap) t.list.keys[at] = order_key(v[e], W::number(first, e, 0));
                ++at;
            }
    }
    __syncthreads();
}

// The list cut to those of its entries that can be among the first `want`, by numbers of entries per bin: between `least`, the smallest logit that can be there, and the largest. Leaves t.listed.
template <typename L> __device__ __forceinline__ void cut_list(L& t, float least, float top, uint32_t want)
{
    constexpr uint32_t kThreads = L::kThreads, kEach = (L::kCap + kThreads - 1) / kThreads, kOwnBins = (kBins + kThreads - 1) / kThreads;
    uint32_t* count = t.list.counts;
    const uint32_t n = t.listed, tid = threadIdx.x;
    const Bins bins{top, 0.999f * (float)kBins / (top - least)};
    uint64_t keys[kEach];
    for (uint32_t i = tid; i < kBins; i += kThreads) count[i] = 0;
    __syncthreads();
    const auto bin_of = [&](uint64_t key) { return (uint32_t)fminf(fmaxf(bins.place(key_logit(key)), 0.0f), (float)(kBins - 1)); };
#pragma unroll
    for (uint32_t e = 0; e < kEach; ++e) {
        keys[e] = tid + e * kThreads < n ? t.list.keys[tid + e * kThreads] : 0;
        if (keys[e]) atomicAdd(&count[bin_of(keys[e])], 1u);
    }
    if (tid == 0) { t.listed = 0; t.found = kBins; }
    __syncthreads();
    uint64_t sum = 0, all;
#pragma unroll
    for (uint32_t e = 0; e < kOwnBins; ++e) if (kOwnBins * tid + e < kBins) sum += count[kOwnBins * tid + e];
    uint64_t at = scan_all<uint64_t>(sum, t, &all);
#pragma unroll
    for (uint32_t e = 0; e < kOwnBins; ++e)
        if (kOwnBins * tid + e < kBins) {
            const uint32_t one = count[kOwnBins * tid + e];
            if (at < want && at + one >= want) t.found = kOwnBins * tid + e;
            at += one;
        }
    __syncthreads();
    const uint32_t last = t.found;
#pragma unroll
    for (uint32_t e = 0; e < kEach; ++e) {
        const bool stays = keys[e] && bin_of(keys[e]) <= last;
        const uint64_t lanes = __ballot(stays);
        uint32_t to = 0;
        if ((tid & 63) == 0 && lanes) to = atomicAdd(&t.listed, (uint32_t)__popcll(lanes));
        to = (uint32_t)__builtin_amdgcn_readfirstlane((int)to) + __builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0));
        if (stays) t.list.keys[to] = keys[e];
    }
    __syncthreads();
}

template <typename T, bool MASK, uint32_t WAVES>
__global__ void __launch_bounds__(64 * WAVES, WAVES == 16 ? 4 : MASK && sizeof(T) == 4 ? 5 : 6) sample_kernel(SampleArgs s)
{
    using L = Lds<WAVES>;
    constexpr uint32_t kWaves = WAVES, kThreads = 64 * WAVES, kCap = L::kCap, kOwnBins = (kBins + kThreads - 1) / kThreads;
    using W = Row<T, MASK>;
    constexpr uint32_t kPer = W::kPer, kChunk = W::kChunk;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    L& t = *(L*)lds;
    const mt_sample_args& a = s.a;
    const uint32_t row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float temperature = a.temperature ? a.temperature[row] : 1.0f, uniform = a.uniform[row], top_p = a.top_p ? a.top_p[row] : 1.0f, min_p = a.min_p ? a.min_p[row] : 0.0f;
    const uint32_t top_k = a.top_k ? (uint32_t)max(a.top_k[row], 0) : 0;
    W x;
    x.x = (const T*)a.logits + row * a.row_stride;
    x.allowed = MASK ? a.allowed + row * a.allowed_stride : nullptr;
    x.n = a.n_classes ? (uint32_t)min(max(a.n_classes[row], 0), (int32_t)a.classes) : a.classes;
    x.share = ceil_div(x.n, kWaves * kChunk) * kChunk;
    const uint32_t first = min(wave * x.share, x.n), end = min(first + x.share, x.n);

    const bool lost = !(temperature >= 0.0f) || uniform != uniform || top_p != top_p || min_p != min_p;
    const bool greedy = temperature < 1.17549435e-38f || top_k == 1 || top_p <= 0.0f;
    const double c = 1.4426950408889634 / (double)(greedy ? 1.0f : temperature);
    const double least = fmin((double)min_p, 1.0);

    // Outcome: nothing yet, or the row's class; in between the bar, the weights and each wave's share of them.
    int32_t id = -1, kept = 0;
    double logprob = kNone;
    bool settled = lost, odd = lost;
    Bar bar{kNone, kNobody};
    Weigh weigh(c, 0.0f);

    // What a pass over the whole row has seen: the largest logit, and whether the row has nothing to draw from.
    float top = kNone;
    const auto largest = [&](const Most& m) __attribute__((always_inline)) {
        odd = __syncthreads_or(m.odd);
        const float w = wave_max(m.x);            // (no lane's is NaN)
        if (lane == 0) t.bars[wave] = w;
        __syncthreads();
        top = t.bars[0];
#pragma unroll
        for (uint32_t v = 1; v < kWaves; ++v) top = fmaxf(top, t.bars[v]);
        __syncthreads();
        odd |= top == __builtin_inff();
        settled = odd || top == kNone;
    };
    // The lanes' largest classes of the waves' first chunks.
    const auto lane_largest = [&]() __attribute__((always_inline)) {
        float m = kNone;
        x.template walk<false>(first, min(first + kChunk, end), lane, [&](const float (&v)[kPer], uint32_t) {
#pragma unroll
            for (uint32_t i = 0; i < kPer; ++i) m = fmaxf(m, v[i]);
        });
        return m;
    };
    // Bins from them: of each wave's 64, the eighth and the eighth last in their order, some 1.4 standard deviations apart; the wave with the largest speaks for all. `lead`: the largest.
    const auto lay_bins = [&](float* lead) __attribute__((always_inline)) {
        const float m = lane_largest(), most = wave_max(m), hi = bar_of(m, 8), lo = bar_of(m, 56);
        __syncthreads();
        if (lane == 0) { t.bars[wave] = lo > kNone ? hi : kNone; t.spreads[wave] = hi - lo; t.share[wave] = (double)most; }
        __syncthreads();
        Bins b{0.0f, 16.0f};
        float at = kNone, lead_x = kNone;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) {
            lead_x = fmaxf(lead_x, (float)t.share[w]);
            if (t.bars[w] > at) { at = t.bars[w]; b.per = 128.0f / t.spreads[w]; }
        }
        if (!(b.per > 1e-30f && b.per < 1e30f)) b.per = 16.0f;
        b.top = (at > kNone ? at : lead_x > kNone && lead_x < 3e38f ? lead_x : 0.0f) + 192.0f / b.per;
        *lead = lead_x > kNone && lead_x < 3e38f ? lead_x : 0.0f;
        __syncthreads();
        return b;
    };
    enum { kPick, kShares, kDigits } next = kShares;      // what remains: look for the class; first sum each wave's share; first find the bar

    if (settled) {
    } else if (greedy) {
        Most m;
        x.template walk<true>(first, end, lane, [&](const float (&v)[kPer], uint32_t base) { m.look(largest_of(v), base); });
        largest(m);
        if (!settled) {
            uint32_t at = kNobody;
            if (m.x == top) {
#pragma unroll
                for (int i = kPer - 1; i >= 0; --i) {
                    const uint32_t j = W::number(m.base, i, lane);
                    if (j < end && x.at(j) == top) at = j;
                }
            }
            id = (int32_t)fold_all<int64_t>((int64_t)at, t, [](int64_t p, int64_t q) { return p < q ? p : q; });
            kept = 1; logprob = 0.0; settled = true;
        }
    } else if (top_k && top_k < x.n) {
        // a value that top_k classes of the first chunks reach, if they are few
        if (tid == 0) t.noted = 0;
        const float m = lane_largest();
        // (of waves with classes for at least half of their lanes each wave's share of top_k; or all of it in one wave)
        const uint32_t full = (uint32_t)__popcll(__ballot(m > kNone));
        __syncthreads();
        if (lane == 0) t.spreads[wave] = (float)full;
        __syncthreads();
        uint32_t waves = 0;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) waves += t.spreads[w] >= 32.0f;
        const uint32_t each = waves ? ceil_div(top_k, waves) : 64;
        const float mine = each <= 32 ? bar_of(m, each) : kNone;
        if (lane == 0) t.bars[wave] = full >= 32 ? mine : __builtin_inff();
        __syncthreads();
        float reached = __builtin_inff();
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) reached = fminf(reached, t.bars[w]);
        if (reached == __builtin_inff()) reached = kNone;
        __syncthreads();
        bool listed = false;
        Most most;
        const auto list_from = [&](float from) __attribute__((always_inline)) {
            x.template walk<true>(first, end, lane, [&](const float (&v)[kPer], uint32_t base) {
                const float m = largest_of(v);
                most.look(m, base);
                note(t, m >= from, base / kPer + lane, lane);
            });
            largest(most);
            list_noted(t, x, from, __builtin_inff());
            return t.listed <= kCap;
        };
        if (reached > kNone || x.n <= kCap) {
            reached = fmaxf(reached, -3.402823466e38f);
            listed = list_from(reached);
        }
        if (!listed && !settled) {
            // classes per bin, then all those of the bins that hold the first top_k
            float lead;
            const Bins bins = lay_bins(&lead);
            for (uint32_t i = tid; i < kWaves * kBins; i += kThreads) t.count[0][i] = 0;
            __syncthreads();
            most = Most{};
            x.template walk<false>(first, end, lane, [&](const float (&v)[kPer], uint32_t base) {
                most.look(largest_of(v), base);
#pragma unroll
                for (uint32_t i = 0; i < kPer; ++i) {
                    const float p = bins.place(v[i]);
                    if (p < (float)kBins) atomicAdd(&t.count[wave][(uint32_t)fmaxf(p, 0.0f)], 1u);
                }
            });
            largest(most);
            uint64_t mine[kOwnBins], sum = 0, all;
#pragma unroll
            for (uint32_t e = 0; e < kOwnBins; ++e) {
                mine[e] = 0;
                if (kOwnBins * tid + e < kBins)
#pragma unroll
                    for (uint32_t w = 0; w < kWaves; ++w) mine[e] += t.count[w][kOwnBins * tid + e];
                sum += mine[e];
            }
            uint64_t at = scan_all<uint64_t>(sum, t, &all);
            if (tid == 0) { t.found = kNobody; t.above = 0; t.noted = 0; }
            __syncthreads();
#pragma unroll
            for (uint32_t e = 0; e < kOwnBins; ++e) {
                if (at < top_k && at + mine[e] >= top_k) { t.found = kOwnBins * tid + e; t.above = at + mine[e]; }
                at += mine[e];
            }
            __syncthreads();
            const uint32_t last = t.found;
            if (!settled && last != kNobody && t.above <= kCap) {
                reached = first_logit(bins, (float)(last + 1), lane);
                listed = list_from(reached);
            }
        }
        if (!settled && listed) {
            // in order: top_k by number, min_p by weight, top_p by sums
            // (one row of 131072 bf16 classes, first 50: 25.4 us without the cut, 20.3 with it; 64 masked rows of 65001: 42.5, 37.0; lists of a few hundred are as fast either way)
            if (t.listed > 400 && 2 * top_k <= t.listed && reached < top) cut_list(t, reached, top, top_k);
            const uint32_t n = t.listed, most_kept = min(n, top_k);
            put_in_order(t, n);
            weigh = Weigh(c, top);
            const Own<L> own(most_kept);
            const float least_x = least_logit(top, c, least, lane);
            double total, at = scan_all<double>(own.weights(t, weigh, least_x), t, &total);
            kept = max((int32_t)sum_all<uint64_t>(own.kept(t, weigh, least_x, at, top_p < 1.0f ? (double)top_p * total : __builtin_inf()), t), 1);
            const uint64_t last = t.list.keys[kept - 1];
            bar = Bar{key_logit(last), (uint32_t)key_class(last)};
            if ((uint32_t)kept <= kThreads) {
                // every kept class by its number: what stands in front of it
                const bool any = tid < (uint32_t)kept;
                const double own_w = any ? t.list.weights[tid] : 0.0, every = sum_all<double>(own_w, t);
                const uint32_t mine_c = any ? (uint32_t)key_class(t.list.keys[tid]) : 0;
                if (tid == 0) t.found = kNobody;
                __syncthreads();
                if (wave * 64 < (uint32_t)kept) {
                    double front = 0;
#pragma unroll 4
                    for (uint32_t i = 0; i < (uint32_t)kept; ++i) front += (uint32_t)key_class(t.list.keys[i]) <= mine_c ? t.list.weights[i] : 0.0;
                    if (any && own_w > 0 && front > (double)uniform * every) atomicMin(&t.found, mine_c);
                }
                __syncthreads();
                uint32_t pick = t.found;
                if (pick == kNobody) pick = (uint32_t)fold_all<int64_t>(any && own_w > 0 ? (int64_t)mine_c : -1, t, [](int64_t p, int64_t q) { return p > q ? p : q; });
                id = (int32_t)pick;
                logprob = weigh.exponent((float)x.x[pick]) * 0.6931471805599453 - log(every);
                settled = true;
            }
        } else if (!settled) next = kDigits;
    } else {
        if (least > 0) {
            Most m;
            x.template walk<true>(first, end, lane, [&](const float (&v)[kPer], uint32_t base) { m.look(largest_of(v), base); });
            largest(m);
            if (!settled) bar.x = least_logit(top, c, least, lane);
        }
        if (settled) {
        } else if (top_p < 1.0f) {
            float lead;
            Bins bins = lay_bins(&lead);
            // They reach 2.5 standard deviations below the middle of a bell-shaped row, whose weights have their own middle sigma c ln 2 deviations higher: where less than what lies below (e^(-z^2/2) is
            // several times that) is to be left out, bins of twice the width, down to 10. One row that is settled digit by digit instead takes 1024 rows of 32768 classes from 87 to 156 us.
            const float z = 2.5f + (float)(c * 0.6931471805599453) * (128.0f / 1.4f) / bins.per;
            if (exp2f(-0.72f * z * z) > 1.0f - top_p) bins.per *= 0.5f;
            if (least > 0) lead = top;
            double rest = 0;
            for (int round = 0; round < 2; ++round) {
                weigh = Weigh(c, lead);
                for (uint32_t i = tid; i < kWaves * kBins; i += kThreads) t.mass[0][i] = 0;
                __syncthreads();
                Most m;
                rest = 0;
                x.template walk<false>(first, end, lane, [&](const float (&v)[kPer], uint32_t base) {
                    m.look(largest_of(v), base);
#pragma unroll
                    for (uint32_t i = 0; i < kPer; ++i) {
                        if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);      // (four at a time: registers)
                        const double w = weigh(v[i]);
                        const float p = bins.place(v[i]);
                        if (v[i] >= bar.x) {
                            if (p < (float)kBins) __hip_atomic_fetch_add(&t.mass[wave][(uint32_t)fmaxf(p, 0.0f)], w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                            else if (v[i] > kNone) rest += w;
                        }
                    }
                });
                largest(m);
                if (settled || fabs(weigh.exponent(top)) <= 900.0) break;
                lead = top;          // (weights of another logit's scale: once more)
            }
            if (!settled) {
                double mine[kOwnBins], sum = 0, in_bins, front = 0;
#pragma unroll
                for (uint32_t e = 0; e < kOwnBins; ++e) {
                    mine[e] = 0;
                    if (kOwnBins * tid + e < kBins)
#pragma unroll
                        for (uint32_t w = 0; w < kWaves; ++w) mine[e] += t.mass[w][kOwnBins * tid + e];
                    sum += mine[e];
                }
                double upto = scan_all<double>(sum, t, &in_bins);
                const double target = (double)top_p * (in_bins + sum_all<double>(rest, t));
                if (tid == 0) { t.found = kNobody; t.noted = 0; }
                __syncthreads();
                uint32_t here = kNobody;
#pragma unroll
                for (uint32_t e = 0; e < kOwnBins; ++e) {
                    if (here == kNobody && kOwnBins * tid + e < kBins && upto + mine[e] >= target) { here = kOwnBins * tid + e; front = upto; }
                    upto += mine[e];
                }
                if (here < kBins) atomicMin(&t.found, here);
                __syncthreads();
                const uint32_t in = t.found;
                if (in == kNobody) next = kDigits;
                else {
                    if (here == in) t.above = __builtin_bit_cast(uint64_t, front);
                    double above_mine = 0;                // of this wave's share
                    for (uint32_t i = lane; i < in; i += 64) above_mine += t.mass[wave][i];
                    above_mine = wave_sum(above_mine);
                    __syncthreads();
                    const double above = __builtin_bit_cast(double, t.above);
                    const float from = fmaxf(first_logit(bins, (float)(in + 1), lane), bar.x), behind = in ? first_logit(bins, (float)in, lane) : __builtin_inff();
                    uint32_t n_above = 0;                 // of this lane's classes
                    x.template walk<true>(first, end, lane, [&](const float (&v)[kPer], uint32_t base) {
                        uint32_t fronts = 0, all = 0;
#pragma unroll
                        for (uint32_t i = 0; i < kPer; ++i) { fronts += v[i] >= behind; all += v[i] >= from; }
                        n_above += fronts;
                        note(t, all != fronts, base / kPer + lane, lane);
                    });
                    const uint64_t all_above = sum_all<uint64_t>(n_above, t);
                    list_noted(t, x, from, behind);
                    const uint32_t n = t.listed;
                    if (n > kCap || n == 0) next = kDigits;
                    else {
                        put_in_order(t, n);
                        const Own<L> own(n);
                        double total, at = above + scan_all<double>(own.weights(t, weigh, kNone), t, &total);
                        const uint32_t in_list = max((uint32_t)sum_all<uint64_t>(own.kept(t, weigh, kNone, at, target), t), 1u);
                        kept = (int32_t)(all_above + in_list);
                        const uint64_t last = t.list.keys[in_list - 1];
                        bar = Bar{key_logit(last), (uint32_t)key_class(last)};
                        double more = 0;                  // the list's part of this wave's share
                        for (uint32_t i = lane; i < in_list; i += 64) {
                            const uint32_t j = (uint32_t)key_class(t.list.keys[i]);
                            if (j >= first && j < end) more += i < kThreads ? t.list.weights[i] : weigh(key_logit(t.list.keys[i]));
                        }
                        more = wave_sum(more);
                        if (lane == 0) t.share[wave] = above_mine + more;
                        __syncthreads();
                        next = kPick;
                    }
                }
            }
        } else {
            // all of them, or all from a weight on: sums for every wave's share
            float lead = top;
            if (!(least > 0)) {
                const float m = wave_max(lane_largest());
                if (lane == 0) t.bars[wave] = m;
                __syncthreads();
#pragma unroll
                for (uint32_t w = 0; w < kWaves; ++w) lead = fmaxf(lead, t.bars[w]);
                __syncthreads();
                if (!(lead > kNone && lead < 3e38f)) lead = 0;
            }
            for (int round = 0; round < 2; ++round) {
                weigh = Weigh(c, lead);
                Most m;
                double sum = 0;
                uint64_t n = 0;
                x.template walk<false>(first, end, lane, [&](const float (&v)[kPer], uint32_t base) {
                    m.look(largest_of(v), base);
#pragma unroll
                    for (uint32_t i = 0; i < kPer; ++i) {
                        if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                        const double w = weigh(v[i]);
                        const bool counts = v[i] > kNone && v[i] >= bar.x;
                        n += (uint32_t)__popcll(__ballot(counts));
                        sum += counts ? w : 0.0;
                    }
                });
                largest(m);
                if (settled) break;
                if (round == 0 && fabs(weigh.exponent(top)) > 900.0) { lead = top; continue; }       // (weights of another logit's scale: once more)
                sum = wave_sum(sum);
                if (lane == 0) t.share[wave] = sum;
                kept = (int32_t)sum_all<uint64_t>(lane == 0 ? n : 0, t);
                next = kPick;
                break;
            }
        }
    }

    if (!settled && next == kDigits) {
        weigh = Weigh(c, top);
        const float least_x = least_logit(top, c, least, lane);
        uint64_t key = 1;
        if (top_k && top_k < x.n)
            key = max(key, reach(x.n, top_k, t, [&](uint32_t j, uint64_t* k) __attribute__((always_inline)) -> uint64_t { const float v = x.at(j); *k = order_key(v, j); return v > kNone; }));
        const uint64_t front = key;
        const auto weight = [&](uint32_t j, uint64_t* k) __attribute__((always_inline)) -> double {
            const float v = x.at(j);
            *k = order_key(v, j);
            return v > kNone && *k >= front && v >= least_x ? weigh(v) : 0.0;
        };
        if (top_p < 1.0f) {
            double sum = 0;
            uint64_t k;
#pragma nounroll
            for (uint32_t j = tid; j < x.n; j += kThreads) sum += weight(j, &k);
            sum = sum_all<double>(sum, t);
            // Whole numbers, so that digits' sums have no order; all of them together 2^61 to 2^62. Their roundings are 2^-42 of the sum for 2^20 classes, and no more than that of any front part that is the
            // answer (whose classes are the largest). Multiples of a part of the *largest* weight instead lose small ones, which together may be what top_p is about.
            const double unit = __builtin_bit_cast(double, (uint64_t)(2107 - (__builtin_bit_cast(uint64_t, sum) >> 52 & 0x7ff)) << 52);
            key = max(key, reach(x.n, (uint64_t)fmax(ceil((double)top_p * sum * unit), 1.0), t, [&](uint32_t j, uint64_t* k) __attribute__((always_inline)) { return (uint64_t)rint(weight(j, k) * unit); }));
        }
        bar = key == 1 || key_logit(key) < least_x ? Bar{least_x, kNobody} : Bar{key_logit(key), (uint32_t)key_class(key)};
        next = kShares;
    }
    if (!settled && next == kShares) {
        double sum = 0;
        uint64_t n = 0;
        x.template walk<false>(first, end, lane, [&](const float (&v)[kPer], uint32_t base) {
#pragma unroll
            for (uint32_t i = 0; i < kPer; ++i) {
                if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                const bool keeps = bar.keeps(v[i], W::number(base, i, lane));
                n += (uint32_t)__popcll(__ballot(keeps));
                if (keeps) sum += weigh(v[i]);
            }
        });
        sum = wave_sum(sum);
        __syncthreads();
        if (lane == 0) t.share[wave] = sum;
        kept = (int32_t)sum_all<uint64_t>(lane == 0 ? n : 0, t);
    }
    if (!settled) {
        // the share that holds the class; of that, a few classes side by side to a thread
        double every = 0, before = 0;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) every += t.share[w];
        const double target = (double)uniform * every;
        uint32_t pick = 0;
        {
            double at = 0;
            bool found = false;
#pragma unroll
            for (uint32_t w = 0; w < kWaves; ++w) {
                const double one = t.share[w];
                if (!found && one > 0) { pick = w; before = at; found = at + one > target; }
                at += one;
            }
        }
        const uint32_t each = ceil_div(ceil_div(x.share, kThreads), 8) * 8, stop = min((pick + 1) * x.share, x.n);
        const uint32_t mine = min(pick * x.share + tid * each, stop), mine_end = min(mine + each, stop);
        double own = 0;
#pragma nounroll
        for (uint32_t j = mine; j < mine_end; j += 8) {
            float v[8];
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) v[e] = j + e < mine_end ? x.at(j + e) : kNone;
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) {
                if (e % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                if (bar.keeps(v[e], j + e)) own += weigh(v[e]);
            }
        }
        if (tid == 0) t.found = kNobody;
        double all;
        const double at = before + scan_all<double>(own, t, &all);
        if (own > 0 && at + own > target) atomicMin(&t.found, tid);
        __syncthreads();
        uint32_t holder = t.found;
        if (holder == kNobody) holder = (uint32_t)fold_all<int64_t>(own > 0 ? (int64_t)tid : 0, t, [](int64_t p, int64_t q) { return p > q ? p : q; });
        __syncthreads();
        if (tid == holder) { t.above = __builtin_bit_cast(uint64_t, at); t.found = mine; }
        __syncthreads();
        if (wave == 0) {
            // its classes, a lane to each
            double so_far = __builtin_bit_cast(double, t.above);
            const uint32_t begin = t.found, close = min(begin + each, stop);
            uint32_t hit = min(begin, x.n - 1);
            for (uint32_t j = begin; j < close; j += 64) {
                const float v = j + lane < close ? x.at(j + lane) : kNone;
                const double w = bar.keeps(v, j + lane) ? weigh(v) : 0.0, upto = so_far + wave_scan(w);
                const uint64_t some = __ballot(w > 0), over = __ballot(w > 0 && upto > target);
                if (some) hit = j + 63 - __builtin_clzll(some);
                if (over) { hit = j + __builtin_ctzll(over); break; }
                so_far += wave_sum(w);
            }
            if (lane == 0) t.words[0] = hit;
        }
        __syncthreads();
        id = (int32_t)t.words[0];
        logprob = weigh.exponent((float)x.x[id]) * 0.6931471805599453 - log(every);
    }
    if (tid == 0) {
        if (odd) { id = -1; kept = -1; logprob = __builtin_nan(""); }
        if (a.ids) a.ids[row] = id;
        if (a.logprobs) a.logprobs[row] = (float)logprob;
        if (a.kept) a.kept[row] = kept;
    }
}

template <typename T, uint32_t WAVES> hipError_t go(const SampleArgs& s, hipStream_t st)
{
    return launch(s.a.allowed ? sample_kernel<T, true, WAVES> : sample_kernel<T, false, WAVES>, dim3(s.a.rows), 64 * WAVES, sizeof(Lds<WAVES>), st, s);
}
// Waves of a workgroup: few where a row has little work for them, many where there are not two rows to a compute unit and much to do (us with 4 / 8 / 16 waves: 1024 rows of 1000 classes at top_p 0.9
// 24.8 / 46.9 / 97, 512 of 8192 29.6 / 30.8 / 54.7, 1024 of 32768 88 / 91 / 148, all of them kept 57 / 52 / 78; 64 masked bf16 rows of 65001 with settings of their own 77 / 52 / 43, one of
// 131072 at top_p 0.9 138 / 88 / 75, with top_k 50 41 / 21 / 25; the last two with top_k before their lists were cut: 16 waves now 37 and 20).
uint32_t waves_for(uint32_t rows, uint32_t classes)
{
    if (classes <= 8192) return 4;
    return rows <= 256 && classes > 32768 ? 16 : 8;
}
template <typename T> hipError_t all_rows(SampleArgs s, hipStream_t st)
{
    mt_sample_args& a = s.a;
    for (uint32_t left = a.rows;; left -= kRowsAtOnce) {
        a.rows = std::min(left, kRowsAtOnce);
        const uint32_t waves = waves_for(a.rows, a.classes);
        const hipError_t e = waves == 4 ? go<T, 4>(s, st) : waves == 16 ? go<T, 16>(s, st) : go<T, 8>(s, st);
        if (e != hipSuccess || left <= kRowsAtOnce) return e;
        const uint64_t n = kRowsAtOnce;
        a.logits = (const T*)a.logits + n * a.row_stride;
        move_rows(a.n_classes, n);
        move_rows(a.allowed, n * a.allowed_stride);
        move_rows(a.uniform, n);
        move_rows(a.temperature, n);
        move_rows(a.top_k, n);
        move_rows(a.top_p, n);
        move_rows(a.min_p, n);
        move_rows(a.ids, n);
        move_rows(a.logprobs, n);
        move_rows(a.kept, n);
    }
}
template <typename T, uint32_t WAVES> hipError_t prepare()
{
    const hipError_t e = hipFuncSetAttribute((const void*)sample_kernel<T, true, WAVES>, hipFuncAttributeMaxDynamicSharedMemorySize, sizeof(Lds<WAVES>));
    return e != hipSuccess ? e : hipFuncSetAttribute((const void*)sample_kernel<T, false, WAVES>, hipFuncAttributeMaxDynamicSharedMemorySize, sizeof(Lds<WAVES>));
}

}  // namespace

hipError_t prepare_sample()
{
    const hipError_t e = prepare<float, 16>();
    return e != hipSuccess ? e : prepare<__bf16, 16>();
}

hipError_t launch_sample(const SampleArgs& s, hipStream_t st) { return s.a.dtype == MT_BF16 ? all_rows<__bf16>(s, st) : all_rows<float>(s, st); }

}  // namespace mt

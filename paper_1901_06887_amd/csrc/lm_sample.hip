// mt_sample: one class for every row of logits, drawn with the row's own settings.
//
// What a row keeps is a front part of its classes in their order (falling logits, lower numbers first among equals), so a row is settled by the last class that it keeps, its `bar`, and by how much weight
// stands in front of the class that a random number picks. Weights are 2^(c (x - x0)) in 64 bits (a polynomial of degree 9, 8e-14 of itself); sums are 64-bit ones in an order that does not depend on timing.
//
// A workgroup to a row, an eighth of its classes to a wave. The bar is found by what the settings ask for:
//   the first class alone (temperature 0, top_k 1, top_p 0): the largest logit, one pass
//   top_k: the lanes' largest first classes give a value that at least top_k classes reach; what reaches it goes into a list in LDS in the same pass. Where those are too many, or top_k is
//     large, numbers of classes per bin (of logits) say in a pass before which classes to list. The list is put in order and settles everything
//   top_p: weight per bin and wave in LDS in the first pass; a second one lists the bin that holds the bar. The weights of what is kept are then known for every wave's eighth
//   neither: sums for every wave's eighth
// The class is then looked for in the eighth that holds it, an eighth of that, and so on down to one chunk. Bins are laid by the lanes' largest first classes, so that neither a few very
// large logits nor many very small ones (masks of the type's lowest value) spoil them: some 90 to a standard deviation of a bell-shaped row. A row for which a list does not suffice (thousands of classes in
// one bin, top_k of thousands) is settled digit by digit of the order's key: right, but sixteen and more passes.
#include "lm_cache_device.h"
#include "lm_logits.h"

namespace mt {
namespace {

constexpr uint32_t kWaves = 8, kThreads = 64 * kWaves;
constexpr uint32_t kBins = 1000;
constexpr uint32_t kCap = 4000;                   // entries of the list
constexpr uint32_t kFewKept = 512;                // kept entries among which every thread looks for its own place
constexpr uint32_t kNobody = 0xffffffffu;

// A constant in scalar registers (the compiler would give every one a pair of vector registers).
__device__ __forceinline__ double scalar(double v) { asm("" : "+s"(v)); return v; }

// A row's weights: 2^(c (x - one)), 1 at `one`.
struct Weigh {
    double c, one;
    __device__ __forceinline__ double exponent(float x) const { return ((double)x - one) * c; }
    __device__ __forceinline__ double operator()(float x) const
    {
        // 2^y = 2^n 2^f, n the nearest whole number (the low bits of y + 1.5 2^52), 2^f a polynomial; y of -1000 and less, -infinity too, count as -1000
        const double y = fmax(exponent(x), -1000.0), t = y + 6755399441055744.0, f = y - (t - 6755399441055744.0);
        double p = fma(scalar(9.16811938851594e-08), f, scalar(1.3255182784592006e-06));
        p = fma(p, f, scalar(1.5258493063907014e-05));
        p = fma(p, f, scalar(0.0001540345603665657));
        p = fma(p, f, scalar(0.0013333547331461978));
        p = fma(p, f, scalar(0.009618129159172244));
        p = fma(p, f, scalar(0.055504108739712246));
        p = fma(p, f, scalar(0.24022650695813708));
        p = fma(p, f, scalar(0.6931471805585505));
        p = fma(p, f, 1.0);
        return __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, p) + (__builtin_bit_cast(uint64_t, t) << 52));
    }
};

struct Lds {
    union {
        double mass[kWaves][kBins];
        uint32_t count[kWaves][kBins];
        struct { uint64_t keys[kCap]; double weights[kCap]; } list;
        uint64_t digits[256];
    };
    uint64_t words[kWaves];
    double share[kWaves];                         // kept weight of every wave's eighth
    float bars[kWaves], spreads[kWaves];
    uint32_t listed, found;
    uint64_t chosen, above;
};

// Inclusive sums over the wave's lanes; the last lane has the total.
template <typename V> __device__ __forceinline__ V wave_scan(V v, uint32_t lane)
{
#pragma unroll
    for (uint32_t d = 1; d < 64; d <<= 1) { const V o = __shfl_up(v, d); if (lane >= d) v += o; }
    return v;
}
template <typename V> __device__ __forceinline__ V wave_sum(V v)
{
#pragma unroll
    for (uint32_t d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
// Over the workgroup, the same in every thread.
template <typename V, typename F> __device__ __forceinline__ V fold_all(V v, Lds& t, F f)
{
    static_assert(sizeof(V) == 8, "");
#pragma unroll
    for (uint32_t d = 32; d; d >>= 1) v = f(v, (V)__shfl_xor(v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) t.words[threadIdx.x >> 6] = __builtin_bit_cast(uint64_t, v);
    __syncthreads();
    v = __builtin_bit_cast(V, t.words[0]);
#pragma unroll
    for (uint32_t w = 1; w < kWaves; ++w) v = f(v, __builtin_bit_cast(V, t.words[w]));
    return v;
}
template <typename V> __device__ __forceinline__ V sum_all(V v, Lds& t) { return fold_all<V>(v, t, [](V a, V b) { return a + b; }); }
// Exclusive sums over the workgroup's threads.
template <typename V> __device__ __forceinline__ V scan_all(V v, Lds& t, V* total)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const V upto = wave_scan(v, lane);
    __syncthreads();
    if (lane == 63) t.words[wave] = __builtin_bit_cast(uint64_t, upto);
    __syncthreads();
    V before = 0, all = 0;
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) { const V o = __builtin_bit_cast(V, t.words[w]); if (w < wave) before += o; all += o; }
    *total = all;
    return before + (upto - v);
}

// Bins of logits, 0 in front; what is in none has kBins or more.
struct Bins {
    float top, per;
    __device__ __forceinline__ float place(float x) const { return (top - x) * per; }
};

// The last class that is kept; everything in front of it is kept too, unless its weight is below `least`.
struct Bar {
    float x;
    uint32_t c;
    double least;
    __device__ __forceinline__ bool keeps(float v, uint32_t at) const { return v > x || (v == x && at <= c && v > kNone); }
};

template <typename T, bool MASK> struct Row {
    static constexpr uint32_t kVecs = sizeof(T) == 4 ? 4 : 2;
    using R = Raw<T, kVecs>;
    static constexpr uint32_t kPer = R::kPer, kChunk = R::kChunk;
    const T* x;
    const uint32_t* allowed;
    uint32_t n, eighth;          // classes that there are; classes of a wave

    __device__ __forceinline__ float at(uint32_t c) const
    {
        if (c >= n || (MASK && !((allowed[c >> 5] >> (c & 31)) & 1))) return kNone;
        return (float)x[c];
    }
    static __device__ __forceinline__ uint32_t number(uint32_t base, int i, uint32_t lane) { return R::first(base, i / R::kVec, lane) + i % R::kVec; }
    // f(logits of a chunk, its first class) for a wave's chunks of classes base .. end - 1
    template <typename F> __device__ __forceinline__ void walk(uint32_t base, uint32_t end, uint32_t lane, F f) const
    {
        if (base >= end) return;
        base = __builtin_amdgcn_readfirstlane(base);
        asm volatile("" : "+s"(base));            // (or the addresses of every pass's first chunk wait in registers)
        R raw;
        raw.template load<MASK>(x, allowed, base, lane, end);
        for (; base < end; base += kChunk) {
            float v[kPer];
            raw.template logits<MASK>(v, base, lane, end);
            if (base + kChunk < end) raw.template load<MASK>(x, allowed, base + kChunk, lane, end);
            f(v, base);
        }
    }
};

// What a pass sees of the largest logit: a lane's largest, and the first class of the chunk that it is in.
struct Most {
    float x = kNone;
    uint32_t base = 0;
    bool odd = false;            // a NaN
    template <uint32_t PER> __device__ __forceinline__ void look(const float (&v)[PER], uint32_t at)
    {
        float m = v[0];
#pragma unroll
        for (uint32_t i = 0; i < PER; ++i) { odd |= v[i] != v[i]; m = fmaxf(m, v[i]); }
        if (m > x) { x = m; base = at; }
    }
};

// The key at which the values of the classes in front of it and its own first reach `target`; amount(c, key) is a class's value. (Digit by digit: every digit is a pass over the row.)
template <typename F> __device__ __forceinline__ uint64_t reach(uint32_t n, uint64_t target, Lds& t, F amount)
{
    uint64_t prefix = 0, before = 0;
#pragma nounroll
    for (int shift = 56; shift >= 0; shift -= 8) {
        __syncthreads();
        if (threadIdx.x < 256) t.digits[threadIdx.x] = 0;
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

// The list's keys in falling order. Up to kThreads of them: every thread counts what is in front of its own; more: a bitonic network whose comparisons all go one way, so that what lies behind the last
// entry can be taken for the smallest and never moves.
__device__ __forceinline__ void put_in_order(Lds& t, uint32_t n)
{
    uint64_t* keys = t.list.keys;
    const uint32_t tid = threadIdx.x;
    if (n <= kThreads) {
        const uint64_t own = tid < n ? keys[tid] : 0;
        uint32_t before = 0;
        if (tid < (n + 63) / 64 * 64)
            for (uint32_t i = 0; i < n; ++i) before += keys[i] > own;
        __syncthreads();
        if (tid < n) keys[before] = own;
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
struct Own {
    uint32_t first, end;
    __device__ __forceinline__ explicit Own(uint32_t n)
    {
        const uint32_t each = ceil_div(n, kThreads);
        first = min(threadIdx.x * each, n);
        end = min(first + each, n);
    }
    // Their weights into the list, and the sum of those that are not below `least`.
    __device__ __forceinline__ double weights(Lds& t, const Weigh& weigh, double least) const
    {
        double sum = 0;
#pragma nounroll
        for (uint32_t i = first; i < end; ++i) {
            const double w = weigh(key_logit(t.list.keys[i]));
            t.list.weights[i] = w;
            if (w >= least) sum += w;
        }
        return sum;
    }
};

template <typename T, bool MASK>
__global__ void __launch_bounds__(kThreads, 4) sample_kernel(SampleArgs s)
{
    using W = Row<T, MASK>;
    constexpr uint32_t kPer = W::kPer, kChunk = W::kChunk;
    __shared__ __attribute__((aligned(16))) Lds t;
    const mt_sample_args& a = s.a;
    const uint32_t row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float temperature = a.temperature ? a.temperature[row] : 1.0f, uniform = a.uniform[row], top_p = a.top_p ? a.top_p[row] : 1.0f, min_p = a.min_p ? a.min_p[row] : 0.0f;
    const uint32_t top_k = a.top_k ? (uint32_t)max(a.top_k[row], 0) : 0;
    W x;
    x.x = (const T*)a.logits + row * a.row_stride;
    x.allowed = MASK ? a.allowed + row * a.allowed_stride : nullptr;
    x.n = a.n_classes ? (uint32_t)min(max(a.n_classes[row], 0), (int32_t)a.classes) : a.classes;
    x.eighth = ceil_div(a.classes, kWaves * kChunk) * kChunk;
    const uint32_t first = min(wave * x.eighth, x.n), end = min(first + x.eighth, x.n);

    const bool lost = !(temperature >= 0.0f) || uniform != uniform || top_p != top_p || min_p != min_p;
    const bool greedy = temperature < 1.17549435e-38f || top_k == 1 || top_p <= 0.0f;
    const double c = 1.4426950408889634 / (double)(greedy ? 1.0f : temperature);
    const double least = fmin((double)min_p, 1.0);
    const auto weigh_from = [&](float at) { return Weigh{c, (double)at}; };

    // Outcome: nothing yet, or the row's class; in between the bar, the weights and each eighth's share of them.
    int32_t id = -1, kept = 0;
    double logprob = kNone;
    bool settled = lost, odd = lost;
    Bar bar{kNone, kNobody, 0.0};
    Weigh weigh = weigh_from(0.0f);

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
    // A wave appends the classes of a chunk that `mine` has a bit for; what doesn't fit is counted alone.
    const auto append = [&](uint32_t mine, const float (&v)[kPer], uint32_t base) __attribute__((always_inline)) {
        if (!__ballot(mine != 0)) return;
        const uint32_t own = (uint32_t)__popc(mine), upto = wave_inclusive_scan(own);
        uint32_t at = 0;
        if (lane == 63) at = atomicAdd(&t.listed, upto);
        at = (uint32_t)__builtin_amdgcn_readlane((int)at, 63) + upto - own;
#pragma unroll
        for (uint32_t i = 0; i < kPer; ++i)
            if (mine >> i & 1) {
                if (at < kCap) t.list.keys[at] = order_key(v[i], W::number(base, i, lane));
                ++at;
            }
    };
    // The lanes' largest classes of the waves' first chunks.
    const auto lane_largest = [&]() __attribute__((always_inline)) {
        float m = kNone;
        x.walk(first, min(first + kChunk, end), lane, [&](const float (&v)[kPer], uint32_t) {
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
    enum { kPick, kShares, kDigits } next = kShares;      // what remains: look for the class; first sum each eighth; first find the bar

    if (settled) {
    } else if (greedy) {
        Most m;
        x.walk(first, end, lane, [&](const float (&v)[kPer], uint32_t base) { m.look(v, base); });
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
        if (tid == 0) t.listed = 0;
        const float m = lane_largest();
        float reached = kNone;
        const uint32_t each = ceil_div(top_k, kWaves);
        if (each <= 48) {
            const float mine = bar_of(m, each), alone = top_k <= 48 ? bar_of(m, top_k) : kNone;
            __syncthreads();
            if (lane == 0) { t.bars[wave] = mine; t.spreads[wave] = alone; }
            __syncthreads();
            reached = t.bars[0];
            float other = t.spreads[0];
#pragma unroll
            for (uint32_t w = 1; w < kWaves; ++w) { reached = fminf(reached, t.bars[w]); other = fmaxf(other, t.spreads[w]); }
            reached = fmaxf(reached, other);
        }
        __syncthreads();
        bool listed = false;
        Most most;
        if (reached > kNone || x.n <= kCap) {
            x.walk(first, end, lane, [&](const float (&v)[kPer], uint32_t base) {
                most.look(v, base);
                uint32_t mine = 0;
#pragma unroll
                for (uint32_t i = 0; i < kPer; ++i) mine |= v[i] >= reached && v[i] > kNone ? 1u << i : 0;
                append(mine, v, base);
            });
            largest(most);
            listed = t.listed <= kCap;
        }
        if (!listed) {
            // classes per bin, then all those of the bins that hold the first top_k
            float lead;
            const Bins bins = lay_bins(&lead);
            for (uint32_t i = tid; i < kWaves * kBins; i += kThreads) t.count[0][i] = 0;
            __syncthreads();
            most = Most{};
            x.walk(first, end, lane, [&](const float (&v)[kPer], uint32_t base) {
                most.look(v, base);
#pragma unroll
                for (uint32_t i = 0; i < kPer; ++i) {
                    const float p = bins.place(v[i]);
                    if (p < (float)kBins) atomicAdd(&t.count[wave][(uint32_t)fmaxf(p, 0.0f)], 1u);
                }
            });
            largest(most);
            uint64_t mine[2] = {0, 0};
#pragma unroll
            for (uint32_t e = 0; e < 2; ++e)
                if (2 * tid + e < kBins)
#pragma unroll
                    for (uint32_t w = 0; w < kWaves; ++w) mine[e] += t.count[w][2 * tid + e];
            uint64_t all;
            const uint64_t before = scan_all<uint64_t>(mine[0] + mine[1], t, &all);
            if (tid == 0) { t.found = kNobody; t.above = 0; t.listed = 0; }
            __syncthreads();
            if (before < top_k && before + mine[0] + mine[1] >= top_k) {
                const bool second = before + mine[0] < top_k;
                t.found = 2 * tid + second;
                t.above = before + mine[0] + (second ? mine[1] : 0);
            }
            __syncthreads();
            const uint32_t last = t.found;
            if (!settled && last != kNobody && t.above <= kCap) {
                __syncthreads();
                x.walk(first, end, lane, [&](const float (&v)[kPer], uint32_t base) {
                    uint32_t mine = 0;
#pragma unroll
                    for (uint32_t i = 0; i < kPer; ++i) mine |= bins.place(v[i]) < (float)(last + 1) ? 1u << i : 0;
                    append(mine, v, base);
                });
                listed = true;
            }
            __syncthreads();
        }
        if (!settled && listed) {
            // in order: top_k by number, min_p by weight, top_p by sums
            __syncthreads();
            const uint32_t n = t.listed;
            put_in_order(t, n);
            weigh = weigh_from(top);
            const uint32_t most_kept = min(n, top_k);
            const Own own(most_kept);
            double total, at = scan_all<double>(own.weights(t, weigh, least), t, &total);
            const double target = top_p < 1.0f ? (double)top_p * total : 2.0 * total;
            uint64_t mine = 0;
            for (uint32_t i = own.first; i < own.end; ++i) {
                const double w = t.list.weights[i];
                if (w < least) break;
                if (i == 0 || at < target) ++mine;
                at += w;
            }
            kept = max((int32_t)sum_all<uint64_t>(mine, t), 1);
            const uint64_t last = t.list.keys[kept - 1];
            bar = Bar{key_logit(last), (uint32_t)key_class(last), 0.0};
            if ((uint32_t)kept <= kFewKept) {
                // every kept class by its number: what stands in front of it
                __syncthreads();
                const uint32_t mine_c = tid < (uint32_t)kept ? (uint32_t)key_class(t.list.keys[tid]) : 0;
                double front = 0, every = 0;
                for (uint32_t i = 0; i < (uint32_t)kept; ++i) {
                    const double one = t.list.weights[i];
                    every += one;
                    if ((uint32_t)key_class(t.list.keys[i]) <= mine_c) front += one;
                }
                if (tid == 0) t.found = kNobody;
                __syncthreads();
                const bool any = tid < (uint32_t)kept && t.list.weights[tid] > 0;
                if (any && front > (double)uniform * every) atomicMin(&t.found, mine_c);
                __syncthreads();
                uint32_t pick = t.found;
                if (pick == kNobody) pick = (uint32_t)fold_all<int64_t>(any ? (int64_t)mine_c : -1, t, [](int64_t p, int64_t q) { return p > q ? p : q; });
                id = (int32_t)pick;
                logprob = weigh.exponent((float)x.x[pick]) * 0.6931471805599453 - log(every);
                settled = true;
            }
        } else if (!settled) next = kDigits;
    } else {
        if (least > 0) {
            Most m;
            x.walk(first, end, lane, [&](const float (&v)[kPer], uint32_t base) { m.look(v, base); });
            largest(m);
            bar.least = least;
        }
        if (settled) {
        } else if (top_p < 1.0f) {
            float lead;
            const Bins bins = lay_bins(&lead);
            if (least > 0) lead = top;
            double rest;
            for (;;) {
                weigh = weigh_from(lead);
                for (uint32_t i = tid; i < kWaves * kBins; i += kThreads) t.mass[0][i] = 0;
                __syncthreads();
                Most m;
                rest = 0;
                x.walk(first, end, lane, [&](const float (&v)[kPer], uint32_t base) {
                    m.look(v, base);
#pragma unroll
                    for (uint32_t i = 0; i < kPer; ++i) {
                        if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);      // (four at a time: registers)
                        const double w = weigh(v[i]);
                        const float p = bins.place(v[i]);
                        if (w >= bar.least) {
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
                double mine[2] = {0, 0};
#pragma unroll
                for (uint32_t e = 0; e < 2; ++e)
                    if (2 * tid + e < kBins)
#pragma unroll
                        for (uint32_t w = 0; w < kWaves; ++w) mine[e] += t.mass[w][2 * tid + e];
                double in_bins;
                const double before = scan_all<double>(mine[0] + mine[1], t, &in_bins);
                const double target = (double)top_p * (in_bins + sum_all<double>(rest, t));
                if (tid == 0) { t.found = kNobody; t.listed = 0; }
                __syncthreads();
                const double upto1 = before + mine[0], upto2 = before + (mine[0] + mine[1]);
                const uint32_t here = upto1 >= target ? 2 * tid : upto2 >= target ? 2 * tid + 1 : kNobody;
                if (here < kBins) atomicMin(&t.found, here);
                __syncthreads();
                const uint32_t in = t.found;
                if (in == kNobody) next = kDigits;
                else {
                    if (here == in) t.above = __builtin_bit_cast(uint64_t, here == 2 * tid ? before : upto1);
                    double above_mine = 0;                // of this wave's eighth
                    for (uint32_t i = lane; i < in; i += 64) above_mine += t.mass[wave][i];
                    above_mine = wave_sum(above_mine);
                    __syncthreads();
                    const double above = __builtin_bit_cast(double, t.above);
                    uint64_t n_above = 0;
                    x.walk(first, end, lane, [&](const float (&v)[kPer], uint32_t base) {
                        uint32_t mine = 0, count = 0;
#pragma unroll
                        for (uint32_t i = 0; i < kPer; ++i) {
                            const float p = bins.place(v[i]);
                            mine |= p < (float)(in + 1) && (in == 0 || p >= (float)in) ? 1u << i : 0;
                            count += in != 0 && p < (float)in;
                        }
                        n_above += count;
                        append(mine, v, base);
                    });
                    n_above = sum_all<uint64_t>(n_above, t);
                    const uint32_t n = t.listed;
                    if (n > kCap || n == 0) next = kDigits;
                    else {
                        put_in_order(t, n);
                        const Own own(n);
                        double total, at = above + scan_all<double>(own.weights(t, weigh, bar.least), t, &total);
                        uint64_t mine = 0;
                        for (uint32_t i = own.first; i < own.end; ++i) {
                            const double w = t.list.weights[i];
                            if (w < bar.least) break;
                            if (i == 0 || at < target) ++mine;
                            at += w;
                        }
                        const uint32_t in_list = max((uint32_t)sum_all<uint64_t>(mine, t), 1u);
                        kept = (int32_t)(n_above + in_list);
                        const uint64_t last = t.list.keys[in_list - 1];
                        bar.x = key_logit(last); bar.c = (uint32_t)key_class(last);
                        double more = 0;                  // the list's share of this wave's eighth
                        for (uint32_t i = lane; i < in_list; i += 64) {
                            const uint32_t j = (uint32_t)key_class(t.list.keys[i]);
                            if (j >= first && j < end) more += t.list.weights[i];
                        }
                        more = wave_sum(more);
                        if (lane == 0) t.share[wave] = above_mine + more;
                        __syncthreads();
                        next = kPick;
                    }
                }
            }
        } else {
            // all of them, or all of a weight: sums for every eighth
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
            for (;;) {
                weigh = weigh_from(lead);
                Most m;
                double sum = 0;
                uint64_t n = 0;
                x.walk(first, end, lane, [&](const float (&v)[kPer], uint32_t base) {
                    m.look(v, base);
                    uint32_t count = 0;
#pragma unroll
                    for (uint32_t i = 0; i < kPer; ++i) {
                        if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                        const double w = weigh(v[i]);
                        const bool counts = v[i] > kNone && w >= bar.least;
                        count += counts;
                        sum += counts ? w : 0.0;
                    }
                    n += count;
                });
                largest(m);
                if (settled) break;
                if (fabs(weigh.exponent(top)) > 900.0) { lead = top; continue; }
                sum = wave_sum(sum);
                if (lane == 0) t.share[wave] = sum;
                kept = (int32_t)sum_all<uint64_t>(n, t);
                next = kPick;
                break;
            }
        }
    }

    if (!settled && next == kDigits) {
        weigh = weigh_from(top);
        const double unit = (double)(1ull << s.bits);
        uint64_t key = 1;
        if (top_k && top_k < x.n)
            key = max(key, reach(x.n, top_k, t, [&](uint32_t j, uint64_t* k) __attribute__((always_inline)) -> uint64_t { const float v = x.at(j); *k = order_key(v, j); return v > kNone; }));
        const uint64_t front = key;
        const auto amount = [&](uint32_t j, uint64_t* k) __attribute__((always_inline)) -> uint64_t {
            const float v = x.at(j);
            *k = order_key(v, j);
            if (!(v > kNone) || *k < front) return 0;
            const double w = weigh(v);
            return w >= least ? (uint64_t)rint(w * unit) : 0;
        };
        if (top_p < 1.0f) {
            uint64_t sum = 0, k;
#pragma nounroll
            for (uint32_t j = tid; j < x.n; j += kThreads) sum += amount(j, &k);
            sum = sum_all<uint64_t>(sum, t);
            key = max(key, reach(x.n, (uint64_t)fmax(ceil((double)top_p * (double)sum), 1.0), t, amount));
        }
        bar = Bar{key == 1 ? kNone : key_logit(key), key == 1 ? kNobody : (uint32_t)key_class(key), least};
        next = kShares;
    }
    if (!settled && next == kShares) {
        double sum = 0;
        uint64_t n = 0;
        x.walk(first, end, lane, [&](const float (&v)[kPer], uint32_t base) {
#pragma unroll
            for (uint32_t i = 0; i < kPer; ++i) {
                if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                if (bar.keeps(v[i], W::number(base, i, lane))) {
                    const double w = weigh(v[i]);
                    if (w >= bar.least) { sum += w; ++n; }
                }
            }
        });
        sum = wave_sum(sum);
        __syncthreads();
        if (lane == 0) t.share[wave] = sum;
        kept = (int32_t)sum_all<uint64_t>(n, t);
    }
    if (!settled) {
        // the eighth that holds the class, an eighth of it, ... the chunk, the class
        double every = 0;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) every += t.share[w];
        const double target = (double)uniform * every;
        double before = 0;
        uint32_t base = 0, len = x.eighth;
        for (;;) {
            uint32_t pick = 0;
            double at = before;
            bool found = false;
#pragma unroll
            for (uint32_t w = 0; w < kWaves; ++w) {
                const double one = t.share[w];
                if (!found && one > 0) { pick = w; before = at; found = at + one > target; }
                at += one;
            }
            base += pick * len;
            const uint32_t stop = min(base + len, x.n);
            if (len <= kChunk) {
                if (wave == 0) {
                    uint32_t hit = kNobody, last = 0;
                    x.walk(base, stop, lane, [&](const float (&v)[kPer], uint32_t from) {
                        constexpr uint32_t kVec = W::R::kVec;
#pragma unroll
                        for (uint32_t i = 0; i < kPer; i += kVec) {
                            double w[kVec], own = 0;
#pragma unroll
                            for (uint32_t e = 0; e < kVec; ++e) {
                                if (e % 2 == 0) __builtin_amdgcn_sched_barrier(0);
                                const uint32_t j = W::number(from, i + e, lane);
                                w[e] = bar.keeps(v[i + e], j) ? weigh(v[i + e]) : 0.0;
                                if (w[e] < bar.least) w[e] = 0;
                                if (w[e] > 0) last = j + 1;
                                own += w[e];
                            }
                            const double upto = wave_scan(own, lane);
                            double so_far = before + (upto - own);
#pragma unroll
                            for (uint32_t e = 0; e < kVec; ++e) {
                                so_far += w[e];
                                if (hit == kNobody && w[e] > 0 && so_far > target) hit = W::number(from, i + e, lane);
                            }
                            before += __shfl(upto, 63);
                        }
                    });
#pragma unroll
                    for (uint32_t d = 32; d; d >>= 1) { hit = min(hit, (uint32_t)__shfl_xor(hit, d)); last = max(last, (uint32_t)__shfl_xor(last, d)); }
                    if (lane == 0) t.found = hit != kNobody ? hit : max(last, 1u) - 1;
                }
                __syncthreads();
                id = (int32_t)t.found;
                break;
            }
            len = ceil_div(len, kWaves * kChunk) * kChunk;
            double sum = 0;
            const uint32_t mine = min(base + wave * len, stop);
            const uint32_t mine_end = min(mine + len, stop);
#pragma nounroll
            for (uint32_t at = mine + lane; at < mine_end; at += 512) {
                float v[8];
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) v[e] = at + 64 * e < mine_end ? x.at(at + 64 * e) : kNone;
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) {
                    if (e % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                    if (bar.keeps(v[e], at + 64 * e)) {
                        const double w = weigh(v[e]);
                        if (w >= bar.least) sum += w;
                    }
                }
            }
            sum = wave_sum(sum);
            __syncthreads();
            if (lane == 0) t.share[wave] = sum;
            __syncthreads();
        }
        logprob = weigh.exponent((float)x.x[id]) * 0.6931471805599453 - log(every);
    }
    if (tid == 0) {
        if (odd) { id = -1; kept = -1; logprob = __builtin_nan(""); }
        if (a.ids) a.ids[row] = id;
        if (a.logprobs) a.logprobs[row] = (float)logprob;
        if (a.kept) a.kept[row] = kept;
    }
}

template <typename T> hipError_t all_rows(SampleArgs s, hipStream_t st)
{
    mt_sample_args& a = s.a;
    for (uint32_t left = a.rows;; left -= kRowsAtOnce) {
        a.rows = std::min(left, kRowsAtOnce);
        const hipError_t e = launch(a.allowed ? sample_kernel<T, true> : sample_kernel<T, false>, dim3(a.rows), kThreads, 0, st, s);
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

}  // namespace

uint64_t sample_scratch_bytes(uint32_t, uint32_t) { return 0; }

hipError_t launch_sample(const SampleArgs& s, hipStream_t st) { return s.a.dtype == MT_BF16 ? all_rows<__bf16>(s, st) : all_rows<float>(s, st); }

}  // namespace mt

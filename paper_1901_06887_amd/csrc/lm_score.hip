// mt_score: log probabilities and ranks of given classes, entropy and the best alternatives of rows of logits, in one pass over them.
//
// With m the largest allowed logit, z = (x - m) / T, S = sum e^z and U = sum z e^z: log p = z - log S and the entropy is log S - U / S, a sum of two
// terms that are not negative.  (x - m) / 2 is what is worked with: x - m itself can leave fp32's range.  U is kept with log2(e) z, the exponent of two, in the place
// of z: where e^z is not 0 that is above -150 at every temperature, so no term of U is large.  Every lane carries its own m, S and U and
// rescales them once per 16 classes; lanes, waves and workgroups are joined at the end.
//
// Alternatives: every wave keeps a list in LDS of what can still be among the best `top` of its classes.  The waves' first 1024 classes set a bar for all of
// them: a value that a quarter of `top` lanes' maxima reach in every wave, so that at least `top` classes do, and few others.  What a wave has in its own
// list is in order in front of its later classes, so of those an equal one doesn't get in; a list that fills up is cut to its best `top` and raises the bar.
// One comparison a lane and 16 classes is what that costs where nothing passes.
//
// Memory bounds many rows (2048 rows of 32768 fp32 classes, one given and one alternative, 56 us, 4.8 TB/s; without either 48 us, 5.6 TB/s), a chain of memory trips
// and the fetch of code that runs once few: one row of 1000 4.4 us, 16 masked rows of 65001 with four given and 20 alternatives 16 us, 9 without alternatives.
#include "lm_device.h"

namespace mt {
namespace {

constexpr float kNone = -__builtin_inff();
constexpr float kLowest = -3.402823466e38f;
constexpr uint32_t kSome = 1024;                  // classes that are enough for a wave
constexpr uint32_t kList = 192;                   // entries of a wave's list
constexpr uint32_t kWaves = 4;                    // waves of a workgroup
constexpr uint32_t kRecords = 1024;               // most rows x parts where workgroups share a row's classes
constexpr uint32_t kMaxParts = 64;                // most workgroups that share one
constexpr uint32_t kPartKeys = kMaxParts / kWaves * MT_SCORE_MAX_TOP / 64;      // keys of a lane where parts are joined

// What a workgroup hands over of its share of a row, to another one on any XCD: every word is stored through to memory and loaded from there
// (agent scope), and the ticket is drawn when the stores have arrived.  Fences of the whole L2 in their place took 4 us more.
struct Part {
    float m, s, u, pad;
    uint32_t in_front[MT_SCORE_MAX_GIVEN];
    uint64_t keys[MT_SCORE_MAX_TOP];
};

template <typename V> __device__ __forceinline__ void hand_over(V* p, V v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename V> __device__ __forceinline__ V take_over(const V* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// A class's logit, -infinity where it is not allowed.
template <typename T>
__device__ __forceinline__ float logit(const T* x, const uint32_t* allowed, uint32_t c, uint32_t n)
{
    if (c >= n || (allowed && !((allowed[c >> 5] >> (c & 31)) & 1))) return kNone;
    return (float)x[c];
}

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

// Half of x - m: with finite x and m this is never out of range.
__device__ __forceinline__ float half_below(float x, float m) { return fmaf(0.5f, x, -0.5f * m); }
__device__ __forceinline__ float log_prob(float x, float m, float inv_t, float log_s) { return half_below(x, m) * inv_t * 2.0f - log_s; }

// Exponents of two below this count as this: two to them is 0 either way, and 0 times this is no NaN.
constexpr float kNothing = -1000.0f;

// Maximum and sums of some classes; nothing yet: {kLowest, 0, 0}.
struct Sums {
    float m, s, u;
    __device__ __forceinline__ void rebase(float to, float scale)
    {
        const float d = half_below(m, to) * scale, f = __builtin_amdgcn_exp2f(d);
        u = f * fmaf(fmaxf(d, kNothing), s, u);
        s *= f;
        m = to;
    }
    __device__ __forceinline__ void join(const Sums& o, float scale)
    {
        const float to = fmaxf(m, o.m);
        Sums q = o;
        q.rebase(to, scale);
        rebase(to, scale);
        s += q.s; u += q.u;
    }
    __device__ __forceinline__ void over_wave(float scale)
    {
        rebase(wave_max(m), scale);
        s = wave_total(s); u = wave_total(u);
    }
};

// Entries among the kStep at `at` that are in front of `key`.
constexpr uint32_t kStep = 8;
__device__ __forceinline__ uint32_t in_front_of(uint64_t key, const uint64_t* at)
{
    uint32_t n = 0;
#pragma unroll
    for (uint32_t k = 0; k < kStep; ++k) n += at[k] > key;
    return n;
}

// A value a little below: what is equal to x is above it.
__device__ __forceinline__ float below(float x) { return x - fmaf(fabsf(x), 1e-6f, 1.2e-38f); }

// Entries of a wave's list in no order, and the bar: a class is kept if its logit is above it.  A bar raised to a value lies a little below it for the rest
// of the chunk, whose classes equal to it may come in front of some in the list, and at the value from the next chunk on.
// (The code is kept short, in loops: a call runs it once, so much of its time is the fetch of the code.)
struct List {
    uint64_t* at;         // LDS, kList entries and kStep more
    uint64_t* best;       // LDS, MT_SCORE_MAX_TOP entries
    uint32_t n;
    float bar, next;
    __device__ __forceinline__ void raise(float to)
    {
        if (to > next) { next = to; bar = below(to); }
    }

    // Leaves the best `top` of the entries, in order, and raises the bar to the last of them.
    __device__ __forceinline__ void cut(uint32_t top, uint32_t lane)
    {
        if (lane < kStep) at[n + lane] = 0;
        wave_sync();
#pragma nounroll
        for (uint32_t j = 0; j < n; j += 64) {
            const uint64_t own = j + lane < n ? at[j + lane] : 0;
            uint32_t before = 0;
#pragma nounroll
            for (uint32_t i = 0; i < n; i += kStep) before += in_front_of(own, at + i);
            if (own && before < top) best[before] = own;
        }
        wave_sync();
        if (n > top) n = top;
        if (lane < n) at[lane] = best[lane];
        wave_sync();
        if (n == top) raise(key_logit(at[top - 1]));
    }

    __device__ __forceinline__ void append(bool keep, uint64_t key)
    {
        const uint64_t lanes = __ballot(keep);
        if (keep) at[n + __builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0))] = key;
        n += (uint32_t)__popcll(lanes);
    }
};
constexpr uint32_t kListRoom = kList - 64;        // entries up to which every lane can still append one

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
                v[i] = u32x4{0, 0, 0, 0};
                if (c + kVec <= classes) v[i] = *(const typename Any<T>::vec16*)(x + c);
                else if (c < classes) {
#pragma unroll
                    for (uint32_t e = 0; e < kVec; ++e)
                        if (c + e < classes) {
                            if constexpr (sizeof(T) == 2) v[i][e / 2] |= (uint32_t)((const uint16_t*)x)[c + e] << (16 * (e % 2));
                            else v[i][e] = ((const uint32_t*)x)[c + e];
                        }
                }
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

// The same for the lanes of all the waves: n values at least reach it.  (Where a wave alone has too few, what n in some other wave reach.)
template <uint32_t WAVES>
__device__ __forceinline__ float bar_of_all(float v, uint32_t n, float* lds, uint32_t wave)
{
    if constexpr (WAVES == 1) return bar_of(v, n);
    float bar = kNone;
#pragma nounroll
    for (int all = 1; all >= 0 && bar == kNone; --all) {
        const float mine = bar_of(v, all ? (n + WAVES - 1) / WAVES : n);
        __syncthreads();
        lds[wave] = mine;
        __syncthreads();
        bar = lds[0];
#pragma unroll
        for (uint32_t w = 1; w < WAVES; ++w) bar = all ? fminf(bar, lds[w]) : fmaxf(bar, lds[w]);
    }
    return bar;
}

// Everything that a wave, then a workgroup, knows of its share of a row.
struct Share {
    Sums sums;
    uint32_t in_front;        // lane g: allowed classes in front of given class g
};

// WAVES waves share a row's part [blockIdx.y]; WAVES 1: every wave of the workgroup has a row of its own.  A lane takes VECS vectors of 16 bytes at a time.
template <typename T, bool TOP, bool MASK, uint32_t WAVES, bool PARTS, uint32_t VECS>
__global__ void __launch_bounds__(64 * kWaves, 4) score_kernel(ScoreArgs s)
{
    using R = Raw<T, VECS>;
    constexpr uint32_t kPer = R::kPer, kChunk = R::kChunk;
    const mt_score_args& a = s.a;
    // (asked for in one go: loads where they are used are as many trips to memory one after the other)
    asm volatile("" :: "s"(a.logits), "s"(a.n_classes), "s"(a.allowed), "s"(a.given), "s"(a.given_ranks), "s"(a.scratch), "s"(a.row_stride), "s"(a.allowed_stride), "s"(a.rows), "s"(a.classes),
                 "s"(a.n_given), "s"(a.top), "s"(s.exp2_scale), "s"(s.parts), "s"(s.part_len));
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t row = WAVES == 1 ? blockIdx.x * kWaves + wave : blockIdx.x;
    if (row >= a.rows) return;                    // (whole waves, and none where a barrier follows)
    __shared__ __attribute__((aligned(16))) uint64_t lists[TOP ? kWaves : 1][TOP ? kList + kStep : 1];
    __shared__ __attribute__((aligned(16))) uint64_t best[TOP ? kWaves : 1][TOP ? MT_SCORE_MAX_TOP : 1];
    const T* x = (const T*)a.logits + row * a.row_stride;
    const uint32_t* allowed = MASK ? a.allowed + row * a.allowed_stride : nullptr;
    const uint32_t part = PARTS ? blockIdx.y : 0;
    const uint32_t part_end = min((uint64_t)(part + 1) * s.part_len, (uint64_t)a.classes);
    const uint32_t wave_len = WAVES == 1 ? s.part_len : ceil_div(s.part_len, WAVES * kChunk) * kChunk;
    uint32_t base = part * s.part_len + (WAVES == 1 ? 0 : wave * wave_len);
    const uint32_t mem_end = base < part_end ? min((uint64_t)base + wave_len, (uint64_t)part_end) : base;      // this wave's classes, and no more are read
    R raw{};
    if (base < mem_end) raw.template load<MASK>(x, allowed, base, lane, mem_end);
    const uint32_t n = a.n_classes ? (uint32_t)min(max(a.n_classes[row], 0), (int32_t)a.classes) : a.classes;
    const uint32_t end = min(mem_end, n);
    // lane g: given class g and its logit
    const int32_t given = lane < a.n_given ? a.given[(uint64_t)row * a.n_given + lane] : -1;
    const float given_x = given >= 0 ? logit(x, allowed, (uint32_t)given, n) : kNone;

    Share w{{kLowest, 0.0f, 0.0f}, 0};
    List list{TOP ? lists[wave] : nullptr, TOP ? best[wave] : nullptr, 0, kNone, kNone};
    __shared__ float wave_bars[WAVES];
    uint32_t first_in_front = 0;      // of given class 0, by this lane's classes
    // (the first time round also without a class: all waves set the bar together)
    for (bool first = true; first || base < end; base += kChunk, first = false) {
        float v[kPer];
        raw.template logits<MASK>(v, base, lane, end);
        if (base + kChunk < end) raw.template load<MASK>(x, allowed, base + kChunk, lane, mem_end);
        float most = v[0];
#pragma unroll
        for (uint32_t i = 1; i < kPer; ++i) most = fmaxf(most, v[i]);
        w.sums.rebase(fmaxf(w.sums.m, most), s.exp2_scale);
#pragma unroll
        for (uint32_t i = 0; i < kPer; ++i) {
            const float h = half_below(v[i], w.sums.m) * s.exp2_scale;
            const float e = __builtin_amdgcn_exp2f(h);
            w.sums.s += e;
            w.sums.u = fmaf(fmaxf(h, kNothing), e, w.sums.u);
        }
        if (a.given_ranks)
            for (uint32_t g = 0; g < a.n_given; ++g) {
                const float at = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, given_x), g));
                const uint32_t c = (uint32_t)__builtin_amdgcn_readlane(given, g);
                uint32_t count = 0;               // of this lane
                if (c < base) {
#pragma unroll
                    for (uint32_t i = 0; i < kPer; ++i) count += v[i] > at;
                } else if (c >= base + kChunk) {
#pragma unroll
                    for (uint32_t i = 0; i < kPer; ++i) count += v[i] >= at;
                } else {
#pragma unroll
                    for (uint32_t i = 0; i < kPer; ++i) count += v[i] > at || (v[i] == at && R::first(base, i / R::kVec, lane) + i % R::kVec < c);
                }
                if (g == 0) first_in_front += count;
                else {
                    count = wave_total(count);
                    if (lane == g) w.in_front += count;
                }
            }
        if constexpr (TOP) {
            list.bar = list.next;
            if (first) {
                // (classes of other waves that reach it come behind this wave's next chunk: an equal one there has to get in)
                const float all = bar_of_all<WAVES>(most, a.top, wave_bars, wave);
                list.raise(WAVES == 1 ? all : below(all));
            }
            const uint64_t lanes = __ballot(most > list.bar);
            if (lanes) {
                if (!first && (uint32_t)__popcll(lanes) >= a.top) list.raise(bar_of(most, a.top));
                uint32_t mine = 0;
#pragma unroll
                for (uint32_t i = 0; i < kPer; ++i) mine |= v[i] > list.bar ? 1u << i : 0;
                if (list.n <= kListRoom && !__ballot((mine & (mine - 1)) != 0)) {       // mostly: one of a lane's at most, its largest
                    const uint32_t i = mine ? __builtin_ctz(mine) : 0;
                    list.append(mine != 0, order_key(most, R::first(base, i / R::kVec, lane) + i % R::kVec));
                    mine = 0;
                }
#pragma nounroll
                while (__ballot(mine != 0)) {
                    const uint32_t i = mine ? __builtin_ctz(mine) : 0;
                    float one = v[0];
#pragma unroll
                    for (uint32_t j = 1; j < kPer; ++j) one = i == j ? v[j] : one;
                    if (list.n > kListRoom) list.cut(a.top, lane);
                    list.append(mine != 0 && one > list.bar, order_key(one, R::first(base, i / R::kVec, lane) + i % R::kVec));
                    mine &= mine - 1;
                }
            }
        }
    }
    first_in_front = wave_total(first_in_front);
    if (lane == 0) w.in_front += first_in_front;
    w.sums.over_wave(s.exp2_scale);
    // The waves' shares to wave 0, the entries of all lists to their places; then, in a row of several parts, the same with what they handed over.
    __shared__ Sums wave_sums[WAVES];
    __shared__ uint32_t wave_n[WAVES], wave_front[WAVES][MT_SCORE_MAX_GIVEN], last;
    for (bool parts_joined = !PARTS;; parts_joined = true) {
        if constexpr (TOP) if (lane < kStep) list.at[list.n + lane] = 0;
        if constexpr (WAVES > 1) {
            if (lane == 0) { wave_sums[wave] = w.sums; wave_n[wave] = list.n; }
            if (lane < MT_SCORE_MAX_GIVEN) wave_front[wave][lane] = w.in_front;
            __syncthreads();
        } else wave_sync();
        uint32_t n = list.n;
        if constexpr (TOP) {
            if constexpr (WAVES > 1) {
                n = 0;
#pragma unroll
                for (uint32_t o = 0; o < WAVES; ++o) n += wave_n[o];
            }
            n = min(n, a.top);
#pragma nounroll
            for (uint32_t j = 0; j < list.n; j += 64) {
                const uint64_t own = j + lane < list.n ? list.at[j + lane] : 0;
                uint32_t before = 0;
#pragma nounroll
                for (uint32_t o = 0; o < WAVES; ++o) {
                    const uint32_t others = WAVES > 1 ? wave_n[o] : list.n;
#pragma nounroll
                    for (uint32_t i = 0; i < others; i += kStep) before += in_front_of(own, lists[WAVES > 1 ? o : wave] + i);
                }
                if (own && before < a.top) best[WAVES > 1 ? 0 : wave][before] = own;
            }
            if constexpr (WAVES > 1) __syncthreads(); else wave_sync();
        }
        if constexpr (WAVES > 1) {
            if (wave == 0) {
#pragma unroll
                for (uint32_t o = 1; o < WAVES; ++o) {
                    w.sums.join(wave_sums[o], s.exp2_scale);
                    if (lane < MT_SCORE_MAX_GIVEN) w.in_front += wave_front[o][lane];
                }
            }
        }
        list.n = n;
        if (parts_joined) break;
        if constexpr (PARTS) {
            // the last workgroup of a row to come here joins the parts of all of them
            uint32_t* tickets = (uint32_t*)a.scratch;
            Part* parts = (Part*)((uint8_t*)a.scratch + kRecords * 4) + (uint64_t)row * s.parts;
            if (wave == 0) {
                Part& p = parts[part];
                if (lane == 0) { hand_over(&p.m, w.sums.m); hand_over(&p.s, w.sums.s); hand_over(&p.u, w.sums.u); }
                if (lane < a.n_given) hand_over(&p.in_front[lane], w.in_front);
                if constexpr (TOP) if (lane < a.top) hand_over(&p.keys[lane], lane < list.n ? best[0][lane] : 0);
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                if (lane == 0) last = __hip_atomic_fetch_add(&tickets[row], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == s.parts - 1;
            }
            __syncthreads();
            if (!last) return;
            if (threadIdx.x == 0) hand_over(&tickets[row], 0u);   // ready for the next call
            // wave v takes parts v, v + 4, ..., a lane each; of their keys every lane takes some
            w = Share{{kLowest, 0.0f, 0.0f}, 0};
            const uint32_t mine = (s.parts - wave + WAVES - 1) / WAVES;
            uint64_t keys[kPartKeys];
            if constexpr (TOP) {
#pragma unroll
                for (uint32_t j = 0; j < kPartKeys; ++j) {
                    const uint32_t i = 64 * j + lane;
                    keys[j] = i < mine * a.top ? take_over(&parts[wave + i / a.top * WAVES].keys[i % a.top]) : 0;
                }
            }
            const bool has = lane < mine;
            const Part& p = parts[has ? wave + lane * WAVES : 0];
            if (has) w.sums = Sums{take_over(&p.m), take_over(&p.s), take_over(&p.u)};
            if (a.given_ranks)
                for (uint32_t g = 0; g < a.n_given; ++g) {
                    const uint32_t count = wave_total(has ? take_over(&p.in_front[g]) : 0u);
                    if (lane == g) w.in_front = count;
                }
            w.sums.over_wave(s.exp2_scale);
            if constexpr (TOP) {
                list.n = 0; list.bar = list.next = kNone;
                float most = kNone;
#pragma unroll
                for (uint32_t j = 0; j < kPartKeys; ++j) if (keys[j]) most = fmaxf(most, key_logit(keys[j]));
                list.raise(bar_of_all<WAVES>(most, a.top, wave_bars, wave));
#pragma nounroll
                for (uint32_t j = 0; j * 64 < mine * a.top; ++j) {
                    uint64_t one = keys[0];
#pragma unroll
                    for (uint32_t k = 1; k < kPartKeys; ++k) one = j == k ? keys[k] : one;
                    if (list.n > kListRoom) list.cut(a.top, lane);
                    list.append(one && key_logit(one) > list.bar, one);
                }
                __syncthreads();                  // (the lists and `best` are read no more)
            }
        }
    }
    if (WAVES > 1 && wave != 0) return;

    // (the largest logit's own term is 1: without a class the sum is 0, with a NaN or +infinity among them it is NaN)
    const bool some = w.sums.s != 0.0f, lost = some && !(w.sums.s < __builtin_inff());
    const float log_s = logf(w.sums.s), nan = __builtin_nanf("");
    if (lane == 0 && a.entropy) a.entropy[row] = lost ? nan : some ? log_s - 0.69314718f * (w.sums.u / w.sums.s) : 0.0f;
    if (lane < a.n_given) {
        const bool there = given_x != kNone;
        const uint64_t to = (uint64_t)row * a.n_given + lane;
        if (a.given_logprobs) a.given_logprobs[to] = !there ? kNone : lost ? nan : log_prob(given_x, w.sums.m, s.inv_t, log_s);
        if (a.given_ranks) a.given_ranks[to] = there && !lost ? (int32_t)w.in_front : -1;
    }
    if constexpr (TOP) {
        if (lane < a.top) {
            const uint64_t key = lane < list.n && !lost ? best[WAVES > 1 ? 0 : wave][lane] : 0;
            const uint64_t to = (uint64_t)row * a.top + lane;
            if (a.top_ids) a.top_ids[to] = key ? key_class(key) : -1;
            if (a.top_logprobs) a.top_logprobs[to] = key ? log_prob(key_logit(key), w.sums.m, s.inv_t, log_s) : lost ? nan : kNone;
        }
    }
}

template <typename T, bool TOP, bool MASK>
hipError_t go(const ScoreArgs& s, hipStream_t st)
{
    // A wave to a row where rows are short, or many for their length (us, four waves / one, 5 alternatives, fp32 and bf16: 256 rows of 1000 classes 7.9 / 6.3 and
    // 7.9 / 6.3, of 4000 7.8 / 11.1 and 7.5 / 9.7; 1024 rows of 2000 10.3 / 8.8 and 9.9 / 8.0, of 4000 11.4 / 13.0 and 10.7 / 11.0, of 8192 15.6 / 17.9 and 13.9 / 14.7, of
    // 10000 18.0 / 22.1 and 17.4 / 16.9, of 16384 21.1 / 28.3 and 18.5 / 21.9; 2048 rows of 4000 17.8 / 15.0 and 17.0 / 13.2, of 12000 31.5 / 31.4 and 30.9 / 23.2, of 24576
    // 47.8 / 52.0 and 38.2 / 35.8).  fp32, with more bytes to wait for, needs two waves to every SIMD.
    const bool many = sizeof(T) == 4 ? s.a.rows >= 2048 && s.a.classes <= 12 * kSome
                                     : s.a.classes <= 24 * kSome && s.a.classes <= (s.a.classes <= kWaves * kSome ? 3 : 10) * (uint64_t)s.a.rows;
    const bool alone = s.a.classes <= 2 * kSome || many;
    // bf16: 32 classes a lane at a time keep the memory busy (2048 rows of 32768 48.8 -> 46.0 us, 256 rows 18.5 -> 15.8), 16 where those are all that a wave has (one row of
    // 1000 5.7 -> 4.5, 256 rows of 4096 9.2 -> 7.4) and where workgroups share a row.
    const bool short_steps = sizeof(T) == 2 && s.a.classes <= (alone ? 1 : kWaves) * kSome;
    constexpr uint32_t kShort = sizeof(T) == 2 ? 2 : 4;
    const dim3 rows(s.a.rows), fours((s.a.rows + kWaves - 1) / kWaves);
    constexpr uint32_t threads = 64 * kWaves;
    if (s.parts > 1) return launch(score_kernel<T, TOP, MASK, kWaves, true, kShort>, dim3(s.a.rows, s.parts), threads, 0, st, s);
    if (alone) return launch(short_steps ? score_kernel<T, TOP, MASK, 1, false, kShort> : score_kernel<T, TOP, MASK, 1, false, 4>, fours, threads, 0, st, s);
    return launch(short_steps ? score_kernel<T, TOP, MASK, kWaves, false, kShort> : score_kernel<T, TOP, MASK, kWaves, false, 4>, rows, threads, 0, st, s);
}

template <typename T>
hipError_t choose(const ScoreArgs& s, hipStream_t st)
{
    const bool top = s.a.top_ids || s.a.top_logprobs, mask = s.a.allowed != nullptr;
    if (top) return mask ? go<T, true, true>(s, st) : go<T, true, false>(s, st);
    return mask ? go<T, false, true>(s, st) : go<T, false, false>(s, st);
}

template <typename T>
hipError_t all_rows(ScoreArgs s, hipStream_t st)
{
    mt_score_args& a = s.a;
    for (uint32_t left = a.rows;; left -= kRowsAtOnce) {
        a.rows = std::min(left, kRowsAtOnce);
        const hipError_t e = choose<T>(s, st);
        if (e != hipSuccess || left <= kRowsAtOnce) return e;
        const uint64_t n = kRowsAtOnce;           // (so many rows are never shared: no scratch)
        a.logits = (const T*)a.logits + n * a.row_stride;
        move_rows(a.n_classes, n);
        move_rows(a.allowed, n * a.allowed_stride);
        move_rows(a.given, n * a.n_given);
        move_rows(a.given_logprobs, n * a.n_given);
        move_rows(a.given_ranks, n * a.n_given);
        move_rows(a.entropy, n);
        move_rows(a.top_ids, n * a.top);
        move_rows(a.top_logprobs, n * a.top);
    }
}

}  // namespace

// A row's classes are shared where there are not enough rows to fill the machine: a part leaves at least a chunk to every wave.  Handing over costs some 4 us,
// and few parts save little (us whole / in parts, 5 alternatives, fp32 and bf16: one row of 16384 10.2 / 10.4 and 9.4 / 10.4, of 24576 12.8 / 10.8 and 10.4 / 10.9, of 65536
// 22.9 / 10.9 and 18.7 / 10.8; 128 rows of 16384 12.6 / 12.8 and 11.2 / 12.8, of 24576 16.0 / 14.8 and 13.3 / 14.2, of 65536 31.7 / 23.5 and 22.8 / 18.7; 256 rows, in four,
// of 32768 20.6 / 20.3 and 16.0 / 19.4, of 65536 35.4 / 29.8 and 23.3 / 24.3, of 131072 65.8 / 43.4 and 39.6 / 33.8).  More work in a row pays sooner: with eight given
// classes 128 rows of 9216 12.6 / 10.1 and 16.3 / 10.0, 256 rows 13.0 / 11.6 and 16.7 / 11.2; with 20 alternatives 256 rows of 32768 30.9 / 21.3 and 23.2 / 20.4.
void score_split(uint32_t rows, uint32_t classes, uint32_t n_given, uint32_t top, uint32_t* parts, uint32_t* part_len)
{
    *parts = 1; *part_len = classes;
    if (rows == 0) return;
    const uint32_t span = kSome * kWaves, spans = (classes + span - 1) / span, want = std::min(kMaxParts, kRecords / rows);
    if (want < 3 || spans < (n_given >= 4 ? 3u : want >= 8 ? 5u : top > 8 ? 8u : 16u)) return;
    *part_len = (spans + want - 1) / want * span;
    *parts = (uint32_t)(((uint64_t)classes + *part_len - 1) / *part_len);
}

uint64_t score_scratch_bytes(uint32_t rows, uint32_t classes, uint32_t n_given, uint32_t top)
{
    uint32_t parts, part_len;
    score_split(rows, classes, n_given, top, &parts, &part_len);
    return parts > 1 ? kRecords * (4 + sizeof(Part)) : 0;
}

hipError_t launch_score(const ScoreArgs& a, hipStream_t s)
{
    return a.a.dtype == MT_BF16 ? all_rows<__bf16>(a, s) : all_rows<float>(a, s);
}

}  // namespace mt

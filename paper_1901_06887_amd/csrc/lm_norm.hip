// mt_add_norm: residual addition, root-mean-square norm and the 8-bit rows, one pass over memory.
//
// h = x + r, y = h * rsqrt(mean(h^2) + eps) * gain, q = e4m3(y / 2^e) with the least e >= -126 for which no |y| of the
// 32 values exceeds 448 * 2^e.  A row is read once and stays in registers between the sum of squares and the outputs; a lane
// holds runs of eight consecutive elements, so a block of 32 is four neighbouring lanes and its maximum two cross-lane moves.  Memory bounds it: 8192 rows of
// 4096 bf16, residual, sum, norm and 8-bit rows 53.5 us, 5.7 TB/s.  One row of 1024 takes 2.5 us, which is the launch and two trips to memory; 333 rows of 1531 fp32
// values 5.1 us (1.7 TB/s: rows that start anywhere, and their ends element by element).
#include "lm_device.h"

namespace mt {
namespace {

constexpr uint32_t kRun = 8;                  // consecutive elements of a lane
// Outputs of more than what the L2s hold (8 x 4 MiB) go past them: 8192 rows of 4096 bf16, sum, norm and 8-bit rows, 65.5 -> 59.7 us, of 2048 30.0 -> 22.7.
constexpr uint64_t kStreamBytes = 32ull << 20;

// 2^e for -126 <= e <= 127
__device__ __forceinline__ float power(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

// e for a block whose largest magnitude is `most` (not NaN, not infinite): 448 is 1.75 * 2^8
__device__ __forceinline__ int block_exponent(float most)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, most);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return most > 0.0f ? max(e, -126) : 0;
}

template <typename T>
struct NormRow {
    const T* x; const T* residual; const float* gain;
    T* sum; T* y; uint8_t* y8; uint8_t* y8_scales;
    bool known;                               // the row's gain exists
};

template <typename T>
__device__ __forceinline__ NormRow<T> norm_row(const mt_norm_args& a, uint32_t row)
{
    NormRow<T> r;
    r.x = (const T*)a.x + row * a.x_stride;
    r.residual = a.residual ? (const T*)a.residual + row * a.residual_stride : nullptr;
    r.known = true;
    uint32_t id = 0;
    if (a.gain_ids) { id = (uint32_t)a.gain_ids[row]; r.known = id < a.n_gains; }
    r.gain = a.gain && r.known ? a.gain + id * a.gain_stride : nullptr;
    r.sum = a.sum ? (T*)a.sum + row * a.sum_stride : nullptr;
    r.y = a.y ? (T*)a.y + row * a.y_stride : nullptr;
    r.y8 = a.y8 ? a.y8 + row * a.y8_stride : nullptr;
    r.y8_scales = a.y8_scales ? a.y8_scales + row * a.y8_scales_stride : nullptr;
    return r;
}

// A lane's run of the row at `at`: h in fp32, zeros past the width.
template <typename T>
__device__ __forceinline__ void load_run(const NormRow<T>& r, uint32_t at, uint32_t width, float (&h)[kRun])
{
    if (at + kRun <= width) {
        load8(r.x + at, h);
        if (r.residual) {
            float q[kRun];
            load8(r.residual + at, q);
#pragma unroll
            for (uint32_t i = 0; i < kRun; ++i) h[i] += q[i];
        }
        return;
    }
    const uint32_t n = at < width ? width - at : 0;
    load_some(r.x + at, n, h);
    if (r.residual) {
        float q[kRun];
        load_some(r.residual + at, n, q);
#pragma unroll
        for (uint32_t i = 0; i < kRun; ++i) h[i] += q[i];
    }
}

// What h is multiplied by: a power of two, then the rest.  They are apart because together they can leave fp32's range where the outputs do not.
struct RowScale { float power, rest; };

// Everything behind the mean: the run's sum, norm and 8-bit values.  All lanes of a block come here together.
template <bool STREAM, typename T>
__device__ __forceinline__ void finish_run(const NormRow<T>& r, uint32_t at, uint32_t width, const float (&h)[kRun], RowScale scale)
{
    const uint32_t n = at >= width ? 0 : width - at < kRun ? width - at : kRun;
    float y[kRun], g[kRun];
    if (r.gain) {
        if (n == kRun) load8(r.gain + at, g); else load_some(r.gain + at, n, g);
    }
#pragma unroll
    for (uint32_t i = 0; i < kRun; ++i) {
        y[i] = h[i] * scale.power * scale.rest;
        if (r.gain) y[i] *= g[i];
        if (!r.known || i >= n) y[i] = 0.0f;
    }
    if (r.sum && n) { if (n == kRun) store8<STREAM>(r.sum + at, h); else store_some(r.sum + at, n, h); }
    if (r.y && n) { if (n == kRun) store8<STREAM>(r.y + at, y); else store_some(r.y + at, n, y); }
    if (!r.y8) return;
    // magnitudes as integers: they order like the values, and a NaN stays above every number
    uint32_t most = 0;
#pragma unroll
    for (uint32_t i = 0; i < kRun; ++i) most = max(most, __builtin_bit_cast(uint32_t, y[i]) & 0x7fffffffu);
    most = max(most, (uint32_t)__shfl_xor((int)most, 1));
    most = max(most, (uint32_t)__shfl_xor((int)most, 2));
    const bool finite = most < 0x7f800000u;
    const int e = finite ? block_exponent(__builtin_bit_cast(float, most)) : 0;
    const float down = power(-e);             // e is at most 119 + 1
    uint32_t q[2];
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
        int w = 0;
        w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i] * down, y[4 * i + 1] * down, w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2] * down, y[4 * i + 3] * down, w, true);
        q[i] = finite ? (uint32_t)w : 0x7f7f7f7fu;
    }
    if (n == kRun) {
        Any<uint8_t>::vec8* to = (Any<uint8_t>::vec8*)(r.y8 + at);
        const u32x2 w = {q[0], q[1]};
        if constexpr (STREAM) __builtin_nontemporal_store(w, to); else *to = w;
    } else
#pragma unroll
        for (uint32_t i = 0; i < kRun; ++i) if (i < n) r.y8[at + i] = (uint8_t)(q[i / 4] >> (8 * (i % 4)));
    if (n && at % MT_MX_BLOCK == 0) r.y8_scales[at / MT_MX_BLOCK] = finite ? (uint8_t)(e + 127) : 0xff;
}

// Over the threads of a row, of what 0 changes nothing; `part`: LDS of a workgroup that has one row.
template <bool MULTI, typename F>
__device__ __forceinline__ uint32_t row_fold(uint32_t v, uint32_t* part, uint32_t t, uint32_t threads, F f)
{
    v = wave_fold(v, f);
    if constexpr (MULTI) {
        if ((t & 63) == 0) part[t >> 6] = v;
        __syncthreads();
        v = 0;
        for (uint32_t w = 0; w < threads / 64; ++w) v = f(v, part[w]);
    }
    return v;
}

// Workgroups of the threads that a row needs (MULTI), or of four waves with a row each.  A thread holds RUNS runs of its row in registers, run j of thread t
// at (j * threads + t) * 8.  LOOP: a row that no workgroup holds is read a second time for the outputs.  STREAM: outputs past the caches.
template <typename T, bool MULTI, uint32_t RUNS, bool LOOP, bool STREAM>
__global__ void __launch_bounds__(MULTI ? 1024 : 256) norm_kernel(mt_norm_args a)
{
    // (asked for in one go: loads where they are used are as many trips to memory one after the other; one row of 1024 2.7 -> 2.5 us, many rows are 1 % slower)
    if constexpr (!STREAM) asm volatile("" :: "s"(a.x), "s"(a.residual), "s"(a.gain), "s"(a.gain_ids), "s"(a.sum), "s"(a.y), "s"(a.y8), "s"(a.y8_scales), "s"(a.x_stride), "s"(a.residual_stride),
                 "s"(a.gain_stride), "s"(a.rows), "s"(a.width), "s"(a.n_gains), "s"(a.eps));
    const uint32_t threads = MULTI ? blockDim.x : 64, span = threads * kRun;
    const uint32_t t = MULTI ? threadIdx.x : threadIdx.x & 63;
    const uint32_t row = MULTI ? blockIdx.x : blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= a.rows) return;                // (whole waves, and only where no barrier follows)
    const NormRow<T> r = norm_row<T>(a, row);
    float h[RUNS][kRun];
    float squares = 0.0f;
    for (uint32_t base = 0; base < (LOOP ? a.width : 1); base += RUNS * span) {
#pragma unroll
        for (uint32_t j = 0; j < RUNS; ++j) load_run(r, base + j * span + t * kRun, a.width, h[j]);
#pragma unroll
        for (uint32_t j = 0; j < RUNS; ++j)
#pragma unroll
            for (uint32_t i = 0; i < kRun; ++i) squares = fmaf(h[j][i], h[j][i], squares);
    }
    __shared__ __attribute__((aligned(16))) uint32_t part[3][MULTI ? 16 : 1];
    const auto add = [](uint32_t p, uint32_t q) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, p) + __builtin_bit_cast(float, q)); };
    squares = __builtin_bit_cast(float, row_fold<MULTI>(__builtin_bit_cast(uint32_t, squares), part[0], t, threads, add));
    RowScale scale{1.0f, 0.0f};
    // Squares beyond fp32's range, or so small that bits of them that count lie below it (2^24 squares lose 2^-126 together): the row is read once more, and its
    // values are brought near 1 by a power of two.  An infinity's row stays as it is, and a row of zeros.  (One comparison, whose rare side lies behind the kernel's code;
    // one row of 1024 2.46 -> 2.53 us.)
    constexpr uint32_t kLeast = 27u << 23, kInfinity = 0x7f800000u;       // 2^-100
    const bool fine = __builtin_bit_cast(uint32_t, squares) - kLeast < kInfinity - kLeast;
    if (__builtin_expect(!fine, 0) && (squares > 1.0f || (squares >= 0.0f && a.eps < 0x1p-100f))) {
        const auto again = [&](auto of_value) {
#pragma nounroll
            for (uint32_t at = t * kRun; at < a.width; at += span) {
                float v[kRun];
                load_run(r, at, a.width, v);
#pragma unroll
                for (uint32_t i = 0; i < kRun; ++i) of_value(v[i]);
            }
        };
        uint32_t most = 0;
        again([&](float v) { most = max(most, __builtin_bit_cast(uint32_t, v) & 0x7fffffffu); });
        most = row_fold<MULTI>(most, part[1], t, threads, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
        if (most != 0 && most < kInfinity) {
            int e = (int)(most >> 23) - 127;
            if (a.eps > 0.0f) e = max(e, ((int)(__builtin_bit_cast(uint32_t, a.eps) >> 23) - 127) >> 1);       // (eps, too, is brought down to 4 at most)
            scale.power = power(-min(max(e, -126), 126));
            squares = 0.0f;
            again([&](float v) { squares = fmaf(v * scale.power, v * scale.power, squares); });
            squares = __builtin_bit_cast(float, row_fold<MULTI>(__builtin_bit_cast(uint32_t, squares), part[2], t, threads, add));
        }
    }
    // (behind the branch: the gain is asked for with it)
    scale.rest = 1.0f / __builtin_sqrtf(squares / (float)a.width + a.eps * scale.power * scale.power);
    for (uint32_t base = 0; base < (LOOP ? a.width : 1); base += RUNS * span) {
#pragma unroll
        for (uint32_t j = 0; j < RUNS; ++j) {
            const uint32_t at = base + j * span + t * kRun;
            if (LOOP) load_run(r, at, a.width, h[j]);
            finish_run<STREAM>(r, at, a.width, h[j], scale);
        }
    }
}

template <typename T, bool MULTI, uint32_t RUNS, bool LOOP = false>
hipError_t go(const mt_norm_args& a, bool stream, hipStream_t s)
{
    const uint32_t grid = MULTI ? a.rows : (a.rows + 3) / 4;
    const uint32_t need = (a.width + kRun * RUNS - 1) / (kRun * RUNS);
    const uint32_t threads = MULTI ? std::min<uint32_t>((need + 63) / 64 * 64, 1024) : 256;
    return launch(stream ? norm_kernel<T, MULTI, RUNS, LOOP, true> : norm_kernel<T, MULTI, RUNS, LOOP, false>, dim3(grid), threads, 0, s, a);
}

template <typename T>
hipError_t choose(const mt_norm_args& a, hipStream_t s)
{
    const uint64_t outputs = (uint64_t)a.rows * a.width * ((a.sum ? sizeof(T) : 0) + (a.y ? sizeof(T) : 0) + (a.y8 ? 1 : 0));
    const bool stream = outputs > kStreamBytes;
    // (one run a thread: with two, 8192 rows of 4096 take 58.5 us instead of 53.8, one row of 4096 3.7 instead of 2.8)
    if (a.width <= 512) return go<T, false, 1>(a, stream, s);
    if (a.width <= 8192) return go<T, true, 1>(a, stream, s);
    if (a.width <= 16384) return go<T, true, 2>(a, stream, s);
    return go<T, true, 2, true>(a, stream, s);
}

template <typename T>
hipError_t all_rows(mt_norm_args a, hipStream_t s)
{
    for (uint32_t left = a.rows;; left -= kRowsAtOnce) {
        a.rows = std::min(left, kRowsAtOnce);
        const hipError_t e = choose<T>(a, s);
        if (e != hipSuccess || left <= kRowsAtOnce) return e;
        const uint64_t n = kRowsAtOnce;
        a.x = (const T*)a.x + n * a.x_stride;
        if (a.residual) a.residual = (const T*)a.residual + n * a.residual_stride;
        move_rows(a.gain_ids, n);
        if (a.sum) a.sum = (T*)a.sum + n * a.sum_stride;
        if (a.y) a.y = (T*)a.y + n * a.y_stride;
        move_rows(a.y8, n * a.y8_stride);
        move_rows(a.y8_scales, n * a.y8_scales_stride);
    }
}

}  // namespace

hipError_t launch_norm(const mt_norm_args& a, hipStream_t s)
{
    return a.dtype == MT_BF16 ? all_rows<__bf16>(a, s) : all_rows<float>(a, s);
}

}  // namespace mt

// Host side of the operators behind language models' answers: argument checks, the 4-bit matrices in a context's
// weight arena, and the grouping of a call's rows into launches.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "lm_internal.h"
#include "../../include/mt_debug.h"

using namespace mt;

namespace {

constexpr uint32_t kMaxFeatures = 1u << 24;
constexpr uint32_t kMinScale4 = 27, kMaxScale4 = 227;       // 2^-100 .. 2^100: no weight and no product of ordinary values leaves fp32's normal range
constexpr uint64_t kMaxGrid = 0xffffffffu / 512;         // a grid holds fewer than 2^32 threads

#define LM_TRY(c, expr)                                                                                                     \
    do {                                                                                                                    \
        const hipError_t e_ = (expr);                                                                                       \
        if (e_ != hipSuccess) {                                                                                             \
            (void)hipGetLastError();                                                                                        \
            return ctx_fail((c), e_ == hipErrorOutOfMemory ? MT_ENOMEM : MT_EDEVICE, "%s: %s", #expr, hipGetErrorString(e_)); \
        }                                                                                                                   \
    } while (0)

inline uint32_t div_up(uint32_t a, uint32_t b) { return (uint32_t)(((uint64_t)a + b - 1) / b); }

// The caller's matrix as tiles (Matrix4); `out` is zeroed.
void pack_matrix4(uint32_t N, uint32_t K, const uint8_t* codes, const uint8_t* scales, const float* bias, uint8_t* out)
{
    const uint32_t kt = div_up(K, kTile4K), nt = div_up(N, kTile4Rows);
    const size_t code_row = (size_t)K / 2 + (K & 1), scale_row = div_up(K, MT_MX_BLOCK);
    for (uint32_t n = 0; n < nt * kTile4Rows; ++n)
        for (uint32_t b = 0; b < kt * 4; ++b) {
            uint8_t* tile = out + ((size_t)(n / kTile4Rows) * kt + b / 4) * kTile4Bytes;
            const uint32_t lane = (b % 4) * kTile4Rows + n % kTile4Rows;
            const bool there = n < N && b < scale_row;
            tile[kTile4Codes + lane] = there ? scales[(size_t)n * scale_row + b] : 127;
            if (!there) continue;
            const size_t from = (size_t)b * 16, len = std::min<size_t>(16, code_row - from);
            std::memcpy(tile + lane * 16, codes + (size_t)n * code_row + from, len);
            if ((K & 1) && b + 1 == scale_row) tile[lane * 16 + len - 1] &= 0x0f;       // the half byte behind the last column
        }
    if (bias) std::memcpy(out + matrix4_tiles_bytes(N, K), bias, (size_t)N * 4);
}

uint64_t matrix4_bytes(uint32_t N, uint32_t K) { return matrix4_tiles_bytes(N, K) + (uint64_t)N * 4; }

bool bad_norm_stride(const void* p, uint64_t stride, uint64_t least) { return p && stride < least; }

}  // namespace

mt_status mt_add_norm(mt_ctx* c, void* hip_stream, const mt_norm_args* a)
{
    if (!c) return MT_EINVAL;
    if (!a) return ctx_fail(c, MT_EINVAL, "null arguments");
    const CtxView v = ctx_view(c);
    if (a->dtype > MT_BF16) return ctx_fail(c, MT_EUNSUPPORTED, "rows of dtype %u", a->dtype);
    if (a->rows && (!a->x || (!a->sum && !a->y && !a->y8))) return ctx_fail(c, MT_EINVAL, "null rows, or no output");
    if (a->rows && (a->y8 == nullptr) != (a->y8_scales == nullptr)) return ctx_fail(c, MT_EINVAL, "8-bit rows and their scales come together");
    if (a->width == 0) return ctx_fail(c, MT_EINVAL, "zero width");
    if (a->width > kMaxFeatures) return ctx_fail(c, MT_EUNSUPPORTED, "rows of %u elements", a->width);
    if (!(a->eps >= 0.0f) || !std::isfinite(a->eps)) return ctx_fail(c, MT_EINVAL, "eps is negative or not finite");
    if (a->gain && a->n_gains == 0) return ctx_fail(c, MT_EINVAL, "a gain, but n_gains is 0");
    if (a->gain_ids && !a->gain) return ctx_fail(c, MT_EINVAL, "gain_ids without a gain");
    const uint64_t w = a->width;
    if (a->x_stride < w || bad_norm_stride(a->residual, a->residual_stride, w) || bad_norm_stride(a->gain, a->gain_stride, w) ||
        bad_norm_stride(a->sum, a->sum_stride, w) || bad_norm_stride(a->y, a->y_stride, w) || bad_norm_stride(a->y8, a->y8_stride, w) ||
        bad_norm_stride(a->y8_scales, a->y8_scales_stride, div_up(a->width, MT_MX_BLOCK)))
        return ctx_fail(c, MT_EINVAL, "a stride is below the width %u", a->width);
    if (v.host_only) return ctx_fail(c, MT_ESTATE, "host-only context cannot run");
    if (a->rows == 0) return MT_OK;
    LM_TRY(c, hipSetDevice(v.device));
    LM_TRY(c, launch_norm(*a, (hipStream_t)hip_stream));
    return MT_OK;
}

mt_status mt_matrix4_footprint_get(uint32_t N, uint32_t K, uint64_t* bytes)
{
    if (!bytes || N == 0 || K == 0) return MT_EINVAL;
    if (N > kMaxFeatures || K > kMaxFeatures) return MT_EUNSUPPORTED;
    *bytes = (matrix4_bytes(N, K) + 255) / 256 * 256;
    return MT_OK;
}

mt_status mt_register_matrix4(mt_ctx* c, uint32_t N, uint32_t K, const uint8_t* codes, const uint8_t* scales, const float* bias, uint32_t* matrix)
{
    if (!c) return MT_EINVAL;
    if (!codes || !scales || !matrix || N == 0 || K == 0) return ctx_fail(c, MT_EINVAL, "null codes, scales or matrix, or no features");
    if (N > kMaxFeatures || K > kMaxFeatures) return ctx_fail(c, MT_EUNSUPPORTED, "%u x %u features", N, K);
    const size_t n_scales = (size_t)N * div_up(K, MT_MX_BLOCK);
    for (size_t i = 0; i < n_scales; ++i)
        if (scales[i] < kMinScale4 || scales[i] > kMaxScale4)
            return ctx_fail(c, MT_EUNSUPPORTED, "scale %u of output %zu is outside %u..%u", scales[i], i / div_up(K, MT_MX_BLOCK), kMinScale4, kMaxScale4);
    const CtxView v = ctx_view(c);
    Matrix4 m;
    m.used = true; m.N = N; m.K = K; m.len = matrix4_bytes(N, K);
    try {
        size_t at = 0;
        while (at < v.matrices->size() && (*v.matrices)[at].used) ++at;
        if (at == v.matrices->size()) v.matrices->push_back(Matrix4{});
        std::vector<uint8_t> image;
        if (!v.host_only) {
            image.assign((size_t)m.len, 0);
            pack_matrix4(N, K, codes, scales, bias, image.data());
            LM_TRY(c, hipSetDevice(v.device));
        }
        const mt_status st = ctx_arena_take(c, m.len, &m.off);
        if (st != MT_OK) return st;
        if (!v.host_only) {
            const hipError_t e = hipMemcpy(v.arena + m.off, image.data(), (size_t)m.len, hipMemcpyHostToDevice);
            if (e != hipSuccess) {
                ctx_arena_give(c, m.off, m.len);
                return ctx_fail(c, MT_EDEVICE, "upload of a matrix failed: %s", hipGetErrorString(e));
            }
        }
        (*v.matrices)[at] = m;
        *matrix = (uint32_t)at;
    } catch (const std::bad_alloc&) {
        return ctx_fail(c, MT_ENOMEM, "no host memory for a matrix of %llu bytes", (unsigned long long)m.len);
    }
    return MT_OK;
}

mt_status mt_unregister_matrix4(mt_ctx* c, uint32_t matrix)
{
    if (!c) return MT_EINVAL;
    const CtxView v = ctx_view(c);
    if (matrix >= v.matrices->size() || !(*v.matrices)[matrix].used) return ctx_fail(c, MT_ENOTFOUND, "no matrix %u", matrix);
    if (!v.host_only) {
        LM_TRY(c, hipSetDevice(v.device));
        LM_TRY(c, hipDeviceSynchronize());
    }
    ctx_arena_give(c, (*v.matrices)[matrix].off, (*v.matrices)[matrix].len);
    (*v.matrices)[matrix] = Matrix4{};
    return MT_OK;
}

mt_status mt_linear4(mt_ctx* c, void* hip_stream, const mt_linear4_args* a, const mt_row_group* groups, uint32_t n_groups)
{
    return mt_linear4_within(c, hip_stream, a, groups, n_groups, UINT32_MAX, UINT32_MAX);       // (as wide as the strides)
}

mt_status mt_linear4_within(mt_ctx* c, void* hip_stream, const mt_linear4_args* a, const mt_row_group* groups, uint32_t n_groups, uint32_t x_width, uint32_t y_width)
{
    if (!c) return MT_EINVAL;
    if (!a || (!groups && n_groups)) return ctx_fail(c, MT_EINVAL, "null arguments or groups");
    const CtxView v = ctx_view(c);
    if (a->x_dtype > MT_MX8 || a->y_dtype > MT_BF16) return ctx_fail(c, MT_EUNSUPPORTED, "rows of dtype %u to dtype %u", a->x_dtype, a->y_dtype);
    if (a->act > MT_ACT_GELU) return ctx_fail(c, MT_EUNSUPPORTED, "activation %u", a->act);
    if (a->rows && (!a->x || !a->y)) return ctx_fail(c, MT_EINVAL, "null rows");
    if (a->rows && (a->x_dtype == MT_MX8) != (a->x_scales != nullptr)) return ctx_fail(c, MT_EINVAL, "scales come with 8-bit rows, and only with them");
    uint64_t next = 0, row_tiles = 0;      // tiles of 16 outputs x 16 rows
    uint32_t most_rows = 0, most_k = 0;
    for (uint32_t g = 0; g < n_groups; ++g) {
        const mt_row_group& r = groups[g];
        if (r.matrix >= v.matrices->size() || !(*v.matrices)[r.matrix].used) return ctx_fail(c, MT_ENOTFOUND, "group %u: no matrix %u", g, r.matrix);
        const Matrix4& m = (*v.matrices)[r.matrix];
        if (r.first_row < next || (uint64_t)r.first_row + r.n_rows > a->rows)
            return ctx_fail(c, MT_EINVAL, "group %u: rows %u..%llu are out of order or outside the %u rows", g, r.first_row, (unsigned long long)r.first_row + r.n_rows, a->rows);
        if (a->x_stride < m.K || a->y_stride < m.N || (a->x_scales && a->x_scales_stride < div_up(m.K, MT_MX_BLOCK)))
            return ctx_fail(c, MT_EINVAL, "group %u: a stride is below the matrix's %u x %u", g, m.N, m.K);
        next = (uint64_t)r.first_row + r.n_rows;
        if (r.n_rows == 0) continue;
        if (x_width < m.K || y_width < m.N)
            return ctx_fail(c, MT_EINVAL, "group %u: rows of %u to %u columns are narrower than the matrix's %u x %u", g, x_width, y_width, m.N, m.K);
        most_rows = std::max(most_rows, r.n_rows);
        most_k = std::max(most_k, m.K);
        row_tiles += (uint64_t)div_up(m.N, kTile4Rows) * div_up(r.n_rows, kTile4Rows);
    }
    if (v.host_only) return ctx_fail(c, MT_ESTATE, "host-only context cannot run");
    if (most_rows == 0) return MT_OK;
    LM_TRY(c, hipSetDevice(v.device));

    const Linear4Shape shape = linear4_shape(row_tiles, most_rows, most_k, v.n_cus, a->x_dtype);
    Linear4Args<kGroups4> k;
    k.call = Linear4Call{v.arena, a->x, a->x_scales, a->y, a->x_stride, a->x_scales_stride, a->y_stride, a->act, 0, a->y_dtype == MT_BF16 ? 1u : 0u};
    uint64_t grid = 0;
    for (uint32_t g = 0; g < n_groups; ++g) {
        const mt_row_group& r = groups[g];
        if (r.n_rows == 0) continue;
        const Matrix4& m = (*v.matrices)[r.matrix];
        const uint64_t wgs = (uint64_t)div_up(m.N, kTile4Rows * shape.nt) * div_up(r.n_rows, kTile4Rows * shape.rt);
        if (wgs > kMaxGrid) return ctx_fail(c, MT_EUNSUPPORTED, "group %u takes %llu workgroups", g, (unsigned long long)wgs);
        if (k.call.n_groups == kGroups4 || grid + wgs > kMaxGrid) {
            LM_TRY(c, launch_linear4(k, shape, a->x_dtype, (uint32_t)grid, (hipStream_t)hip_stream));
            k.call.n_groups = 0; grid = 0;
        }
        k.groups[k.call.n_groups++] = Group4{m.off, m.N, m.K, r.first_row, r.n_rows, (uint32_t)grid};
        grid += wgs;
    }
    LM_TRY(c, launch_linear4(k, shape, a->x_dtype, (uint32_t)grid, (hipStream_t)hip_stream));
    return MT_OK;
}

int mt_debug_linear4_shape(uint64_t tiles, uint32_t most_rows, uint32_t most_k, uint32_t compute_units, uint32_t x_dtype, uint32_t* outputs, uint32_t* rows)
{
    const Linear4Shape s = linear4_shape(tiles, most_rows, most_k, compute_units, x_dtype);
    if (outputs) *outputs = s.nt * kTile4Rows;
    if (rows) *rows = s.rt * kTile4Rows;
    return s.through_lds ? 1 : 0;
}

mt_status mt_score_scratch_get(uint32_t rows, uint32_t classes, uint32_t n_given, uint32_t top, uint64_t* bytes)
{
    if (!bytes || classes == 0 || n_given > MT_SCORE_MAX_GIVEN || top > MT_SCORE_MAX_TOP) return MT_EINVAL;
    *bytes = score_scratch_bytes(rows, classes, n_given, top);
    return MT_OK;
}

mt_status mt_score(mt_ctx* c, void* hip_stream, const mt_score_args* a)
{
    if (!c) return MT_EINVAL;
    if (!a) return ctx_fail(c, MT_EINVAL, "null arguments");
    const CtxView v = ctx_view(c);
    if (a->dtype > MT_BF16) return ctx_fail(c, MT_EUNSUPPORTED, "logits of dtype %u", a->dtype);
    if (a->classes == 0 || a->classes > (uint32_t)INT32_MAX) return ctx_fail(c, MT_EINVAL, "%u classes", a->classes);
    if (a->n_given > MT_SCORE_MAX_GIVEN || a->top > MT_SCORE_MAX_TOP)
        return ctx_fail(c, MT_EINVAL, "%u given classes or %u alternatives are more than %u or %u", a->n_given, a->top, MT_SCORE_MAX_GIVEN, MT_SCORE_MAX_TOP);
    if (a->rows && !a->logits) return ctx_fail(c, MT_EINVAL, "null logits");
    if (a->rows == 0) {
        if (v.host_only) return ctx_fail(c, MT_ESTATE, "host-only context cannot run");
        return MT_OK;
    }
    if ((a->given != nullptr) != (a->n_given != 0) || (!a->given && (a->given_logprobs || a->given_ranks)))
        return ctx_fail(c, MT_EINVAL, "given classes, their number and their outputs come together");
    if (a->top == 0 && (a->top_ids || a->top_logprobs)) return ctx_fail(c, MT_EINVAL, "outputs for alternatives, but top is 0");
    if (!a->given_logprobs && !a->given_ranks && !a->entropy && !a->top_ids && !a->top_logprobs) return ctx_fail(c, MT_EINVAL, "no output");
    if (a->row_stride < a->classes || (a->allowed && a->allowed_stride < div_up(a->classes, 32)))
        return ctx_fail(c, MT_EINVAL, "a stride is below the %u classes", a->classes);
    if (!(a->temperature >= FLT_MIN) || !std::isfinite(a->temperature)) return ctx_fail(c, MT_EINVAL, "temperature is not positive, normal and finite");
    const uint64_t need = score_scratch_bytes(a->rows, a->classes, a->n_given, a->top);
    if (need && (!a->scratch || a->scratch_bytes < need || (uintptr_t)a->scratch % 16))
        return ctx_fail(c, MT_EINVAL, "the call needs %llu bytes of scratch on a 16-byte boundary", (unsigned long long)need);
    if (v.host_only) return ctx_fail(c, MT_ESTATE, "host-only context cannot run");
    LM_TRY(c, hipSetDevice(v.device));
    ScoreArgs k;
    k.a = *a;
    k.inv_t = (float)(1.0 / (double)a->temperature);
    k.exp2_scale = (float)(2.0 * 1.4426950408889634 / (double)a->temperature);       // (at 2^-126, the smallest, below 2^128)
    score_split(a->rows, a->classes, a->n_given, a->top, &k.parts, &k.part_len);
    LM_TRY(c, launch_score(k, (hipStream_t)hip_stream));
    return MT_OK;
}

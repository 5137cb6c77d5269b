// Shared between the host side of the operators behind language models' answers (lm_api.cpp, the context in mt_api.cpp) and their kernels (lm_*.hip).
// Not part of the public ABI.
#pragma once
#include <vector>

#include "mt_internal.h"

namespace mt {

// A 4-bit matrix as it lies in the arena: tiles of 16 outputs x 128 of the fan-in, [output tile][k tile], then the fp32 biases, zeros where there are none.
// A tile is one operand of the matrix instructions: lane l holds output l % 16 and the 32 values of k block l / 16, 16 bytes of
// codes in lane order, then 64 bytes of scales in lane order; outputs and k past the matrix are zero with scale 1.
constexpr uint32_t kTile4Rows = 16, kTile4K = 128, kTile4Codes = 1024, kTile4Bytes = kTile4Codes + 64;
struct Matrix4 {
    bool used = false;
    uint32_t N = 0, K = 0;
    uint64_t off = 0, len = 0;       // the arena block
};
inline __host__ __device__ uint64_t matrix4_tiles_bytes(uint32_t N, uint32_t K)
{
    return (uint64_t)((N + kTile4Rows - 1) / kTile4Rows) * ((K + kTile4K - 1) / kTile4K) * kTile4Bytes;
}
constexpr uint32_t kGroups4 = 64;    // groups of one launch: a lane each, and 2 KiB of kernel arguments
struct Group4 {
    uint64_t off;                    // arena offset of the matrix
    uint32_t N, K, row0, n_rows;
    uint32_t wg_base;                // workgroups of the launch's groups before this one
};
struct Linear4Call {
    const uint8_t* arena;
    const void* x; const uint8_t* x_scales; void* y;
    uint64_t x_stride, x_scales_stride, y_stride;
    uint32_t act, n_groups, y_bf16;
};
// What a kernel is given.  The small form is the front of the large one: with its 350 bytes of arguments instead of 2100 a call takes the host 4.0 us instead of 4.3.
constexpr uint32_t kFewGroups4 = 8;
template <uint32_t GROUPS> struct Linear4Args {
    Linear4Call call;
    Group4 groups[GROUPS];
};
static_assert(sizeof(Linear4Args<kGroups4>) <= 4096, "kernel arguments");
struct ScoreArgs {
    mt_score_args a;
    float inv_t, exp2_scale;         // 1 / temperature, and 2 log2(e) / temperature (finite)
    uint32_t parts, part_len;        // workgroups that share a row, and classes of one of them
};
// A launch and its error.
template <typename A, typename B> hipError_t launch(void (*kernel)(A), dim3 grid, uint32_t threads, uint32_t lds, hipStream_t s, const B& args)
{
    static_assert(sizeof(B) >= sizeof(A), "the kernel's arguments, or more behind them");
    void* p[] = {(void*)&args};
    return hipLaunchKernel((const void*)kernel, grid, dim3(threads), p, lds, s);
}
hipError_t launch_norm(const mt_norm_args& a, hipStream_t s);
struct Linear4Shape { uint32_t rt, nt; bool through_lds; };      // tiles of 16 rows and of 16 outputs that a workgroup serves, and how it takes its rows
Linear4Shape linear4_shape(uint64_t row_tiles, uint32_t most_rows, uint32_t most_k, uint32_t n_cus, uint32_t x_dtype);      // row_tiles: of 16 outputs x 16 rows
hipError_t prepare_linear4();      // once per device, before the first launch: lets kernels ask for more than 64 KiB of LDS
hipError_t launch_linear4(const Linear4Args<kGroups4>& a, Linear4Shape shape, uint32_t x_dtype, uint32_t grid, hipStream_t s);
void score_split(uint32_t rows, uint32_t classes, uint32_t n_given, uint32_t top, uint32_t* parts, uint32_t* part_len);
uint64_t score_scratch_bytes(uint32_t rows, uint32_t classes, uint32_t n_given, uint32_t top);
hipError_t launch_score(const ScoreArgs& a, hipStream_t s);

// What lm_api.cpp sees of a context (mt_api.cpp defines it).
struct CtxView {
    bool host_only;
    int device;
    uint32_t n_cus;
    uint8_t* arena;
    std::vector<Matrix4>* matrices;
};
CtxView ctx_view(mt_ctx* c);
mt_status ctx_fail(mt_ctx* c, mt_status st, const char* fmt, ...);
mt_status ctx_arena_take(mt_ctx* c, uint64_t len, uint64_t* off);   // in a cache context models give way; waits for the device there
void ctx_arena_give(mt_ctx* c, uint64_t off, uint64_t len);

}  // namespace mt

// Shared between the host side of the calls on language models' caches (lm_cache_api.cpp) and their kernels (lm_kv_write.hip, lm_attend.hip, lm_pages.hip, lm_sample.hip).
// Not part of the public ABI.
#pragma once
#include "lm_internal.h"

namespace mt {

struct KvWriteArgs {
    mt_kv_cache c;
    mt_kv_batch b;
    mt_kv_write_args a;
};
hipError_t launch_kv_write(const KvWriteArgs& a, hipStream_t s);

// Places (tokens of a sequence) that rows first .. last - 1 of a call fill, row r being token length - (after - r) of a table of `reach` tokens: begin .. stop - 1.
struct Places { int32_t begin, stop; };
inline __host__ __device__ Places places_of_rows(int32_t length, int32_t first, int32_t last, int32_t after, int32_t reach)
{
    const int32_t from = length - (after - first), to = length - (after - last);
    const Places p{from > 0 ? from : 0, to < reach ? to : reach};
    return p.begin < p.stop ? p : Places{0, 0};
}

struct AttendArgs {
    mt_kv_cache c;
    mt_kv_batch b;
    mt_attend_args a;
};
uint64_t attend_scratch_bytes(const mt_kv_cache& c, const mt_kv_batch& b, uint32_t q_heads, uint32_t max_length);
hipError_t launch_attend(const AttendArgs& a, hipStream_t s);

// A cache's work memory: the pages that a call moves, and what its steps hand to each other.
struct PageMoves { uint32_t n, held, pad[2]; };          // pairs that follow; pages held, where a call counts them
struct PageWork {
    PageMoves* head;
    int32_t* moves;          // [2 * most_moves]: from, to
    int32_t* map;            // [n_pages]: where a page went (of those that moved)
    uint32_t* was;           // [seqs]
};
inline __host__ __device__ uint64_t page_work_bytes(uint32_t n_pages, uint32_t seqs)
{
    const uint64_t moves = n_pages > seqs ? n_pages : seqs;
    return (sizeof(PageMoves) + 8 * moves + 4 * (uint64_t)n_pages + 4 * (uint64_t)seqs + 15) / 16 * 16;
}
inline __host__ __device__ PageWork page_work(const mt_kv_cache& c)
{
    const uint64_t moves = c.n_pages > c.seqs ? c.n_pages : c.seqs;
    PageWork w;
    w.head = (PageMoves*)c.work;
    w.moves = (int32_t*)(w.head + 1);
    w.map = w.moves + 2 * moves;
    w.was = (uint32_t*)(w.map + c.n_pages);
    return w;
}
struct PagesArgs {
    mt_kv_cache c;
    const int32_t *first, *second;       // the call's lists
    int32_t* out;
    uint32_t n;
};
hipError_t prepare_pages();      // once per device: lets kernels ask for more than 64 KiB of LDS
hipError_t launch_kv_grow(const PagesArgs& a, hipStream_t s);
hipError_t launch_kv_fork(const PagesArgs& a, hipStream_t s);
hipError_t launch_kv_free(const PagesArgs& a, hipStream_t s);
hipError_t launch_kv_compact(const PagesArgs& a, hipStream_t s);
hipError_t launch_kv_copy(const PagesArgs& a, hipStream_t s);

struct SampleArgs {
    mt_sample_args a;
};
hipError_t prepare_sample();     // once per device, as prepare_pages
hipError_t launch_sample(const SampleArgs& a, hipStream_t s);

}  // namespace mt

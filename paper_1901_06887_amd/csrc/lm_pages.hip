// Calls on the pages of a cache: room for tokens, forks, release, compaction, copies.
//
// What a call decides it decides in one workgroup: prefix sums over the list's entries say what each takes, one pass over the pages' counts finds
// the lowest-numbered free ones.  Whole numbers throughout, so results do not depend on timing.  Pages that move are then copied by the whole machine, from a list
// that the first launch leaves in the cache's work memory.
//
// The books are one workgroup's chains of trips to memory: release 2.2 us (one sequence) to 4.6 (thousands of pages), growth 3.6 to 8.7, a fork 6.1, compaction 6.8. The copies run at the rate of
// a large copy: 2 GB read and written in two launches of 210 us each, 5.0 TB/s.
#include "lm_cache_device.h"

namespace mt {
namespace {

constexpr uint32_t kThreads = 1024, kWaves = kThreads / 64;
constexpr uint32_t kNobody = 0xffffffffu;
constexpr uint32_t kRefs = 16;                    // counts that a thread looks at in one go

// Exclusive prefix sums over the workgroup; every thread gets the total.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* total, uint32_t* lds)
{
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63, upto = wave_inclusive_scan(v);
    __syncthreads();
    if (lane == 63) lds[wave] = upto;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) { const uint32_t n = lds[w]; all += n; before += w < wave ? n : 0; }
    *total = all;
    return before + upto - v;
}

// A thread's kRefs counts from page `first` on; 1 (held) behind the last.
__device__ __forceinline__ void load_refs(const int32_t* refs, uint32_t first, uint32_t n, int32_t (&v)[kRefs])
{
    if (first + kRefs <= n) {
#pragma unroll
        for (uint32_t i = 0; i < kRefs / 4; ++i) {
            const u32x4 w = *(const Any<float>::vec16*)(refs + first + 4 * i);
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) v[4 * i + e] = (int32_t)w[e];
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < kRefs; ++i) v[i] = first + i < n ? refs[first + i] : 1;
    }
}

// The first `want` free pages into `to`; returns how many of them there are.
__device__ uint32_t find_free(const mt_kv_cache& c, uint32_t want, int32_t* to, uint32_t* lds)
{
    uint32_t found = 0;
    for (uint32_t base = 0; base < c.n_pages && found < want; base += kThreads * kRefs) {
        int32_t v[kRefs];
        const uint32_t first = base + threadIdx.x * kRefs;
        load_refs(c.refs, min(first, c.n_pages), c.n_pages, v);
        uint32_t mine = 0, total;
#pragma unroll
        for (uint32_t i = 0; i < kRefs; ++i) mine += v[i] <= 0;
        uint32_t at = found + block_scan(mine, &total, lds);
#pragma unroll
        for (uint32_t i = 0; i < kRefs; ++i)
            if (v[i] <= 0) {
                if (at < want) to[at] = (int32_t)(first + i);
                ++at;
            }
        found = min(found + total, want);
    }
    __syncthreads();
    return found;
}

__device__ __forceinline__ uint32_t pages_for(uint64_t tokens, uint32_t page_tokens) { return (uint32_t)((tokens + page_tokens - 1) / page_tokens); }

// LDS of the kernels that take pages: who names a sequence first, then the scans' and the entries' words.
struct Entry { int32_t seq; uint32_t from, take, at; };       // table entries from, from + 1, ... take pages at, at + 1, ... of the free ones
struct Taking {
    uint32_t scan[kWaves];
    Entry entries[kThreads];
    uint32_t first_by[1];        // [seqs]
};

__device__ void name_firsts(Taking& t, const mt_kv_cache& c, const int32_t* seqs, uint32_t n)
{
    for (uint32_t s = threadIdx.x; s < c.seqs; s += kThreads) t.first_by[s] = kNobody;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
        const uint32_t s = seqs ? (uint32_t)seqs[i] : i;
        if (s < c.seqs) atomicMin(&t.first_by[s], i);
    }
    __syncthreads();
}

// What entry i of mt_kv_grow asks for.
struct Wish { int32_t seq; bool can; uint32_t have, take; int64_t length; };
__device__ __forceinline__ Wish grow_wish(const Taking& t, const PagesArgs& p, uint32_t i)
{
    Wish w{-1, false, 0, 0, 0};
    if (i >= p.n) return w;
    const uint32_t s = p.first ? (uint32_t)p.first[i] : i;
    if (s >= p.c.seqs || t.first_by[s] != i) return w;
    const int64_t tokens = p.second[i], was = max(p.c.lengths[s], 0);
    if (tokens < 0 || (was + tokens + p.c.page_tokens - 1) / p.c.page_tokens > p.c.table_width) return w;
    w.seq = (int32_t)s; w.can = true; w.length = was + tokens;
    w.have = pages_for(was, p.c.page_tokens);
    w.take = pages_for(w.length, p.c.page_tokens) - w.have;
    return w;
}

__global__ void __launch_bounds__(kThreads) grow_kernel(PagesArgs p)
{
    extern __shared__ Taking lds[];
    Taking& t = lds[0];
    const mt_kv_cache& c = p.c;
    const PageWork work = page_work(c);
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    name_firsts(t, c, p.first, p.n);
    uint64_t asked = 0;
    for (uint32_t base = 0; base < p.n; base += kThreads) {
        uint32_t total;
        block_scan(grow_wish(t, p, base + threadIdx.x).take, &total, t.scan);
        asked += total;
    }
    const uint32_t there = find_free(c, (uint32_t)min(asked, (uint64_t)c.n_pages), work.moves, t.scan);
    uint64_t given = 0;
    for (uint32_t base = 0; base < p.n; base += kThreads) {
        const Wish w = grow_wish(t, p, base + threadIdx.x);
        uint32_t total;
        const uint32_t before = block_scan(w.take, &total, t.scan);
        const bool granted = w.can && (w.take == 0 || given + before + w.take <= there);
        t.entries[threadIdx.x] = Entry{w.seq, w.have, granted ? w.take : 0, (uint32_t)(given + before)};
        __syncthreads();
        if (granted) c.lengths[w.seq] = (int32_t)w.length;
        if (p.out && base + threadIdx.x < p.n) p.out[base + threadIdx.x] = granted;
        for (uint32_t e = wave; e < min(kThreads, p.n - base); e += kWaves) {
            const Entry one = t.entries[e];
            for (uint32_t i = lane; i < one.take; i += 64) {
                const int32_t page = work.moves[one.at + i];
                c.table[(uint64_t)one.seq * c.table_stride + one.from + i] = page;
                c.refs[page] = 1;
            }
        }
        given += total;
        __syncthreads();
    }
}

__global__ void __launch_bounds__(kThreads) fork_kernel(PagesArgs p)
{
    extern __shared__ Taking lds[];
    Taking& t = lds[0];
    const mt_kv_cache& c = p.c;
    const PageWork work = page_work(c);
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    name_firsts(t, c, p.second, p.n);
    // (lengths as they are before the call: bit 31 says that the entry can be served)
    uint32_t asked = 0;
    for (uint32_t base = 0; base < p.n; base += kThreads) {
        const uint32_t i = base + threadIdx.x;
        uint32_t was = 0;
        if (i < p.n) {
            const uint32_t parent = (uint32_t)p.first[i], child = (uint32_t)p.second[i];
            if (parent < c.seqs && child < c.seqs && t.first_by[child] == i && c.lengths[child] == 0) {
                const uint32_t length = (uint32_t)max(c.lengths[parent], 0);
                if (pages_for(length, c.page_tokens) <= c.table_width) was = 1u << 31 | length;
            }
            work.was[i] = was;
        }
        asked += __syncthreads_count((was & 0x7fffffffu) % c.page_tokens != 0);
    }
    int32_t* free_pages = work.map;
    const uint32_t there = find_free(c, min(asked, c.n_pages), free_pages, t.scan);
    uint32_t given = 0;
    for (uint32_t base = 0; base < p.n; base += kThreads) {
        const uint32_t i = base + threadIdx.x, was = i < p.n ? work.was[i] : 0, length = was & 0x7fffffffu;
        const uint32_t take = length % c.page_tokens != 0;
        uint32_t total;
        const uint32_t before = block_scan(take, &total, t.scan);
        const bool granted = (was >> 31) && (take == 0 || given + before + take <= there);
        const int32_t child = granted ? p.second[i] : -1;
        t.entries[threadIdx.x] = Entry{child, length, granted ? 1u : 0u, given + before};
        __syncthreads();
        if (p.out && i < p.n) p.out[i] = granted;
        for (uint32_t e = wave; e < min(kThreads, p.n - base); e += kWaves) {
            const Entry one = t.entries[e];
            if (!one.take) continue;
            const int32_t* from = c.table + (uint64_t)(uint32_t)p.first[base + e] * c.table_stride;
            int32_t* to = c.table + (uint64_t)one.seq * c.table_stride;
            const uint32_t full = one.from / c.page_tokens;
            for (uint32_t j = lane; j < full; j += 64) {
                const int32_t page = from[j];
                to[j] = page;
                if ((uint32_t)page < c.n_pages) atomicAdd(&c.refs[page], 1);
            }
            if (lane == 0) {
                c.lengths[one.seq] = (int32_t)one.from;
                if (one.from % c.page_tokens) {
                    const int32_t page = free_pages[one.at];
                    work.moves[2 * one.at] = from[full];
                    work.moves[2 * one.at + 1] = page;
                    to[full] = page;
                    c.refs[page] = 1;
                }
            }
        }
        given += total;
        __syncthreads();
    }
    if (threadIdx.x == 0) work.head->n = min(given, there);
}

// A wave to an entry.
__global__ void __launch_bounds__(256) free_kernel(PagesArgs p)
{
    const mt_kv_cache& c = p.c;
    const uint32_t lane = threadIdx.x & 63, i = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i >= p.n) return;
    const uint32_t s = (uint32_t)p.first[i];
    if (s >= c.seqs) return;
    int32_t was = 0;
    if (lane == 0) was = atomicExch(&c.lengths[s], 0);        // (of a sequence that stands twice one entry finds the pages)
    was = __builtin_amdgcn_readfirstlane(was);
    const uint32_t held = min(pages_for((uint32_t)max(was, 0), c.page_tokens), c.table_width);
    for (uint32_t j = lane; j < held; j += 64) {
        int32_t* at = c.table + (uint64_t)s * c.table_stride + j;
        const int32_t page = *at;
        *at = -1;
        if ((uint32_t)page < c.n_pages) atomicSub(&c.refs[page], 1);
    }
}

__global__ void __launch_bounds__(kThreads) compact_kernel(PagesArgs p)
{
    __shared__ uint32_t scan[kWaves];
    const mt_kv_cache& c = p.c;
    const PageWork work = page_work(c);
    uint32_t held = 0;
    int32_t v[kRefs];
    for (uint32_t base = 0; base < c.n_pages; base += kThreads * kRefs) {
        const uint32_t first = base + threadIdx.x * kRefs;
        load_refs(c.refs, min(first, c.n_pages), c.n_pages, v);
        uint32_t mine = 0, total;
#pragma unroll
        for (uint32_t i = 0; i < kRefs; ++i) mine += first + i < c.n_pages && v[i] > 0;
        block_scan(mine, &total, scan);
        held += total;
    }
    uint32_t holes = 0, movers = 0;
    for (uint32_t base = 0; base < c.n_pages; base += kThreads * kRefs) {
        const uint32_t first = base + threadIdx.x * kRefs;
        load_refs(c.refs, min(first, c.n_pages), c.n_pages, v);
        uint32_t mine = 0, total;                 // free ones below `held` in the lower half, held ones from there on in the upper: 16384 at most of either
#pragma unroll
        for (uint32_t i = 0; i < kRefs; ++i) mine += first + i < held ? v[i] <= 0 : (uint32_t)(first + i < c.n_pages && v[i] > 0) << 16;
        const uint32_t before = block_scan(mine, &total, scan);
        uint32_t at_hole = holes + (before & 0xffff), at_mover = movers + (before >> 16);
        holes += total & 0xffff;
        movers += total >> 16;
#pragma unroll
        for (uint32_t i = 0; i < kRefs; ++i) {
            if (first + i < held && v[i] <= 0) work.moves[2 * at_hole++ + 1] = (int32_t)(first + i);
            if (first + i >= held && first + i < c.n_pages && v[i] > 0) work.moves[2 * at_mover++] = (int32_t)(first + i);
        }
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < movers; i += kThreads) {
        const int32_t from = work.moves[2 * i], to = work.moves[2 * i + 1];
        work.map[from] = to;
        c.refs[to] = c.refs[from];
        c.refs[from] = 0;
    }
    if (threadIdx.x == 0) {
        work.head->n = movers;
        work.head->held = held;
        if (p.out) *p.out = (int32_t)held;
    }
}

// The tables behind a compaction: a wave to a sequence.
__device__ void follow(const PagesArgs& p, const PageWork& work, uint32_t held)
{
    const mt_kv_cache& c = p.c;
    const uint32_t lane = threadIdx.x & 63, waves = gridDim.x * 4;
    for (uint32_t s = blockIdx.x * 4 + (threadIdx.x >> 6); s < c.seqs; s += waves) {
        const uint32_t n = min(pages_for((uint32_t)max(c.lengths[s], 0), c.page_tokens), c.table_width);
        for (uint32_t j = lane; j < n; j += 64) {
            int32_t* at = c.table + (uint64_t)s * c.table_stride + j;
            const uint32_t page = (uint32_t)*at;
            if (page >= held && page < c.n_pages) *at = work.map[page];
        }
    }
}

// Pages from and to of a list, whole: every workgroup takes pieces of kPiece bytes, 16 bytes a thread at a time.
constexpr uint32_t kPiece = 16384;
enum class Moves { kForked, kCompacted, kGiven, kClaimed };      // a list of the call's: every piece looks through what is behind its pair, or work.map says whose a page is
struct Block { uint8_t* base; uint64_t page, layer; uint32_t bytes; };       // a page of one layer in one of the cache's four parts

template <Moves WHAT>
__global__ void __launch_bounds__(256) copy_pages_kernel(PagesArgs p)
{
    const mt_kv_cache& c = p.c;
    const PageWork work = page_work(c);
    constexpr bool given = WHAT == Moves::kGiven || WHAT == Moves::kClaimed;
    const uint32_t n = given ? p.n : work.head->n;
    if constexpr (WHAT == Moves::kCompacted) follow(p, work, work.head->held);
    const uint32_t es = c.dtype == MT_F32 ? 4 : c.dtype == MT_BF16 ? 2 : 1;
    const uint32_t page = c.heads * c.page_tokens * c.head_dim * es, scales = c.dtype == MT_KV8 ? c.heads * c.page_tokens : 0;
    const uint32_t pieces = ceil_div(page, kPiece), scale_pieces = ceil_div(scales, kPiece), each = 2 * (pieces + scale_pieces);
    const uint64_t all = (uint64_t)n * c.layers * each;
    for (uint64_t i = blockIdx.x; i < all; i += gridDim.x) {
        const uint32_t pair = (uint32_t)(i / (c.layers * each)), rest = (uint32_t)(i % (c.layers * each)), layer = rest / each;
        uint32_t piece = rest % each;
        const uint32_t from = (uint32_t)(given ? p.first[pair] : work.moves[2 * pair]), to = (uint32_t)(given ? p.second[pair] : work.moves[2 * pair + 1]);
        if (from >= c.n_pages || to >= c.n_pages || from == to) continue;
        if constexpr (WHAT == Moves::kGiven) {
            bool again = false;
            for (uint32_t j = pair + 1 + threadIdx.x; j < n; j += 256) again |= (uint32_t)p.second[j] == to;
            if (__syncthreads_or(again)) continue;
        }
        if constexpr (WHAT == Moves::kClaimed)
            if ((uint32_t)work.map[to] != pair + 1) continue;
        const bool second = piece >= pieces + scale_pieces;
        if (second) piece -= pieces + scale_pieces;
        const bool of_scales = piece >= pieces;
        uint8_t* base = of_scales ? (second ? c.v_scales : c.k_scales) + layer * c.scales_layer_stride : (uint8_t*)(second ? c.v : c.k) + layer * c.layer_stride * es;
        const uint64_t stride = of_scales ? c.scales_page_stride : c.page_stride * es;
        const uint32_t begin = (of_scales ? piece - pieces : piece) * kPiece, bytes = min(kPiece, (of_scales ? scales : page) - begin);
        const uint8_t* src = base + from * stride + begin;
        uint8_t* dst = base + to * stride + begin;
        for (uint32_t at = threadIdx.x * 16; at < bytes; at += 256 * 16) *(u32x4*)(dst + at) = *(const u32x4*)(src + at);
    }
}

// work.map: for every page the last pair, counted from 1, that names it as its target; 0 for none.
__global__ void __launch_bounds__(256) unclaim_kernel(PagesArgs p)
{
    int32_t* map = page_work(p.c).map;
    for (uint64_t i = blockIdx.x * 256 + threadIdx.x; i < p.c.n_pages; i += gridDim.x * 256) map[i] = 0;
}
__global__ void __launch_bounds__(256) claim_kernel(PagesArgs p)
{
    uint32_t* map = (uint32_t*)page_work(p.c).map;
    for (uint64_t i = blockIdx.x * 256 + threadIdx.x; i < p.n; i += gridDim.x * 256) {
        const uint32_t to = (uint32_t)p.second[i];
        if (to < p.c.n_pages) atomicMax(&map[to], (uint32_t)i + 1);
    }
}

template <Moves WHAT> hipError_t copy_pages(const PagesArgs& p, uint64_t most, hipStream_t s)
{
    const uint64_t page = (uint64_t)p.c.heads * p.c.page_tokens * p.c.head_dim * value_bytes(p.c.dtype), work = most * p.c.layers * 2 * ((page + kPiece - 1) / kPiece + (p.c.dtype == MT_KV8));
    return launch(copy_pages_kernel<WHAT>, dim3((uint32_t)std::min<uint64_t>(std::max<uint64_t>(work, 1), 2048)), 256, 0, s, p);
}

uint32_t taking_bytes(const PagesArgs& p) { return sizeof(Taking) + 4 * p.c.seqs; }

}  // namespace

hipError_t prepare_pages()
{
    constexpr int most = sizeof(Taking) + 4 * MT_KV_MAX_SEQS;
    const hipError_t e = hipFuncSetAttribute((const void*)grow_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, most);
    return e != hipSuccess ? e : hipFuncSetAttribute((const void*)fork_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, most);
}

hipError_t launch_kv_grow(const PagesArgs& p, hipStream_t s) { return launch(grow_kernel, dim3(1), kThreads, taking_bytes(p), s, p); }
hipError_t launch_kv_fork(const PagesArgs& p, hipStream_t s)
{
    const hipError_t e = launch(fork_kernel, dim3(1), kThreads, taking_bytes(p), s, p);
    return e != hipSuccess ? e : copy_pages<Moves::kForked>(p, p.n, s);
}
hipError_t launch_kv_free(const PagesArgs& p, hipStream_t s) { return launch(free_kernel, dim3((p.n + 3) / 4), 256, 0, s, p); }
hipError_t launch_kv_compact(const PagesArgs& p, hipStream_t s)
{
    const hipError_t e = launch(compact_kernel, dim3(1), kThreads, 0, s, p);
    return e != hipSuccess ? e : copy_pages<Moves::kCompacted>(p, p.c.n_pages, s);
}
hipError_t launch_kv_copy(const PagesArgs& p, hipStream_t s)
{
    // Looking through the list is work that grows with its square (us looked through / looked up, pages of 4 KiB: 1 pair 5.7 / 13.9, 2048 8.9 / 13.2, 4096 18.5 / 16.6, 8192 42 / 24, 65536 1406 / 237; of 128 KiB:
    // 1024 115 / 117, 4096 464 / 440).
    if (p.n < 4096) return copy_pages<Moves::kGiven>(p, p.n, s);
    const auto blocks = [](uint64_t n) { return dim3((uint32_t)std::min<uint64_t>((n + 255) / 256, 2048)); };
    hipError_t e = launch(unclaim_kernel, blocks(p.c.n_pages), 256, 0, s, p);
    if (e == hipSuccess) e = launch(claim_kernel, blocks(p.n), 256, 0, s, p);
    return e != hipSuccess ? e : copy_pages<Moves::kClaimed>(p, p.n, s);
}

}  // namespace mt

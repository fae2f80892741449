// Who holds which page of a cache: sequences that share pages become
// continuations of others, get room for tokens, give pages back, and the pages
// in use move to the front.  Contract: include/dart_cache.h.
//
// Each call is one cluster of 8 CTAs (a small pool's one CTA): its work is a few scans over the pages and
// over the tables' entries, a chain of dependent loads, which the cluster's barriers
// join in one launch (a launch for each phase would add 2 us to each).  Pages are
// divided over the threads in runs, so that ranks of free pages and pages in use
// are sums of the runs before; tables over the warps in units of 128 entries, of
// which the ones that a call does not touch cost one comparison.
//
// All counts are integers: sums by atomics do not depend on their order.  What a
// phase decides by is never changed before the barrier behind it.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "../../include/dart.h"
#include "../../include/dart_cache.h"
#include "dart_cache.cuh"
#include "dart_device.cuh"
#include "dart_kernels.h"

namespace dart {
namespace {

constexpr int kCtas = 8, kThreads = 1024, kWarps = kThreads / 32;
constexpr int kUnit = 128;     // table entries of a unit: four a lane
// A pool of at most this size is one CTA's work, whose barriers cost less: one prompt continued in
// four ways 14.5 us instead of 16.5, a pool of 8 sequences compacted 18.6 instead of 20.7; 40
// sequences of 251 pages (80 units) 26.8 instead of 21.0.
constexpr int kOnePages = 4096, kOneUnits = 64;
constexpr int kDevNoRoom = 8;  // value in *status

// What reserve has found out about a sequence: places of its new pages' numbers and pair.
struct Grant {
    int count, pair;      // new pages; 1: one of them is a copy
    int old_end, need;    // entries [old_end, need) are all new, shared ones lie before
    int first, offset;    // first entry to look at; place of its pages in the list of free ones, -1: none
    int pair_at, old_new; // place of its pair; new pages before old_end
};

struct PoolArgs {
    int num_pages, page_log2, nseq, max_pages, chunks, run;  // chunks: units of a row; run: pages of a thread (a multiple of 4)
    int ctas;                                                // of the cluster; 1: no cluster
    int32_t *refs, *table, *held, *lens, *pairs, *count;
    const int32_t *parents, *n_rows;
    int32_t* granted;  // may be NULL
    // workspace
    int32_t* row;    // [nseq][max_pages]: select: new rows; reserve: which entries are new
    int32_t* list;   // [num_pages]: free pages, or holes, in ascending order
    int32_t* map;    // [num_pages]: where a page moves
    int32_t* seq;    // [nseq][2]: select: pages and length afterwards
    Grant* grant;    // [nseq]
    int32_t* sums;   // [2][kCtas]
    int* status;
};

__device__ __forceinline__ void bad_page(const PoolArgs& a) {
    if (a.status) atomicOr(a.status, kDevBounds);
}
__device__ __forceinline__ bool in_pool(const PoolArgs& a, int page) { return page >= 0 && page < a.num_pages; }
__device__ __forceinline__ int held_of(const PoolArgs& a, int s) { return min(max(__ldcg(a.held + s), 0), a.max_pages); }
__device__ __forceinline__ int len_of(const PoolArgs& a, int s) { return min(max(__ldcg(a.lens + s), 0), a.max_pages << a.page_log2); }
__device__ __forceinline__ int pages_of(const PoolArgs& a, int tokens) { return (tokens + (1 << a.page_log2) - 1) >> a.page_log2; }
// Pages that sequence s has with `rows` tokens more.
__device__ __forceinline__ long long need_of(const PoolArgs& a, int s, int rows) {
    return (static_cast<long long>(len_of(a, s)) + rows + (1 << a.page_log2) - 1) >> a.page_log2;
}

// body(s, i0): entries i0 .. of sequence s, for every unit of the tables, by a warp.
template <typename Body>
__device__ __forceinline__ void each_unit(const PoolArgs& a, Body&& body) {
    const int units = a.nseq * a.chunks;
    for (int u = blockIdx.x * kWarps + (threadIdx.x >> 5); u < units; u += a.ctas * kWarps) {
        const int s = a.chunks == 1 ? u : u / a.chunks;
        body(s, (u - s * a.chunks) * kUnit);
    }
}

// Between two phases: what the cluster wrote before is seen after it (by loads from L2).
__device__ __forceinline__ void next_phase(const PoolArgs& a) {
    if (a.ctas == 1) {
        __syncthreads();
    } else {
        __syncwarp();
        cluster_sync_all();
    }
}

// Exclusive sum over the block and its total; `part` is used by this call alone until
// the block's next barrier but one.
__device__ __forceinline__ int block_sum(int x, int* part, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int upto = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(kFull, upto, o);
        if (lane >= o) upto += y;
    }
    __syncthreads();
    if (lane == 31) part[warp] = upto;
    __syncthreads();
    const int mine = lane < kWarps ? part[lane] : 0;
    int before = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(kFull, before, o);
        if (lane >= o) before += y;
    }
    *total = __shfl_sync(kFull, before, 31);
    return __shfl_sync(kFull, before - mine, warp) + upto - x;
}

// refs of pages p .. p + 3 (past the pool: `none`).
__device__ __forceinline__ int4 refs4(const PoolArgs& a, int p, int none) {
    if (p + 4 <= a.num_pages) return __ldcg(reinterpret_cast<const int4*>(a.refs + p));
    int4 r = make_int4(none, none, none, none);
    if (p < a.num_pages) r.x = __ldcg(a.refs + p);
    if (p + 1 < a.num_pages) r.y = __ldcg(a.refs + p + 1);
    if (p + 2 < a.num_pages) r.z = __ldcg(a.refs + p + 2);
    return r;
}
// Pages in use among [p0, p1).
__device__ __forceinline__ int used_among(const PoolArgs& a, int p0, int p1) {
    int n = 0;
#pragma unroll 4
    for (int p = p0; p < p1; p += 4) {
        const int4 r = refs4(a, p, 0);
        n += (r.x > 0) + (r.y > 0) + (r.z > 0) + (r.w > 0);
    }
    return n;
}

// ------------------------------------------------------------ select

__global__ void __launch_bounds__(kThreads, 1) pool_select_kernel(const __grid_constant__ PoolArgs a) {
    const int lane = threadIdx.x & 31;
    pdl_trigger();
    pdl_wait();
    each_unit(a, [&](int s, int i0) {
        int p = ld_plain(a.parents + s);
        if (p < -1 || p >= a.nseq) {
            if (i0 == 0 && lane == 0) bad_page(a);
            p = s;
        }
        const bool change = p != s;
        const int have = change ? held_of(a, s) : 0;
        const int len = p >= 0 ? __ldcg(a.lens + p) : 0, keep = change && p >= 0 ? min(held_of(a, p), pages_of(a, len_of(a, p))) : 0;
        if (i0 == 0 && lane == 0) *reinterpret_cast<int2*>(a.seq + 2 * s) = make_int2(change ? keep : -1, len);
        if (i0 >= max(have, keep)) return;
#pragma unroll
        for (int e = 0; e < kUnit / 32; e++) {
            const int i = i0 + 32 * e + lane;
            if (i < have) {
                const int page = __ldcg(a.table + static_cast<long long>(s) * a.max_pages + i);
                if (in_pool(a, page))
                    atomicAdd(a.refs + page, -1);
                else
                    bad_page(a);
            }
            if (i < keep) {
                const int page = __ldcg(a.table + static_cast<long long>(p) * a.max_pages + i);
                if (in_pool(a, page))
                    atomicAdd(a.refs + page, 1);
                else
                    bad_page(a);
                __stcg(a.row + static_cast<long long>(s) * a.max_pages + i, page);
            }
        }
    });
    next_phase(a);
    each_unit(a, [&](int s, int i0) {
        const int2 now = __ldcg(reinterpret_cast<const int2*>(a.seq + 2 * s));
        if (now.x < 0) return;
        if (i0 == 0 && lane == 0) {
            a.held[s] = now.x;
            a.lens[s] = now.y;
        }
#pragma unroll
        for (int e = 0; e < kUnit / 32; e++) {
            const int i = i0 + 32 * e + lane;
            if (i < now.x) a.table[static_cast<long long>(s) * a.max_pages + i] = __ldcg(a.row + static_cast<long long>(s) * a.max_pages + i);
        }
    });
}

// ------------------------------------------------------------ reserve

__global__ void __launch_bounds__(kThreads, 1) pool_reserve_kernel(const __grid_constant__ PoolArgs a) {
    __shared__ int part[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = blockIdx.x;
    pdl_trigger();
    pdl_wait();
    // free pages of this thread's run, of the CTA
    const long long run0 = (static_cast<long long>(rank) * kThreads + tid) * a.run;
    const int p0 = static_cast<int>(min(run0, static_cast<long long>(a.num_pages))), p1 = min(p0 + a.run, a.num_pages);
    int cta_free;
    const int free_before = block_sum((p1 - p0) - used_among(a, p0, p1), part, &cta_free);
    if (tid == 0) __stcg(a.sums + rank, cta_free);
    // what each sequence needs: a warp each
    for (int s = rank * kWarps + warp; s < a.nseq; s += a.ctas * kWarps) {
        const int len = len_of(a, s), rows = ld_plain(a.n_rows + s), have = held_of(a, s), page = 1 << a.page_log2;
        const long long need64 = rows > 0 ? need_of(a, s, rows) : 0;
        Grant g{};
        const bool fits = need64 <= a.max_pages;
        if (!fits && lane == 0 && a.status) atomicOr(a.status, kDevNoRoom);
        g.need = fits ? static_cast<int>(need64) : 0;
        const int first = len >> a.page_log2;
        g.first = min(first, have);
        g.old_end = min(max(have, g.first), max(g.need, g.first));  // (shared ones are looked for up to here)
        for (int i0 = g.first; i0 < g.old_end; i0 += 32) {
            const int i = i0 + lane;
            bool fresh = false;
            if (i < g.old_end) {
                const int at = __ldcg(a.table + static_cast<long long>(s) * a.max_pages + i);
                if (in_pool(a, at))
                    fresh = __ldcg(a.refs + at) > 1;
                else
                    bad_page(a);
            }
            const unsigned all = __ballot_sync(kFull, fresh);
            if (i < g.old_end) __stcg(a.row + static_cast<long long>(s) * a.max_pages + i, fresh ? g.count + __popc(all & ((1u << lane) - 1u)) : -1);
            if (i0 == g.first && first < have && (len & (page - 1))) g.pair = all & 1u;  // (entry `first`: lane 0)
            g.count += __popc(all);
        }
        g.old_new = g.count;
        g.count += max(g.need - g.old_end, 0);
        if (lane == 0) {
            const int4* src = reinterpret_cast<const int4*>(&g);
            __stcg(reinterpret_cast<int4*>(a.grant + s), src[0]);
            __stcg(reinterpret_cast<int4*>(a.grant + s) + 1, src[1]);
        }
    }
    next_phase(a);
    // every CTA: places in the list of free pages, CTA by CTA
    int all_free = 0, cta_before = 0;
    for (int c = 0; c < a.ctas; c++) {
        const int n = __ldcg(a.sums + c);
        if (c < rank) cta_before += n;
        all_free += n;
    }
    int places = 0, copies = 0;  // granted so far
    long long asked = 0;         // (of all sequences, granted or not)
    for (int s0 = 0; s0 < a.nseq; s0 += kThreads) {
        const int s = s0 + tid;
        int2 want = make_int2(0, 0);
        int rows = 0;
        if (s < a.nseq) {
            want = __ldcg(reinterpret_cast<const int2*>(a.grant + s));
            rows = ld_plain(a.n_rows + s);
        }
        const bool fits = rows > 0 && need_of(a, min(s, a.nseq - 1), rows) <= a.max_pages;
        int tile;  // (at most nseq * max_pages, 2^30)
        const int before = block_sum(want.x, part, &tile);
        const bool granted = asked + before + want.x <= all_free;
        int ok, pairs;
        block_sum(granted ? want.x : 0, part, &ok);
        const int pair_at = copies + block_sum(granted ? want.y : 0, part, &pairs);
        if (s < a.nseq && (s0 / kThreads) % a.ctas == rank) {
            if (!granted && want.x > 0 && a.status) atomicOr(a.status, kDevNoRoom);
            __stcg(&a.grant[s].offset, granted && want.x > 0 ? static_cast<int>(asked) + before : -1);
            __stcg(&a.grant[s].pair_at, pair_at);
            if (a.granted) a.granted[s] = fits && (granted || want.x == 0) ? rows : 0;
        }
        places += ok;
        copies += pairs;
        asked += tile;
    }
    if (rank == 0 && tid == 0) *a.count = copies;
    {
        int at = cta_before + free_before;
        if (at < places)
            for (int p = p0; p < p1; p += 4) {
                const int4 r = refs4(a, p, 1);
                const int v[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (v[e] <= 0) {
                        if (at < places) __stcg(a.list + at, p + e);
                        at++;
                    }
            }
    }
    next_phase(a);
    // the shared pages' replacements: a warp a sequence
    for (int s = rank * kWarps + warp; s < a.nseq; s += a.ctas * kWarps) {
        Grant g;
        int4* dst = reinterpret_cast<int4*>(&g);
        dst[0] = __ldcg(reinterpret_cast<const int4*>(a.grant + s));
        dst[1] = __ldcg(reinterpret_cast<const int4*>(a.grant + s) + 1);
        if (g.offset < 0) continue;
        for (int i = g.first + lane; i < g.old_end; i += 32) {
            const int n = __ldcg(a.row + static_cast<long long>(s) * a.max_pages + i);
            if (n < 0) continue;
            const int page = __ldcg(a.list + g.offset + n);
            int32_t* at = a.table + static_cast<long long>(s) * a.max_pages + i;
            const int old = __ldcg(at);
            atomicAdd(a.refs + old, -1);
            a.refs[page] = 1;
            *at = page;
            if (g.pair && i == g.first) *reinterpret_cast<int2*>(a.pairs + 2 * g.pair_at) = make_int2(old, page);
        }
        if (lane == 0 && g.need > g.old_end) a.held[s] = g.need;
    }
    // the others
    each_unit(a, [&](int s, int i0) {
        const int4 g = __ldcg(reinterpret_cast<const int4*>(a.grant + s)), h = __ldcg(reinterpret_cast<const int4*>(a.grant + s) + 1);
        const int from = g.z, to = g.w, offset = h.y + h.w;
        if (h.y < 0 || i0 >= to) return;
#pragma unroll
        for (int e = 0; e < kUnit / 32; e++) {
            const int i = i0 + 32 * e + lane;
            if (i < from || i >= to) continue;
            const int page = __ldcg(a.list + offset + i - from);
            a.refs[page] = 1;
            a.table[static_cast<long long>(s) * a.max_pages + i] = page;
        }
    });
}

// ------------------------------------------------------------ trim

__global__ void __launch_bounds__(kThreads, 1) pool_trim_kernel(const __grid_constant__ PoolArgs a) {
    const int lane = threadIdx.x & 31;
    pdl_trigger();
    pdl_wait();
    each_unit(a, [&](int s, int i0) {
        const int have = held_of(a, s), need = pages_of(a, len_of(a, s));
        if (i0 >= have || i0 + kUnit <= need) return;
#pragma unroll
        for (int e = 0; e < kUnit / 32; e++) {
            const int i = i0 + 32 * e + lane;
            if (i < need || i >= have) continue;
            const int page = __ldcg(a.table + static_cast<long long>(s) * a.max_pages + i);
            if (in_pool(a, page))
                atomicAdd(a.refs + page, -1);
            else
                bad_page(a);
        }
    });
    next_phase(a);  // (every unit has seen the counts that change now)
    for (int s = blockIdx.x * kThreads + threadIdx.x; s < a.nseq; s += a.ctas * kThreads) a.held[s] = min(held_of(a, s), pages_of(a, len_of(a, s)));
}

// ------------------------------------------------------------ compact

__global__ void __launch_bounds__(kThreads, 1) pool_compact_kernel(const __grid_constant__ PoolArgs a) {
    __shared__ int part[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, rank = blockIdx.x;
    pdl_trigger();
    pdl_wait();
    const long long run0 = (static_cast<long long>(rank) * kThreads + tid) * a.run;
    const int p0 = static_cast<int>(min(run0, static_cast<long long>(a.num_pages))), p1 = min(p0 + a.run, a.num_pages);
    int cta_used;
    int before = block_sum(used_among(a, p0, p1), part, &cta_used);  // pages in use before this run
    if (tid == 0) __stcg(a.sums + rank, cta_used);
    next_phase(a);
    int n = 0;
    for (int c = 0; c < a.ctas; c++) {
        const int x = __ldcg(a.sums + c);
        if (c < rank) before += x;
        n += x;
    }
    // free pages below n in order: page p is the (p - pages in use before it)-th
    int at = before, holes = 0;
    const int low_end = min(p1, max(n, p0));
    for (int p = p0; p < low_end; p += 4) {
        const int4 r = refs4(a, p, 1);
        const int v[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int e = 0; e < 4; e++) {
            if (p + e >= low_end) break;
            if (v[e] > 0) {
                at++;
            } else {
                __stcg(a.list + (p + e - at), p + e);
                holes++;
            }
        }
    }
    int cta_holes;
    block_sum(holes, part, &cta_holes);
    if (tid == 0) __stcg(a.sums + kCtas + rank, cta_holes);
    next_phase(a);
    int moves = 0;
    for (int c = 0; c < a.ctas; c++) moves += __ldcg(a.sums + kCtas + c);
    // pages in use from n on (the counts below n change meanwhile, these are this thread's alone)
    int k = at - (n - moves);
    for (int p = low_end; p < p1; p++) {
        const int users = __ldcg(a.refs + p);
        int to = p;
        if (users > 0) {
            to = __ldcg(a.list + k);
            *reinterpret_cast<int2*>(a.pairs + 2 * k) = make_int2(p, to);
            a.refs[to] = users;
            a.refs[p] = 0;
            k++;
        }
        __stcg(a.map + p, to);
    }
    if (rank == 0 && tid == 0) *a.count = moves;
    next_phase(a);
    each_unit(a, [&](int s, int i0) {
        const int have = held_of(a, s);
        if (i0 >= have) return;
#pragma unroll
        for (int e = 0; e < kUnit / 32; e++) {
            const int i = i0 + 32 * e + lane;
            if (i >= have) continue;
            int32_t* x = a.table + static_cast<long long>(s) * a.max_pages + i;
            const int page = __ldcg(x);
            if (!in_pool(a, page))
                bad_page(a);
            else if (page >= n)
                *x = __ldcg(a.map + page);
        }
    });
}

// ------------------------------------------------------------ host

bool valid_pool(const dart_page_pool* p) {
    if (!p || p->num_pages < 1 || p->nseq < 1 || p->max_pages < 1) return false;
    if (p->page_size != 16 && p->page_size != 32 && p->page_size != 64 && p->page_size != 128) return false;
    if (p->num_pages > (1 << 30)) return false;
    return static_cast<long long>(p->nseq) * p->max_pages <= (1ll << 30) && static_cast<long long>(p->max_pages) * p->page_size <= (1ll << 30);
}
bool aligned(const void* p, uintptr_t n) { return p && (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

struct PoolWs {
    size_t row, list, map, seq, grant, sums, total;
};
PoolWs pool_ws(const dart_page_pool& p) {
    auto up = [](size_t n) { return (n + 255) & ~static_cast<size_t>(255); };
    PoolWs w{};
    w.list = up(static_cast<size_t>(p.nseq) * p.max_pages * 4);
    w.map = w.list + up(static_cast<size_t>(p.num_pages) * 4);
    w.seq = w.map + up(static_cast<size_t>(p.num_pages) * 4);
    w.grant = w.seq + up(static_cast<size_t>(p.nseq) * 8);
    w.sums = w.grant + up(static_cast<size_t>(p.nseq) * sizeof(Grant));
    w.total = w.sums + up(2 * kCtas * 4);
    return w;
}

// What all calls check, and the arguments they share; DART_OK or an error.
int pool_args(const dart_page_pool* pool, const void* lens, bool needs_lens, const void* workspace, size_t bytes, bool needs_ws, int* status,
              PoolArgs* a) {
    if (!valid_pool(pool) || !aligned(pool->refs, 16) || !aligned(pool->table, 4) || !aligned(pool->held, 4)) return DART_ERR_INVALID;
    if ((needs_lens && !aligned(lens, 4)) || (status && !aligned(status, 4))) return DART_ERR_INVALID;
    const PoolWs w = pool_ws(*pool);
    if (needs_ws && (!aligned(workspace, 256) || bytes < w.total)) return DART_ERR_INVALID;
    if (const int rc = check_device()) return rc;
    *a = PoolArgs{};
    a->num_pages = pool->num_pages;
    while ((1 << a->page_log2) < pool->page_size) a->page_log2++;
    a->nseq = pool->nseq;
    a->max_pages = pool->max_pages;
    a->chunks = (pool->max_pages + kUnit - 1) / kUnit;
    a->ctas = pool->num_pages <= kOnePages && static_cast<long long>(a->nseq) * a->chunks <= kOneUnits ? 1 : kCtas;
    a->run = ((pool->num_pages + a->ctas * kThreads - 1) / (a->ctas * kThreads) + 3) / 4 * 4;
    a->refs = pool->refs;
    a->table = pool->table;
    a->held = pool->held;
    a->lens = const_cast<int32_t*>(static_cast<const int32_t*>(lens));
    a->status = status;
    if (needs_ws) {
        uint8_t* ws = static_cast<uint8_t*>(const_cast<void*>(workspace));
        a->row = reinterpret_cast<int32_t*>(ws);
        a->list = reinterpret_cast<int32_t*>(ws + w.list);
        a->map = reinterpret_cast<int32_t*>(ws + w.map);
        a->seq = reinterpret_cast<int32_t*>(ws + w.seq);
        a->grant = reinterpret_cast<Grant*>(ws + w.grant);
        a->sums = reinterpret_cast<int32_t*>(ws + w.sums);
    }
    return DART_OK;
}

int launch_pool(void (*kernel)(PoolArgs), const PoolArgs& a, void* stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = a.ctas == 1 ? launch_pdl(kernel, dim3(1), dim3(kThreads), 0, st, a) : launch_pdl_cluster(kernel, dim3(kCtas), dim3(kThreads), 0, st, kCtas, a);
    return e == cudaSuccess ? DART_OK : DART_ERR_CUDA;
}

int reserve(const dart_page_pool* pool, const int32_t* lens, const int32_t* n_rows, int32_t* granted, int32_t* pairs, int max_pairs, int32_t* count,
            void* workspace, size_t workspace_bytes, int* status, void* stream) {
    PoolArgs a;
    if (!aligned(n_rows, 4) || !aligned(pairs, 8) || !aligned(count, 4) || !pool || max_pairs < pool->nseq) return DART_ERR_INVALID;
    if (const int rc = pool_args(pool, lens, true, workspace, workspace_bytes, true, status, &a)) return rc;
    a.n_rows = n_rows;
    a.granted = granted;
    a.pairs = pairs;
    a.count = count;
    return launch_pool(pool_reserve_kernel, a, stream);
}

}  // namespace
}  // namespace dart

using namespace dart;

extern "C" {

size_t dart_page_pool_workspace(const dart_page_pool* pool) { return valid_pool(pool) ? pool_ws(*pool).total : 0; }

int dart_page_pool_select(const dart_page_pool* pool, const int32_t* parents, int32_t* lens, void* workspace, size_t workspace_bytes,
                          int* status, void* stream) {
    PoolArgs a;
    if (!aligned(parents, 4)) return DART_ERR_INVALID;
    if (const int rc = pool_args(pool, lens, true, workspace, workspace_bytes, true, status, &a)) return rc;
    a.parents = parents;
    return launch_pool(pool_select_kernel, a, stream);
}

int dart_page_pool_reserve(const dart_page_pool* pool, const int32_t* lens, const int32_t* n_rows, int32_t* pairs, int max_pairs,
                           int32_t* count, void* workspace, size_t workspace_bytes, int* status, void* stream) {
    return reserve(pool, lens, n_rows, nullptr, pairs, max_pairs, count, workspace, workspace_bytes, status, stream);
}

int dart_page_pool_reserve_rows(const dart_page_pool* pool, const int32_t* lens, const int32_t* n_rows, int32_t* granted, int32_t* pairs,
                                int max_pairs, int32_t* count, void* workspace, size_t workspace_bytes, int* status, void* stream) {
    if (!aligned(granted, 4)) return DART_ERR_INVALID;
    return reserve(pool, lens, n_rows, granted, pairs, max_pairs, count, workspace, workspace_bytes, status, stream);
}

int dart_page_pool_trim(const dart_page_pool* pool, const int32_t* lens, int* status, void* stream) {
    PoolArgs a;
    if (const int rc = pool_args(pool, lens, true, nullptr, 0, false, status, &a)) return rc;
    return launch_pool(pool_trim_kernel, a, stream);
}

int dart_page_pool_compact(const dart_page_pool* pool, int32_t* pairs, int max_pairs, int32_t* count, void* workspace,
                           size_t workspace_bytes, int* status, void* stream) {
    PoolArgs a;
    if (!aligned(pairs, 8) || !aligned(count, 4) || !pool || max_pairs < pool->num_pages / 2) return DART_ERR_INVALID;
    if (const int rc = pool_args(pool, nullptr, false, workspace, workspace_bytes, true, status, &a)) return rc;
    a.pairs = pairs;
    a.count = count;
    return launch_pool(pool_compact_kernel, a, stream);
}

}  // extern "C"

// Tree attention over the paged cache.  Contract: include/dart_cache.h.
//
// A unit of work is 16 query rows of one kv head of one sequence (a row = a
// tree row and one of the G query heads that share the kv head) against all
// keys that the rows may see: the sequence's cache, then its tree rows, both
// in chunks of 16 keys.  The chunks of all units form one list, which the
// CTAs (one per SM) share evenly, so that ragged lengths and a single long
// sequence load every SM alike; lengths are read on the device, so the split
// is made there.  A CTA's eight warps take its chunks in turn, each with its
// own ring of TMA stages and its own running maximum, sum and accumulators:
// nothing is exchanged before the unit's end, where the warps' results are
// merged through shared memory.  A unit that several CTAs share is left as
// partial results in the workspace, which a second kernel joins in order.
//
// The products are warp-wide 16 x 8 x 16 matrix instructions: with at most 16
// rows a chunk of bf16 keys takes 8 KB from HBM for 32 of them, far below any
// tensor rate, and keys and probabilities stay in registers (a 128-row tile
// of the tensor-memory path would be 7/8 empty).  HBM bounds it.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "../../include/dart.h"
#include "../../include/dart_cache.h"
#include "dart_cache.cuh"
#include "dart_kernels.h"

namespace dart {

bool valid_cache(const dart_kv_cache* c);
bool valid_cache_pointers(const dart_kv_cache* c);

namespace {

constexpr int kUnitRows = 16;
constexpr int kChunk = 16;                 // keys
constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kMaxCtas = 256;              // workspace slots: 2 per CTA
constexpr int kMergeBytes = 4 * 64 * 32 * 4;  // accumulators of four warps
constexpr float kSlack = 8.0f;             // log2 units a score may exceed the row's reference by

struct Part {  // a unit's partial result
    float o[kUnitRows][kHeadDim];
    float2 ml[kUnitRows];  // reference (log2 units), sum
};

struct PagedArgs {
    int nseq, B, Hq, Hkv, G, nrg, max_pages, page_log2, num_pages, mw;
    long long pool_rows;
    const int32_t *table, *lens, *depths, *n_nodes;
    const uint64_t* mask;
    const __nv_bfloat16 *q, *k, *v;
    long long q_stride, k_stride, v_stride;
    const float *ks, *vs;
    __nv_bfloat16* out;
    Part* parts;  // [CTAs][2]: of the unit begun before the CTA's range, of the unit that goes on after it
    int* status;
    float sl2;  // scale * log2(e)
    RopeTurns turns;
};

// ------------------------------------------------------------ the schedule

__device__ __forceinline__ int seq_len(const PagedArgs& a, int s) {
    const long long most = static_cast<long long>(a.max_pages) << a.page_log2;
    return static_cast<int>(min(max(static_cast<long long>(__ldg(a.lens + s)), 0ll), most));
}
__device__ __forceinline__ int seq_nodes(const PagedArgs& a, int s) {
    return a.B > 0 ? min(max(__ldg(a.n_nodes + s), 0), a.B) : 0;
}

// A place in the list of chunks: sequence, unit of the sequence (row group
// fastest, then kv head), chunk of the unit.
struct Place {
    int s, unit, chunk;
    int len, nodes, ctx_chunks, chunks, units;  // of the sequence
    __device__ __forceinline__ void load(const PagedArgs& a) {
        len = seq_len(a, s);
        nodes = seq_nodes(a, s);
        ctx_chunks = (len + kChunk - 1) / kChunk;
        chunks = ctx_chunks + (nodes + 1 + kChunk - 1) / kChunk;
        units = a.Hkv * (((nodes + 1) * a.G + kUnitRows - 1) / kUnitRows);
    }
    __device__ __forceinline__ int groups(const PagedArgs& a) const { return units / a.Hkv; }
    __device__ __forceinline__ void advance(const PagedArgs& a, int by) {
        chunk += by;
        while (chunk >= chunks) {
            chunk -= chunks;
            if (++unit == units) {
                unit = 0;
                if (++s >= a.nseq) {
                    chunk = 0;
                    return;
                }
                load(a);
            }
        }
    }
};

// Chunks of all sequences before sequence `upto`, by one warp.
__device__ __forceinline__ long long chunks_before(const PagedArgs& a, int upto, int lane) {
    long long n = 0;
    for (int s = lane; s < upto; s += 32) {
        Place p{};
        p.s = s;
        p.load(a);
        n += static_cast<long long>(p.units) * p.chunks;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(kFull, n, o);
    return n;
}

// The place of chunk x of the list (0 <= x < all), by one warp.
__device__ __forceinline__ Place find_place(const PagedArgs& a, long long x, int lane) {
    long long done = 0;
    for (int s0 = 0; s0 < a.nseq; s0 += 32) {
        Place p{};
        p.s = s0 + lane;
        long long n = 0;
        if (p.s < a.nseq) {
            p.load(a);
            n = static_cast<long long>(p.units) * p.chunks;
        }
        long long upto = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(kFull, upto, o);
            if (lane >= o) upto += y;
        }
        const unsigned hit = __ballot_sync(kFull, p.s < a.nseq && x < done + upto);
        if (hit) {
            const int l = __ffs(hit) - 1;
            const long long rest = x - done - __shfl_sync(kFull, upto - n, l);
            Place r{};
            r.s = s0 + l;
            r.load(a);
            r.unit = static_cast<int>(rest / r.chunks);
            r.chunk = static_cast<int>(rest % r.chunks);
            return r;
        }
        done += __shfl_sync(kFull, upto, 31);
    }
    Place r{};
    r.s = a.nseq;
    return r;
}

// CTAs that get work (at least one chunk per warp each), and where CTA c's
// share begins.
__device__ __forceinline__ int active_ctas(long long all, int ctas) {
    return static_cast<int>(min(static_cast<long long>(ctas), (all + kWarps - 1) / kWarps));
}
__device__ __forceinline__ long long share_begin(long long all, int ctas, int c) { return all * c / ctas; }
__device__ __forceinline__ int share_of_chunk(long long all, int ctas, long long x) {
    return static_cast<int>(((x + 1) * ctas - 1) / all);
}

// ------------------------------------------------------------ fragments

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two e4m3 codes (low, high byte) as an f16 pair: exact.
__device__ __forceinline__ uint32_t e4m3_to_f16(uint32_t two) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(static_cast<uint16_t>(two)));
    return r;
}
// Two e4m3 codes in bytes 1 and 3 of x (bytes 0 and 2: anything) as a bf16
// pair: sign, then exponent and mantissa four bits down, and a product with
// 2^120 for the difference of the exponents' biases (exact, subnormals too).
__device__ __forceinline__ uint32_t e4m3_to_bf16(uint32_t x) {
    const uint32_t y = ((x >> 4) & 0x07F007F0u) | (x & 0x80008000u);
    const __nv_bfloat162 by = __halves2bfloat162(__ushort_as_bfloat16(0x7B80), __ushort_as_bfloat16(0x7B80));  // 2^120
    const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&y), by);
    return *reinterpret_cast<const uint32_t*>(&r);
}

// Row of a 16-key chunk behind key slot (n-tile q, column n) of the products:
// chosen so that both the reads of K (lanes g, t: row slot_row(q, g), 16-byte
// pieces t, t + 4, ...) and of V (rows slot_row(q, 2t + e), piece g) touch
// every bank once under the 128-byte swizzle.
__device__ __forceinline__ int slot_row(int q, int n) {
    return q * 8 + ((((n >> 2) ^ n) & 1) << 2) + (n & 2) + (n & 1);
}

__device__ __forceinline__ uint32_t swz(int row, int piece) {  // byte offset in a tile of 128-byte rows
    return static_cast<uint32_t>(row * 128 + ((piece ^ (row & 7)) << 4));
}

template <bool kFp8>
struct Geo {
    static constexpr int kKeyBytes = kFp8 ? kHeadDim : 2 * kHeadDim;
    static constexpr int kTile = kChunk * kKeyBytes;             // K or V of a chunk
    static constexpr int kStage = 2 * kTile + (kFp8 ? 128 : 0);  // K, V, scales of both
    static constexpr int kStages = kFp8 ? 5 : 3;
    static constexpr int kRing = kWarps * kStages * 2 * kTile;
    static constexpr int kScales = kFp8 ? kWarps * kStages * 128 : 0;
    // ring, merge buffer (the query rows before it), scales, statistics, barriers
    static constexpr int kSmem = kRing + kMergeBytes + kScales + kWarps * kUnitRows * 8 + kUnitRows * 4 + kWarps * kStages * 8 + 64;
};

// Element of the head behind column n of n-tile j of the output products.
template <bool kFp8>
__device__ __forceinline__ int out_dim(int n, int j) {
    return kFp8 ? 16 * n + j : (j < 8 ? 8 * n + j : 64 + 8 * n + j - 8);
}
// 16-byte piece (8 bf16) of a row of the head that step pair i of thread t
// covers; i and i + 2 are 64 elements apart, as RoPE's pairs are.
template <bool kFp8>
__device__ __forceinline__ int k_piece(int i, int t) {
    return kFp8 ? 8 * (i >> 1) + 2 * t + (i & 1) : 8 * (i >> 1) + t + 4 * (i & 1);
}

struct Frags {
    uint32_t q[8][4];   // queries, hi (bf16) or scaled f16 (e4m3 cache): steps of 16 elements
    uint32_t lo[8][4];  // what the hi part leaves (bf16 cache)
    float acc[16][4];
    float m[2], l[2];   // rows g and g + 8
};

template <bool kFp8>
__global__ void __launch_bounds__(kThreads, 1)
    paged_rows_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                      const __grid_constant__ PagedArgs a) {
    using G_ = Geo<kFp8>;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* merge = smem + G_::kRing;
    uint8_t* scales = merge + kMergeBytes;
    float2* stat = reinterpret_cast<float2*>(scales + G_::kScales);       // [warps][16 rows]
    float* row_scale = reinterpret_cast<float*>(stat + kWarps * kUnitRows);
    uint64_t* bars = reinterpret_cast<uint64_t*>(row_scale + kUnitRows);  // [warps][stages]
    int* flags = reinterpret_cast<int*>(bars + kWarps * G_::kStages);
    volatile int* abort = flags;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    pdl_trigger();
    uint8_t* ring = smem + warp * G_::kStages * 2 * G_::kTile;
    uint8_t* my_scales = scales + warp * G_::kStages * 128;
    uint64_t* bar = bars + warp * G_::kStages;
    if (lane == 0)
        for (int i = 0; i < G_::kStages; i++) mbar_init(bar + i, 1);
    if (tid == 0) *abort = 0;
    fence_mbar_init();
    __syncthreads();
    pdl_wait();

    // rows of no node: zeros
    for (long long i = blockIdx.x; i < static_cast<long long>(a.nseq) * (a.B + 1); i += gridDim.x) {
        const int s = static_cast<int>(i / (a.B + 1)), r = static_cast<int>(i % (a.B + 1));
        if (r <= seq_nodes(a, s)) continue;
        uint4* o = reinterpret_cast<uint4*>(a.out + i * a.Hq * kHeadDim);
        for (int j = tid; j < a.Hq * kHeadDim / 8; j += kThreads) o[j] = make_uint4(0, 0, 0, 0);
    }

    const long long all = chunks_before(a, a.nseq, lane);
    const int ctas = active_ctas(all, gridDim.x);
    if (static_cast<int>(blockIdx.x) >= ctas) return;
    const long long begin = share_begin(all, ctas, blockIdx.x), end = share_begin(all, ctas, blockIdx.x + 1);
    Place unit = find_place(a, begin, lane);  // of the unit at hand; its chunk: where the CTA's part begins
    Place load = unit, use = unit;            // of this warp's next chunk to load, to work on
    load.advance(a, warp);
    use = load;
    long long load_at = begin + warp, use_at = begin + warp;
    int n_load = 0, n_use = 0;
    bool ok = true;
    const uint64_t policy = a.nrg == 1 ? l2_policy_evict_first() : l2_policy_evict_last();

    // The page of a chunk, one chunk ahead of its load.
    auto page_of = [&](const Place& p) -> int {
        if (p.s >= a.nseq || p.chunk >= p.ctx_chunks) return 0;
        return __ldg(a.table + static_cast<long long>(p.s) * a.max_pages + ((p.chunk * kChunk) >> a.page_log2));
    };
    int page = load_at < end ? page_of(load) : 0;
    auto issue = [&]() {  // loads the chunk at `load` (tree chunks are read when they are worked on)
        if (load.chunk < load.ctx_chunks) {
            if (lane == 0) {
                const int st = n_load % G_::kStages;
                const int head = load.unit / load.groups(a);
                long long row = a.pool_rows;  // past the pool: zeros
                if (page >= 0 && page < a.num_pages)
                    row = ((static_cast<long long>(page) * a.Hkv + head) << a.page_log2) +
                          ((load.chunk * kChunk) & ((1 << a.page_log2) - 1));
                else if (a.status)
                    atomicOr(a.status, kDevBounds);
                uint8_t* k = ring + st * 2 * G_::kTile;
                uint8_t* v = k + G_::kTile;
                mbar_arrive_expect_tx(bar + st, G_::kStage);
                tma_load_2d(k, &tmK, bar + st, 0, static_cast<int>(row), policy);
                if (!kFp8) tma_load_2d(k + G_::kTile / 2, &tmK, bar + st, 64, static_cast<int>(row), policy);
                tma_load_2d(v, &tmV, bar + st, 0, static_cast<int>(row), policy);
                if (!kFp8) tma_load_2d(v + G_::kTile / 2, &tmV, bar + st, 64, static_cast<int>(row), policy);
                if (kFp8) {
                    const long long sr = row < a.pool_rows ? row : 0;
                    bulk_load(my_scales + st * 128, a.ks + sr, 64, bar + st);
                    bulk_load(my_scales + st * 128 + 64, a.vs + sr, 64, bar + st);
                }
            }
            n_load++;
        }
        load_at += kWarps;
        if (load_at < end) {
            load.advance(a, kWarps);
            page = page_of(load);
        }
    };
    while (load_at < end && n_load < G_::kStages) issue();

    Frags f;
    for (long long at = begin; at < end;) {
        // ---- this CTA's part of a unit: chunks [at, at + part) of the list
        const int part = static_cast<int>(min(static_cast<long long>(unit.chunks - unit.chunk), end - at));
        const int groups = unit.groups(a), head = unit.unit / groups, row0 = (unit.unit % groups) * kUnitRows;
        const int s = unit.s, len = unit.len, nodes = unit.nodes;
        const long long seq_row = static_cast<long long>(s) * (a.B + 1);
        __syncthreads();  // the merge buffer is free
        {
            // the unit's queries, rotated: 16 threads a row, 4 pairs each
            const int r = tid >> 4, p0 = (tid & 15) * 4, b = (row0 + r) / a.G;
            float lo[4] = {0.0f, 0.0f, 0.0f, 0.0f}, hi[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (b <= nodes) {
                const int pos = len + (b > 0 ? __ldg(a.depths + static_cast<long long>(s) * a.B + b - 1) : 0);
                const __nv_bfloat16* q = a.q + (seq_row + b) * a.q_stride + (head * a.G + (row0 + r) % a.G) * kHeadDim + p0;
                const uint2 x = *reinterpret_cast<const uint2*>(q), y = *reinterpret_cast<const uint2*>(q + 64);
                const float xl[4] = {bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y)};
                const float xh[4] = {bf16_lo(y.x), bf16_hi(y.x), bf16_lo(y.y), bf16_hi(y.y)};
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    float sn, cs;
                    rope_sincos(a.turns.f[p0 + e], pos, &sn, &cs);
                    lo[e] = xl[e] * cs - xh[e] * sn;
                    hi[e] = xh[e] * cs + xl[e] * sn;
                }
            }
            uint8_t* d = merge + r * 256 + p0 * 2;
            if (kFp8) {
                // scaled by a power of two to a largest element in [1, 2): f16 then
                // rounds it to 2^-11 whatever the queries' magnitude
                float mx = 0.0f;
#pragma unroll
                for (int e = 0; e < 4; e++) mx = fmaxf(mx, fmaxf(fabsf(lo[e]), fabsf(hi[e])));
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, o));
                const int ex = min(max(static_cast<int>(__float_as_uint(mx) >> 23) - 127, -100), 120);
                const float down = __uint_as_float(static_cast<uint32_t>(127 - ex) << 23);
                if ((tid & 15) == 0) row_scale[r] = a.sl2 * __uint_as_float(static_cast<uint32_t>(127 + ex) << 23);
                __half2 w[4] = {__floats2half2_rn(lo[0] * down, lo[1] * down), __floats2half2_rn(lo[2] * down, lo[3] * down),
                                __floats2half2_rn(hi[0] * down, hi[1] * down), __floats2half2_rn(hi[2] * down, hi[3] * down)};
                *reinterpret_cast<uint2*>(d) = *reinterpret_cast<uint2*>(w);
                *reinterpret_cast<uint2*>(d + 128) = *reinterpret_cast<uint2*>(w + 2);
            } else {
                // bf16 and what it leaves: with one bf16 term the queries' rounding
                // alone would move the output as much as its own rounding does
                const uint32_t h[4] = {pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3]), pack_bf16x2(hi[0], hi[1]),
                                       pack_bf16x2(hi[2], hi[3])};
                *reinterpret_cast<uint2*>(d) = make_uint2(h[0], h[1]);
                *reinterpret_cast<uint2*>(d + 128) = make_uint2(h[2], h[3]);
                d += kUnitRows * 256;
                *reinterpret_cast<uint2*>(d) = make_uint2(pack_bf16x2(lo[0] - bf16_lo(h[0]), lo[1] - bf16_hi(h[0])),
                                                          pack_bf16x2(lo[2] - bf16_lo(h[1]), lo[3] - bf16_hi(h[1])));
                *reinterpret_cast<uint2*>(d + 128) = make_uint2(pack_bf16x2(hi[0] - bf16_lo(h[2]), hi[1] - bf16_hi(h[2])),
                                                                pack_bf16x2(hi[2] - bf16_lo(h[3]), hi[3] - bf16_hi(h[3])));
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int off = k_piece<kFp8>(i, t) * 16;
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const uint4 x = *reinterpret_cast<const uint4*>(merge + (g + 8 * h) * 256 + off);
                f.q[2 * i][h] = x.x;
                f.q[2 * i][2 + h] = x.y;
                f.q[2 * i + 1][h] = x.z;
                f.q[2 * i + 1][2 + h] = x.w;
                if (!kFp8) {
                    const uint4 y = *reinterpret_cast<const uint4*>(merge + (kUnitRows + g + 8 * h) * 256 + off);
                    f.lo[2 * i][h] = y.x;
                    f.lo[2 * i][2 + h] = y.y;
                    f.lo[2 * i + 1][h] = y.z;
                    f.lo[2 * i + 1][2 + h] = y.w;
                }
            }
        }
        const float rs[2] = {kFp8 ? row_scale[g] : a.sl2, kFp8 ? row_scale[g + 8] : a.sl2};
#pragma unroll
        for (int j = 0; j < 16; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) f.acc[j][e] = 0.0f;
        f.m[0] = f.m[1] = -INFINITY;
        f.l[0] = f.l[1] = 0.0f;

        // ---- this warp's chunks of the part
        while (use_at < at + part) {
            const bool ctx = use.chunk < use.ctx_chunks;
            const int st = n_use % G_::kStages;
            const uint8_t* kt = ring + st * 2 * G_::kTile;
            const uint8_t* vt = kt + G_::kTile;
            const float* sck = reinterpret_cast<const float*>(my_scales + st * 128);
            const int key0 = ctx ? use.chunk * kChunk : (use.chunk - use.ctx_chunks) * kChunk;
            const int live = ctx ? len : nodes + 1;  // keys below it exist
            if (ctx && ok) {
                const bool got = mbar_wait_inline(bar + st, static_cast<uint32_t>(n_use / G_::kStages) & 1u, abort);
                if (!__all_sync(kFull, got)) {
                    ok = false;
                    *abort = 1;
                    if (a.status && lane == 0) atomicOr(a.status, kDevTimeout);
                }
            }
            if (ok) {
                float sc[2][4];  // [key half][row g: keys 2t, 2t + 1; row g + 8: the same]
#pragma unroll
                for (int q = 0; q < 2; q++)
#pragma unroll
                    for (int e = 0; e < 4; e++) sc[q][e] = 0.0f;
                if (ctx) {
#pragma unroll
                    for (int q = 0; q < 2; q++) {
                        const int row = slot_row(q, g);
                        if (kFp8) {
#pragma unroll
                            for (int c = 0; c < 2; c++) {
                                const uint4 x = *reinterpret_cast<const uint4*>(kt + swz(row, t + 4 * c));
                                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                                for (int e = 0; e < 4; e++)
                                    mma_f16(sc[q], f.q[4 * c + e], e4m3_to_f16(w[e]), e4m3_to_f16(w[e] >> 16));
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; i++) {
                                const uint4 x = *reinterpret_cast<const uint4*>(kt + (i >> 1) * (G_::kTile / 2) + swz(row, t + 4 * (i & 1)));
                                mma_bf16(sc[q], f.q[2 * i], x.x, x.y);
                                mma_bf16(sc[q], f.q[2 * i + 1], x.z, x.w);
                                mma_bf16(sc[q], f.lo[2 * i], x.x, x.y);
                                mma_bf16(sc[q], f.lo[2 * i + 1], x.z, x.w);
                            }
                        }
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < 2; q++) {
                        if (key0 + 8 * q > nodes) break;
                        const int j = key0 + slot_row(q, g);
                        uint32_t w[4][4];
#pragma unroll
                        for (int i = 0; i < 4; i++)
#pragma unroll
                            for (int e = 0; e < 4; e++) w[i][e] = 0u;
                        if (j <= nodes) {
                            const int pos = len + (j > 0 ? __ldg(a.depths + static_cast<long long>(s) * a.B + j - 1) : 0);
                            const __nv_bfloat16* k = a.k + (seq_row + j) * a.k_stride + head * kHeadDim;
#pragma unroll
                            for (int i = 0; i < 2; i++) {
                                const int d0 = 8 * k_piece<kFp8>(i, t);
                                const uint4 x = __ldg(reinterpret_cast<const uint4*>(k + d0));
                                const uint4 y = __ldg(reinterpret_cast<const uint4*>(k + d0 + 64));
                                const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                                for (int e = 0; e < 4; e++) {
                                    float s0, c0, s1, c1;
                                    rope_sincos(a.turns.f[d0 + 2 * e], pos, &s0, &c0);
                                    rope_sincos(a.turns.f[d0 + 2 * e + 1], pos, &s1, &c1);
                                    const float x0 = bf16_lo(xw[e]), x1 = bf16_hi(xw[e]), y0 = bf16_lo(yw[e]), y1 = bf16_hi(yw[e]);
                                    w[i][e] = pack_bf16x2(x0 * c0 - y0 * s0, x1 * c1 - y1 * s1);
                                    w[i + 2][e] = pack_bf16x2(y0 * c0 + x0 * s0, y1 * c1 + x1 * s1);
                                }
                            }
                        }
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 4; i++)
#pragma unroll
                            for (int h = 0; h < 2; h++) {
                                if (kFp8) {  // the queries as bf16: tree keys may leave f16's range
                                    uint32_t qb[4];
#pragma unroll
                                    for (int e = 0; e < 4; e++) {
                                        const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&f.q[2 * i + h][e]));
                                        qb[e] = pack_bf16x2(x.x, x.y);
                                    }
                                    mma_bf16(sc[q], qb, w[i][2 * h], w[i][2 * h + 1]);
                                } else {
                                    mma_bf16(sc[q], f.q[2 * i + h], w[i][2 * h], w[i][2 * h + 1]);
                                    mma_bf16(sc[q], f.lo[2 * i + h], w[i][2 * h], w[i][2 * h + 1]);
                                }
                            }
                    }
                }

                // scores in log2 units, hidden keys -inf
                float mx[2] = {-INFINITY, -INFINITY};
                const bool part_hidden = key0 + kChunk > live || !ctx;
#pragma unroll
                for (int q = 0; q < 2; q++)
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        const int key = slot_row(q, 2 * t + e);
                        const float by = kFp8 && ctx ? sck[key] : 1.0f;
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            float x = sc[q][2 * h + e] * (rs[h] * by);
                            if (part_hidden) {
                                bool see = key0 + key < live;
                                if (!ctx && see && key0 + key > 0) {
                                    const int b = (row0 + g + 8 * h) / a.G, bit = key0 + key - 1;
                                    see = b > 0 && b <= nodes &&
                                          ((__ldg(a.mask + (static_cast<long long>(s) * a.B + b - 1) * a.mw + (bit >> 6)) >> (bit & 63)) & 1ull);
                                }
                                if (!see) x = -INFINITY;
                            }
                            sc[q][2 * h + e] = x;
                            mx[h] = fmaxf(mx[h], x);
                        }
                    }
                if (__any_sync(kFull, mx[0] > f.m[0] + kSlack || mx[1] > f.m[1] + kSlack)) {
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        float x = fmaxf(mx[h], __shfl_xor_sync(kFull, mx[h], 1));
                        x = fmaxf(f.m[h], fmaxf(x, __shfl_xor_sync(kFull, x, 2)));
                        const float alpha = f.m[h] == -INFINITY ? 0.0f : exp2_fast(f.m[h] - x);
                        f.m[h] = x;
                        f.l[h] *= alpha;
#pragma unroll
                        for (int j = 0; j < 16; j++) {
                            f.acc[j][2 * h] *= alpha;
                            f.acc[j][2 * h + 1] *= alpha;
                        }
                    }
                }
                uint32_t p[4];
#pragma unroll
                for (int q = 0; q < 2; q++)
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        const float ref = f.m[h] == -INFINITY ? 0.0f : f.m[h];
                        float w[2];
#pragma unroll
                        for (int e = 0; e < 2; e++) {
                            w[e] = exp2_fast(sc[q][2 * h + e] - ref);
                            f.l[h] += w[e];
                            if (kFp8 && ctx) {
                                const int key = slot_row(q, 2 * t + e);
                                w[e] = key0 + key < live ? w[e] * sck[16 + key] : 0.0f;
                            }
                        }
                        p[2 * q + h] = pack_bf16x2(w[0], w[1]);
                    }

                // O += P V
                if (ctx && kFp8) {
                    uint4 x[2][2];
#pragma unroll
                    for (int q = 0; q < 2; q++)
#pragma unroll
                        for (int e = 0; e < 2; e++) {
                            const int row = slot_row(q, 2 * t + e);
                            x[q][e] = *reinterpret_cast<const uint4*>(vt + swz(row, g));
                            if (key0 + row >= live) x[q][e] = make_uint4(0, 0, 0, 0);  // (NaN codes may lie there)
                        }
#pragma unroll
                    for (int w = 0; w < 4; w++) {
                        auto word = [&](int q, int e) { return w == 0 ? x[q][e].x : w == 1 ? x[q][e].y : w == 2 ? x[q][e].z : x[q][e].w; };
#pragma unroll
                        for (int b = 0; b < 4; b++) {
                            const uint32_t sel = ((4u + b) << 12) | (static_cast<uint32_t>(b) << 4);
                            mma_bf16(f.acc[4 * w + b], p, e4m3_to_bf16(__byte_perm(word(0, 0), word(0, 1), sel)),
                                     e4m3_to_bf16(__byte_perm(word(1, 0), word(1, 1), sel)));
                        }
                    }
                } else {
#pragma unroll
                    for (int half = 0; half < 2; half++) {
                        uint4 x[2][2];
#pragma unroll
                        for (int q = 0; q < 2; q++)
#pragma unroll
                            for (int e = 0; e < 2; e++) {
                                const int row = slot_row(q, 2 * t + e);
                                x[q][e] = make_uint4(0, 0, 0, 0);
                                if (key0 + row < live) {
                                    if (ctx)
                                        x[q][e] = *reinterpret_cast<const uint4*>(vt + half * (G_::kTile / 2) + swz(row, g));
                                    else
                                        x[q][e] = __ldg(reinterpret_cast<const uint4*>(a.v + (seq_row + key0 + row) * a.v_stride +
                                                                                       head * kHeadDim + 8 * (kFp8 ? 2 * g + half : g + 8 * half)));
                                }
                            }
#pragma unroll
                        for (int w = 0; w < 4; w++) {
                            auto word = [&](int q, int e) { return w == 0 ? x[q][e].x : w == 1 ? x[q][e].y : w == 2 ? x[q][e].z : x[q][e].w; };
                            mma_bf16(f.acc[8 * half + 2 * w], p, __byte_perm(word(0, 0), word(0, 1), 0x5410),
                                     __byte_perm(word(1, 0), word(1, 1), 0x5410));
                            mma_bf16(f.acc[8 * half + 2 * w + 1], p, __byte_perm(word(0, 0), word(0, 1), 0x7632),
                                     __byte_perm(word(1, 0), word(1, 1), 0x7632));
                        }
                    }
                }
            }
            __syncwarp();  // every lane has read the stage
            if (ctx) n_use++;
            use_at += kWarps;
            if (use_at < end) use.advance(a, kWarps);
            while (ok && load_at < end && n_load - n_use < G_::kStages) issue();
        }

        // ---- the warps' results into one
#pragma unroll
        for (int h = 0; h < 2; h++) {
            f.l[h] += __shfl_xor_sync(kFull, f.l[h], 1);
            f.l[h] += __shfl_xor_sync(kFull, f.l[h], 2);
            if (t == 0) stat[warp * kUnitRows + g + 8 * h] = make_float2(f.m[h], f.l[h]);
        }
        __syncthreads();  // (the queries before the merge buffer have been read)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            float top = -INFINITY;
            for (int w = 0; w < kWarps; w++) top = fmaxf(top, stat[w * kUnitRows + g + 8 * h].x);
            const float by = f.m[h] == -INFINITY ? 0.0f : exp2_fast(f.m[h] - top);
#pragma unroll
            for (int j = 0; j < 16; j++) {
                f.acc[j][2 * h] *= by;
                f.acc[j][2 * h + 1] *= by;
            }
        }
        float* buf = reinterpret_cast<float*>(merge) + (warp & 3) * 64 * 32 + lane;
        if (warp >= 4)
#pragma unroll
            for (int j = 0; j < 16; j++)
#pragma unroll
                for (int e = 0; e < 4; e++) buf[(4 * j + e) * 32] = f.acc[j][e];
        __syncthreads();
        if (warp < 4)
#pragma unroll
            for (int j = 0; j < 16; j++)
#pragma unroll
                for (int e = 0; e < 4; e++) buf[(4 * j + e) * 32] += f.acc[j][e];
        __syncthreads();
        {
            const int r = tid >> 4, d8 = tid & 15, b = (row0 + r) / a.G;
            const int n = kFp8 ? d8 >> 1 : d8 & 7, j0 = kFp8 ? (d8 & 1) * 8 : (d8 >> 3) * 8;
            const float* src = reinterpret_cast<const float*>(merge) + ((r >> 3) * 2 + (n & 1)) * 32 + (r & 7) * 4 + (n >> 1);
            if (b <= nodes) {
                float top = -INFINITY, l = 0.0f;
                for (int w = 0; w < kWarps; w++) top = fmaxf(top, stat[w * kUnitRows + r].x);
                for (int w = 0; w < kWarps; w++) {
                    const float2 x = stat[w * kUnitRows + r];
                    if (x.x != -INFINITY) l += x.y * exp2_fast(x.x - top);
                }
                float o[8];
#pragma unroll
                for (int k = 0; k < 8; k++) {
                    o[k] = 0.0f;
#pragma unroll
                    for (int w = 0; w < 4; w++) o[k] += src[w * 64 * 32 + (j0 + k) * 128];
                }
                if (unit.chunk == 0 && part == unit.chunks) {
                    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
                    __nv_bfloat16* d = a.out + ((seq_row + b) * a.Hq + head * a.G + (row0 + r) % a.G) * kHeadDim + 8 * d8;
                    *reinterpret_cast<uint4*>(d) = make_uint4(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv),
                                                              pack_bf16x2(o[4] * inv, o[5] * inv), pack_bf16x2(o[6] * inv, o[7] * inv));
                } else {
                    Part* d = a.parts + 2 * blockIdx.x + (unit.chunk > 0 ? 0 : 1);
                    float4* w = reinterpret_cast<float4*>(&d->o[r][8 * d8]);
                    w[0] = make_float4(o[0], o[1], o[2], o[3]);
                    w[1] = make_float4(o[4], o[5], o[6], o[7]);
                    if (d8 == 0) d->ml[r] = make_float2(top, l);
                }
            }
        }
        at += part;
        unit.advance(a, part);
    }
    if (!ok) {  // copies in flight land before the CTA ends
        const unsigned long long t0 = globaltimer_ns();
        for (int i = n_use; i < n_load; i++)
            while (!mbar_try_wait(bar + i % G_::kStages, static_cast<uint32_t>(i / G_::kStages) & 1u))
                if (globaltimer_ns() - t0 > kWaitLimitNs) break;
    }
}

// Joins the parts of the units that several CTAs shared, in the order of
// their keys.  One block per unit; 16 threads a row, 8 elements each.
__global__ void __launch_bounds__(kThreads) paged_join_kernel(const __grid_constant__ PagedArgs a, int grid_ctas) {
    pdl_trigger();
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31;
    const int per = a.Hkv * a.nrg, s = blockIdx.x / per;
    Place p{};
    p.s = s;
    p.unit = blockIdx.x % per;
    p.load(a);
    if (p.unit >= p.units) return;
    const long long all = chunks_before(a, a.nseq, lane);
    const int ctas = active_ctas(all, grid_ctas);
    const long long first = chunks_before(a, s, lane) + static_cast<long long>(p.unit) * p.chunks;
    const int c0 = share_of_chunk(all, ctas, first), c1 = share_of_chunk(all, ctas, first + p.chunks - 1);
    if (c0 == c1) return;
    const int groups = p.groups(a), head = p.unit / groups, row0 = (p.unit % groups) * kUnitRows;
    const int r = tid >> 4, d8 = tid & 15, b = (row0 + r) / a.G;
    if (b > p.nodes) return;
    auto slot = [&](int c) { return a.parts + 2 * c + (share_begin(all, ctas, c) > first ? 0 : 1); };
    float top = -INFINITY;
    for (int c = c0; c <= c1; c++) top = fmaxf(top, slot(c)->ml[r].x);
    float l = 0.0f, o[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    for (int c = c0; c <= c1; c++) {
        const Part* x = slot(c);
        const float2 ml = x->ml[r];
        if (ml.x == -INFINITY) continue;
        const float by = exp2_fast(ml.x - top);
        const float4 u = *reinterpret_cast<const float4*>(&x->o[r][8 * d8]), v = *reinterpret_cast<const float4*>(&x->o[r][8 * d8 + 4]);
        l += ml.y * by;
        o[0] += u.x * by;
        o[1] += u.y * by;
        o[2] += u.z * by;
        o[3] += u.w * by;
        o[4] += v.x * by;
        o[5] += v.y * by;
        o[6] += v.z * by;
        o[7] += v.w * by;
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    __nv_bfloat16* d = a.out + ((static_cast<long long>(s) * (a.B + 1) + b) * a.Hq + head * a.G + (row0 + r) % a.G) * kHeadDim + 8 * d8;
    *reinterpret_cast<uint4*>(d) = make_uint4(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv),
                                              pack_bf16x2(o[4] * inv, o[5] * inv), pack_bf16x2(o[6] * inv, o[7] * inv));
}

// ------------------------------------------------------------ host

bool valid_cfg(const dart_paged_attn_config* c, const dart_kv_cache* cache) {
    if (!c || !valid_cache(cache)) return false;
    if (c->nseq < 1 || c->B < 0 || c->B > 1024 || c->max_pages < 1 || c->Hq < cache->Hkv || c->Hq % cache->Hkv) return false;
    const int G = c->Hq / cache->Hkv;
    if (G != 1 && G != 2 && G != 4 && G != 8 && G != 16) return false;
    if (!(c->rope_theta > 1.0f) || !std::isfinite(c->rope_theta) || !(c->scale > 0.0f) || !std::isfinite(c->scale)) return false;
    // positions (with the tree's depths) and the numbers of rows are 32-bit
    if (static_cast<long long>(c->max_pages) * cache->page_size > (1ll << 30)) return false;
    return static_cast<long long>(c->nseq) * (c->B + 1) * c->Hq <= (1ll << 30);
}

// Rows of dh elements (the whole pool) in boxes of 16 rows by 128 bytes.
bool encode_pool(CUtensorMap* m, const void* base, long long rows, bool fp8) {
    EncodeTiledFn fn = tensor_map_encoder();
    if (!fn) return false;
    const cuuint64_t dims[2] = {kHeadDim, static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(kHeadDim) * (fp8 ? 1 : 2)};
    const cuuint32_t box[2] = {fp8 ? 128u : 64u, kChunk}, estr[2] = {1, 1};
    return fn(m, fp8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides,
              box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The device's number of SMs; 0 if it is not sm_103a, -1 on an error.  The
// shared-memory opt-in of the kernels is set on the first call per device.
int device_sms(int dev) {
    static std::atomic<int> known[64];
    if (dev < 0 || dev >= 64) return -1;
    const int k = known[dev].load(std::memory_order_acquire);
    if (k) return k;
    int major = 0, minor = 0, sms = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return -1;
    if (major != 10 || minor != 3) return 0;
    if (cudaFuncSetAttribute(paged_rows_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, Geo<false>::kSmem) != cudaSuccess ||
        cudaFuncSetAttribute(paged_rows_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, Geo<true>::kSmem) != cudaSuccess)
        return -1;
    known[dev].store(sms, std::memory_order_release);
    return sms;
}

}  // namespace
}  // namespace dart

using namespace dart;

extern "C" {

size_t dart_paged_attention_workspace(const dart_paged_attn_config* cfg, const dart_kv_cache* cache) {
    if (!valid_cfg(cfg, cache)) return 0;
    return sizeof(Part) * 2 * kMaxCtas;
}

int dart_paged_attention(const dart_paged_attn_config* cfg, const dart_kv_cache* cache, const int32_t* page_table,
                         const int32_t* lens, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                         const void* v, int64_t v_stride, const int32_t* depths, const uint64_t* mask,
                         const int32_t* n_nodes, void* out, void* workspace, size_t workspace_bytes, int* status,
                         void* stream) {
    if (!valid_cfg(cfg, cache) || !valid_cache_pointers(cache)) return DART_ERR_INVALID;
    const dart_paged_attn_config& c = *cfg;
    auto al = [](const void* p, uintptr_t n) { return p && (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
    if (!al(page_table, 4) || !al(lens, 4) || !al(q, 16) || !al(k, 16) || !al(v, 16) || !al(out, 16) || !al(workspace, 256))
        return DART_ERR_INVALID;
    if (c.B > 0 && (!al(depths, 4) || !al(mask, 8) || !al(n_nodes, 4))) return DART_ERR_INVALID;
    if (status && !al(status, 4)) return DART_ERR_INVALID;
    const int64_t width = static_cast<int64_t>(cache->Hkv) * kHeadDim;
    if (q_stride < static_cast<int64_t>(c.Hq) * kHeadDim || k_stride < width || v_stride < width) return DART_ERR_INVALID;
    if (q_stride % 8 || k_stride % 8 || v_stride % 8) return DART_ERR_INVALID;
    if (workspace_bytes < dart_paged_attention_workspace(cfg, cache)) return DART_ERR_INVALID;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return DART_ERR_CUDA;
    const int sms = device_sms(dev);
    if (sms <= 0) return sms < 0 ? DART_ERR_CUDA : DART_ERR_UNSUPPORTED;

    const bool fp8 = cache->dtype == DART_KV_E4M3;
    PagedArgs a{};
    a.nseq = c.nseq;
    a.B = c.B;
    a.Hq = c.Hq;
    a.Hkv = cache->Hkv;
    a.G = c.Hq / cache->Hkv;
    a.nrg = ((c.B + 1) * a.G + kUnitRows - 1) / kUnitRows;
    a.max_pages = c.max_pages;
    while ((1 << a.page_log2) < cache->page_size) a.page_log2++;
    a.num_pages = cache->num_pages;
    a.mw = (c.B + 63) / 64;
    a.pool_rows = static_cast<long long>(cache->num_pages) * cache->Hkv * cache->page_size;
    a.table = page_table;
    a.lens = lens;
    a.depths = depths;
    a.n_nodes = n_nodes;
    a.mask = mask;
    a.q = static_cast<const __nv_bfloat16*>(q);
    a.k = static_cast<const __nv_bfloat16*>(k);
    a.v = static_cast<const __nv_bfloat16*>(v);
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.ks = cache->k_scale;
    a.vs = cache->v_scale;
    a.out = static_cast<__nv_bfloat16*>(out);
    a.parts = static_cast<Part*>(workspace);
    a.status = status;
    a.sl2 = static_cast<float>(static_cast<double>(c.scale) * 1.4426950408889634);
    a.turns = rope_turns(c.rope_theta);
    CUtensorMap tmK, tmV;
    if (!encode_pool(&tmK, cache->k, a.pool_rows, fp8) || !encode_pool(&tmV, cache->v, a.pool_rows, fp8)) return DART_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int ctas = std::min(sms, kMaxCtas);
    const cudaError_t e = fp8 ? launch_pdl(paged_rows_kernel<true>, dim3(ctas), dim3(kThreads), Geo<true>::kSmem, st, tmK, tmV, a)
                              : launch_pdl(paged_rows_kernel<false>, dim3(ctas), dim3(kThreads), Geo<false>::kSmem, st, tmK, tmV, a);
    if (e != cudaSuccess) return DART_ERR_CUDA;
    if (launch_pdl(paged_join_kernel, dim3(c.nseq * a.Hkv * a.nrg), dim3(kThreads), 0, st, a, ctas) != cudaSuccess) return DART_ERR_CUDA;
    return DART_OK;
}

}  // extern "C"

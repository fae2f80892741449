// Tree attention over the paged cache for more than 16 query rows per kv head:
// 128-row tiles on the tensor cores (tcgen05, operands and accumulators in
// tensor memory).  Contract: include/dart_cache.h.
//
// Launches of a call:
//   paged_prep_kernel  rotated queries, one row per (kv head, tree row, head
//       of the group), with bf16 pages as two bf16 terms; and, per sequence and kv head, the "side" keys and
//       values: the last len % 128 cache tokens (in bf16), the tree rows
//       (keys rotated), zeros up to a multiple of 128.  So all other cache
//       tiles are whole, need no mask, and nothing unwritten is ever read.
//   paged_widen_kernel  e4m3 pages that several query tiles read: as f16 tiles.
//   paged_tiles_kernel  a unit is 128 query rows of a kv head against the
//       whole cache tiles and the side tiles that its rows may see.  The
//       tiles of all units form one list that the CTAs (one per SM) share
//       evenly: ragged lengths, one long sequence and many short ones load
//       every SM alike.  A CTA runs through its units without a pause: loads
//       run ahead across units, and a unit's queries are written while the
//       last product of the unit before runs.
//   paged_tiles_join_kernel  joins the units that several CTAs shared.
//
// Roles in a CTA: warp 0 loads tiles by TMA, page by page (K ring, V ring);
// warp 1 issues the MMAs; warps 2-9 are two softmax warpgroups (thread = query
// row = TMEM lane; warpgroup wg owns key and output columns [64 wg, 64 wg +
// 64), the two warps of a lane quarter exchange maxima and sums).  With e4m3
// pages all operands are f16: four more warps turn raw tiles into f16, each
// key's codes times its scale over a power of two that the tile (K) or the
// unit so far (V) has in common; queries and side rows are f16 with a power
// of two per row.  So nothing can overflow, and the softmax has one factor a
// tile to apply instead of one a key (64 broadcast reads of a key's scale from
// shared memory, twice, took 0.5 us of a tile's 1.6).  TMEM (512 columns): S
// [0,128), O [128,256), P [256,384) in two buffers, Q [384,448), and with bf16
// pages what the queries' first bf16 term leaves, [448,512).
// A row's running maximum is raised (and O rescaled) only when a tile exceeds
// it by more than 2^8.  Every wait is bounded.
//
// Measured: a tile takes 1.07 us from bf16 pages (24 MMAs of 64 cycles are 0.8) and
// 1.05 from widened ones (16 MMAs, 0.53); eight trees of 512 nodes over up to 4096
// keys take 241 and 270 us with everything around.  With the first term of the
// queries alone bf16 pages took 0.90 and 211 us, at an error against 64 bits of
// 0.0029 of the output instead of 0.0023 (its own rounding is 0.0017).  What a tile takes
// beside its MMAs is the chain of the softmax's instructions (two warps a
// scheduler, in step because they share rows: exponentials 0.3 us, maxima, the
// exchange, 0.1 us for each wait) beside the issuing warp's, which is almost as
// long.  Tried, when those eight trees took 235 us with bf16 pages: four softmax warpgroups of 32
// columns (287 us: the fixed part of the instructions doubles); CTA pairs with half
// of K and V each (383: one more hop in every exchange); S in two buffers and P in
// one (262); later, mask words read a tile ahead (216 instead of 211: registers).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cstdint>
#include <cstring>

#include "../../include/dart.h"
#include "dart_kernels.h"
#include "dart_paged.cuh"
#include "dart_tmem.cuh"

namespace dart {
namespace {

// Where K and V tiles come from: bf16 pages; e4m3 pages, converted in the CTA;
// e4m3 pages that paged_widen_kernel has laid out as f16 tiles before.
enum Source { kPages, kCodes, kWidened };
constexpr int kRows = 128;               // query rows per unit (MMA M)
constexpr int kKeys = 128;               // keys per tile
constexpr int kHalf = kKeys * 128;       // 128 rows of one 128-byte swizzle column
constexpr int kTile = 2 * kHalf;         // 128 keys of bf16
constexpr int kSoft = 256;               // softmax threads
constexpr int kPairBar = 2;              // named barriers 2 .. 5
constexpr int kConvBar = 6;              // 6: the warps that convert K, 7: V
constexpr float kSlack8 = 8.0f;          // log2 units: P <= 2^8 between rescales
// What a unit costs beside its tiles (its queries, its result, the pause between
// its last tile and the next unit's first), in tiles: eight trees of 512 nodes over
// 4096 bf16 keys 241 us with 3 and 4, 245 with 6; e4m3 273, 270, 274.
constexpr int kTileCost = 4;
constexpr int kMinTiles = 2;             // of a share (one tree of 20 nodes over 500 keys: 1 18.5 us, 2 17.9, 4 19.8)
constexpr uint32_t kSCol = 0, kOCol = 128, kPCol = 256, kQCol = 384, kQLoCol = 448;

// Rows that threads of a warp read or write one each are kept a 16-byte piece
// after the other: piece c of row r of a 128-row tile at [c][r].
struct TilePart {
    float4 o[kHeadDim / 4][kRows];
    float2 ml[kRows];
};

struct TileArgs {
    PagedArgs p;
    int sk;                    // side keys per sequence and kv head (a multiple of 128)
    int nqt;                    // query tiles of a kv head of a full tree
    // bf16, or f16 (e4m3 pages) with a factor per row:
    uint4* qr;                  // [nseq][Hkv][nqt][16 pieces][128 rows]
    uint4* q_lo;                // bf16: what the first term leaves, the same way
    uint4 *side_k, *side_v;     // [nseq][Hkv][sk] rows; e4m3 pages: [nseq][Hkv][sk / 128][16 pieces][128]
    float* q_scale;             // [nseq][Hkv][nqt][128], with scale * log2(e) in it
    float *side_ks, *side_vs;   // [nseq][Hkv][sk]
    // kWidened: all tiles of a kv head, f16 times a power of two each of K and V
    int wide_tiles;             // room per sequence and kv head
    uint4 *wide_k, *wide_v;     // [nseq][Hkv][wide_tiles * 128] rows
    float2* wide_refs;          // [nseq][Hkv][wide_tiles]
};

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// Two e4m3 codes as an f16 pair: exact.
__device__ __forceinline__ uint32_t codes_to_f16(uint32_t two) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(static_cast<uint16_t>(two)));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16x2(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// ------------------------------------------------------------ preparation

// 16 of a row's 128 values: elements 8 p .. 8 p + 7 and 64 + 8 p .. of lane p of
// a group of 8.
struct Piece {
    float lo[8], hi[8];
};
__device__ __forceinline__ Piece unpack_piece(const uint4& a, const uint4& b) {
    const uint32_t u[4] = {a.x, a.y, a.z, a.w}, w[4] = {b.x, b.y, b.z, b.w};
    Piece x;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        x.lo[2 * e] = bf16_lo(u[e]);
        x.lo[2 * e + 1] = bf16_hi(u[e]);
        x.hi[2 * e] = bf16_lo(w[e]);
        x.hi[2 * e + 1] = bf16_hi(w[e]);
    }
    return x;
}
// As bf16, or as f16 scaled by a power of two to a largest element of the row
// in [1, 2); returns the factor that undoes it.  (All lanes of the warp.)
template <bool kF16>
__device__ __forceinline__ float pack_piece(const Piece& x, uint4* lo, uint4* hi) {
    float down = 1.0f, factor = 1.0f;
    if (kF16) {
        float mx = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; e++) mx = fmaxf(mx, fmaxf(fabsf(x.lo[e]), fabsf(x.hi[e])));
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, o));
        const int ex = min(max(static_cast<int>(__float_as_uint(mx) >> 23) - 127, -100), 120);
        down = __uint_as_float(static_cast<uint32_t>(127 - ex) << 23);
        factor = __uint_as_float(static_cast<uint32_t>(127 + ex) << 23);
    }
    auto two = [&](float a, float b) { return kF16 ? pack_f16x2(a * down, b * down) : pack_bf16x2(a, b); };
    *lo = make_uint4(two(x.lo[0], x.lo[1]), two(x.lo[2], x.lo[3]), two(x.lo[4], x.lo[5]), two(x.lo[6], x.lo[7]));
    *hi = make_uint4(two(x.hi[0], x.hi[1]), two(x.hi[2], x.hi[3]), two(x.hi[4], x.hi[5]), two(x.hi[6], x.hi[7]));
    return factor;
}

// Blocks 0 .. B of a sequence: a tree row's keys and values (side rows), head by
// head by groups of 8 threads, and its rotated queries; blocks from B + 1 on: the
// side rows that are no tree rows.
constexpr int kPrepThreads = 256, kGroups = kPrepThreads / 8;
template <bool kFp8>
__global__ void __launch_bounds__(kPrepThreads) paged_prep_kernel(const __grid_constant__ TileArgs ta, const uint8_t* pool_k, const uint8_t* pool_v) {
    __shared__ float2 turn_of[kHeadDim / 2];  // cos, sin
    const PagedArgs& a = ta.p;
    const int tid = threadIdx.x, p = tid & 7, group = tid >> 3, s = blockIdx.x, b = blockIdx.y;
    const long long in = static_cast<long long>(s) * (a.B + 1) + b;
    const int rows = a.Hq + 2 * a.Hkv;  // queries, keys, values of a tree row
    auto source = [&](int i) {
        return i < a.Hq ? a.q + in * a.q_stride + i * kHeadDim
                        : i < a.Hq + a.Hkv ? a.k + in * a.k_stride + (i - a.Hq) * kHeadDim : a.v + in * a.v_stride + (i - a.Hq - a.Hkv) * kHeadDim;
    };
    constexpr int kBatch = 2;  // rows of a group on their way at a time
    uint4 raw[kBatch][2];
    auto fetch = [&](int i0) {
#pragma unroll
        for (int u = 0; u < kBatch; u++) {
            const int i = i0 + u * kGroups + group;
            raw[u][0] = raw[u][1] = make_uint4(0u, 0u, 0u, 0u);
            if (i < rows) {
                raw[u][0] = ld_plain(reinterpret_cast<const uint4*>(source(i)) + p);
                raw[u][1] = ld_plain(reinterpret_cast<const uint4*>(source(i)) + 8 + p);
            }
        }
    };
    pdl_wait();
    pdl_trigger();  // (after the wait: the next kernel reads lengths and pages before its own)
    if (b <= a.B) fetch(0);  // (whatever the length and the number of nodes are)
    const int depth = b > 0 && b <= a.B ? ld_plain(a.depths + static_cast<long long>(s) * a.B + b - 1) : 0;
    const int len = seq_len(a, s), nodes = seq_nodes(a, s), tail = len % kKeys;
    const int end = (tail + nodes) / kKeys * kKeys + kKeys;  // side rows that a tile reads
    auto put_side = [&](int kv, int head, int j, const uint4& lo, const uint4& hi) {
        uint4* d = kv ? ta.side_v : ta.side_k;
        const long long row = (static_cast<long long>(s) * a.Hkv + head) * ta.sk + j;
        if (kFp8) {
            d += (row >> 7) * (16 * kKeys) + (row & 127);
            d[p * kKeys] = lo;
            d[(8 + p) * kKeys] = hi;
        } else {
            d[row * 16 + p] = lo;
            d[row * 16 + 8 + p] = hi;
        }
    };
    auto put_scale = [&](int kv, int head, int j, float x) {
        if (kFp8 && p == 0) (kv ? ta.side_vs : ta.side_ks)[(static_cast<long long>(s) * a.Hkv + head) * ta.sk + j] = x;
    };
    if (b > a.B) {
        int j = b - a.B - 1;  // of the side rows that are no tree rows: before them, then after them
        if (j >= tail) j += nodes + 1;
        if (j >= end) return;
        // a token of the cache: its codes or values as they are; zeros after the nodes
        const int key = len - tail + j;
        const int page = j < tail ? ld_plain(a.table + static_cast<long long>(s) * a.max_pages + (key >> a.page_log2)) : -1;
        const bool there = page >= 0 && page < a.num_pages;
        if (j < tail && !there && a.status && tid == 0) atomicOr(a.status, kDevBounds);
        for (int i = group; i < 2 * a.Hkv; i += kGroups) {
            const int kv = i >= a.Hkv, head = i - kv * a.Hkv;
            const long long row = there ? ((static_cast<long long>(page) * a.Hkv + head) << a.page_log2) + (key & ((1 << a.page_log2) - 1)) : 0;
            const uint8_t* pool = kv ? pool_v : pool_k;
            uint4 lo = make_uint4(0u, 0u, 0u, 0u), hi = lo;
            if (there && kFp8) {
                const uint2 x = *reinterpret_cast<const uint2*>(pool + row * kHeadDim + 8 * p), y = *reinterpret_cast<const uint2*>(pool + row * kHeadDim + 64 + 8 * p);
                lo = make_uint4(codes_to_f16(x.x), codes_to_f16(x.x >> 16), codes_to_f16(x.y), codes_to_f16(x.y >> 16));
                hi = make_uint4(codes_to_f16(y.x), codes_to_f16(y.x >> 16), codes_to_f16(y.y), codes_to_f16(y.y >> 16));
            } else if (there) {
                lo = reinterpret_cast<const uint4*>(pool)[row * 16 + p];
                hi = reinterpret_cast<const uint4*>(pool)[row * 16 + 8 + p];
            }
            put_side(kv, head, j, lo, hi);
            if (kFp8) put_scale(kv, head, j, there ? ld_plain((kv ? a.vs : a.ks) + row) : 0.0f);
        }
        return;
    }
    if (b > nodes) {  // no node: zeros as output
        uint4* out = reinterpret_cast<uint4*>(a.out + in * a.Hq * kHeadDim);
        for (int i = tid; i < a.Hq * 16; i += kPrepThreads) out[i] = make_uint4(0u, 0u, 0u, 0u);
        return;
    }
    if (tid < kHeadDim / 2) {
        float sn, cs;
        rope_sincos(a.turns.f[tid], len + depth, &sn, &cs);
        turn_of[tid] = make_float2(cs, sn);
    }
    __syncthreads();
    for (int i0 = 0; i0 < rows; i0 += kBatch * kGroups) {
        if (i0 > 0) fetch(i0);
#pragma unroll
        for (int u = 0; u < kBatch; u++) {
            if (i0 + u * kGroups >= rows) break;  // (whole warps stay together)
            const int i = i0 + u * kGroups + group;
            Piece x = unpack_piece(raw[u][0], raw[u][1]);
            if (i < a.Hq + a.Hkv)
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const float2 t = turn_of[8 * p + e];
                    const float lo = x.lo[e], hi = x.hi[e];
                    x.lo[e] = lo * t.x - hi * t.y;
                    x.hi[e] = hi * t.x + lo * t.y;
                }
            uint4 lo, hi;
            const float factor = pack_piece<kFp8>(x, &lo, &hi);
            if (i < a.Hq) {
                const int head = i >> a.g_log2, row = (b << a.g_log2) + (i & (a.G - 1));
                const long long tile = (static_cast<long long>(s) * a.Hkv + head) * ta.nqt + (row >> 7);
                uint4* d = ta.qr + tile * (16 * kRows) + (row & 127);
                d[p * kRows] = lo;
                d[(8 + p) * kRows] = hi;
                if (!kFp8) {
                    // with one bf16 term the queries' rounding alone would move the output as
                    // much as its own rounding does
                    const Piece y = unpack_piece(lo, hi);
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        x.lo[e] -= y.lo[e];
                        x.hi[e] -= y.hi[e];
                    }
                    pack_piece<false>(x, &lo, &hi);
                    d = ta.q_lo + tile * (16 * kRows) + (row & 127);
                    d[p * kRows] = lo;
                    d[(8 + p) * kRows] = hi;
                }
                if (kFp8 && p == 0) ta.q_scale[tile * kRows + (row & 127)] = factor * a.sl2;
            } else if (i < rows) {
                const int kv = i >= a.Hq + a.Hkv, head = i - a.Hq - kv * a.Hkv;
                put_side(kv, head, tail + b, lo, hi);
                put_scale(kv, head, tail + b, factor);
            }
        }
    }
}

// The logarithm of a power of two.
__device__ __forceinline__ float log2_of(float x) { return static_cast<float>(static_cast<int>(__float_as_uint(x) >> 23) - 127); }
// A power of two above x >= 0.
__device__ __forceinline__ float above(float x) {
    return __uint_as_float((min(max(__float_as_uint(x) >> 23, 27u), 252u) + 1u) << 23);
}

// ------------------------------------------------------------ e4m3 pages as f16 tiles

// One block per tile of a sequence and kv head (whole cache tiles, then side
// tiles): codes times their key's scale over a power of two that the tile's
// keys (and, apart, values) have in common, rounded once to f16.  Converting in
// the tiles kernel costs 0.8 us a tile of every unit, and this 2 us a tile once.
__global__ void __launch_bounds__(256) paged_widen_kernel(const __grid_constant__ TileArgs ta, const uint8_t* pool_k, const uint8_t* pool_v) {
    __shared__ float scale_of[2 * kKeys];
    __shared__ int row_of[kKeys];  // of the pool; -1: no such page
    __shared__ float top_of[8];
    const PagedArgs& a = ta.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int head = blockIdx.x % a.Hkv, s = blockIdx.x / a.Hkv, t = blockIdx.y;
    pdl_wait();
    pdl_trigger();
    const int len = seq_len(a, s), nodes = seq_nodes(a, s), whole = len / kKeys, tail = len % kKeys;
    if (t > whole + (tail + nodes) / kKeys) return;
    const bool cache_tile = t < whole;
    const long long side = (static_cast<long long>(s) * a.Hkv + head) * ta.sk + (t - whole) * kKeys;
    if (cache_tile && tid < kKeys) {
        const int at = t * kKeys + tid;
        const int page = ld_plain(a.table + static_cast<long long>(s) * a.max_pages + (at >> a.page_log2));
        const bool there = page >= 0 && page < a.num_pages;
        if (!there && a.status) atomicOr(a.status, kDevBounds);
        row_of[tid] = there ? static_cast<int>(((static_cast<long long>(page) * a.Hkv + head) << a.page_log2) + (at & ((1 << a.page_log2) - 1))) : -1;
    }
    __syncthreads();
    // groups of 8 lanes a row, 16 elements a lane: on their way while the scales are compared
    const int p = tid & 7, group = tid >> 3;
    constexpr int kRounds = 2 * kKeys / 32;
    uint4 c[kRounds];
    if (cache_tile)
#pragma unroll
        for (int i = 0; i < kRounds; i++) {
            const int row = row_of[(i * 32 + group) & 127];
            c[i] = make_uint4(0u, 0u, 0u, 0u);
            if (row >= 0) c[i] = ld_plain(reinterpret_cast<const uint4*>(i >= kRounds / 2 ? pool_v : pool_k) + static_cast<long long>(row) * 8 + p);
        }
    {
        const int kv = tid >> 7, key = tid & 127;
        float sc = 0.0f;
        if (!cache_tile)
            sc = __ldcg((kv ? ta.side_vs : ta.side_ks) + side + key);
        else if (row_of[key] >= 0)
            sc = ld_plain((kv ? a.vs : a.ks) + row_of[key]);
        scale_of[tid] = sc;
        const float top = __uint_as_float(__reduce_max_sync(kFull, __float_as_uint(fmaxf(sc, 0.0f))));
        if (lane == 0) top_of[warp] = top;
    }
    __syncthreads();
    float ref[2];
#pragma unroll
    for (int kv = 0; kv < 2; kv++) ref[kv] = above(fmaxf(fmaxf(top_of[4 * kv], top_of[4 * kv + 1]), fmaxf(top_of[4 * kv + 2], top_of[4 * kv + 3])));
    const long long tile = (static_cast<long long>(s) * a.Hkv + head) * ta.wide_tiles + t;
    if (tid == 0) ta.wide_refs[tile] = make_float2(ref[0], ref[1]);
#pragma unroll
    for (int i = 0; i < kRounds; i++) {
        const int kv = i >= kRounds / 2, key = (i * 32 + group) & 127;
        const __half2 by = __float2half2_rn(scale_of[kv * kKeys + key] * __uint_as_float(0x7F000000u - __float_as_uint(ref[kv])));
        uint32_t x[8];
        if (cache_tile) {
            const uint32_t w[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
#pragma unroll
            for (int e = 0; e < 4; e++) {
                x[2 * e] = codes_to_f16(w[e]);
                x[2 * e + 1] = codes_to_f16(w[e] >> 16);
            }
        } else {
            const uint4* src = (kv ? ta.side_v : ta.side_k) + (side >> 7) * (16 * kKeys) + key;
            const uint4 y = __ldcg(src + 2 * p * kKeys), z = __ldcg(src + (2 * p + 1) * kKeys);
            x[0] = y.x;
            x[1] = y.y;
            x[2] = y.z;
            x[3] = y.w;
            x[4] = z.x;
            x[5] = z.y;
            x[6] = z.z;
            x[7] = z.w;
        }
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&x[e]), by);
            x[e] = *reinterpret_cast<const uint32_t*>(&r);
        }
        uint4* d = (kv ? ta.wide_v : ta.wide_k) + (tile * kKeys + key) * 16 + 2 * p;
        d[0] = make_uint4(x[0], x[1], x[2], x[3]);
        d[1] = make_uint4(x[4], x[5], x[6], x[7]);
    }
}

// ------------------------------------------------------------ the schedule

// A place in the list: kv heads of a sequence one after the other, the units
// (query tiles) of a head one after the other.  A unit's length in the list is
// its tiles (its last row sees tree rows up to itself) and kTileCost.
struct TilePlace {
    int s, head, qt, tile;
    int len, nodes, whole, tail, nqt;  // of the sequence: whole cache tiles, cache tokens beside them, units per head
    __device__ __forceinline__ void load(const PagedArgs& a) {
        len = seq_len(a, s);
        nodes = seq_nodes(a, s);
        whole = len / kKeys;
        tail = len % kKeys;
        nqt = (((nodes + 1) << a.g_log2) + kRows - 1) / kRows;
    }
    __device__ __forceinline__ int tiles(const PagedArgs& a, int q) const {
        return whole + (tail + min(((q + 1) * kRows - 1) >> a.g_log2, nodes)) / kKeys + 1;
    }
    __device__ __forceinline__ int head_cost(const PagedArgs& a) const {
        int n = 0;
        for (int q = 0; q < nqt; q++) n += tiles(a, q) + kTileCost;
        return n;
    }
    __device__ __forceinline__ void next_unit(const PagedArgs& a) {
        tile = 0;
        if (++qt == nqt) {
            qt = 0;
            if (++head == a.Hkv) {
                head = 0;
                if (++s < a.nseq) load(a);
            }
        }
    }
};

// By one warp: the list's length and, then, the place x of it (of its first 32
// sequences a head's length is kept).
struct TileList {
    long long all;
    int own;
    __device__ __forceinline__ static int length(const PagedArgs& a, int s) {
        if (s >= a.nseq) return 0;
        TilePlace p{};
        p.s = s;
        p.load(a);
        return p.head_cost(a);
    }
    __device__ __forceinline__ TileList(const PagedArgs& a, int lane) {
        own = length(a, lane);
        long long n = own;
        for (int s = lane + 32; s < a.nseq; s += 32) n += length(a, s);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(kFull, n, o);
        all = n * a.Hkv;
    }
    __device__ __forceinline__ TilePlace find(const PagedArgs& a, long long x, int lane) const {
        long long done = 0;
        TilePlace r{};
        for (int s0 = 0; s0 < a.nseq; s0 += 32) {
            int cost = s0 == 0 ? own : length(a, s0 + lane);
            const long long n = static_cast<long long>(a.Hkv) * cost;
            long long upto = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long y = __shfl_up_sync(kFull, upto, o);
                if (lane >= o) upto += y;
            }
            const unsigned hit = __ballot_sync(kFull, x < done + upto);
            if (hit) {
                const int l = __ffs(hit) - 1;
                const long long rest = x - done - __shfl_sync(kFull, upto - n, l);
                cost = __shfl_sync(kFull, cost, l);
                r.s = s0 + l;
                r.load(a);
                r.head = place_div(rest, cost);
                r.tile = static_cast<int>(rest - static_cast<long long>(r.head) * cost);
                for (int t; r.tile >= (t = r.tiles(a, r.qt) + kTileCost); r.qt++) r.tile -= t;
                return r;
            }
            done += __shfl_sync(kFull, upto, 31);
        }
        r.s = a.nseq;
        return r;
    }
};

// A share's parts of units, one after the other.
struct Walk {
    TilePlace p;
    long long left;  // places of the share from p on
    int s, head, qt, t0, t1, tiles, whole, tail, nodes;  // the part at hand: tiles [t0, t1) of a unit of `tiles`
    __device__ __forceinline__ bool next(const PagedArgs& a) {
        while (left > 0 && p.s < a.nseq) {  // (s: in case the lengths change under the call)
            tiles = p.tiles(a, p.qt);
            t0 = p.tile;
            t1 = static_cast<int>(min(static_cast<long long>(tiles), t0 + left));
            s = p.s;
            head = p.head;
            qt = p.qt;
            whole = p.whole;
            tail = p.tail;
            nodes = p.nodes;
            left -= tiles + kTileCost - t0;
            p.next_unit(a);
            if (t0 < t1) return true;
        }
        return false;
    }
};

// ------------------------------------------------------------ the tiles

// Registers move between warpgroups, out of the 4 x 128 a thread that the
// e4m3 kernel is launched with (128 are too few for the softmax's 64 scores a
// thread).
constexpr int kRegsIssue = 96, kRegsSoft = 160, kRegsConvert = 96;
static_assert(kRegsIssue + 2 * kRegsSoft + kRegsConvert <= 4 * 128, "more than the launch has");
template <int kRegs>
__device__ __forceinline__ void reg_less() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs));
}
template <int kRegs>
__device__ __forceinline__ void reg_more() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs));
}

// D[tmem] (+)= A[tmem] * B[smem] at fixed offsets from the operands' bases, by
// one lane of a converged warp: operands that the whole warp agrees on stay in
// uniform registers, while a single thread's would be moved there one by one for
// every product (66 cycles each, as long as the product takes).  `lo`: address >>
// 4, and the leading offset of an MN-major operand.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);  // stride, version, 128-byte swizzle
template <int kAOff, int kBOff>
__device__ __forceinline__ void mma_at(uint32_t tmem_d, uint32_t tmem_a, uint32_t lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p, e;\n .reg .b32 x, y;\n .reg .b64 d;\n setp.ne.b32 p, %4, 0;\n add.u32 x, %1, %5;\n add.u32 y, %2, %6;\n"
        " mov.b64 d, {y, %7};\n elect.sync _|e, 0xffffffff;\n @e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], d, %3, p;\n}\n" ::"r"(tmem_d),
        "r"(tmem_a), "r"(lo), "r"(idesc), "r"(accumulate), "n"(kAOff), "n"(kBOff), "r"(kDescHigh)
        : "memory");
}
__device__ __forceinline__ void commit_elected(uint64_t* bar) {
    asm volatile(
        "{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n"
        " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(smem_u32(bar))
        : "memory");
}
// S = Q K^T (K-major K: 32 bytes a step, 64 elements a swizzle column) and
// O += P V (MN-major V: 16 keys of 128 bytes a step).
template <bool kFirst, int kk = 0>
__device__ __forceinline__ void mma_s(uint32_t d, uint32_t q, uint32_t k_lo, uint32_t idesc) {
    mma_at<kk * 8, ((kk >> 2) * kHalf + (kk & 3) * 32) / 16>(d, q, k_lo, idesc, kFirst && kk == 0 ? 0u : 1u);
    if constexpr (kk + 1 < kHeadDim / 16) mma_s<kFirst, kk + 1>(d, q, k_lo, idesc);
}
template <int kk = 0>
__device__ __forceinline__ void mma_pv(uint32_t d, uint32_t p, uint32_t v_lo, uint32_t idesc, uint32_t first) {
    mma_at<kk * 8, kk * 2048 / 16>(d, p, v_lo, idesc, kk > 0 ? 1u : 1u - first);
    if constexpr (kk + 1 < kKeys / 16) mma_pv<kk + 1>(d, p, v_lo, idesc, first);
}

template <Source kSource>
struct TGeo {
    static constexpr bool kConv = kSource == kCodes;
    // Three operand tiles of K and of V; converted ones two of each, and raw tiles of
    // half the size before them.
    static constexpr int kStages = kConv ? 2 : 3;
    static constexpr int kRawK = kConv ? 3 : 0, kRawV = kConv ? 2 : 0;
    static constexpr int kRing = 4;  // a tile's factors outlive its operands
    static constexpr int kOps = 2 * kStages * kTile;
    static constexpr int kRaw = (kRawK + kRawV) * kHalf;
    static constexpr int kRawScales = (kRawK + kRawV) * kKeys * 4;
    static constexpr int kBars = 4 * kStages + 2 * (kRawK + kRawV) + (kConv ? kRing : 0) + 9;
    static constexpr int kExchange = 4 * kRows * 4 + 16 * 4 + kRing * 8 + kRing * 4 * 4;
    static constexpr int kSmem = kOps + kRaw + kRawScales + kBars * 8 + kExchange + 16;
    // kCodes: warpgroups (producer, MMA, two idle warps), softmax, softmax, converters
    static constexpr int kThreads = kConv ? 512 : 64 + kSoft;
    static constexpr int kFirstSoft = kConv ? 4 : 2;
};

__device__ __forceinline__ uint32_t tile_swz(int row, int piece) { return static_cast<uint32_t>(row * 128 + ((piece ^ (row & 7)) << 4)); }

// 8 x 8 pieces of 16 bytes, a row per lane of 8: afterwards lane j has piece j of
// all 8 rows.
__device__ __forceinline__ void transpose8(uint4 (&y)[8], int lane) {
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {
        const bool up = lane & o;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (i & o) continue;
            uint4 &a = y[i], &b = y[i | o];  // (this lane keeps a if its bit is clear, else b)
            const uint4 give = up ? a : b;
            uint4 got;
            got.x = __shfl_xor_sync(kFull, give.x, o);
            got.y = __shfl_xor_sync(kFull, give.y, o);
            got.z = __shfl_xor_sync(kFull, give.z, o);
            got.w = __shfl_xor_sync(kFull, give.w, o);
            if (up)
                a = got;
            else
                b = got;
        }
    }
}

// A wait of a whole warp: where the phase has ended already, as it has most of the
// time, one poll and one vote.
__device__ __forceinline__ bool soon(uint64_t* bar, uint32_t parity, volatile int* abort) {
    return __all_sync(kFull, mbar_try_wait(bar, parity)) || warp_wait<1>(bar, parity, abort);
}

// Bits [o, o + 64) of a row of mask words (o >= -128; bits outside are 0).
__device__ __forceinline__ uint64_t mask_bits(const uint64_t* m, int mw, int o) {
    if (o <= -64) return 0ull;
    if (o < 0) return ld_plain(m) << -o;
    const int w = o >> 6, sh = o & 63;
    uint64_t r = w < mw ? ld_plain(m + w) >> sh : 0ull;
    if (sh && w + 1 < mw) r |= ld_plain(m + w + 1) << (64 - sh);
    return r;
}

template <Source kSource>
__global__ void __launch_bounds__(TGeo<kSource>::kThreads, 1)
    paged_tiles_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                       const __grid_constant__ CUtensorMap tmSk, const __grid_constant__ CUtensorMap tmSv,
                       const __grid_constant__ TileArgs ta) {
    using G_ = TGeo<kSource>;
    constexpr bool kConv = kSource == kCodes;  // converting warps
    constexpr bool kF16 = kSource != kPages;   // f16 operands, with a factor per row of Q and per tile of K and V
    constexpr int kStages = G_::kStages;
    const PagedArgs& a = ta.p;
    extern __shared__ __align__(1024) uint8_t tiles_smem[];
    uint8_t* sK = tiles_smem;
    uint8_t* sV = sK + kStages * kTile;
    uint8_t* rK = sV + kStages * kTile;  // raw tiles
    uint8_t* rV = rK + G_::kRawK * kHalf;
    float* raw_scales = reinterpret_cast<float*>(rV + G_::kRawV * kHalf);  // [raw K stages, raw V stages][key]
    uint64_t* k_full = reinterpret_cast<uint64_t*>(raw_scales + (G_::kRawK + G_::kRawV) * kKeys);
    uint64_t* k_empty = k_full + kStages;   // S of the tile done
    uint64_t* v_full = k_empty + kStages;
    uint64_t* v_empty = v_full + kStages;   // PV of the tile done
    uint64_t* rk_full = v_empty + kStages;
    uint64_t* rk_empty = rk_full + G_::kRawK;
    uint64_t* rv_full = rk_empty + G_::kRawK;
    uint64_t* rv_empty = rv_full + G_::kRawV;
    uint64_t* sc_full = rv_empty + G_::kRawV;
    uint64_t* s_full = sc_full + (kConv ? G_::kRing : 0);
    uint64_t* s_empty = s_full + 1;         // softmax has S in registers
    uint64_t* p_full = s_empty + 1;         // [2] by P buffer (P(n + 1) may be there before P(n) is waited for)
    uint64_t* pv_done = p_full + 2;         // [2] by P buffer
    uint64_t* q_ready = pv_done + 2;
    uint64_t* o_free = q_ready + 1;         // the unit's O has been read
    uint64_t* tdown = o_free + 1;
    float* xch = reinterpret_cast<float*>(k_full + G_::kBars);  // [2][warpgroup][128] row max / sum exchange
    int* xok = reinterpret_cast<int*>(xch + 4 * kRows);         // [2][warpgroup][4] "no wait failed"
    float2* tile_ref = reinterpret_cast<float2*>(xok + 16);      // [tile % 4] powers of two of K and V
    float* conv_top = reinterpret_cast<float*>(tile_ref + G_::kRing);  // [K, V][tile % 4][warp] largest scales
    int* misc = reinterpret_cast<int*>(conv_top + 4 * G_::kRing);      // TMEM base, abort
    volatile int* abort = &misc[1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_trigger();

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; i++) {
            mbar_init(&k_full[i], kConv ? 64 : 1);
            mbar_init(&k_empty[i], 1);
            mbar_init(&v_full[i], kConv ? 64 : 1);
            mbar_init(&v_empty[i], 1);
        }
        for (int i = 0; i < G_::kRawK; i++) {
            mbar_init(&rk_full[i], 1);
            mbar_init(&rk_empty[i], 64);
        }
        for (int i = 0; i < G_::kRawV; i++) {
            mbar_init(&rv_full[i], 1);
            mbar_init(&rv_empty[i], 64);
        }
        if (kConv)
            for (int i = 0; i < G_::kRing; i++) mbar_init(&sc_full[i], 2);
        mbar_init(s_full, 1);
        mbar_init(s_empty, kSoft / 32);
        for (int i = 0; i < 2; i++) {
            mbar_init(&p_full[i], kSoft / 32);
            mbar_init(&pv_done[i], 1);
        }
        mbar_init(q_ready, kSoft / 32);
        mbar_init(o_free, kSoft / 32);
        mbar_init(tdown, 1);
        misc[1] = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(reinterpret_cast<uint32_t*>(&misc[0]), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = static_cast<uint32_t>(misc[0]);
    // The preparation kernel lets this one start when all before it has ended:
    // lengths, page numbers and pages may be read at once, only what it writes
    // has to be waited for (pdl_wait below).
    Walk w{};
    {
        const TileList list(a, lane);
        const Shares shares(list.all, gridDim.x, kMinTiles);
        if (static_cast<int>(blockIdx.x) < shares.count) {
            w.left = shares.length(blockIdx.x);
            w.p = list.find(a, shares.begin(blockIdx.x), lane);
        }
        if (threadIdx.x == 0) {
            a.plan->places[blockIdx.x] = make_int4(w.p.s, w.p.head * 256 + w.p.qt, w.p.tile, w.left > 0 ? w.p.tiles(a, w.p.qt) : 0);
            a.plan->nodes[blockIdx.x] = w.p.nodes;
            if (blockIdx.x == 0) a.plan->count = shares.count;
        }
    }

    if (warp < G_::kFirstSoft) {
        if (kConv) reg_less<kRegsIssue>();
        if (warp == 0) {
            // ---------------------------------------------------------- loads: the whole warp, a lane per page
            const int per_tile = kKeys >> a.page_log2;  // pages of a tile
            const uint64_t policy = (a.B + 1) * a.G <= kRows ? l2_policy_evict_first() : l2_policy_evict_last();
            auto page_at = [&](int t) {
                return kSource != kWidened && t < w.whole && lane < per_tile
                           ? __ldcg(a.table + static_cast<long long>(w.s) * a.max_pages + static_cast<long long>(t) * per_tile + lane)
                           : 0;
            };
            int n = 0;       // bf16: tiles so far; e4m3: whole cache tiles so far
            bool have = w.next(a), ok = true, waited = kSource == kWidened, k_ahead = false;  // (k_ahead: tile n's K is on its way, its V is not)
            if (waited) pdl_wait();
            int t = w.t0, page = have ? page_at(t) : 0;
            while (have && ok) {
                // this tile, then the next one's page numbers, which are there when it is its turn
                const int head = w.head, s = w.s, tt = t, my_page = page;
                const bool cache_tile = kSource != kWidened && tt < w.whole;
                const int laid_row = kSource == kWidened ? ((s * a.Hkv + head) * ta.wide_tiles + tt) * kKeys : (s * a.Hkv + head) * ta.sk + (tt - w.whole) * kKeys;
                if (++t == w.t1) {
                    have = w.next(a);
                    t = w.t0;
                }
                if (have) page = page_at(t);
                if (kConv && !cache_tile) continue;  // (the converting warps read side tiles themselves)
                if (!cache_tile && !waited) {
                    pdl_wait();
                    waited = true;
                }
                long long row = a.pool_rows;  // past the pool: zeros
                if (cache_tile && lane < per_tile) {
                    if (my_page >= 0 && my_page < a.num_pages)
                        row = (static_cast<long long>(my_page) * a.Hkv + head) << a.page_log2;
                    else if (a.status)
                        atomicOr(a.status, kDevBounds);
                }
                for (int kv = 0; kv < 2 && ok; kv++) {
                    const int stages = kConv ? (kv ? G_::kRawV : G_::kRawK) : kStages;
                    const int st = n % stages;
                    uint64_t* full = (kConv ? (kv ? rv_full : rk_full) : (kv ? v_full : k_full)) + st;
                    uint64_t* empty = (kConv ? (kv ? rv_empty : rk_empty) : (kv ? v_empty : k_empty)) + st;
                    uint8_t* dst = kConv ? (kv ? rV : rK) + st * kHalf : (kv ? sV : sK) + st * kTile;
                    const CUtensorMap* tm = cache_tile ? (kv ? &tmV : &tmK) : (kv ? &tmSv : &tmSk);
                    ok = warp_wait<kWaitPolls>(empty, (static_cast<uint32_t>(n / stages) & 1u) ^ 1u, abort);
                    if (!ok) break;
                    k_ahead = kv == 0;
                    if (lane == 0)
                        mbar_arrive_expect_tx(full, kConv ? kHalf + kKeys * 4 : kTile);
                    __syncwarp();
                    if (!cache_tile) {
                        if (lane < 2)
                            tma_load_2d(dst + lane * kHalf, tm, full, 64 * lane, laid_row, policy);
                    } else if (lane < per_tile) {
                        const uint32_t at = static_cast<uint32_t>(lane << a.page_log2) * 128;
                        tma_load_2d(dst + at, tm, full, 0, static_cast<int>(row), policy);
                        if (!kConv) tma_load_2d(dst + kHalf + at, tm, full, 64, static_cast<int>(row), policy);
                        if (kConv) {
                            const long long sr = row < a.pool_rows ? row : 0;
                            bulk_load(raw_scales + (kv * G_::kRawK + st) * kKeys + (lane << a.page_log2), (kv ? a.vs : a.ks) + sr, 4u << a.page_log2, full);
                        }
                    }
                }
                if (ok) n++;
            }
            if (!ok && lane == 0) attn_timeout(a.status, abort);
            // The last copies land before the CTA ends, whoever gives up a wait, and when (in a
            // good run their readers have waited for them, and this costs nothing).
            for (int kv = 0; kv < 2; kv++) {
                const int stages = kConv ? (kv ? G_::kRawV : G_::kRawK) : kStages;
                uint64_t* full = kConv ? (kv ? rv_full : rk_full) : (kv ? v_full : k_full);
                const int fills = n + (kv == 0 && k_ahead ? 1 : 0);
                for (int i = max(fills - stages, 0); i < fills; i++)
                    if (lane == 0) attn_drain(&full[i % stages], static_cast<uint32_t>(i / stages) & 1u);
            }
        } else if (warp == 1) {
            // ---------------------------------------------------------- MMAs
            {
                // (operand types: bf16 1, f16 0 in bits 7 and 10)
                constexpr uint32_t idesc_s = idesc_bf16_f32(kRows, kKeys) & (kF16 ? ~((1u << 7) | (1u << 10)) : ~0u);
                constexpr uint32_t idesc_pv = (idesc_bf16_f32(kRows, kHeadDim) & (kF16 ? ~((1u << 7) | (1u << 10)) : ~0u)) | (1u << 16);  // B (= V) MN-major
                const uint32_t k_lo = smem_u32(sK) >> 4, v_lo = smem_u32(sV) >> 4, base = __shfl_sync(kFull, tmem, 0);
                auto issue_s = [&](int n) -> bool {
                    const int st = n % kStages;
                    if (!soon(&k_full[st], static_cast<uint32_t>(n / kStages) & 1u, abort) ||
                        (n > 0 && !soon(s_empty, static_cast<uint32_t>(n - 1) & 1u, abort)))
                        return false;
                    tc_fence_after();
                    const uint32_t k = __shfl_sync(kFull, (k_lo + st * (kTile >> 4)) & 0x3FFFu, 0);
                    mma_s<true>(base + kSCol, base + kQCol, k, idesc_s);
                    if (!kF16) mma_s<false>(base + kSCol, base + kQLoCol, k, idesc_s);
                    commit_elected(s_full);
                    commit_elected(&k_empty[st]);
                    return true;
                };
                bool have = w.next(a), ok = true;
                int n = 0, part = 0, t = w.t0;
                if (have) ok = soon(q_ready, 0, abort) && issue_s(0);
                while (have && ok) {
                    // tile t of part `part`; S of the part's next tile first
                    const bool first = t == w.t0, last = t + 1 == w.t1;
                    if (!last) ok = issue_s(n + 1);
                    const int st = n % kStages;
                    ok = ok && soon(&p_full[n & 1], static_cast<uint32_t>(n >> 1) & 1u, abort) &&
                         soon(&v_full[st], static_cast<uint32_t>(n / kStages) & 1u, abort) &&
                         (!first || part == 0 || soon(o_free, static_cast<uint32_t>(part - 1) & 1u, abort));
                    if (!ok) break;
                    tc_fence_after();
                    mma_pv(base + kOCol, base + kPCol + __shfl_sync(kFull, n & 1, 0) * 64,
                           __shfl_sync(kFull, ((v_lo + st * (kTile >> 4)) & 0x3FFFu) | ((kHalf >> 4) << 16), 0), idesc_pv, __shfl_sync(kFull, first ? 1u : 0u, 0));
                    commit_elected(&v_empty[st]);
                    commit_elected(&pv_done[n & 1]);
                    t++;
                    if (last) {
                        have = w.next(a);
                        t = w.t0;
                        part++;
                        if (have) ok = soon(q_ready, static_cast<uint32_t>(part) & 1u, abort) && issue_s(n + 1);
                    }
                    n++;
                }
                if (!ok) {
                    if (lane == 0) attn_timeout(a.status, abort);
                    __syncwarp();
                    commit_elected(tdown);
                    attn_drain(tdown, 0);
                }
            }
        }
    } else if (warp < G_::kFirstSoft + 8) {
        // ---------------------------------------------------------- softmax
        if (kConv) reg_more<kRegsSoft>();
        const int qd = warp & 3, wg = (warp - G_::kFirstSoft) >> 2, cb = wg * 64;
        const int r = qd * 32 + lane;  // query row of the unit = TMEM lane
        const int pair_bar = kPairBar + qd;
        const uint32_t tl = tmem + (static_cast<uint32_t>(qd * 32) << 16);
        auto arrive = [&](uint64_t* bar) {  // of the whole warp
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
        };
        // The maximum or sum of a row and "no wait failed" of the lane quarter's two warps:
        // two places in turn, so that one barrier an exchange is enough.
        int turn = 0;
        auto exchange = [&](float x, bool& ok) {
            float* xc = xch + turn * 2 * kRows;
            int* xo = xok + turn * 8;
            turn ^= 1;
            xc[wg * kRows + r] = x;
            if (lane == 0) xo[wg * 4 + qd] = ok ? 1 : 0;
            named_bar_sync(pair_bar, 64);
            ok = ok && xo[(1 - wg) * 4 + qd] != 0;
            return xc[(1 - wg) * kRows + r];
        };
        // this thread's half of its row's query into tensor memory
        auto load_q = [&]() {
            const bool in = w.qt * kRows + r < (w.nodes + 1) << a.g_log2;
            const long long at = ((static_cast<long long>(w.s) * a.Hkv + w.head) * ta.nqt + w.qt) * (16 * kRows) + 8 * wg * kRows + r;
            uint32_t q[kF16 ? 1 : 2][32];
#pragma unroll
            for (int i = 0; i < (kF16 ? 1 : 2); i++)
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const uint4 y = in ? __ldcg((i ? ta.q_lo : ta.qr) + at + e * kRows) : make_uint4(0u, 0u, 0u, 0u);
                    q[i][4 * e] = y.x;
                    q[i][4 * e + 1] = y.y;
                    q[i][4 * e + 2] = y.z;
                    q[i][4 * e + 3] = y.w;
                }
            tmem_st32(tl + kQCol + wg * 32, q[0]);
            if (!kF16) tmem_st32(tl + kQLoCol + wg * 32, q[kF16 ? 0 : 1]);
            tmem_wait_st();
            arrive(q_ready);
        };
        bool have = w.next(a), ok = true;
        pdl_wait();
        if (have) load_q();
        int n = 0;
        while (have) {
            const int s = w.s, head = w.head, t0 = w.t0, t1 = w.t1, whole = w.whole, tail = w.tail, nodes = w.nodes;
            const bool full_unit = t0 == 0 && t1 == w.tiles;
            const int row = w.qt * kRows + r, b = row >> a.g_log2;
            const bool row_ok = b <= nodes;
            // m_run: the row's reference.  f16: O is in units of vref, the largest of the
            // tiles' powers of two so far; P has a factor 2^7 (at most 2^15), so that 2^-31
            // of the largest weight still counts, and its tile's power of two over vref
            constexpr float kBoost = kF16 ? 7.0f : 0.0f;
            float m_run = -INFINITY, l = 0.0f, vref = 0.0f;
            float rs = a.sl2;  // scores in log2 units = products * rs (f16: * the tile's power of two of K)
            if (kF16 && row_ok) rs = __ldcg(ta.q_scale + ((static_cast<long long>(s) * a.Hkv + head) * ta.nqt + w.qt) * kRows + r);
            float2 ref_ahead = make_float2(1.0f, 1.0f);  // (kWidened: read a tile ahead)
            const float2* refs = ta.wide_refs + (static_cast<long long>(s) * a.Hkv + head) * ta.wide_tiles;
            if (kSource == kWidened) ref_ahead = __ldcg(refs + t0);
            for (int t = t0; t < t1; t++, n++) {
                // visible keys of this row among this warpgroup's 64 of the tile
                // (of a whole cache tile all, in a row of no node too: it is not written)
                uint64_t vis = ~0ull;
                bool all_seen = true;
                if (t >= whole) {
                    const int o = (t - whole) * kKeys + cb - tail - 1;  // tree node of the first key (negative: cache, row 0)
                    vis = 0ull;
                    if (b > 0 && row_ok && o < b) {  // (bits beyond the row's own are not used)
                        vis = mask_bits(a.mask + (static_cast<long long>(s) * a.B + b - 1) * a.mw, a.mw, o);
                        if (b - o < 64) vis &= (1ull << (b - o)) - 1ull;
                    }
                    if (o < 0) vis |= o <= -64 ? ~0ull : (1ull << -o) - 1ull;
                    all_seen = __all_sync(kFull, vis == ~0ull);
                }
                // Both warps of the lane quarter reach the exchange of every iteration and
                // leave the loop at the same point: a failed wait is exchanged with the row
                // max and acted on after it.
                if (kConv && ok && !soon(&sc_full[n % G_::kRing], static_cast<uint32_t>(n / G_::kRing) & 1u, abort)) ok = false;
                if (ok && !soon(s_full, static_cast<uint32_t>(n) & 1u, abort)) ok = false;
                if (!ok) attn_timeout(a.status, abort);
                float sv[64];
                float mx = -INFINITY, rt = rs, vtile = 0.0f;
                if (ok) {
                    if (kF16) {  // (before s_empty: after S(n + 1) the place may be written again)
                        const float2 ref = kConv ? tile_ref[n % G_::kRing] : ref_ahead;
                        // not 0, where both factors are tiny (rows of zeros): hidden keys are -inf by now
                        rt = fmaxf(rt * ref.x, FLT_MIN);
                        vtile = ref.y;
                        if (kSource == kWidened && t + 1 < t1) ref_ahead = __ldcg(refs + t + 1);
                    }
                    tc_fence_after();
                    tmem_ld64(tl + kSCol + cb, sv);
                    arrive(s_empty);
                    if (!all_seen) {
#pragma unroll
                        for (int c = 0; c < 64; c++)
                            if (!((vis >> c) & 1ull)) sv[c] = -INFINITY;
                    }
                    // (four chains: one alone would be a third of the tile's time in latencies)
                    float m4[4] = {sv[0], sv[1], sv[2], sv[3]};
#pragma unroll
                    for (int c = 4; c < 60; c += 8)
#pragma unroll
                        for (int e = 0; e < 4; e++) m4[e] = max3(m4[e], sv[c + e], sv[c + 4 + e]);
                    mx = max3(max3(m4[0], m4[1], sv[60]), max3(m4[2], m4[3], sv[61]), fmaxf(sv[62], sv[63]));
                }
                mx = fmaxf(mx, exchange(mx, ok));
                if (!ok) break;
                const float mx2 = mx * rt;
                const bool higher = mx2 > m_run + kSlack8;
                const bool resc = higher || (kF16 && vtile > vref);  // (vref: the same in every thread)
                const float m_new = higher ? mx2 : m_run;
                const float alpha = higher ? ex2(m_run - m_new) : 1.0f;
                float alpha_o = alpha, down = 1.0f;  // (down: P's part for the tile's power of two; 2^-60 is as good as nothing)
                if (kF16) {
                    const float vnew = fmaxf(vref, vtile);
                    const float inv = __uint_as_float(0x7F000000u - __float_as_uint(vnew));  // (powers of two: exact)
                    alpha_o *= vref * inv;
                    down = fmaxf(vtile * inv, 8.6736173798840355e-19f);
                    vref = vnew;
                }
                // P buffer n & 1 was last read by PV(n - 2), which was issued before S(n) and so
                // ended before s_full's arrival; O must be stable (PV(n - 1) done) only when
                // it is rescaled.  On a timeout this tile is skipped; the pair leaves the loop
                // together at the next exchange.
                if (t > t0 && __any_sync(kFull, resc)) {
                    if (!soon(&pv_done[(n - 1) & 1], static_cast<uint32_t>((n - 1) >> 1) & 1u, abort)) {
                        attn_timeout(a.status, abort);
                        ok = false;
                        continue;
                    }
                    tc_fence_after();
#pragma unroll
                    for (int c0 = 0; c0 < 64; c0 += 16) {
                        float o[16];
                        tmem_ld16(tl + kOCol + cb + c0, o);
#pragma unroll
                        for (int e = 0; e < 16; e++) o[e] *= alpha_o;
                        tmem_st16(tl + kOCol + cb + c0, o);
                    }
                    tmem_wait_st();
                }
                l *= alpha;
                m_run = m_new;
                // P = 2^(s - m) as pairs of V's operand type (bf16 or f16, which a product's
                // operands share; the sum has the unrounded weights); hidden keys hold -inf and give 0 (so does
                // every key of a row that has seen no visible key: m = -inf)
                const float nm = m_run == -INFINITY ? 0.0f : kBoost - m_run + (kF16 ? log2_of(down) : 0.0f);
                float2 sum0 = make_float2(0.0f, 0.0f), sum1 = sum0;
                uint32_t pk[32];
#pragma unroll
                for (int c = 0; c < 64; c += 4) {
                    float2 x = fma2(make_float2(sv[c], sv[c + 1]), make_float2(rt, rt), make_float2(nm, nm));
                    float2 z = fma2(make_float2(sv[c + 2], sv[c + 3]), make_float2(rt, rt), make_float2(nm, nm));
                    x = make_float2(ex2(x.x), ex2(x.y));
                    z = make_float2(ex2(z.x), ex2(z.y));
                    sum0 = add2(sum0, x);
                    sum1 = add2(sum1, z);
                    pk[c >> 1] = kF16 ? pack_f16x2(x.x, x.y) : pack_bf16x2(x.x, x.y);
                    pk[(c >> 1) + 1] = kF16 ? pack_f16x2(z.x, z.y) : pack_bf16x2(z.x, z.y);
                }
                sum0 = add2(sum0, sum1);
                const float lsum = sum0.x + sum0.y;
                tmem_st32(tl + kPCol + (n & 1) * 64 + wg * 32, pk);
                tmem_wait_st();
                l += kF16 ? lsum * __uint_as_float(0x7F000000u - __float_as_uint(down)) : lsum;  // (1 / down)
                arrive(&p_full[n & 1]);
                if (t + 1 == t1) {
                    // the next part's queries, while the last PV runs: all products with this
                    // part's have been seen
                    have = w.next(a);
                    if (have) load_q();
                }
            }
            // the pair leaves together: an `ok` lost after the last exchange is exchanged here
            if (ok && !soon(&pv_done[(n - 1) & 1], static_cast<uint32_t>((n - 1) >> 1) & 1u, abort)) {
                attn_timeout(a.status, abort);
                ok = false;
            }
            l += exchange(l, ok);
            if (!ok) break;
            tc_fence_after();
            float o[64];
            tmem_ld64(tl + kOCol + cb, o);
            arrive(o_free);
            if (full_unit) {
                // rows in whole lines: 8 lanes exchange their rows' 8 pieces
                const float inv = l > 0.0f ? (kF16 ? vref : 1.0f) / l : 0.0f;
                uint4 y[8];
#pragma unroll
                for (int e = 0; e < 8; e++)
                    y[e] = make_uint4(pack_bf16x2(o[8 * e] * inv, o[8 * e + 1] * inv), pack_bf16x2(o[8 * e + 2] * inv, o[8 * e + 3] * inv),
                                      pack_bf16x2(o[8 * e + 4] * inv, o[8 * e + 5] * inv), pack_bf16x2(o[8 * e + 6] * inv, o[8 * e + 7] * inv));
                transpose8(y, lane);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const int their = row - (lane & 7) + e, tb = their >> a.g_log2;  // row of lane 8 (lane / 8) + e
                    if (tb <= nodes)
                        reinterpret_cast<uint4*>(a.out + ((static_cast<long long>(s) * (a.B + 1) + tb) * a.Hq + head * a.G + (their & (a.G - 1))) * kHeadDim + cb)[lane & 7] = y[e];
                }
            } else if (row_ok) {
                TilePart* d = reinterpret_cast<TilePart*>(a.parts) + 2 * blockIdx.x + (t0 > 0 ? 0 : 1);
#pragma unroll
                for (int e = 0; e < 16; e++) {
                    const float by = kF16 ? vref : 1.0f;
                    d->o[wg * 16 + e][r] = make_float4(o[4 * e] * by, o[4 * e + 1] * by, o[4 * e + 2] * by, o[4 * e + 3] * by);
                }
                if (wg == 0) d->ml[r] = make_float2(m_run, l);
            }
        }
    } else if constexpr (kConv) {
        // ---------------------------------------------------------- raw tiles to operands (e4m3): a thread per key
        reg_less<kRegsConvert>();
        // Two warps for K, two for V, on their own; a thread takes keys `key` and key + 64.
        const int cw = warp - (G_::kFirstSoft + 8), kv = cw >> 1, key = (cw & 1) * 32 + lane;
        uint64_t* raw_full = kv ? rv_full : rk_full;
        uint64_t* raw_empty = kv ? rv_empty : rk_empty;
        uint64_t* op_full = kv ? v_full : k_full;
        uint64_t* op_empty = kv ? v_empty : k_empty;
        const uint8_t* raw_tile = kv ? rV : rK;
        uint8_t* op_tile = kv ? sV : sK;
        const int raw_stages = kv ? G_::kRawV : G_::kRawK;
        const float* side_scale = kv ? ta.side_vs : ta.side_ks;
        const uint4* side_rows = kv ? ta.side_v : ta.side_k;
        float* pair_top = conv_top + kv * 2 * G_::kRing;
        bool ok = true, stop = false, waited = false;
        int n = 0, raw = 0;  // tiles, whole cache tiles so far
        // The two warps meet at a barrier in every tile, so they leave together: one whose
        // wait failed says so at the next tile's.
        while (!stop && w.next(a)) {
            for (int t = w.t0; t < w.t1; t++, n++) {
                const bool cache_tile = t < w.whole;
                if (!cache_tile && !waited) {
                    pdl_wait();
                    waited = true;
                }
                const int st = n % kStages, rs = raw % raw_stages;
                const long long side = (static_cast<long long>(w.s) * a.Hkv + w.head) * ta.sk + (t - w.whole) * kKeys + key;
                if (ok && cache_tile && !soon(&raw_full[rs], static_cast<uint32_t>(raw / raw_stages) & 1u, abort)) ok = false;
                float sc[2];
#pragma unroll
                for (int h = 0; h < 2; h++)
                    sc[h] = cache_tile ? raw_scales[(kv * G_::kRawK + rs) * kKeys + key + 64 * h] : __ldcg(side_scale + side + 64 * h);
                const float mine = fmaxf(fmaxf(sc[0], sc[1]), 0.0f);
                float top = __uint_as_float(__reduce_max_sync(kFull, __float_as_uint(mine)));
                if (lane == 0) pair_top[(n % G_::kRing) * 2 + (cw & 1)] = ok ? top : -1.0f;
                named_bar_sync(kConvBar + kv, 64);
                const float2 both = *reinterpret_cast<const float2*>(pair_top + (n % G_::kRing) * 2);
                if (fminf(both.x, both.y) < 0.0f) {
                    ok = false;
                    stop = true;
                    break;
                }
                const float ref = above(fmaxf(both.x, both.y));
                if (key == 0) {
                    (kv ? tile_ref[n % G_::kRing].y : tile_ref[n % G_::kRing].x) = ref;
                    mbar_arrive(&sc_full[n % G_::kRing]);
                }
                if (!soon(&op_empty[st], (static_cast<uint32_t>(n / kStages) & 1u) ^ 1u, abort)) {
                    ok = false;
                    if (cache_tile) raw++;
                    continue;
                }
                const float inv = __uint_as_float(0x7F000000u - __float_as_uint(ref));  // 1 / ref
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    // the key's scale over the common power of two, at most 1, rounded to f16: that
                    // moves the key's scores or its values by 2^-12 of themselves at most, as
                    // much as the rounding of an operand does
                    const __half2 by = __float2half2_rn(sc[h] * inv);
                    auto times = [&](uint32_t x) {
                        const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&x), by);
                        return *reinterpret_cast<const uint32_t*>(&r);
                    };
                    const int row = key + 64 * h;
                    uint8_t* dst = op_tile + st * kTile;
                    uint4 x[8];
                    if (cache_tile) {
                        const uint8_t* src = raw_tile + rs * kHalf;
#pragma unroll
                        for (int c = 0; c < 8; c++) x[c] = *reinterpret_cast<const uint4*>(src + tile_swz(row, c));
#pragma unroll
                        for (int c = 0; c < 8; c++) {
                            uint8_t* d = dst + (c >> 2) * kHalf;
                            *reinterpret_cast<uint4*>(d + tile_swz(row, (2 * c) & 7)) =
                                make_uint4(times(codes_to_f16(x[c].x)), times(codes_to_f16(x[c].x >> 16)), times(codes_to_f16(x[c].y)), times(codes_to_f16(x[c].y >> 16)));
                            *reinterpret_cast<uint4*>(d + tile_swz(row, (2 * c + 1) & 7)) =
                                make_uint4(times(codes_to_f16(x[c].z)), times(codes_to_f16(x[c].z >> 16)), times(codes_to_f16(x[c].w)), times(codes_to_f16(x[c].w >> 16)));
                        }
                    } else {
                        const uint4* src = side_rows + (side >> 7) * (16 * kKeys) + row;
#pragma unroll
                        for (int q = 0; q < 2; q++) {
#pragma unroll
                            for (int c = 0; c < 8; c++) x[c] = __ldcg(src + (8 * q + c) * kKeys);
#pragma unroll
                            for (int c = 0; c < 8; c++)
                                *reinterpret_cast<uint4*>(dst + q * kHalf + tile_swz(row, c)) = make_uint4(times(x[c].x), times(x[c].y), times(x[c].z), times(x[c].w));
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the MMAs read it
                mbar_arrive(&op_full[st]);
                if (cache_tile) {
                    // Only now, when what was read from it is in use: an arrival right after the
                    // loads let the slot be refilled before they had returned.
                    mbar_arrive(&raw_empty[rs]);
                    raw++;
                }
            }
        }
        if (!ok) attn_timeout(a.status, abort);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// Joins the parts of the units that several CTAs shared, in the order of
// their keys.  Blocks 8 (i - 1) .. + 7 work if share i begins inside a unit that
// share i - 1 began: 16 rows each, 16 threads (8 elements each) a row.
__global__ void __launch_bounds__(256) paged_tiles_join_kernel(const __grid_constant__ PagedArgs a) {
    pdl_trigger();
    const int tid = threadIdx.x, lane = tid & 31, i = blockIdx.x / 8 + 1, eighth = blockIdx.x % 8;
    pdl_wait();
    // all that has to be known in one go (the kernel is a chain of loads)
    const int count = a.plan->count, nodes = a.plan->nodes[i];
    const int4 at = a.plan->places[i], prev = a.plan->places[i - 1];
    const int4 next = a.plan->places[min(i + 1 + lane, kMaxSms - 1)];
    if (i >= count || at.z == 0 || at.z >= at.w) return;  // (from at.w on the place stands for a unit's other costs)
    if (prev.x == at.x && prev.y == at.y && prev.z > 0) return;
    const int s = at.x, head = at.y / 256, qt = at.y % 256;
    const int r = eighth * 16 + (tid & 15), d8 = tid >> 4, row = qt * kRows + r, b = row >> a.g_log2;
    const int c0 = i - 1;
    int c1 = i;  // the last share that holds tiles of the unit
    {
        const unsigned out = __ballot_sync(kFull, !(i + 1 + lane < count && next.x == at.x && next.y == at.y && next.z < at.w));
        if (out) {
            c1 += __ffs(out) - 1;
        } else {
            c1 += 32;
            for (; c1 + 1 < count; c1++) {
                const int4 x = a.plan->places[c1 + 1];
                if (x.x != at.x || x.y != at.y || x.z >= at.w) break;
            }
        }
    }
    if (b > nodes) return;
    float top = -INFINITY, l = 0.0f, o[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int c = c0; c <= c1; c++) {
        const TilePart* x = static_cast<const TilePart*>(a.parts) + 2 * c + (c < i ? 1 : 0);
        const float2 ml = x->ml[r];
        const float4 y = x->o[2 * d8][r], z = x->o[2 * d8 + 1][r];
        const bool any = ml.x != -INFINITY;
        const float up = fmaxf(top, ml.x), old = top == -INFINITY ? 0.0f : ex2(top - up), by = any ? ex2(ml.x - up) : 0.0f;
        top = up;
        l = l * old + (any ? ml.y * by : 0.0f);
        const float v[8] = {y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
#pragma unroll
        for (int k = 0; k < 8; k++) o[k] = o[k] * old + (any ? v[k] * by : 0.0f);
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    __nv_bfloat16* d = a.out + ((static_cast<long long>(s) * (a.B + 1) + b) * a.Hq + head * a.G + (row & (a.G - 1))) * kHeadDim + 8 * d8;
    *reinterpret_cast<uint4*>(d) = make_uint4(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv),
                                              pack_bf16x2(o[4] * inv, o[5] * inv), pack_bf16x2(o[6] * inv, o[7] * inv));
}

// e4m3 pages are widened first where a kv head has at least this many query
// tiles, each of which would convert all keys again (a tile of a unit takes 1.05
// us from f16 tiles and 1.9 converted), and where the f16 tiles of the longest
// sequences take at most 4 GB.  Eight trees over 4096 keys, widened / converted:
// 4 query tiles 96 / 97 us, 5 113 / 120, 8 150 / 184; one over 2048, 3 tiles 28.4 /
// 23.8; one over 16384, 4 tiles 73 / 70.
constexpr int kWidenTiles = 4;
constexpr size_t kWidenBytes = static_cast<size_t>(4) << 30;

// Workspace: partial results, queries, side rows, their factors, f16 tiles.
struct TileWs {
    int sk, nqt, wide_tiles;
    size_t q, q_lo, k, v, qs, ks, vs, wk, wv, refs, total;
};
TileWs tile_ws(int nseq, int B, int Hq, const dart_kv_cache& cache, int max_pages) {
    TileWs w{};
    const int Hkv = cache.Hkv;
    w.sk = (kKeys - 1 + B + 1 + kKeys - 1) / kKeys * kKeys;
    w.nqt = ((B + 1) * (Hq / Hkv) + kRows - 1) / kRows;
    const size_t heads = static_cast<size_t>(nseq) * Hkv, q_rows = heads * w.nqt * kRows;
    auto up = [](size_t n) { return (n + 255) & ~static_cast<size_t>(255); };
    w.q = up(sizeof(SharePlan) + sizeof(TilePart) * 2 * kMaxSms);
    w.q_lo = w.q + up(q_rows * kHeadDim * 2);
    w.k = w.q_lo + (cache.dtype == DART_KV_BF16 ? up(q_rows * kHeadDim * 2) : 0);
    w.v = w.k + up(heads * w.sk * kHeadDim * 2);
    w.qs = w.v + up(heads * w.sk * kHeadDim * 2);
    w.ks = w.qs + up(q_rows * 4);
    w.vs = w.ks + up(heads * w.sk * 4);
    w.wk = w.vs + up(heads * w.sk * 4);
    const long long tiles = static_cast<long long>(max_pages) * cache.page_size / kKeys + w.sk / kKeys;
    const size_t each = heads * tiles * kTile;
    if (cache.dtype == DART_KV_E4M3 && w.nqt >= kWidenTiles && each <= kWidenBytes / 2 && tiles <= 65535) w.wide_tiles = static_cast<int>(tiles);
    const size_t wide = w.wide_tiles ? each : 0;
    w.wv = w.wk + wide;
    w.refs = w.wv + wide;
    w.total = w.refs + up(heads * w.wide_tiles * 8);
    return w;
}

}  // namespace

size_t paged_tiles_workspace(const dart_paged_attn_config& c, const dart_kv_cache& cache) {
    return tile_ws(c.nseq, c.B, c.Hq, cache, c.max_pages).total;
}

template <Source kSource>
static bool allow_smem() {
    return cudaFuncSetAttribute(paged_tiles_kernel<kSource>, cudaFuncAttributeMaxDynamicSharedMemorySize, TGeo<kSource>::kSmem) == cudaSuccess;
}
bool paged_tiles_prepare_device() { return allow_smem<kPages>() && allow_smem<kCodes>() && allow_smem<kWidened>(); }

template <Source kSource>
static cudaError_t launch_tiles(int sms, cudaStream_t st, const CUtensorMap& k, const CUtensorMap& v, const CUtensorMap& side_k,
                                const CUtensorMap& side_v, const TileArgs& ta) {
    return launch_pdl(paged_tiles_kernel<kSource>, dim3(sms), dim3(TGeo<kSource>::kThreads), TGeo<kSource>::kSmem, st, k, v, side_k, side_v, ta);
}

int launch_paged_tiles(PagedArgs a, const dart_kv_cache& cache, uint8_t* workspace, int sms, cudaStream_t st) {
    const bool fp8 = cache.dtype == DART_KV_E4M3;
    const TileWs w = tile_ws(a.nseq, a.B, a.Hq, cache, a.max_pages);
    const bool wide = w.wide_tiles > 0;
    TileArgs ta{};
    ta.p = a;
    ta.sk = w.sk;
    ta.nqt = w.nqt;
    ta.qr = reinterpret_cast<uint4*>(workspace + w.q);
    ta.q_lo = reinterpret_cast<uint4*>(workspace + w.q_lo);
    ta.side_k = reinterpret_cast<uint4*>(workspace + w.k);
    ta.side_v = reinterpret_cast<uint4*>(workspace + w.v);
    ta.q_scale = reinterpret_cast<float*>(workspace + w.qs);
    ta.side_ks = reinterpret_cast<float*>(workspace + w.ks);
    ta.side_vs = reinterpret_cast<float*>(workspace + w.vs);
    ta.wide_tiles = w.wide_tiles;
    ta.wide_k = reinterpret_cast<uint4*>(workspace + w.wk);
    ta.wide_v = reinterpret_cast<uint4*>(workspace + w.wv);
    ta.wide_refs = reinterpret_cast<float2*>(workspace + w.refs);
    const long long heads = static_cast<long long>(a.nseq) * a.Hkv, side_rows = heads * w.sk;
    CUtensorMap tmK, tmV, tmSk, tmSv;
    // f16 tiles are 16-bit rows to the copies, as bf16 rows are
    const bool maps = wide ? encode_rows(&tmK, ta.wide_k, heads * w.wide_tiles * kKeys, false, kKeys) && encode_rows(&tmV, ta.wide_v, heads * w.wide_tiles * kKeys, false, kKeys)
                           : encode_rows(&tmK, cache.k, a.pool_rows, fp8, cache.page_size) && encode_rows(&tmV, cache.v, a.pool_rows, fp8, cache.page_size) &&
                                 encode_rows(&tmSk, ta.side_k, side_rows, false, kKeys) && encode_rows(&tmSv, ta.side_v, side_rows, false, kKeys);
    if (!maps) return DART_ERR_CUDA;
    if (wide) {
        tmSk = tmK;  // (side tiles lie among the others)
        tmSv = tmV;
    }
    // tree rows, up to 127 cache tokens before them, up to 127 rows of zeros after them
    const dim3 prep(static_cast<unsigned>(a.nseq), static_cast<unsigned>(a.B + 1 + 2 * (kKeys - 1)));
    const uint8_t *pk = static_cast<const uint8_t*>(cache.k), *pv = static_cast<const uint8_t*>(cache.v);
    cudaError_t e = fp8 ? launch_pdl(paged_prep_kernel<true>, prep, dim3(kPrepThreads), 0, st, ta, pk, pv)
                        : launch_pdl(paged_prep_kernel<false>, prep, dim3(kPrepThreads), 0, st, ta, pk, pv);
    if (e == cudaSuccess && wide)
        e = launch_pdl(paged_widen_kernel, dim3(static_cast<unsigned>(heads), static_cast<unsigned>(w.wide_tiles)), dim3(256), 0, st, ta, pk, pv);
    if (e == cudaSuccess)
        e = wide ? launch_tiles<kWidened>(sms, st, tmK, tmV, tmSk, tmSv, ta)
                 : fp8 ? launch_tiles<kCodes>(sms, st, tmK, tmV, tmSk, tmSv, ta) : launch_tiles<kPages>(sms, st, tmK, tmV, tmSk, tmSv, ta);
    if (e == cudaSuccess) e = launch_pdl(paged_tiles_join_kernel, dim3(8 * (sms - 1)), dim3(256), 0, st, a);
    return e == cudaSuccess ? DART_OK : DART_ERR_CUDA;
}

}  // namespace dart

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
//   paged_widen_kernel  e4m3 or e2m1 pages that several query tiles read: as f16 tiles.
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
// 64), the two warps of a lane quarter exchange maxima and sums).  With e4m3 or e2m1
// pages all operands are f16: four more warps turn raw tiles into f16, each
// key's codes times its scale over a power of two that the tile (K) or the
// unit so far (V) has in common; queries and side rows are f16 with a power
// of two per row.  So nothing can overflow, and the softmax has one factor a
// tile to apply instead of one a key (64 broadcast reads of a key's scale from
// shared memory, twice, took 0.5 us of a tile's 1.6).  TMEM (512 columns): S
// [0,256) in two buffers, each of which P takes over (S(n + 1) is there when the softmax
// comes to it), O [256,384), Q [384,448), and with bf16 pages what the queries' first
// bf16 term leaves, [448,512).
// A row's running maximum is raised (and O rescaled) only when a tile exceeds
// it by more than 2^8.  Every wait is bounded.
//
// Measured: a tile takes 1.07 us from bf16 pages (24 MMAs of 66 cycles are 0.8), 1.05 from
// widened ones (16 MMAs, 0.53), 1.4 from e2m1 pages that the CTA converts; eight trees of 512
// nodes over up to 4096 keys take 234 and 243 (e4m3 248) us with everything around.  With the first
// term of the queries alone bf16 pages took 0.90 and 211 us, at an error against 64 bits of
// 0.0029 of the output instead of 0.0023 (its own rounding is 0.0017).  What a tile takes
// beside its MMAs is the chain of the softmax: about 580 cycles from one tile's P to the next
// one's scores, 670 to the row's maximum, 830 to P, most of them latencies of operations
// that share a queue (TMEM loads and stores, barriers, exchanges).  Registers and
// instructions count: what is spilled goes to L2, since shared memory leaves the L1 cache no
// room (a part's numbers are in shared memory for that; without, 480 bytes of spills, one tree of
// 17 rows over 131072 e2m1 keys 126 us instead of 91; the next part's queries fetched a tile
// early, at 312 bytes, 370 us for the eight trees), and four kinds of warps share the
// instruction cache (the two keys of a converting thread unrolled, 64 trees of 32 rows over
// up to 4096 e2m1 keys 176 us instead of 140; eight converting warps, and so 96 registers, 148).
// Tried: four softmax warpgroups of 32 columns (287 us where two took 235: the
// fixed part of the instructions doubles); CTA pairs with half of K and V each (383: one more
// hop in every exchange); two streams of tiles, of four warps with 128 columns a thread or of eight
// warps with 64, scores read twice (307 both, where one stream took 270: S(n + 2) waits for
// PV(n)); weights formed before the maximum is known (274).
// Where they take 255: PV(n) and S(n + 2) issued in one go (257) and the next tile's scores
// loaded while P is stored (280: tensor memory serves the products meanwhile).
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

// Where K and V tiles come from: bf16 pages; e4m3 or e2m1 pages, converted in the
// CTA; pages of either that paged_widen_kernel has laid out as f16 tiles before.
enum Source { kPages, kCodes, kCodes4, kWidened };
constexpr int kRows = 128;               // query rows per unit (MMA M)
constexpr int kKeys = 128;               // keys per tile
constexpr int kHalf = kKeys * 128;       // 128 rows of one 128-byte swizzle column
constexpr int kTile = 2 * kHalf;         // 128 keys of bf16
constexpr int kSoft = 256;               // softmax threads
constexpr int kPairBar = 2;              // named barriers 2 .. 5
constexpr float kSlack8 = 8.0f;          // log2 units: P <= 2^8 between rescales
// What a unit costs beside its tiles (its queries, its result, the pause between
// its last tile and the next unit's first), in tiles: eight trees of 512 nodes over
// 4096 bf16 keys 241 us with 3 and 4, 245 with 6; e4m3 273, 270, 274; e2m1 262, 255, 258.
// Where a tile takes longer, because the CTA converts it, one less: 64 trees of 32
// rows over up to 4096 e2m1 keys 143 us with 3, 144 with 4.
constexpr int kTileCost = 4, kTileCostConverted = 3;
constexpr int kMinTiles = 2;             // of a share (one tree of 20 nodes over 500 keys: 1 18.5 us, 2 17.9, 4 19.8)
constexpr uint32_t kSCol = 0, kOCol = 256, kQCol = 384, kQLoCol = 448;  // S: two of 128 columns

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

// The first blocks of a sequence take kTree tree rows each: their keys and values (side
// rows) and rotated queries, head by head by groups of 8 threads.  The others take
// kTokens side rows each that are no tree rows: tokens of the cache before them and, with bf16
// pages, zeros after them (who reads f16 side rows puts zeros there itself).  Bound by
// latencies: 64 trees of 32 rows 61 us with a row a block, 254 of them without a tree row.
constexpr int kPrepThreads = 256, kGroups = kPrepThreads / 8, kTokens = 16;
template <int kType, int kTree>
__global__ void __launch_bounds__(kPrepThreads) paged_prep_kernel(const __grid_constant__ TileArgs ta, const uint8_t* pool_k, const uint8_t* pool_v) {
    constexpr bool kF16 = kType != DART_KV_BF16;
    __shared__ float2 turn_of[kTree][kHeadDim / 2];  // cos, sin; of element 8 p + e at [8 e + p]
    __shared__ int row_of[kTokens];                  // of the pool, of head 0; -1: no such page
    const PagedArgs& a = ta.p;
    const int tid = threadIdx.x, p = tid & 7, group = tid >> 3, s = blockIdx.x;
    const int tree_blocks = (a.B + kTree) / kTree;  // of B + 1 rows
    const bool tree = static_cast<int>(blockIdx.y) < tree_blocks;
    const int b0 = blockIdx.y * kTree, b_end = min(b0 + kTree, a.B + 1);
    const long long in = static_cast<long long>(s) * (a.B + 1);
    const int rows = a.Hq + 2 * a.Hkv, jobs = (b_end - b0) * rows;  // queries, keys, values of a tree row
    auto source = [&](int job) {
        const int b = b0 + job / rows, i = job % rows;
        return i < a.Hq ? a.q + (in + b) * a.q_stride + i * kHeadDim
                        : i < a.Hq + a.Hkv ? a.k + (in + b) * a.k_stride + (i - a.Hq) * kHeadDim : a.v + (in + b) * a.v_stride + (i - a.Hq - a.Hkv) * kHeadDim;
    };
    constexpr int kBatch = 2;  // rows of a group on their way at a time
    uint4 ahead[kBatch][2];
    auto fetch = [&](int job0) {
#pragma unroll
        for (int u = 0; u < kBatch; u++) {
            const int job = job0 + u * kGroups + group;
            ahead[u][0] = ahead[u][1] = make_uint4(0u, 0u, 0u, 0u);
            if (job < jobs) {
                const uint4* src = reinterpret_cast<const uint4*>(source(job));
                ahead[u][0] = ld_plain(src + p);
                ahead[u][1] = ld_plain(src + 8 + p);
            }
        }
    };
    pdl_wait();
    pdl_trigger();  // (after the wait: the next kernel reads lengths and pages before its own)
    if (tree) fetch(0);  // (whatever the length and the number of nodes are)
    const int len = seq_len(a, s), nodes = seq_nodes(a, s), tail = len % kKeys;
    // piece i of side row j (of 16 bytes)
    auto side_piece = [&](int kv, int head, int j, int i) {
        const long long row = (static_cast<long long>(s) * a.Hkv + head) * ta.sk + j;
        return (kv ? ta.side_v : ta.side_k) + (kF16 ? (row >> 7) * (16 * kKeys) + i * kKeys + (row & 127) : row * 16 + i);
    };
    auto side_scale = [&](int kv, int head, int j) { return (kv ? ta.side_vs : ta.side_ks) + (static_cast<long long>(s) * a.Hkv + head) * ta.sk + j; };
    if (!tree) {
        const int list = tail + (kF16 ? 0 : (tail + nodes) / kKeys * kKeys + kKeys - (tail + nodes + 1));  // side rows that are no tree rows
        const int j0 = (blockIdx.y - tree_blocks) * kTokens, j_end = min(j0 + kTokens, list);
        if (j0 >= j_end) return;
        if (tid < j_end - j0) {
            const int j = j0 + tid, key = len - tail + j;
            int row = -1;
            if (j < tail) {
                const int page = ld_plain(a.table + static_cast<long long>(s) * a.max_pages + (key >> a.page_log2));
                if (page >= 0 && page < a.num_pages)
                    row = static_cast<int>(((static_cast<long long>(page) * a.Hkv) << a.page_log2) + (key & ((1 << a.page_log2) - 1)));
                else if (a.status)
                    atomicOr(a.status, kDevBounds);
            }
            row_of[tid] = row;
        }
        __syncthreads();
        if (kF16) {
            // a warp a head's keys or values: 16 tokens by 2 of their 8 blocks of 16 elements at a time
            const int warp = tid >> 5, token = tid & 15, first = (tid >> 4) & 1;
            const bool in = j0 + token < j_end;  // (whole warps stay together)
            const int row0 = in ? row_of[token] : -1;
            for (int i = warp; i < 2 * a.Hkv; i += kPrepThreads / 32) {
                const int kv = i >= a.Hkv, head = i - kv * a.Hkv, j = j0 + token;
                const long long row = row0 + (static_cast<long long>(head) << a.page_log2);
                const uint8_t* src = (kv ? pool_v : pool_k) + row * row_bytes(kType);
                uint4 x[4];
                uint32_t block[4];
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const int c = 2 * e + first;
                    x[e] = make_uint4(0u, 0u, 0u, 0u);
                    block[e] = 0u;
                    if (row0 < 0) continue;
                    if (kType == DART_KV_E2M1) {
                        const uint2 y = ld_plain(reinterpret_cast<const uint2*>(src) + c);
                        x[e].x = y.x;
                        x[e].y = y.y;
                        block[e] = ld_plain((kv ? a.vb : a.kb) + row * kBlocks + c);
                    } else {
                        x[e] = ld_plain(reinterpret_cast<const uint4*>(src) + c);
                    }
                }
                uint32_t any = 0;  // (a row of zeros has no part in the tile's power of two)
#pragma unroll
                for (int e = 0; e < 4; e++) any |= kType == DART_KV_E2M1 ? block[e] & 0x7Fu : e4m3_bits(x[e]);
                any |= __shfl_xor_sync(kFull, any, 16);
                if (!in) continue;
                if (first == 0) *side_scale(kv, head, j) = any ? ld_plain((kv ? a.vs : a.ks) + row) : 0.0f;
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    uint32_t y[8];
                    if (kType == DART_KV_E2M1) {
                        const uint32_t by = e4m3_f16(block[e] | block[e] << 8);
                        uint32_t lo[4], hi[4];
                        e2m1_f16(x[e].x, lo);
                        e2m1_f16(x[e].y, hi);
#pragma unroll
                        for (int k = 0; k < 4; k++) {
                            y[k] = mul_f16x2(lo[k], by);
                            y[4 + k] = mul_f16x2(hi[k], by);
                        }
                    } else {
                        const uint32_t w[4] = {x[e].x, x[e].y, x[e].z, x[e].w};
#pragma unroll
                        for (int k = 0; k < 4; k++) {
                            y[2 * k] = e4m3_f16(w[k]);
                            y[2 * k + 1] = e4m3_f16(w[k] >> 16);
                        }
                    }
                    uint4* d = side_piece(kv, head, j, 2 * (2 * e + first));
                    d[0] = make_uint4(y[0], y[1], y[2], y[3]);
                    d[kKeys] = make_uint4(y[4], y[5], y[6], y[7]);
                }
            }
        } else {
            for (int i = group; i < (j_end - j0) * 2 * a.Hkv; i += kGroups) {
                const int token = i / (2 * a.Hkv), rest = i % (2 * a.Hkv), kv = rest >= a.Hkv, head = rest - kv * a.Hkv;
                int j = j0 + token;
                uint4 lo = make_uint4(0u, 0u, 0u, 0u), hi = lo;
                if (row_of[token] >= 0) {
                    const uint4* src = reinterpret_cast<const uint4*>(kv ? pool_v : pool_k) + (row_of[token] + (static_cast<long long>(head) << a.page_log2)) * 16;
                    lo = src[p];
                    hi = src[8 + p];
                }
                if (j >= tail) j += nodes + 1;
                uint4* d = side_piece(kv, head, j, p);
                d[0] = lo;
                d[8] = hi;
            }
        }
        return;
    }
    for (int b = max(b0, nodes + 1); b < b_end; b++) {  // no node: zeros as output
        uint4* out = reinterpret_cast<uint4*>(a.out + (in + b) * a.Hq * kHeadDim);
        for (int i = tid; i < a.Hq * 16; i += kPrepThreads) out[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    if (b0 > nodes) return;
    if (tid < kTree * (kHeadDim / 2)) {
        const int b = b0 + tid / (kHeadDim / 2), e = tid % (kHeadDim / 2);
        if (b <= nodes) {
            const int depth = b > 0 ? ld_plain(a.depths + static_cast<long long>(s) * a.B + b - 1) : 0;
            float sn, cs;
            rope_sincos(a.turns.f[e], len + depth, &sn, &cs);
            turn_of[tid / (kHeadDim / 2)][8 * (e % 8) + e / 8] = make_float2(cs, sn);
        }
    }
    __syncthreads();
    for (int job0 = 0; job0 < jobs; job0 += kBatch * kGroups) {
        uint4 raw[kBatch][2];
#pragma unroll
        for (int u = 0; u < kBatch; u++) {
            raw[u][0] = ahead[u][0];
            raw[u][1] = ahead[u][1];
        }
        if (kTree > 1 || job0 + kBatch * kGroups < jobs) fetch(job0 + kBatch * kGroups);
#pragma unroll
        for (int u = 0; u < kBatch; u++) {
            if (job0 + u * kGroups >= jobs) break;  // (whole warps stay together)
            const int job = min(job0 + u * kGroups + group, jobs - 1), tr = job / rows, b = b0 + tr, i = job % rows;
            const bool use = job0 + u * kGroups + group < jobs && b <= nodes;
            Piece x = unpack_piece(raw[u][0], raw[u][1]);
            if (i < a.Hq + a.Hkv)
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const float2 t = turn_of[tr][8 * e + p];
                    const float lo = x.lo[e], hi = x.hi[e];
                    x.lo[e] = lo * t.x - hi * t.y;
                    x.hi[e] = hi * t.x + lo * t.y;
                }
            uint4 lo, hi;
            const float factor = pack_piece<kF16>(x, &lo, &hi);
            if (!use) continue;
            if (i < a.Hq) {
                const int head = i >> a.g_log2, row = (b << a.g_log2) + (i & (a.G - 1));
                const long long tile = (static_cast<long long>(s) * a.Hkv + head) * ta.nqt + (row >> 7);
                uint4* d = ta.qr + tile * (16 * kRows) + (row & 127);
                d[p * kRows] = lo;
                d[(8 + p) * kRows] = hi;
                if (!kF16) {
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
                if (kF16 && p == 0) ta.q_scale[tile * kRows + (row & 127)] = factor * a.sl2;
            } else {
                const int kv = i >= a.Hq + a.Hkv, head = i - a.Hq - kv * a.Hkv;
                uint4* d = side_piece(kv, head, tail + b, p);
                d[0] = lo;
                d[kF16 ? 8 * kKeys : 8] = hi;
                if (kF16 && p == 0) *side_scale(kv, head, tail + b) = factor;
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

// The warp's largest x >= 0.
__device__ __forceinline__ float largest_of(float x) { return __uint_as_float(__reduce_max_sync(kFull, __float_as_uint(x))); }
// The largest scale of a tile of e4m3 codes among rows that are not all 0.  By a warp.
__device__ __noinline__ float largest_in_use(const uint8_t* tile, const float* scales) {
    float most = 0.0f;
#pragma unroll 1
    for (int row = threadIdx.x & 31; row < kKeys; row += 32)
        if (row_in_use<DART_KV_E4M3>(tile, nullptr, row)) most = fmaxf(most, scales[row]);
    return largest_of(most);
}

// ------------------------------------------------------------ e4m3 or e2m1 pages as f16 tiles

// One block per tile of a sequence and kv head (whole cache tiles, then side
// tiles): codes times their key's scale (e2m1: and block scale) over a power of two
// that the tile's keys (and, apart, values) have in common: that factor rounded to f16 and
// its product with the code again (both exact where scales are powers of two).
template <int kType>
__global__ void __launch_bounds__(256) paged_widen_kernel(const __grid_constant__ TileArgs ta, const uint8_t* pool_k, const uint8_t* pool_v) {
    __shared__ float scale_of[2 * kKeys];
    __shared__ int row_of[kKeys];  // of the pool; -1: no such page
    __shared__ float top_of[8];
    __shared__ bool used[2 * kKeys];
    const PagedArgs& a = ta.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int head = blockIdx.x % a.Hkv, s = blockIdx.x / a.Hkv, t = blockIdx.y;
    // Cache tiles need nothing of the preparation, which lets this kernel start when all before
    // it has ended.  (The last tiles of a head are never of the cache, so this kernel does
    // not end before the preparation.)
    pdl_trigger();
    const int len = seq_len(a, s), nodes = seq_nodes(a, s), whole = len / kKeys, tail = len % kKeys;
    const bool cache_tile = t < whole;
    if (!cache_tile) pdl_wait();
    if (t > whole + (tail + nodes) / kKeys) return;
    const int live = cache_tile ? kKeys : tail + nodes + 1 - (t - whole) * kKeys;  // rows of a side tile that exist
    const long long side = (static_cast<long long>(s) * a.Hkv + head) * ta.sk + (t - whole) * kKeys;
    if (cache_tile && tid < kKeys) {
        const int at = t * kKeys + tid;
        const int page = ld_plain(a.table + static_cast<long long>(s) * a.max_pages + (at >> a.page_log2));
        const bool there = page >= 0 && page < a.num_pages;
        if (!there && a.status) atomicOr(a.status, kDevBounds);
        row_of[tid] = there ? static_cast<int>(((static_cast<long long>(page) * a.Hkv + head) << a.page_log2) + (at & ((1 << a.page_log2) - 1))) : -1;
    }
    __syncthreads();
    // groups of 8 lanes a row, 16-byte pieces p and 8 + p of it a lane: on their way while the scales are compared
    const int p = tid & 7, group = tid >> 3;
    constexpr int kRounds = 2 * kKeys / 32;
    uint4 c[kRounds];  // codes of both pieces (e2m1: a word each, and the row's block scales)
    if (cache_tile)
#pragma unroll
        for (int i = 0; i < kRounds; i++) {
            const int row = row_of[(i * 32 + group) & 127];
            c[i] = make_uint4(0u, 0u, 0u, 0u);
            if (row < 0) continue;
            const uint8_t* pool = i >= kRounds / 2 ? pool_v : pool_k;
            if (kType == DART_KV_E2M1) {
                const uint32_t* src = reinterpret_cast<const uint32_t*>(pool + static_cast<long long>(row) * row_bytes(kType));
                const uint2 block = ld_plain(reinterpret_cast<const uint2*>(i >= kRounds / 2 ? a.vb : a.kb) + row);
                c[i] = make_uint4(ld_plain(src + p), ld_plain(src + 8 + p), block.x, block.y);
            } else {
                const uint2* src = reinterpret_cast<const uint2*>(pool + static_cast<long long>(row) * row_bytes(kType));
                const uint2 x = ld_plain(src + p), y = ld_plain(src + 8 + p);
                c[i] = make_uint4(x.x, x.y, y.x, y.y);
            }
        }
    {
        const int kv = tid >> 7, key = tid & 127;
        float sc = 0.0f;
        if (!cache_tile)
            sc = key < live ? __ldcg((kv ? ta.side_vs : ta.side_ks) + side + key) : 0.0f;
        else if (row_of[key] >= 0)
            sc = ld_plain((kv ? a.vs : a.ks) + row_of[key]);
        if (cache_tile) {
            // rows of zeros have no part in the powers of two
#pragma unroll
            for (int i = 0; i < kRounds; i++) {
                if (kType == DART_KV_E2M1) {  // (the same in all lanes of the row)
                    if (p == 0) used[i * 32 + group] = e2m1_in_use(make_uint2(c[i].z, c[i].w));
                } else {
                    const unsigned rows = __ballot_sync(kFull, e4m3_bits(c[i]) != 0u);
                    if (p == 0) used[i * 32 + group] = (rows >> (lane & 24) & 0xFFu) != 0u;
                }
            }
            __syncthreads();
            if (!used[tid]) sc = 0.0f;
        }
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
        const float factor = scale_of[kv * kKeys + key] * __uint_as_float(0x7F000000u - __float_as_uint(ref[kv]));
        float of[2] = {factor, factor};
        uint32_t x[2][4];
        if (cache_tile && kType == DART_KV_E2M1) {
            const uint32_t block = e4m3_f16(__byte_perm(c[i].z, c[i].w, (p >> 1) * 0x11 + 0x40));
            const float2 by = __half22float2(*reinterpret_cast<const __half2*>(&block));
            of[0] *= by.x;
            of[1] *= by.y;
            e2m1_f16(c[i].x, x[0]);
            e2m1_f16(c[i].y, x[1]);
        } else if (cache_tile) {
            const uint32_t w[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
#pragma unroll
            for (int e = 0; e < 4; e++) {
                x[e >> 1][2 * (e & 1)] = e4m3_f16(w[e]);
                x[e >> 1][2 * (e & 1) + 1] = e4m3_f16(w[e] >> 16);
            }
        } else {
            const uint4* src = (kv ? ta.side_v : ta.side_k) + (side >> 7) * (16 * kKeys) + key;
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const uint4 y = key < live ? __ldcg(src + (8 * h + p) * kKeys) : make_uint4(0u, 0u, 0u, 0u);
                x[h][0] = y.x;
                x[h][1] = y.y;
                x[h][2] = y.z;
                x[h][3] = y.w;
            }
        }
        uint4* d = (kv ? ta.wide_v : ta.wide_k) + (tile * kKeys + key) * 16 + p;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const __half2 by = __float2half2_rn(of[h]);
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&x[h][e]), by);
                x[h][e] = *reinterpret_cast<const uint32_t*>(&r);
            }
            d[8 * h] = make_uint4(x[h][0], x[h][1], x[h][2], x[h][3]);
        }
    }
}

// ------------------------------------------------------------ the schedule

// A place in the list: kv heads of a sequence one after the other, the units
// (query tiles) of a head one after the other.  A unit's length in the list is
// its tiles (its last row sees tree rows up to itself) and unit_cost.
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
        for (int q = 0; q < nqt; q++) n += tiles(a, q) + a.unit_cost;
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
                for (int t; r.tile >= (t = r.tiles(a, r.qt) + a.unit_cost); r.qt++) r.tile -= t;
                return r;
            }
            done += __shfl_sync(kFull, upto, 31);
        }
        r.s = a.nseq;
        return r;
    }
};

// A share's parts of units, one after the other.
struct UnitPart {
    int s, head, qt, t0, t1, tiles, whole, tail, nodes;  // tiles [t0, t1) of a unit of `tiles`
};
struct Walk : UnitPart {  // (the part at hand)
    TilePlace p;
    long long left;  // places of the share from p on
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
            left -= tiles + a.unit_cost - t0;
            p.next_unit(a);
            if (t0 < t1) return true;
        }
        return false;
    }
};

// The softmax warps have no registers for that: theirs is in shared memory, and so are
// the part at hand and the next one.
struct WalkSlot {
    Walk walk;
    UnitPart part[2];
    __device__ __forceinline__ bool next(const PagedArgs& a, int which, int lane) {  // by a whole warp
        int more = 0;
        __syncwarp();
        if (lane == 0) {
            Walk w = walk;
            more = w.next(a);
            walk = w;
            part[which] = w;
        }
        __syncwarp();
        return __shfl_sync(kFull, more, 0) != 0;
    }
};

// ------------------------------------------------------------ the tiles

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
// O += P V (MN-major V: 16 keys of 128 bytes a step; P of keys 64 .. 127 lies 64
// columns behind that of keys 0 .. 63).
template <bool kFirst, int kk = 0>
__device__ __forceinline__ void mma_s(uint32_t d, uint32_t q, uint32_t k_lo, uint32_t idesc) {
    mma_at<kk * 8, ((kk >> 2) * kHalf + (kk & 3) * 32) / 16>(d, q, k_lo, idesc, kFirst && kk == 0 ? 0u : 1u);
    if constexpr (kk + 1 < kHeadDim / 16) mma_s<kFirst, kk + 1>(d, q, k_lo, idesc);
}
template <int kk = 0>
__device__ __forceinline__ void mma_pv(uint32_t d, uint32_t p, uint32_t v_lo, uint32_t idesc, uint32_t first) {
    mma_at<(kk >> 2) * 64 + (kk & 3) * 8, kk * 2048 / 16>(d, p, v_lo, idesc, kk > 0 ? 1u : 1u - first);
    if constexpr (kk + 1 < kKeys / 16) mma_pv<kk + 1>(d, p, v_lo, idesc, first);
}

template <Source kSource>
struct TGeo {
    static constexpr bool kConv = kSource == kCodes || kSource == kCodes4, kFour = kSource == kCodes4;
    // Three operand tiles of K and of V; converted ones two of each, and raw tiles of
    // half or a quarter of the size before them.
    static constexpr int kStages = kConv ? 2 : 3;
    static constexpr int kRawK = kConv ? 3 : 0, kRawV = kFour ? 3 : kConv ? 2 : 0;
    static constexpr int kRing = 8;  // a tile's factors outlive its operands: S runs up to two tiles ahead of the softmax, K two ahead of S
    static constexpr int kOps = 2 * kStages * kTile;
    static constexpr int kRawTile = kFour ? kHalf / 2 : kHalf;
    static constexpr int kRaw = (kRawK + kRawV) * kRawTile;
    static constexpr int kRawScale = kFour ? 4 + kBlocks : 4;  // bytes of a key
    static constexpr int kRawScales = (kRawK + kRawV) * kKeys * kRawScale;
    static constexpr int kBars = 4 * kStages + 2 * (kRawK + kRawV) + (kConv ? kRing : 0) + 9;
    static constexpr int kExchange = 4 * kRows * 4 + 16 * 4 + kRing * 8 + (kSoft / 32) * static_cast<int>(sizeof(WalkSlot));
    static constexpr int kSmem = kOps + kRaw + kRawScales + kBars * 8 + kExchange + 16;
    // loads, MMAs, 8 softmax warps, kConv: 2 that convert K, 2 V
    static constexpr int kFirstSoft = 2, kFirstConv = kFirstSoft + kSoft / 32;
    static constexpr int kThreads = 32 * (kFirstConv + (kConv ? 4 : 0));
};

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

// The two words of a row of mask words that hold bits [o, o + 64) (o >= -128), and
// those bits (outside the row they are 0).
struct MaskWords {
    uint64_t first, second;
    __device__ __forceinline__ void load(const uint64_t* m, int mw, int o) {
        const int w = max(o, 0) >> 6;
        first = o > -64 && w < mw ? ld_plain(m + w) : 0ull;
        second = o > 0 && w + 1 < mw ? ld_plain(m + w + 1) : 0ull;
    }
    __device__ __forceinline__ uint64_t bits(int o) const {
        if (o <= -64) return 0ull;
        if (o <= 0) return first << -o;
        const int sh = o & 63;
        return first >> sh | (sh ? second << (64 - sh) : 0ull);
    }
};

template <Source kSource>
__global__ void __launch_bounds__(TGeo<kSource>::kThreads, 1)
    paged_tiles_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                       const __grid_constant__ CUtensorMap tmSk, const __grid_constant__ CUtensorMap tmSv,
                       const __grid_constant__ TileArgs ta) {
    using G_ = TGeo<kSource>;
    constexpr bool kConv = G_::kConv;          // converting warps
    constexpr bool kFour = G_::kFour;
    constexpr bool kF16 = kSource != kPages;   // f16 operands, with a factor per row of Q and per tile of K and V
    constexpr int kStages = G_::kStages;
    const PagedArgs& a = ta.p;
    extern __shared__ __align__(1024) uint8_t tiles_smem[];
    uint8_t* sK = tiles_smem;
    uint8_t* sV = sK + kStages * kTile;
    uint8_t* rK = sV + kStages * kTile;  // raw tiles
    uint8_t* rV = rK + G_::kRawK * G_::kRawTile;
    float* raw_scales = reinterpret_cast<float*>(rV + G_::kRawV * G_::kRawTile);  // [raw K stages, raw V stages][key]
    uint8_t* raw_blocks = reinterpret_cast<uint8_t*>(raw_scales + (G_::kRawK + G_::kRawV) * kKeys);  // [the same][key][8]
    uint64_t* k_full = reinterpret_cast<uint64_t*>(reinterpret_cast<uint8_t*>(raw_scales) + G_::kRawScales);
    uint64_t* k_empty = k_full + kStages;   // S of the tile done
    uint64_t* v_full = k_empty + kStages;
    uint64_t* v_empty = v_full + kStages;   // PV of the tile done
    uint64_t* rk_full = v_empty + kStages;
    uint64_t* rk_empty = rk_full + G_::kRawK;
    uint64_t* rv_full = rk_empty + G_::kRawK;
    uint64_t* rv_empty = rv_full + G_::kRawV;
    uint64_t* sc_full = rv_empty + G_::kRawV;
    uint64_t* s_full = sc_full + (kConv ? G_::kRing : 0);  // [2] by S buffer
    uint64_t* p_full = s_full + 2;          // [2] the same (P(n + 1) may be there before P(n) is waited for)
    uint64_t* pv_done = p_full + 2;         // [2]
    uint64_t* q_ready = pv_done + 2;
    uint64_t* o_free = q_ready + 1;         // the unit's O has been read
    uint64_t* tdown = o_free + 1;
    float* xch = reinterpret_cast<float*>(k_full + G_::kBars);  // [2][warpgroup][128] row max / sum exchange
    int* xok = reinterpret_cast<int*>(xch + 4 * kRows);         // [2][warpgroup][4] "no wait failed"
    float2* tile_ref = reinterpret_cast<float2*>(xok + 16);      // [tile % kRing] powers of two of K and V
    WalkSlot* slots = reinterpret_cast<WalkSlot*>(tile_ref + G_::kRing);  // [softmax warp]
    int* misc = reinterpret_cast<int*>(slots + kSoft / 32);      // TMEM base, abort
    volatile int* abort = &misc[1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_trigger();

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; i++) {
            mbar_init(&k_full[i], kConv ? 2 : 1);
            mbar_init(&k_empty[i], 1);
            mbar_init(&v_full[i], kConv ? 2 : 1);
            mbar_init(&v_empty[i], 1);
        }
        for (int i = 0; i < G_::kRawK; i++) {
            mbar_init(&rk_full[i], 1);
            mbar_init(&rk_empty[i], 2);
        }
        for (int i = 0; i < G_::kRawV; i++) {
            mbar_init(&rv_full[i], 1);
            mbar_init(&rv_empty[i], 2);
        }
        if (kConv)
            for (int i = 0; i < G_::kRing; i++) mbar_init(&sc_full[i], 2);
        for (int i = 0; i < 2; i++) {
            mbar_init(&s_full[i], 1);
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
                    uint8_t* dst = kConv ? (kv ? rV : rK) + st * G_::kRawTile : (kv ? sV : sK) + st * kTile;
                    const CUtensorMap* tm = cache_tile ? (kv ? &tmV : &tmK) : (kv ? &tmSv : &tmSk);
                    ok = warp_wait<kWaitPolls>(empty, (static_cast<uint32_t>(n / stages) & 1u) ^ 1u, abort);
                    if (!ok) break;
                    k_ahead = kv == 0;
                    if (lane == 0)
                        mbar_arrive_expect_tx(full, kConv ? G_::kRawTile + kKeys * G_::kRawScale : kTile);
                    __syncwarp();
                    if (!cache_tile) {
                        if (lane < 2)
                            tma_load_2d(dst + lane * kHalf, tm, full, 64 * lane, laid_row, policy);
                    } else if (lane < per_tile) {
                        const uint32_t at = static_cast<uint32_t>(lane << a.page_log2) * (kFour ? 64 : 128);
                        tma_load_2d(dst + at, tm, full, 0, static_cast<int>(row), policy);
                        if (!kConv) tma_load_2d(dst + kHalf + at, tm, full, 64, static_cast<int>(row), policy);
                        if (kConv) {
                            const long long sr = row < a.pool_rows ? row : 0;
                            const int first = (kv * G_::kRawK + st) * kKeys + (lane << a.page_log2);
                            bulk_load(raw_scales + first, (kv ? a.vs : a.ks) + sr, 4u << a.page_log2, full);
                            if (kFour) bulk_load(raw_blocks + first * kBlocks, (kv ? a.vb : a.kb) + sr * kBlocks, static_cast<uint32_t>(kBlocks) << a.page_log2, full);
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
                // S(n + 1) takes the place of P(n - 1): products run in the order of their issue, and
                // PV(n - 1) was issued before it.
                auto issue_s = [&](int n) -> bool {
                    const int st = n % kStages;
                    if (!soon(&k_full[st], static_cast<uint32_t>(n / kStages) & 1u, abort)) return false;
                    tc_fence_after();
                    const uint32_t k = __shfl_sync(kFull, (k_lo + st * (kTile >> 4)) & 0x3FFFu, 0), d = base + kSCol + __shfl_sync(kFull, n & 1, 0) * kKeys;
                    mma_s<true>(d, base + kQCol, k, idesc_s);
                    if (!kF16) mma_s<false>(d, base + kQLoCol, k, idesc_s);
                    commit_elected(&s_full[n & 1]);
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
                    mma_pv(base + kOCol, base + kSCol + __shfl_sync(kFull, n & 1, 0) * kKeys,
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
                if (!ok && lane == 0) attn_timeout(a.status, abort);
                // The last products end before tensor memory is given back, whoever gives up a wait (in a good
                // run the softmax has waited for them, and this costs nothing).
                __syncwarp();
                commit_elected(tdown);
                attn_drain(tdown, 0);
            }
        }
    } else if (warp < G_::kFirstConv) {
        // ---------------------------------------------------------- softmax
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
        WalkSlot& slot = slots[warp - G_::kFirstSoft];
        if (lane == 0) slot.walk = w;
        int which = 0;  // of the slot's parts: the next one
        bool have = slot.next(a, 0, lane), ok = true;
        float rs = a.sl2;  // scores in log2 units = products * rs (f16: * the tile's power of two of K)
        float2 ref_ahead = make_float2(1.0f, 1.0f);  // (kWidened: a tile's powers of two, read a tile ahead)
        auto refs = [&](const UnitPart& u) { return ta.wide_refs + (static_cast<long long>(u.s) * a.Hkv + u.head) * ta.wide_tiles; };
        // this thread's half of its row's query into tensor memory, and what else the part begins with
        auto load_q = [&](const UnitPart& u) {
            const bool in = u.qt * kRows + r < (u.nodes + 1) << a.g_log2;
            const long long unit = (static_cast<long long>(u.s) * a.Hkv + u.head) * ta.nqt + u.qt, at = unit * (16 * kRows) + 8 * wg * kRows + r;
#pragma unroll
            for (int i = 0; i < (kF16 ? 1 : 2); i++) {
                uint32_t q[32];
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const uint4 y = in ? __ldcg((i ? ta.q_lo : ta.qr) + at + e * kRows) : make_uint4(0u, 0u, 0u, 0u);
                    q[4 * e] = y.x;
                    q[4 * e + 1] = y.y;
                    q[4 * e + 2] = y.z;
                    q[4 * e + 3] = y.w;
                }
                if (kF16) rs = in ? __ldcg(ta.q_scale + unit * kRows + r) : a.sl2;
                if (kSource == kWidened) ref_ahead = __ldcg(refs(u) + u.t0);
                tmem_st32(tl + (i ? kQLoCol : kQCol) + wg * 32, q);
            }
            tmem_wait_st();
            arrive(q_ready);
        };
        pdl_wait();
        if (have) load_q(slot.part[0]);
        int n = 0, part = 0;
        while (have) {
            const UnitPart& u = slot.part[which];
            which ^= 1;
            const int t1 = u.t1, whole = u.whole;
            auto node = [&]() { return (u.qt * kRows + r) >> a.g_log2; };  // tree row of this row
            const bool idle = !__any_sync(kFull, node() <= u.nodes);  // (in both warps of the lane quarter)
            // m_run: the row's reference.  f16: O is in units of vref, the largest of the
            // tiles' powers of two so far; P has a factor 2^7 (at most 2^15), so that 2^-31
            // of the largest weight still counts, and its tile's power of two over vref
            constexpr float kBoost = kF16 ? 7.0f : 0.0f;
            float m_run = -INFINITY, l = 0.0f, vref = 0.0f;
            // Mask words of side tiles, read a tile ahead.  first_node: tree node of the first key of
            // this half of tile t (negative: cache, row 0).
            auto first_node = [&](int t) { return (t - whole) * kKeys + cb - u.tail - 1; };
            MaskWords words{};
            auto fetch_words = [&](int t) {
                if (t < whole) return;
                const int b = node(), o = first_node(t);
                if (b > 0 && b <= u.nodes && o < b) words.load(a.mask + (static_cast<long long>(u.s) * a.B + b - 1) * a.mw, a.mw, o);
            };
            fetch_words(u.t0);
            for (int t = u.t0; t < t1; t++, n++) {
                // visible keys of this row among this warpgroup's 64 of the tile
                // (of a whole cache tile all, in a row of no node too: it is not written)
                uint64_t vis = ~0ull;
                bool all_seen = true;
                if (t >= whole && !idle) {
                    const int b = node(), o = first_node(t);
                    vis = 0ull;
                    if (b > 0 && b <= u.nodes && o < b) {  // (bits beyond the row's own are not used)
                        vis = words.bits(o);
                        if (b - o < 64) vis &= (1ull << (b - o)) - 1ull;
                    }
                    if (o < 0) vis |= o <= -64 ? ~0ull : (1ull << -o) - 1ull;
                    all_seen = __all_sync(kFull, vis == ~0ull);
                }
                if (t + 1 < t1) fetch_words(t + 1);
                // Both warps of the lane quarter reach the exchange of every iteration and
                // leave the loop at the same point: a failed wait is exchanged with the row
                // max and acted on after it.
                if (kConv && ok && !soon(&sc_full[n % G_::kRing], static_cast<uint32_t>(n / G_::kRing) & 1u, abort)) ok = false;
                if (ok && !soon(&s_full[n & 1], static_cast<uint32_t>(n >> 1) & 1u, abort)) ok = false;
                if (!ok) attn_timeout(a.status, abort);
                if (idle) {  // rows of no node: nothing of them is read
                    if (!ok) break;
                    arrive(&p_full[n & 1]);
                    if (t + 1 == t1) {
                        have = slot.next(a, which, lane);
                        if (have) load_q(slot.part[which]);
                    }
                    continue;
                }
                const uint32_t s_at = tl + kSCol + (n & 1) * kKeys + cb;
                float sv[64];
                float mx = -INFINITY, rt = rs, vtile = 0.0f;
                if (ok) {
                    if (kF16) {
                        const float2 ref = kConv ? tile_ref[n % G_::kRing] : ref_ahead;
                        // not 0, where both factors are tiny (rows of zeros): hidden keys are -inf by now
                        rt = fmaxf(rt * ref.x, FLT_MIN);
                        vtile = ref.y;
                        if (kSource == kWidened && t + 1 < t1) ref_ahead = __ldcg(refs(u) + t + 1);
                    }
                    tc_fence_after();
                    tmem_ld64(s_at, sv);
                    if (!all_seen) {
#pragma unroll
                        for (int c = 0; c < 64; c++)
                            if (!((vis >> c) & 1ull)) sv[c] = -INFINITY;
                    }
                    // (four chains: one alone would be a third of the tile's time in latencies)
                    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < 64; c += 8)
#pragma unroll
                        for (int e = 0; e < 4; e++) m4[e] = max3(m4[e], sv[c + e], sv[c + 4 + e]);
                    mx = max3(m4[0], m4[1], fmaxf(m4[2], m4[3]));
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
                // P takes the place of the scores that this thread has read; O must be stable
                // (PV(n - 1) done) only when it is rescaled.  On a timeout this tile is skipped; the pair leaves the loop
                // together at the next exchange.
                if (t > u.t0 && __any_sync(kFull, resc)) {
                    if (!soon(&pv_done[(n - 1) & 1], static_cast<uint32_t>((n - 1) >> 1) & 1u, abort)) {
                        attn_timeout(a.status, abort);
                        ok = false;
                        continue;
                    }
                    tc_fence_after();
#pragma unroll(kConv ? 1 : 4)  // (the less code, the better)
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
#pragma unroll
                for (int h = 0; h < 64; h += 32) {
                    uint32_t pk[16];
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const int c = h + i;
                        float2 x = fma2(make_float2(sv[c], sv[c + 1]), make_float2(rt, rt), make_float2(nm, nm));
                        float2 z = fma2(make_float2(sv[c + 2], sv[c + 3]), make_float2(rt, rt), make_float2(nm, nm));
                        x = make_float2(ex2(x.x), ex2(x.y));
                        z = make_float2(ex2(z.x), ex2(z.y));
                        sum0 = add2(sum0, x);
                        sum1 = add2(sum1, z);
                        pk[i >> 1] = kF16 ? pack_f16x2(x.x, x.y) : pack_bf16x2(x.x, x.y);
                        pk[(i >> 1) + 1] = kF16 ? pack_f16x2(z.x, z.y) : pack_bf16x2(z.x, z.y);
                    }
                    tmem_st16u(s_at + (h >> 1), pk);
                }
                sum0 = add2(sum0, sum1);
                const float lsum = sum0.x + sum0.y;
                tmem_wait_st();
                l += kF16 ? lsum * __uint_as_float(0x7F000000u - __float_as_uint(down)) : lsum;  // (1 / down)
                arrive(&p_full[n & 1]);
                if (t + 1 == t1) {
                    // the next part's queries, while the last PV runs: all products with this
                    // part's have been seen
                    have = slot.next(a, which, lane);
                    if (have) load_q(slot.part[which]);
                }
            }
            // The pair leaves together: an `ok` lost after the last exchange is exchanged here, in a
            // part without rows too (the next one may have some, and barriers that both have to reach).
            if (ok && (!soon(&pv_done[(n - 1) & 1], static_cast<uint32_t>((n - 1) >> 1) & 1u, abort) || a.test_wait_fails(warp, part++))) {
                attn_timeout(a.status, abort);
                ok = false;
            }
            if (idle) {
                exchange(0.0f, ok);
                if (!ok) break;
                arrive(o_free);
                continue;
            }
            l += exchange(l, ok);
            if (!ok) break;
            tc_fence_after();
            const int b = node(), row = u.qt * kRows + r;
            const bool row_ok = b <= u.nodes;
            if (u.t0 == 0 && t1 == u.tiles) {
                // rows in whole lines: 8 lanes exchange their rows' 8 pieces
                const float inv = l > 0.0f ? (kF16 ? vref : 1.0f) / l : 0.0f;
                uint4 y[8];
#pragma unroll
                for (int h = 0; h < 8; h += 4) {
                    float o[32];
                    tmem_ld32(tl + kOCol + cb + 8 * h, o);
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        y[h + e] = make_uint4(pack_bf16x2(o[8 * e] * inv, o[8 * e + 1] * inv), pack_bf16x2(o[8 * e + 2] * inv, o[8 * e + 3] * inv),
                                              pack_bf16x2(o[8 * e + 4] * inv, o[8 * e + 5] * inv), pack_bf16x2(o[8 * e + 6] * inv, o[8 * e + 7] * inv));
                }
                arrive(o_free);
                transpose8(y, lane);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const int their = row - (lane & 7) + e, tb = their >> a.g_log2;  // row of lane 8 (lane / 8) + e
                    if (tb <= u.nodes)
                        reinterpret_cast<uint4*>(a.out + ((static_cast<long long>(u.s) * (a.B + 1) + tb) * a.Hq + u.head * a.G + (their & (a.G - 1))) * kHeadDim + cb)[lane & 7] = y[e];
                }
            } else {
                TilePart* d = reinterpret_cast<TilePart*>(a.parts) + 2 * blockIdx.x + (u.t0 > 0 ? 0 : 1);
#pragma unroll(kConv ? 1 : 2)
                for (int h = 0; h < 16; h += 8) {
                    float o[32];
                    tmem_ld32(tl + kOCol + cb + 4 * h, o);
                    if (h == 8) arrive(o_free);
                    if (!row_ok) continue;
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        const float by = kF16 ? vref : 1.0f;
                        d->o[wg * 16 + h + e][r] = make_float4(o[4 * e] * by, o[4 * e + 1] * by, o[4 * e + 2] * by, o[4 * e + 3] * by);
                    }
                }
                if (row_ok && wg == 0) d->ml[r] = make_float2(m_run, l);
            }
        }
    } else if constexpr (kConv) {
        // ---------------------------------------------------------- raw tiles to operands: a thread per two keys
        // Two warps for K, two for V, each on its own: a warp looks at all the tile's scales for
        // itself, which costs less than to meet the others.
        const int cw = warp - G_::kFirstConv, kv = cw >> 1, row0 = (cw & 1) * 32 + lane;
        uint64_t* raw_full = kv ? rv_full : rk_full;
        uint64_t* raw_empty = kv ? rv_empty : rk_empty;
        uint64_t* op_full = kv ? v_full : k_full;
        uint64_t* op_empty = kv ? v_empty : k_empty;
        const uint8_t* raw_tile = kv ? rV : rK;
        uint8_t* op_tile = kv ? sV : sK;
        const int raw_stages = kv ? G_::kRawV : G_::kRawK;
        const float* side_scale = kv ? ta.side_vs : ta.side_ks;
        const uint4* side_rows = kv ? ta.side_v : ta.side_k;
        bool ok = true, waited = false;
        int n = 0, raw = 0;  // tiles, whole cache tiles so far
        while (ok && w.next(a)) {
            float unit_top = 0.0f;  // the largest power of two of this part's tiles so far
            for (int t = w.t0; t < w.t1; t++, n++) {
                const bool cache_tile = t < w.whole;
                if (!cache_tile && !waited) {
                    pdl_wait();
                    waited = true;
                }
                const int st = n % kStages, rs = raw % raw_stages;
                const long long side = (static_cast<long long>(w.s) * a.Hkv + w.head) * ta.sk + (t - w.whole) * kKeys;
                ok = !cache_tile || soon(&raw_full[rs], static_cast<uint32_t>(raw / raw_stages) & 1u, abort);
                if (!ok) break;
                const float* scale_of = raw_scales + (kv * G_::kRawK + rs) * kKeys;
                const int live = cache_tile ? kKeys : w.tail + w.nodes + 1 - (t - w.whole) * kKeys;  // rows that exist
                float4 four;
                if (cache_tile) {
                    four = reinterpret_cast<const float4*>(scale_of)[lane];
                } else {
                    const float* of = side_scale + side;
                    auto scale = [&](int i) { return i < live ? __ldcg(of + i) : 0.0f; };
                    four = make_float4(scale(lane), scale(lane + 32), scale(lane + 64), scale(lane + 96));
                }
                auto largest = [&]() { return largest_of(fmaxf(max3(four.x, four.y, four.z), fmaxf(four.w, 0.0f))); };
                float top = largest();
                ok = soon(&op_empty[st], (static_cast<uint32_t>(n / kStages) & 1u) ^ 1u, abort);
                if (!ok) break;
                if (cache_tile && top >= unit_top) {
                    // (once a part, mostly) Rows of zeros have no part in it.  Of e4m3 codes one row of the
                    // largest scale is looked at first: 64 trees of 32 rows over up to 4096 keys 142 us
                    // without any of this, 146 with it, 151 where all rows are looked at.
                    if (kFour) {
                        const uint4* of = reinterpret_cast<const uint4*>(raw_blocks + ((kv * G_::kRawK + rs) * kKeys + 4 * lane) * kBlocks);
                        const uint4 x = of[0], y = of[1];
                        if (!e2m1_in_use(make_uint2(x.x, x.y))) four.x = 0.0f;
                        if (!e2m1_in_use(make_uint2(x.z, x.w))) four.y = 0.0f;
                        if (!e2m1_in_use(make_uint2(y.x, y.y))) four.z = 0.0f;
                        if (!e2m1_in_use(make_uint2(y.z, y.w))) four.w = 0.0f;
                        top = largest();
                    } else {
                        const int place = four.x == top ? 0 : four.y == top ? 1 : four.z == top ? 2 : four.w == top ? 3 : 4;
                        const int row = __ffs(__ballot_sync(kFull, place < 4)) - 1;  // (of a lane; 0 where all scales are NaN or negative)
                        const uint8_t* tile = raw_tile + rs * G_::kRawTile;
                        if (!e4m3_row_in_use(tile, max(4 * row + __shfl_sync(kFull, place, max(row, 0)), 0) & (kKeys - 1), lane)) top = largest_in_use(tile, scale_of);
                    }
                }
                const float ref = above(top);
                unit_top = fmaxf(unit_top, ref);
                if (row0 == 0) {
                    (kv ? tile_ref[n % G_::kRing].y : tile_ref[n % G_::kRing].x) = ref;
                    mbar_arrive(&sc_full[n % G_::kRing]);
                }
                const float inv = __uint_as_float(0x7F000000u - __float_as_uint(ref));  // 1 / ref
                if (kFour && cache_tile) {
                    // codes times (block scale * scale over the common power of two), rounded to f16:
                    // exact where the scale is a power of two, as the cache writes leave it.  Two
                    // blocks at a time, the next two on their way: those trees 140 us, one of 17 rows
                    // over 131072 keys 91; without the loop 149 and 93, one step at a time 135 and 101.
                    const uint8_t* src = raw_tile + rs * G_::kRawTile;
                    const uint8_t* bl = raw_blocks + (kv * G_::kRawK + rs) * kKeys * kBlocks;
                    uint8_t* dst = op_tile + st * kTile;
                    uint4 ahead = *reinterpret_cast<const uint4*>(src + swz64(row0, 0));
                    uint32_t b_ahead = *reinterpret_cast<const uint16_t*>(bl + row0 * kBlocks);
                    float s_ahead = scale_of[row0];
#pragma unroll 2
                    for (int i = 0; i < 8; i++) {
                        const int row = row0 + 64 * (i >> 2), c = i & 3, nr = row0 + 64 * ((i + 1) >> 2 & 1), nc = (i + 1) & 3;
                        const uint4 y = ahead;
                        const float part = fminf(s_ahead * inv, 1.0f);
                        const uint32_t wide = e4m3_f16(b_ahead);
                        ahead = *reinterpret_cast<const uint4*>(src + swz64(nr, nc));
                        b_ahead = *reinterpret_cast<const uint16_t*>(bl + nr * kBlocks + 2 * nc);
                        s_ahead = scale_of[nr];
                        const float2 of = __half22float2(*reinterpret_cast<const __half2*>(&wide));
                        uint8_t* d = dst + (c >> 1) * kHalf;
#pragma unroll
                        for (int e = 0; e < 2; e++) {
                            const __half2 by = __float2half2_rn((e ? of.y : of.x) * part);
                            const uint32_t f = *reinterpret_cast<const uint32_t*>(&by);
                            uint32_t lo[4], hi[4];
                            e2m1_f16(e ? y.z : y.x, lo);
                            e2m1_f16(e ? y.w : y.y, hi);
                            *reinterpret_cast<uint4*>(d + swz(row, (4 * c + 2 * e) & 7)) = make_uint4(mul_f16x2(lo[0], f), mul_f16x2(lo[1], f), mul_f16x2(lo[2], f), mul_f16x2(lo[3], f));
                            *reinterpret_cast<uint4*>(d + swz(row, (4 * c + 2 * e + 1) & 7)) = make_uint4(mul_f16x2(hi[0], f), mul_f16x2(hi[1], f), mul_f16x2(hi[2], f), mul_f16x2(hi[3], f));
                        }
                    }
                } else {
#pragma unroll 1
                    for (int row = row0; row < kKeys; row += 64) {
                        const float sc = cache_tile ? scale_of[row] : row < live ? __ldcg(side_scale + side + row) : 0.0f;
                        // the key's scale over the common power of two, at most 1, rounded to f16: that
                        // moves the key's scores or its values by 2^-12 of themselves at most, as
                        // much as the rounding of an operand does (a row of zeros may have a larger one)
                        const float part = fminf(sc * inv, 1.0f);
                        const __half2 by = __float2half2_rn(part);
                        auto times = [&](uint32_t x) {
                            const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&x), by);
                            return *reinterpret_cast<const uint32_t*>(&r);
                        };
                        uint8_t* dst = op_tile + st * kTile;
                        uint4 x[8];
                        if (cache_tile) {
                            const uint8_t* src = raw_tile + rs * G_::kRawTile;
#pragma unroll
                            for (int c = 0; c < 8; c++) x[c] = *reinterpret_cast<const uint4*>(src + swz(row, c));
#pragma unroll
                            for (int c = 0; c < 8; c++) {
                                uint8_t* d = dst + (c >> 2) * kHalf;
                                *reinterpret_cast<uint4*>(d + swz(row, (2 * c) & 7)) =
                                    make_uint4(times(e4m3_f16(x[c].x)), times(e4m3_f16(x[c].x >> 16)), times(e4m3_f16(x[c].y)), times(e4m3_f16(x[c].y >> 16)));
                                *reinterpret_cast<uint4*>(d + swz(row, (2 * c + 1) & 7)) =
                                    make_uint4(times(e4m3_f16(x[c].z)), times(e4m3_f16(x[c].z >> 16)), times(e4m3_f16(x[c].w)), times(e4m3_f16(x[c].w >> 16)));
                            }
                        } else {
                            const uint4* src = side_rows + (side >> 7) * (16 * kKeys) + row;
#pragma unroll 1
                            for (int q = 0; q < 2; q++) {
                                if (row >= live) {
#pragma unroll
                                    for (int c = 0; c < 8; c++) *reinterpret_cast<uint4*>(dst + q * kHalf + swz(row, c)) = make_uint4(0u, 0u, 0u, 0u);
                                    continue;
                                }
#pragma unroll
                                for (int c = 0; c < 8; c++) x[c] = __ldcg(src + (8 * q + c) * kKeys);
#pragma unroll
                                for (int c = 0; c < 8; c++)
                                    *reinterpret_cast<uint4*>(dst + q * kHalf + swz(row, c)) = make_uint4(times(x[c].x), times(x[c].y), times(x[c].z), times(x[c].w));
                            }
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the MMAs read it
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&op_full[st]);
                    // Only now, when what was read from it is in use: an arrival right after the
                    // loads let the slot be refilled before they had returned.
                    if (cache_tile) mbar_arrive(&raw_empty[rs]);
                }
                raw += cache_tile;
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
// share i - 1 began: 16 rows each, 16 threads (8 elements each) a row.  kBatch parts are on their
// way at a time: eight where a unit has several (107 registers), two where most have one or two,
// so that more blocks run at once (2 and 8: one tree of 300 nodes over 2048 bf16 keys 30.7 and 32.1 us,
// eight of 127 over up to 4096 66.5 and 70.5; one of 64 over 2048 22.5 and 20.4, of 16 over
// 131072 100.7 and 94.4).
template <int kBatch>
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
    for (int c = c0; c <= c1; c += kBatch) {
        float2 ml[kBatch];
        float4 y[kBatch], z[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; u++) {
            ml[u] = make_float2(-INFINITY, 0.0f);
            if (c + u > c1) continue;
            const TilePart* x = static_cast<const TilePart*>(a.parts) + 2 * (c + u) + (c + u < i ? 1 : 0);
            ml[u] = x->ml[r];
            y[u] = x->o[2 * d8][r];
            z[u] = x->o[2 * d8 + 1][r];
        }
#pragma unroll
        for (int u = 0; u < kBatch; u++) {
            if (ml[u].x == -INFINITY) continue;
            const float up = fmaxf(top, ml[u].x), old = top == -INFINITY ? 0.0f : ex2(top - up), by = ex2(ml[u].x - up);
            top = up;
            l = l * old + ml[u].y * by;
            const float v[8] = {y[u].x, y[u].y, y[u].z, y[u].w, z[u].x, z[u].y, z[u].z, z[u].w};
#pragma unroll
            for (int k = 0; k < 8; k++) o[k] = o[k] * old + v[k] * by;
        }
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    __nv_bfloat16* d = a.out + ((static_cast<long long>(s) * (a.B + 1) + b) * a.Hq + head * a.G + (row & (a.G - 1))) * kHeadDim + 8 * d8;
    *reinterpret_cast<uint4*>(d) = make_uint4(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv),
                                              pack_bf16x2(o[4] * inv, o[5] * inv), pack_bf16x2(o[6] * inv, o[7] * inv));
}

// e4m3 and e2m1 pages are widened first where a kv head has at least this many query
// tiles, each of which would convert all keys again (a tile of a unit takes 1.05
// us from f16 tiles and 1.4 converted), and where the f16 tiles of the longest
// sequences take at most 4 GB.  Widened / converted, eight trees over up to 4096 keys, 64
// of them, two over up to 16384: 4 query tiles e4m3 81 / 81, 582 / 527, 86 / 76 us, e2m1 79 / 79,
// 560 / 505, 82 / 77; 5 tiles (64 trees: up to 2048 keys) e4m3 93 / 100, 399 / 460, 97 / 90, e2m1
// 90 / 97, 391 / 436, 94 / 93.
constexpr int kWidenTiles = 5;
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
    if (cache.dtype != DART_KV_BF16 && w.nqt >= kWidenTiles && each <= kWidenBytes / 2 && tiles <= 65535) w.wide_tiles = static_cast<int>(tiles);
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
bool paged_tiles_prepare_device() { return allow_smem<kPages>() && allow_smem<kCodes>() && allow_smem<kCodes4>() && allow_smem<kWidened>(); }

template <Source kSource>
static cudaError_t launch_tiles(int sms, cudaStream_t st, const CUtensorMap& k, const CUtensorMap& v, const CUtensorMap& side_k,
                                const CUtensorMap& side_v, const TileArgs& ta) {
    return launch_pdl(paged_tiles_kernel<kSource>, dim3(sms), dim3(TGeo<kSource>::kThreads), TGeo<kSource>::kSmem, st, k, v, side_k, side_v, ta);
}

int launch_paged_tiles(PagedArgs a, const dart_kv_cache& cache, uint8_t* workspace, int sms, cudaStream_t st) {
    const bool e4m3 = cache.dtype == DART_KV_E4M3, e2m1 = cache.dtype == DART_KV_E2M1;
    const TileWs w = tile_ws(a.nseq, a.B, a.Hq, cache, a.max_pages);
    const bool wide = w.wide_tiles > 0;
    TileArgs ta{};
    a.unit_cost = wide || !(e4m3 || e2m1) ? kTileCost : kTileCostConverted;
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
    const bool maps = wide ? encode_rows(&tmK, ta.wide_k, heads * w.wide_tiles * kKeys, DART_KV_BF16, kKeys) && encode_rows(&tmV, ta.wide_v, heads * w.wide_tiles * kKeys, DART_KV_BF16, kKeys)
                           : encode_rows(&tmK, cache.k, a.pool_rows, cache.dtype, cache.page_size) && encode_rows(&tmV, cache.v, a.pool_rows, cache.dtype, cache.page_size) &&
                                 encode_rows(&tmSk, ta.side_k, side_rows, DART_KV_BF16, kKeys) && encode_rows(&tmSv, ta.side_v, side_rows, DART_KV_BF16, kKeys);
    if (!maps) return DART_ERR_CUDA;
    if (wide) {
        tmSk = tmK;  // (side tiles lie among the others)
        tmSv = tmV;
    }
    // Four tree rows a block from this many rows on (bf16 / e4m3 / e2m1, four and one a block: eight trees of
    // 96 nodes over up to 4096 keys 67.4 and 63.6 / 84.6 and 81.8 / 81.7 and 79.3 us, of 150 79.6 and 78.9 / 93.8 and
    // 96.8 / 91.1 and 94.0, of 512 234 and 239 / 248 and 253 / 245 and 249; 32 of 31 over up to 2048 52.7 and
    // 54.2 / 60.5 and 59.4 / 57.3 and 56.9).
    const bool four = static_cast<long long>(a.nseq) * (a.B + 1) >= 7 * sms;
    const int tree_blocks = four ? (a.B + 4) / 4 : a.B + 1;
    // up to 127 cache tokens before the tree rows and, in bf16, up to 127 rows of zeros after them
    const int others = e4m3 || e2m1 ? kKeys - 1 : 2 * (kKeys - 1);
    const dim3 prep(static_cast<unsigned>(a.nseq), static_cast<unsigned>(tree_blocks + (others + kTokens - 1) / kTokens));
    const uint8_t *pk = static_cast<const uint8_t*>(cache.k), *pv = static_cast<const uint8_t*>(cache.v);
    const dim3 pb(kPrepThreads), wg(static_cast<unsigned>(heads), static_cast<unsigned>(w.wide_tiles)), wb(256);
    auto prepare = [&](auto* kernel) { return launch_pdl(kernel, prep, pb, 0, st, ta, pk, pv); };
    cudaError_t e = e2m1   ? prepare(four ? paged_prep_kernel<DART_KV_E2M1, 4> : paged_prep_kernel<DART_KV_E2M1, 1>)
                    : e4m3 ? prepare(four ? paged_prep_kernel<DART_KV_E4M3, 4> : paged_prep_kernel<DART_KV_E4M3, 1>)
                           : prepare(four ? paged_prep_kernel<DART_KV_BF16, 4> : paged_prep_kernel<DART_KV_BF16, 1>);
    if (e == cudaSuccess && wide)
        e = e2m1 ? launch_pdl(paged_widen_kernel<DART_KV_E2M1>, wg, wb, 0, st, ta, pk, pv) : launch_pdl(paged_widen_kernel<DART_KV_E4M3>, wg, wb, 0, st, ta, pk, pv);
    if (e == cudaSuccess)
        e = wide   ? launch_tiles<kWidened>(sms, st, tmK, tmV, tmSk, tmSv, ta)
            : e2m1 ? launch_tiles<kCodes4>(sms, st, tmK, tmV, tmSk, tmSv, ta)
            : e4m3 ? launch_tiles<kCodes>(sms, st, tmK, tmV, tmSk, tmSv, ta)
                   : launch_tiles<kPages>(sms, st, tmK, tmV, tmSk, tmSv, ta);
    if (e == cudaSuccess) e = launch_pdl(heads * w.nqt * 4 <= sms ? paged_tiles_join_kernel<8> : paged_tiles_join_kernel<2>, dim3(8 * (sms - 1)), dim3(256), 0, st, a);
    return e == cudaSuccess ? DART_OK : DART_ERR_CUDA;
}

}  // namespace dart

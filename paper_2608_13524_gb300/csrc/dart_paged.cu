// Tree attention over the paged cache.  Contract: include/dart_cache.h.
//
// paged_rows_kernel: few query rows a sequence (decoding), bound by HBM.  A
// unit of work is the query rows of one kv head of one sequence (a row = a tree
// row and one of the G query heads that share the kv head) against all keys
// that the rows may see: the sequence's cache, then its tree rows, in chunks
// of 16 (bf16), 32 (e4m3) or 64 (e2m1) keys.  The chunks of all units form one list,
// which the warps of the GPU share evenly, so that ragged lengths and a single
// long sequence load every SM alike; lengths are read on the device, so the
// split is made there.  A warp streams its chunks through a ring of TMA stages
// of its own and keeps its own running maximum, sum and accumulators: no warp
// waits for another.  Units that several warps share are left as partial
// results in the workspace, which paged_join_kernel joins in order.
//
// The products are warp-wide 16 x 8 x 16 matrix instructions with keys (for
// S^T = K Q^T) and head dimensions (O^T = V^T P^T) along the 16 and rows along
// the 8, once for up to 8 rows and twice (kN = 2) for up to 16: with rows along
// the 16, 8 rows took as many products and accumulators as 16.  A chunk of 16
// bf16 keys takes 8 KB from HBM for 24 kN of them, far below any tensor rate,
// and scores and probabilities stay in registers (a 128-row tile of the
// tensor-memory path would be 7/8 empty or more).
//
// Measured, 64 sequences of up to 8192 keys, 8 kv heads, one token each: bf16
// pages 170 us, 6.4 TB/s, 94 % of the measured copy bandwidth; e4m3 pages 94 us,
// 6.0 TB/s, 88 %, where the conversions (64 codes a thread and chunk) come
// second; a call of a few keys takes 12 us, a chain of two launches and six or
// seven dependent loads.  With rows along the 16 and 8 warps e4m3 took 116 us.
// e2m1 pages 80 us (4.1 TB/s, 60 %): 331 instructions per 16 keys, half of them the
// conversions and the products with block scales, issue 56 % active with 2.75 warps a
// scheduler, DRAM 52 %.  Larger chunks pay the copies' issue (six a chunk) less often and
// give the scores' products four chains instead of two: 91 us with chunks of 32 keys.
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
#include "dart_kernels.h"
#include "dart_paged.cuh"
#include "dart_ring.h"

namespace dart {

bool encode_rows(CUtensorMap* m, const void* base, long long rows, int type, int box_rows) {
    EncodeTiledFn fn = tensor_map_encoder();
    if (!fn) return false;
    const bool bytes = type != DART_KV_BF16, four = type == DART_KV_E2M1;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(four ? kHeadDim / 2 : kHeadDim), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(row_bytes(type))};
    const cuuint32_t box[2] = {type == DART_KV_E4M3 ? 128u : 64u, static_cast<cuuint32_t>(box_rows)}, estr[2] = {1, 1};
    return fn(m, bytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides,
              box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, four ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace {

constexpr float kSlack = 8.0f;  // log2 units a score may exceed the row's reference by

template <int kN>
struct Part {  // a unit's partial result
    float o[8 * kN][kHeadDim];
    float2 ml[8 * kN];  // reference (log2 units), sum
};

// Warps of a CTA: as many as their registers allow (for up to 8 rows 168 a
// thread; 10 warps: e4m3 93 us instead of 95, pages of 16 tokens 99 instead of
// 96; for up to 16 rows 6 warps instead of 8: 76 us instead of 65).
// e2m1, up to 8 rows: 11, as many as shared memory holds two chunks of 64 keys for (64
// sequences of up to 8192 keys, one token each: 9 warps 94 us, 10 85, 11 80; chunks of 32
// keys with 12 warps 91, 14 95, 16 86).
__host__ __device__ constexpr int rows_warps(int type, int n) { return n > 1 ? 8 : type == DART_KV_E2M1 ? 11 : 12; }

// A unit whose cache values are measured by less than this is measured by 1 once tree rows
// come to it: their weights are 128 over that, which times a tree value has to be a float.
constexpr float kSmallRef = 9.31322574615478515625e-10f;  // 2^-30

// ------------------------------------------------------------ the schedule

// Chunk sizes, and what a unit costs beside its chunks (queries, tree rows,
// the result), in chunks: its list is that much longer, so that warps with
// many short units get fewer of them.  kTokenCost: without a tree (256 sequences of
// up to 1024 e4m3 keys 56.5 us at 1, 54 at 2, 55.5 at 3, 56.5 at 6; bf16 97 at 2, 95 at
// 3 to 7, 97 at 9).  kUnitCost: 64 trees of 3 nodes over 4096 keys, bf16 105 us at 3,
// 100 at 6, 98 at 9; e4m3 71, 65, 65 at 2, 4, 6.  Chunks of 64 keys: half of that (1024
// sequences of up to 512 e2m1 keys, kTokenCost 1 162 us, 2 166; trees of 3 nodes, kUnitCost 2,
// 4, 6: 64 over up to 1000 keys 42, 41, 41 us, 16 over up to 16384 64, 65, 66).  Chunks of 32 e2m1
// keys for up to 16 rows: 40, 75.
template <int kType, int kN>
struct Chunk {
    static constexpr int kKeys = kType == DART_KV_BF16 ? 16 : kType == DART_KV_E2M1 ? 64 : 32;
    static constexpr int kUnitCost = kType == DART_KV_BF16 ? 9 : kKeys == 64 ? (kN == 1 ? 3 : 4) : 6, kTokenCost = kType == DART_KV_BF16 ? 5 : kKeys == 64 ? 1 : 2;
};

// A place in the list of chunks: sequence, kv head, chunk of the unit.
template <int kType, int kN>
struct Place {
    int s, head, chunk;
    int len, nodes, ctx_chunks, chunks, cost;  // of the sequence; cost: the unit's length in the list
    __device__ __forceinline__ void load(const PagedArgs& a) {
        constexpr int kKeys = Chunk<kType, kN>::kKeys;
        len = seq_len(a, s);
        nodes = seq_nodes(a, s);
        ctx_chunks = (len + kKeys - 1) / kKeys;
        chunks = ctx_chunks + (nodes + 1 + 15) / 16;  // (tree rows: 16 at a time)
        cost = chunks + (a.B == 0 ? Chunk<kType, kN>::kTokenCost : Chunk<kType, kN>::kUnitCost);
    }
    __device__ __forceinline__ void next_unit(const PagedArgs& a) {
        chunk = 0;
        if (++head == a.Hkv) {
            head = 0;
            if (++s < a.nseq) load(a);
        }
    }
};

// By one warp: the list's length and, then, the place x of it (of its first 32
// sequences the lengths are kept).
template <int kType, int kN>
struct List {
    long long all, own;  // own: length of sequence `lane`
    __device__ __forceinline__ static long long length(const PagedArgs& a, int s) {
        if (s >= a.nseq) return 0;
        Place<kType, kN> p{};
        p.s = s;
        p.load(a);
        return static_cast<long long>(a.Hkv) * p.cost;
    }
    __device__ __forceinline__ List(const PagedArgs& a, int lane) {
        own = length(a, lane);
        long long n = own;
        for (int s = lane + 32; s < a.nseq; s += 32) n += length(a, s);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(kFull, n, o);
        all = n;
    }
    __device__ __forceinline__ Place<kType, kN> find(const PagedArgs& a, long long x, int lane) const {
        long long done = 0;
        Place<kType, kN> r{};
        for (int s0 = 0; s0 < a.nseq; s0 += 32) {
            const long long n = s0 == 0 ? own : length(a, s0 + lane);
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
                r.s = s0 + l;
                r.load(a);
                r.head = place_div(rest, r.cost);
                r.chunk = static_cast<int>(rest - static_cast<long long>(r.head) * r.cost);
                return r;
            }
            done += __shfl_sync(kFull, upto, 31);
        }
        r.s = a.nseq;
        return r;
    }
};

// Shares: one per warp, each at least this long (values around it make no
// difference: shares are shorter than that in the smallest calls alone).  Chunks of 64
// keys: one token over 500 12.8 us with 1, 14.9 with 2.
constexpr int min_share(int chunk_keys) { return chunk_keys == 64 ? 1 : 2; }

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
// The e4m3 codes of the low or the high half of a word as an f16 pair: exact.
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) {
    uint32_t r;
    asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %1;\n cvt.rn.f16x2.e4m3x2 %0, l;\n}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) {
    uint32_t r;
    asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %1;\n cvt.rn.f16x2.e4m3x2 %0, h;\n}" : "=r"(r) : "r"(w));
    return r;
}
// The transpose of an 8 x 8 matrix of 16-bit values (lane 4 r + c: row r,
// columns 2 c, 2 c + 1).
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// Row of a 16-key chunk behind key slot 8 q + n of the products: chosen so that
// both the reads of K (lanes g, t: row slot_row(q, g), 16-byte
// pieces t, t + 4, ...) and of V (rows slot_row(q, 2t + e), piece g) touch
// every bank once under the 128-byte swizzle.
__device__ __forceinline__ int slot_row(int q, int n) {
    return q * 8 + ((((n >> 2) ^ n) & 1) << 2) + (n & 2) + (n & 1);
}
// The same for 64-byte rows of e2m1 codes and their swizzle: 8-byte pieces t, t + 4 of row
// slot_row4(q, g), piece g of rows slot_row4(q, 2t + e).
__device__ __forceinline__ int slot_row4(int q, int n) { return q * 8 + (((n ^ (n >> 2)) & 1) << 2) + ((n >> 2) << 1) + ((n >> 1) & 1); }

// The unit that a warp comes to next and the places of its share from there on: in shared
// memory, for want of registers.
template <int kType, int kN>
struct NextUnit {
    Place<kType, kN> at;
    long long left;
};

template <int kType, int kN>
struct Geo {
    static constexpr int kKeys = Chunk<kType, kN>::kKeys;
    static constexpr int kSubs = kKeys / 16;                             // products of 16 keys
    static constexpr int kTile = kKeys * row_bytes(kType);               // K or V of a chunk
    static constexpr int kWarps = rows_warps(kType, kN), kThreads = 32 * kWarps;
    static constexpr int kStages = kType == DART_KV_E2M1 ? 2 : kN == 1 ? 2 : 3;
    static constexpr int kRing = kWarps * kStages * 2 * kTile;           // 192 KB (e2m1: 176, 128)
    // e4m3, e2m1: a key's scale; e2m1: its block scales
    static constexpr int kScale = (kType == DART_KV_BF16 ? 0 : 4) + (kType == DART_KV_E2M1 ? kBlocks : 0);
    static constexpr int kScales = kWarps * kStages * 2 * kKeys * kScale;
    static constexpr int kTurns = kWarps * (kHeadDim / 2) * 8;            // a position's angles, of each warp
    static constexpr int kBars = kWarps * kStages * 8;
    static constexpr int kSmem = kRing + kScales + kTurns + kBars + kWarps * static_cast<int>(sizeof(NextUnit<kType, kN>));
};

// 16-byte piece (8 bf16) of a row of the head that step pair i of thread t
// covers; i and i + 2 are 64 elements apart, as RoPE's pairs are.
template <bool kF16>
__device__ __forceinline__ int k_piece(int i, int t) {
    return kF16 ? 8 * (i >> 1) + 2 * t + (i & 1) : 8 * (i >> 1) + t + 4 * (i & 1);
}

template <int kType, int kN>
__global__ void __launch_bounds__(32 * rows_warps(kType, kN), 1)
    paged_rows_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                      const __grid_constant__ PagedArgs a) {
    using G_ = Geo<kType, kN>;
    constexpr bool kF16 = kType != DART_KV_BF16;   // f16 operands; a scale a key
    constexpr bool kFour = kType == DART_KV_E2M1;  // block scales beside it
    constexpr int kWarps = G_::kWarps, kThreads = G_::kThreads;
    constexpr int kKeys = G_::kKeys, kSubs = G_::kSubs, kTile = G_::kTile, kStages = G_::kStages;
    extern __shared__ __align__(1024) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    pdl_trigger();
    uint8_t* ring = smem + warp * kStages * 2 * kTile;
    float* scales = reinterpret_cast<float*>(smem + G_::kRing) + warp * kStages * 2 * kKeys;  // [stage][K, V][key]
    uint8_t* blocks = smem + G_::kRing + kWarps * kStages * 2 * kKeys * 4 + warp * kStages * 2 * kKeys * kBlocks;  // [stage][K, V][key][8]
    float2* turns = reinterpret_cast<float2*>(smem + G_::kRing + G_::kScales) + warp * (kHeadDim / 2);
    uint64_t* bar = reinterpret_cast<uint64_t*>(smem + G_::kRing + G_::kScales + G_::kTurns) + warp * kStages;
    if (lane == 0) {
        for (int i = 0; i < kStages; i++) mbar_init(bar + i, 1);
        fence_mbar_init();
    }
    __syncwarp();
    pdl_wait();

    // rows of no node: zeros
    if (a.B > 0)
        for (long long i = blockIdx.x; i < static_cast<long long>(a.nseq) * (a.B + 1); i += gridDim.x) {
            const int s = static_cast<int>(i / (a.B + 1)), r = static_cast<int>(i % (a.B + 1));
            if (r <= seq_nodes(a, s)) continue;
            uint4* o = reinterpret_cast<uint4*>(a.out + i * a.Hq * kHeadDim);
            for (int j = tid; j < a.Hq * kHeadDim / 8; j += kThreads) o[j] = make_uint4(0, 0, 0, 0);
        }

    const List<kType, kN> list(a, lane);
    const int share = warp * gridDim.x + blockIdx.x;
    const Shares shares(list.all, kWarps * gridDim.x, min_share(kKeys));
    if (share >= shares.count) return;
    Place<kType, kN> load = list.find(a, shares.begin(share), lane);
    int to_load = load.s < a.nseq ? shares.length(share) : 0;  // places of this share not yet loaded
    NextUnit<kType, kN>& next = reinterpret_cast<NextUnit<kType, kN>*>(smem + G_::kRing + G_::kScales + G_::kTurns + G_::kBars)[warp];
    if (lane == 0) {
        a.plan->places[share] = make_int4(load.s, load.head, load.chunk, load.chunks);
        a.plan->nodes[share] = load.nodes;
        if (share == 0) a.plan->count = shares.count;
        next.at = load;
        next.left = to_load;
    }
    __syncwarp();
    StageRing<kStages> fills;
    bool failed = false;
    int none = 0;
    volatile int* abort = &none;  // (a warp waits for no other)
    const uint64_t policy = l2_policy_evict_first();  // (every key is read once)
    const int page_mask = (1 << a.page_log2) - 1, pool_rows = static_cast<int>(a.pool_rows);
    constexpr int kRow = kType == DART_KV_BF16 ? 128 : row_bytes(kType);  // of a tile in shared memory (bf16: two halves)

    // Moves `load` to the next chunk of the cache in this share (or past it).
    auto settle = [&]() {
        while (to_load > 0 && load.chunk >= load.ctx_chunks) {
            to_load -= load.cost - load.chunk;
            load.next_unit(a);
            if (load.s >= a.nseq) to_load = 0;
        }
    };
    // row of a 16-key chunk behind a key slot
    auto row_of = [](int q, int n) { return kFour ? slot_row4(q, n) : slot_row(q, n); };
    auto page_at = [&](int key) {
        return ld_plain(a.table + static_cast<long long>(load.s) * a.max_pages + (key >> a.page_log2));
    };
    // A chunk's tokens lie in up to kKeys / 16 pages, one after the other: lane h has page h
    // of `load`'s, read a chunk ahead of its use (-2: no token falls there).
    constexpr int kKeysLog2 = kKeys == 16 ? 4 : kKeys == 32 ? 5 : 6;
    const int seg_log2 = min(a.page_log2, kKeysLog2), segs = kKeys >> seg_log2;
    int page = 0;
    auto look_up = [&]() {
        settle();
        if (to_load <= 0) return;
        const int key = load.chunk * kKeys + ((lane & (segs - 1)) << seg_log2);
        page = key < load.len ? page_at(key) : -2;
    };
    auto issue = [&]() {  // loads the chunk at `load`: a lane a page
        const int st = fills.stage(fills.filled);
        if (lane == 0) mbar_arrive_expect_tx(bar + st, 2 * kTile + 2 * kKeys * G_::kScale);
        __syncwarp();
        if (lane < segs) {
            uint8_t* k = ring + st * 2 * kTile + (lane << seg_log2) * kRow;
            uint8_t* v = k + kTile;
            const bool there = page >= 0 && page < a.num_pages;
            if (!there && page != -2 && a.status) atomicOr(a.status, kDevBounds);
            const int from = there ? ((page * a.Hkv + load.head) << a.page_log2) + ((load.chunk * kKeys) & page_mask) : 0;
            const int row = there ? from : pool_rows;  // past the pool: zeros
            tma_load_2d(k, &tmK, bar + st, 0, row, policy);
            tma_load_2d(v, &tmV, bar + st, 0, row, policy);
            if (kF16) {
                float* sc = scales + st * 2 * kKeys + (lane << seg_log2);
                bulk_load(sc, a.ks + from, 4u << seg_log2, bar + st);
                bulk_load(sc + kKeys, a.vs + from, 4u << seg_log2, bar + st);
                if (kFour) {
                    uint8_t* bl = blocks + (st * 2 * kKeys + (lane << seg_log2)) * kBlocks;
                    bulk_load(bl, a.kb + static_cast<long long>(from) * kBlocks, static_cast<uint32_t>(kBlocks) << seg_log2, bar + st);
                    bulk_load(bl + kKeys * kBlocks, a.vb + static_cast<long long>(from) * kBlocks, static_cast<uint32_t>(kBlocks) << seg_log2, bar + st);
                }
            } else {
                tma_load_2d(k + kTile / 2, &tmK, bar + st, 64, row, policy);
                tma_load_2d(v + kTile / 2, &tmV, bar + st, 64, row, policy);
            }
        }
        fills.filled++;
        to_load--;
        load.chunk++;
        look_up();
    };
    look_up();
    while (to_load > 0 && fills.room()) issue();

    // (s: in case the lengths change under the call, which leaves its results open)
    while (next.left > 0 && next.at.s < a.nseq) {
        // ---- this warp's part of a unit: chunks [c0, c1)
        const int c0 = next.at.chunk, chunks = next.at.chunks, c1 = static_cast<int>(min(static_cast<long long>(chunks), c0 + next.left));
        const int s = next.at.s, head = next.at.head, len = next.at.len, nodes = next.at.nodes, ctx_chunks = next.at.ctx_chunks;
        const long long seq_row = static_cast<long long>(s) * (a.B + 1);
        __syncwarp();
        if (lane == 0) {
            Place<kType, kN> p = next.at;
            next.left -= p.cost - c0;
            p.next_unit(a);
            next.at = p;
        }
        __syncwarp();
        if (c0 >= c1) continue;  // (the part of a unit's length that stands for its other costs)

        // Single tokens all have the position `len`: its angles once, two a lane, instead of
        // the 16 of every thread's pieces, for the queries and again for the key (1024
        // sequences of up to 512 e4m3 keys 211 us with those, 115 so).
        if (a.B == 0) {
            __syncwarp();
#pragma unroll
            for (int h = 0; h < 2; h++) {
                float sn, cs;
                rope_sincos(a.turns.f[32 * h + lane], len, &sn, &cs);
                turns[32 * h + lane] = make_float2(cs, sn);
            }
            __syncwarp();
        }
        // cosines and sines of elements d0 .. d0 + 7 at a position
        auto angles = [&](int d0, int pos, float (&cs)[8], float (&sn)[8]) {
            if (a.B == 0) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float4 x = *reinterpret_cast<const float4*>(turns + d0 + e);
                    cs[e] = x.x;
                    sn[e] = x.y;
                    cs[e + 1] = x.z;
                    sn[e + 1] = x.w;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++) rope_sincos(a.turns.f[d0 + e], pos, &sn[e], &cs[e]);
            }
        };
        // the queries of rows 8 n + g, rotated, as operands: step pair i covers the 8
        // elements of piece k_piece(i, t) in steps 2 i, 2 i + 1
        uint32_t q[kN][8][2], lo[kN][8][2];
        float rs[kN][2];  // of rows 8 n + 2 t, + 1: scores in log2 units = products * rs
#pragma unroll
        for (int n = 0; n < kN; n++) {
            const int r = 8 * n + g, b = r >> a.g_log2;
            float x[4][8];
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int e = 0; e < 8; e++) x[i][e] = 0.0f;
            if (b <= nodes) {
                const int pos = len + (b > 0 ? ld_plain(a.depths + static_cast<long long>(s) * a.B + b - 1) : 0);
                const __nv_bfloat16* src = a.q + (seq_row + b) * a.q_stride + (head * a.G + (r & (a.G - 1))) * kHeadDim;
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const int d0 = 8 * k_piece<kF16>(i, t);
                    const uint4 u = ld_plain(reinterpret_cast<const uint4*>(src + d0)), w = ld_plain(reinterpret_cast<const uint4*>(src + d0 + 64));
                    const uint32_t uw[4] = {u.x, u.y, u.z, u.w}, ww[4] = {w.x, w.y, w.z, w.w};
                    float cs[8], sn[8];
                    angles(d0, pos, cs, sn);
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        const float x1 = e & 1 ? bf16_hi(uw[e >> 1]) : bf16_lo(uw[e >> 1]);
                        const float x2 = e & 1 ? bf16_hi(ww[e >> 1]) : bf16_lo(ww[e >> 1]);
                        x[i][e] = x1 * cs[e] - x2 * sn[e];
                        x[i + 2][e] = x2 * cs[e] + x1 * sn[e];
                    }
                }
            }
            float down = 1.0f, up = a.sl2;
            if (kF16) {
                // scaled by a power of two to a largest element in [1, 2): f16 then
                // rounds it to 2^-11 whatever the query's magnitude
                float mx = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; i++)
#pragma unroll
                    for (int e = 0; e < 8; e++) mx = fmaxf(mx, fabsf(x[i][e]));
                mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, 2));
                const int ex = min(max(static_cast<int>(__float_as_uint(mx) >> 23) - 127, -100), 120);
                down = __uint_as_float(static_cast<uint32_t>(127 - ex) << 23);
                up *= __uint_as_float(static_cast<uint32_t>(127 + ex) << 23);
            }
            rs[n][0] = __shfl_sync(kFull, up, 8 * t);
            rs[n][1] = __shfl_sync(kFull, up, 8 * t + 4);
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int e = 0; e < 4; e++) {  // words of the piece: elements 2 e, 2 e + 1
                    uint32_t w;
                    if (kF16) {
                        w = pack_f16(x[i][2 * e] * down, x[i][2 * e + 1] * down);
                    } else {
                        // bf16 and what it leaves: with one bf16 term the queries' rounding
                        // alone would move the output as much as its own rounding does
                        w = pack_bf16x2(x[i][2 * e], x[i][2 * e + 1]);
                        lo[n][2 * i + (e >> 1)][e & 1] = pack_bf16x2(x[i][2 * e] - bf16_lo(w), x[i][2 * e + 1] - bf16_hi(w));
                    }
                    q[n][2 * i + (e >> 1)][e & 1] = w;
                }
        }
        // O^T: product j has elements j of piece g (bf16 pages) or 16 g + j (e4m3) in [0, 1],
        // the same 64 (bf16) or 8 further in [2, 3], of rows 8 n + 2 t, + 1
        float acc[kN][8][4], m[kN][2], l[kN][2];
        // e4m3: the accumulators are in units of vref / 128, vref a power of two
        // above every value scale so far, so that f16 probabilities (p <= 2^8 times
        // scale / vref <= 1 times 2^7) neither overflow nor lose small weights
        // (2^-31 of the largest still counts)
        float vref = 0.0f;
#pragma unroll
        for (int n = 0; n < kN; n++) {
            m[n][0] = m[n][1] = -INFINITY;
            l[n][0] = l[n][1] = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; j++)
#pragma unroll
                for (int e = 0; e < 4; e++) acc[n][j][e] = 0.0f;
        }

        // New scores sc[sub][n][2 qq + e] of key slot 8 qq + g and row 8 n + 2 t + e:
        // raises the references where one is exceeded by more than 2^8, and turns the
        // scores into probabilities.
        auto soften = [&](auto& sc) {
            constexpr int subs = sizeof(sc) / sizeof(sc[0]);
            float mx[kN][2];
            bool over = false;
#pragma unroll
            for (int n = 0; n < kN; n++)
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    mx[n][e] = -INFINITY;
#pragma unroll
                    for (int j = 0; j < subs; j++) mx[n][e] = fmaxf(mx[n][e], fmaxf(sc[j][n][e], sc[j][n][2 + e]));
                    over |= mx[n][e] > m[n][e] + kSlack;
                }
            if (__any_sync(kFull, over)) {
#pragma unroll
                for (int n = 0; n < kN; n++)
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        float x = mx[n][e];
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) x = fmaxf(x, __shfl_xor_sync(kFull, x, o));
                        x = fmaxf(m[n][e], x);
                        const float alpha = m[n][e] == -INFINITY ? 0.0f : exp2_fast(m[n][e] - x);
                        m[n][e] = x;
                        l[n][e] *= alpha;
#pragma unroll
                        for (int j = 0; j < 8; j++) {
                            acc[n][j][e] *= alpha;
                            acc[n][j][2 + e] *= alpha;
                        }
                    }
            }
#pragma unroll
            for (int n = 0; n < kN; n++)
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const float ref = m[n][e] == -INFINITY ? 0.0f : m[n][e];
#pragma unroll
                    for (int j = 0; j < subs; j++)
#pragma unroll
                        for (int qq = 0; qq < 2; qq++) {
                            const float w = exp2_fast(sc[j][n][2 * qq + e] - ref);
                            l[n][e] += w;
                            sc[j][n][2 * qq + e] = w;
                        }
                }
        };
        // O^T += V^T P^T of 16 keys with bf16 values: piece(half, q, e) = 16 bytes of
        // key slot (q, 2 t + e): piece g of each half of the row (bf16 pages), or
        // pieces 2 g, 2 g + 1 (tree rows beside e4m3 pages).  P is rounded to bf16, the
        // type of V, which a product's operands share; that moves the output about as much
        // as its own rounding does (0.0021 to 0.0023 of it in all, for 0.0017).  The sum l
        // has the unrounded weights.
        auto values_bf16 = [&](const float (&w)[kN][4], auto&& piece) {
            uint32_t p[kN][2];
#pragma unroll
            for (int n = 0; n < kN; n++) {
                p[n][0] = transpose_8x8(pack_bf16x2(w[n][0], w[n][1]));
                p[n][1] = transpose_8x8(pack_bf16x2(w[n][2], w[n][3]));
            }
            uint32_t x[2][2][2][4];  // [half][q][e][word]
#pragma unroll
            for (int half = 0; half < 2; half++)
#pragma unroll
                for (int qq = 0; qq < 2; qq++)
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        const uint4 y = piece(half, qq, e);
                        x[half][qq][e][0] = y.x;
                        x[half][qq][e][1] = y.y;
                        x[half][qq][e][2] = y.z;
                        x[half][qq][e][3] = y.w;
                    }
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const uint32_t sel = h ? 0x7632 : 0x5410;
                    const uint32_t v[4] = {__byte_perm(x[0][0][0][j], x[0][0][1][j], sel), __byte_perm(x[1][0][0][j], x[1][0][1][j], sel),
                                           __byte_perm(x[0][1][0][j], x[0][1][1][j], sel), __byte_perm(x[1][1][0][j], x[1][1][1][j], sel)};
#pragma unroll
                    for (int n = 0; n < kN; n++) mma_bf16(acc[n][2 * j + h], v, p[n][0], p[n][1]);
                }
        };

        // ---- the cache
        const int c_ctx = min(c1, ctx_chunks);
        for (int c = c0; c < c_ctx; c++) {
            const int st = fills.stage(fills.used), key0 = c * kKeys;
            uint8_t* kt = ring + st * 2 * kTile;
            uint8_t* vt = kt + kTile;
            const float* sck = scales + st * 2 * kKeys;
            uint8_t* blk = blocks + st * 2 * kKeys * kBlocks;
            if (!failed) {
                const bool got = mbar_wait_inline(bar + st, fills.parity(fills.used), abort);
                if (!__all_sync(kFull, got)) {
                    failed = true;
                    if (a.status && lane == 0) atomicOr(a.status, kDevTimeout);
                }
            }
            if (!failed) {
                const int there = len - key0;  // keys of the chunk that exist
                if (there < kKeys) {
                    // anything may lie behind the last one: zeros for V, which P = 0 would
                    // not hide (these stores are ordered before the slot's next copy below)
                    if (kFour) {  // (in any order: the rows are whole)
                        for (int i = lane; i < (kKeys - there) * 4; i += 32)
                            *reinterpret_cast<uint4*>(vt + there * 64 + i * 16) = make_uint4(0, 0, 0, 0);
                        for (int i = lane; i < kKeys - there; i += 32) *reinterpret_cast<uint2*>(blk + (kKeys + there + i) * kBlocks) = make_uint2(0, 0);
                    } else {
                        for (int i = lane; i < (kKeys - there) * 8; i += 32) {
#pragma unroll
                            for (int half = 0; half < (kF16 ? 1 : 2); half++)
                                *reinterpret_cast<uint4*>(vt + half * (kTile / 2) + swz(there + (i >> 3), i & 7)) = make_uint4(0, 0, 0, 0);
                        }
                    }
                    __syncwarp();
                }
                float sc[kSubs][kN][4];  // [16 keys][8 rows][slot g: rows 2t, 2t + 1; slot 8 + g: the same]
#pragma unroll
                for (int j = 0; j < kSubs; j++)
#pragma unroll
                    for (int n = 0; n < kN; n++)
#pragma unroll
                        for (int e = 0; e < 4; e++) sc[j][n][e] = 0.0f;
                if constexpr (kFour) {
                    // step by step for all subs in turn: products that do not wait for one another
#pragma unroll
                    for (int i = 0; i < 2; i++) {  // block t + 4 i of all keys
                        uint2 x[kSubs][2];
                        uint32_t by[kSubs][2];
#pragma unroll
                        for (int j = 0; j < kSubs; j++)
#pragma unroll
                            for (int qq = 0; qq < 2; qq++) {
                                const int row = 16 * j + row_of(qq, g);
                                x[j][qq] = *reinterpret_cast<const uint2*>(kt + swz64(row, (t + 4 * i) >> 1) + 8 * (t & 1));
                                const uint32_t b = *reinterpret_cast<const uint32_t*>(blk + row * kBlocks + 4 * i);
                                by[j][qq] = e4m3_f16(__byte_perm(b, 0u, t * 0x11));
                            }
#pragma unroll
                        for (int w = 0; w < 2; w++)
#pragma unroll
                            for (int h = 0; h < 2; h++)
#pragma unroll
                                for (int j = 0; j < kSubs; j++) {
                                    uint32_t k[4];
#pragma unroll
                                    for (int qq = 0; qq < 2; qq++) {
                                        uint32_t two[2];
                                        e2m1_f16(w ? x[j][qq].y : x[j][qq].x, h, two);
                                        k[qq] = mul_f16x2(two[0], by[j][qq]);
                                        k[2 + qq] = mul_f16x2(two[1], by[j][qq]);
                                    }
#pragma unroll
                                    for (int n = 0; n < kN; n++) mma_f16(sc[j][n], k, q[n][4 * i + 2 * w + h][0], q[n][4 * i + 2 * w + h][1]);
                                }
                    }
                } else if constexpr (kF16) {
#pragma unroll
                    for (int i = 0; i < 2; i++)
#pragma unroll
                        for (int j = 0; j < kSubs; j++) {
                            const uint4 x = *reinterpret_cast<const uint4*>(kt + swz(16 * j + slot_row(0, g), t + 4 * i));
                            const uint4 y = *reinterpret_cast<const uint4*>(kt + swz(16 * j + slot_row(1, g), t + 4 * i));
                            const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                            for (int e = 0; e < 4; e++) {
                                const uint32_t k[4] = {codes_lo(xw[e]), codes_lo(yw[e]), codes_hi(xw[e]), codes_hi(yw[e])};
#pragma unroll
                                for (int n = 0; n < kN; n++) mma_f16(sc[j][n], k, q[n][4 * i + e][0], q[n][4 * i + e][1]);
                            }
                        }
                } else {
                    float sl[kSubs][kN][4];
#pragma unroll
                    for (int j = 0; j < kSubs; j++)
#pragma unroll
                        for (int n = 0; n < kN; n++)
#pragma unroll
                            for (int e = 0; e < 4; e++) sl[j][n][e] = 0.0f;
#pragma unroll
                    for (int i = 0; i < 4; i++)
#pragma unroll
                        for (int j = 0; j < kSubs; j++) {
                            const uint8_t* half = kt + (i >> 1) * (kTile / 2);
                            const uint4 x = *reinterpret_cast<const uint4*>(half + swz(16 * j + slot_row(0, g), t + 4 * (i & 1)));
                            const uint4 y = *reinterpret_cast<const uint4*>(half + swz(16 * j + slot_row(1, g), t + 4 * (i & 1)));
                            const uint32_t k0[4] = {x.x, y.x, x.y, y.y}, k1[4] = {x.z, y.z, x.w, y.w};
#pragma unroll
                            for (int n = 0; n < kN; n++) {
                                mma_bf16(sc[j][n], k0, q[n][2 * i][0], q[n][2 * i][1]);
                                mma_bf16(sl[j][n], k0, lo[n][2 * i][0], lo[n][2 * i][1]);
                                mma_bf16(sc[j][n], k1, q[n][2 * i + 1][0], q[n][2 * i + 1][1]);
                                mma_bf16(sl[j][n], k1, lo[n][2 * i + 1][0], lo[n][2 * i + 1][1]);
                            }
                        }
#pragma unroll
                    for (int j = 0; j < kSubs; j++)
#pragma unroll
                        for (int n = 0; n < kN; n++)
#pragma unroll
                            for (int e = 0; e < 4; e++) sc[j][n][e] += sl[j][n][e];
                }
                float vs[kSubs][2];  // value scales of slots g, 8 + g
#pragma unroll
                for (int j = 0; j < kSubs; j++)
#pragma unroll
                    for (int qq = 0; qq < 2; qq++) {
                        const int key = 16 * j + row_of(qq, g);
                        const float by = kF16 ? sck[key] : 1.0f;
                        vs[j][qq] = kF16 ? sck[kKeys + key] : 1.0f;
#pragma unroll
                        for (int n = 0; n < kN; n++)
#pragma unroll
                            for (int e = 0; e < 2; e++) sc[j][n][2 * qq + e] *= kF16 ? rs[n][e] * by : rs[n][e];
                    }
                if (there < kKeys) {
#pragma unroll
                    for (int j = 0; j < kSubs; j++)
#pragma unroll
                        for (int qq = 0; qq < 2; qq++)
                            if (16 * j + row_of(qq, g) >= there) {
#pragma unroll
                                for (int n = 0; n < kN; n++) sc[j][n][2 * qq] = sc[j][n][2 * qq + 1] = -INFINITY;
                                vs[j][qq] = 0.0f;
                            }
                }
                if constexpr (kF16) {
                    float top = 0.0f;
#pragma unroll
                    for (int j = 0; j < kSubs; j++) top = fmaxf(top, fmaxf(vs[j][0], vs[j][1]));
                    if (__any_sync(kFull, top > vref)) {
                        // (rare) Rows of zeros have no part in it.  Of e4m3 codes one of the largest
                        // scale's rows is looked at first: the rest is code that is not at hand.
                        top = __uint_as_float(__reduce_max_sync(kFull, __float_as_uint(top)));  // (not negative)
                        bool look = kFour;
                        if (!kFour) {
                            int row = -1;
#pragma unroll
                            for (int j = 0; j < kSubs; j++)
#pragma unroll
                                for (int qq = 0; qq < 2; qq++)
                                    if (vs[j][qq] == top) row = 16 * j + row_of(qq, g);
                            look = !e4m3_row_in_use(vt, __shfl_sync(kFull, row, __ffs(__ballot_sync(kFull, row >= 0)) - 1), lane);
                        }
                        if (look) {
                            top = 0.0f;
#pragma unroll 1
                            for (int row = lane; row < kKeys; row += 32)
                                if (row_in_use<kType>(vt, blk + kKeys * kBlocks, row)) top = fmaxf(top, sck[kKeys + row]);
                            top = __uint_as_float(__reduce_max_sync(kFull, __float_as_uint(top)));
                        }
                        if (top > vref) {
                            const float raised = __uint_as_float(min(max(__float_as_uint(top) >> 23, 27u), 252u) + 1u << 23);
                            const float alpha = vref / raised;
                            vref = raised;
#pragma unroll
                            for (int n = 0; n < kN; n++)
#pragma unroll
                                for (int j = 0; j < 8; j++)
#pragma unroll
                                    for (int e = 0; e < 4; e++) acc[n][j][e] *= alpha;
                        }
                    }
                }
                soften(sc);
                if constexpr (kF16) {
                    const float inv = vref > 0.0f ? 128.0f / vref : 0.0f;  // (0: all scales are)
#pragma unroll
                    for (int u = 0; u < kSubs; u++) {
                        const float w0 = fminf(vs[u][0] * inv, 128.0f), w1 = fminf(vs[u][1] * inv, 128.0f);  // (more: rows of zeros)
                        uint32_t p[kN][2];
#pragma unroll
                        for (int n = 0; n < kN; n++) {
                            p[n][0] = transpose_8x8(pack_f16(sc[u][n][0] * w0, sc[u][n][1] * w0));
                            p[n][1] = transpose_8x8(pack_f16(sc[u][n][2] * w1, sc[u][n][3] * w1));
                        }
                        if constexpr (kFour) {
                            // block g of two neighbouring slots' keys: words of 8 codes, and both block scales
                            uint2 x[2][2];
                            uint32_t by[2];
#pragma unroll
                            for (int qq = 0; qq < 2; qq++) {
                                uint32_t b[2];
#pragma unroll
                                for (int e = 0; e < 2; e++) {
                                    const int row = 16 * u + row_of(qq, 2 * t + e);
                                    x[qq][e] = *reinterpret_cast<const uint2*>(vt + swz64(row, g >> 1) + 8 * (g & 1));
                                    b[e] = *reinterpret_cast<const uint32_t*>(blk + (kKeys + row) * kBlocks + (g & 4));
                                }
                                by[qq] = e4m3_f16(__byte_perm(b[0], b[1], (g & 3) * 0x11 + 0x40));
                            }
#pragma unroll
                            for (int odd = 0; odd < 2; odd++) {  // elements 2 j + odd of both words
                                constexpr uint32_t kLow = 0x0F0F0F0Fu;
                                uint32_t v[2][2][4];  // [keys][word][j]
#pragma unroll
                                for (int qq = 0; qq < 2; qq++)
#pragma unroll
                                    for (int w = 0; w < 2; w++) {
                                        const uint32_t c0 = w ? x[qq][0].y : x[qq][0].x, c1 = w ? x[qq][1].y : x[qq][1].x;
                                        e2m1_f16(odd ? ((c0 >> 4) & kLow) | (c1 & ~kLow) : (c0 & kLow) | ((c1 << 4) & ~kLow), v[qq][w]);
#pragma unroll
                                        for (int j = 0; j < 4; j++) v[qq][w][j] = mul_f16x2(v[qq][w][j], by[qq]);
                                    }
#pragma unroll
                                for (int j = 0; j < 4; j++) {
                                    const uint32_t both[4] = {v[0][0][j], v[0][1][j], v[1][0][j], v[1][1][j]};
#pragma unroll
                                    for (int n = 0; n < kN; n++) mma_f16(acc[n][2 * j + odd], both, p[n][0], p[n][1]);
                                }
                            }
                        } else {
                            uint32_t x[2][2][4];
#pragma unroll
                            for (int qq = 0; qq < 2; qq++)
#pragma unroll
                                for (int e = 0; e < 2; e++) {
                                    const uint4 y = *reinterpret_cast<const uint4*>(vt + swz(16 * u + slot_row(qq, 2 * t + e), g));
                                    x[qq][e][0] = y.x;
                                    x[qq][e][1] = y.y;
                                    x[qq][e][2] = y.z;
                                    x[qq][e][3] = y.w;
                                }
#pragma unroll
                            for (int w = 0; w < 2; w++)
#pragma unroll
                                for (int b = 0; b < 2; b++) {
                                    // elements 4 w + 2 b, + 1 of piece g (words w), and 8 further (words 2 + w), of
                                    // both keys of a pair
                                    const uint32_t sel = b ? 0x7362 : 0x5140;
                                    const uint32_t v0 = __byte_perm(x[0][0][w], x[0][1][w], sel), v1 = __byte_perm(x[0][0][2 + w], x[0][1][2 + w], sel);
                                    const uint32_t v2 = __byte_perm(x[1][0][w], x[1][1][w], sel), v3 = __byte_perm(x[1][0][2 + w], x[1][1][2 + w], sel);
                                    const uint32_t first[4] = {codes_lo(v0), codes_lo(v1), codes_lo(v2), codes_lo(v3)};
                                    const uint32_t second[4] = {codes_hi(v0), codes_hi(v1), codes_hi(v2), codes_hi(v3)};
#pragma unroll
                                    for (int n = 0; n < kN; n++) {
                                        mma_f16(acc[n][4 * w + 2 * b], first, p[n][0], p[n][1]);
                                        mma_f16(acc[n][4 * w + 2 * b + 1], second, p[n][0], p[n][1]);
                                    }
                                }
                        }
                    }
                } else {
                    values_bf16(sc[0], [&](int half, int qq, int e) {
                        return *reinterpret_cast<const uint4*>(vt + half * (kTile / 2) + swz(slot_row(qq, 2 * t + e), g));
                    });
                }
                if (there < kKeys) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            __syncwarp();  // every lane has read the stage
            fills.passed(failed);
            if (!failed && to_load > 0) issue();
        }

        // ---- the tree rows, 16 at a time, read and rotated here (keys rounded to bf16, as a
        // bf16 cache holds them later)
        for (int c = max(c0, ctx_chunks); c < c1; c++) {
            const int key0 = (c - ctx_chunks) * 16;
            uint32_t w[2][4][4];  // [key slot 8 qq + g][piece][word]
#pragma unroll
            for (int qq = 0; qq < 2; qq++) {
                const int j = key0 + slot_row(qq, g);
#pragma unroll
                for (int i = 0; i < 4; i++)
#pragma unroll
                    for (int e = 0; e < 4; e++) w[qq][i][e] = 0u;
                if (j <= nodes) {
                    const int pos = len + (j > 0 ? ld_plain(a.depths + static_cast<long long>(s) * a.B + j - 1) : 0);
                    const __nv_bfloat16* k = a.k + (seq_row + j) * a.k_stride + head * kHeadDim;
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        const int d0 = 8 * k_piece<kF16>(i, t);
                        const uint4 x = ld_plain(reinterpret_cast<const uint4*>(k + d0));
                        const uint4 y = ld_plain(reinterpret_cast<const uint4*>(k + d0 + 64));
                        const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
                        float cs[8], sn[8];
                        angles(d0, pos, cs, sn);
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            const float k0 = cs[2 * e], s0 = sn[2 * e], k1 = cs[2 * e + 1], s1 = sn[2 * e + 1];
                            const float x0 = bf16_lo(xw[e]), x1 = bf16_hi(xw[e]), y0 = bf16_lo(yw[e]), y1 = bf16_hi(yw[e]);
                            w[qq][i][e] = pack_bf16x2(x0 * k0 - y0 * s0, x1 * k1 - y1 * s1);
                            w[qq][i + 2][e] = pack_bf16x2(y0 * k0 + x0 * s0, y1 * k1 + x1 * s1);
                        }
                    }
                }
            }
            __syncwarp();
            float sc[1][kN][4];
#pragma unroll
            for (int n = 0; n < kN; n++)
#pragma unroll
                for (int e = 0; e < 4; e++) sc[0][n][e] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const uint32_t k[4] = {w[0][i >> 1][2 * (i & 1)], w[1][i >> 1][2 * (i & 1)], w[0][i >> 1][2 * (i & 1) + 1], w[1][i >> 1][2 * (i & 1) + 1]};
#pragma unroll
                for (int n = 0; n < kN; n++) {
                    if (kF16) {
                        // the queries as one bf16 term (rounded once more, by as much as the
                        // tree keys are): tree keys may leave f16's range
                        uint32_t qb[2];
#pragma unroll
                        for (int e = 0; e < 2; e++) {
                            const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&q[n][i][e]));
                            qb[e] = pack_bf16x2(x.x, x.y);
                        }
                        mma_bf16(sc[0][n], k, qb[0], qb[1]);
                    } else {
                        mma_bf16(sc[0][n], k, q[n][i][0], q[n][i][1]);
                        mma_bf16(sc[0][n], k, lo[n][i][0], lo[n][i][1]);
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < kN; n++)
#pragma unroll
                for (int qq = 0; qq < 2; qq++)
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        const int j = key0 + slot_row(qq, g), b = (8 * n + 2 * t + e) >> a.g_log2;
                        bool see = j <= nodes && b <= nodes;
                        if (see && j > 0)
                            see = j <= b && ((ld_plain(a.mask + (static_cast<long long>(s) * a.B + b - 1) * a.mw + ((j - 1) >> 6)) >> ((j - 1) & 63)) & 1ull);
                        sc[0][n][2 * qq + e] = see ? sc[0][n][2 * qq + e] * rs[n][e] : -INFINITY;
                    }
            soften(sc);
            if (kF16) {
                if (vref < kSmallRef) {
#pragma unroll
                    for (int n = 0; n < kN; n++)
#pragma unroll
                        for (int j = 0; j < 8; j++)
#pragma unroll
                            for (int e = 0; e < 4; e++) acc[n][j][e] *= vref;
                    vref = 1.0f;
                }
                const float inv = 128.0f / vref;
#pragma unroll
                for (int n = 0; n < kN; n++)
#pragma unroll
                    for (int e = 0; e < 4; e++) sc[0][n][e] *= inv;
            }
            values_bf16(sc[0], [&](int half, int qq, int e) {
                const int j = key0 + slot_row(qq, 2 * t + e);
                if (j > nodes) return make_uint4(0, 0, 0, 0);
                return ld_plain(reinterpret_cast<const uint4*>(a.v + (seq_row + j) * a.v_stride + head * kHeadDim + 8 * (kF16 ? 2 * g + half : g + 8 * half)));
            });
        }

        // ---- the result, or this part of it
        const bool whole = c0 == 0 && c1 == chunks;
        Part<kN>* part = static_cast<Part<kN>*>(a.parts) + 2 * static_cast<long long>(share) + (c0 > 0 ? 0 : 1);
#pragma unroll
        for (int n = 0; n < kN; n++)
#pragma unroll
            for (int e = 0; e < 2; e++) {
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) l[n][e] += __shfl_xor_sync(kFull, l[n][e], o);
                const int r = 8 * n + 2 * t + e, b = r >> a.g_log2;
                if (b > nodes) continue;
                float by = kF16 ? vref * 0.0078125f : 1.0f;
                if (whole) by = l[n][e] > 0.0f ? by / l[n][e] : 0.0f;
#pragma unroll
                for (int half = 0; half < 2; half++) {
                    const int d = kF16 ? 16 * g + 8 * half : 64 * half + 8 * g;  // of the 8 elements
                    float o[8];
#pragma unroll
                    for (int k = 0; k < 8; k++) o[k] = acc[n][k][2 * half + e] * by;
                    if (whole) {
                        __nv_bfloat16* dst = a.out + ((seq_row + b) * a.Hq + head * a.G + (r & (a.G - 1))) * kHeadDim + d;
                        *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]),
                                                                    pack_bf16x2(o[4], o[5]), pack_bf16x2(o[6], o[7]));
                    } else {
                        float4* dst = reinterpret_cast<float4*>(&part->o[r][d]);
                        dst[0] = make_float4(o[0], o[1], o[2], o[3]);
                        dst[1] = make_float4(o[4], o[5], o[6], o[7]);
                    }
                }
                if (!whole && g == 0) part->ml[r] = make_float2(m[n][e], l[n][e]);
            }
    }
    if (failed) {  // copies in flight land before the CTA ends
        const unsigned long long t0 = globaltimer_ns();
        for (int i = fills.used; i < fills.filled; i++)
            while (!mbar_try_wait(bar + fills.stage(i), fills.parity(i)))
                if (globaltimer_ns() - t0 > kWaitLimitNs) break;
    }
}

// Joins the parts of the units that several warps shared, in the order of
// their keys.  Block i works if share i begins inside a unit that share i - 1
// began: 16 threads (8 elements each) per row, and as many more groups of
// threads as fit, each with every n-th part, joined in order through shared
// memory.
constexpr int kJoinThreads = 256;
template <int kN>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(const __grid_constant__ PagedArgs a) {
    __shared__ float2 ml_of[8 * kN];
    __shared__ float sum_of[8 * kN][kHeadDim];
    __shared__ int ends[kJoinThreads / 32];
    pdl_trigger();
    const int tid = threadIdx.x, lane = tid & 31, i = blockIdx.x + 1;
    pdl_wait();
    // all that has to be known in one go (the kernel is a chain of loads)
    const int count = a.plan->count, nodes = a.plan->nodes[i];
    const int4 at = a.plan->places[i], prev = a.plan->places[i - 1];
    int4 next = a.plan->places[min(i + 1 + tid, kMaxShares - 1)];
    if (i >= count || at.z == 0 || at.z >= at.w) return;  // (from at.w on the place stands for a unit's other costs)
    if (prev.x == at.x && prev.y == at.y && prev.z > 0) return;
    // the last share that holds chunks of the unit
    int end = i;
    for (int from = i + 1;; from += kJoinThreads) {
        if (from > i + 1) next = a.plan->places[min(from + tid, kMaxShares - 1)];
        const bool in = from + tid < count && next.x == at.x && next.y == at.y && next.z < at.w;
        const unsigned out = __ballot_sync(kFull, !in);
        if (lane == 0) ends[tid >> 5] = out ? __ffs(out) - 1 : 32;
        __syncthreads();
        int n = 0;
        for (int w = 0; w < kJoinThreads / 32; w++) {
            n += ends[w];
            if (ends[w] < 32) break;
        }
        end += n;
        __syncthreads();
        if (n < kJoinThreads) break;
    }
    const int s = at.x, head = at.y, rows = (nodes + 1) << a.g_log2;
    int span = 1;  // rows rounded up to a power of two
    while (span < rows) span *= 2;
    const int slot_of_row = tid >> 4, d8 = tid & 15, r = slot_of_row % span, part0 = slot_of_row / span, step = kJoinThreads / 16 / span;
    const bool live = r < rows;
    // share i - 1 began the unit (its second slot), the others went on with it
    auto slot = [&](int c) { return static_cast<const Part<kN>*>(a.parts) + 2 * static_cast<long long>(c) + (c < i ? 1 : 0); };
    const int c0 = i - 1, c1 = end;
    float top = -INFINITY, l = 0.0f, o[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int kBatch = 4;  // parts on their way at a time
    for (int first = c0 + part0; live && first <= c1; first += kBatch * step) {
        float2 ml[kBatch];
        float4 y[kBatch], z[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; u++) {
            const int c = first + u * step;
            ml[u] = make_float2(-INFINITY, 0.0f);
            if (c > c1) continue;
            const Part<kN>* x = slot(c);
            ml[u] = x->ml[r];
            y[u] = *reinterpret_cast<const float4*>(&x->o[r][8 * d8]);
            z[u] = *reinterpret_cast<const float4*>(&x->o[r][8 * d8 + 4]);
        }
#pragma unroll
        for (int u = 0; u < kBatch; u++) {
            if (ml[u].x == -INFINITY) continue;
            const float up = fmaxf(top, ml[u].x), old = top == -INFINITY ? 0.0f : exp2_fast(top - up), by = exp2_fast(ml[u].x - up);
            top = up;
            l = l * old + ml[u].y * by;
            const float w[8] = {y[u].x, y[u].y, y[u].z, y[u].w, z[u].x, z[u].y, z[u].z, z[u].w};
#pragma unroll
            for (int k = 0; k < 8; k++) o[k] = o[k] * old + w[k] * by;
        }
    }
    // the groups' results, one after the other
    for (int q = 1; q < step; q++) {
        __syncthreads();
        if (part0 == q) {
#pragma unroll
            for (int k = 0; k < 8; k++) sum_of[r][8 * d8 + k] = o[k];
            if (d8 == 0) ml_of[r] = make_float2(top, l);
        }
        __syncthreads();
        if (part0 == 0 && live && ml_of[r].x != -INFINITY) {
            const float2 ml = ml_of[r];
            const float up = fmaxf(top, ml.x), old = top == -INFINITY ? 0.0f : exp2_fast(top - up), by = exp2_fast(ml.x - up);
            top = up;
            l = l * old + ml.y * by;
#pragma unroll
            for (int k = 0; k < 8; k++) o[k] = o[k] * old + sum_of[r][8 * d8 + k] * by;
        }
    }
    if (part0 != 0 || !live) return;
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    __nv_bfloat16* d = a.out + ((static_cast<long long>(s) * (a.B + 1) + (r >> a.g_log2)) * a.Hq + head * a.G + (r & (a.G - 1))) * kHeadDim + 8 * d8;
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
    return static_cast<long long>(c->nseq) * (c->B + 1) * c->Hq <= (1ll << 30) &&
           static_cast<long long>(c->nseq) * cache->Hkv * (c->B + 256) <= (1ll << 30);
}

#ifdef DART_DEBUG
struct {
    int warp, part;
} fail_at = {-1, -1};  // (dart_test_paged_wait)
#endif

// Which kernel: a few rows are streamed from HBM, more are 128-row tiles of the
// tensor-memory path (64 sequences, 16 rows a kv head, up to 4096 keys, here and there: bf16
// pages 103 and 109 us, e4m3 66 and 141, e2m1 82 and 136; 16 over up to 16384 107 and 99, 64 and
// 101, 67 and 104).
constexpr int kFewRows = 16;
bool few_rows(const dart_paged_attn_config& c, const dart_kv_cache& cache) { return (c.B + 1) * (c.Hq / cache.Hkv) <= kFewRows; }

template <int kType>
bool allow_rows_smem() {
    return cudaFuncSetAttribute(paged_rows_kernel<kType, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, Geo<kType, 1>::kSmem) == cudaSuccess &&
           cudaFuncSetAttribute(paged_rows_kernel<kType, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, Geo<kType, 2>::kSmem) == cudaSuccess;
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
    if (!allow_rows_smem<DART_KV_BF16>() || !allow_rows_smem<DART_KV_E4M3>() || !allow_rows_smem<DART_KV_E2M1>())
        return -1;
    if (!paged_tiles_prepare_device()) return -1;
    known[dev].store(sms, std::memory_order_release);
    return sms;
}

template <int kN>
constexpr size_t rows_workspace() {
    constexpr int kWarps = std::max(rows_warps(DART_KV_BF16, kN), rows_warps(DART_KV_E2M1, kN));
    static_assert(kWarps * kMaxSms <= kMaxShares, "the plan holds every share");
    return sizeof(SharePlan) + sizeof(Part<kN>) * 2 * kWarps * kMaxSms;
}

template <int kType, int kN>
int launch_rows(const PagedArgs& a, const dart_kv_cache& cache, int ctas, cudaStream_t st) {
    using G_ = Geo<kType, kN>;
    const int box = std::min(cache.page_size, Chunk<kType, kN>::kKeys);
    CUtensorMap tmK, tmV;
    if (!encode_rows(&tmK, cache.k, a.pool_rows, kType, box) || !encode_rows(&tmV, cache.v, a.pool_rows, kType, box)) return DART_ERR_CUDA;
    if (launch_pdl(paged_rows_kernel<kType, kN>, dim3(ctas), dim3(G_::kThreads), G_::kSmem, st, tmK, tmV, a) != cudaSuccess) return DART_ERR_CUDA;
    return launch_pdl(paged_join_kernel<kN>, dim3(G_::kWarps * ctas - 1), dim3(kJoinThreads), 0, st, a) == cudaSuccess ? DART_OK : DART_ERR_CUDA;
}

}  // namespace
}  // namespace dart

using namespace dart;

extern "C" {

int dart_test_paged_wait(int warp, int part) {
#ifdef DART_DEBUG
    fail_at = {warp, part};
    return DART_OK;
#else
    return warp < 0 && part < 0 ? DART_OK : DART_ERR_UNSUPPORTED;
#endif
}

size_t dart_paged_attention_workspace(const dart_paged_attn_config* cfg, const dart_kv_cache* cache) {
    if (!valid_cfg(cfg, cache)) return 0;
    if (few_rows(*cfg, *cache)) return (cfg->B + 1) * (cfg->Hq / cache->Hkv) <= 8 ? rows_workspace<1>() : rows_workspace<2>();
    return paged_tiles_workspace(*cfg, *cache);
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

    PagedArgs a{};
    a.nseq = c.nseq;
    a.B = c.B;
    a.Hq = c.Hq;
    a.Hkv = cache->Hkv;
    a.G = c.Hq / cache->Hkv;
    while ((1 << a.g_log2) < a.G) a.g_log2++;
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
    a.kb = static_cast<const uint8_t*>(cache->k_block);
    a.vb = static_cast<const uint8_t*>(cache->v_block);
    a.out = static_cast<__nv_bfloat16*>(out);
#ifdef DART_DEBUG
    a.fail_warp = fail_at.warp;
    a.fail_part = fail_at.part;
#endif
    a.plan = static_cast<SharePlan*>(workspace);
    a.parts = static_cast<uint8_t*>(workspace) + sizeof(SharePlan);
    a.status = status;
    a.sl2 = static_cast<float>(static_cast<double>(c.scale) * 1.4426950408889634);
    a.turns = rope_turns(c.rope_theta);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!few_rows(c, *cache)) return launch_paged_tiles(a, *cache, static_cast<uint8_t*>(workspace), std::min(sms, kMaxSms), st);
    const int ctas = std::min(sms, kMaxSms);
    const bool eight = (c.B + 1) * a.G <= 8;
    if (cache->dtype == DART_KV_E2M1) return eight ? launch_rows<DART_KV_E2M1, 1>(a, *cache, ctas, st) : launch_rows<DART_KV_E2M1, 2>(a, *cache, ctas, st);
    if (cache->dtype == DART_KV_E4M3) return eight ? launch_rows<DART_KV_E4M3, 1>(a, *cache, ctas, st) : launch_rows<DART_KV_E4M3, 2>(a, *cache, ctas, st);
    return eight ? launch_rows<DART_KV_BF16, 1>(a, *cache, ctas, st) : launch_rows<DART_KV_BF16, 2>(a, *cache, ctas, st);
}

}  // extern "C"

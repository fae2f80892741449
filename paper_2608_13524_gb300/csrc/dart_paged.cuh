// What the two kernels of the paged attention share: arguments, and the even
// division of a list of work over shares (a unit's place in the list is known
// to everyone, so is who holds which part of it).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>

#include "../../include/dart_cache.h"
#include "dart_cache.cuh"

namespace dart {

constexpr int kMaxSms = 160, kMaxShares = 12 * kMaxSms;  // shares are counted by SMs; the workspace has room for this many

// Where the shares of a call begin, for the kernel that joins split units:
// places[i] = sequence, unit, place in the unit, places of the unit that are
// work; nodes[i]: nodes of the sequence.
struct SharePlan {
    int count, pad[3];
    int4 places[kMaxShares];
    int nodes[kMaxShares];
};

struct PagedArgs {
    int nseq, B, Hq, Hkv, G, g_log2, max_pages, page_log2, num_pages, mw;
    int unit_cost;  // (tiles) what a unit costs beside its tiles, in tiles
    long long pool_rows;
    const int32_t *table, *lens, *depths, *n_nodes;
    const uint64_t* mask;
    const __nv_bfloat16 *q, *k, *v;
    long long q_stride, k_stride, v_stride;
    const float *ks, *vs;
    const uint8_t *kb, *vb;  // block scales (e2m1)
    __nv_bfloat16* out;
    void* parts;  // partial results, two per share: of the unit begun before it, of the unit that goes on after it
    SharePlan* plan;
    int* status;
    float sl2;  // scale * log2(e)
    RopeTurns turns;
    // Debug builds: whether the last wait of a softmax warp's part is to count as failed (dart_test_paged_wait).
#ifdef DART_DEBUG
    int fail_warp, fail_part;
    __device__ __forceinline__ bool test_wait_fails(int warp, int part) const { return warp == fail_warp && part == fail_part; }
#else
    __device__ __forceinline__ bool test_wait_fails(int, int) const { return false; }
#endif
};

__device__ __forceinline__ int seq_len(const PagedArgs& a, int s) {
    const long long most = static_cast<long long>(a.max_pages) << a.page_log2;
    return static_cast<int>(min(max(static_cast<long long>(__ldcg(a.lens + s)), 0ll), most));
}
__device__ __forceinline__ int seq_nodes(const PagedArgs& a, int s) {
    return a.B > 0 ? min(max(__ldcg(a.n_nodes + s), 0), a.B) : 0;
}

// A list of length `all` in `count` shares of all / count places, the first
// all % count of them one longer.
struct Shares {
    long long each;
    int more, count;
    __device__ __forceinline__ Shares(long long all, int most, int least) {
        count = static_cast<int>(min(static_cast<long long>(most), (all + least - 1) / least));
        if (all < (1ll << 32)) {  // (a 64-bit division takes long)
            const uint32_t q = static_cast<uint32_t>(all) / static_cast<uint32_t>(count);
            each = q;
            more = static_cast<int>(static_cast<uint32_t>(all) - q * static_cast<uint32_t>(count));
        } else {
            each = all / count;
            more = static_cast<int>(all - each * count);
        }
    }
    __device__ __forceinline__ long long begin(int i) const { return each * i + min(i, more); }
    __device__ __forceinline__ int length(int i) const { return static_cast<int>(each) + (i < more); }
};

// x / d of a place in a sequence's part of the list.
__device__ __forceinline__ int place_div(long long x, int d) {
    return x < (1ll << 32) ? static_cast<int>(static_cast<uint32_t>(x) / static_cast<uint32_t>(d)) : static_cast<int>(x / d);
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Byte offset of 16-byte piece `piece` of a row in a tile of 128-byte rows, of 64-byte rows.
__device__ __forceinline__ uint32_t swz(int row, int piece) {
    return static_cast<uint32_t>(row * 128 + ((piece ^ (row & 7)) << 4));
}
__device__ __forceinline__ uint32_t swz64(int row, int piece) {
    return static_cast<uint32_t>(row * 64 + ((piece ^ ((row >> 1) & 3)) << 4));
}

// The same of a row of a tile in shared memory: by one thread, and of e4m3 codes by a warp.
template <int kType>
__device__ __forceinline__ bool row_in_use(const uint8_t* tile, const uint8_t* blocks, int row) {
    if (kType == DART_KV_E2M1) return e2m1_in_use(*reinterpret_cast<const uint2*>(blocks + row * kBlocks));
    uint32_t any = 0;
#pragma unroll
    for (int c = 0; c < 8; c++) any |= e4m3_bits(*reinterpret_cast<const uint4*>(tile + swz(row, c)));
    return any != 0u;
}
__device__ __forceinline__ bool e4m3_row_in_use(const uint8_t* tile, int row, int lane) {
    return __any_sync(kFull, (*reinterpret_cast<const uint32_t*>(tile + row * kHeadDim + 4 * lane) & 0x7F7F7F7Fu) != 0u);
}

bool valid_cache(const dart_kv_cache* c);
bool valid_cache_pointers(const dart_kv_cache* c);
// Rows of dh elements of type DART_KV_* (the whole pool) in boxes of box_rows rows
// by 128 bytes (e2m1: 64, a whole row), swizzled over as many.
bool encode_rows(CUtensorMap* m, const void* base, long long rows, int type, int box_rows);

// 128-row tiles on the tensor-memory path (dart_paged_tiles.cu).
size_t paged_tiles_workspace(const dart_paged_attn_config& c, const dart_kv_cache& cache);
bool paged_tiles_prepare_device();  // kernel attributes, once per device
int launch_paged_tiles(PagedArgs a, const dart_kv_cache& cache, uint8_t* workspace, int sms, cudaStream_t st);

}  // namespace dart

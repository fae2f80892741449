// Which branch of the draft tree the target's probabilities keep.  Contract:
// include/dart_verify.h.
//
// One cluster of 8 or 16 CTAs walks the tree of a sequence, a row of logits at
// a time: a row's sum of exponentials is needed only if the walk comes there
// (three or four of a few hundred rows), so the walk reads what it cannot do
// without instead of every row of the tree.  Each CTA takes its part of the
// row, the warps' maxima and sums are exchanged through distributed shared
// memory, and every warp takes the same decision from them: one cluster
// barrier per step.  The walk is a chain of dependent rows, bound by latency:
// a step loads its vectors into registers before anything else, has the rows
// of the first children fetched into L2 while its own sums are made, and the
// noise, which only the last row wants, is copied to shared memory meanwhile.
// Measured, V = 151936, bf16, mean over 16 inputs: 18.4 us for walks of 3.5 rows, 38.4
// for eight of which the longest has 8.2, so 4.3 us a row (3.4 where it is in L2: its
// share 0.8, the sums and the two merges, a cluster barrier, the decision) and 3.4
// beside the rows; V = 4096 greedily 10.5 us for 2.8 rows.  2 MB of rows and noise at
// 0.1 TB/s, so bandwidth is not in question.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cfloat>
#include <cmath>
#include <cstddef>
#include <cstdint>
#include <type_traits>

#include "../../include/dart.h"
#include "../../include/dart_verify.h"
#include "dart_device.cuh"
#include "dart_kernels.h"

namespace dart {
namespace {

constexpr int kVerifyThreads = 512;
constexpr int kVerifyWarps = kVerifyThreads / 32;
constexpr int kMaxNodes = 1024;
constexpr int kNodesPerThread = kMaxNodes / kVerifyThreads;
constexpr int kHeld = 4;            // vectors of a row that a thread holds in registers
constexpr int kFetched = 4;         // children whose rows are fetched ahead
constexpr float kLeastLog2 = -126.0f;  // of exp((z - m) / T): below it a token is as good as masked
constexpr int kNoise = 20480;       // noise in shared memory (80 KB): the shares of V <= 163000

struct VerifyArgs {
    int B, V;
    long long ld;
    float T, unit, inv_t;  // temperature, the softmax's (1 for T = 0), its reciprocal
    const void* logits;
    const int32_t *tokens, *parents, *n_nodes;
    const float *u, *noise;
    int32_t *n_rows, *rows, *out_tokens;
    float* logp;
};

// NaN counts as -inf (fmaxf takes the number), +inf as the largest number of the logits' type
// (a bf16 one, too: single elements and vectors have to agree).
constexpr float kBf16Max = 3.38953138925153547590470800371487866880e38f;  // 0x7F7F
__device__ __forceinline__ float clean(float z, float most) { return fminf(fmaxf(z, -INFINITY), most); }
__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float fast_log2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void fetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

template <typename T>
__device__ __forceinline__ float load_logit(const T* row, int i);
template <>
__device__ __forceinline__ float load_logit<float>(const float* row, int i) {
    return clean(ld_plain(row + i), FLT_MAX);
}
template <>
__device__ __forceinline__ float load_logit<__nv_bfloat16>(const __nv_bfloat16* row, int i) {
    return clean(__bfloat162float(ld_plain(row + i)), kBf16Max);
}

// The logits of one 16-byte vector: cleaned words, their values, and the values'
// maximum (bf16: two at a time).
template <typename T>
struct Vec;
template <>
struct Vec<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ uint4 clean4(const uint4& w) {
        auto one = [](uint32_t x) { return __float_as_uint(clean(__uint_as_float(x), FLT_MAX)); };
        return make_uint4(one(w.x), one(w.y), one(w.z), one(w.w));
    }
    static __device__ __forceinline__ void get(const uint4& w, float (&z)[4]) {
        z[0] = __uint_as_float(w.x);
        z[1] = __uint_as_float(w.y);
        z[2] = __uint_as_float(w.z);
        z[3] = __uint_as_float(w.w);
    }
    static __device__ __forceinline__ float top(const uint4& w) {
        return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
    }
};
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int n = 8;
    static __device__ __forceinline__ uint32_t clean2(uint32_t w) {
        const __nv_bfloat162 low = __halves2bfloat162(__ushort_as_bfloat16(0xFF80), __ushort_as_bfloat16(0xFF80));   // -inf
        const __nv_bfloat162 high = __halves2bfloat162(__ushort_as_bfloat16(0x7F7F), __ushort_as_bfloat16(0x7F7F));  // kBf16Max
        const __nv_bfloat162 r = __hmin2(__hmax2(*reinterpret_cast<const __nv_bfloat162*>(&w), low), high);
        return *reinterpret_cast<const uint32_t*>(&r);
    }
    static __device__ __forceinline__ uint4 clean4(const uint4& w) {
        return make_uint4(clean2(w.x), clean2(w.y), clean2(w.z), clean2(w.w));
    }
    static __device__ __forceinline__ void get(const uint4& w, float (&z)[8]) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; e++) {
            z[2 * e] = __uint_as_float(u[e] << 16);
            z[2 * e + 1] = __uint_as_float(u[e] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ float top(const uint4& w) {
        auto two = [](uint32_t x) { return *reinterpret_cast<const __nv_bfloat162*>(&x); };
        const __nv_bfloat162 r = __hmax2(__hmax2(two(w.x), two(w.y)), __hmax2(two(w.z), two(w.w)));
        return fmaxf(__low2float(r), __high2float(r));
    }
};

// A row's share of this CTA: 16-byte vectors [v0, v1) from element `first`
// on, and, for the first CTA, the elements before and after all vectors.
struct Share {
    int first, v0, v1, tail;  // (tail: first element after the vectors)
};
template <typename T, int kCtas>
__device__ __forceinline__ Share share_of(const T* row, int V, int rank) {
    Share s;
    const int mis = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
    s.first = min(V, mis ? Vec<T>::n - mis : 0);
    const int nv = (V - s.first) / Vec<T>::n;
    s.v0 = static_cast<int>(static_cast<long long>(nv) * rank / kCtas);
    s.v1 = static_cast<int>(static_cast<long long>(nv) * (rank + 1) / kCtas);
    s.tail = s.first + nv * Vec<T>::n;
    return s;
}

// The first kHeld vectors of this thread; what is not there is -inf.
template <typename T>
__device__ __forceinline__ void hold(const T* row, const Share& s, uint4 (&held)[kHeld]) {
    const uint4* vec = reinterpret_cast<const uint4*>(row + s.first);
    const uint32_t none = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
#pragma unroll
    for (int q = 0; q < kHeld; q++) {
        const int v = s.v0 + threadIdx.x + q * kVerifyThreads;
        held[q] = v < s.v1 ? ld_plain(vec + v) : make_uint4(none, none, none, none);
    }
}
// The element that this thread has beside vectors, -1 if none.
__device__ __forceinline__ int odd_one(const Share& s, int V, int rank) {
    const int i = threadIdx.x;
    if (rank != 0 || i >= s.first + V - s.tail) return -1;
    return i < s.first ? i : s.tail + i - s.first;
}

struct alignas(16) RowStat {  // of a row, or of a part of it (sent as one 16-byte store)
    float m, sum;  // largest logit, sum of exp((z - m) / T)
    int arg, pad;  // the lowest token that has it
};
static_assert(sizeof(RowStat) == 16, "one 16-byte store");

// All lanes' parts into one, the same in every lane.
__device__ __forceinline__ RowStat warp_merge_stat(const RowStat& a, float c) {
    RowStat r;
    r.m = f32_unord(__reduce_max_sync(kFull, f32_ord(a.m)));
    float sum = r.m == -INFINITY ? 0.0f : a.sum * fast_exp2((a.m - r.m) * c);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
    r.sum = sum;
    r.arg = __reduce_min_sync(kFull, a.m == r.m && r.m != -INFINITY ? a.arg : 0x7FFFFFFF);
    r.pad = 0;
    return r;
}
__device__ __forceinline__ void st_cluster_v4(uint32_t local, uint32_t rank, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(mapa_u32(local, rank)), "r"(a), "r"(b), "r"(c), "r"(d)
                 : "memory");
}

struct Kids {  // children of a row, ascending
    int node[kMaxNodes], token[kMaxNodes];
    float z[kMaxNodes], e[kMaxNodes];  // logit; exp((z - m) / T), -1 for a repeated token (more than 32 children)
};

template <int kCtas>
struct VerifySmem {
    RowStat peer[2][kCtas * kVerifyWarps];  // (by the parity of the exchange)
    int parent[kMaxNodes], token[kMaxNodes];
    Kids kids[2];                  // (by the parity of the step: a warp may still read the step before)
    int count[2][kVerifyWarps];
    uint32_t child[kVerifyThreads];  // bit n q + e: element e of the thread's held vector q is a child's token
    float noise[];                   // of the share's first kNoise elements
};

// The whole cluster's merge of one RowStat per thread; every thread gets it.
template <int kCtas>
__device__ __forceinline__ RowStat cluster_merge(VerifySmem<kCtas>& sm, const RowStat& a, int rank, int parity, float c) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const RowStat w = warp_merge_stat(a, c);
    if (lane < kCtas)
        st_cluster_v4(smem_u32(&sm.peer[parity][rank * kVerifyWarps + warp]), lane, __float_as_uint(w.m), __float_as_uint(w.sum),
                      static_cast<uint32_t>(w.arg), 0u);
    __syncwarp();
    cluster_sync_all();
    RowStat all[kCtas * kVerifyWarps / 32];
    RowStat r{-INFINITY, 0.0f, 0x7FFFFFFF, 0};
#pragma unroll
    for (int i = 0; i < kCtas * kVerifyWarps / 32; i++) {
        all[i] = sm.peer[parity][32 * i + lane];
        r.m = fmaxf(r.m, all[i].m);
    }
    if (r.m != -INFINITY)
#pragma unroll
        for (int i = 0; i < kCtas * kVerifyWarps / 32; i++) {
            r.sum += all[i].sum * fast_exp2((all[i].m - r.m) * c);
            if (all[i].m == r.m) r.arg = min(r.arg, all[i].arg);
        }
    return warp_merge_stat(r, c);
}

template <typename T, int kCtas>
__global__ void __launch_bounds__(kVerifyThreads, 1) verify_tree_kernel(const VerifyArgs a) {
    extern __shared__ __align__(16) uint8_t verify_smem[];
    VerifySmem<kCtas>& sm = *reinterpret_cast<VerifySmem<kCtas>*>(verify_smem);
    constexpr int n = Vec<T>::n;
    pdl_trigger();
    const int rank = static_cast<int>(cluster_ctarank()), s = blockIdx.x / kCtas;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int R = a.B + 1;
    const T* base = static_cast<const T*>(a.logits) + static_cast<long long>(s) * R * a.ld;
    const float* noise = a.noise + static_cast<long long>(s) * a.V;
    const bool sampling = a.T > 0.0f;
    const float c = a.inv_t * 1.4426950408889634f;
    cluster_started_arrive();
    sm.child[tid] = 0;
    pdl_wait();
    int row = 0;
    Share share = share_of<T, kCtas>(base, a.V, rank);
    uint4 held[kHeld];
    hold(base, share, held);
    float u = sampling ? ld_plain(a.u + static_cast<long long>(s) * R) : 0.0f;
    const int nn = min(max(ld_plain(a.n_nodes + s), 0), a.B);
    for (int i = tid; i < nn; i += kVerifyThreads) {
        const int p = ld_plain(a.parents + static_cast<long long>(s) * a.B + i), t = ld_plain(a.tokens + static_cast<long long>(s) * a.B + i);
        // a child comes after its parent, which ends every walk
        sm.parent[i] = p >= -1 && p < i && t >= 0 && t < a.V ? p + 1 : -1;
        sm.token[i] = t;
    }
    // noise of the tokens [noise0, noise0 + noise_n) in shared memory: where the share's
    // vectors lie, give or take what another row's alignment moves them by
    const int noise0 = max(0, share.first + share.v0 * n - n), noise_n = min(min(kNoise, (share.v1 - share.v0 + 3) * n), a.V - noise0);
    if (sampling)
        for (int i = tid; i < noise_n; i += kVerifyThreads)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(sm.noise + i)), "l"(noise + noise0 + i) : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");
    __syncthreads();
    cluster_started_wait();  // the peers' shared memory may be written from here on

    int parity = 0;  // of the exchange
    for (int step = 0;; step++) {
        const T* z_row = base + static_cast<long long>(row) * a.ld;
        Kids& kids = sm.kids[step & 1];
        // the row's children in ascending order
        int mine[kNodesPerThread], n_mine = 0, before = 0, in_warp = 0;
#pragma unroll
        for (int q = 0; q < kNodesPerThread; q++) {
            const int i = tid * kNodesPerThread + q;
            const bool is = i < nn && sm.parent[i] == row;
            const unsigned ball = __ballot_sync(kFull, is);
            mine[q] = is ? n_mine : -1;
            n_mine += is;
            before += __popc(ball & ((1u << lane) - 1u));
            in_warp += __popc(ball);
        }
        if (lane == 0) sm.count[step & 1][warp] = in_warp;
        __syncthreads();
        int nk = lane < kVerifyWarps ? sm.count[step & 1][lane] : 0;
        before += __reduce_add_sync(kFull, lane < warp ? nk : 0);
        nk = __reduce_add_sync(kFull, nk);
        float mine_z[kNodesPerThread];
#pragma unroll
        for (int q = 0; q < kNodesPerThread; q++)
            if (mine[q] >= 0) {
                const int i = tid * kNodesPerThread + q, t = sm.token[i], at = before + mine[q];
                mine_z[q] = load_logit(z_row, t);  // (stored below, when it is there)
                kids.node[at] = i;
                kids.token[at] = t;
            }

        // the row's maximum, sum of exponentials and best token: this thread's
        const uint4* vec = reinterpret_cast<const uint4*>(z_row + share.first);
        const int v_more = share.v0 + tid + kHeld * kVerifyThreads, odd = odd_one(share, a.V, rank);
        const float odd_z = odd >= 0 ? load_logit(z_row, odd) : -INFINITY;
        RowStat st{odd_z, 0.0f, odd, 0};
#pragma unroll
        for (int q = 0; q < kHeld; q++) {
            held[q] = Vec<T>::clean4(held[q]);
            st.m = fmaxf(st.m, Vec<T>::top(held[q]));
        }
        for (int v = v_more; v < share.v1; v += kVerifyThreads) st.m = fmaxf(st.m, Vec<T>::top(Vec<T>::clean4(ld_plain(vec + v))));
        if (st.m != -INFINITY) {
            auto add = [&](const uint4& w) {
                float z[n], x = 0.0f;
                Vec<T>::get(w, z);
#pragma unroll
                for (int e = 0; e < n; e++) x += fast_exp2((z[e] - st.m) * c);
                st.sum += x;
            };
            if (odd >= 0) st.sum += fast_exp2((odd_z - st.m) * c);
#pragma unroll
            for (int q = 0; q < kHeld; q++) add(held[q]);
            for (int v = v_more; v < share.v1; v += kVerifyThreads) add(Vec<T>::clean4(ld_plain(vec + v)));
        }
        if (!sampling && __any_sync(kFull, st.m != -INFINITY)) {
            const float top = f32_unord(__reduce_max_sync(kFull, f32_ord(st.m)));
            if (st.m == top && top != -INFINITY) {  // (few lanes)
                st.arg = odd_z == top ? odd : 0x7FFFFFFF;
                auto seek = [&](const uint4& w, int v) {
                    float z[n];
                    Vec<T>::get(w, z);
#pragma unroll
                    for (int e = n - 1; e >= 0; e--)
                        if (z[e] == top) st.arg = min(st.arg, share.first + v * n + e);
                };
#pragma unroll
                for (int q = 0; q < kHeld; q++) seek(held[q], share.v0 + tid + q * kVerifyThreads);
                for (int v = v_more; v < share.v1; v += kVerifyThreads) seek(Vec<T>::clean4(ld_plain(vec + v)), v);
            }
        }
#pragma unroll
        for (int q = 0; q < kNodesPerThread; q++)
            if (mine[q] >= 0) kids.z[before + mine[q]] = mine_z[q];
        __syncthreads();
        {  // rows that may be next: four warps each
            const int k = warp % kFetched;
            if (k < nk) {
                const T* r = base + static_cast<long long>(kids.node[k] + 1) * a.ld;
                const Share sh = share_of<T, kCtas>(r, a.V, rank);
                const char* lo = reinterpret_cast<const char*>(r + sh.first) + static_cast<long long>(sh.v0) * 16;
                const int bytes = (sh.v1 - sh.v0) * 16;
                for (int i = ((warp / kFetched) * 32 + lane) * 128; i < bytes; i += kVerifyThreads / kFetched * 128) fetch_l2(lo + i);
            }
        }
        st = cluster_merge<kCtas>(sm, st, rank, parity, c);
        parity ^= 1;
        const float m = st.m == -INFINITY ? 0.0f : st.m;
        const float total = st.sum;
        int tok = !sampling && st.m != -INFINITY ? st.arg : -1;

        // the decision, the same in every warp: the child that is kept, else (T > 0)
        // the last one with a probability
        int next = -1, last = -1;
        const float goal = u * total;
        if (nk > 32) {  // (repeated tokens are looked for by all threads)
            for (int k = tid; k < nk; k += kVerifyThreads) {
                bool again = false;
                const int t = kids.token[k];
                for (int j = 0; j < k; j++) again |= kids.token[j] == t;
                kids.e[k] = again ? -1.0f : expf((kids.z[k] - m) * a.inv_t);
            }
            __syncthreads();
        }
        float run = 0.0f;
        for (int k0 = 0; k0 < nk && next < 0; k0 += 32) {
            const int k = k0 + lane, t = k < nk ? kids.token[k] : -1 - lane;
            float e = -1.0f;
            if (nk > 32) {
                if (k < nk) e = kids.e[k];
            } else {
                const unsigned same = __match_any_sync(kFull, t);
                if (k < nk && !(same & ((1u << lane) - 1u))) e = expf((kids.z[k] - m) * a.inv_t);
            }
            if (sampling) {
                const unsigned pos = __ballot_sync(kFull, e > 0.0f);
                if (pos) last = k0 + 31 - __clz(pos);
                float x = fmaxf(e, 0.0f);
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const float y = __shfl_up_sync(kFull, x, o);
                    if (lane >= o) x += y;
                }
                x += run;
                // (e: the lanes' sums are rounded each in its own order, so one without a share
                // of its own may lie above its neighbour's)
                const unsigned hit = __ballot_sync(kFull, e > 0.0f && goal < x);
                if (hit) next = k0 + __ffs(hit) - 1;
                run = __shfl_sync(kFull, x, 31);
            } else {
                const unsigned hit = __ballot_sync(kFull, e >= 0.0f && t == tok);
                if (hit) next = k0 + __ffs(hit) - 1;
            }
        }

        if (next < 0 && sampling) {
            // the largest p / e among the tokens of no child
            for (int k = tid; k < nk; k += kVerifyThreads) {
                const int at = kids.token[k] - share.first, v = at / n - share.v0;
                if (at >= 0 && v >= 0 && v < min(share.v1 - share.v0, kHeld * kVerifyThreads))
                    atomicOr(&sm.child[v % kVerifyThreads], 1u << ((v / kVerifyThreads) * n + at % n));
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncthreads();
            const uint32_t child = sm.child[tid];
            RowStat w{-INFINITY, 0.0f, 0x7FFFFFFF, 0};
            const float least = m + kLeastLog2 / c;
            auto offer = [&](float z, float e, int t) {  // (tokens of a thread are not in ascending order only at the odd ones)
                const float x = (z - m) * c - fast_log2(e);
                if (z >= least && (x > w.m || (x == w.m && t < w.arg))) {
                    w.m = x;
                    w.arg = t;
                }
            };
            auto is_child = [&](int t) {
                bool yes = false;
                for (int k = 0; k < nk; k++) yes |= kids.token[k] == t;
                return yes;
            };
#pragma unroll
            for (int q = 0; q < kHeld; q++) {
                const int v = share.v0 + tid + q * kVerifyThreads, t0 = share.first + v * n;
                if (v < share.v1) {
                    float z[n];
                    Vec<T>::get(held[q], z);
#pragma unroll
                    for (int e = 0; e < n; e++) {
                        const int i = t0 + e - noise0;
                        const float x = i >= 0 && i < noise_n ? sm.noise[i] : ld_plain(noise + t0 + e);
                        if (!((child >> (q * n + e)) & 1u)) offer(z[e], x, t0 + e);
                    }
                }
            }
            for (int v = v_more; v < share.v1; v += kVerifyThreads) {
                float z[n];
                Vec<T>::get(Vec<T>::clean4(ld_plain(vec + v)), z);
#pragma unroll
                for (int e = 0; e < n; e++) {
                    const int t = share.first + v * n + e;
                    if (!is_child(t)) offer(z[e], ld_plain(noise + t), t);
                }
            }
            if (odd >= 0 && !is_child(odd)) offer(odd_z, ld_plain(noise + odd), odd);
            w = cluster_merge<kCtas>(sm, w, rank, parity, 0.0f);
            parity ^= 1;
            if (w.m != -INFINITY)
                tok = w.arg;
            else
                next = last;  // nothing with a probability is left beside the children
            if (next >= 0) {
                sm.child[tid] = 0;
                __syncthreads();
            }
        }
        const bool stop = next < 0;
        const int here = row;
        float z_tok = -INFINITY;
        if (!stop) {
            tok = kids.token[next];
            z_tok = kids.z[next];
            row = kids.node[next] + 1;
            share = share_of<T, kCtas>(base + static_cast<long long>(row) * a.ld, a.V, rank);
            hold(base + static_cast<long long>(row) * a.ld, share, held);
            if (sampling) u = ld_plain(a.u + static_cast<long long>(s) * R + row);
        }
        if (rank == kCtas - 1 && warp == kVerifyWarps - 1 && lane == 0) {
            const long long o = static_cast<long long>(s) * R + step;
            if (stop && tok >= 0) z_tok = load_logit(z_row, tok);
            a.rows[o] = here;
            a.out_tokens[o] = tok;
            a.logp[o] = tok >= 0 ? (z_tok - m) / a.unit - logf(total) : 0.0f;
            if (stop) a.n_rows[s] = step + 1;
        }
        if (stop) {
            if (rank == 0)
                for (int i = step + 1 + tid; i < R; i += kVerifyThreads) {
                    a.rows[static_cast<long long>(s) * R + i] = -1;
                    a.out_tokens[static_cast<long long>(s) * R + i] = -1;
                    a.logp[static_cast<long long>(s) * R + i] = 0.0f;
                }
            break;
        }
    }
}

// Clusters of kCtas CTAs of this kernel that fit the current device at once
// (0: an error); the kernel's attributes are set on the first call per device.
template <typename T, int kCtas>
int clusters_at_once(int dev) {
    static std::atomic<int> known[64];
    if (dev < 0 || dev >= 64) return 0;
    const int k = known[dev].load(std::memory_order_acquire);
    if (k) return k;
    constexpr int bytes = sizeof(VerifySmem<kCtas>) + kNoise * 4;
    auto kernel = verify_tree_kernel<T, kCtas>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return 0;
    if (kCtas > 8 && cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kCtas);
    cfg.blockDim = dim3(kVerifyThreads);
    cfg.dynamicSmemBytes = bytes;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kCtas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int most = 0;
    if (cudaOccupancyMaxActiveClusters(&most, kernel, &cfg) != cudaSuccess || most < 1) return 0;
    known[dev].store(most, std::memory_order_release);
    return most;
}

template <typename T>
int launch_verify(const VerifyArgs& a, int nseq, int dev, cudaStream_t st) {
    // 16 CTAs a sequence up to half as many again as run at once (the last begin when
    // the first end), else 8.  V = 151936, 16 CTAs / 8: one sequence 27.6 / 31.1 us,
    // four 13.7 / 16.9 (short walks), eight 31.2 / 36.2, ten 27.7 / 32.0, fourteen 42.7 /
    // 32.0, 64 134 / 91; V = 32000, eight 34.3 / 33.4.
    const int large = clusters_at_once<T, 16>(dev), small = clusters_at_once<T, 8>(dev);
    if (!large || !small) return DART_ERR_CUDA;
    auto go = [&](auto ctas) {
        constexpr int kCtas = decltype(ctas)::value;
        return launch_pdl_cluster(verify_tree_kernel<T, kCtas>, dim3(static_cast<unsigned>(nseq) * kCtas), dim3(kVerifyThreads),
                                  sizeof(VerifySmem<kCtas>) + kNoise * 4, st, kCtas, a);
    };
    const cudaError_t e = nseq <= large + large / 2 ? go(std::integral_constant<int, 16>{}) : go(std::integral_constant<int, 8>{});
    return e == cudaSuccess ? DART_OK : DART_ERR_CUDA;
}

}  // namespace
}  // namespace dart

using namespace dart;

extern "C" int dart_verify_tree(const dart_verify_config* cfg, const void* logits, const int32_t* tokens,
                                const int32_t* parents, const int32_t* n_nodes, const float* u, const float* noise,
                                int32_t* n_rows, int32_t* rows, int32_t* out_tokens, float* logp, void* stream) {
    if (!cfg || cfg->nseq < 1 || cfg->B < 1 || cfg->B > kMaxNodes || cfg->V < 1 || cfg->V >= (1 << 24)) return DART_ERR_INVALID;
    if ((cfg->dtype != DART_F32 && cfg->dtype != DART_BF16) || cfg->ld < cfg->V) return DART_ERR_INVALID;
    const float T = cfg->temperature;  // (below 1e-6 a difference of logits over T may leave the floats)
    if (!std::isfinite(T) || (T != 0.0f && T < 1e-6f)) return DART_ERR_INVALID;
    if (cfg->nseq > 2147483647 / 16) return DART_ERR_INVALID;
    auto al4 = [](const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 3u) == 0; };
    if (!logits || (reinterpret_cast<uintptr_t>(logits) & 15u)) return DART_ERR_INVALID;
    if (!al4(tokens) || !al4(parents) || !al4(n_nodes) || !al4(n_rows) || !al4(rows) || !al4(out_tokens) || !al4(logp))
        return DART_ERR_INVALID;
    if (T > 0.0f && (!al4(u) || !al4(noise))) return DART_ERR_INVALID;
    int dev = 0, major = 0, minor = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess)
        return DART_ERR_CUDA;
    if (major != 10 || minor != 3) return DART_ERR_UNSUPPORTED;
    VerifyArgs a{};
    a.B = cfg->B;
    a.V = cfg->V;
    a.ld = cfg->ld;
    a.T = T;
    a.unit = T > 0.0f ? T : 1.0f;
    a.inv_t = 1.0f / a.unit;
    a.logits = logits;
    a.tokens = tokens;
    a.parents = parents;
    a.n_nodes = n_nodes;
    a.u = u;
    a.noise = noise;
    a.n_rows = n_rows;
    a.rows = rows;
    a.out_tokens = out_tokens;
    a.logp = logp;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return cfg->dtype == DART_BF16 ? launch_verify<__nv_bfloat16>(a, cfg->nseq, dev, st) : launch_verify<float>(a, cfg->nseq, dev, st);
}

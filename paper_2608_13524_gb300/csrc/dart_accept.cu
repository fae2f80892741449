// Which branch of the draft tree the target's probabilities keep.  Contract:
// include/dart_verify.h.
//
// One cluster of 8 CTAs walks the tree of a sequence, a row of logits at a
// time: a row's sum of exponentials is needed only if the walk comes there
// (three or four of a few hundred rows), so the walk reads what it cannot do
// without instead of every row of the tree.  Each CTA takes an eighth of the
// row (running maximum and sum per thread, one pass), the eight partial
// results are exchanged through distributed shared memory, and every CTA
// takes the same decision from them: one cluster barrier per step.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cfloat>
#include <cmath>
#include <cstddef>
#include <cstdint>

#include "../../include/dart.h"
#include "../../include/dart_verify.h"
#include "dart_device.cuh"
#include "dart_kernels.h"

namespace dart {
namespace {

constexpr int kVerifyCtas = 8;  // cluster size (portable)
constexpr int kVerifyThreads = 512;
constexpr int kVerifyWarps = kVerifyThreads / 32;
constexpr int kMaxNodes = 1024;
constexpr int kNodesPerThread = kMaxNodes / kVerifyThreads;

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

// NaN counts as -inf, +inf as the largest float.
__device__ __forceinline__ float clean(float z) { return z == z ? fminf(z, FLT_MAX) : -INFINITY; }

template <typename T>
__device__ __forceinline__ float load_logit(const T* row, int i);
template <>
__device__ __forceinline__ float load_logit<float>(const float* row, int i) {
    return clean(__ldg(row + i));
}
template <>
__device__ __forceinline__ float load_logit<__nv_bfloat16>(const __nv_bfloat16* row, int i) {
    return clean(__bfloat162float(__ldg(row + i)));
}

// The logits of one 16-byte vector.
template <typename T>
struct Vec;
template <>
struct Vec<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ void get(const uint4& w, float (&z)[4]) {
        z[0] = clean(__uint_as_float(w.x));
        z[1] = clean(__uint_as_float(w.y));
        z[2] = clean(__uint_as_float(w.z));
        z[3] = clean(__uint_as_float(w.w));
    }
};
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int n = 8;
    static __device__ __forceinline__ void get(const uint4& w, float (&z)[8]) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; e++) {
            z[2 * e] = clean(__uint_as_float(u[e] << 16));
            z[2 * e + 1] = clean(__uint_as_float(u[e] & 0xFFFF0000u));
        }
    }
};

// A row's share of this CTA: 16-byte vectors [v0, v1) from element `first`
// on, and, for the first CTA, the elements before and after all vectors.
struct Share {
    int first, v0, v1, tail;  // (tail: first element after the vectors)
};
template <typename T>
__device__ __forceinline__ Share share_of(const T* row, int V, int rank) {
    Share s;
    const int mis = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
    s.first = min(V, mis ? Vec<T>::n - mis : 0);
    const int nv = (V - s.first) / Vec<T>::n;
    s.v0 = static_cast<int>(static_cast<long long>(nv) * rank / kVerifyCtas);
    s.v1 = static_cast<int>(static_cast<long long>(nv) * (rank + 1) / kVerifyCtas);
    s.tail = s.first + nv * Vec<T>::n;
    return s;
}

// f(token, logit) for every element of the share.
template <typename T, typename F>
__device__ __forceinline__ void for_share(const T* row, int V, const Share& s, int rank, F&& f) {
    constexpr int n = Vec<T>::n, kUnroll = 4;
    const uint4* vec = reinterpret_cast<const uint4*>(row + s.first);
    int v = s.v0 + threadIdx.x;
    for (; v + (kUnroll - 1) * kVerifyThreads < s.v1; v += kUnroll * kVerifyThreads) {
        uint4 w[kUnroll];
#pragma unroll
        for (int q = 0; q < kUnroll; q++) w[q] = __ldg(vec + v + q * kVerifyThreads);
#pragma unroll
        for (int q = 0; q < kUnroll; q++) {
            float z[n];
            Vec<T>::get(w[q], z);
            f(s.first + (v + q * kVerifyThreads) * n, z);
        }
    }
    for (; v < s.v1; v += kVerifyThreads) {
        float z[n];
        Vec<T>::get(__ldg(vec + v), z);
        f(s.first + v * n, z);
    }
    if (rank == 0) {
        const int extra = s.first + (V - s.tail);
        if (static_cast<int>(threadIdx.x) < extra) {
            const int i = static_cast<int>(threadIdx.x) < s.first ? threadIdx.x : s.tail + (threadIdx.x - s.first);
            float z[1] = {load_logit(row, i)};
            f(i, z);
        }
    }
}

struct alignas(16) RowStat {  // of a row, or of a part of it (sent as two 16-byte stores)
    float m, sum;    // largest logit, sum of exp((z - m) / T)
    int finite, pad;  // tokens of finite logit
    uint64_t key;    // largest logit, lowest token
};

static_assert(sizeof(RowStat) == 32 && offsetof(RowStat, key) == 16, "two 16-byte stores");

__device__ __forceinline__ void stat_merge(RowStat& a, const RowStat& b, float c) {
    const float m = fmaxf(a.m, b.m);
    if (m != -INFINITY)
        a.sum = (a.m == -INFINITY ? 0.0f : a.sum * exp2f((a.m - m) * c)) + (b.m == -INFINITY ? 0.0f : b.sum * exp2f((b.m - m) * c));
    a.m = m;
    a.finite += b.finite;
    a.key = a.key > b.key ? a.key : b.key;
}
__device__ __forceinline__ RowStat stat_shfl(const RowStat& a, int o) {
    RowStat b;
    b.m = __shfl_xor_sync(kFull, a.m, o);
    b.sum = __shfl_xor_sync(kFull, a.sum, o);
    b.finite = __shfl_xor_sync(kFull, a.finite, o);
    b.pad = 0;
    b.key = shfl_xor_u64(a.key, o);
    return b;
}
__device__ __forceinline__ void st_cluster_v4(uint32_t local, uint32_t rank, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(mapa_u32(local, rank)), "r"(a), "r"(b), "r"(c), "r"(d)
                 : "memory");
}

struct VerifySmem {
    RowStat peer[2][kVerifyCtas];   // by the parity of the exchange
    RowStat warp[kVerifyWarps];
    int parent[kMaxNodes], token[kMaxNodes];
    int kid[kMaxNodes], kid_token[kMaxNodes];  // children of the present row, ascending
    float kid_z[kMaxNodes], kid_e[kMaxNodes];
    int count[kVerifyWarps + 1];
    int decided, bonus;
};

// The whole cluster's merge of one RowStat per thread; every thread gets it.
__device__ __forceinline__ RowStat cluster_merge(VerifySmem& sm, RowStat a, int rank, int parity, float c) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) stat_merge(a, stat_shfl(a, o), c);
    if (lane == 0) sm.warp[warp] = a;
    __syncthreads();
    if (warp == 0) {
        RowStat b{-INFINITY, 0.0f, 0, 0, 0ull};
        if (lane < kVerifyWarps) b = sm.warp[lane];
#pragma unroll
        for (int o = kVerifyWarps / 2; o > 0; o >>= 1) stat_merge(b, stat_shfl(b, o), c);
        b = RowStat{__shfl_sync(kFull, b.m, 0), __shfl_sync(kFull, b.sum, 0), __shfl_sync(kFull, b.finite, 0), 0, shfl_u64(b.key, 0)};
        if (lane < kVerifyCtas) {
            const uint32_t at = smem_u32(&sm.peer[parity][rank]);
            st_cluster_v4(at, lane, __float_as_uint(b.m), __float_as_uint(b.sum), static_cast<uint32_t>(b.finite), 0u);
            st_cluster_v4(at + 16, lane, static_cast<uint32_t>(b.key), static_cast<uint32_t>(b.key >> 32), 0u, 0u);
        }
        __syncwarp();
    }
    cluster_sync_all();
    RowStat r = sm.peer[parity][0];
    for (int p = 1; p < kVerifyCtas; p++) stat_merge(r, sm.peer[parity][p], c);
    return r;
}

template <typename T>
__global__ void __launch_bounds__(kVerifyThreads, 1) verify_tree_kernel(const VerifyArgs a) {
    __shared__ VerifySmem sm;
    pdl_trigger();
    const int rank = static_cast<int>(cluster_ctarank()), s = blockIdx.x / kVerifyCtas;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int R = a.B + 1;
    cluster_started_arrive();
    pdl_wait();
    const int nn = min(max(__ldg(a.n_nodes + s), 0), a.B);
    const bool sampling = a.T > 0.0f;
    for (int i = tid; i < nn; i += kVerifyThreads) {
        const int p = __ldg(a.parents + static_cast<long long>(s) * a.B + i), t = __ldg(a.tokens + static_cast<long long>(s) * a.B + i);
        // a child comes after its parent, which ends every walk
        sm.parent[i] = p >= -1 && p < i && t >= 0 && t < a.V ? p + 1 : -1;
        sm.token[i] = t;
    }
    const float c = a.inv_t * 1.4426950408889634f;
    const T* base = static_cast<const T*>(a.logits) + static_cast<long long>(s) * R * a.ld;
    __syncthreads();
    cluster_started_wait();  // the peers' shared memory may be written from here on

    int row = 0, step = 0;
    for (;; step++) {
        const T* z_row = base + static_cast<long long>(row) * a.ld;
        const Share share = share_of(z_row, a.V, rank);
        // children of this row in ascending order, and their logits
        int mine[kNodesPerThread], n_mine = 0;
        unsigned ball[kNodesPerThread];
#pragma unroll
        for (int q = 0; q < kNodesPerThread; q++) {
            const int i = tid * kNodesPerThread + q;
            const bool is = i < nn && sm.parent[i] == row;
            ball[q] = __ballot_sync(kFull, is);
            mine[q] = is ? n_mine : -1;
            n_mine += is;
        }
        int before = 0, in_warp = 0;
#pragma unroll
        for (int q = 0; q < kNodesPerThread; q++) {
            before += __popc(ball[q] & ((1u << lane) - 1u));
            in_warp += __popc(ball[q]);
        }
        if (lane == 0) sm.count[warp] = in_warp;
        __syncthreads();
        int nk = 0;
        for (int w = 0; w < kVerifyWarps; w++) {
            if (w < warp) before += sm.count[w];
            nk += sm.count[w];
        }
#pragma unroll
        for (int q = 0; q < kNodesPerThread; q++)
            if (mine[q] >= 0) {
                const int i = tid * kNodesPerThread + q, t = sm.token[i], at = before + mine[q];
                sm.kid[at] = i;
                sm.kid_token[at] = t;
                sm.kid_z[at] = load_logit(z_row, t);
            }

        // the row's maximum, sum of exponentials and best token
        RowStat st{-INFINITY, 0.0f, 0, 0, 0ull};
        for_share(z_row, a.V, share, rank, [&](int tok, auto& z) {
            constexpr int n = sizeof(z) / sizeof(float);
            float mx = z[0];
#pragma unroll
            for (int e = 1; e < n; e++) mx = fmaxf(mx, z[e]);
            if (mx > st.m) {
                st.sum = st.m == -INFINITY ? 0.0f : st.sum * exp2f((st.m - mx) * c);
                st.m = mx;
#pragma unroll
                for (int e = n - 1; e >= 0; e--)
                    if (z[e] == mx) st.key = make_key(mx, static_cast<uint32_t>(tok + e));
            }
            if (st.m != -INFINITY) {
#pragma unroll
                for (int e = 0; e < n; e++) {
                    st.sum += exp2f((z[e] - st.m) * c);
                    st.finite += z[e] > -INFINITY;
                }
            }
        });
        st = cluster_merge(sm, st, rank, step & 1, c);
        const float m = st.m == -INFINITY ? 0.0f : st.m;
        const float total = st.sum;
        const int best = st.key ? static_cast<int>(key_idx(st.key)) : -1;

        // the decision, the same in every CTA
        for (int k = tid; k < nk; k += kVerifyThreads) {
            bool again = false;
            const int t = sm.kid_token[k];
            for (int j = 0; j < k; j++) again |= sm.kid_token[j] == t;
            // a repeated token has no share; -1 marks it
            sm.kid_e[k] = again ? -1.0f : expf((sm.kid_z[k] - m) / a.unit);
        }
        __syncthreads();
        if (warp == 0) {
            int next = -1;
            if (sampling) {
                const float t = __ldg(a.u + static_cast<long long>(s) * R + row) * total;
                float run = 0.0f;
                int last = -1, finite = 0;
                for (int k0 = 0; k0 < nk && next < 0; k0 += 32) {
                    const int k = k0 + lane;
                    const float e = k < nk ? sm.kid_e[k] : -1.0f;
                    finite += __popc(__ballot_sync(kFull, e >= 0.0f && sm.kid_z[min(k, nk - 1)] > -INFINITY));
                    const unsigned pos = __ballot_sync(kFull, e > 0.0f);
                    if (pos) last = k0 + 31 - __clz(pos);
                    float x = fmaxf(e, 0.0f);
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const float y = __shfl_up_sync(kFull, x, o);
                        if (lane >= o) x += y;
                    }
                    x += run;
                    const unsigned hit = __ballot_sync(kFull, k < nk && t < x);
                    if (hit) next = k0 + __ffs(hit) - 1;
                    run = __shfl_sync(kFull, x, 31);
                }
                if (next < 0 && finite == st.finite) next = last;  // nothing is left beside the children
            } else {
                for (int k0 = 0; k0 < nk && next < 0; k0 += 32) {
                    const int k = k0 + lane;
                    const unsigned hit = __ballot_sync(kFull, k < nk && sm.kid_e[k] >= 0.0f && sm.kid_token[k] == best);
                    if (hit) next = k0 + __ffs(hit) - 1;
                }
            }
            if (lane == 0) sm.decided = next;
        }
        __syncthreads();
        const int next = sm.decided;
        const long long o = static_cast<long long>(s) * R + step;
        if (next >= 0) {
            if (rank == 0 && tid == 0) {
                a.rows[o] = row;
                a.out_tokens[o] = sm.kid_token[next];
                a.logp[o] = (sm.kid_z[next] - m) / a.unit - logf(total);
            }
            row = sm.kid[next] + 1;
            __syncthreads();  // the children's arrays are free
            continue;
        }

        int tok = best;
        if (sampling) {
            // the largest p / e among the tokens of no child
            const float* noise = a.noise + static_cast<long long>(s) * a.V;
            float top = -INFINITY;
            int arg = -1;
            for_share(z_row, a.V, share, rank, [&](int t0, auto& z) {
                constexpr int n = sizeof(z) / sizeof(float);
#pragma unroll
                for (int e = 0; e < n; e++) {
                    const float w = (z[e] - m) / a.T - logf(__ldg(noise + t0 + e));
                    if (w > top || (w == top && t0 + e < arg)) {
                        bool child = false;
                        for (int k = 0; k < nk; k++) child |= sm.kid_token[k] == t0 + e;
                        if (!child) {
                            top = w;
                            arg = t0 + e;
                        }
                    }
                }
            });
            RowStat w{-INFINITY, 0.0f, 0, 0, arg >= 0 ? make_key(top, static_cast<uint32_t>(arg)) : 0ull};
            w = cluster_merge(sm, w, rank, (step + 1) & 1, c);
            tok = w.key ? static_cast<int>(key_idx(w.key)) : -1;
        }
        if (rank == 0) {
            if (tid == 0) {
                a.rows[o] = row;
                a.out_tokens[o] = tok;
                a.logp[o] = tok >= 0 ? (load_logit(z_row, tok) - m) / a.unit - logf(total) : 0.0f;
                a.n_rows[s] = step + 1;
            }
            for (int i = step + 1 + tid; i < R; i += kVerifyThreads) {
                a.rows[static_cast<long long>(s) * R + i] = -1;
                a.out_tokens[static_cast<long long>(s) * R + i] = -1;
                a.logp[static_cast<long long>(s) * R + i] = 0.0f;
            }
        }
        break;
    }
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
    if (cfg->nseq > 2147483647 / kVerifyCtas) return DART_ERR_INVALID;
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
    const dim3 grid(static_cast<unsigned>(cfg->nseq) * kVerifyCtas), block(kVerifyThreads);
    const cudaError_t e = cfg->dtype == DART_BF16
                              ? launch_pdl_cluster(verify_tree_kernel<__nv_bfloat16>, grid, block, 0, st, kVerifyCtas, a)
                              : launch_pdl_cluster(verify_tree_kernel<float>, grid, block, 0, st, kVerifyCtas, a);
    return e == cudaSuccess ? DART_OK : DART_ERR_CUDA;
}

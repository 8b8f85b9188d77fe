// Balance of a model's experts over all replicas' tokens: the picks' counts, and the load-balancing loss (with the z loss)
// together with the gradient of the routers' logits.  Both are sums over every replica's rows, the case of paper
// Section 4.1, "Non-elementwise operators".
//
// The gradient needs a token's own row and the counts, which no logit enters, so loss and gradient are one pass: a row is
// read once into the registers of a few lanes and its gradient written from there.
#include <cuda_bf16.h>
#include <math.h>

#include "ws_internal.h"

namespace {

constexpr int kMaxReplicas = 512;
constexpr int kMaxExperts = 1024;
constexpr int kBlock = 256;

// What a launch names travels in its parameters, in a table of the size it needs.
template <int NP>
struct RouterTab {
    const void* in[NP];            // [layers of the launch][replicas] picks or logits
    void* out[NP];                 // ... dlogits
    const unsigned char* valid[NP];// [replicas]
    int tokens[NP];                // [replicas]
    int chunk0[NP];                // [replicas] first chunk of a replica's tokens
};

struct RouterParams {
    int replicas, experts, topk;
    int chunks;                    // chunks of a layer
    int rows;                      // tokens of a chunk
    int layer0;                    // first layer of the launch
};

// The replica that a chunk belongs to.
template <int NP>
__device__ __forceinline__ int replica_of(const RouterTab<NP>& tab, int replicas, int chunk) {
    int lo = 0, hi = replicas - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.chunk0[mid] <= chunk) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// ------------------------------------------------------------------ counts ---
// A CTA counts a chunk in shared memory and adds its counts to the layer's, integers, so in any order.
template <typename I, int NP>
__global__ void __launch_bounds__(kBlock) counts_kernel(const RouterParams P, const __grid_constant__ RouterTab<NP> tab, unsigned long long* counts) {
    __shared__ int hist[kMaxExperts + 1];
    const int layer = blockIdx.y, E = P.experts;
    for (int e = threadIdx.x; e <= E; e += kBlock) hist[e] = 0;
    __syncthreads();
    const int rep = replica_of(tab, P.replicas, blockIdx.x);
    const long long row0 = (long long)(blockIdx.x - tab.chunk0[rep]) * P.rows;
    const int n = (int)min((long long)P.rows, tab.tokens[rep] - row0);
    const unsigned char* valid = tab.valid[rep];
    const I* picks = (const I*)tab.in[layer * P.replicas + rep] + row0 * P.topk;
    for (int i = threadIdx.x; i < n * P.topk; i += kBlock) {
        if (valid && !valid[row0 + i / P.topk]) continue;
        const I e = picks[i];
        if (e >= 0 && e < E) atomicAdd(&hist[(int)e], 1);
    }
    for (int i = threadIdx.x; i < n; i += kBlock)
        if (!valid || valid[row0 + i]) atomicAdd(&hist[E], 1);
    __syncthreads();
    for (int e = threadIdx.x; e <= E; e += kBlock)
        if (hist[e]) atomicAdd(counts + (long long)(P.layer0 + layer) * (E + 1) + e, (unsigned long long)hist[e]);
}

// ----------------------------------------------------------------- balance ---
struct BalanceParams {
    RouterParams r;
    const long long* counts;
    const float* upstream;
    float* loss;
    double2* partials;             // [layers][chunks]
    long long ld, dld;
    double coef, z;
    int accumulate;
    int lanes;                     // lanes of a row, a power of two
};

__device__ __forceinline__ float get(const float* p) { return __ldcs(p); }
__device__ __forceinline__ float get(const __nv_bfloat16* p) {
    return __uint_as_float((unsigned)__ldcs(reinterpret_cast<const unsigned short*>(p)) << 16);
}
__device__ __forceinline__ void put(float* p, float x) { __stcs(p, x); }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) {
    const __nv_bfloat16 b = __float2bfloat16_rn(x);
    __stcs(reinterpret_cast<unsigned short*>(p), *reinterpret_cast<const unsigned short*>(&b));
}
// V consecutive elements: one, or 16 bytes of them
template <typename X, int V>
__device__ __forceinline__ void load_v(const X* p, float* o) {
    if constexpr (V == 1) {
        o[0] = get(p);
    } else if constexpr (sizeof(X) == 4) {
        const float4 v = __ldcs(reinterpret_cast<const float4*>(p));
        o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
    } else {
        const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p));
        const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o[2 * i] = __uint_as_float(w[i] << 16);
            o[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}
template <typename X, int V>
__device__ __forceinline__ void store_v(X* p, const float* x) {
    if constexpr (V == 1) {
        put(p, x[0]);
    } else if constexpr (sizeof(X) == 4) {
        __stcs(reinterpret_cast<float4*>(p), make_float4(x[0], x[1], x[2], x[3]));
    } else {
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const unsigned*>(&b);
        }
        __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
    }
}

// Sums of the layer's two losses from those of its chunks, in the chunks' order.
__device__ __forceinline__ void write_loss(const BalanceParams& P, int layer, double bal, double z, double tokens) {
    const double inv = tokens > 0.0 ? 1.0 / tokens : 0.0;
    P.loss[2 * layer] = (float)(P.coef * P.r.experts * inv * bal);
    P.loss[2 * layer + 1] = P.z == 0.0 ? 0.f : (float)(P.z * inv * z);
}

__device__ __forceinline__ void sum2(double& a, double& b) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
    }
}

// X: the logits' type.  A row lies on P.lanes lanes; lane q holds the C vectors of V elements at (c lanes + q) V.
template <typename X, int V, int C, bool SIG, int NP>
__global__ void __launch_bounds__(kBlock) balance_kernel(const __grid_constant__ BalanceParams P, const __grid_constant__ RouterTab<NP> tab) {
    __shared__ double2 part[kBlock / 32];
    asm volatile("griddepcontrol.launch_dependents;");
    const int E = P.r.experts, G = P.lanes, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int q = lane & (G - 1), sub = lane / G, per_warp = 32 / G;
    const int layer = P.r.layer0 + blockIdx.y;
    const int rep = replica_of(tab, P.r.replicas, blockIdx.x);
    const long long row0 = (long long)(blockIdx.x - tab.chunk0[rep]) * P.r.rows;
    const int n = (int)min((long long)P.r.rows, tab.tokens[rep] - row0);
    const unsigned char* valid = tab.valid[rep];
    const X* in = (const X*)tab.in[blockIdx.y * P.r.replicas + rep];
    X* out = (X*)tab.out[blockIdx.y * P.r.replicas + rep];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const long long* counts = P.counts + (long long)layer * (E + 1);
    const double tokens = (double)counts[E];
    const double inv = tokens > 0.0 ? 1.0 / tokens : 0.0, up = P.upstream ? (double)*P.upstream : 1.0;
    const float slope = (float)(up * P.coef * E * inv), zslope = (float)(2.0 * up * P.z * inv);
    float share[C * V];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = (c * G + q) * V + v;
            share[c * V + v] = e < E ? (float)((double)counts[e] * inv / P.r.topk) : 0.f;
        }
    double bal = 0.0, zsum = 0.0;
    for (int i0 = warp * per_warp; i0 < n; i0 += (kBlock / 32) * per_warp) {
        const int i = i0 + sub;
        const long long row = row0 + i;
        const bool there = i < n, live = there && (!valid || valid[row]);
        float x[C * V], y[C * V];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int e = (c * G + q) * V;
#pragma unroll
            for (int v = 0; v < V; ++v) x[c * V + v] = -INFINITY;
            if (live && e < E) load_v<X, V>(in + row * P.ld + e, x + c * V);
        }
        float top = -INFINITY;
#pragma unroll
        for (int c = 0; c < C * V; ++c) top = fmaxf(top, x[c]);
        for (int o = G >> 1; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        // Softmax: exp(x - top).  Sigmoid scores of a row whose largest logit is below -40 are exp(x) to the last bit of
        // fp32, and only their ratios count: there they are exp(x - top) too, where the scores themselves would vanish.
        const float shift = top > -INFINITY ? top : 0.f;
        float total = 0.f, inner = 0.f;
#pragma unroll
        for (int c = 0; c < C * V; ++c) {
            float s;
            if (!SIG || top < -40.f) {
                s = expf(x[c] - shift);
                if (SIG) y[c] = 1.f;
            } else {
                const float u = expf(-fabsf(x[c])), d = 1.f / (1.f + u);
                s = x[c] >= 0.f ? d : u * d;
                y[c] = x[c] >= 0.f ? u * d : d;
            }
            x[c] = s;
            total += s;
            inner = fmaf(share[c], s, inner);
        }
        for (int o = G >> 1; o > 0; o >>= 1) {
            total += __shfl_xor_sync(0xffffffffu, total, o);
            inner += __shfl_xor_sync(0xffffffffu, inner, o);
        }
        const bool empty = total == 0.f;                  // no expert that the token can pick
        const float scale = empty ? 0.f : 1.f / total;
        inner *= scale;
        const float lse = SIG || empty ? 0.f : shift + logf(total);
        if (live && q == 0) {
            bal += inner;
            zsum += (double)lse * lse;
        }
        if (there && out && (live || !P.accumulate)) {
            const float zl = zslope * lse;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int e = (c * G + q) * V;
                if (e >= E) continue;
                float d[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const int k = c * V + v;
                    const float p = x[k] * scale, g = slope * (share[k] - inner);
                    d[v] = live ? (SIG ? p * g * y[k] : p * (P.z == 0.0 ? g : g + zl)) : 0.f;
                }
                X* at = out + row * P.dld + e;
                if (P.accumulate) {
                    float old[V];
                    load_v<X, V>(at, old);
#pragma unroll
                    for (int v = 0; v < V; ++v) d[v] += old[v];
                }
                store_v<X, V>(at, d);
            }
        }
    }
    if (!P.loss) return;
    sum2(bal, zsum);
    if (lane == 0) part[warp] = make_double2(bal, zsum);
    __syncthreads();
    if (threadIdx.x == 0) {
        bal = zsum = 0.0;
        for (int k = 0; k < kBlock / 32; ++k) {
            bal += part[k].x;
            zsum += part[k].y;
        }
        if (P.r.chunks == 1) write_loss(P, layer, bal, zsum, tokens);
        else P.partials[(long long)layer * P.r.chunks + blockIdx.x] = make_double2(bal, zsum);
    }
}

__global__ void __launch_bounds__(kBlock) balance_loss_kernel(const __grid_constant__ BalanceParams P) {
    __shared__ double2 part[kBlock / 32];
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int layer = blockIdx.x;
    const double2* p = P.partials + (long long)layer * P.r.chunks;
    double bal = 0.0, zsum = 0.0;
    for (int i = threadIdx.x; i < P.r.chunks; i += kBlock) {
        bal += p[i].x;
        zsum += p[i].y;
    }
    sum2(bal, zsum);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = make_double2(bal, zsum);
    __syncthreads();
    if (threadIdx.x == 0) {
        bal = zsum = 0.0;
        for (int k = 0; k < kBlock / 32; ++k) {
            bal += part[k].x;
            zsum += part[k].y;
        }
        write_loss(P, layer, bal, zsum, (double)P.counts[(long long)layer * (P.r.experts + 1) + P.r.experts]);
    }
}

// -------------------------------------------------------------------- host ---
template <typename... KArgs, typename... Args>
void launch(void (*kernel)(KArgs...), dim3 grid, cudaStream_t st, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kBlock);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// The part of a set that both calls read.
ws_status check_set(const ws_router_set* s) {
    if (!s || !s->tokens) return WS_ERR_INVALID_ARG;
    if (s->layers < 1 || s->layers > 65535 || s->replicas < 1 || s->replicas > kMaxReplicas) return WS_ERR_INVALID_ARG;
    if (s->experts < 1 || s->experts > kMaxExperts || s->topk < 1 || s->topk > s->experts) return WS_ERR_INVALID_ARG;
    for (int k = 0; k < s->replicas; ++k)
        if (s->tokens[k] < 0 || s->tokens[k] > 0x7fffffffLL) return WS_ERR_INVALID_ARG;
    return WS_OK;
}
ws_status check_balance(const ws_router_set* s) {
    const ws_status st = check_set(s);
    if (st != WS_OK) return st;
    if (s->dtype != WS_F32 && s->dtype != WS_BF16) return WS_ERR_DTYPE;
    if (s->score != WS_SOFTMAX && s->score != WS_SIGMOID) return WS_ERR_INVALID_ARG;
    if (!s->logits || s->logits_ld < s->experts || (s->dlogits && s->dlogits_ld < s->experts)) return WS_ERR_INVALID_ARG;
    if (s->logits_ld > (1LL << 31) || (s->dlogits && s->dlogits_ld > (1LL << 31))) return WS_ERR_INVALID_ARG;
    return WS_OK;
}

// A layer's tokens in chunks of `rows` that lie in one replica each; at least one chunk.
long long chunks_of(const ws_router_set* s, long long rows) {
    long long n = 0;
    for (int k = 0; k < s->replicas; ++k) n += (s->tokens[k] + rows - 1) / rows;
    return n > 0 ? n : 1;
}
template <int NP>
void fill(RouterTab<NP>& tab, const ws_router_set* s, const void* const* in, void* const* out, int layer0, int layers, int rows) {
    for (int i = 0; i < layers * s->replicas; ++i) {
        tab.in[i] = in ? in[(long long)layer0 * s->replicas + i] : nullptr;
        tab.out[i] = out ? out[(long long)layer0 * s->replicas + i] : nullptr;
    }
    int at = 0;
    for (int k = 0; k < s->replicas; ++k) {
        tab.valid[k] = s->valid ? s->valid[k] : nullptr;
        tab.tokens[k] = (int)s->tokens[k];
        tab.chunk0[k] = at;
        at += (int)((s->tokens[k] + rows - 1) / rows);
    }
}

template <int NP>
void launch_counts(const ws_router_set* s, RouterParams P, int layers, int64_t* counts, cudaStream_t st) {
    RouterTab<NP> tab;
    fill(tab, s, s->picks, nullptr, P.layer0, layers, P.rows);
    const dim3 grid(P.chunks, layers);
    if (s->index_bytes == 4) counts_kernel<int, NP><<<grid, kBlock, 0, st>>>(P, tab, (unsigned long long*)counts);
    else counts_kernel<long long, NP><<<grid, kBlock, 0, st>>>(P, tab, (unsigned long long*)counts);
}

template <typename X, int V, int C, int NP>
void launch_score(const ws_router_set* s, const BalanceParams& P, const RouterTab<NP>& tab, dim3 grid, cudaStream_t st) {
    if (s->score == WS_SIGMOID) launch(balance_kernel<X, V, C, true, NP>, grid, st, P, tab);
    else launch(balance_kernel<X, V, C, false, NP>, grid, st, P, tab);
}
template <typename X, int NP>
void launch_shape(const ws_router_set* s, bool wide, const BalanceParams& P, const RouterTab<NP>& tab, dim3 grid, cudaStream_t st) {
    constexpr int V = 16 / sizeof(X);
    const int v = wide ? V : 1, c = (s->experts + 32 * v - 1) / (32 * v);       // vectors of a lane
    if (wide) {
        if (c <= 1) launch_score<X, V, 1>(s, P, tab, grid, st);
        else if (c <= 2) launch_score<X, V, 2>(s, P, tab, grid, st);
        else if (c <= 4 || V == 8) launch_score<X, V, 4>(s, P, tab, grid, st);
        else if constexpr (V == 4) launch_score<X, V, 8>(s, P, tab, grid, st);
    } else {
        if (c <= 1) launch_score<X, 1, 1>(s, P, tab, grid, st);
        else if (c <= 2) launch_score<X, 1, 2>(s, P, tab, grid, st);
        else if (c <= 4) launch_score<X, 1, 4>(s, P, tab, grid, st);
        else if (c <= 8) launch_score<X, 1, 8>(s, P, tab, grid, st);
        else if (c <= 16) launch_score<X, 1, 16>(s, P, tab, grid, st);
        else launch_score<X, 1, 32>(s, P, tab, grid, st);
    }
}
template <int NP>
void launch_balance(const ws_router_set* s, bool wide, const BalanceParams& P, int layers, cudaStream_t st) {
    RouterTab<NP> tab;
    fill(tab, s, s->logits, s->dlogits, P.r.layer0, layers, P.r.rows);
    const dim3 grid(P.r.chunks, layers);
    if (s->dtype == WS_F32) launch_shape<float>(s, wide, P, tab, grid, st);
    else launch_shape<__nv_bfloat16>(s, wide, P, tab, grid, st);
}

int balance_rows(const ws_router_set* s) {
    // about 64 KB read and written by a CTA
    const int bytes = s->experts * (s->dtype == WS_F32 ? 8 : 4);
    int rows = 2048;
    while (rows > 32 && (long long)rows * bytes > (64 << 10)) rows >>= 1;
    return rows;
}

}  // namespace

extern "C" ws_status ws_router_counts(const ws_router_set* s, int64_t* counts, int32_t accumulate, void* stream) {
    WsRange range_("ws_router_counts");
    const ws_status ok = check_set(s);
    if (ok != WS_OK) return ok;
    if (!counts || !s->picks || (s->index_bytes != 4 && s->index_bytes != 8)) return WS_ERR_INVALID_ARG;
    if (!aligned(counts, 8)) return WS_ERR_ALIGNMENT;
    for (long long i = 0; i < (long long)s->layers * s->replicas; ++i) {
        if (s->tokens[i % s->replicas] == 0) continue;
        if (!s->picks[i]) return WS_ERR_INVALID_ARG;
        if (!aligned(s->picks[i], s->index_bytes)) return WS_ERR_ALIGNMENT;
    }
    cudaStream_t st = (cudaStream_t)stream;
    if (!accumulate) {
        const cudaError_t e = cudaMemsetAsync(counts, 0, sizeof(int64_t) * (size_t)s->layers * (s->experts + 1), st);
        if (e != cudaSuccess) return ws_cuda_fail(e, "ws_router_counts");
    }
    RouterParams P = {};
    P.replicas = s->replicas;
    P.experts = s->experts;
    P.topk = s->topk;
    P.rows = 4096 / s->topk > 256 ? 4096 / s->topk : 256;
    const long long chunks = chunks_of(s, P.rows);
    if (chunks > 0x7fffffffLL) return WS_ERR_TOO_LARGE;
    P.chunks = (int)chunks;
    const int most = kMaxReplicas / s->replicas;
    for (int l = 0; l < s->layers; l += most) {
        const int layers = s->layers - l < most ? s->layers - l : most, np = layers * s->replicas;
        P.layer0 = l;
        if (np <= 16) launch_counts<16>(s, P, layers, counts, st);
        else if (np <= 128) launch_counts<128>(s, P, layers, counts, st);
        else launch_counts<kMaxReplicas>(s, P, layers, counts, st);
        const ws_status r = ws_check_launch("ws_router_counts");
        if (r != WS_OK) return r;
    }
    return WS_OK;
}

extern "C" size_t ws_balance_workspace_bytes(const ws_router_set* s) {
    if (check_balance(s) != WS_OK) return 0;
    return 16 + sizeof(double2) * (size_t)s->layers * (size_t)chunks_of(s, balance_rows(s));
}

extern "C" ws_status ws_balance_loss(const ws_router_set* s, const int64_t* counts, float* loss, double coef, double z_coef,
                                     const float* upstream, int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream) {
    WsRange range_("ws_balance_loss");
    const ws_status ok = check_balance(s);
    if (ok != WS_OK) return ok;
    if (!counts || (!loss && !s->dlogits) || !isfinite(coef) || !isfinite(z_coef)) return WS_ERR_INVALID_ARG;
    if (s->score == WS_SIGMOID && z_coef != 0.0) return WS_ERR_INVALID_ARG;
    if (!aligned(counts, 8) || !aligned(loss, 4) || !aligned(upstream, 4)) return WS_ERR_ALIGNMENT;
    const size_t eb = s->dtype == WS_F32 ? 4 : 2;
    bool wide = s->experts * eb % 16 == 0 && s->logits_ld * eb % 16 == 0 && (!s->dlogits || s->dlogits_ld * eb % 16 == 0);
    for (long long i = 0; i < (long long)s->layers * s->replicas; ++i) {
        if (s->tokens[i % s->replicas] == 0) continue;
        const void* d = s->dlogits ? s->dlogits[i] : nullptr;
        if (!s->logits[i] || (s->dlogits && !d)) return WS_ERR_INVALID_ARG;
        if (!aligned(s->logits[i], eb) || !aligned(d, eb)) return WS_ERR_ALIGNMENT;
        wide = wide && aligned(s->logits[i], 16) && aligned(d, 16);
    }
    if (!workspace || workspace_bytes < ws_balance_workspace_bytes(s)) return WS_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return WS_ERR_ALIGNMENT;
    BalanceParams P = {};
    P.r.replicas = s->replicas;
    P.r.experts = s->experts;
    P.r.topk = s->topk;
    P.r.rows = balance_rows(s);
    const long long chunks = chunks_of(s, P.r.rows);
    if (chunks > 0x7fffffffLL) return WS_ERR_TOO_LARGE;
    P.r.chunks = (int)chunks;
    P.counts = (const long long*)counts;
    P.upstream = upstream;
    P.loss = loss;
    P.partials = (double2*)workspace;
    P.ld = s->logits_ld;
    P.dld = s->dlogits_ld;
    P.coef = coef;
    P.z = z_coef;
    P.accumulate = accumulate;
    const int v = wide ? (int)(16 / eb) : 1, vecs = (s->experts + v - 1) / v;
    P.lanes = 1;
    while (P.lanes < 32 && P.lanes < vecs) P.lanes <<= 1;
    cudaStream_t st = (cudaStream_t)stream;
    const int most = kMaxReplicas / s->replicas;
    for (int l = 0; l < s->layers; l += most) {
        const int layers = s->layers - l < most ? s->layers - l : most, np = layers * s->replicas;
        P.r.layer0 = l;
        if (np <= 16) launch_balance<16>(s, wide, P, layers, st);
        else if (np <= 128) launch_balance<128>(s, wide, P, layers, st);
        else launch_balance<kMaxReplicas>(s, wide, P, layers, st);
        const ws_status r = ws_check_launch("ws_balance_loss");
        if (r != WS_OK) return r;
    }
    if (loss && P.r.chunks > 1) launch(balance_loss_kernel, dim3(s->layers), st, P);
    return ws_check_launch("ws_balance_loss");
}

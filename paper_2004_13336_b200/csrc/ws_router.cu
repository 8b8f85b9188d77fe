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
constexpr int kMaxPointers = 512;    // (layer, replica) pairs of a launch
constexpr int kMaxCtas = 1184;       // CTAs of a launch of ws_balance_loss
constexpr int kMaxExperts = 1024;
constexpr int kBlock = 256;

// What a launch names travels in its parameters, in a table of the size it needs.
template <int NP, int NR>
struct RouterTab {
    const void* in[NP];            // [layers of the launch][replicas] picks or logits
    const unsigned char* valid[NR];// [replicas]
    int tokens[NR];                // [replicas]
    int chunk0[NR];                // [replicas] first chunk of a replica's tokens
};
template <int NP, int NR>
struct BalanceTab : RouterTab<NP, NR> {
    void* out[NP];                 // [layers of the launch][replicas] dlogits
};

struct RouterParams {
    int replicas, experts, topk;
    int chunks;                    // chunks of a layer
    int rows;                      // tokens of a chunk
    int layer0;                    // first layer of the launch
    unsigned magic;                // ceil(2^32 / topk)
    int columns;                   // counters of an expert
};

// The replica that a chunk belongs to.
template <int NP, int NR>
__device__ __forceinline__ int replica_of(const RouterTab<NP, NR>& tab, int replicas, int chunk) {
    int lo = 0, hi = replicas - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.chunk0[mid] <= chunk) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// ------------------------------------------------------------------ counts ---
constexpr int kCountBlock = 512, kCountWarps = kCountBlock / 32;
// Every expert has several counters side by side, a lane's by its number modulo theirs, as many as fit: fewer lanes meet on one.
constexpr int kCounters = 2048;

// Counts a thread's share (first, first + step, ... of the 16-byte vectors, or of the picks) of `n` tokens' picks into its column
// `hist`, and returns how many of its share of the tokens exist.  Fewer than 2^22 picks: a pick's token is found by a product
// (magic = ceil(2^32 / topk)).  A pass's loads are all issued before the first count.
template <typename I, bool MASKED, int B>
__device__ __forceinline__ void count_vectors(const uint4* p, const unsigned char* valid, int nv, unsigned topk, unsigned magic, unsigned E, int first, int step,
                                              int* hist, int columns) {
    constexpr int VE = 16 / sizeof(I);
    for (int i = first; i < nv; i += step * B) {
        uint4 v[B];
        unsigned char ok[MASKED ? B * VE : 1];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const int ib = i + step * b;
            v[b] = make_uint4(~0u, ~0u, ~0u, ~0u);
            if (ib < nv) v[b] = __ldcs(p + ib);
            if constexpr (MASKED)
#pragma unroll
                for (int j = 0; j < VE; ++j) {
                    const unsigned at = ib < nv ? ib * VE + j : 0;
                    ok[b * VE + j] = valid[topk == 1 ? at : __umulhi(at, magic)];
                }
        }
#pragma unroll
        for (int b = 0; b < B; ++b) {
            unsigned e[VE];
            if constexpr (VE == 4) {
                e[0] = v[b].x; e[1] = v[b].y; e[2] = v[b].z; e[3] = v[b].w;
            } else {
                e[0] = v[b].y ? ~0u : v[b].x; e[1] = v[b].w ? ~0u : v[b].z;
            }
#pragma unroll
            for (int j = 0; j < VE; ++j)
                if (e[j] < E && (!MASKED || ok[b * VE + j])) atomicAdd(hist + e[j] * columns, 1);
        }
    }
}
template <typename I, int BM>
__device__ __forceinline__ int count_picks(const I* picks, const unsigned char* valid, int n, unsigned topk, unsigned magic, unsigned E, int first, int step,
                                           int* hist, int columns) {
    constexpr int VE = 16 / sizeof(I);
    const int total = n * (int)topk;
    int done = 0;
    if ((reinterpret_cast<uintptr_t>(picks) & 15u) == 0) {
        const int nv = total / VE;
        if (valid) count_vectors<I, true, BM>((const uint4*)picks, valid, nv, topk, magic, E, first, step, hist, columns);
        else count_vectors<I, false, 4>((const uint4*)picks, valid, nv, topk, magic, E, first, step, hist, columns);
        done = nv * VE;
    }
    auto exists = [&](unsigned at) { return !valid || valid[topk == 1 ? at : __umulhi(at, magic)]; };
    for (int i = done + first; i < total; i += step) {
        const I e = picks[i];
        if (exists(i) && e >= 0 && e < (I)E) atomicAdd(hist + (int)e * columns, 1);
    }
    if (!valid) return first == 0 ? n : 0;
    int live = 0;
    for (int i = first; i < n; i += step) live += valid[i] != 0;
    return live;
}

// Row y of the grid counts layer y in shared memory.  CLUSTER: the row is a cluster, whose warps take the layer's chunks in turn
// and which adds its CTAs' counts up over distributed shared memory, so that nothing has to be cleared in front of the
// launch; else a CTA takes a chunk and adds its counts to the layer's, integers, so in any order.
template <typename I, bool CLUSTER, int NP, int NR>
__global__ void __launch_bounds__(kCountBlock, CLUSTER ? 2 : 4) counts_kernel(const RouterParams P, const __grid_constant__ RouterTab<NP, NR> tab, long long* counts,
                                                             int accumulate) {
    __shared__ int hist[kCounters], sums[kMaxExperts + 1];
    const int E = P.experts, layer = blockIdx.y, warp = threadIdx.x >> 5;
    const int columns = P.columns;
    if (CLUSTER) asm volatile("griddepcontrol.launch_dependents;");
    for (int i = threadIdx.x; i < columns * E; i += kCountBlock) hist[i] = 0;
    if (threadIdx.x == 0) sums[E] = 0;
    __syncthreads();
    if (CLUSTER) asm volatile("griddepcontrol.wait;" ::: "memory");
    int live = 0;
    for (int chunk = CLUSTER ? blockIdx.x * kCountWarps + warp : blockIdx.x; chunk < P.chunks; chunk += CLUSTER ? gridDim.x * kCountWarps : gridDim.x) {
        const int rep = replica_of(tab, P.replicas, chunk);
        const long long row0 = (long long)(chunk - tab.chunk0[rep]) * P.rows;
        const int n = (int)min((long long)P.rows, tab.tokens[rep] - row0);
        const unsigned char* valid = tab.valid[rep];
        live += count_picks<I, CLUSTER || sizeof(I) == 8 ? 4 : 2>((const I*)tab.in[layer * P.replicas + rep] + row0 * P.topk, valid ? valid + row0 : nullptr, n, P.topk, P.magic, E,
                            CLUSTER ? threadIdx.x & 31 : threadIdx.x, CLUSTER ? 32 : kCountBlock, hist + (threadIdx.x & (columns - 1)), columns);
    }
    live = __reduce_add_sync(0xffffffffu, live);
    if ((threadIdx.x & 31) == 0 && live) atomicAdd(sums + E, live);
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += kCountBlock) {
        int sum = 0;
        for (int k = 0; k < columns; ++k) sum += hist[e * columns + ((e + k) & (columns - 1))];      // (every lane in a bank of its own)
        sums[e] = sum;
    }
    long long* out = counts + (long long)(P.layer0 + layer) * (E + 1);
    if constexpr (CLUSTER) {
        const int rank = blockIdx.x, ctas = gridDim.x;
        auto meet = [] { asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory"); };
        meet();
        const unsigned own = (unsigned)__cvta_generic_to_shared(sums);
        for (int e = rank * kCountBlock + threadIdx.x; e <= E; e += ctas * kCountBlock) {
            long long sum = 0;
            for (int k = 0; k < ctas; ++k) {
                unsigned at;
                int c;
                asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(own + 4 * e), "r"(k));
                asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c) : "r"(at) : "memory");
                sum += c;
            }
            out[e] = accumulate ? out[e] + sum : sum;
        }
        meet();                    // (shared memory stays until everybody has read it)
    } else {
        __syncthreads();
        for (int e = threadIdx.x; e <= E; e += kCountBlock)
            if (sums[e]) atomicAdd((unsigned long long*)out + e, (unsigned long long)sums[e]);
    }
}

// ----------------------------------------------------------------- balance ---
struct BalanceParams {
    RouterParams r;
    const long long* counts;
    const float* upstream;
    float* loss;
    double2* partials;             // [layers][slots]
    long long ld, dld;
    double coef, z;
    double slope, zslope;          // coef experts, 2 z
    int accumulate;
    int lanes;                     // lanes of a row, a power of two
    int layers;                    // layers of the launch
    int sms;                       // multiprocessors of the device
    int whole;                     // an item is a layer, else a chunk of a layer's tokens
    int team;                      // warps that share a replica's rows, a power of two
    int slots;                     // CTAs of a layer, at most
};
// A launch's items are dealt out to its CTAs in runs of consecutive ones: `extra` CTAs get per_cta + 1, the others per_cta.
struct Deal {
    long long per_cta;
    int extra;
    __host__ __device__ Deal(long long items, int ctas) : per_cta(items / ctas), extra((int)(items % ctas)) {}
    __device__ __forceinline__ long long first(int cta) const { return cta * per_cta + (cta < extra ? cta : extra); }
    __device__ __forceinline__ int cta_of(long long item) const {
        const long long big = extra * (per_cta + 1);
        return (int)(item < big ? item / (per_cta + 1) : extra + (item - big) / per_cta);
    }
};

// 2^x and 1/x to 2 units in the last place of fp32, results below 2^-126 as 0: next to a row's largest score they are.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.4426950408889634f;

// Two fp32 numbers in a register pair: one instruction adds, multiplies or multiplies and adds both.
struct F2 {
    unsigned long long v;
    __device__ __forceinline__ F2() {}
    __device__ __forceinline__ F2(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ void get(float& a, float& b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
};
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return d;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
    F2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
    return d;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
    F2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
    return d;
}

// V consecutive logits as they lie in memory: one, or 16 bytes of them.
template <typename X, int V>
struct Raw {
    unsigned w[V == 1 ? 1 : 4];
    __device__ __forceinline__ void load(const X* p) {
        if constexpr (V > 1) {
            const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p));
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else if constexpr (sizeof(X) == 4) {
            w[0] = __ldcs(reinterpret_cast<const unsigned*>(p));
        } else {
            w[0] = (unsigned)__ldcs(reinterpret_cast<const unsigned short*>(p)) << 16;
        }
    }
    // -infinity: experts that do not exist
    __device__ __forceinline__ void none() {
#pragma unroll
        for (int i = 0; i < (V == 1 ? 1 : 4); ++i) w[i] = V == 1 || sizeof(X) == 4 ? 0xff800000u : 0xff80ff80u;
    }
    __device__ __forceinline__ float top() const {
        if constexpr (V == 8) {         // two at a time
            __nv_bfloat162 m = reinterpret_cast<const __nv_bfloat162&>(w[0]);
#pragma unroll
            for (int i = 1; i < 4; ++i) m = __hmax2(m, reinterpret_cast<const __nv_bfloat162&>(w[i]));
            return fmaxf(__low2float(m), __high2float(m));
        } else {
            float m = get(0);
#pragma unroll
            for (int i = 1; i < V; ++i) m = fmaxf(m, get(i));
            return m;
        }
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (V == 1 || sizeof(X) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
};
template <typename X, int V>
__device__ __forceinline__ void store_v(X* p, const float* x) {
    if constexpr (V == 1 && sizeof(X) == 4) {
        __stcs(p, x[0]);
    } else if constexpr (V == 1) {
        const __nv_bfloat16 b = __float2bfloat16_rn(x[0]);
        __stcs(reinterpret_cast<unsigned short*>(p), *reinterpret_cast<const unsigned short*>(&b));
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
// Over the G lanes of a row.
__device__ __forceinline__ float row_max(float x, int G) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (o < G) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}
__device__ __forceinline__ void row_sum2(float& a, float& b, int G) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (o < G) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
}

// The rows' pass.  Its floor is the copy of the logits; what it has to do per element meanwhile is an exponential, a few
// packed additions and products and, with bf16, taking the pairs apart and putting them together, and per row three sums over
// its lanes (18 instructions an element of bf16 rows of 64, where 22 fit into the copy's time).  So a lane holds 16 elements where a row
// has so many, the launch is one wave of CTAs that walk runs of consecutive rows (the counts are read once a layer and CTA), and the next
// row is on its way while the present one is worked on.  us: 43 M bf16 logits in rows of 64 (24 layers, 8 replicas, z loss) 40,
// 26 at the copy bandwidth (lanes of 8 elements 48, CTAs of 64 KB instead of one wave 58, single fp32 instructions 48); 134 M
// fp32 sigmoid logits in rows of 256 177, softmax 189, 164 at the copy bandwidth (sigmoid in CTAs of 64 KB 264).
//
// Resident CTAs per SM by the elements of a lane.
__host__ __device__ constexpr int balance_ctas(int elems, bool sig) {
    return elems > 16 ? 1 : elems > 8 ? (sig ? 2 : 3) : (sig ? 4 : 4);
}

// X: the logits' type.  A row lies on P.lanes lanes; lane q holds the C vectors of V elements at (c lanes + q) V.
template <typename X, int V, int C, bool SIG, int NP, int NR>
__global__ void __launch_bounds__(kBlock, balance_ctas(C * V, SIG)) balance_kernel(const __grid_constant__ BalanceParams P, const Deal deal,
                                                                                   const __grid_constant__ BalanceTab<NP, NR> tab) {
    constexpr int N = C * V, H = (N + 1) / 2;             // elements of a lane, pairs
    __shared__ __align__(16) float shares[kMaxExperts];       // (32 lanes hold at most 32 elements each)
    __shared__ double2 part[kBlock / 32];
    asm volatile("griddepcontrol.launch_dependents;");
    const int E = P.r.experts, G = P.lanes, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int q = lane & (G - 1), sub = lane / G, per_warp = 32 / G;
    // The warps that share a replica's rows: all of them, or in a whole layer of several replicas a part for each.
    const int team = P.team, first = (warp & (team - 1)) * per_warp, stride = team * per_warp;
    const int mine = (E / V - q + G - 1) / G;             // vectors of this lane that exist
    const int per_layer = P.whole ? 1 : P.r.chunks;
    const long long end = deal.first(blockIdx.x + 1);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const float up = P.upstream ? *P.upstream : 1.f;
    for (long long item = deal.first(blockIdx.x); item < end;) {
        const int layer = item <= 0x7fffffffLL ? (int)item / per_layer : (int)(item / per_layer);
        const long long layer_end = min(end, (long long)(layer + 1) * per_layer);

        // The rows of a run: consecutive items in one replica.
        int n, run, rep = warp / team;
        const X* in;
        X* out;
        const unsigned char* valid;
        Raw<X, V> next[C];
        // Of the rows i (read next) and i + stride: whether the token exists.  A row is read once that is known.
        bool live1, live2;
        auto exists = [&](int i) { return i < n && (!valid || valid[i]); };
        auto fetch = [&] {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                next[c].none();
                if (live1 && c < mine) next[c].load(in + c * G * V);
            }
        };
        auto open = [&] {
            long long row0 = 0;
            if (P.whole) {
                n = rep < P.r.replicas ? tab.tokens[rep] : 0;
                if (n == 0) {          // (the pointers of a replica without tokens are nothing)
                    live1 = live2 = false;
                    out = nullptr;
                    return;
                }
            } else {
                const int chunk = (int)(item - (long long)layer * per_layer);
                rep = replica_of(tab, P.r.replicas, chunk);
                const int rep_end = rep + 1 < P.r.replicas ? tab.chunk0[rep + 1] : P.r.chunks;
                run = (int)min(layer_end - item, (long long)(rep_end - chunk));
                row0 = (long long)(chunk - tab.chunk0[rep]) * P.r.rows;
                n = (int)min((long long)run * P.r.rows, tab.tokens[rep] - row0);
            }
            const int i = first + sub;
            valid = tab.valid[rep];
            if (valid) valid += row0;
            in = (const X*)tab.in[layer * P.r.replicas + rep] + (row0 + i) * P.ld + q * V;
            out = (X*)tab.out[layer * P.r.replicas + rep];
            if (out) out += (row0 + i) * P.dld + q * V;
            live1 = exists(i);
            live2 = exists(i + stride);
            fetch();
        };
        open();                        // the first rows are on their way while the counts are read

        const long long* counts = P.counts + (long long)(P.r.layer0 + layer) * (E + 1);
        const float tokens = (float)counts[E], inv = tokens > 0.f ? 1.f / tokens : 0.f, inv_picks = inv / P.r.topk;
        // (in 64 bits: neither factor needs to be an fp32 number for the product to be one)
        const float slope = (float)(up * P.slope * inv), zslope = P.z == 0.0 ? 0.f : (float)(up * P.zslope * inv);
        __syncthreads();               // (the layer before is done with its shares)
        for (int e = threadIdx.x; e < C * G * V; e += kBlock) shares[e] = e < E ? (float)counts[e] * inv_picks : 0.f;
        __syncthreads();
        F2 share[H];
        {
            float f[2 * H];
#pragma unroll
            for (int k = 0; k < 2 * H; ++k) f[k] = k < N ? shares[(k / V * G + q) * V + k % V] : 0.f;
#pragma unroll
            for (int h = 0; h < H; ++h) share[h] = F2(f[2 * h], f[2 * h + 1]);
        }

        double bal = 0.0, zsum = 0.0;
        for (;;) {
            for (int i0 = first; i0 < n; i0 += stride) {
                Raw<X, V> x[C];
#pragma unroll
                for (int c = 0; c < C; ++c) x[c] = next[c];
                const bool live = live1;
                in += stride * P.ld;
                live1 = live2;
                fetch();
                live2 = exists(i0 + sub + 2 * stride);

                auto get = [&](int k) { return k < N ? x[k / V].get(k % V) : -INFINITY; };
                auto row_top = [&] {
                    float top = x[0].top();
#pragma unroll
                    for (int c = 1; c < C; ++c) top = fmaxf(top, x[c].top());
                    top = row_max(top, G);
                    return top > -INFINITY ? top : 0.f;
                };
                F2 s[H], y[SIG ? H : 1];
                float total, inner, shift = 0.f;
                // exp(v - shift) with the difference formed first: right for any v and shift
                auto far_exponentials = [&] {
#pragma unroll
                    for (int h = 0; h < H; ++h) s[h] = F2(exp2_fast((get(2 * h) - shift) * kLog2e), exp2_fast((get(2 * h + 1) - shift) * kLog2e));
                };
                // the scores' sum and that of share times score, over the row
                auto sums = [&] {
                    F2 t(0.f, 0.f), u(0.f, 0.f);
#pragma unroll
                    for (int h = 0; h < H; ++h) {
                        t = add2(t, s[h]);
                        u = fma2(share[h], s[h], u);
                    }
                    float a, b;
                    t.get(a, b);
                    total = a + b;
                    u.get(a, b);
                    inner = a + b;
                    row_sum2(total, inner, G);
                };
                if constexpr (SIG) {
#pragma unroll
                    for (int h = 0; h < H; ++h) {          // 1 / (1 + t) with t = exp(-v), and its complement t / (1 + t)
                        float a, b;
                        mul2(F2(get(2 * h), get(2 * h + 1)), F2(-kLog2e, -kLog2e)).get(a, b);
                        const F2 t(exp2_fast(a), exp2_fast(b));
                        add2(t, F2(1.f, 1.f)).get(a, b);
                        s[h] = F2(rcp_fast(a), rcp_fast(b));
                        mul2(s[h], t).get(a, b);
                        y[h] = F2(fminf(a, 1.f), fminf(b, 1.f));           // (0 * infinity: 1)
                    }
                    sums();
                    if (__any_sync(0xffffffffu, total < 1e-17f)) {
                        // All scores of a row are below 2^-56 (its largest logit below -39): they are exp(v) to the last bit,
                        // their complements 1, and only their ratios count, which exp(v - top) keeps where the scores vanish.
                        F2 keep[H];
#pragma unroll
                        for (int h = 0; h < H; ++h) keep[h] = s[h];
                        const bool low = total < 1e-17f;
                        const float total0 = total, inner0 = inner;
                        shift = row_top();
                        far_exponentials();
                        sums();
                        if (low) {
#pragma unroll
                            for (int h = 0; h < H; ++h) y[h] = F2(1.f, 1.f);
                        } else {
                            total = total0;
                            inner = inner0;
#pragma unroll
                            for (int h = 0; h < H; ++h) s[h] = keep[h];
                        }
                    }
                } else {
                    shift = row_top();
                    // v log2 e - shift log2 e in one fma, whose second term is rounded: every exponent of the row is off by half
                    // a unit in the last place of it, the same for all, so the scores' ratios stay and the sum's logarithm
                    // moves by less than shift's own rounding.  Below 2^20 that is 2^-4 at most; from some 2^31 on the
                    // scores would all vanish or overflow.
                    if (__any_sync(0xffffffffu, !(fabsf(shift) < 1048576.f))) {
                        far_exponentials();
                    } else {
                        const float bias = -shift * kLog2e;
#pragma unroll
                        for (int h = 0; h < H; ++h) {
                            float a, b;
                            fma2(F2(get(2 * h), get(2 * h + 1)), F2(kLog2e, kLog2e), F2(bias, bias)).get(a, b);
                            s[h] = F2(exp2_fast(a), exp2_fast(b));
                        }
                    }
                    sums();
                }
                const bool empty = total == 0.f;                  // no expert that the token can pick
                const float scale = empty ? 0.f : rcp_fast(total);
                inner *= scale;
                float lse = 0.f;
                // (__logf is off by up to 2^-21 next to 1, where the sum is when one expert has most of it)
                if (!SIG && P.z != 0.0) lse = empty ? 0.f : shift + logf(total);
                if (live && q == 0) {
                    bal += inner;
                    zsum += (double)lse * lse;
                }
                if (out) {
                    if (i0 + sub < n && (live || !P.accumulate)) {
                        // p_e (slope (f_e - inner) + zslope lse) with p_e = s_e scale; a token that does not exist has scores 0, and
                        // no factors either: an infinite one (an overflowed loss scale) would make NaN of them
                        const float a = empty ? 0.f : slope * scale, b = empty ? 0.f : (SIG ? -slope * inner : zslope * lse - slope * inner) * scale;
                        float d[2 * H];
#pragma unroll
                        for (int h = 0; h < H; ++h) {
                            F2 g = mul2(s[h], fma2(F2(a, a), share[h], F2(b, b)));
                            if constexpr (SIG) g = mul2(g, y[h]);
                            g.get(d[2 * h], d[2 * h + 1]);
                        }
#pragma unroll
                        for (int c = 0; c < C; ++c) {
                            if (c >= mine) continue;
                            X* at = out + c * G * V;
                            if (P.accumulate) {
                                Raw<X, V> old;
                                old.load(at);
#pragma unroll
                                for (int v = 0; v < V; ++v) d[c * V + v] += old.get(v);
                            }
                            store_v<X, V>(at, d + c * V);
                        }
                    }
                    out += stride * P.dld;
                }
            }
            if (P.whole) {
                rep += (kBlock / 32) / team;
                if (rep >= P.r.replicas) break;
            } else {
                item += run;
                if (item == layer_end) break;
            }
            open();
        }
        item = layer_end;

        if (P.loss) {
            sum2(bal, zsum);
            if (lane == 0) part[warp] = make_double2(bal, zsum);
            __syncthreads();
            if (threadIdx.x == 0) {
                bal = zsum = 0.0;
                for (int k = 0; k < kBlock / 32; ++k) {
                    bal += part[k].x;
                    zsum += part[k].y;
                }
                if (P.whole) write_loss(P, P.r.layer0 + layer, bal, zsum, (double)counts[E]);
                else P.partials[(long long)(P.r.layer0 + layer) * P.slots + blockIdx.x - deal.cta_of((long long)layer * per_layer)] = make_double2(bal, zsum);
            }
        }
    }
}

// The losses of a launch's layers from what its CTAs left.
__global__ void __launch_bounds__(kBlock) balance_loss_kernel(const __grid_constant__ BalanceParams P, const Deal deal) {
    __shared__ double2 part[kBlock / 32];
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int layer = P.r.layer0 + blockIdx.x;
    const long long item0 = (long long)blockIdx.x * P.r.chunks;
    const int count = deal.cta_of(item0 + P.r.chunks - 1) - deal.cta_of(item0) + 1;
    const double2* p = P.partials + (long long)layer * P.slots;
    double bal = 0.0, zsum = 0.0;
    for (int i = threadIdx.x; i < count; i += kBlock) {
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
// With programmatic dependent launch; `cluster` CTAs along x to a cluster.
template <typename... KArgs, typename... Args>
void launch_cluster(void (*kernel)(KArgs...), dim3 grid, int block, int cluster, cudaStream_t st, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}
template <typename... KArgs, typename... Args>
void launch(void (*kernel)(KArgs...), dim3 grid, cudaStream_t st, const Args&... args) {
    launch_cluster(kernel, grid, kBlock, 1, st, args...);
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
template <int NP, int NR>
void fill(RouterTab<NP, NR>& tab, const ws_router_set* s, const void* const* in, int layer0, int layers, int rows) {
    for (int i = 0; i < layers * s->replicas; ++i) tab.in[i] = in[(long long)layer0 * s->replicas + i];
    int at = 0;
    for (int k = 0; k < s->replicas; ++k) {
        tab.valid[k] = s->valid ? s->valid[k] : nullptr;
        tab.tokens[k] = (int)s->tokens[k];
        tab.chunk0[k] = at;
        at += (int)((s->tokens[k] + rows - 1) / rows);
    }
}

// ctas: CTAs of a layer, a cluster or not
template <int NP, int NR>
void launch_counts(const ws_router_set* s, const RouterParams& P, int layers, int ctas, bool cluster, int64_t* counts, int accumulate, cudaStream_t st) {
    RouterTab<NP, NR> tab;
    fill(tab, s, s->picks, P.layer0, layers, P.rows);
    const dim3 grid(ctas, layers);
    long long* out = (long long*)counts;
    if (cluster) {
        if (s->index_bytes == 4) launch_cluster(counts_kernel<int, true, NP, NR>, grid, kCountBlock, ctas, st, P, tab, out, accumulate);
        else launch_cluster(counts_kernel<long long, true, NP, NR>, grid, kCountBlock, ctas, st, P, tab, out, accumulate);
    } else {
        if (s->index_bytes == 4) counts_kernel<int, false, NP, NR><<<grid, kCountBlock, 0, st>>>(P, tab, out, 1);
        else counts_kernel<long long, false, NP, NR><<<grid, kCountBlock, 0, st>>>(P, tab, out, 1);
    }
}

template <typename X, int V, int C, int NP, int NR>
Deal launch_score(const ws_router_set* s, const BalanceParams& P, const BalanceTab<NP, NR>& tab, cudaStream_t st) {
    const bool sig = s->score == WS_SIGMOID;
    const long long items = (long long)P.layers * (P.whole ? 1 : P.r.chunks), most = (long long)P.sms * balance_ctas(C * V, sig);
    const int grid = (int)(items < most ? items : most < kMaxCtas ? most : kMaxCtas);
    const Deal deal(items, grid);
    if (sig) launch(balance_kernel<X, V, C, true, NP, NR>, dim3(grid), st, P, deal, tab);
    else launch(balance_kernel<X, V, C, false, NP, NR>, dim3(grid), st, P, deal, tab);
    return deal;
}
// A lane holds up to 16 elements of a row in vectors (fewer shuffles, and less of what every lane does once a row), up to 8 single
// ones (rows off the 16-byte boundaries: bf16 rows of 60, 15.7 M, 41 us, with 2 elements 77, with 16 40; fp32 rows of 33 29, 55, 30),
// more where 32 lanes do not hold the row that way.  Short fp32 rows keep two lanes side by side (rows of 16 20 -> 17; bf16 16 -> 19).
template <typename X, int NP, int NR>
Deal launch_shape(const ws_router_set* s, bool wide, BalanceParams& P, const BalanceTab<NP, NR>& tab, cudaStream_t st) {
    constexpr int V = 16 / sizeof(X);
    const int vecs = wide ? s->experts / V : s->experts;
    int c = 1;
    while (2 * c * (wide ? V : 1) <= (wide ? 16 : 8) && (wide && V == 4 && vecs > 2 ? 4 : 2) * c <= vecs) c *= 2;
    while ((vecs + c - 1) / c > 32) c *= 2;
    P.lanes = 1;
    while (P.lanes * c < vecs) P.lanes *= 2;
    if (wide) {
        if (c == 1) return launch_score<X, V, 1>(s, P, tab, st);
        if (c == 2) return launch_score<X, V, 2>(s, P, tab, st);
        if (c == 4) return launch_score<X, V, 4>(s, P, tab, st);
        if constexpr (V == 4) return launch_score<X, V, 8>(s, P, tab, st);
    }
    if (c == 1) return launch_score<X, 1, 1>(s, P, tab, st);
    if (c == 2) return launch_score<X, 1, 2>(s, P, tab, st);
    if (c == 4) return launch_score<X, 1, 4>(s, P, tab, st);
    if (c == 8) return launch_score<X, 1, 8>(s, P, tab, st);
    if (c == 16) return launch_score<X, 1, 16>(s, P, tab, st);
    return launch_score<X, 1, 32>(s, P, tab, st);
}
template <int NP, int NR>
Deal launch_balance(const ws_router_set* s, bool wide, BalanceParams& P, cudaStream_t st) {
    BalanceTab<NP, NR> tab;
    fill(tab, s, s->logits, P.r.layer0, P.layers, P.r.rows);
    for (int i = 0; i < P.layers * s->replicas; ++i) tab.out[i] = s->dlogits ? s->dlogits[(long long)P.r.layer0 * s->replicas + i] : nullptr;
    return s->dtype == WS_F32 ? launch_shape<float>(s, wide, P, tab, st) : launch_shape<__nv_bfloat16>(s, wide, P, tab, st);
}

// Multiprocessors of the current device, asked for once per thread and device.
int device_sms() {
    static thread_local int known = -1, sms = 148;
    int dev = 0;
    if (cudaGetDevice(&dev) == cudaSuccess && dev != known && cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess) known = dev;
    return sms;
}

// How a layer's tokens are cut up: tokens of a chunk, chunks, whether a CTA takes the whole layer.
struct Cut {
    int rows, whole;
    long long chunks;
    int slots;
};
Cut balance_cut(const ws_router_set* s) {
    Cut c;
    const int bytes = s->experts * (s->dtype == WS_F32 ? 4 : 2);
    c.rows = 512;
    while (c.rows > 8 && c.rows * bytes > (16 << 10)) c.rows >>= 1;
    long long total = 0;
    for (int k = 0; k < s->replicas; ++k) total += s->tokens[k];
    c.whole = total <= 2 * c.rows;
    c.chunks = chunks_of(s, c.rows);
    c.slots = (int)(c.chunks < kMaxCtas ? c.chunks : kMaxCtas);
    return c;
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
    RouterParams P = {};
    P.replicas = s->replicas;
    P.experts = s->experts;
    P.topk = s->topk;
    P.magic = s->topk > 1 ? (unsigned)(((1ULL << 32) + s->topk - 1) / s->topk) : 0;
    // Chunks of about 512 picks, one for a warp; a power of two of tokens, so that chunks of aligned picks are aligned.
    // A cluster of up to 8 CTAs a layer, while none of its warps has more than 2 chunks.  us, a cluster / chunks of 8192 picks:
    // 24 layers of 65 K picks 6.8 / 11, 1 of 65 K 5.3 / 7.4, 48 of 33 K 5.9 / 16; 1 of 262 K 13.2 / 6.3, 8 of 262 K 19 / 8.2
    // (a cluster's few CTAs count some 2 picks a cycle each).  4 layers of 2.1 M 64-bit picks, chunks of 8192 / 16384: 19.5 / 17.6.
    P.rows = 4;
    while (2 * P.rows * s->topk <= 512) P.rows *= 2;
    long long chunks = chunks_of(s, P.rows);
    const bool cluster = chunks <= 8 * kCountWarps * 2;
    int ctas = 1;
    if (cluster) {
        while (ctas < 8 && ctas * kCountWarps < chunks) ctas *= 2;
    } else {
        // a CTA's chunk: 8192 picks, more where that would be more CTAs than are resident
        while (2 * P.rows * s->topk <= 8192) P.rows *= 2;
        while ((chunks = chunks_of(s, P.rows)) * s->layers > 4LL * device_sms() && 2 * P.rows * s->topk <= 65536) P.rows *= 2;
        if (chunks > 0x7fffffffLL) return WS_ERR_TOO_LARGE;
        ctas = (int)chunks;
        if (!accumulate) {
            const cudaError_t e = cudaMemsetAsync(counts, 0, sizeof(int64_t) * (size_t)s->layers * (s->experts + 1), st);
            if (e != cudaSuccess) return ws_cuda_fail(e, "ws_router_counts");
        }
    }
    P.chunks = (int)chunks;
    P.columns = cluster ? 8 : 4;
    while (P.columns * s->experts > kCounters) P.columns >>= 1;
    const int most = kMaxPointers / s->replicas;
    for (int l = 0; l < s->layers; l += most) {
        const int layers = s->layers - l < most ? s->layers - l : most, np = layers * s->replicas;
        P.layer0 = l;
        if (np <= 32) launch_counts<32, 32>(s, P, layers, ctas, cluster, counts, accumulate, st);
        else if (s->replicas <= 32) launch_counts<kMaxPointers, 32>(s, P, layers, ctas, cluster, counts, accumulate, st);
        else launch_counts<kMaxPointers, kMaxReplicas>(s, P, layers, ctas, cluster, counts, accumulate, st);
        const ws_status r = ws_check_launch("ws_router_counts");
        if (r != WS_OK) return r;
    }
    return WS_OK;
}

extern "C" size_t ws_balance_workspace_bytes(const ws_router_set* s) {
    if (check_balance(s) != WS_OK) return 0;
    return sizeof(double2) * (size_t)s->layers * (size_t)balance_cut(s).slots;
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
    const Cut cut = balance_cut(s);
    if (cut.chunks > 0x7fffffffLL) return WS_ERR_TOO_LARGE;
    P.r.rows = cut.rows;
    P.r.chunks = (int)cut.chunks;
    P.whole = cut.whole;
    P.team = kBlock / 32;
    for (int k = 1; cut.whole && k < s->replicas && P.team > 1; k *= 2) P.team /= 2;
    P.slots = cut.slots;
    P.sms = device_sms();
    P.counts = (const long long*)counts;
    P.upstream = upstream;
    P.loss = loss;
    P.partials = (double2*)workspace;
    P.ld = s->logits_ld;
    P.dld = s->dlogits_ld;
    P.coef = coef;
    P.z = z_coef;
    P.slope = coef * s->experts;
    P.zslope = 2.0 * z_coef;
    P.accumulate = accumulate;
    cudaStream_t st = (cudaStream_t)stream;
    const int most = kMaxPointers / s->replicas;
    for (int l = 0; l < s->layers; l += most) {
        P.layers = s->layers - l < most ? s->layers - l : most;
        P.r.layer0 = l;
        const Deal deal = P.layers * s->replicas <= 32 ? launch_balance<32, 32>(s, wide, P, st)
                         : s->replicas <= 32          ? launch_balance<kMaxPointers, 32>(s, wide, P, st)
                                                      : launch_balance<kMaxPointers, kMaxReplicas>(s, wide, P, st);
        if (loss && !P.whole) launch(balance_loss_kernel, dim3(P.layers), st, P, deal);
        const ws_status r = ws_check_launch("ws_balance_loss");
        if (r != WS_OK) return r;
    }
    return WS_OK;
}

// Dropout of the replicas' weights: ws_unpack_dropout hands the sharded weights out to the replicas' tensors, each replica
// under a mask of its own, and ws_reduce_dropout, its adjoint, sums the replicas' gradients under the same masks into the
// sharded layout (reverse formatting of paper Section 4.2; formatting and sum of Sections 2.2, 5.1).
//
// A mask is a function of (seed, step, replica, tensor, element) and is drawn where it is used.  A tile starts at a
// multiple of 8 elements of its tensor in either layout, so the 8 elements of a vector are those of one random block.
#include "ws_kernels.cuh"

namespace {

using namespace wsk;

constexpr int kRounds = 7;

struct DropParams {
    const WsTile* tiles;
    long long tile_lo;      // first tile of this launch
    long long ntl;          // tiles per shard (concatenated layout: of this launch)
    long long nitems;
    long long S;
    int r0;                 // first shard of this launch; `flat` starts with it
    int concat;
    const void* const* table;   // [T][nsets]
    int nsets;
    unsigned key[2 * kRounds];  // the two key words of every round
    unsigned thr;           // T << 16
    float scale;
    unsigned step;
    const unsigned* step_dev;
    unsigned replica;
#ifdef WS_DEBUG_BOUNDS
    unsigned* bounds;
    long long flat_elems;
#endif
};

// Philox4x32: a round multiplies two of the words by constants to 64 bits and mixes the halves with the others and the key.
__device__ __forceinline__ uint4 philox(const DropParams& P, unsigned c0, unsigned c1, unsigned c2, unsigned c3) {
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
        c0 = (unsigned)(b >> 32) ^ c1 ^ P.key[2 * i];
        c1 = (unsigned)b;
        c2 = (unsigned)(a >> 32) ^ c3 ^ P.key[2 * i + 1];
        c3 = (unsigned)a;
    }
    return make_uint4(c0, c1, c2, c3);
}
// Which of a block's elements are kept, without taking the halves apart: the high half of w is at least T where w >= T 2^16,
// the low half where w 2^16 >= T 2^16.
__device__ __forceinline__ bool kept(const uint4& w, int i, unsigned thr) {
    const unsigned x = i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w;
    return (i & 1 ? x : x << 16) >= thr;
}

// 8 elements as fp32.  WIDE: fp32 as one 256-bit access, else as two of 128 bits; bf16 is one of 128 either way.
template <bool BF, bool WIDE>
__device__ __forceinline__ Fv<8> load8(const void* base, long long e) {
    if constexpr (BF) {
        return widen<true, 8>(load_grad<true, 8>(base, e));
    } else if constexpr (WIDE) {
        return load_f32<8>((const float*)base + e);
    } else {
        const Fv<4> a = load_f32<4>((const float*)base + e), b = load_f32<4>((const float*)base + e + 4);
        Fv<8> o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.f[i] = i < 4 ? a.f[i & 3] : b.f[i & 3];
        return o;
    }
}
template <bool BF, bool WIDE>
__device__ __forceinline__ void store8(void* base, long long e, const Fv<8>& x) {
    if constexpr (BF) {
        store_bf16<8>((unsigned short*)base + e, x);
    } else if constexpr (WIDE) {
        store_f32<8>((float*)base + e, x);
    } else {
        store_f32<4>((float*)base + e, Fv<4>{x.f[0], x.f[1], x.f[2], x.f[3]});
        store_f32<4>((float*)base + e + 4, Fv<4>{x.f[4], x.f[5], x.f[6], x.f[7]});
    }
}
template <bool BF>
__device__ __forceinline__ void store8_partial(void* base, long long e, const Fv<8>& x, int n) {
    if constexpr (BF) store_bf16_partial<8>((unsigned short*)base + e, x, n);
    else store_f32_partial<8>((float*)base + e, x, n);
}

// What a launch's item is: its tile, where it lies in `flat` and in the tensor.
struct DropItem {
    long long flat0;     // first element in `flat`
    long long elem0;     // ... in the tensor, a multiple of 8
    long long nvalid;    // elements that exist in the tensor
    int nvec, seg;
    bool ok;
};
__device__ __forceinline__ DropItem item_of(const DropParams& P, long long item) {
    DropItem d;
    const long long r = P.concat ? 0 : item / P.ntl;             // shard, counted from r0
    const WsTile tl = P.tiles[P.tile_lo + (item - r * P.ntl)];
    const long long shard = P.concat ? tl.shard : P.r0 + r;
    d.flat0 = (shard - P.r0) * P.S + tl.pos;
    d.elem0 = shard * tl.piece + tl.poff;
    const long long nv = tl.vt - shard * tl.piece;
    d.nvalid = nv < 0 ? 0 : nv > tl.len ? (long long)tl.len : nv;
    d.nvec = tl.len >> 3;
    d.seg = tl.seg;
    d.ok = true;
#ifdef WS_DEBUG_BOUNDS
    if (d.flat0 < 0 || d.flat0 + tl.len > P.flat_elems) {
        if ((threadIdx.x & 31) == 0 && P.bounds) atomicOr(P.bounds, (unsigned)WS_BOUNDS_FLAT);
        d.ok = false;
    }
#endif
    return d;
}

// FBF, TBF: flat buffer, tensors in bf16.  SHORT: a warp per tile, else a CTA.
template <bool FBF, bool TBF, bool WIDE, bool SHORT>
__global__ void __launch_bounds__(256) hand_out_kernel(const __grid_constant__ DropParams P, const void* __restrict__ flat) {
    asm volatile("griddepcontrol.launch_dependents;");
    const int per_cta = SHORT ? blockDim.x >> 5 : 1;
    const int first = SHORT ? threadIdx.x & 31 : threadIdx.x, step = SHORT ? 32 : blockDim.x;
    for (long long item = (long long)blockIdx.x * per_cta + (SHORT ? threadIdx.x >> 5 : 0); item < P.nitems; item += (long long)gridDim.x * per_cta) {
        const DropItem d = item_of(P, item);
        const void* const* sets = P.table + (long long)d.seg * P.nsets;
        // plan and pointer tables were uploaded before; the previous kernel of the stream may own the data
        asm volatile("griddepcontrol.wait;" ::: "memory");
        if (!d.ok) continue;
        const unsigned now = P.step + (P.step_dev ? *P.step_dev : 0u);
        for (int i = first; i < d.nvec; i += step) {
            const long long have = d.nvalid - 8LL * i;
            if (have <= 0) break;
            Fv<8> x = load8<FBF, WIDE>(flat, d.flat0 + 8LL * i);
#pragma unroll
            for (int e = 0; e < 8; ++e) x.f[e] *= P.scale;
            const long long j = (d.elem0 >> 3) + i;
            for (int k = 0; k < P.nsets; ++k) {
                const uint4 w = philox(P, (unsigned)j, now, (unsigned)d.seg, P.replica + k + ((unsigned)(j >> 32) << 16));
                Fv<8> y;
#pragma unroll
                for (int e = 0; e < 8; ++e) y.f[e] = kept(w, e, P.thr) ? x.f[e] : 0.f;
                void* t = const_cast<void*>(sets[k]);
                if (have >= 8) store8<TBF, WIDE>(t, 8 * j, y);
                else store8_partial<TBF>(t, 8 * j, y, (int)have);
            }
        }
    }
}

// Adds x to (s, c) with compensation, as kahan1, but an infinite sum stays infinite.
__device__ __forceinline__ void kahan_inf(float& s, float& c, float x) {
    const float y = x - c, t = s + y;
    c = fabsf(t) < INFINITY ? (t - s) - y : 0.f;
    s = t;
}

// The copies are summed in blocks of 4 whose loads are issued together; the blocks of more than 8 copies with compensation.
constexpr int kSumBlock = 4;
template <bool FBF, bool TBF, bool WIDE, bool SHORT>
__global__ void __launch_bounds__(256) sum_kernel(const __grid_constant__ DropParams P, void* __restrict__ flat) {
    asm volatile("griddepcontrol.launch_dependents;");
    const int per_cta = SHORT ? blockDim.x >> 5 : 1;
    const int first = SHORT ? threadIdx.x & 31 : threadIdx.x, step = SHORT ? 32 : blockDim.x;
    for (long long item = (long long)blockIdx.x * per_cta + (SHORT ? threadIdx.x >> 5 : 0); item < P.nitems; item += (long long)gridDim.x * per_cta) {
        const DropItem d = item_of(P, item);
        const void* const* sets = P.table + (long long)d.seg * P.nsets;
        asm volatile("griddepcontrol.wait;" ::: "memory");
        if (!d.ok) continue;
        const unsigned now = P.step + (P.step_dev ? *P.step_dev : 0u);
        for (int i = first; i < d.nvec; i += step) {
            const long long have = d.nvalid - 8LL * i;
            const long long j = (d.elem0 >> 3) + i;
            Fv<8> sum, comp;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum.f[e] = comp.f[e] = 0.f;
            for (int k0 = 0; have > 0 && k0 < P.nsets; k0 += kSumBlock) {
                GradRaw<TBF, 8> raw[kSumBlock];
#pragma unroll
                for (int q = 0; q < kSumBlock; ++q) {
                    const int k = k0 + q < P.nsets ? k0 + q : k0;
                    if (have >= 8) {
                        if constexpr (TBF) {
                            raw[q] = load_grad<true, 8>(sets[k], 8 * j);
                        } else {
                            const Fv<8> v = load8<false, WIDE>(sets[k], 8 * j);
#pragma unroll
                            for (int e = 0; e < 8; ++e) raw[q].f[e] = v.f[e];
                        }
                    } else {
                        raw[q] = load_grad_partial<TBF, 8>(sets[k], 8 * j, (int)have);
                    }
                }
                Fv<8> block;
#pragma unroll
                for (int q = 0; q < kSumBlock; ++q) {
                    const uint4 w = philox(P, (unsigned)j, now, (unsigned)d.seg, P.replica + k0 + q + ((unsigned)(j >> 32) << 16));
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float v = k0 + q < P.nsets && kept(w, e, P.thr) ? raw_elem<TBF, 8>(raw[q], e) : 0.f;
                        block.f[e] = q == 0 ? v : block.f[e] + v;
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (P.nsets > 8) kahan_inf(sum.f[e], comp.f[e], block.f[e]);
                    else sum.f[e] += block.f[e];
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum.f[e] = e < have ? sum.f[e] * P.scale : 0.f;
            store8<FBF, WIDE>(flat, d.flat0 + 8LL * i, sum);
        }
    }
}

template <typename... KArgs, typename... Args>
void launch(void (*kernel)(KArgs...), long long grid, int block, cudaStream_t st, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)block);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}

template <bool FBF, bool TBF, bool WIDE, bool SHORT>
void launch_op(bool sum, void* flat, long long grid, int threads, cudaStream_t st, const DropParams& P) {
    if (sum) launch(sum_kernel<FBF, TBF, WIDE, SHORT>, grid, threads, st, P, flat);
    else launch(hand_out_kernel<FBF, TBF, WIDE, SHORT>, grid, threads, st, P, (const void*)flat);
}
template <bool FBF, bool TBF>
void launch_types(bool sum, bool wide, bool is_short, void* flat, long long grid, int threads, cudaStream_t st, const DropParams& P) {
    if constexpr (FBF && TBF) {         // no fp32 access: WIDE says nothing
        (is_short ? launch_op<FBF, TBF, true, true> : launch_op<FBF, TBF, true, false>)(sum, flat, grid, threads, st, P);
    } else {
        if (wide) (is_short ? launch_op<FBF, TBF, true, true> : launch_op<FBF, TBF, true, false>)(sum, flat, grid, threads, st, P);
        else (is_short ? launch_op<FBF, TBF, false, true> : launch_op<FBF, TBF, false, false>)(sum, flat, grid, threads, st, P);
    }
}

ws_status run(bool sum, const ws_plan* p, int32_t r, void* flat, ws_dtype flat_dtype, const ws_tensor_table* table, const ws_dropout* drop,
              void* stream) {
    if (!p || !flat || !table || !table->dev || !drop) return WS_ERR_INVALID_ARG;
    if (r < -1 || r >= p->R) return WS_ERR_INVALID_ARG;
    if (table->T != p->T || table->nsets < 1 || table->nsets > 1024) return WS_ERR_INVALID_ARG;
    if (!(drop->p >= 0.0 && drop->p < 1.0)) return WS_ERR_INVALID_ARG;      // (refuses NaN)
    if (drop->replica < 0 || (long long)drop->replica + table->nsets > 65536) return WS_ERR_INVALID_ARG;
    if ((flat_dtype != WS_F32 && flat_dtype != WS_BF16) || (table->dtype != WS_F32 && table->dtype != WS_BF16)) return WS_ERR_DTYPE;
    if (!p->d_tiles) return WS_ERR_NOT_UPLOADED;
    if (!ws_aligned16(flat) || (reinterpret_cast<uintptr_t>(drop->step_dev) & 3u) != 0) return WS_ERR_ALIGNMENT;
    DropParams P = {};
    P.tiles = p->d_tiles;
    P.S = p->S;
    P.concat = p->layout == WS_LAYOUT_CONCAT;
    P.r0 = r < 0 ? 0 : r;
    if (P.concat) {
        P.tile_lo = r < 0 ? 0 : p->shard_tile_begin[r];
        P.nitems = P.ntl = (r < 0 ? p->ntiles : p->shard_tile_begin[r + 1]) - P.tile_lo;
    } else {
        P.ntl = p->ntiles;
        P.nitems = p->ntiles * (r < 0 ? p->R : 1);
    }
    if (P.nitems < 1) return WS_OK;
    P.table = (const void* const*)table->dev;
    P.nsets = table->nsets;
    for (int i = 0; i < kRounds; ++i) {
        P.key[2 * i] = (unsigned)drop->seed + i * 0x9E3779B9u;
        P.key[2 * i + 1] = (unsigned)(drop->seed >> 32) + i * 0xBB67AE85u;
    }
    const double t = floor(drop->p * 65536.0 + 0.5);
    const unsigned dropped = t < 65535.0 ? (unsigned)t : 65535u;
    P.thr = dropped << 16;
    P.scale = (float)(65536.0 / (65536.0 - dropped));
    P.step = drop->step;
    P.step_dev = drop->step_dev;
    P.replica = (unsigned)drop->replica;
#ifdef WS_DEBUG_BOUNDS
    P.bounds = ws_bounds_word();
    P.flat_elems = (r < 0 ? (long long)p->R : 1) * p->S;
#endif
    const bool wide = table->min_align >= 32 && (reinterpret_cast<uintptr_t>(flat) & 31u) == 0;
    // a warp per tile where tiles are short (ws_pack's rule, in elements of the wider type)
    const long long tile = p->ntiles > 0 ? (P.concat ? p->S * p->R : p->S) / p->ntiles : p->K;
    const bool is_short = P.nitems > 32LL * p->sms && tile <= 768 && p->longest <= 128 << 10;
    int threads = is_short ? 128 : 256;
    while (!is_short && threads > 64 && p->K / 8 < 2 * threads) threads >>= 1;
    const int per_cta = is_short ? threads / 32 : 1;
    long long grid = (P.nitems + per_cta - 1) / per_cta;
    if (grid > 0x7fffffffLL) grid = 0x7fffffffLL;
    cudaStream_t st = (cudaStream_t)stream;
    if (flat_dtype == WS_BF16) (table->dtype == WS_BF16 ? launch_types<true, true> : launch_types<true, false>)(sum, wide, is_short, flat, grid, threads, st, P);
    else (table->dtype == WS_BF16 ? launch_types<false, true> : launch_types<false, false>)(sum, wide, is_short, flat, grid, threads, st, P);
    return ws_check_launch(sum ? "ws_reduce_dropout" : "ws_unpack_dropout");
}

}  // namespace

extern "C" ws_status ws_unpack_dropout(const ws_plan* plan, int32_t r, const void* flat, ws_dtype flat_dtype, const ws_tensor_table* lists,
                                       const ws_dropout* drop, void* stream) {
    WsRange range_("ws_unpack_dropout");
    return run(false, plan, r, const_cast<void*>(flat), flat_dtype, lists, drop, stream);
}

extern "C" ws_status ws_reduce_dropout(const ws_plan* plan, int32_t r, const ws_tensor_table* grads, const ws_dropout* drop, void* flat,
                                       ws_dtype flat_dtype, void* stream) {
    WsRange range_("ws_reduce_dropout");
    return run(true, plan, r, flat, flat_dtype, grads, drop, stream);
}

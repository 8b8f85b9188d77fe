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

// sum += x where element i of the block is kept: an addition under a predicate, without a choice in front of it (the
// integer and choice instructions are what these kernels have most of).
__device__ __forceinline__ void add_kept(float& sum, float x, const uint4& w, int i, unsigned thr) {
    const unsigned h = i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w;
    asm("{\n\t.reg .pred p;\n\tsetp.ge.u32 p, %1, %2;\n\t@p add.f32 %0, %0, %3;\n\t}" : "+f"(sum) : "r"(i & 1 ? h : h << 16), "r"(thr), "f"(x));
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

// What a launch's item is: its tile, where it lies in `flat` and in the tensor.
struct DropItem {
    long long flat0;     // first element in `flat`
    long long block0;    // first run of 8 elements in the tensor
    int nvalid;          // elements that exist in the tensor
    int nvec, seg;
    bool ok;
};
__device__ __forceinline__ DropItem item_of(const DropParams& P, long long item) {
    DropItem d;
    // shard, counted from r0 (a division of 64 bits is a tenth of a tile's instructions)
    const long long r = P.concat ? 0 : P.nitems <= 0xffffffffLL ? (long long)((unsigned)item / (unsigned)P.ntl) : item / P.ntl;
    const WsTile tl = P.tiles[P.tile_lo + (item - r * P.ntl)];
    const long long shard = P.concat ? tl.shard : P.r0 + r;
    d.flat0 = (shard - P.r0) * P.S + tl.pos;
    d.block0 = (shard * tl.piece + tl.poff) >> 3;
    const long long nv = tl.vt - shard * tl.piece;
    d.nvalid = nv < 0 ? 0 : nv > tl.len ? tl.len : (int)nv;
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
__device__ __forceinline__ uint4 block_of(const DropParams& P, const DropItem& d, int i, unsigned now, int k) {
    const long long j = d.block0 + i;
    return philox(P, (unsigned)j, now, (unsigned)d.seg, P.replica + k + ((unsigned)(j >> 32) << 16));
}

// 8 scaled elements as they are stored; `masked` of them: the dropped ones 0.
template <bool TBF>
struct Copy {
    Fv<8> x;
    __device__ __forceinline__ explicit Copy(const Fv<8>& v) : x(v) {}
    __device__ __forceinline__ Copy masked(const uint4& w, unsigned thr) const {
        Copy y(*this);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (!kept(w, e, thr)) y.x.f[e] = 0.f;
        return y;
    }
    template <bool WIDE>
    __device__ __forceinline__ void store(void* t, long long e) const { store8<false, WIDE>(t, e, x); }
    __device__ __forceinline__ void store(void* t, long long e, int n) const { store_f32_partial<8>((float*)t + e, x, n); }
};
template <>
struct Copy<true> {                // rounded once, whatever the number of sets
    unsigned x[4];
    __device__ __forceinline__ explicit Copy(const Fv<8>& v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v.f[2 * i], v.f[2 * i + 1]);
            x[i] = *reinterpret_cast<const unsigned*>(&b);
        }
    }
    __device__ __forceinline__ Copy masked(const uint4& w, unsigned thr) const {
        Copy y(*this);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!kept(w, 2 * i, thr)) y.x[i] &= 0xffff0000u;
            if (!kept(w, 2 * i + 1, thr)) y.x[i] &= 0x0000ffffu;
        }
        return y;
    }
    template <bool WIDE>
    __device__ __forceinline__ void store(void* t, long long e) const {
        __stcs(reinterpret_cast<uint4*>((unsigned short*)t + e), make_uint4(x[0], x[1], x[2], x[3]));
    }
    __device__ __forceinline__ void store(void* t, long long e, int n) const {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) ((unsigned short*)t)[e + i] = (unsigned short)(i & 1 ? x[i / 2] >> 16 : x[i / 2]);
    }
};

// Hands U vectors, i, i + step, ..., out to every set; FULL: all their elements exist.
template <bool FBF, bool TBF, bool WIDE, int U, bool FULL>
__device__ __forceinline__ void hand_out(const DropParams& P, const DropItem& d, const void* flat, const void* const* sets, int i, int step, unsigned now) {
    Fv<8> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = load8<FBF, WIDE>(flat, d.flat0 + 8LL * (i + u * step));
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[u].f[e] *= P.scale;
#pragma unroll 1
    for (int k = 0; k < P.nsets; ++k) {
        void* t = const_cast<void*>(sets[k]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int iu = i + u * step;
            const Copy<TBF> y = Copy<TBF>(x[u]).masked(block_of(P, d, iu, now, k), P.thr);
            if (FULL) y.template store<WIDE>(t, 8 * (d.block0 + iu));
            else y.store(t, 8 * (d.block0 + iu), d.nvalid - 8 * iu);
        }
    }
}

// FBF, TBF: flat buffer, tensors in bf16.  SHORT: a warp per tile, else a CTA.  A thread holds U vectors of its tile, whose
// loads are issued together, and writes them to one set after the other.
template <bool FBF, bool TBF, bool WIDE, bool SHORT, int U, int MINB>
__global__ void __launch_bounds__(256, MINB) hand_out_kernel(const __grid_constant__ DropParams P, const void* __restrict__ flat) {
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
        const int full = d.nvalid >> 3;
        int i = first;
        for (; i + (U - 1) * step < full; i += U * step) hand_out<FBF, TBF, WIDE, U, true>(P, d, flat, sets, i, step, now);
        if (U > 1)
#pragma unroll 1
            for (; i < full; i += step) hand_out<FBF, TBF, WIDE, 1, true>(P, d, flat, sets, i, step, now);
        if (i == full && (d.nvalid & 7)) hand_out<FBF, TBF, WIDE, 1, false>(P, d, flat, sets, i, step, now);       // the tensor's last elements
    }
}

// Adds x to (s, c) with compensation, as kahan1, but an infinite sum stays infinite.
__device__ __forceinline__ void kahan_inf(float& s, float& c, float x) {
    const float y = x - c, t = s + y;
    c = fabsf(t) < INFINITY ? (t - s) - y : 0.f;
    s = t;
}

// Sums U vectors, i, i + step, ..., of all sets.  The copies are taken in blocks of KB whose loads are issued together;
// COMP: more than 8 copies, whose blocks are added with compensation.
template <bool FBF, bool TBF, bool WIDE, int KB, int U, bool COMP, bool FULL>
__device__ __forceinline__ void sum_up(const DropParams& P, const DropItem& d, void* flat, const void* const* sets, int i, int step, unsigned now) {
    Fv<8> sum[U], comp[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[u].f[e] = comp[u].f[e] = 0.f;
#pragma unroll 1
    for (int k0 = 0; k0 < P.nsets; k0 += KB) {
        GradRaw<TBF, 8> raw[U][KB];
#pragma unroll
        for (int q = 0; q < KB; ++q) {
            if (KB > 1 && k0 + q >= P.nsets) break;
            const void* g = sets[k0 + q];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int iu = i + u * step;
                if constexpr (!FULL) {
                    raw[u][q] = load_grad_partial<TBF, 8>(g, 8 * (d.block0 + iu), d.nvalid - 8 * iu);
                } else if constexpr (TBF) {
                    raw[u][q] = load_grad<true, 8>(g, 8 * (d.block0 + iu));
                } else {
                    const Fv<8> v = load8<false, WIDE>(g, 8 * (d.block0 + iu));
#pragma unroll
                    for (int e = 0; e < 8; ++e) raw[u][q].f[e] = v.f[e];
                }
            }
        }
        Fv<8> block[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) block[u].f[e] = COMP ? 0.f : sum[u].f[e];
#pragma unroll
        for (int q = 0; q < KB; ++q) {
            if (KB > 1 && k0 + q >= P.nsets) break;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint4 w = block_of(P, d, i + u * step, now, k0 + q);
#pragma unroll
                for (int e = 0; e < 8; ++e) add_kept(block[u].f[e], raw_elem<TBF, 8>(raw[u][q], e), w, e, P.thr);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (COMP) kahan_inf(sum[u].f[e], comp[u].f[e], block[u].f[e]);
                else sum[u].f[e] = block[u].f[e];
            }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int iu = i + u * step, have = d.nvalid - 8 * iu;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[u].f[e] = FULL || e < have ? sum[u].f[e] * P.scale : 0.f;
        store8<FBF, WIDE>(flat, d.flat0 + 8LL * iu, sum[u]);
    }
}

template <bool FBF, bool TBF, bool WIDE, bool SHORT, int KB, int U, bool COMP, int MINB>
__global__ void __launch_bounds__(256, MINB) sum_kernel(const __grid_constant__ DropParams P, void* __restrict__ flat) {
    asm volatile("griddepcontrol.launch_dependents;");
    const int per_cta = SHORT ? blockDim.x >> 5 : 1;
    const int first = SHORT ? threadIdx.x & 31 : threadIdx.x, step = SHORT ? 32 : blockDim.x;
    for (long long item = (long long)blockIdx.x * per_cta + (SHORT ? threadIdx.x >> 5 : 0); item < P.nitems; item += (long long)gridDim.x * per_cta) {
        const DropItem d = item_of(P, item);
        const void* const* sets = P.table + (long long)d.seg * P.nsets;
        asm volatile("griddepcontrol.wait;" ::: "memory");
        if (!d.ok) continue;
        const unsigned now = P.step + (P.step_dev ? *P.step_dev : 0u);
        const int full = d.nvalid >> 3;
        int i = first;
        for (; i + (U - 1) * step < full; i += U * step) sum_up<FBF, TBF, WIDE, KB, U, COMP, true>(P, d, flat, sets, i, step, now);
        if (U > 1)
#pragma unroll 1
            for (; i < full; i += step) sum_up<FBF, TBF, WIDE, KB, 1, COMP, true>(P, d, flat, sets, i, step, now);
        if (i == full && (d.nvalid & 7)) {          // the tensor's last elements
            sum_up<FBF, TBF, WIDE, 1, 1, COMP, false>(P, d, flat, sets, i, step, now);
            i += step;
        }
        for (; i < d.nvec; i += step) store8<FBF, WIDE>(flat, d.flat0 + 8LL * i, Fv<8>{});             // padding
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

// How a call's tiles are cut up: tiles, elements of the plan's tile and of the average one, a warp per tile or a CTA.
struct Shape {
    long long items;
    int tile;
    long long average;
    bool is_short;
};
// CTAs of `most` threads, fewer where a tile would not give each of them `unroll` vectors.
template <typename Kernel, typename Flat>
void launch_tiles(Kernel kernel, const Shape& s, int most, int unroll, cudaStream_t st, const DropParams& P, Flat flat) {
    int threads = s.is_short ? 128 : most;
    while (!s.is_short && threads > 32 && s.tile / 8 < unroll * threads) threads >>= 1;
    const int per_cta = s.is_short ? threads / 32 : 1;
    const long long grid = (s.items + per_cta - 1) / per_cta;
    launch(kernel, grid < 0x7fffffffLL ? grid : 0x7fffffffLL, threads, st, P, flat);
}

// Drawing the masks is what these kernels do beside the copy: 14 products of 32 x 32 bits and as many three-way exclusive ors
// per block of 8 elements and set, and a comparison and a choice per element.  On bf16 tensors that is 10 instructions an
// element, half of them of the integer pipe's half rate, near what the copy leaves time for; fp32 tensors have twice the time.
// So small CTAs (a long tile's latencies overlap with other tiles'), registers for many of them, no more loads in flight than
// that needs.  us in runs of 0.6 s, whose power takes the SM clock from 1.96 GHz to 1.6 to 1.8, by threads of a CTA: 335 M elements
// from bf16 to one bf16 list 256 264, 128 241, 64 231 (205 at the copy bandwidth; 216 in runs of 60 ms); the sum of one bf16
// list 259 / 244 / 240, of 2 of 61 M 91 / 91 / 83 (75), of 4 of 1.56 G 3186 / 3116 / 3118 (2859); 4 bf16 lists from an fp32
// state of 451 M 960 / 883 / 908 (828).  With 3 CTAs of 256 an SM the sum of 4 lists takes 3378.  More than 8 bf16
// lists: blocks of 8 halve the compensation's steps, 16 lists of 61 M 476 -> 438 (338).
template <bool FBF, bool TBF, bool WIDE, bool SHORT>
void launch_op(bool sum, void* flat, const Shape& s, cudaStream_t st, const DropParams& P) {
    const void* from = flat;
    if (!sum) {
        // Four vectors in flight need tiles that have them; without, with many lists, a draw's latency is all there is (us, 4 / 1:
        // 16 lists of 2 M in 64 shards 50 / 29, in 16 shards 42 / 24, 3 lists of 45 M in 64 shards 70 / 74).
        if constexpr (FBF && TBF) {
            if (P.nsets <= 3 || s.average >= 1536) launch_tiles(hand_out_kernel<true, true, WIDE, SHORT, 4, 5>, s, 64, 4, st, P, from);
            else launch_tiles(hand_out_kernel<true, true, WIDE, SHORT, 1, 5>, s, 64, 1, st, P, from);
        } else if (P.nsets == 1) {
            launch_tiles(hand_out_kernel<FBF, TBF, WIDE, SHORT, 2, 3>, s, 64, 2, st, P, from);
        } else {
            launch_tiles(hand_out_kernel<FBF, TBF, WIDE, SHORT, 2, 1>, s, 128, 2, st, P, from);
        }
    } else if (P.nsets == 1) {
        launch_tiles(sum_kernel<FBF, TBF, WIDE, SHORT, 1, 2, false, TBF ? 5 : 4>, s, 64, 2, st, P, flat);
    } else if (P.nsets == 2) {
        launch_tiles(sum_kernel<FBF, TBF, WIDE, SHORT, 2, TBF ? 2 : 1, false, 4>, s, 64, TBF ? 2 : 1, st, P, flat);
    } else if (P.nsets <= 8) {
        launch_tiles(sum_kernel<FBF, TBF, WIDE, SHORT, 4, 1, false, TBF ? 6 : 3>, s, 128, 1, st, P, flat);
    } else {
        launch_tiles(sum_kernel<FBF, TBF, WIDE, SHORT, TBF ? 8 : 4, 1, true, TBF ? 3 : 4>, s, TBF ? 64 : 128, 1, st, P, flat);
    }
}
template <bool FBF, bool TBF>
void launch_types(bool sum, bool wide, void* flat, const Shape& s, cudaStream_t st, const DropParams& P) {
    if constexpr (FBF && TBF) {         // no fp32 access: WIDE says nothing
        (s.is_short ? launch_op<FBF, TBF, true, true> : launch_op<FBF, TBF, true, false>)(sum, flat, s, st, P);
    } else {
        if (wide) (s.is_short ? launch_op<FBF, TBF, true, true> : launch_op<FBF, TBF, true, false>)(sum, flat, s, st, P);
        else (s.is_short ? launch_op<FBF, TBF, false, true> : launch_op<FBF, TBF, false, false>)(sum, flat, s, st, P);
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
    // A warp per tile where tiles are short and many, and not long enough in any place to leave a warp walking alone (ws_pack's
    // rule, in elements).  us, a CTA / a warp per tile: 64 shards of 47 M in tiles of 900, sum of one bf16 list 56 / 42, fp32 to one
    // list 64 / 61; 16 bf16 lists of 4 M in tiles of 660, whose draws are enough work for a CTA, 42 / 53, 8 of 2 M 15 / 22.
    const long long tile = p->ntiles > 0 ? (P.concat ? p->S * p->R : p->S) / p->ntiles : p->K;
    const Shape s{P.nitems, p->K, tile, P.nitems > 32LL * p->sms && tile <= (P.nsets <= 2 ? 1024 : P.nsets <= 4 ? 768 : 256) && p->longest <= 128 << 10};
    cudaStream_t st = (cudaStream_t)stream;
    if (flat_dtype == WS_BF16) (table->dtype == WS_BF16 ? launch_types<true, true> : launch_types<true, false>)(sum, wide, flat, s, st, P);
    else (table->dtype == WS_BF16 ? launch_types<false, true> : launch_types<false, false>)(sum, wide, flat, s, st, P);
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

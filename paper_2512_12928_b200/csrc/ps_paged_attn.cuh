// The frame of the attention of one new token per row over a paged cache whose lengths and block tables are on the
// device: how the work is cut, the walk over a share's tiles, softmax states, segment ends and the join.  What a tile is
// (its types, how it comes to shared memory and is multiplied) is a Worker's matter: ps_paged_attn.cu has one for caches of
// 16 bits, ps_quant_attn.cu one for 8 bits.
//
// Softmax: the reference m of a head is raised only when a score exceeds it by more than kSlack, so that a tile needs
// one vote instead of a maximum over the lanes; weights stay below 2^kSlack and sums in 32 bits lose nothing by it.
//
// Work: the rows' tiles form one sequence (with two places more for each row's start and end, which cost about two tiles'
// time) that is cut into equal shares, one per CTA, from the lengths each CTA reads itself: no plan is made on the host or
// by another kernel.  A row cut by a share's end leaves partial results (m, sum, accumulators) in the workspace, which a
// second kernel (paged_join_kernel) combines in order.  The join is a second launch rather than a last-arrival counter in
// the first: the workspace then needs no initial state, and neither a replayed graph nor a call that shares it in turn can
// find a stale counter.  It is launched early, but its CTAs (64 registers a thread) do not fit beside one of the first
// kernel (8 warps of 199 to 251 registers a thread, or 16 of 128), so they start as those leave.
//
// Warps: a CTA works on `units` (KV head, group of at most 16 query heads) times `subs` token slices (a power of two);
// the units of a token are neighbours in memory.  The slices' states are combined through shared memory at a segment's
// end, where only a unit's own warps wait for one another.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdio>
#include <type_traits>

#include "ps_internal.h"
#include "ps_kvswap.h"

namespace {

constexpr int kMaxUnits = 8;          // of a CTA
constexpr int kMaxGroup = 16;         // query heads of a unit
constexpr int kJoinThreads = 256;
constexpr int32_t kMaxTokens = INT32_MAX - 1024;   // of a row, so that a tile's end cannot wrap
constexpr int kStatusBadId = 2, kStatusLength = 5;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;

struct AttnParams {
    const void *kpool, *vpool, *q;
    void* out;
    float* lse;
    const int32_t* tables;
    const int32_t* ctx;
    int32_t* status;
    float* part_o;       // [cta][2][unit][row][D]
    float2* part_ml;     // [cta][2][unit][row]
    int4* cuts;          // [cta]: the segment that this CTA did not finish: {row, chunk, parts, first CTA}; parts 0: none
    int64_t k_block_stride, v_block_stride, q_stride, out_stride;
    const float *k_scale, *v_scale;  // of an 8-bit cache: [block][KV head]
    uint32_t k_step, v_step, row_step;         // from block to block and token to token, in steps of 16 bytes
    uint32_t k_scale_step, v_scale_step;       // from block to block, in bytes
    bool near;                       // both pools have one step, and 32 bits count a pool's steps
    int64_t room;        // tokens a table row has room for
    uint64_t block_magic;
    int32_t batch, table_stride, num_blocks, block_size, window;
    int32_t hkv, hq, group;          // group: query heads per KV head
    int32_t splits, rows;            // a KV head's query heads are cut into `splits` units of `rows` heads
    int32_t units, chunks, subs;     // units per CTA, CTAs' worth of units per row, token slices
    int32_t ctas;                    // of the main kernel
    int32_t step_log2;               // tokens of a tile of all slices
    int32_t segment;                 // places that a segment's start and end take in the sequence that is shared out
    float scale_log2e;
};

// ------------------------------------------------------------------------------------------------ pieces

template <typename T> struct Num;
template <> struct Num<__nv_bfloat16> {
    static constexpr float kLift = 0.f, kSlack = 8.f;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
    static __device__ __forceinline__ void mma(float (&d)[4], const uint4& a, uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
    }
};
template <> struct Num<__half> {
    // p is rounded to fp16 for the product with V, and fp16 loses relative precision below 2^-14.  So p is computed
    // 2^kLift times larger (the sum carries the same factor, and both cancel): at most 2^(kLift + kSlack) = 2^14.
    static constexpr float kLift = 8.f, kSlack = 6.f;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
    static __device__ __forceinline__ void mma(float (&d)[4], const uint4& a, uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
    }
};

__device__ __forceinline__ uint4 ldsm(uint32_t a) {
    uint4 v;
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint4 ldsm_t(uint32_t a) {
    uint4 v;
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
// 16 bytes to shared memory, read once; zeros where bytes is 0, and then src is not read
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint32_t bytes, uint64_t policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src), "r"(bytes), "l"(policy)
                 : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {   // all but the newest N groups have landed
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint64_t read_once_policy() {
    uint64_t pol;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
    return pol;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// t / block_size for 0 <= t < 2^31: magic is 2^64 / block_size rounded up (block_size > 1)
__device__ __forceinline__ int32_t block_of(int32_t t, const AttnParams& p) {
    const uint32_t low = __umulhi((uint32_t)t, (uint32_t)p.block_magic);
    return p.block_size == 1 ? t : (int32_t)((t * (uint64_t)(uint32_t)(p.block_magic >> 32) + low) >> 32);
}

// Tokens that are attended of a row of n: [first, end).
__device__ __forceinline__ void row_span(const AttnParams& p, int32_t n, int32_t* first, int32_t* end) {
    const int32_t e = (int64_t)n > p.room ? (int32_t)p.room : max(n, 0);
    *end = e;
    *first = p.window > 0 && e > p.window ? e - p.window : 0;
}
// Tiles of a row of n; an empty row still has a result to write.
__device__ __forceinline__ int32_t row_tiles(const AttnParams& p, int32_t n) {
    int32_t first, end;
    row_span(p, n, &first, &end);
    return end > first ? (end - first + (1 << p.step_log2) - 1) >> p.step_log2 : 1;
}

// Where a unit's queries are: heads [h0, h0 + n).
__device__ __forceinline__ void unit_heads(const AttnParams& p, int unit, int* kv, int* h0, int* n) {
    *kv = p.splits == 1 ? unit : unit / p.splits;
    const int s = unit - *kv * p.splits;
    *h0 = *kv * p.group + s * p.rows;
    *n = min(p.rows, p.group - s * p.rows);
}

// A segment is a row and a chunk of units.  It takes p.segment places of the sequence that is cut into shares for its start
// and end, then one for each of its tiles.  What a share has of one:
struct Part {
    int32_t b, chunk;
    int32_t h0, n;                           // the warp's unit: query heads [h0, h0 + n)
    int32_t lo, count, tiles;                // tiles [lo, lo + count) of the segment's
    int32_t base;                            // place of the segment's first tile
};

// The tiles of a CTA's share, one after the other, as they are requested.
struct Walk {
    int32_t b, chunk, len;                   // row b of len tokens
    int32_t next_len;                        // of row b + 1, asked for while row b is worked on
    int32_t t, end;                          // the next tile's first token, and where the row's end
    int32_t left;                            // tiles of the segment still to be requested; 0: of the share
    int32_t place;                           // where the next segment's first tile is
    __device__ __forceinline__ void look_ahead(const AttnParams& p) { next_len = b + 1 < p.batch ? p.ctx[b + 1] : 0; }
    // Begins with tile i of the segment, at a place before share_end.
    __device__ __forceinline__ Part enter(const AttnParams& p, int32_t i, int32_t at, int32_t share_end) {
        int32_t first;
        row_span(p, len, &first, &end);
        if (end != len && p.status) *(volatile int32_t*)p.status = kStatusLength;
        const int32_t tiles = row_tiles(p, len);
        t = first + (i << p.step_log2);
        left = min(tiles - i, share_end - at);
        place = at - i + tiles + p.segment;
        return {b, chunk, 0, 0, i, left, tiles, at - i};
    }
    // To the next segment, whose first tile is before the share's end.
    __device__ __forceinline__ void step(const AttnParams& p) {
        if (++chunk < p.chunks) return;
        chunk = 0;
        ++b;
        len = next_len;
        look_ahead(p);
    }
};

// The softmax state of a warp.  Lane (g = lane / 4, c = lane % 4) holds heads 8 t + 2 c and 8 t + 2 c + 1 of column tile t:
// the reference m of the weights p = 2^(s - m), the sum over the tokens it has seen itself, and acc[t][j] = dims
// 16 j + g of both heads, dims 16 j + 8 + g of both.  m is kNothing before the first token: finite, so that
// differences from it are never NaN, and as a reference as good as any for scores as low as that.
constexpr float kNothing = -3.0e38f;
template <int D, int NT>
struct State {
    float m[NT][2], l[NT][2];
    float acc[NT][D / 16][4];
};

template <int D, int NT>
__device__ __forceinline__ void state_reset(State<D, NT>& st) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            st.m[t][h] = kNothing;
            st.l[t][h] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) st.acc[t][j][i] = 0.f;
    }
}

__device__ __forceinline__ float weight_for(float m, float top) { return m == top ? 1.f : ex2(m - top); }
__device__ __forceinline__ float inverse_sum(float l) { return l > 0.f ? 1.f / l : l == 0.f ? 0.f : CUDART_NAN_F; }
template <typename T>
__device__ __forceinline__ float natural_log_sum(float m, float l) {
    return l == 0.f ? -CUDART_INF_F : (m - Num<T>::kLift + log2f(l)) * kLn2;
}
template <typename T>
__device__ __forceinline__ void store4(T* dst, const float4& o, float f) {
    uint2 w;
    w.x = Num<T>::pack(o.x * f, o.y * f);
    w.y = Num<T>::pack(o.z * f, o.w * f);
    *reinterpret_cast<uint2*>(dst) = w;
}

// -------------------------------------------------------------------------------------------- main kernel

// A barrier of a unit's warps; other units go their own way.
__device__ __forceinline__ void slices_meet(const AttnParams& p, int unit_in_cta) {
    if (p.subs > 1) asm volatile("bar.sync %0, %1;" ::"r"(1 + unit_in_cta), "r"(32 * p.subs) : "memory");
    else __syncwarp();
}

template <typename W>
__global__ void __launch_bounds__(W::kWarps * 32, 1)
paged_attn_kernel(const __grid_constant__ AttnParams p) {
    constexpr int kMaxWarps = W::kWarps;
    using R = typename W::Stages;
    using T = typename W::Type;
    constexpr int D = W::kDim, NT = W::kColumns;
    extern __shared__ unsigned char smem_raw[];   // rings of the warps
    // the pieces' places are exclusive-ored within 128 bytes
    unsigned char* smem = smem_raw + (-(uint32_t)__cvta_generic_to_shared(smem_raw) & 127);
    __shared__ float2 sh_ml[kMaxWarps][8 * NT];
    __shared__ int sh_sum[kMaxWarps];
    __shared__ int4 sh_begin;          // where the share begins: row, chunk, tile; the row's length
    __shared__ int sh_place;
    constexpr int kParts = R::kStages + 1;   // those whose tiles are in the ring, or being attended, and one entered
    __shared__ Part sh_parts[kMaxWarps][kParts];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int nwarps = blockDim.x >> 5;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    W wk(p, (uint32_t)__cvta_generic_to_shared(smem));
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // This CTA's share of the sequence row 0 chunk 0, row 0 chunk 1, ..., row 1 chunk 0, ...
    const int per = (p.batch + blockDim.x - 1) / blockDim.x;
    const int b_lo = min(p.batch, (int)threadIdx.x * per), b_hi = min(p.batch, b_lo + per);
    int mine = 0, len = 0;
#pragma unroll 4
    for (int b = b_lo; b < b_hi; ++b) {
        len = p.ctx[b];
        mine += (row_tiles(p, len) + p.segment) * p.chunks;
    }
    int before = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int n = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += n;
    }
    if (lane == 31) sh_sum[warp] = before;
    __syncthreads();
    int sums = lane < nwarps ? sh_sum[lane] : 0;
#pragma unroll
    for (int o = 1; o < kMaxWarps; o <<= 1) {
        const int n = __shfl_up_sync(0xffffffffu, sums, o);
        if (lane >= o) sums += n;
    }
    const int total = __shfl_sync(0xffffffffu, sums, kMaxWarps - 1);
    const int earlier = __shfl_sync(0xffffffffu, sums, max(warp - 1, 0));
    before += (warp > 0 ? earlier : 0) - mine;
    const int share = (total + gridDim.x - 1) / gridDim.x;
    const int begin = share * blockIdx.x, end = min(total, begin + share);
    if (begin >= before && begin < before + mine) {
        int a = before, b = b_lo;                // and of a single row the length is still there
        if (per > 1)
#pragma unroll 1
            for (;; ++b) {
                len = p.ctx[b];
                const int n = (row_tiles(p, len) + p.segment) * p.chunks;
                if (begin < a + n) break;
                a += n;
            }
        const int tiles = row_tiles(p, len);
        int chunk = 0, i = begin - a;
        if (p.chunks > 1) {
            chunk = i / (tiles + p.segment);
            i -= chunk * (tiles + p.segment);
        }
        i = max(i - p.segment, 0);                // a share that begins in a segment's first places has its first tile
        sh_begin = make_int4(b, chunk, i, len);
        sh_place = a + chunk * (tiles + p.segment) + p.segment + i;
        // the first block ids, into L1 while the CTA meets
        int32_t first, last;
        row_span(p, len, &first, &last);
        const int32_t t = first + (i << p.step_log2);
        if (t < last) {
            uint32_t unused;
            asm volatile("ld.global.ca.b32 %0, [%1];" : "=r"(unused) : "l"(p.tables + (int64_t)b * p.table_stride + block_of(t, p)));
        }
    }
    __syncthreads();
    int4 cut = make_int4(0, 0, 0, 0);
    if (begin < end && sh_place < end) {         // else there is no tile in it
        Walk walk;                               // to the tile that is requested next
        int32_t parts = 0, part = 0;             // entered, and attended: parts part to parts - 1 wait in sh_parts
        auto enter = [&](int32_t i, int32_t at) {
            Part s = walk.enter(p, i, at, end);
            const int unit = s.chunk * p.units + wk.unit_in_cta;
            int kv = 0;
            if (unit < p.hkv * p.splits) unit_heads(p, unit, &kv, &s.h0, &s.n);      // else the unit does not exist: no heads
            wk.enter(s, kv);
            if (lane == 0) sh_parts[warp][parts % kParts] = s;
            ++parts;
        };
        const int4 start = sh_begin;
        walk.b = start.x;
        walk.chunk = start.y;
        walk.len = start.w;
        walk.look_ahead(p);
        enter(start.z, sh_place);
        wk.load_ids(walk.t, walk.end);
        int slot = 0;                            // stage that is filled next
        typename W::Softmax st;
        int32_t left = 0, due = 0;               // tiles of the part to be attended, and of those requested
#pragma unroll 1
        for (int fill = R::kStages - 1; walk.left > 0 || due > 0;) {
            copies_wait<R::kStages - 2>();
            __syncwarp();                        // the other lanes' copies too, and they have left the stage before
            const int filled = slot;             // the stage that the tile before left
            slot = slot + 1 == R::kStages ? 0 : slot + 1;       // the oldest
            const uint32_t on = wk.masks[0];
#pragma unroll
            for (int i = 0; i + 1 < R::kStages - 1; ++i) wk.masks[i] = wk.masks[i + 1];
            typename W::Keys k;
            wk.read_keys(slot, k);               // in the first rounds what it reads is not used
            if (walk.left > 0) {
                wk.masks[R::kStages - 2] = wk.copy_tile(filled);
                ++due;
                walk.t += 1 << p.step_log2;
                if (--walk.left == 0 && walk.place < end) {
                    walk.step(p);
                    enter(0, walk.place);
                }
                if (walk.left > 0) wk.load_ids(walk.t, walk.end);
            }
            copies_commit();
            if (fill > 0) {                      // the first rounds only fill the ring
                --fill;
                continue;
            }
            if (left == 0) {
                const Part& s = sh_parts[warp][part % kParts];
                left = s.count;
                wk.reset(st);
                wk.load_query(s.b, s.h0, s.n);
            }
            wk.attend(slot, k, on, st);
            --due;
            if (--left == 0) {
                const Part s = sh_parts[warp][part % kParts];
                ++part;
                const bool seg_end = s.lo + s.count == s.tiles;
                const int32_t h0 = s.h0, n = s.n, lo = s.lo;
                const bool whole = lo == 0 && seg_end;
                // The states of the slices go through the stage that has just been read, heads as rows, and come
                // back as rows of four dims a lane.  (The places' exclusive or keeps the writes free of conflicts.)
                float* own = reinterpret_cast<float*>(smem + warp * R::kWarpBytes + slot * R::kStageBytes);
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int r = 8 * t + 2 * wk.c + h;
                        wk.put_sums(own + r * D, st, t, h);
                        float l = st.l[t][h];
                        l += __shfl_xor_sync(0xffffffffu, l, 4);
                        l += __shfl_xor_sync(0xffffffffu, l, 8);
                        l += __shfl_xor_sync(0xffffffffu, l, 16);
                        if (wk.g == 0) sh_ml[warp][r] = make_float2(wk.reference(st, t, h), l);
                    }
                slices_meet(p, wk.unit_in_cta);
                constexpr int kLanes = D / 4, kHeads = 32 / kLanes;      // heads that a warp works on at a time
                const int dim = 4 * (lane % kLanes);
                auto put = [&](int r, const float4& o, float m, float l) {
                    if (whole) {
                        store4((T*)p.out + s.b * p.out_stride + (int64_t)(h0 + r) * D + dim, o, inverse_sum(l));
                        if (p.lse && dim == 0) p.lse[(int64_t)s.b * p.hq + h0 + r] = natural_log_sum<T>(m, l);
                    } else {
                        const int64_t part = (((int64_t)blockIdx.x * 2 + (lo == 0)) * p.units + wk.unit_in_cta) * p.rows + r;
                        *reinterpret_cast<float4*>(p.part_o + part * D + dim) = o;
                        if (dim == 0) p.part_ml[part] = make_float2(m, l);
                    }
                };
                auto get = [&](int w, int r) {
                    return *reinterpret_cast<const float4*>(smem + w * R::kWarpBytes + slot * R::kStageBytes +
                                                            4 * (r * D + (dim ^ (8 * (r >> 1 & 3)))));
                };
                if (p.subs == 1) {
#pragma unroll 4
                    for (int r = lane / kLanes; r < n; r += kHeads) put(r, get(warp, r), sh_ml[warp][r].x, sh_ml[warp][r].y);
                } else {
                    // eight parts are loaded at a time: of all slices of one, two or four heads
                    auto combine = [&](auto slices) {
                        constexpr int kSlices = decltype(slices)::value, kAtOnce = kSlices < 8 ? 8 / kSlices : 1;
                        constexpr int kStep = kSlices * kHeads;
#pragma unroll 1
                        for (int r0 = wk.sub * kHeads + lane / kLanes; r0 < n; r0 += kAtOnce * kStep) {
                            float m[kAtOnce], l[kAtOnce];
                            float4 o[kAtOnce];
#pragma unroll
                            for (int h = 0; h < kAtOnce; ++h) {
                                const int r = min(r0 + h * kStep, n - 1);
                                m[h] = kNothing;
                                l[h] = 0.f;
                                o[h] = make_float4(0.f, 0.f, 0.f, 0.f);
                                float2 ml[kSlices];
#pragma unroll
                                for (int i = 0; i < kSlices; ++i) {
                                    ml[i] = sh_ml[wk.unit_in_cta + i * p.units][r];
                                    m[h] = fmaxf(m[h], ml[i].x);
                                }
#pragma unroll
                                for (int i = 0; i < kSlices; ++i) {
                                    const float4 x = get(wk.unit_in_cta + i * p.units, r);
                                    const float f = weight_for(ml[i].x, m[h]);
                                    l[h] += ml[i].y * f;
                                    o[h].x += x.x * f;
                                    o[h].y += x.y * f;
                                    o[h].z += x.z * f;
                                    o[h].w += x.w * f;
                                }
                            }
#pragma unroll
                            for (int h = 0; h < kAtOnce; ++h)
                                if (r0 + h * kStep < n) put(r0 + h * kStep, o[h], m[h], l[h]);
                        }
                    };
                    if (p.subs == 2) combine(std::integral_constant<int, 2>());
                    else if (p.subs == 4) combine(std::integral_constant<int, 4>());
                    else if (kMaxWarps == 8 || p.subs == 8) combine(std::integral_constant<int, 8>());
                    else combine(std::integral_constant<int, kMaxWarps>());
                }
                slices_meet(p, wk.unit_in_cta);      // the stage is free again
                if (!seg_end) {
                    const int from = s.base / share;      // the CTAs of the segment's first and last tile
                    cut = make_int4(s.b, s.chunk, (s.base + s.tiles - 1) / share - from + 1, from);
                }
            }
        }
    }
    if (threadIdx.x == 0) p.cuts[blockIdx.x] = cut;
}

// Combines the parts of the rows that a share's end cut.  cuts[i] names the segment that CTA i of the main kernel did
// not finish: its row and chunk, its number of parts and the CTA that it begins in.  The parts are slot 1 of that CTA
// and slot 0 of those that follow.  The CTAs of all cuts of a segment share its work items, (unit, query head) pairs:
// nothing has to be counted or listed first.  What an item costs is latency, so its loads do not wait for one
// another: parts are requested while the weights are made from all parts' m.  Where a segment has as many CTAs to
// share it as items (a long row on much of the chip), an item is a CTA's, whose slices of D / 4 threads take every
// eighth or sixteenth part; else it is a warp's.  Sums are taken in a fixed order, so a result does not depend on timing.
template <typename T, int D>
struct Joiner {
    static constexpr int kLanes = D / 4;     // a lane owns 4 dims
    const AttnParams& p;
    int4 cut;                                // row, chunk, parts, first CTA
    int64_t slot0, step;
    int h0, r, per;

    __device__ __forceinline__ Joiner(const AttnParams& pp) : p(pp), per(pp.units * pp.rows) {}

    // Item k of a segment; false if that unit or head does not exist.
    __device__ __forceinline__ bool set(const int4& segment, int k) {
        cut = segment;
        const int u = k / p.rows, unit = cut.y * p.units + u;
        int kv, n;
        unit_heads(p, unit, &kv, &h0, &n);
        r = k - u * p.rows;
        step = 2 * (int64_t)per;             // from one CTA's slots to the next's
        slot0 = (int64_t)cut.w * step + k;
        return kv < p.hkv && r < n;
    }
    __device__ __forceinline__ int64_t slot(int q) const { return slot0 + q * step + (q == 0 ? per : 0); }
    __device__ __forceinline__ float4 load(int q, int lane) const {
        return __ldcg(reinterpret_cast<const float4*>(p.part_o + slot(q) * D) + lane);
    }
    // The slice's sum of weight_of(q) times part q over q = slice, slice + slices, ...; the first parts are in x already.
    template <int kAhead, typename W>
    __device__ __forceinline__ float4 sum(float4 (&x)[kAhead], int slice, int slices, int rounds, int lane, W weight_of) const {
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int q0 = slice; rounds > 0; --rounds, q0 += kAhead * slices)
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int q = q0 + i * slices;
                const float w = weight_of(q);
                o.x += x[i].x * w;
                o.y += x[i].y * w;
                o.z += x[i].z * w;
                o.w += x[i].w * w;
                const int next = q + kAhead * slices;
                if (next < cut.z) x[i] = load(next, lane);
            }
        return o;
    }
    template <int kAhead>
    __device__ __forceinline__ void request(float4 (&x)[kAhead], int slice, int slices, int lane) const {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int q = slice + i * slices;
            x[i] = q < cut.z ? load(q, lane) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
    __device__ __forceinline__ void store(const float4& o, float m, float l, int lane) const {
        store4((T*)p.out + cut.x * p.out_stride + (int64_t)(h0 + r) * D + 4 * lane, o, inverse_sum(l));
        if (p.lse && lane == 0) p.lse[(int64_t)cut.x * p.hq + h0 + r] = natural_log_sum<T>(m, l);
    }
};

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads, 4)
paged_join_kernel(const __grid_constant__ AttnParams p) {
    using J = Joiner<T, D>;
    constexpr int kLanes = J::kLanes, kWarps = kJoinThreads / 32;
    extern __shared__ float weight[];        // [ctas], then [ctas] sums
    float* sums = weight + p.ctas;
    __shared__ float4 sm_o[kJoinThreads / kLanes][kLanes];
    __shared__ float sm_m[kWarps], sm_l[kWarps];
    const int tid = threadIdx.x, warp = tid >> 5;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    // grid: (CTAs per cut, cuts)
    const int4 cut = __ldcg(p.cuts + blockIdx.y);
    if (cut.z == 0) return;
    const int first = (blockIdx.y - cut.w) * gridDim.x + blockIdx.x, sharers = (cut.z - 1) * gridDim.x;
    const bool wide = cut.z > 32 || sharers >= p.units * p.rows;   // a CTA per item; else a warp
    J j(p);
#pragma unroll 1
    for (int item = first; wide && item < j.per; item += sharers) {
        if (!j.set(cut, item)) continue;
        constexpr int kSlices = kJoinThreads / kLanes, kAhead = 4;
        const int lane = tid % kLanes, slice = tid / kLanes, parts = j.cut.z;
        float4 x[kAhead];
        j.request(x, slice, kSlices, lane);
        float m = kNothing, l = 0.f;
#pragma unroll 1
        for (int q = tid; q < parts; q += kJoinThreads) {
            const float2 ml = __ldcg(p.part_ml + j.slot(q));
            weight[q] = ml.x;
            sums[q] = ml.y;
            m = fmaxf(m, ml.x);
        }
        m = warp_max(m);
        if ((tid & 31) == 0) sm_m[warp] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWarps; ++w) m = fmaxf(m, sm_m[w]);
#pragma unroll 1
        for (int q = tid; q < parts; q += kJoinThreads) {
            weight[q] = weight_for(weight[q], m);
            l += sums[q] * weight[q];
        }
        l = warp_sum(l);
        if ((tid & 31) == 0) sm_l[warp] = l;
        __syncthreads();
        const int rounds = (parts + kAhead * kSlices - 1) / (kAhead * kSlices);
        float4 o = j.sum(x, slice, kSlices, rounds, lane, [&](int q) { return q < parts ? weight[q] : 0.f; });
        sm_o[slice][lane] = o;
        __syncthreads();
        if (slice == 0) {
#pragma unroll 4
            for (int q = 1; q < kSlices; ++q) {
                const float4 y = sm_o[q][lane];
                o.x += y.x;
                o.y += y.y;
                o.z += y.z;
                o.w += y.w;
            }
            l = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) l += sm_l[w];
            j.store(o, m, l, lane);
        }
        __syncthreads();                     // what is shared is free again
    }
#pragma unroll 1
    for (int item = first * kWarps + warp; !wide && item < j.per; item += sharers * kWarps) {
        if (!j.set(cut, item)) continue;
        constexpr int kSlices = 32 / kLanes, kAhead = 4 / kSlices;
        const int lane = (tid & 31) % kLanes, slice = (tid & 31) / kLanes, parts = j.cut.z;
        float4 x[kAhead];
        j.request(x, slice, kSlices, lane);
        const float2 ml = (tid & 31) < parts ? __ldcg(p.part_ml + j.slot(tid & 31)) : make_float2(kNothing, 0.f);
        const float m = warp_max(ml.x), w = weight_for(ml.x, m), l = warp_sum(ml.y * w);
        const int rounds = (parts + kAhead * kSlices - 1) / (kAhead * kSlices);
        float4 o = j.sum(x, slice, kSlices, rounds, lane, [&](int q) {
            const float v = __shfl_sync(0xffffffffu, w, q & 31);
            return q < parts ? v : 0.f;
        });
        if (kSlices == 2) {
            o.x += __shfl_xor_sync(0xffffffffu, o.x, 16);
            o.y += __shfl_xor_sync(0xffffffffu, o.y, 16);
            o.z += __shfl_xor_sync(0xffffffffu, o.z, 16);
            o.w += __shfl_xor_sync(0xffffffffu, o.w, 16);
        }
        if (slice == 0) j.store(o, m, l, lane);
    }
}

// ---------------------------------------------------------------------------------------------------- host

// Of a kernel: tokens that a warp takes at a time, and most warps of a CTA.
struct Tiling {
    int32_t tile, warps;
};
// How the heads are dealt to warps.
struct Layout {
    int32_t splits, rows, units, chunks, subs, ctas, step_log2;
    int nt;                                // column tiles of 8 heads of a unit
    size_t part_o, part_ml, cuts, bytes;   // offsets and size of the workspace
};
// Units per CTA: all of a token's, up to the warps, so that a CTA reads whole rows of the pools and combines nothing at
// a segment's end.  For one or two rows fewer, whose warps share the tokens: a long row is then cut into a quarter as
// many parts, and a short one may not be cut at all (one row of 8 KV heads of 128: 300 tokens 7.5 instead of 7.7 us,
// 4096 9.7 instead of 10.8, 32768 29.1 instead of 30.3; but 4 rows of 30000 80.4 instead of 78.6 us).
template <typename TilingOf>
Layout layout_of(int32_t batch, int32_t hkv, int32_t hq, int32_t dim, TilingOf tiling_of, int sms) {
    Layout y{};
    const int32_t group = hq / hkv;
    y.splits = (group + kMaxGroup - 1) / kMaxGroup;
    y.rows = (group + y.splits - 1) / y.splits;
    y.nt = (y.rows + 7) / 8;
    const int32_t all = hkv * y.splits;
    const Tiling tiling = tiling_of(dim, y.nt);
    const int32_t most = (int64_t)batch * all <= 2 * kMaxUnits ? 2 : kMaxUnits;
    y.chunks = (all + most - 1) / most;
    y.units = (all + y.chunks - 1) / y.chunks;
    for (y.subs = 1; 2 * y.subs * y.units <= tiling.warps; y.subs *= 2) {}
    for (y.step_log2 = 0; (1 << y.step_log2) < tiling.tile * y.subs; ++y.step_log2) {}
    y.ctas = sms;                          // the rings leave no shared memory for more
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    const size_t slots = (size_t)y.ctas * 2 * y.units * y.rows;
    y.part_o = 0;
    y.part_ml = up(slots * dim * sizeof(float));
    y.cuts = y.part_ml + up(slots * sizeof(float2));
    y.bytes = y.cuts + up((size_t)y.ctas * sizeof(int4));
    return y;
}

constexpr int kMaxDevices = 64;

// Rings of all warps, and room to begin on a 128-byte boundary.
template <typename W>
constexpr int attn_smem(int warps) { return 128 + warps * W::Stages::kWarpBytes; }

template <typename... W>
cudaError_t allow_smem() {
    cudaError_t e = cudaSuccess;
    ((e = e != cudaSuccess ? e : cudaFuncSetAttribute(paged_attn_kernel<W>, cudaFuncAttributeMaxDynamicSharedMemorySize, attn_smem<W>(W::kWarps))), ...);
    return e;
}

// SM count of the current device; looked up once per device.  The kernels' shared memory limit is raised there too.
template <typename... W>
cudaError_t device_sms(int* sms) {
    static std::atomic<int> known[kMaxDevices];
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    *sms = known[dev].load(std::memory_order_acquire);
    if (*sms > 0) return cudaSuccess;
    e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = allow_smem<W...>();
    if (e == cudaSuccess) known[dev].store(*sms, std::memory_order_release);
    return e;
}

template <typename W>
cudaError_t launch_main(const AttnParams& p, const Layout& y, cudaStream_t s) {
    return ps::launch_dependent(paged_attn_kernel<W>, dim3((unsigned)y.ctas), dim3((unsigned)(32 * y.units * y.subs)),
                                (size_t)attn_smem<W>(y.units * y.subs), s, p);
}
// W1, W2: the workers for units of up to 8 and up to 16 query heads.
template <typename W1, typename W2>
cudaError_t launch_attn(const AttnParams& p, const Layout& y, bool may_cut, cudaStream_t s) {
    cudaError_t e = y.nt == 1 ? launch_main<W1>(p, y, s) : launch_main<W2>(p, y, s);
    if (e == cudaSuccess && may_cut) {
        // Four CTAs of a cut at most, so that all fit the chip at once: those of a second round would begin only when the first
        // has waited for the main kernel.  (64 rows of 4096 tokens and one of 32768, 64 query heads on 8: 179.9 us in 16 bits
        // and 100.3 in 8, with eight CTAs a cut of three an SM 182.4 and 101.7.)
        const dim3 grid((unsigned)std::min(4, (y.units * y.rows + kJoinThreads / 32 - 1) / (kJoinThreads / 32)), (unsigned)(y.ctas - 1));
        e = ps::launch_dependent(paged_join_kernel<typename W1::Type, W1::kDim>, grid, dim3(kJoinThreads), (size_t)y.ctas * 2 * sizeof(float), s, p);
    }
    return e;
}

const char* shape_error(int32_t hkv, int32_t hq, int32_t dim) {
    if (hkv <= 0 || hq <= 0 || hq % hkv != 0) return "num_q_heads must be a positive multiple of num_kv_heads";
    if (dim != 64 && dim != 128) return "head_dim must be 64 or 128";
    if (hq / hkv > 64) return "at most 64 query heads per KV head";
    if (hkv > 1024) return "at most 1024 KV heads";
    return nullptr;
}

template <typename TilingOf, typename Sms>
int32_t workspace_of(int32_t hkv, int32_t hq, int32_t dim, TilingOf tiling_of, Sms sms_here, int64_t* bytes) {
    if (!bytes || shape_error(hkv, hq, dim)) return PS_ERR_INVALID;
    int sms = 0;
    if (sms_here(&sms) != cudaSuccess) {
        cudaGetLastError();
        return PS_ERR_CUDA;
    }
    *bytes = (int64_t)std::max(layout_of(1, hkv, hq, dim, tiling_of, sms).bytes, layout_of(1 << 30, hkv, hq, dim, tiling_of, sms).bytes);
    return PS_OK;
}

bool on_bytes(const void* q, int64_t stride_bytes, int bytes) { return reinterpret_cast<uintptr_t>(q) % bytes == 0 && stride_bytes % bytes == 0; }
constexpr const char* kUneven = "pools, q, out and their strides must be multiples of 16 bytes";

// Returns PS_ERR_INVALID with a text that begins with the entry point's name.
struct Refusal {
    const char* name;
    char* buf;
    int32_t cap;
    int32_t operator()(const char* text) const {
        if (buf && cap > 0) snprintf(buf, (size_t)cap, "%s: %s", name, text);
        return PS_ERR_INVALID;
    }
};

struct CacheShape {
    int32_t hkv, dim, block_size, num_blocks;
};

// Checks a call's arguments (Args: ps_paged_attn_args or ps_quant_attn_args; `pools` checks the cache's own) and fills in
// all parameters but the cache's.  Nothing to do for a batch of 0.
template <typename Args, typename TilingOf, typename Sms, typename Pools>
int32_t plan_call(const Args& a, const CacheShape& c, TilingOf tiling_of, Sms sms_here, Pools pools, const Refusal& refuse, AttnParams* params,
                  Layout* layout, bool* may_cut) {
    if (refuse.buf && refuse.cap > 0) refuse.buf[0] = 0;
    if (const char* m = shape_error(c.hkv, a.num_q_heads, c.dim)) return refuse(m);
    if (a.batch < 0 || c.block_size <= 0 || c.num_blocks <= 0 || a.table_stride <= 0 || a.window < 0)
        return refuse("negative count or non-positive size");
    if (a.dtype != PS_DTYPE_BF16 && a.dtype != PS_DTYPE_FP16) return refuse("dtype must be PS_DTYPE_BF16 or PS_DTYPE_FP16");
    if (!(a.scale == a.scale) || a.scale - a.scale != 0.f) return refuse("scale is not finite");
    if (a.batch == 0) return PS_OK;
    if (!a.q || !a.out || !a.block_tables || !a.ctx_lens || !a.workspace) return refuse("null pointer");
    if (const char* m = pools()) return refuse(m);
    if (!on_bytes(a.q, 2 * a.q_stride, 16) || !on_bytes(a.out, 2 * a.out_stride, 16)) return refuse(kUneven);
    const int64_t width = (int64_t)a.num_q_heads * c.dim;
    if (a.batch > 1 && a.out_stride < width) return refuse("rows of out overlap");
    // In place a row's queries are loaded by the CTAs that attend it before its result is stored: by the CTA that has the
    // whole row, or behind all of them by the join.
    if (!(a.out == a.q && (a.out_stride == a.q_stride || a.batch == 1)) &&
        ps::rows_meet(ps::RowSet{a.out, a.out_stride, width}, ps::RowSet{a.q, a.q_stride, width}, a.batch))
        return refuse("out overlaps q by another stride or in part");
    // The places of all segments are counted in 32 bits.  A segment has a place for every tile that its table row has room
    // for and at most 4 more, and a tile's tokens times the KV heads are 24 (3 KV heads of 33 query heads each) times a
    // row's segments or more: with 1024 more tokens a row, 2^34 tokens times KV heads always fit.
    const int64_t room = std::min<int64_t>((int64_t)a.table_stride * c.block_size, kMaxTokens);
    const Layout places = layout_of(a.batch, c.hkv, a.num_q_heads, c.dim, tiling_of, 1);
    if ((room >> places.step_log2) + 4 > (1 << 30) / ((int64_t)a.batch * places.chunks))
        return refuse("the tables of the batch have room for more than 2^30 tiles of tokens");
    int sms = 0;
    if (cudaError_t e = sms_here(&sms); e != cudaSuccess) {
        char where[64];
        snprintf(where, sizeof where, "%s: device", refuse.name);
        return ps::launch_fail(refuse.buf, refuse.cap, where, e);
    }
    const Layout y = layout_of(a.batch, c.hkv, a.num_q_heads, c.dim, tiling_of, sms);
    if (a.workspace_bytes < (int64_t)y.bytes || (reinterpret_cast<uintptr_t>(a.workspace) & 255)) {
        char text[128];
        snprintf(text, sizeof text, "the workspace is smaller than %s_workspace says, or not on a 256-byte boundary", refuse.name);
        return refuse(text);
    }
    AttnParams& p = *params;
    p.q = a.q, p.out = a.out, p.lse = a.lse;
    p.tables = a.block_tables, p.ctx = a.ctx_lens, p.status = a.status_word;
    char* ws = (char*)a.workspace;
    p.part_o = (float*)(ws + y.part_o);
    p.part_ml = (float2*)(ws + y.part_ml);
    p.cuts = (int4*)(ws + y.cuts);
    p.q_stride = a.q_stride, p.out_stride = a.out_stride;
    p.room = room;
    p.block_magic = c.block_size > 1 ? ~0ull / (uint64_t)c.block_size + 1 : 0;
    p.batch = a.batch, p.table_stride = a.table_stride, p.num_blocks = c.num_blocks, p.block_size = c.block_size, p.window = a.window;
    p.hkv = c.hkv, p.hq = a.num_q_heads, p.group = a.num_q_heads / c.hkv;
    p.splits = y.splits, p.rows = y.rows, p.units = y.units, p.chunks = y.chunks, p.subs = y.subs, p.ctas = y.ctas;
    p.step_log2 = y.step_log2;
    p.scale_log2e = (a.scale != 0.f ? a.scale : 1.f / sqrtf((float)c.dim)) * kLog2e;
    // A segment's start and end take about the time of two tiles.  Not counted (1 in brackets), 200 rows of 10 to 100 tokens
    // take 20.2 instead of 17.2 us (17.9), 33 ragged rows with a window 19.6 instead of 18.1 (18.8), 64 rows of 1024 to
    // 4096 102.4 either way.  With few segments a CTA has one whatever it costs.
    p.segment = (int64_t)a.batch * y.chunks >= y.ctas / 8 ? 2 : 0;
    // rows that cannot be longer than one tile are never cut
    const int64_t longest = a.window > 0 && a.window < p.room ? a.window : p.room;
    *may_cut = longest > (int64_t)1 << p.step_log2;
    *layout = y;
    return PS_OK;
}

}  // namespace

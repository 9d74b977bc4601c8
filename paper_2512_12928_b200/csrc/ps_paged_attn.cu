// ps_paged_attn: attention of one new token per row over a paged KV cache, with the lengths and block tables on the
// device.  Nothing about the batch but its size is known on the host, so the call can be replayed from a graph.
//
//   out[b][h] = sum_t p_t V[t][h / G] / sum_t p_t,   p_t = 2^(s_t - m),   s_t = log2(e) scale q[b][h] . K[t][h / G],
//   max(0, ctx_b - window) <= t < ctx_b,   m = max_t s_t (running),   lse = ln 2 (m + log2 sum_t p_t)
//
// Bound: HBM, for up to 16 query heads on a KV head.  A token and KV head cost 4 D bytes and 4 G D flops, and the card
// would compute faster than it loads up to G = 64; but a unit (see Warps) has at most 16 query heads, and with more of them
// every unit of a KV head copies the tiles for itself, 2 to 4 times the cache's bytes in all (the 672 MB case below with
// 16 query heads on each of 8 KV heads 110.5 us, with 20 155, 32 167, 64 294).  Every warp streams its own tiles of 16 or
// 32 tokens (4 KiB of K and of V) through a ring of three in shared memory (cp.async, 16 bytes a lane, whole 128-byte
// lines), across the ends of rows, and no barrier lies between HBM and the tensor cores.  Tokens may lie anywhere; what is
// not attended is filled with zeros instead of being read.
// Measured: 672 MB of cache (64 rows of 1024 to 4096 tokens, 32 query heads on 8 KV heads of 128, bf16) 101.5 us, or
// 6.6 TB/s, which is what a copy reaches; about 6 us of it pass before the first tile is there and in the join, and
// bound small calls (one row of 300 tokens: 7.0 us).  Heads of 64 need as many instructions for half the bytes and
// reach 0.9 of that rate, 0.77 with 16 query heads on a KV head.
//
// Products: a group has few query heads, so they are the narrow side: S^T = K Q^T and O^T = V^T P^T as
// mma.m16n8k16 with tokens, then dims, as the 16 rows and 8 heads as the columns.  K comes through ldmatrix and V
// through its transposing form, both without bank conflicts (16-byte pieces exclusive-ored with the token's number);
// P^T leaves the first product as pairs of heads and enters the second as pairs of tokens, which is one movmatrix.
// With heads as the rows instead, half of every product was padding for up to 8 heads and V's pairs cost 32 byte
// permutes a tile: 159 us for 672 MB of cache (64 rows, 32 query heads on 8 KV heads of 128), where this form took 106.
// (The tile shapes of tcgen05.mma have 64 or 128 rows and its P would go through shared or tensor memory; the
// tensor cores are idle most of the time either way.)
//
// Softmax: the reference m of a head is raised only when a score exceeds it by more than kSlack, so that a tile needs
// one vote instead of a maximum over the lanes; weights stay below 2^kSlack and sums in 32 bits lose nothing by it.
// For the product with V a weight is split into two numbers of the inputs' type: one alone makes the result's error
// 1.4 times what its own rounding costs, and the second product costs less than 1 % of the time.  A third number gains
// nothing: of the 672 MB case's outputs in bf16 0.3 % are not the nearest to the exact value either way (0.08 % of a sum in
// plain 32-bit arithmetic), which then is the tensor cores' order and rounding of sums.
//
// Work: the rows' tiles form one sequence (with two places more for each row's start and end, which cost about two tiles'
// time) that is cut into equal shares, one per CTA, from the lengths each CTA reads itself: no plan is made on the host or
// by another kernel.  A row cut by a share's end leaves partial results (m, sum, accumulators) in the workspace, which a
// second kernel (paged_join_kernel) combines in order.  The join is a second launch rather than a last-arrival counter in
// the first: the workspace then needs no initial state, and neither a replayed graph nor a call that shares it in turn can
// find a stale counter.  It is launched early, but its CTAs (80 registers a thread) do not fit beside one of 8
// warps of the first kernel (207 to 249), so they start as those leave.
//
// Warps: a CTA works on `units` (KV head, group of at most 16 query heads) times `subs` token slices (a power of two);
// the units of a token are neighbours in memory.  The slices' states are combined through shared memory at a segment's
// end.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "ps_internal.h"
#include "ps_kvswap.h"

namespace {

constexpr int kMaxWarps = 8;
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
    return p.block_size == 1 ? t : (int32_t)__umul64hi((uint64_t)(uint32_t)t, p.block_magic);
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
    *kv = unit / p.splits;
    const int s = unit - *kv * p.splits;
    *h0 = *kv * p.group + s * p.rows;
    *n = min(p.rows, p.group - s * p.rows);
}

// The tiles of a CTA's share, one after the other: row b, chunk of its units, tile i of the row's `tiles`, at `place` of
// the sequence that is cut into shares: a segment (row and chunk) takes p.segment places for its start and end, then one
// for each tile.
struct Cursor {
    int32_t b, chunk, i, tiles, first, end, place;
    int32_t next_len;                        // of row b + 1, asked for while row b is worked on
    __device__ __forceinline__ void row(const AttnParams& p, int32_t len) {
        row_span(p, len, &first, &end);
        tiles = row_tiles(p, len);
        if (end != len && p.status) *(volatile int32_t*)p.status = kStatusLength;
    }
    __device__ __forceinline__ bool ends_segment() const { return i + 1 == tiles; }
    __device__ __forceinline__ int32_t next_place(const AttnParams& p) const { return place + 1 + (ends_segment() ? p.segment : 0); }
    __device__ __forceinline__ void next(const AttnParams& p, int32_t share_end) {
        place = next_place(p);
        if (++i < tiles) return;
        i = 0;
        if (++chunk < p.chunks) return;
        chunk = 0;
        ++b;
        if (place < share_end) row(p, next_len);
        look_ahead(p);
    }
    __device__ __forceinline__ void look_ahead(const AttnParams& p) { next_len = b + 1 < p.batch ? p.ctx[b + 1] : 0; }
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

// -------------------------------------------------------------------------------------------- main kernel

template <int D>
struct Ring {
    static constexpr int kStages = 3;
    static constexpr int kTokens = 2048 / D;                 // of a tile: 16 or 32, products take 16 at a time
    static constexpr int kRowBytes = 2 * D;
    static constexpr int kSideBytes = kTokens * kRowBytes;   // keys, then values
    static constexpr int kStageBytes = 2 * kSideBytes;
    static constexpr int kWarpBytes = kStages * kStageBytes;
};

template <typename T, int D, int NT>
struct Worker {
    using R = Ring<D>;
    static constexpr int kSub = R::kTokens / 16;             // groups of 16 tokens in a tile
    const AttnParams& p;
    const int lane, g, c, unit_in_cta, sub;
    const uint32_t ring;                       // the warp's first stage
    const uint64_t policy;
    uint32_t put;                              // this lane's place in a stage: row lane / 8 and, in place, piece lane % 8
    uint32_t k_at[4], v_at[4];                 // what this lane reads of a stage: pieces 2 j + .. of its row of the four parts
    uint32_t q[NT][D / 16][2];                 // query head 8 t + g, dims 16 j + 2 c and 16 j + 8 + 2 c
    const T *k_src, *v_src;                    // pools at this lane's head and piece
    const int32_t* table;
    int32_t id, at;                            // block and place of token lane % kTokens; at = -1: no token
    bool idle;                                 // the unit does not exist
    uint32_t mask, next_mask;                  // which tokens of the two oldest tiles in the ring are attended

    __device__ __forceinline__ Worker(const AttnParams& pp, uint32_t smem)
        : p(pp), lane(threadIdx.x & 31), g((threadIdx.x & 31) >> 2), c(threadIdx.x & 3), unit_in_cta((threadIdx.x >> 5) % pp.units),
          sub((threadIdx.x >> 5) / pp.units), ring(smem + (threadIdx.x >> 5) * R::kWarpBytes), policy(read_once_policy()), mask(0),
          next_mask(0) {
        const int x = lane & 7, up = lane >> 4, mid = lane >> 3 & 1;
        put = (lane >> 3) * R::kRowBytes + (((lane & 7) ^ (lane >> 3)) << 4);   // rows 4 to 7 of 8: piece ^ 4
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            k_at[j] = (x + 8 * mid) * R::kRowBytes + (((2 * j + up) ^ x) << 4);
            v_at[j] = R::kSideBytes + (x + 8 * up) * R::kRowBytes + (((2 * j + mid) ^ x) << 4);
        }
    }

    __device__ __forceinline__ void load_query(int b, int h0, int n) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const T* src = (const T*)p.q + b * p.q_stride + (int64_t)(h0 + 8 * t + g) * D + 2 * c;
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    q[t][j][h] = 8 * t + g < n ? *reinterpret_cast<const uint32_t*>(src + 16 * j + 8 * h) : 0u;
        }
    }

    // The row and chunk of the tiles to come.
    __device__ __forceinline__ void enter(const Cursor& cur) {
        int kv, h0, n;
        unit_heads(p, cur.chunk * p.units + unit_in_cta, &kv, &h0, &n);
        idle = kv >= p.hkv;
        const int64_t o = idle ? 0 : (int64_t)kv * D + 8 * (lane & 7);
        k_src = (const T*)p.kpool + o;
        v_src = (const T*)p.vpool + o;
        table = p.tables + (int64_t)cur.b * p.table_stride;
        // the unit's queries, into L1: they are loaded when its tiles have come, and then nothing hides their latency
        if (!idle && lane < n * D / 64) {
            uint32_t unused;
            asm volatile("ld.global.ca.b32 %0, [%1];" : "=r"(unused) : "l"((const T*)p.q + cur.b * p.q_stride + (int64_t)h0 * D + lane * 64));
        }
    }

    // Looks the tile's tokens up.
    __device__ __forceinline__ void load_ids(const Cursor& cur) {
        const int32_t t = cur.first + R::kTokens * ((cur.i << (p.step_log2 - (D == 128 ? 4 : 5))) + sub) + lane % R::kTokens;
        id = 0;
        at = -1;
        if (t < cur.end) {
            const int32_t blk = block_of(t, p);
            at = t - blk * p.block_size;
            id = table[blk];
        }
    }

    // Requests the tile that load_ids looked up, into a stage; returns which of its tokens are attended.
    __device__ __forceinline__ uint32_t copy_tile(int stage) {
        const bool known = (unsigned)id < (unsigned)p.num_blocks;
        if (at >= 0 && !known && p.status) *(volatile int32_t*)p.status = kStatusBadId;
        const bool read = at >= 0 && known && !idle;
        const uint32_t on = __ballot_sync(0xffffffffu, read);
        // where the lane's token lies in the pools; what is not read has the address of the first block's first token
        const int64_t in_block = (int64_t)at * p.hkv * D;
        const int64_t k_off = read ? id * p.k_block_stride + in_block : 0, v_off = read ? id * p.v_block_stride + in_block : 0;
        const uint32_t dst = ring + stage * R::kStageBytes + put;
#pragma unroll
        for (int i = 0; i < R::kTokens / 4; ++i) {
            const int row = 4 * i + (lane >> 3);
            const uint32_t bytes = (on >> row & 1) << 4;
            const int64_t ko = __shfl_sync(0xffffffffu, k_off, row);
            const int64_t vo = p.k_block_stride == p.v_block_stride ? ko : __shfl_sync(0xffffffffu, v_off, row);
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
                const uint32_t to = (dst ^ (64 * (i & 1))) + 4 * i * R::kRowBytes + 128 * j;
                copy16(to, k_src + ko + 64 * j, bytes, policy);
                copy16(to + R::kSideBytes, v_src + vo + 64 * j, bytes, policy);
            }
        }
        return on;
    }

    // The keys of the tile in a stage.
    __device__ __forceinline__ void read_keys(int stage, uint4 (&k)[kSub][D / 16]) const {
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int j = 0; j < D / 16; ++j) k[u][j] = ldsm(ring + stage * R::kStageBytes + 16 * u * R::kRowBytes + k_at[j % 4] + 128 * (j / 4));
    }
    // Attends that tile; `on`: its tokens that count.
    __device__ __forceinline__ void attend(int stage, const uint4 (&k)[kSub][D / 16], uint32_t on, State<D, NT>& st) {
        const uint32_t src = ring + stage * R::kStageBytes;
        constexpr int kChains = 2 / kSub;        // two chains of products either way
        float s[kSub][NT][4], s2[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s2[t][i] = 0.f;
#pragma unroll
                for (int u = 0; u < kSub; ++u) s[u][t][i] = 0.f;
            }
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int u = 0; u < kSub; ++u)
#pragma unroll
                for (int t = 0; t < NT; ++t) Num<T>::mma(kChains == 2 && (j & 1) ? s2[t] : s[u][t], k[u][j], q[t][j][0], q[t][j][1]);
        uint4 v[kSub][D / 16];                   // asked for before the softmax
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int j = 0; j < D / 16; ++j) v[u][j] = ldsm_t(src + 16 * u * R::kRowBytes + v_at[j % 4] + 128 * (j / 4));
        // s[u][t][0], [1]: token 16 u + g, heads 8t + 2c, + 1; [2], [3]: token 16 u + 8 + g.  The weights' exponents:
        float e[kSub][NT][4];
        bool over = false;
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x = s[u][t][i] + (kChains == 2 ? s2[t][i] : 0.f);
                    x = on >> (16 * u + g + 4 * (i & 2)) & 1 ? x * p.scale_log2e : -CUDART_INF_F;
                    s[u][t][i] = x;
                    e[u][t][i] = x - st.m[t][i & 1];
                    over |= e[u][t][i] > Num<T>::kSlack;
                }
        if (__any_sync(0xffffffffu, over)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float mx = fmaxf(s[0][t][h], s[0][t][2 + h]);
                    if (kSub == 2) mx = fmaxf(mx, fmaxf(s[kSub - 1][t][h], s[kSub - 1][t][2 + h]));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                    mx = fmaxf(mx, st.m[t][h]);
                    const float alpha = ex2(st.m[t][h] - mx);
                    st.m[t][h] = mx;
                    st.l[t][h] *= alpha;
#pragma unroll
                    for (int j = 0; j < D / 16; ++j) {
                        st.acc[t][j][h] *= alpha;
                        st.acc[t][j][2 + h] *= alpha;
                    }
#pragma unroll
                    for (int u = 0; u < kSub; ++u) {
                        e[u][t][h] = s[u][t][h] - mx;
                        e[u][t][2 + h] = s[u][t][2 + h] - mx;
                    }
                }
        }
        // P^T: tokens 2c, 2c + 1 and 2c + 8, 2c + 9 (of 16) of head 8t + g, as the sum of two numbers of the inputs' type
        uint32_t pt[kSub][NT][2], rest[kSub][NT][2];
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int i = 0; i < 4; ++i) e[u][t][i] = ex2(e[u][t][i] + Num<T>::kLift);
                st.l[t][0] += e[u][t][0] + e[u][t][2];
                st.l[t][1] += e[u][t][1] + e[u][t][3];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t v = Num<T>::pack(e[u][t][2 * i], e[u][t][2 * i + 1]);
                    const float2 f = Num<T>::unpack(v);
                    pt[u][t][i] = transpose8(v);
                    rest[u][t][i] = transpose8(Num<T>::pack(e[u][t][2 * i] - f.x, e[u][t][2 * i + 1] - f.y));
                }
            }
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    Num<T>::mma(st.acc[t][j], v[u][j], pt[u][t][0], pt[u][t][1]);
                    Num<T>::mma(st.acc[t][j], v[u][j], rest[u][t][0], rest[u][t][1]);
                }
    }
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

template <typename T, int D, int NT>
__global__ void __launch_bounds__(kMaxWarps * 32, 1)
paged_attn_kernel(const __grid_constant__ AttnParams p) {
    using R = Ring<D>;
    extern __shared__ unsigned char smem_raw[];   // rings of the warps
    // the pieces' places are exclusive-ored within 128 bytes
    unsigned char* smem = smem_raw + (-(uint32_t)__cvta_generic_to_shared(smem_raw) & 127);
    __shared__ float2 sh_ml[kMaxWarps][8 * NT];
    __shared__ int sh_sum[kMaxWarps];
    __shared__ int4 sh_begin;          // where the share begins: row, chunk, tile; the row's length
    __shared__ int sh_place;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int nwarps = blockDim.x >> 5;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    Worker<T, D, NT> wk(p, (uint32_t)__cvta_generic_to_shared(smem));
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
    Cursor cur;
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
        int a = before;
        cur.b = b_lo;                            // and of a single row the length is still there
        if (per > 1)
#pragma unroll 1
            for (;; ++cur.b) {
                len = p.ctx[cur.b];
                const int n = (row_tiles(p, len) + p.segment) * p.chunks;
                if (begin < a + n) break;
                a += n;
            }
        cur.row(p, len);
        cur.chunk = 0;
        cur.i = begin - a;
        if (p.chunks > 1) {
            cur.chunk = cur.i / (cur.tiles + p.segment);
            cur.i -= cur.chunk * (cur.tiles + p.segment);
        }
        cur.i = max(cur.i - p.segment, 0);        // a share that begins in a segment's first places has its first tile
        sh_begin = make_int4(cur.b, cur.chunk, cur.i, len);
        sh_place = a + cur.chunk * (cur.tiles + p.segment) + p.segment + cur.i;
        // the first block ids, into L1 while the CTA meets
        const int32_t t = cur.first + (cur.i << p.step_log2);
        if (t < cur.end) {
            uint32_t unused;
            asm volatile("ld.global.ca.b32 %0, [%1];" : "=r"(unused) : "l"(p.tables + (int64_t)cur.b * p.table_stride + block_of(t, p)));
        }
    }
    __syncthreads();
    int4 cut = make_int4(0, 0, 0, 0);
    if (begin < end && sh_place < end) {         // else there is no tile in it
        const int4 start = sh_begin;
        cur.b = start.x;
        cur.chunk = start.y;
        cur.i = start.z;
        cur.place = sh_place;
        cur.look_ahead(p);
        cur.row(p, start.w);
        Cursor ahead = cur;                      // the tile that is requested next
        int slot = 0;                            // stage that is filled next
        wk.enter(ahead);
        wk.load_ids(ahead);
        State<D, NT> st;
        int kv = 0, h0 = 0, n = 0;
        int32_t lo = 0;
        bool fresh = true;
#pragma unroll 1
        for (int fill = R::kStages - 1; cur.place < end;) {
            copies_wait<R::kStages - 2>();
            __syncwarp();                        // the other lanes' copies too, and they have left the stage before
            const int filled = slot;             // the stage that the tile before left
            slot = slot + 1 == R::kStages ? 0 : slot + 1;       // the oldest
            const uint32_t on = wk.mask;
            wk.mask = wk.next_mask;
            uint4 k[Worker<T, D, NT>::kSub][D / 16];
            wk.read_keys(slot, k);               // in the first rounds what it reads is not used
            if (ahead.place < end) {
                wk.next_mask = wk.copy_tile(filled);
                ahead.next(p, end);
                if (ahead.place < end) {
                    if (ahead.i == 0) wk.enter(ahead);
                    wk.load_ids(ahead);
                }
            }
            copies_commit();
            if (fill > 0) {                      // the first rounds only fill the ring
                --fill;
                continue;
            }
            const int unit = cur.chunk * p.units + wk.unit_in_cta;
            if (fresh) {
                state_reset(st);
                n = 0;
                if (unit < p.hkv * p.splits) unit_heads(p, unit, &kv, &h0, &n);
                wk.load_query(cur.b, h0, n);
                lo = cur.i;
                fresh = false;
            }
            wk.attend(slot, k, on, st);
            const bool seg_end = cur.ends_segment();
            if (seg_end || cur.next_place(p) >= end) {
                const bool whole = lo == 0 && seg_end;
                // The states of the slices go through the stage that has just been read, heads as rows, and come
                // back as rows of four dims a lane.  (The places' exclusive or keeps the writes free of conflicts.)
                float* own = reinterpret_cast<float*>(smem + warp * R::kWarpBytes + slot * R::kStageBytes);
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int r = 8 * t + 2 * wk.c + h;
#pragma unroll
                        for (int j = 0; j < D / 16; ++j)
#pragma unroll
                            for (int e = 0; e < 2; ++e) own[r * D + ((16 * j + 8 * e + wk.g) ^ (8 * wk.c))] = st.acc[t][j][2 * e + h];
                        float l = st.l[t][h];
                        l += __shfl_xor_sync(0xffffffffu, l, 4);
                        l += __shfl_xor_sync(0xffffffffu, l, 8);
                        l += __shfl_xor_sync(0xffffffffu, l, 16);
                        if (wk.g == 0) sh_ml[warp][r] = make_float2(st.m[t][h], l);
                    }
                if (p.subs > 1) __syncthreads(); else __syncwarp();
                constexpr int kLanes = D / 4, kHeads = 32 / kLanes;      // heads that a warp works on at a time
                const int dim = 4 * (lane % kLanes);
                auto put = [&](int r, const float4& o, float m, float l) {
                    if (whole) {
                        store4((T*)p.out + cur.b * p.out_stride + (int64_t)(h0 + r) * D + dim, o, inverse_sum(l));
                        if (p.lse && dim == 0) p.lse[(int64_t)cur.b * p.hq + h0 + r] = natural_log_sum<T>(m, l);
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
                        constexpr int kSlices = decltype(slices)::value, kAtOnce = kMaxWarps / kSlices;
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
                    else combine(std::integral_constant<int, 8>());
                }
                if (p.subs > 1) __syncthreads(); else __syncwarp();      // the stage is free again
                if (!seg_end) {
                    const int from = (cur.place - cur.i) / share;      // the CTAs of the segment's first and last tile
                    cut = make_int4(cur.b, cur.chunk, (cur.place + cur.tiles - cur.i - 1) / share - from + 1, from);
                }
                fresh = true;
            }
            cur.next(p, end);
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
__global__ void __launch_bounds__(kJoinThreads, 3)
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
        constexpr int kSlices = kJoinThreads / kLanes, kAhead = 6;
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
        constexpr int kSlices = 32 / kLanes, kAhead = 8 / kSlices;
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
Layout layout_of(int32_t batch, int32_t hkv, int32_t hq, int32_t dim, int sms) {
    Layout y{};
    const int32_t group = hq / hkv;
    y.splits = (group + kMaxGroup - 1) / kMaxGroup;
    y.rows = (group + y.splits - 1) / y.splits;
    y.nt = (y.rows + 7) / 8;
    const int32_t all = hkv * y.splits;
    const int32_t most = (int64_t)batch * all <= 2 * kMaxWarps ? 2 : kMaxWarps;
    y.chunks = (all + most - 1) / most;
    y.units = (all + y.chunks - 1) / y.chunks;
    for (y.subs = 1; 2 * y.subs * y.units <= kMaxWarps; y.subs *= 2) {}
    for (y.step_log2 = dim == 128 ? 4 : 5; (1 << y.step_log2) < 2048 / dim * y.subs; ++y.step_log2) {}   // Ring::kTokens
    y.ctas = sms;                          // the rings take an SM's shared memory
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
static_assert(Ring<64>::kWarpBytes == Ring<128>::kWarpBytes, "one size for both");
int attn_smem(int warps) { return 128 + warps * Ring<128>::kWarpBytes; }

template <typename T, int D, int NT>
cudaError_t allow_smem() {
    return cudaFuncSetAttribute(paged_attn_kernel<T, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, attn_smem(kMaxWarps));
}

// SM count of the current device; looked up once per device.  The kernels' shared memory limit is raised there too.
cudaError_t device_sms(int* sms) {
    static std::atomic<int> known[kMaxDevices];
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    *sms = known[dev].load(std::memory_order_acquire);
    if (*sms > 0) return cudaSuccess;
    e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = allow_smem<__nv_bfloat16, 64, 1>();
    if (e == cudaSuccess) e = allow_smem<__nv_bfloat16, 64, 2>();
    if (e == cudaSuccess) e = allow_smem<__nv_bfloat16, 128, 1>();
    if (e == cudaSuccess) e = allow_smem<__nv_bfloat16, 128, 2>();
    if (e == cudaSuccess) e = allow_smem<__half, 64, 1>();
    if (e == cudaSuccess) e = allow_smem<__half, 64, 2>();
    if (e == cudaSuccess) e = allow_smem<__half, 128, 1>();
    if (e == cudaSuccess) e = allow_smem<__half, 128, 2>();
    if (e == cudaSuccess) known[dev].store(*sms, std::memory_order_release);
    return e;
}

template <typename T, int D, int NT>
cudaError_t launch_main(const AttnParams& p, const Layout& y, cudaStream_t s) {
    return ps::launch_dependent(paged_attn_kernel<T, D, NT>, dim3((unsigned)y.ctas), dim3((unsigned)(32 * y.units * y.subs)),
                                (size_t)attn_smem(y.units * y.subs), s, p);
}
template <typename T, int D>
cudaError_t launch_attn(const AttnParams& p, const Layout& y, bool may_cut, cudaStream_t s) {
    cudaError_t e = y.nt == 1 ? launch_main<T, D, 1>(p, y, s) : launch_main<T, D, 2>(p, y, s);
    if (e == cudaSuccess && may_cut) {
        const dim3 grid((unsigned)((y.units * y.rows + kJoinThreads / 32 - 1) / (kJoinThreads / 32)), (unsigned)(y.ctas - 1));
        e = ps::launch_dependent(paged_join_kernel<T, D>, grid, dim3(kJoinThreads), (size_t)y.ctas * 2 * sizeof(float), s, p);
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

}  // namespace

extern "C" int32_t ps_paged_attn_workspace(int32_t num_kv_heads, int32_t num_q_heads, int32_t head_dim, int64_t* bytes) {
    if (!bytes || shape_error(num_kv_heads, num_q_heads, head_dim)) return PS_ERR_INVALID;
    int sms = 0;
    if (device_sms(&sms) != cudaSuccess) {
        cudaGetLastError();
        return PS_ERR_CUDA;
    }
    *bytes = (int64_t)std::max(layout_of(1, num_kv_heads, num_q_heads, head_dim, sms).bytes,
                               layout_of(1 << 30, num_kv_heads, num_q_heads, head_dim, sms).bytes);
    return PS_OK;
}

extern "C" int32_t ps_paged_attn(const ps_paged_attn_args* args, void* stream, char* err_buf, int32_t err_cap) {
    using ps::arg_fail;
    if (err_buf && err_cap > 0) err_buf[0] = 0;
    auto bad = [&](const char* m) { return arg_fail(err_buf, err_cap, PS_ERR_INVALID, m); };
    if (!args) return bad("ps_paged_attn: null arguments");
    const ps_paged_attn_args a = *args;
    if (const char* m = shape_error(a.num_kv_heads, a.num_q_heads, a.head_dim)) {
        char text[128];
        snprintf(text, sizeof text, "ps_paged_attn: %s", m);
        return bad(text);
    }
    if (a.batch < 0 || a.block_size <= 0 || a.num_gpu_blocks <= 0 || a.table_stride <= 0 || a.window < 0)
        return bad("ps_paged_attn: negative count or non-positive size");
    if (a.dtype != PS_DTYPE_BF16 && a.dtype != PS_DTYPE_FP16) return bad("ps_paged_attn: dtype must be PS_DTYPE_BF16 or PS_DTYPE_FP16");
    if (!(a.scale == a.scale) || a.scale - a.scale != 0.f) return bad("ps_paged_attn: scale is not finite");
    if (a.batch == 0) return PS_OK;
    if (!a.kpool || !a.vpool || !a.q || !a.out || !a.block_tables || !a.ctx_lens || !a.workspace) return bad("ps_paged_attn: null pointer");
    auto on = [](const void* q, int64_t stride, int bytes) {
        return (reinterpret_cast<uintptr_t>(q) % bytes) == 0 && (stride * 2) % bytes == 0;
    };
    const int64_t block_elems = (int64_t)a.block_size * a.num_kv_heads * a.head_dim;
    if (a.num_gpu_blocks > 1 && (a.k_block_stride < block_elems || a.v_block_stride < block_elems))
        return bad("ps_paged_attn: a pool's block stride is smaller than a block");
    if (!on(a.kpool, a.k_block_stride, 16) || !on(a.vpool, a.v_block_stride, 16) || !on(a.q, a.q_stride, 16) || !on(a.out, a.out_stride, 16))
        return bad("ps_paged_attn: pools, q, out and their strides must be multiples of 16 bytes");
    const int64_t width = (int64_t)a.num_q_heads * a.head_dim;
    if (a.batch > 1 && a.out_stride < width) return bad("ps_paged_attn: rows of out overlap");
    // In place a row's queries are loaded by the CTAs that attend it before its result is stored: by the CTA that has the
    // whole row, or behind all of them by the join.
    if (!(a.out == a.q && (a.out_stride == a.q_stride || a.batch == 1)) &&
        ps::rows_meet({a.out, a.out_stride, width}, {a.q, a.q_stride, width}, a.batch))
        return bad("ps_paged_attn: out overlaps q by another stride or in part");
    // The places of all segments are counted in 32 bits.  A segment has a place for every tile that its table row has room
    // for and at most 4 more, and a tile's tokens times the KV heads are 24 (3 KV heads of 33 query heads each) times a
    // row's segments or more: with 1024 more tokens a row, 2^34 tokens times KV heads always fit.
    const int64_t room = std::min<int64_t>((int64_t)a.table_stride * a.block_size, kMaxTokens);
    const Layout places = layout_of(a.batch, a.num_kv_heads, a.num_q_heads, a.head_dim, 1);
    if ((room >> places.step_log2) + 4 > (1 << 30) / ((int64_t)a.batch * places.chunks))
        return bad("ps_paged_attn: the tables of the batch have room for more than 2^30 tiles of tokens");
    int sms = 0;
    cudaError_t e = device_sms(&sms);
    if (e != cudaSuccess) return ps::launch_fail(err_buf, err_cap, "ps_paged_attn: device", e);
    const Layout y = layout_of(a.batch, a.num_kv_heads, a.num_q_heads, a.head_dim, sms);
    if (a.workspace_bytes < (int64_t)y.bytes || (reinterpret_cast<uintptr_t>(a.workspace) & 255))
        return bad("ps_paged_attn: the workspace is smaller than ps_paged_attn_workspace says, or not on a 256-byte boundary");
    AttnParams p{};
    p.kpool = a.kpool, p.vpool = a.vpool, p.q = a.q, p.out = a.out, p.lse = a.lse;
    p.tables = a.block_tables, p.ctx = a.ctx_lens, p.status = a.status_word;
    char* ws = (char*)a.workspace;
    p.part_o = (float*)(ws + y.part_o);
    p.part_ml = (float2*)(ws + y.part_ml);
    p.cuts = (int4*)(ws + y.cuts);
    p.k_block_stride = a.k_block_stride, p.v_block_stride = a.v_block_stride, p.q_stride = a.q_stride, p.out_stride = a.out_stride;
    p.room = room;
    p.block_magic = a.block_size > 1 ? ~0ull / (uint64_t)a.block_size + 1 : 0;
    p.batch = a.batch, p.table_stride = a.table_stride, p.num_blocks = a.num_gpu_blocks, p.block_size = a.block_size, p.window = a.window;
    p.hkv = a.num_kv_heads, p.hq = a.num_q_heads, p.group = a.num_q_heads / a.num_kv_heads;
    p.splits = y.splits, p.rows = y.rows, p.units = y.units, p.chunks = y.chunks, p.subs = y.subs, p.ctas = y.ctas;
    p.step_log2 = y.step_log2;
    p.scale_log2e = (a.scale != 0.f ? a.scale : 1.f / sqrtf((float)a.head_dim)) * kLog2e;
    // A segment's start and end take about the time of two tiles.  Not counted (1 in brackets), 200 rows of 10 to 100 tokens
    // take 20.2 instead of 17.2 us (17.9), 33 ragged rows with a window 19.6 instead of 18.1 (18.8), 64 rows of 1024 to
    // 4096 102.4 either way.  With few segments a CTA has one whatever it costs.
    p.segment = (int64_t)a.batch * y.chunks >= y.ctas / 8 ? 2 : 0;
    // rows that cannot be longer than one tile are never cut
    const int64_t longest = a.window > 0 && a.window < p.room ? a.window : p.room;
    const bool may_cut = longest > (int64_t)1 << p.step_log2;
    cudaStream_t s = (cudaStream_t)stream;
    if (a.dtype == PS_DTYPE_BF16)
        e = a.head_dim == 128 ? launch_attn<__nv_bfloat16, 128>(p, y, may_cut, s) : launch_attn<__nv_bfloat16, 64>(p, y, may_cut, s);
    else
        e = a.head_dim == 128 ? launch_attn<__half, 128>(p, y, may_cut, s) : launch_attn<__half, 64>(p, y, may_cut, s);
    if (e != cudaSuccess) return ps::launch_fail(err_buf, err_cap, "ps_paged_attn", e);
    return PS_OK;
}

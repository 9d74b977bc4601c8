// ps_paged_attn: attention of one new token per row over a paged KV cache, with the lengths and block tables on the
// device.  Nothing about the batch but its size is known on the host, so the call can be replayed from a graph.
//
//   out[b][h] = sum_t p_t V[t][h / G] / sum_t p_t,   p_t = 2^(s_t - m),   s_t = log2(e) scale q[b][h] . K[t][h / G],
//   max(0, ctx_b - window) <= t < ctx_b,   m = max_t s_t (running),   lse = ln 2 (m + log2 sum_t p_t)
//
// Bound: HBM.  A token and KV head cost 4 D bytes and 4 G D flops; up to G = 64 the card computes faster than it
// loads.  So the kernel is built around the loads:
//
//  * Fragments come straight from global memory.  mma.m16n8k16 contracts over k, and the order of k is free as long
//    as both operands use the same one; so is the order of the 8 columns of a product.  A lane therefore loads 32
//    contiguous bytes of a key row, which are its B operands of four products (the query is loaded in the same
//    order), and for V 16 bytes (D = 64) or 32 bytes (D = 128) of four token rows, whose halves are paired by byte
//    permutes.  No shared memory, no barrier, no transposing load lies between HBM and the tensor cores, tokens may
//    lie anywhere (any block size, any block stride), and every warp runs on its own.
//    (The tile shapes of tcgen05.mma need 64 or 128 rows; a group of at most 16 query heads would leave most idle.)
//  * The next tile's keys are requested before the softmax of the present one and its values before the next
//    products, so a warp has 4 to 8 KiB in flight throughout.
//
// Work: the rows' tiles form one sequence that is cut into equal shares, one per CTA, from the lengths each CTA
// reads itself: no plan is made on the host or by another kernel.  A row cut by a share's end leaves partial
// results (m, sum, accumulators) in the workspace, which a second kernel (paged_join_kernel) combines in order.
// The join is a second launch rather than a last-arrival counter in the first: the workspace then needs no
// initial state, and neither a replayed graph nor a call that shares it in turn can find a stale counter.
//
// Warps: a CTA works on `units` (KV head, group of at most 16 query heads) times `subs` token slices; the units of a
// token are neighbours in memory.  The slices' states are combined through shared memory at a segment's end.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

#include <atomic>
#include <cmath>

#include "ps_internal.h"
#include "ps_kvswap.h"

namespace {

constexpr int kMaxWarps = 8;
constexpr int kTile = 16;             // tokens of a warp's tile
constexpr int kMaxGroup = 16;         // query heads of a unit
constexpr int kCtaFactor = 1;         // CTAs per SM
constexpr int kJoinThreads = 128;
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
    int4* cuts;          // [cta]: a segment that begins in this CTA and ends in a later one: {row, chunk, parts, 0}
    int64_t k_block_stride, v_block_stride, q_stride, out_stride;
    int64_t room;        // tokens a table row has room for
    uint64_t block_magic;
    int32_t batch, table_stride, num_blocks, block_size, window;
    int32_t hkv, hq, group;          // group: query heads per KV head
    int32_t splits, rows;            // a KV head's query heads are cut into `splits` units of `rows` heads
    int32_t units, chunks, subs;     // units per CTA, CTAs' worth of units per row, token slices
    float scale_log2e;
};

// ------------------------------------------------------------------------------------------------ pieces

template <typename T> struct Num;
template <> struct Num<__nv_bfloat16> {
    static constexpr float kLift = 0.f;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    static __device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                               uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};
template <> struct Num<__half> {
    // p is rounded to fp16 for the product with V.  Its largest value is 1 and fp16 loses relative precision below
    // 2^-14, so p is computed 2^14 times larger (the sum carries the same factor, and both cancel).
    static constexpr float kLift = 14.f;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    static __device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                               uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};

__device__ __forceinline__ void ld32(const void* p, uint32_t* r) {   // 32 bytes, read once
    asm volatile("ld.global.nc.L1::no_allocate.L2::evict_first.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "l"(p));
}
__device__ __forceinline__ void ld16(const void* p, uint32_t* r) {
    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "l"(p));
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

// Tokens of row b that are attended: [first, end).
__device__ __forceinline__ void row_span(const AttnParams& p, int b, int32_t* first, int32_t* end) {
    const int32_t n = p.ctx[b];
    int32_t e = n < 0 ? 0 : n;
    if ((int64_t)e > p.room) e = (int32_t)p.room;
    if (e != n && p.status) *(volatile int32_t*)p.status = kStatusLength;
    *end = e;
    *first = p.window > 0 && e > p.window ? e - p.window : 0;
}
__device__ __forceinline__ int32_t row_tiles(const AttnParams& p, int b) {
    int32_t first, end;
    row_span(p, b, &first, &end);
    const int32_t step = kTile * p.subs;
    return end > first ? (end - first + step - 1) / step : 1;   // an empty row still has a result to write
}

// Where a unit's queries are: heads [h0, h0 + n).
__device__ __forceinline__ void unit_heads(const AttnParams& p, int unit, int* kv, int* h0, int* n) {
    *kv = unit / p.splits;
    const int s = unit - *kv * p.splits;
    *h0 = *kv * p.group + s * p.rows;
    *n = min(p.rows, p.group - s * p.rows);
}

// A tile's tokens: lane l < 16 holds block id and place in the block of token l (-1: not attended).
struct TileIds {
    int32_t id, at;
};

// The softmax state of a warp: rows lane / 4 and lane / 4 + 8, dims [D/4 * c, D/4 * (c + 1)) with c = lane % 4;
// acc[j][0], acc[j][1] are the dims D/4 * c + j and D/4 * c + D/8 + j of the first row, [2], [3] of the second.
template <int D>
struct State {
    float m[2], l[2];
    float acc[D / 8][4];
};

// -------------------------------------------------------------------------------------------- main kernel

template <typename T, int D, int MR>
struct Worker {
    static constexpr int KC = D / 64;          // 32-byte pieces of a key row per lane
    static constexpr int VW = D / 16;          // registers of a value row per lane
    const AttnParams& p;
    const int lane, g, c;
    uint32_t q0[KC][8], q1[KC][8];             // query rows g and g + 8 in the key's order
    uint32_t k[2][KC][8];                      // keys of tokens g and g + 8
    uint32_t v[4][VW];                         // values of tokens 2c, 2c + 1, 2c + 8, 2c + 9
    TileIds ids;
    uint32_t mask, next_mask;                  // tokens of the tile that are attended

    __device__ __forceinline__ Worker(const AttnParams& pp) : p(pp), lane(threadIdx.x & 31), g((threadIdx.x & 31) >> 2), c(threadIdx.x & 3) {}

    __device__ __forceinline__ void load_query(int b, int h0, int n) {
        const T* q = (const T*)p.q + b * p.q_stride + (int64_t)h0 * D;
#pragma unroll
        for (int j = 0; j < KC; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) q0[j][i] = q1[j][i] = 0;
            if (g < n) {
                ld16(q + g * D + 64 * j + 16 * c, q0[j]);
                ld16(q + g * D + 64 * j + 16 * c + 8, q0[j] + 4);
            }
            if (MR == 16 && g + 8 < n) {
                ld16(q + (g + 8) * D + 64 * j + 16 * c, q1[j]);
                ld16(q + (g + 8) * D + 64 * j + 16 * c + 8, q1[j] + 4);
            }
        }
    }

    __device__ __forceinline__ void load_ids(const int32_t* table, int32_t t0, int32_t end) {
        const int32_t t = t0 + (lane & 15);
        ids.id = -1;
        ids.at = 0;
        if (t < end) {
            const int32_t blk = block_of(t, p);
            const int32_t id = __ldg(table + blk);
            ids.at = t - blk * p.block_size;
            if ((unsigned)id < (unsigned)p.num_blocks) ids.id = id;
            else if (p.status) *(volatile int32_t*)p.status = kStatusBadId;
        }
        next_mask = __ballot_sync(0xffffffffu, ids.id >= 0) & 0xffffu;
    }

    __device__ __forceinline__ void load_keys(int kv) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int32_t id = __shfl_sync(0xffffffffu, ids.id, g + 8 * r), at = __shfl_sync(0xffffffffu, ids.at, g + 8 * r);
            const T* row = (const T*)p.kpool + id * p.k_block_stride + ((int64_t)at * p.hkv + kv) * D + 16 * c;
            if (next_mask == 0xffffu) {
#pragma unroll
                for (int j = 0; j < KC; ++j) ld32(row + 64 * j, k[r][j]);
            } else {
#pragma unroll
                for (int j = 0; j < KC; ++j) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) k[r][j][i] = 0;
                    if (id >= 0) ld32(row + 64 * j, k[r][j]);
                }
            }
        }
    }

    __device__ __forceinline__ void load_values(int kv) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int tok = 2 * c + (r & 1) + 8 * (r >> 1);
            const int32_t id = __shfl_sync(0xffffffffu, ids.id, tok), at = __shfl_sync(0xffffffffu, ids.at, tok);
            const T* row = (const T*)p.vpool + id * p.v_block_stride + ((int64_t)at * p.hkv + kv) * D + (D / 8) * g;
            if (next_mask == 0xffffu) {
                if constexpr (D == 128) ld32(row, v[r]); else ld16(row, v[r]);
            } else {   // a value that is not attended must not reach the product, where 0 times a NaN is a NaN
#pragma unroll
                for (int i = 0; i < VW; ++i) v[r][i] = 0;
                if (id >= 0) {
                    if constexpr (D == 128) ld32(row, v[r]); else ld16(row, v[r]);
                }
            }
        }
    }

    // Attends this warp's tiles of tokens [t_lo, t_hi): those with index = sub modulo subs.
    __device__ __forceinline__ void run(const int32_t* table, int32_t t_lo, int32_t t_hi, int sub, int kv, State<D>& st) {
        const int32_t step = kTile * p.subs;
        int32_t t = t_lo + kTile * sub;
        if (t >= t_hi) return;
        load_ids(table, t, t_hi);
        mask = next_mask;
        load_keys(kv);
        load_values(kv);
        t += step;
        bool more = t < t_hi;
        if (more) load_ids(table, t, t_hi);
        while (true) {
            float s[2][4];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                s[r][0] = s[r][1] = s[r][2] = s[r][3] = 0.f;
#pragma unroll
                for (int j = 0; j < KC; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        Num<T>::mma(s[r], q0[j][2 * i], MR == 16 ? q1[j][2 * i] : 0u, q0[j][2 * i + 1],
                                    MR == 16 ? q1[j][2 * i + 1] : 0u, k[r][j][2 * i], k[r][j][2 * i + 1]);
            }
            if (more) load_keys(kv);
            // scores in base 2; columns 2c, 2c + 1 of the two products are tokens 8r + 2c, 8r + 2c + 1
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int i = 0; i < MR / 4; ++i) s[r][i] *= p.scale_log2e;
            if (mask != 0xffffu) {
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int i = 0; i < MR / 4; ++i)
                        if (!(mask >> (8 * r + 2 * c + (i & 1)) & 1)) s[r][i] = -CUDART_INF_F;
            }
            bool grown = false;
            float m_new[2], alpha[2];
#pragma unroll
            for (int h = 0; h < MR / 8; ++h) {
                float mx = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                m_new[h] = fmaxf(st.m[h], mx);
                grown |= m_new[h] > st.m[h];
            }
            if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
                for (int h = 0; h < MR / 8; ++h) {
                    // a row that has seen nothing has m = -inf and sum 0: its factor is 0 and not a NaN
                    alpha[h] = st.m[h] == m_new[h] ? 1.f : ex2(st.m[h] - m_new[h]);
                    st.m[h] = m_new[h];
                    st.l[h] *= alpha[h];
#pragma unroll
                    for (int j = 0; j < D / 8; ++j) {
                        st.acc[j][2 * h] *= alpha[h];
                        st.acc[j][2 * h + 1] *= alpha[h];
                    }
                }
            }
            uint32_t a[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int h = 0; h < MR / 8; ++h) {
                const float m = st.m[h] == -CUDART_INF_F ? 0.f : st.m[h] - Num<T>::kLift;
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float e0 = ex2(s[r][2 * h] - m), e1 = ex2(s[r][2 * h + 1] - m);
                    st.l[h] += e0 + e1;
                    a[2 * r + h] = Num<T>::pack(e0, e1);
                }
            }
#pragma unroll
            for (int j = 0; j < D / 8; ++j) {
                const uint32_t sel = j & 1 ? 0x7632u : 0x5410u;
                Num<T>::mma(st.acc[j], a[0], a[1], a[2], a[3], __byte_perm(v[0][j / 2], v[1][j / 2], sel),
                            __byte_perm(v[2][j / 2], v[3][j / 2], sel));
            }
            if (!more) break;
            load_values(kv);
            mask = next_mask;
            t += step;
            more = t < t_hi;
            if (more) load_ids(table, t, t_hi);
        }
    }
};

template <int D, int MR>
__device__ __forceinline__ void state_reset(State<D>& st) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        st.m[h] = -CUDART_INF_F;
        st.l[h] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < D / 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) st.acc[j][i] = 0.f;
}

// Joins another state into st: weights 2^(m - max), 0 for a side that has seen nothing.
__device__ __forceinline__ void join_weights(float m, float m2, float* m_new, float* w, float* w2) {
    *m_new = fmaxf(m, m2);
    *w = m == *m_new ? 1.f : ex2(m - *m_new);
    *w2 = m2 == *m_new ? 1.f : ex2(m2 - *m_new);
}

template <typename T, int D, int MR>
__global__ void __launch_bounds__(kMaxWarps * 32, 1)
paged_attn_kernel(const __grid_constant__ AttnParams p) {
    extern __shared__ float4 xchg[];   // [(subs - 1) * units][MR / 8 * (D / 16 + 1)][32]
    constexpr int kXchg = MR / 8 * (D / 16) + 1;
    __shared__ long long sh_sum[kMaxWarps];
    __shared__ long long sh_at;        // tiles before the CTA's first row
    __shared__ int sh_row;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int nwarps = blockDim.x >> 5;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // This CTA's share of the sequence row 0 chunk 0, row 0 chunk 1, ..., row 1 chunk 0, ...
    const int per = (p.batch + blockDim.x - 1) / blockDim.x;
    const int b_lo = min(p.batch, (int)threadIdx.x * per), b_hi = min(p.batch, b_lo + per);
    long long mine = 0;
    for (int b = b_lo; b < b_hi; ++b) mine += row_tiles(p, b);
    mine *= p.chunks;
    long long before = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long n = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += n;
    }
    if (lane == 31) sh_sum[warp] = before;
    __syncthreads();
    long long total = 0;
    before -= mine;
    for (int w = 0; w < nwarps; ++w) {
        if (w < warp) before += sh_sum[w];
        total += sh_sum[w];
    }
    const long long share = (total + gridDim.x - 1) / gridDim.x;
    const long long begin = share * blockIdx.x, end = min(total, begin + share);
    if (begin >= before && begin < before + mine) {
        long long at = before;
        int b = b_lo;
        while (true) {
            const long long n = (long long)row_tiles(p, b) * p.chunks;
            if (begin < at + n) break;
            at += n;
            ++b;
        }
        sh_row = b;
        sh_at = at;
    }
    __syncthreads();
    int4 cut = make_int4(0, 0, 0, 0);
    if (begin < end) {
        int b = sh_row;
        long long seg = sh_at;      // where the row's first chunk begins
        int32_t first, last;
        row_span(p, b, &first, &last);
        int32_t tiles = row_tiles(p, b);
        int chunk = (int)((begin - seg) / tiles);
        seg += (long long)chunk * tiles;
        const int unit_in_cta = warp % p.units, sub = warp / p.units;
        Worker<T, D, MR> wk(p);
        for (long long at = begin; at < end;) {
            const long long seg_end = seg + tiles;
            const int32_t lo = (int32_t)(at - seg), hi = (int32_t)(min(end, seg_end) - seg);
            const int32_t step = kTile * p.subs;
            // of 64 bits where 32 could wrap: lengths go up to 2^31 - 1
            const int32_t t_lo = first + lo * step, t_hi = (int32_t)min((int64_t)last, (int64_t)first + (int64_t)hi * step);
            const int unit = chunk * p.units + unit_in_cta;
            const bool busy = unit < p.hkv * p.splits;
            int kv = 0, h0 = 0, n = 0;
            State<D> st;
            state_reset<D, MR>(st);
            if (busy) {
                unit_heads(p, unit, &kv, &h0, &n);
                wk.load_query(b, h0, n);
                wk.run(p.tables + (int64_t)b * p.table_stride, t_lo, t_hi, sub, kv, st);
#pragma unroll
                for (int h = 0; h < MR / 8; ++h) {
                    st.l[h] += __shfl_xor_sync(0xffffffffu, st.l[h], 1);
                    st.l[h] += __shfl_xor_sync(0xffffffffu, st.l[h], 2);
                }
            }
            if (p.subs > 1) {
                if (sub > 0) {
                    float4* x = xchg + ((sub - 1) * p.units + unit_in_cta) * kXchg * 32 + lane;
                    x[0] = make_float4(st.m[0], st.l[0], st.m[1], st.l[1]);
#pragma unroll
                    for (int j = 0; j < D / 16; ++j) {
                        if constexpr (MR == 16) {
                            x[(1 + 2 * j) * 32] = make_float4(st.acc[2 * j][0], st.acc[2 * j][1], st.acc[2 * j][2], st.acc[2 * j][3]);
                            x[(2 + 2 * j) * 32] =
                                make_float4(st.acc[2 * j + 1][0], st.acc[2 * j + 1][1], st.acc[2 * j + 1][2], st.acc[2 * j + 1][3]);
                        } else {
                            x[(1 + j) * 32] = make_float4(st.acc[2 * j][0], st.acc[2 * j][1], st.acc[2 * j + 1][0], st.acc[2 * j + 1][1]);
                        }
                    }
                }
                __syncthreads();
                if (sub == 0)
                    for (int o = 0; o < p.subs - 1; ++o) {
                        const float4* x = xchg + (o * p.units + unit_in_cta) * kXchg * 32 + lane;
                        const float4 ml = x[0];
                        float w[2], w2[2];
                        join_weights(st.m[0], ml.x, &st.m[0], &w[0], &w2[0]);
                        join_weights(st.m[1], ml.z, &st.m[1], &w[1], &w2[1]);
                        st.l[0] = st.l[0] * w[0] + ml.y * w2[0];
                        st.l[1] = st.l[1] * w[1] + ml.w * w2[1];
#pragma unroll
                        for (int j = 0; j < D / 16; ++j) {
                            if constexpr (MR == 16) {
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const float4 y = x[(1 + 2 * j + e) * 32];
                                    float(&d)[4] = st.acc[2 * j + e];
                                    d[0] = d[0] * w[0] + y.x * w2[0];
                                    d[1] = d[1] * w[0] + y.y * w2[0];
                                    d[2] = d[2] * w[1] + y.z * w2[1];
                                    d[3] = d[3] * w[1] + y.w * w2[1];
                                }
                            } else {
                                const float4 y = x[(1 + j) * 32];
                                st.acc[2 * j][0] = st.acc[2 * j][0] * w[0] + y.x * w2[0];
                                st.acc[2 * j][1] = st.acc[2 * j][1] * w[0] + y.y * w2[0];
                                st.acc[2 * j + 1][0] = st.acc[2 * j + 1][0] * w[0] + y.z * w2[0];
                                st.acc[2 * j + 1][1] = st.acc[2 * j + 1][1] * w[0] + y.w * w2[0];
                            }
                        }
                    }
                __syncthreads();
            }
            const bool whole = lo == 0 && hi == tiles;
            if (busy && sub == 0) {
                const int gg = lane >> 2, cc = lane & 3;
#pragma unroll
                for (int h = 0; h < MR / 8; ++h) {
                    const int r = gg + 8 * h;
                    if (r >= n) continue;
                    if (whole) {
                        const float inv = st.l[h] > 0.f ? 1.f / st.l[h] : st.l[h] == 0.f ? 0.f : CUDART_NAN_F;
                        T* o = (T*)p.out + b * p.out_stride + (int64_t)(h0 + r) * D + (D / 4) * cc;
                        // dims D/4 c + j are acc[j][0], dims D/4 c + D/8 + j acc[j][1]
#pragma unroll
                        for (int e = 0; e < 2; ++e)
#pragma unroll
                            for (int j = 0; j < D / 8; j += 8) {
                                uint4 w;
                                w.x = Num<T>::pack(st.acc[j][2 * h + e] * inv, st.acc[j + 1][2 * h + e] * inv);
                                w.y = Num<T>::pack(st.acc[j + 2][2 * h + e] * inv, st.acc[j + 3][2 * h + e] * inv);
                                w.z = Num<T>::pack(st.acc[j + 4][2 * h + e] * inv, st.acc[j + 5][2 * h + e] * inv);
                                w.w = Num<T>::pack(st.acc[j + 6][2 * h + e] * inv, st.acc[j + 7][2 * h + e] * inv);
                                *reinterpret_cast<uint4*>(o + e * (D / 8) + j) = w;
                            }
                        if (p.lse && cc == 0)
                            p.lse[(int64_t)b * p.hq + h0 + r] =
                                st.l[h] == 0.f ? -CUDART_INF_F : (st.m[h] - Num<T>::kLift + log2f(st.l[h])) * kLn2;
                    } else {
                        const int64_t slot = (((int64_t)blockIdx.x * 2 + (lo == 0)) * p.units + unit_in_cta) * p.rows + r;
                        float* o = p.part_o + slot * D + (D / 4) * cc;
#pragma unroll
                        for (int e = 0; e < 2; ++e)
#pragma unroll
                            for (int j = 0; j < D / 8; j += 4)
                                *reinterpret_cast<float4*>(o + e * (D / 8) + j) =
                                    make_float4(st.acc[j][2 * h + e], st.acc[j + 1][2 * h + e], st.acc[j + 2][2 * h + e], st.acc[j + 3][2 * h + e]);
                        if (cc == 0) p.part_ml[slot] = make_float2(st.m[h], st.l[h]);
                    }
                }
            }
            if (lo == 0 && hi < tiles) cut = make_int4(b, chunk, (int)((seg_end - 1) / share) - (int)blockIdx.x + 1, 0);
            at = seg + hi;
            if (at == seg_end && at < end) {
                seg = seg_end;
                if (++chunk == p.chunks) {
                    chunk = 0;
                    ++b;
                    row_span(p, b, &first, &last);
                    tiles = row_tiles(p, b);
                }
            }
        }
    }
    if (threadIdx.x == 0) p.cuts[blockIdx.x] = cut;
}

// Combines the parts of the rows that a share's end cut: CTA i of the main kernel names in cuts[i] the segment that
// begins in it and goes on, whose parts are slot 1 of CTA i and slot 0 of the CTAs that follow.  Work items are
// (segment, unit, query head), dealt to the CTAs in turn; a CTA's slices of D / 4 threads take every fourth or eighth
// part each, and the slices are combined in order, so a result does not depend on timing.
template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads)
paged_join_kernel(const __grid_constant__ AttnParams p, int32_t ctas) {
    constexpr int kLanes = D / 4;            // a lane owns 4 dims
    constexpr int kSlices = kJoinThreads / kLanes;
    extern __shared__ int4 list[];           // [ctas]: the cuts; .w is the CTA that a segment begins in
    __shared__ float sm_m[kSlices], sm_l[kSlices];
    __shared__ float4 sm_o[kSlices][kLanes];
    __shared__ int sm_count[kJoinThreads / 32];
    const int lane = threadIdx.x % kLanes, slice = threadIdx.x / kLanes;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    int count = 0;
    for (int i0 = 0; i0 < ctas; i0 += kJoinThreads) {
        const int i = i0 + threadIdx.x;
        const int4 cut = i < ctas ? __ldcg(p.cuts + i) : make_int4(0, 0, 0, 0);
        const unsigned some = __ballot_sync(0xffffffffu, cut.z != 0);
        if ((threadIdx.x & 31) == 0) sm_count[threadIdx.x >> 5] = __popc(some);
        __syncthreads();
        int at = count + __popc(some & ((1u << (threadIdx.x & 31)) - 1));
        for (int w = 0; w < kJoinThreads / 32; ++w) {
            if (w < (int)(threadIdx.x >> 5)) at += sm_count[w];
            count += sm_count[w];
        }
        if (cut.z != 0) list[at] = make_int4(cut.x, cut.y, cut.z, i);
        __syncthreads();
    }
    const int per = p.units * p.rows;
    for (int item = blockIdx.x; item < count * per; item += gridDim.x) {
        {
            const int seg = item / per, k = item - seg * per;
            const int4 cut = list[seg];
            const int i = cut.w;
            const int u = k / p.rows, r = k - u * p.rows;
            const int unit = cut.y * p.units + u;
            if (unit >= p.hkv * p.splits) continue;
            int kv, h0, n;
            unit_heads(p, unit, &kv, &h0, &n);
            if (r >= n) continue;
            float m = -CUDART_INF_F, l = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int q = slice; q < cut.z; q += kSlices) {
                const int64_t slot = (((int64_t)(i + q) * 2 + (q == 0)) * p.units + u) * p.rows + r;
                const float2 ml = __ldcg(p.part_ml + slot);
                const float4 x = __ldcg(reinterpret_cast<const float4*>(p.part_o + slot * D) + lane);
                float w, w2;
                join_weights(m, ml.x, &m, &w, &w2);
                l = l * w + ml.y * w2;
                o.x = o.x * w + x.x * w2;
                o.y = o.y * w + x.y * w2;
                o.z = o.z * w + x.z * w2;
                o.w = o.w * w + x.w * w2;
            }
            __syncthreads();
            if (lane == 0) {
                sm_m[slice] = m;
                sm_l[slice] = l;
            }
            sm_o[slice][lane] = o;
            __syncthreads();
            if (slice == 0) {
#pragma unroll
                for (int q = 1; q < kSlices; ++q) {
                    float w, w2;
                    join_weights(m, sm_m[q], &m, &w, &w2);
                    const float4 x = sm_o[q][lane];
                    l = l * w + sm_l[q] * w2;
                    o.x = o.x * w + x.x * w2;
                    o.y = o.y * w + x.y * w2;
                    o.z = o.z * w + x.z * w2;
                    o.w = o.w * w + x.w * w2;
                }
                const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : CUDART_NAN_F;
                uint2 w;
                w.x = Num<T>::pack(o.x * inv, o.y * inv);
                w.y = Num<T>::pack(o.z * inv, o.w * inv);
                *reinterpret_cast<uint2*>((T*)p.out + cut.x * p.out_stride + (int64_t)(h0 + r) * D + 4 * lane) = w;
                if (p.lse && lane == 0)
                    p.lse[(int64_t)cut.x * p.hq + h0 + r] = l == 0.f ? -CUDART_INF_F : (m - Num<T>::kLift + log2f(l)) * kLn2;
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------------- host

// How the heads are dealt to warps; the same for a shape on every call.
struct Layout {
    int32_t splits, rows, units, chunks, subs, ctas;
    int mr;
    size_t part_o, part_ml, cuts, bytes;   // offsets and size of the workspace
};

Layout layout_of(int32_t hkv, int32_t hq, int32_t dim, int sms) {
    Layout y{};
    const int32_t group = hq / hkv;
    y.splits = (group + kMaxGroup - 1) / kMaxGroup;
    y.rows = (group + y.splits - 1) / y.splits;
    y.mr = y.rows <= 8 ? 8 : 16;
    const int32_t all = hkv * y.splits;
    y.chunks = (all + kMaxWarps - 1) / kMaxWarps;
    y.units = (all + y.chunks - 1) / y.chunks;
    y.subs = kMaxWarps / y.units;
    y.ctas = sms * kCtaFactor;
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    const size_t slots = (size_t)y.ctas * 2 * y.units * y.rows;
    y.part_o = 0;
    y.part_ml = up(slots * dim * sizeof(float));
    y.cuts = y.part_ml + up(slots * sizeof(float2));
    y.bytes = y.cuts + up((size_t)y.ctas * sizeof(int4));
    return y;
}

constexpr int kMaxDevices = 64;

// SM count of the current device; looked up once per device.  The kernels' shared memory limit is raised there too.
template <typename T, int D, int MR>
cudaError_t allow_smem() {
    return cudaFuncSetAttribute(paged_attn_kernel<T, D, MR>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (kMaxWarps - 1) * (MR / 8 * (D / 16) + 1) * 32 * (int)sizeof(float4));
}
cudaError_t device_sms(int* sms) {
    static std::atomic<int> known[kMaxDevices];
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    *sms = known[dev].load(std::memory_order_acquire);
    if (*sms > 0) return cudaSuccess;
    e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = allow_smem<__nv_bfloat16, 64, 8>();
    if (e == cudaSuccess) e = allow_smem<__nv_bfloat16, 64, 16>();
    if (e == cudaSuccess) e = allow_smem<__nv_bfloat16, 128, 8>();
    if (e == cudaSuccess) e = allow_smem<__nv_bfloat16, 128, 16>();
    if (e == cudaSuccess) e = allow_smem<__half, 64, 8>();
    if (e == cudaSuccess) e = allow_smem<__half, 64, 16>();
    if (e == cudaSuccess) e = allow_smem<__half, 128, 8>();
    if (e == cudaSuccess) e = allow_smem<__half, 128, 16>();
    if (e == cudaSuccess) known[dev].store(*sms, std::memory_order_release);
    return e;
}

template <typename T, int D>
cudaError_t launch_attn(const AttnParams& p, const Layout& y, bool may_cut, cudaStream_t s) {
    const dim3 block((unsigned)(32 * y.units * y.subs));
    const size_t smem = (size_t)(y.subs - 1) * y.units * (y.mr / 8 * (D / 16) + 1) * 32 * sizeof(float4);
    cudaError_t e = y.mr == 8 ? ps::launch_dependent(paged_attn_kernel<T, D, 8>, dim3((unsigned)y.ctas), block, smem, s, p)
                              : ps::launch_dependent(paged_attn_kernel<T, D, 16>, dim3((unsigned)y.ctas), block, smem, s, p);
    if (e == cudaSuccess && may_cut)
        e = ps::launch_dependent(paged_join_kernel<T, D>, dim3((unsigned)y.ctas * 8), dim3(kJoinThreads),
                                 (size_t)y.ctas * sizeof(int4), s, p, y.ctas);
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
    *bytes = (int64_t)layout_of(num_kv_heads, num_q_heads, head_dim, sms).bytes;
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
    if (!on(a.kpool, a.k_block_stride, 32) || !on(a.vpool, a.v_block_stride, 32))
        return bad("ps_paged_attn: pools and their block strides must be multiples of 32 bytes");
    if (!on(a.q, a.q_stride, 16) || !on(a.out, a.out_stride, 16))
        return bad("ps_paged_attn: q, out and their row strides must be multiples of 16 bytes");
    if (a.batch > 1 && a.out_stride < (int64_t)a.num_q_heads * a.head_dim) return bad("ps_paged_attn: rows of out overlap");
    int sms = 0;
    cudaError_t e = device_sms(&sms);
    if (e != cudaSuccess) return ps::launch_fail(err_buf, err_cap, "ps_paged_attn: device", e);
    const Layout y = layout_of(a.num_kv_heads, a.num_q_heads, a.head_dim, sms);
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
    p.room = (int64_t)a.table_stride * a.block_size;
    if (p.room > kMaxTokens) p.room = kMaxTokens;
    p.block_magic = a.block_size > 1 ? ~0ull / (uint64_t)a.block_size + 1 : 0;
    p.batch = a.batch, p.table_stride = a.table_stride, p.num_blocks = a.num_gpu_blocks, p.block_size = a.block_size, p.window = a.window;
    p.hkv = a.num_kv_heads, p.hq = a.num_q_heads, p.group = a.num_q_heads / a.num_kv_heads;
    p.splits = y.splits, p.rows = y.rows, p.units = y.units, p.chunks = y.chunks, p.subs = y.subs;
    p.scale_log2e = (a.scale != 0.f ? a.scale : 1.f / sqrtf((float)a.head_dim)) * kLog2e;
    // rows that cannot be longer than one tile are never cut
    const int64_t longest = a.window > 0 && a.window < p.room ? a.window : p.room;
    const bool may_cut = longest > (int64_t)kTile * y.subs;
    cudaStream_t s = (cudaStream_t)stream;
    if (a.dtype == PS_DTYPE_BF16)
        e = a.head_dim == 128 ? launch_attn<__nv_bfloat16, 128>(p, y, may_cut, s) : launch_attn<__nv_bfloat16, 64>(p, y, may_cut, s);
    else
        e = a.head_dim == 128 ? launch_attn<__half, 128>(p, y, may_cut, s) : launch_attn<__half, 64>(p, y, may_cut, s);
    if (e != cudaSuccess) return ps::launch_fail(err_buf, err_cap, "ps_paged_attn", e);
    return PS_OK;
}

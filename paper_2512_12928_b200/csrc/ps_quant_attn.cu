// ps_quant_attn: attention of one new token per row over a paged cache of 8-bit codes with a scale for each block and KV
// head, K[t] = a_t k_t and V[t] = b_t v_t with whole numbers or 8-bit floats k_t, v_t.
//
//   out[b][h] = sum_t p_t b_t v_t / sum_t p_t,   p_t = 2^(s_t - m),   s_t = log2(e) scale a_t (q[b][h] . k_t)
//
// with the frame of ps_paged_attn.cuh: the sequence's cut, the walk, segment ends and the join are ps_paged_attn's.
//
// Bound: HBM, and next to it the instructions that a code costs: a token and KV head are half the bytes of a 16-bit cache's and
// as many products and weights.  Measured: 337 MB of cache (64 rows of 1024 to 4096 tokens, 32 query heads on 8 KV heads of 128)
// 62.7 us in int8 and 60.0 in 8-bit floats (16 bits: 101), about 7 us of which pass before the first tile is there, where rows
// end and in the join; 1.07 GB (rows of 8192) 175 and 168 us, of which a copy would take 167; one row of 500 tokens 9.1.  Heads
// of 64 take 63.1 us for as many bytes in int8; 16 query heads on a KV head of 128 85 and 75 us, of 64 98 and 88.  More than 16
// copy the tiles once for every 16, as in 16 bits.
//
// Products: S^T = K Q^T and O^T = V^T P^T as in ps_paged_attn.cu, tokens and then dims as the 16 rows of a product.  A tile of
// 16 or 32 tokens comes to shared memory as it lies in the pool (cp.async, 16 bytes a lane).  ldmatrix sees pairs of codes as its
// elements: a lane gets four neighbouring dims of a token's key, and through the transposing form two neighbouring dims of
// two tokens' values.  Which dims and tokens a product's rows and columns stand for is free, so what comes together stays
// together: of values row g is dim 2g and row g + 8 dim 2g + 1, and queries are laid out as keys come.
//
// Codes are widened to fp16 between ldmatrix and the product; every code is exact there.  Queries in fp16 are multiplied as they
// are.  Those in bf16 are multiplied by a power of two that puts their head's largest magnitude next to 2^13, and the scores by
// its inverse: what is above 2^-27 of the largest stays exact, and what is below is off by 2^-38 of it at most.
// (Keys in int8 could enter mma.m16n8k32 as they are, with a query as a whole number in three digits of 8 bits: the case above in
// 62.0 us, rows of 8192 in 173.  But then a query has 22 bits from its head's largest value on, and with one dim 2^12 times the
// others, which meets codes near zero, a score lost 3e-4.  A fourth digit spills registers: 70.9 us.)
//
// Scales: a_t multiplies a score in 32 bits.  b_t goes into the weight, p_t (b_t / r) with r a power of two next to the
// largest b that the warp has met, so that weights stay within fp16; sums are multiplied by r where a segment ends.  A weight
// is the sum of two fp16 numbers: with one, a tenth of the results in bf16 were not the nearest to the exact value (0.02 % with
// two, 0.06 % in plain 32-bit arithmetic), for 2 % of the time (9 % with 9 to 16 query heads on a KV head).
#include <cuda_fp8.h>

#include "ps_paged_attn.cuh"

namespace {

// Four codes of a register as two pairs of fp16 numbers.
struct Int8 {
    static constexpr bool kAlternate = true;             // keys come as codes 0 and 2, 1 and 3
    // a byte b with its top bit turned is k + 128; as the low bits of 0x6400 = 1024 that is 1152 + k, exactly
    static __device__ __forceinline__ uint32_t widen(uint32_t x) {
        uint32_t r;
        asm("{\n.reg .b32 v;\nlop3.b32 v, %1, 0x00ff00ff, 0x64806480, 0x6a;\nsub.f16x2 %0, v, %2;\n}" : "=r"(r) : "r"(x), "r"(0x64806480u));
        return r;
    }
    static __device__ __forceinline__ void values(uint32_t x, uint32_t& lo, uint32_t& hi) {      // codes 0 and 2, 1 and 3
        lo = widen(x);
        hi = widen(x >> 8);
    }
    static __device__ __forceinline__ void keys(uint32_t x, uint32_t& lo, uint32_t& hi) { values(x, lo, hi); }
};
struct E4m3 {
    static constexpr bool kAlternate = false;
    static __device__ __forceinline__ void keys(uint32_t x, uint32_t& lo, uint32_t& hi) {        // codes 0 and 1, 2 and 3
        asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %2;\ncvt.rn.f16x2.e4m3x2 %0, l;\ncvt.rn.f16x2.e4m3x2 %1, h;\n}" : "=r"(lo), "=r"(hi) : "r"(x));
    }
    static __device__ __forceinline__ void values(uint32_t x, uint32_t& lo, uint32_t& hi) { keys(__byte_perm(x, 0, 0x3120), lo, hi); }
};

// d = a b (first), or d + a b
__device__ __forceinline__ void mma_f16(bool first, float (&d)[4], const uint4& a, uint32_t b0, uint32_t b1) {
    if (first)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                     : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                     : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1), "f"(0.f));
    else
        Num<__half>::mma(d, a, b0, b1);
}

// Tiles of 16 U tokens, and as many bytes on their way for either head size.
template <int D, int NT, int U, int Warps>
struct Ring {
    static constexpr int kTokens = 16 * U;                   // of a tile
    static constexpr int kRowBytes = D;
    static constexpr int kSideBytes = kTokens * kRowBytes;   // keys, then values, then their scales
    static constexpr int kTileBytes = 2 * kSideBytes + 2 * kTokens * (int)sizeof(float);
    static constexpr int kStateBytes = 8 * NT * D * (int)sizeof(float);      // a stage takes a unit's sums where a segment ends
    static constexpr int kStageBytes = kTileBytes > kStateBytes ? kTileBytes : kStateBytes;
    static constexpr int kStages = (Warps == 16 ? 13056 : 26112) / kStageBytes;
    static constexpr int kWarpBytes = kStages * kStageBytes;
};

template <int D, int NT>
struct QuantState : State<D, NT> {
    float inv_ref;                             // 1 / r
};

// Warps of a CTA, of which an SM has one: 16 of 128 registers a thread for units of up to 8 query heads, 8 for up to 16, which need
// twice as many.  A warp's instructions wait for one another more than for memory, and four a scheduler fill the gaps (64 rows
// of 1024 to 4096 tokens, 32 query heads on 8 of 128: 62.7 us in int8 with 16 warps and 72.4 with 8, 60.0 and 70.1 in 8-bit
// floats; of 64 dims and 2048 to 8192 tokens 63.1 and 73.9 in int8).  Short calls pay for it (one row of 300 tokens: 9.1 and 8.0,
// 200 rows of 10 to 100 19.4 and 17.2).  What 16 warps' registers do not hold costs more than it gives for 16 heads of 64 (88 us
// with 8 warps, 93 with 16).
// As two CTAs of 8 warps they do not wait for one another where a row ends, but a row has twice as many parts and what lies
// next to one another is not read at the same time (the same in int8: 66.6 us, and 17.6 for the short rows).
constexpr int warps_of(int nt) { return nt == 1 ? 16 : 8; }
constexpr int groups_of(int dim, int nt) { return nt == 1 && dim == 128 ? 1 : 2; }     // of 16 tokens, in a tile

template <typename T, typename C, int D, int NT>
struct Worker {
    static constexpr int U = groups_of(D, NT), kWarps = warps_of(NT);
    using Stages = Ring<D, NT, U, kWarps>;
    using R = Stages;
    using Type = T;
    using Softmax = QuantState<D, NT>;
    using Keys = uint4[U][D / 32];
    using N = Num<__half>;
    static constexpr int kDim = D, kColumns = NT;
    static constexpr int kPieces = D / 16;     // of a token's row, 16 bytes each
    static constexpr int kRows = 32 / kPieces; // of a warp's copy
    const AttnParams& p;
    const int lane, g, c, unit_in_cta, sub;
    const uint32_t ring;                       // the warp's first stage
    const uint64_t policy;
    const int32_t my_token;                    // of a tile of all slices: the one that this lane looks up
    const uint32_t scale_put;                  // the place of its scale in a stage
    uint32_t put;                              // this lane's place in a stage: row lane / kPieces and, in place, piece lane % kPieces
    uint32_t get;                              // what this lane reads of a stage's half: piece 0 or 1 of its row; piece 2 j + .. is at get ^ 32 j
    // query head 8 t + g, dims 32 j + 4 c + .. of four and dims 32 j + 16 + 4 c + .. of four, in the order of the keys' codes
    uint32_t q[NT][D / 32][4];
    float factor[NT][2];                       // of the scores of heads 8 t + 2 c and 8 t + 2 c + 1, with log2(e) scale in it
    const unsigned char *k_src, *v_src;        // pools at this lane's head and piece
    const float* scale_src;                    // scales of the head: keys', and with one group of tokens the upper lanes' values'
    const int32_t* table;
    int32_t id, at;                            // block and place of token lane % kTokens; at = -1: no token
    bool idle;                                 // the unit does not exist
    uint32_t masks[R::kStages - 1];            // which tokens of the tiles in the ring are attended, the oldest first

    __device__ __forceinline__ Worker(const AttnParams& pp, uint32_t smem)
        : p(pp), lane(threadIdx.x & 31), g((threadIdx.x & 31) >> 2), c(threadIdx.x & 3), unit_in_cta((threadIdx.x >> 5) % pp.units),
          sub((threadIdx.x >> 5) / pp.units), ring(smem + (threadIdx.x >> 5) * R::kWarpBytes), policy(read_once_policy()),
          my_token(R::kTokens * sub + lane % R::kTokens),
          // tokens g, 8 + g, .. next to one another; with one group of tokens the upper lanes have the values' scales
          scale_put(2 * R::kSideBytes + 4 * (2 * U * (lane & 7) + (lane % R::kTokens >> 3)) + (U == 1 ? 4 * (lane & 16) : 0)), masks{} {
        const int x = lane & 7, up = lane >> 4, mid = lane >> 3 & 1, row = lane / kPieces;
        put = row * D + (((lane % kPieces) ^ swap(row)) << 4);
        get = (x + 8 * mid) * D + ((up ^ swap(x)) << 4);
    }

    // A token's pieces are exclusive-ored with this, so that eight tokens' same piece lie in different banks.
    static __device__ __forceinline__ int swap(int token) { return D == 128 ? token & 7 : token >> 1 & 3; }

    __device__ __forceinline__ void load_query(int b, int h0, int n) {
        constexpr bool kScaled = std::is_same_v<T, __nv_bfloat16>;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const T* src = (const T*)p.q + b * p.q_stride + (int64_t)(h0 + 8 * t + g) * D + 4 * c;
            uint2 v[D / 16];
#pragma unroll
            for (int j = 0; j < D / 16; ++j) v[j] = 8 * t + g < n ? *reinterpret_cast<const uint2*>(src + 16 * j) : make_uint2(0u, 0u);
            float up = 1.f, down = 1.f;
            if constexpr (kScaled) {
                uint32_t most = 0;
#pragma unroll
                for (int j = 0; j < D / 16; ++j) most = __vimax3_u16x2(most, v[j].x & 0x7fff7fffu, v[j].y & 0x7fff7fffu);
                most = max(most & 0xffffu, most >> 16);
                most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
                most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
                // 2^(top - e) for a magnitude of 2^e, and its inverse: both are normal numbers
                constexpr int kTop = 13;
                const uint32_t bits = __float_as_uint(Num<T>::unpack(most).x);
                const int e = min(max((int)(bits >> 23), kTop + 1), 254);
                up = __uint_as_float((uint32_t)(254 + kTop - e) << 23);
                down = __uint_as_float((uint32_t)(e - kTop) << 23);
            }
            factor[t][0] = p.scale_log2e * __shfl_sync(0xffffffffu, down, 8 * c);
            factor[t][1] = p.scale_log2e * __shfl_sync(0xffffffffu, down, 8 * c + 4);
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                const float2 a = Num<T>::unpack(v[j].x), e = Num<T>::unpack(v[j].y);
                q[t][j / 2][2 * (j % 2)] = N::pack(a.x * up, (C::kAlternate ? e.x : a.y) * up);
                q[t][j / 2][2 * (j % 2) + 1] = N::pack((C::kAlternate ? a.y : e.x) * up, e.y * up);
            }
        }
    }

    // The part whose tiles come next.
    __device__ __forceinline__ void enter(const Part& s, int kv) {
        idle = s.n == 0;
        const int64_t o = (int64_t)kv * D + 16 * (lane % kPieces);
        k_src = (const unsigned char*)p.kpool + o;
        v_src = (const unsigned char*)p.vpool + o;
        scale_src = (U == 2 || lane < 16 ? p.k_scale : p.v_scale) + kv;
        table = p.tables + (int64_t)s.b * p.table_stride;
        // the unit's queries, into L1: they are loaded when its tiles have come, and then nothing hides their latency
        if (lane < s.n * D / 64) {
            uint32_t unused;
            asm volatile("ld.global.ca.b32 %0, [%1];" : "=r"(unused) : "l"((const T*)p.q + s.b * p.q_stride + (int64_t)s.h0 * D + lane * 64));
        }
    }

    // Looks up the tokens of the tile that the slices' from token t0 on are, in a row that ends at `end`.
    __device__ __forceinline__ void load_ids(int32_t t0, int32_t end) {
        const int32_t t = t0 + my_token;
        id = 0;
        at = -1;
        if (t < end) {
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
        const uint32_t base = ring + stage * R::kStageBytes, dst = base + put;
        // what is not read has the address of the first block's first token
        const uint32_t blk = read ? id : 0, place = read ? at : 0;
        if (on == 0xffffffffu && p.near) copy_rows<true>(blk, place, on, dst);       // as nearly always
        else copy_rows<false>(blk, place, on, dst);
        const uint32_t four = read ? 4 : 0;
        if (U == 1) {
            copy4(base + scale_put, bytes_on(scale_src, blk, lane < 16 ? p.k_scale_step : p.v_scale_step), four);
        } else {
            copy4(base + scale_put, bytes_on(scale_src, blk, p.k_scale_step), four);
            copy4(base + scale_put + 4 * R::kTokens, bytes_on(scale_src + (p.v_scale - p.k_scale), blk, p.v_scale_step), four);
        }
        return on;
    }
    // The rows of a tile: a lane's token lies in block blk at `place`.  kAll: all are read, and p.near holds.
    template <bool kAll>
    __device__ __forceinline__ void copy_rows(uint32_t blk, uint32_t place, uint32_t on, uint32_t dst) {
        const uint32_t off = blk * p.k_step + place * p.row_step;
#pragma unroll
        for (int i = 0; i < R::kTokens / kRows; ++i) {
            const int row = kRows * i + lane / kPieces;
            const uint32_t to = (D == 128 ? dst ^ (64 * (i & 1)) : dst) + kRows * i * D;     // rows 4 to 7 of 8: piece ^ 4
            if (kAll) {
                const uint32_t o = __shfl_sync(0xffffffffu, off, row);
                copy_whole(to, bytes_on(k_src, o, 16), policy);
                copy_whole(to + R::kSideBytes, bytes_on(v_src, o, 16), policy);
            } else {
                const uint32_t bytes = (on >> row & 1) << 4;
                const uint64_t b = __shfl_sync(0xffffffffu, blk, row), in_block = __shfl_sync(0xffffffffu, place, row) * (uint64_t)p.row_step;
                copy16(to, k_src + 16 * (b * p.k_step + in_block), bytes, policy);
                copy16(to + R::kSideBytes, v_src + 16 * (b * p.v_step + in_block), bytes, policy);
            }
        }
    }
    static __device__ __forceinline__ void copy_whole(uint32_t dst, const void* src, uint64_t policy) {
        asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
    }
    static __device__ __forceinline__ const void* bytes_on(const void* src, uint32_t n, uint32_t step) {      // n steps on
        uint64_t a;
        asm("mad.wide.u32 %0, %1, %2, %3;" : "=l"(a) : "r"(n), "r"(step), "l"(src));
        return reinterpret_cast<const void*>(a);
    }
    static __device__ __forceinline__ void copy4(uint32_t dst, const void* src, uint32_t bytes) {
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
    }
    static __device__ __forceinline__ void floats(uint32_t src, float (&v)[2]) {
        asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v[0]), "=f"(v[1]) : "r"(src) : "memory");
    }
    static __device__ __forceinline__ void floats(uint32_t src, float (&v)[4]) {
        asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(src) : "memory");
    }

    // The keys of the tile in a stage: k[u][j] has 32 dims of 16 tokens.
    __device__ __forceinline__ void read_keys(int stage, Keys& k) const {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < D / 32; ++j) k[u][j] = ldsm(((ring + stage * R::kStageBytes + get) ^ 32 * j) + 16 * u * D);
    }

    __device__ __forceinline__ void reset(Softmax& st) const {
        state_reset(static_cast<State<D, NT>&>(st));
        st.inv_ref = 1.7014118e38f;            // 2^127: any scale raises the reference, and 0 times it is 0
    }
    __device__ __forceinline__ void put_sums(float* row, const Softmax& st, int t, int h) const {
        const float ref = 1.f / st.inv_ref;
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
            *reinterpret_cast<float2*>(row + ((16 * j + 2 * g) ^ (8 * c))) = make_float2(st.acc[t][j][h] * ref, st.acc[t][j][2 + h] * ref);
    }
    // st.m is the reference less N::kLift, so that weights are 2^N::kLift times larger; the frame knows of 2^Num<T>::kLift.
    __device__ __forceinline__ float reference(const Softmax& st, int t, int h) const { return st.m[t][h] + Num<T>::kLift; }

    // Attends the tile in a stage; `on`: its tokens that count.
    __device__ __forceinline__ void attend(int stage, const Keys& k, uint32_t on, Softmax& st) {
        const uint32_t src = ring + stage * R::kStageBytes;
        float s[U][NT][4];
#pragma unroll
        for (int j = 0; j < D / 32; ++j)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint4 x = k[u][j];       // tokens 0 to 7 and 8 to 15 of 16 dims, then of the next 16
                uint4 a, b;
                C::keys(x.x, a.x, a.z);
                C::keys(x.y, a.y, a.w);
                C::keys(x.z, b.x, b.z);
                C::keys(x.w, b.y, b.w);
#pragma unroll
                for (int t = 0; t < NT; ++t) mma_f16(j == 0, s[u][t], a, q[t][j][0], q[t][j][1]);
#pragma unroll
                for (int t = 0; t < NT; ++t) N::mma(s[u][t], b, q[t][j][2], q[t][j][3]);
            }
        uint4 v[U][D / 32];                    // asked for before the softmax
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < D / 32; ++j) v[u][j] = ldsm_t(((src + get) ^ 32 * j) + R::kSideBytes + 16 * u * D);
        float ks[2 * U], vs[2 * U];            // of tokens g, 8 + g, ..
        floats(src + 2 * R::kSideBytes + 8 * U * g, ks);
        floats(src + 2 * R::kSideBytes + 4 * R::kTokens + 8 * U * g, vs);
        // s[u][t][0], [1]: token 16 u + g, heads 8t + 2c, + 1; [2], [3]: token 16 u + 8 + g; each to be multiplied by the token's
        // scale and the head's factor.  The weights' exponents, and the largest of them: max does not see a NaN, which then gives a
        // NaN weight
        float e[U][NT][4], w[2 * U], top = 0.f, most = 0.f;
        auto by = [&](int u, int t, int i) { return ks[2 * u + (i >> 1)] * factor[t][i & 1]; };
        auto attended = [&](int u, int i) { return on >> (16 * u + g + 4 * (i & 2)) & 1; };
#pragma unroll
        for (int i = 0; i < 2 * U; ++i) {
            w[i] = vs[i] * st.inv_ref;
            most = fmaxf(most, fabsf(w[i]));
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int u = 0; u < U; ++u) e[u][t][i] = fmaf(s[u][t][i], by(u, t, i), -st.m[t][i & 1]);
        if (on != 0xffffffffu)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (!attended(u, i)) e[u][t][i] = -CUDART_INF_F;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int u = 0; u < U; ++u) top = fmaxf(top, e[u][t][i]);
        const bool over = top > N::kSlack + N::kLift || most > 2.f;
        if (__any_sync(0xffffffffu, over)) {
            // the reference of the values' scales: the power of two below the largest, or the present one
            float largest = 0.f;
#pragma unroll
            for (int i = 0; i < 2 * U; ++i) largest = fmaxf(largest, fabsf(vs[i]));
            const uint32_t ex = min(__reduce_max_sync(0xffffffffu, __float_as_uint(largest)) >> 23, 252u);
            const float inv = fminf(st.inv_ref, __uint_as_float((254u - ex) << 23));
            const float sink = inv / st.inv_ref;
            st.inv_ref = inv;
#pragma unroll
            for (int i = 0; i < 2 * U; ++i) w[i] = vs[i] * inv;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float x[U][2], mx = -CUDART_INF_F;
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            x[u][i] = attended(u, 2 * i) ? s[u][t][2 * i + h] * by(u, t, 2 * i + h) : -CUDART_INF_F;
                            mx = fmaxf(mx, x[u][i]);
                        }
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                    mx = fmaxf(mx - N::kLift, st.m[t][h]);
                    const float alpha = ex2(st.m[t][h] - mx);
                    st.m[t][h] = mx;
                    st.l[t][h] *= alpha;
#pragma unroll
                    for (int j = 0; j < D / 16; ++j) {
                        st.acc[t][j][h] *= alpha * sink;
                        st.acc[t][j][2 + h] *= alpha * sink;
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        e[u][t][h] = x[u][0] - mx;
                        e[u][t][2 + h] = x[u][1] - mx;
                    }
                }
        }
        // P^T: tokens 2c, 2c + 1 and 2c + 8, 2c + 9 (of 16) of head 8t + g, as the sum of two fp16 numbers
        uint32_t pt[U][NT][2], rest[U][NT][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int i = 0; i < 4; ++i) e[u][t][i] = ex2(e[u][t][i]);
                st.l[t][0] += e[u][t][0] + e[u][t][2];
                st.l[t][1] += e[u][t][1] + e[u][t][3];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float x = e[u][t][2 * i] * w[2 * u + i], y = e[u][t][2 * i + 1] * w[2 * u + i];
                    const uint32_t pair = N::pack(x, y);
                    pt[u][t][i] = transpose8(pair);
                    const float2 f = N::unpack(pair);
                    rest[u][t][i] = transpose8(N::pack(x - f.x, y - f.y));
                }
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                const uint4 x = v[u][j];       // tokens 0 to 7 and 8 to 15 of 16 dims, then of the next 16
                uint4 a, b;
                C::values(x.x, a.x, a.y);
                C::values(x.y, a.z, a.w);
                C::values(x.z, b.x, b.y);
                C::values(x.w, b.z, b.w);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    N::mma(st.acc[t][2 * j], a, pt[u][t][0], pt[u][t][1]);
                    N::mma(st.acc[t][2 * j + 1], b, pt[u][t][0], pt[u][t][1]);
                    N::mma(st.acc[t][2 * j], a, rest[u][t][0], rest[u][t][1]);
                    N::mma(st.acc[t][2 * j + 1], b, rest[u][t][0], rest[u][t][1]);
                }
            }
    }
};

// ---------------------------------------------------------------------------------------------------- host

Tiling tiling_of(int32_t dim, int32_t nt) { return {16 * groups_of(dim, nt), warps_of(nt)}; }

template <typename T, typename C, int D>
cudaError_t launch(const AttnParams& p, const Layout& y, bool may_cut, cudaStream_t s) {
    return launch_attn<Worker<T, C, D, 1>, Worker<T, C, D, 2>>(p, y, may_cut, s);
}
template <typename T, typename C>
cudaError_t launch(const AttnParams& p, int32_t dim, const Layout& y, bool may_cut, cudaStream_t s) {
    return dim == 128 ? launch<T, C, 128>(p, y, may_cut, s) : launch<T, C, 64>(p, y, may_cut, s);
}
cudaError_t sms_here(int* sms) {
    using B = __nv_bfloat16;
    using H = __half;
    return device_sms<Worker<B, Int8, 64, 1>, Worker<B, Int8, 64, 2>, Worker<B, Int8, 128, 1>, Worker<B, Int8, 128, 2>,
                      Worker<B, E4m3, 64, 1>, Worker<B, E4m3, 64, 2>, Worker<B, E4m3, 128, 1>, Worker<B, E4m3, 128, 2>,
                      Worker<H, Int8, 64, 1>, Worker<H, Int8, 64, 2>, Worker<H, Int8, 128, 1>, Worker<H, Int8, 128, 2>,
                      Worker<H, E4m3, 64, 1>, Worker<H, E4m3, 64, 2>, Worker<H, E4m3, 128, 1>, Worker<H, E4m3, 128, 2>>(sms);
}

}  // namespace

extern "C" int32_t ps_quant_attn_workspace(int32_t num_kv_heads, int32_t num_q_heads, int32_t head_dim, int64_t* bytes) {
    return workspace_of(num_kv_heads, num_q_heads, head_dim, tiling_of, sms_here, bytes);
}

extern "C" int32_t ps_quant_attn(const ps_quant_attn_args* args, void* stream, char* err_buf, int32_t err_cap) {
    const Refusal refuse{"ps_quant_attn", err_buf, err_cap};
    if (!args) return refuse("null arguments");
    const ps_quant_attn_args a = *args;
    const ps_quant_cache& c = a.cache;
    if (c.codes != PS_CODE_INT8 && c.codes != PS_CODE_E4M3) return refuse("codes must be PS_CODE_INT8 or PS_CODE_E4M3");
    AttnParams p{};
    Layout y{};
    bool may_cut = false;
    auto pools = [&]() -> const char* {
        if (!c.kpool || !c.vpool || !c.k_scale || !c.v_scale) return "null pointer";
        const int64_t block = (int64_t)c.block_size * c.num_kv_heads * c.head_dim;
        if (c.num_gpu_blocks > 1 && (c.k_block_stride < block || c.v_block_stride < block || c.k_scale_stride < c.num_kv_heads ||
                                     c.v_scale_stride < c.num_kv_heads))
            return "a pool's block stride is smaller than a block, or its scales' than a block's";
        if (std::max(c.k_block_stride, c.v_block_stride) >> 36 || std::max(c.k_scale_stride, c.v_scale_stride) >> 30)
            return "blocks lie 2^36 bytes apart or more, or scales 2^30 floats";
        if (!on_bytes(c.k_scale, 0, 4) || !on_bytes(c.v_scale, 0, 4)) return "scales must be on 4-byte boundaries";
        if (!on_bytes(c.kpool, c.k_block_stride, 16) || !on_bytes(c.vpool, c.v_block_stride, 16)) return kUneven;
        return nullptr;
    };
    const int32_t rc =
        plan_call(a, {c.num_kv_heads, c.head_dim, c.block_size, c.num_gpu_blocks}, tiling_of, sms_here, pools, refuse, &p, &y, &may_cut);
    if (rc != PS_OK || a.batch == 0) return rc;
    p.kpool = c.kpool, p.vpool = c.vpool, p.k_scale = c.k_scale, p.v_scale = c.v_scale;
    p.k_step = (uint32_t)(c.k_block_stride >> 4), p.v_step = (uint32_t)(c.v_block_stride >> 4);
    p.k_scale_step = (uint32_t)(4 * c.k_scale_stride), p.v_scale_step = (uint32_t)(4 * c.v_scale_stride);
    p.row_step = (uint32_t)(c.num_kv_heads * (c.head_dim / 16));
    p.near = p.k_step == p.v_step && (double)c.num_gpu_blocks * (double)c.k_block_stride < 68719476736.0;      // 2^36
    cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e;
    if (a.dtype == PS_DTYPE_BF16)
        e = c.codes == PS_CODE_INT8 ? launch<__nv_bfloat16, Int8>(p, c.head_dim, y, may_cut, s) : launch<__nv_bfloat16, E4m3>(p, c.head_dim, y, may_cut, s);
    else
        e = c.codes == PS_CODE_INT8 ? launch<__half, Int8>(p, c.head_dim, y, may_cut, s) : launch<__half, E4m3>(p, c.head_dim, y, may_cut, s);
    if (e != cudaSuccess) return ps::launch_fail(err_buf, err_cap, "ps_quant_attn", e);
    return PS_OK;
}

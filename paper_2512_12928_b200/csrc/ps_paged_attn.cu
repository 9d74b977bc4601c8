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
// The cut of the work, the warps, the ends of segments and the join are the frame's (ps_paged_attn.cuh).
#include "ps_paged_attn.cuh"

namespace {

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
    using Stages = R;
    using Type = T;
    using Softmax = State<D, NT>;
    static constexpr int kDim = D, kColumns = NT, kWarps = 8;
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
    uint32_t masks[R::kStages - 1];            // which tokens of the tiles in the ring are attended, the oldest first
    using Keys = uint4[kSub][D / 16];

    __device__ __forceinline__ Worker(const AttnParams& pp, uint32_t smem)
        : p(pp), lane(threadIdx.x & 31), g((threadIdx.x & 31) >> 2), c(threadIdx.x & 3), unit_in_cta((threadIdx.x >> 5) % pp.units),
          sub((threadIdx.x >> 5) / pp.units), ring(smem + (threadIdx.x >> 5) * R::kWarpBytes), policy(read_once_policy()),
          masks{} {
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

    // The part whose tiles come next.
    __device__ __forceinline__ void enter(const Part& s, int kv) {
        idle = s.n == 0;
        const int64_t o = (int64_t)kv * D + 8 * (lane & 7);
        k_src = (const T*)p.kpool + o;
        v_src = (const T*)p.vpool + o;
        table = p.tables + (int64_t)s.b * p.table_stride;
        // the unit's queries, into L1: they are loaded when its tiles have come, and then nothing hides their latency
        if (lane < s.n * D / 64) {
            uint32_t unused;
            asm volatile("ld.global.ca.b32 %0, [%1];" : "=r"(unused) : "l"((const T*)p.q + s.b * p.q_stride + (int64_t)s.h0 * D + lane * 64));
        }
    }

    // Looks up the tokens of the tile that the slices' from token t0 on are, in a row that ends at `end`.
    __device__ __forceinline__ void load_ids(int32_t t0, int32_t end) {
        const int32_t t = t0 + R::kTokens * sub + lane % R::kTokens;
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
    __device__ __forceinline__ void read_keys(int stage, Keys& k) const {
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int j = 0; j < D / 16; ++j) k[u][j] = ldsm(ring + stage * R::kStageBytes + 16 * u * R::kRowBytes + k_at[j % 4] + 128 * (j / 4));
    }
    __device__ __forceinline__ void reset(Softmax& st) const { state_reset(st); }
    // One head's sums over tokens to its row of shared memory: the row's places are exclusive-ored with 8 c.
    __device__ __forceinline__ void put_sums(float* row, const Softmax& st, int t, int h) const {
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) row[(16 * j + 8 * e + g) ^ (8 * c)] = st.acc[t][j][2 * e + h];
    }
    // What the head's weights and sums refer to.
    __device__ __forceinline__ float reference(const Softmax& st, int t, int h) const { return st.m[t][h]; }
    // Attends that tile; `on`: its tokens that count.
    __device__ __forceinline__ void attend(int stage, const Keys& k, uint32_t on, State<D, NT>& st) {
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

// ---------------------------------------------------------------------------------------------------- host

Tiling tiling_of(int32_t dim, int32_t) { return {dim == 128 ? Ring<128>::kTokens : Ring<64>::kTokens, 8}; }

template <typename T, int D>
cudaError_t launch(const AttnParams& p, const Layout& y, bool may_cut, cudaStream_t s) {
    return launch_attn<Worker<T, D, 1>, Worker<T, D, 2>>(p, y, may_cut, s);
}
cudaError_t sms_here(int* sms) {
    using B = __nv_bfloat16;
    using H = __half;
    return device_sms<Worker<B, 64, 1>, Worker<B, 64, 2>, Worker<B, 128, 1>, Worker<B, 128, 2>, Worker<H, 64, 1>, Worker<H, 64, 2>,
                      Worker<H, 128, 1>, Worker<H, 128, 2>>(sms);
}

}  // namespace

extern "C" int32_t ps_paged_attn_workspace(int32_t num_kv_heads, int32_t num_q_heads, int32_t head_dim, int64_t* bytes) {
    return workspace_of(num_kv_heads, num_q_heads, head_dim, tiling_of, sms_here, bytes);
}

extern "C" int32_t ps_paged_attn(const ps_paged_attn_args* args, void* stream, char* err_buf, int32_t err_cap) {
    const Refusal refuse{"ps_paged_attn", err_buf, err_cap};
    if (!args) return refuse("null arguments");
    const ps_paged_attn_args a = *args;
    AttnParams p{};
    Layout y{};
    bool may_cut = false;
    auto pools = [&]() -> const char* {
        if (!a.kpool || !a.vpool) return "null pointer";
        const int64_t block_elems = (int64_t)a.block_size * a.num_kv_heads * a.head_dim;
        if (a.num_gpu_blocks > 1 && (a.k_block_stride < block_elems || a.v_block_stride < block_elems))
            return "a pool's block stride is smaller than a block";
        if (!on_bytes(a.kpool, 2 * a.k_block_stride, 16) || !on_bytes(a.vpool, 2 * a.v_block_stride, 16)) return kUneven;
        return nullptr;
    };
    const int32_t rc = plan_call(a, {a.num_kv_heads, a.head_dim, a.block_size, a.num_gpu_blocks}, tiling_of, sms_here, pools, refuse, &p, &y, &may_cut);
    if (rc != PS_OK || a.batch == 0) return rc;
    p.kpool = a.kpool, p.vpool = a.vpool;
    p.k_block_stride = a.k_block_stride, p.v_block_stride = a.v_block_stride;
    cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e;
    if (a.dtype == PS_DTYPE_BF16)
        e = a.head_dim == 128 ? launch<__nv_bfloat16, 128>(p, y, may_cut, s) : launch<__nv_bfloat16, 64>(p, y, may_cut, s);
    else
        e = a.head_dim == 128 ? launch<__half, 128>(p, y, may_cut, s) : launch<__half, 64>(p, y, may_cut, s);
    if (e != cudaSuccess) return ps::launch_fail(err_buf, err_cap, "ps_paged_attn", e);
    return PS_OK;
}

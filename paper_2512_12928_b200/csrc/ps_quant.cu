// ps_quant_append and ps_quant_read: a paged cache of 8-bit codes with one scale for each block and KV head, written from
// 16-bit keys and values and read back into 16 bits.
//
//   need = max |x| / Q over the call's tokens of a block and head,   scale' = max(scale, need, 2^-100),
//   code = round(x / scale'),   and codes that are there: round(code scale / scale') where scale' > scale
//
// Bound: memory; a value written is 2 bytes read and 1 written, a value read back 1 and 2.  A scale needs all of its
// block's new values before the first code can be rounded, so a warp takes one block's tokens of one head ("unit") and holds
// them in registers between the two: 16 tokens of 128 dims are 4 vectors of 32 bytes a lane.  Larger blocks have several warps.
// Measured (8 KV heads of 128, bf16): 9350 tokens of prompt chunks appended in 13.7 us, whose bytes would take 8.9; a decode
// batch's 200 of 4 heads 2.3, one 2.0, all where no scale rises (where nearly all do 3, 1.2 and 0.7 us more).  71000 tokens read
// back in 68.3 us, or 6.4 TB/s, which is what a copy reaches; 300 in 2.3.
// What the append spends above its bytes are two rounds and a half of CTAs, in each of which slots, then rows, then the maximum
// over a warp wait for one another, and a unit's own instructions.  (With the values in shared memory instead of registers, by
// cp.async, and more warps on an SM: 18.6 us where registers took 15.5.)
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <math_constants.h>

#include <algorithm>

#include "ps_internal.h"
#include "ps_kvswap.h"

namespace {

constexpr int kThreads = 256;
constexpr int kMaxDim = 512, kMaxHeads = 1024;
constexpr int kStatusBadSlot = 1;
constexpr float kLeastScale = 7.888609052210118e-31f;   // 2^-100: its reciprocal is finite

template <typename T> struct Num;
template <> struct Num<__nv_bfloat16> {
    static constexpr uint32_t kInf = 0x7f80;
    static __device__ __forceinline__ float2 unpack(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
};
template <> struct Num<__half> {
    static constexpr uint32_t kInf = 0x7c00;
    static __device__ __forceinline__ float2 unpack(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
};

struct Int8 {
    static constexpr float kTop = 127.f;
    // Codes of four values times r.  The exact product is rounded to a whole number by the addition: 1.5 2^23 + n has n as its
    // low bits.
    static __device__ __forceinline__ uint32_t pack(const float4& v, float r) {
        auto one = [&](float x) { return __float_as_uint(fmaf(x, r, 12582912.f)); };
        return __byte_perm(__byte_perm(one(v.x), one(v.y), 0x0040), __byte_perm(one(v.z), one(v.w), 0x0040), 0x5410);
    }
    // Four codes.  A byte with its top bit turned is n + 128; as the low bits of 2^23 that is 2^23 + 128 + n, exactly.
    static __device__ __forceinline__ float4 unpack(uint32_t v) {
        const uint32_t x = v ^ 0x80808080u;
        auto one = [&](uint32_t select) { return __uint_as_float(__byte_perm(x, 0x4b000000u, select)) - 8388736.f; };
        return make_float4(one(0x7540), one(0x7541), one(0x7542), one(0x7543));
    }
};
struct E4m3 {
    static constexpr float kTop = 448.f;
    static __device__ __forceinline__ uint32_t pack(const float4& v, float r) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(__fmul_rn(v.x, r), __fmul_rn(v.y, r)), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(__fmul_rn(v.z, r), __fmul_rn(v.w, r)), __NV_SATFINITE, __NV_E4M3);
        return __byte_perm(lo, hi, 0x5410);
    }
    static __device__ __forceinline__ float4 unpack(uint32_t v) {
        const float2 a = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)v, __NV_E4M3)));
        const float2 b = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v >> 16), __NV_E4M3)));
        return make_float4(a.x, a.y, b.x, b.y);
    }
};

// W values that are loaded and stored at once.
template <int Bytes> struct Bits;
template <> struct Bits<1> { using type = uint8_t; };
template <> struct Bits<2> { using type = uint16_t; };
template <> struct Bits<4> { using type = uint32_t; };
template <> struct Bits<8> { using type = uint2; };
template <> struct Bits<16> { using type = uint4; };
template <> struct Bits<32> { using type = uint4; };     // in two halves, or by one access of 32 bytes
template <int Bytes>
struct alignas(Bytes < 4 ? 4 : Bytes > 16 ? 16 : Bytes) Vec {
    uint32_t w[(Bytes + 3) / 4];             // a value of one or two bytes is the low ones of a word
    __device__ __forceinline__ void load(const void* p) {
        using B = typename Bits<Bytes>::type;
        if constexpr (Bytes == 32)
            asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                         : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p) : "memory");
        else if constexpr (Bytes < 4) w[0] = *static_cast<const B*>(p);
        else *reinterpret_cast<B*>(w) = *static_cast<const B*>(p);
    }
    __device__ __forceinline__ void store(void* p) const {
        using B = typename Bits<Bytes>::type;
        if constexpr (Bytes == 32)
            asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
                         "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
        else if constexpr (Bytes < 4) *static_cast<B*>(p) = (B)w[0];
        else *static_cast<B*>(p) = *reinterpret_cast<const B*>(w);
    }
};

// slot / size: magic is 2^64 / size rounded up, which is exact where slot * size < 2^64
__device__ __forceinline__ int64_t block_of(int64_t slot, uint64_t magic) {
    return magic == 0 ? slot : (int64_t)__umul64hi((uint64_t)slot, magic);     // 0: blocks of one token
}

struct Side {                     // keys or values
    const void* rows;             // 16-bit rows: read by the append, written by the read-back
    unsigned char* pool;
    float* scale;
    int64_t row_stride, block_stride, scale_stride;
};
struct QuantParams {
    Side side[2];
    const int64_t* slots;
    int32_t* status;
    int64_t num_slots;
    uint64_t block_magic;
    int32_t tokens, hkv, dim, block_size, sides, tok_per_cta;
    int32_t team;                 // warps of a unit
    int32_t row_vecs, row_magic;  // vectors of a head's row; 2^16 / row_vecs rounded up
    int32_t row_step, piece_step, team_row_step, team_piece_step;      // 32 vectors on, and 32 team
};

// ------------------------------------------------------------------------------------------------ append

// Vectors of w values of a lane that stay in registers between maximum and rounding.
constexpr __host__ __device__ int held_of(int w) { return w == 16 ? 4 : 8; }

// A segment is a run of tokens that go to one block.  A warp has one head of keys or values, and the segments that begin
// among the CTA's tokens; it finds them for itself, without barriers.  kTeam: blocks are larger than what a warp holds, and
// several warps have a head together; the CTA looks up 256 tokens at once, so that few CTAs find nothing.  kEven: a row's
// vectors divide a team's lanes, so that a lane has the same piece of every row it has.
template <typename T, typename C, int W, bool kEven, bool kTeam, int kCtas>
__global__ void __launch_bounds__(kThreads, kCtas)
quant_append_kernel(const __grid_constant__ QuantParams p) {
    constexpr int kHold = held_of(W);
    constexpr int kWindow = kTeam ? kThreads : 32;           // tokens that are looked up at once, from the one before on
    __shared__ int32_t blocks[kWindow], places[kWindow];     // these only with teams
    __shared__ uint32_t changes[kThreads / 32], zeros[kThreads / 32], tops[2][kThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, team = kTeam ? p.team : 1;
    const int team_in_cta = warp / team, lane_in_team = threadIdx.x - 32 * team * team_in_cta;
    const int unit = (kThreads / 32) / team * blockIdx.y + team_in_cta;
    if (!kTeam && unit >= p.sides * p.hkv) return;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int head = unit < p.hkv ? unit : unit - p.hkv;
    const Side& side = p.side[unit < p.hkv ? 0 : 1];
    // The vectors of a segment, rows first: this lane has every 32nd, or with the team `together` every one that is 32 team on.
    bool together = false;
    int row0, piece0, row_step, piece_step;
    auto deal = [&] {
        const int me = kTeam && together ? lane_in_team : lane;
        row0 = me * p.row_magic >> 16, piece0 = me - row0 * p.row_vecs;
        row_step = kTeam && together ? p.team_row_step : p.row_step, piece_step = kTeam && together ? p.team_piece_step : p.piece_step;
    };
    deal();
    auto next = [&](int& row, int& piece) {
        row += row_step;
        if (kEven) return;
        piece += piece_step;
        if (piece >= p.row_vecs) {
            piece -= p.row_vecs;
            ++row;
        }
    };
    auto meet_team = [&] { asm volatile("bar.sync %0, %1;" ::"r"(1 + team_in_cta), "r"(32 * team) : "memory"); };
    int turn = 0;
    const uint32_t place_bytes = p.hkv * p.dim;
    const int32_t t0 = blockIdx.x * p.tok_per_cta;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    // What begins among the CTA's tokens mostly ends within the window, too
    const int32_t t = t0 - 1 + (kTeam ? threadIdx.x : lane);
    int64_t slot = t >= 0 && t < p.tokens ? p.slots[t] : -1;
    if (slot >= p.num_slots) {
        if (p.status) *(volatile int32_t*)p.status = kStatusBadSlot;
        slot = -1;
    }
    const int32_t block = slot < 0 ? -1 : (int32_t)block_of(slot, p.block_magic);
    const int32_t my_place = (int32_t)slot - block * p.block_size;          // modulo 2^32: a place is less

    // Tokens [first, first + len) of the window, or more where the segment goes on behind it.
    auto segment = [&](int first, int len, int32_t blk, bool begun) {
        const bool ends = first + len < kWindow;
        const int64_t block_begin = (int64_t)blk * p.block_size;
        while (!ends) {
            const int32_t u = t0 - 1 + first + len + lane;
            const int64_t s = u < p.tokens ? p.slots[u] : -1;
            const uint32_t out = __ballot_sync(0xffffffffu, s < block_begin || s - block_begin >= p.block_size);
            const int more = out ? __ffs(out) - 1 : 32;
            begun |= __any_sync(0xffffffffu, lane < more && s == block_begin);
            len += more;
            if (more < 32) break;
        }
        const int32_t token0 = t0 - 1 + first;
        const T* src = (const T*)side.rows + token0 * side.row_stride + (int64_t)head * p.dim;
        unsigned char* pool = side.pool + blk * side.block_stride + (int64_t)head * p.dim;
        float* scale_at = side.scale + blk * side.scale_stride + head;
        auto from = [&](int row, int piece) { return src + (int64_t)row * (int32_t)side.row_stride + piece * W; };
        const float old = begun ? 0.f : *scale_at;
        Vec<2 * W> held[kHold];
        uint32_t most = 0;                   // of both halves of a word
        auto meet = [&](const Vec<2 * W>& x) {
#pragma unroll
            for (int i = 0; i < W / 2; i += 2) most = __vimax3_u16x2(most, x.w[i] & 0x7fff7fffu, x.w[i + 1] & 0x7fff7fffu);
            if (W == 1) most = max(most, x.w[0] & 0x7fffu);
        };
        int row = row0, piece = piece0;
#pragma unroll
        for (int i = 0; i < kHold; ++i) {
            if (row < len) held[i].load(from(row, piece));
            next(row, piece);
        }
        int row2 = row0, piece2 = piece0;
#pragma unroll
        for (int i = 0; i < kHold; ++i) {
            if (row2 < len) meet(held[i]);
            next(row2, piece2);
        }
        while (row < len) {
            Vec<2 * W> x;
            x.load(from(row, piece));
            meet(x);
            next(row, piece);
        }
        most = __reduce_max_sync(0xffffffffu, max(most & 0xffff, most >> 16));
        if (kTeam && together) {             // all warps have the old scale by then, too
            if (lane == 0) tops[turn][warp] = most;
            meet_team();
            most = __reduce_max_sync(0xffffffffu, tops[turn][team_in_cta * team + lane % team]);
            turn ^= 1;
        }
        const float need = Num<T>::unpack(most).x * (1.f / C::kTop);
        const float now = most >= Num<T>::kInf || old != old ? CUDART_NAN_F : fmaxf(fmaxf(old, need), kLeastScale);
        const float r = 1.f / now;
        if (!begun && now > old) {           // the codes that are there, all places of the block
            const float f = __fmul_rn(old, r);
            int q = row0, c = piece0;
            while (q < p.block_size) {
                // on their way at once: as many as the registers of two CTAs an SM hold (64 blocks of 64 / 256 tokens that
                // all grow: 8.6 / 26 us with four, 13 / 56 with one)
                constexpr int kMany = kCtas == 2 ? 4 : 1;
                Vec<W> x[kMany];
                unsigned char* at[kMany];
                bool there[kMany];
#pragma unroll
                for (int k = 0; k < kMany; ++k) {
                    at[k] = pool + (uint32_t)q * (uint64_t)place_bytes + c * W;
                    there[k] = q < p.block_size;
                    if (there[k]) x[k].load(at[k]);
                    next(q, c);
                }
#pragma unroll
                for (int k = 0; k < kMany; ++k) {
                    if (!there[k]) continue;
#pragma unroll
                    for (int i = 0; i < (W + 3) / 4; ++i) x[k].w[i] = C::pack(C::unpack(x[k].w[i]), f);
                    x[k].store(at[k]);
                }
            }
            __syncwarp();                    // the new tokens' codes come on top
        }
        if (kTeam && together && !begun) meet_team();
        auto put = [&](const Vec<2 * W>& x, uint32_t place, int piece) {
            Vec<W> y;
#pragma unroll
            for (int i = 0; i < (W + 3) / 4; ++i) {
                const float2 lo = Num<T>::unpack(x.w[2 * i]), hi = W > 1 ? Num<T>::unpack(x.w[2 * i + (W > 1)]) : lo;
                y.w[i] = C::pack(make_float4(lo.x, lo.y, hi.x, hi.y), r);
            }
            y.store(pool + place * (uint64_t)place_bytes + piece * W);
        };
        auto place_of = [&](int row) { return (uint32_t)(p.slots[token0 + row] - block_begin); };
        row = row0, piece = piece0;
#pragma unroll
        for (int i = 0; i < kHold; ++i) {
            uint32_t place = kTeam ? 0 : __shfl_sync(0xffffffffu, my_place, first + row);
            if (row < len) {
                if (kTeam && first + row < kWindow) place = places[first + row];
                else if (!ends && first + row >= kWindow) place = place_of(row);
                put(held[i], place, piece);
            }
            next(row, piece);
        }
        while (row < len) {
            Vec<2 * W> x;
            x.load(from(row, piece));
            put(x, place_of(row), piece);
            next(row, piece);
        }
        if (kTeam && together ? lane_in_team == 0 : lane == 0) *scale_at = now;
    };

    if constexpr (kTeam) {
        blocks[threadIdx.x] = block;
        places[threadIdx.x] = my_place;
        __syncthreads();
        const uint32_t change = __ballot_sync(0xffffffffu, threadIdx.x > 0 && block != blocks[max((int)threadIdx.x - 1, 0)]);
        const uint32_t zero = __ballot_sync(0xffffffffu, slot >= 0 && my_place == 0);
        if (lane == 0) changes[warp] = change, zeros[warp] = zero;
        __syncthreads();
        if (unit >= p.sides * p.hkv) return;
        // the words of a mask from bit `from` on, one a lane
        auto word_from = [&](const uint32_t* mask, int from) {
            const int n = from - 32 * lane;
            return lane >= kThreads / 32 || n >= 32 ? 0u : n <= 0 ? mask[lane] : mask[lane] & (0xffffffffu << n);
        };
        auto first_from = [&](const uint32_t* mask, int from) {
            const uint32_t w = word_from(mask, from), any = __ballot_sync(0xffffffffu, w != 0);
            const int at = any ? __ffs(any) - 1 : 0, in_word = __ffs(__shfl_sync(0xffffffffu, w, at)) - 1;
            return any ? 32 * at + in_word : kWindow;
        };
        // What a warp holds goes to one after the other of the team's warps, what is longer to all of them together.
        int whose = 0;
        for (int first = first_from(changes, 1); first <= p.tok_per_cta;) {
            const int end = first_from(changes, first + 1);
            if (blocks[first] >= 0) {
                together = end == kWindow || (end - first) * p.row_vecs > 32 * kHold;
                deal();
                if (together || whose++ % team == warp % team)
                    segment(first, end - first, blocks[first], first_from(zeros, first) < end);
            }
            first = end;
        }
    } else {
        const int32_t before = __shfl_up_sync(0xffffffffu, block, 1);
        uint32_t starts = __ballot_sync(0xffffffffu, lane > 0 && lane <= p.tok_per_cta && block >= 0 && block != before);
        for (; starts; starts &= starts - 1) {
            const int first = __ffs(starts) - 1;
            const int32_t blk = __shfl_sync(0xffffffffu, block, first);
            const uint32_t other = __ballot_sync(0xffffffffu, block != blk) & (0xffffffffu << first);
            const int len = (other ? __ffs(other) - 1 : 32) - first;
            segment(first, len, blk, __any_sync(0xffffffffu, lane >= first && lane < first + len && my_place == 0));
        }
    }
}

// -------------------------------------------------------------------------------------------------- read

// Where a token lies: found once for a CTA's tokens and kept in shared memory.
struct Place {
    int64_t codes, scales;        // offsets in the pool and its scales; codes < 0: nothing of it is written
};

// A thread has one vector of a token, the same of every `at_once`-th token.
constexpr int kAhead = 4;        // tokens that it has on their way at once (17.1 us where 2 took 20.0 and 8 22.6)
constexpr int kMaxTokens = 256;   // of a CTA
template <typename T, typename C, int W>
__global__ void __launch_bounds__(kThreads, 4)
quant_read_kernel(const __grid_constant__ QuantParams p) {
    __shared__ Place place[2][kMaxTokens];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int side_vecs = p.hkv * p.dim / W, per = p.sides * side_vecs;     // vectors of a token
    const int lanes = min(per, kThreads), at_once = kThreads / lanes;
    const int k0 = threadIdx.x / lanes, row_vecs = p.dim / W;
    const int32_t t0 = blockIdx.x * p.tok_per_cta;
    const int n = min(p.tok_per_cta, p.tokens - t0);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (threadIdx.x < n) {
        const int64_t slot = p.slots[t0 + threadIdx.x];
        const bool live = slot >= 0 && slot < p.num_slots;
        if (slot >= p.num_slots && p.status) *(volatile int32_t*)p.status = kStatusBadSlot;
        const int64_t blk = block_of(live ? slot : 0, p.block_magic), in_block = (slot - blk * p.block_size) * ((int64_t)p.hkv * p.dim);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const Side& s = p.side[i < p.sides ? i : 0];
            place[i][threadIdx.x] = {live ? blk * s.block_stride + in_block : -1, blk * s.scale_stride};
        }
    }
    __syncthreads();
    if (k0 >= at_once) return;
    for (int j = threadIdx.x - k0 * lanes; j < per; j += lanes) {
        const int which = j < side_vecs ? 0 : 1, vec = j - which * side_vecs;
        const Side& side = p.side[which];
        const unsigned char* pool = side.pool + vec * W;
        const float* scales = side.scale + vec / row_vecs;
        T* rows = (T*)side.rows + t0 * side.row_stride + vec * W;
        for (int k = k0; k < n; k += kAhead * at_once) {
            bool live[kAhead];
            Vec<W> x[kAhead];
            float scale[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const Place at = place[which][min(k + i * at_once, n - 1)];
                live[i] = k + i * at_once < n && at.codes >= 0;
                if (!live[i]) continue;
                x[i].load(pool + at.codes);
                scale[i] = scales[at.scales];
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (!live[i]) continue;
                Vec<2 * W> y;
#pragma unroll
                for (int h = 0; h < (W + 3) / 4; ++h) {
                    const float4 v = C::unpack(x[i].w[h]);
                    y.w[2 * h] = Num<T>::pack(v.x * scale[i], v.y * scale[i]);
                    if (W > 2) y.w[2 * h + (W > 2)] = Num<T>::pack(v.z * scale[i], v.w * scale[i]);
                }
                y.store(rows + (k + i * at_once) * side.row_stride);
            }
        }
    }
}

// -------------------------------------------------------------------------------------------------- host

struct Given {                    // one side as the caller gave it
    const void* rows;
    void* pool;
    float* scale;
    int64_t row_stride, block_stride, scale_stride;
};

// Fills in p; *p.sides is 0 where there is nothing to do.  Returns the text of what is wrong, or null.
const char* plan(const ps_quant_cache& c, const Given (&given)[2], const int64_t* slots, int32_t* status, int32_t tokens, int32_t dtype,
                 bool rows_written, QuantParams* params) {
    if (tokens < 0 || c.block_size <= 0 || c.num_gpu_blocks <= 0) return "negative count or non-positive size";
    if (tokens > INT32_MAX - 1024) return "too many tokens";   // so that what a warp looks ahead cannot wrap
    if (c.block_size > INT32_MAX - 4096) return "block_size must be below 2^31 - 4096";    // nor the places that a lane takes at once
    if (c.num_kv_heads <= 0 || c.num_kv_heads > kMaxHeads || c.head_dim <= 0 || c.head_dim > kMaxDim)
        return "num_kv_heads must be from 1 to 1024, head_dim from 1 to 512";
    if (dtype != PS_DTYPE_BF16 && dtype != PS_DTYPE_FP16) return "dtype must be PS_DTYPE_BF16 or PS_DTYPE_FP16";
    if (c.codes != PS_CODE_INT8 && c.codes != PS_CODE_E4M3) return "codes must be PS_CODE_INT8 or PS_CODE_E4M3";
    if (tokens == 0) return nullptr;         // tensors without elements have no address
    const int64_t width = (int64_t)c.num_kv_heads * c.head_dim, block = width * c.block_size;
    QuantParams& p = *params;
    ps::RowSet sets[2][3];
    for (const Given& g : given) {
        if (!g.rows && !g.pool && !g.scale) continue;
        if (!g.rows || !g.pool || !g.scale) return "keys and values need rows, codes and scales, or none of them";
        if (c.num_gpu_blocks > 1 && (g.block_stride < block || g.scale_stride < c.num_kv_heads))
            return "a pool's block stride is smaller than a block, or its scales' than a block's";
        if (reinterpret_cast<uintptr_t>(g.scale) % 4 || reinterpret_cast<uintptr_t>(g.rows) % 2) return "scales or rows are not aligned to their elements";
        if (tokens > 1 && (g.row_stride > INT32_MAX || g.row_stride < INT32_MIN)) return "rows lie 2^31 elements apart or more";
        if (rows_written && tokens > 1 && g.row_stride < width && -g.row_stride < width) return "rows of k_out or v_out overlap";
        sets[p.sides][0] = {g.rows, g.row_stride, width, 2};
        sets[p.sides][1] = {g.pool, g.block_stride, block, 1};
        sets[p.sides][2] = {g.scale, g.scale_stride, c.num_kv_heads, 4};
        p.side[p.sides++] = {g.rows, (unsigned char*)g.pool, g.scale, g.row_stride, g.block_stride, g.scale_stride};
    }
    if (p.sides == 0) return "neither keys nor values are given";
    if (!slots) return "null pointer";
    // slots are divided by block_size as block_of says
    if ((double)c.num_gpu_blocks * c.block_size * c.block_size >= 18e18) return "num_gpu_blocks * block_size^2 must be below 1.8e19";
    // whatever is written is apart from everything else
    auto count = [&](int kind) -> int64_t { return kind == 0 ? tokens : c.num_gpu_blocks; };
    for (int i = 0; i < 3 * p.sides; ++i)
        for (int j = 0; j < i; ++j) {
            const bool written = rows_written ? i % 3 == 0 || j % 3 == 0 : i % 3 != 0 || j % 3 != 0;
            if (written && ps::rows_meet(sets[i / 3][i % 3], count(i % 3), sets[j / 3][j % 3], count(j % 3)))
                return "what is written overlaps another argument";
        }
    p.slots = slots, p.status = status;
    p.num_slots = (int64_t)c.num_gpu_blocks * c.block_size;
    p.block_magic = c.block_size > 1 ? ~0ull / (uint64_t)c.block_size + 1 : 0;
    p.tokens = tokens, p.hkv = c.num_kv_heads, p.dim = c.head_dim, p.block_size = c.block_size;
    return nullptr;
}

// Whether w values can be moved at once everywhere.
bool fits(const QuantParams& p, int w) {
    bool ok = p.dim % w == 0;
    for (int i = 0; i < p.sides; ++i) {
        const Side& s = p.side[i];
        ok = ok && reinterpret_cast<uintptr_t>(s.rows) % (2 * w) == 0 && s.row_stride % w == 0 &&
             reinterpret_cast<uintptr_t>(s.pool) % w == 0 && s.block_stride % w == 0;
    }
    return ok;
}

template <typename T, typename C>
cudaError_t launch_append(QuantParams p, cudaStream_t s) {
    // Where a block and the call have more tokens than a warp holds in registers, it has a team of up to 8 warps (9350 tokens of 8
    // heads of 128 in blocks of 64 / 256 / 1024: 17 / 21 / 43 us instead of 21 / 71 / 245, 256 in one block 5.9 instead of 31; a
    // batch's 64 single tokens in blocks of 64 4.4 instead of 2.4, which the 256 tokens that a CTA looks up cost).
    const int w = fits(p, 16) ? 16 : fits(p, 8) ? 8 : 1, units = p.sides * p.hkv;
    p.row_vecs = p.dim / w;
    p.team = 1;
    while (p.team < 8 && 32 * held_of(w) * p.team < (int64_t)std::min(p.block_size, p.tokens) * p.row_vecs) p.team *= 2;
    const int at_once = kThreads / 32 / p.team;              // units of a CTA
    const unsigned groups = (unsigned)((units + at_once - 1) / at_once);
    // Few tokens: one a CTA and warp, so that they spread over the chip.  Many: 16, of which a block of 16 tokens begins
    // one, with teams 128, while that leaves every SM 16 warps (9350 tokens of 8 heads of 128: 1 / 4 / 8 / 16 tokens a CTA
    // 51 / 22 / 17 / 15.5 us when this was chosen, 200 of 4 heads 2.8 / 5.6 / 9.5 / 17).  A CTA of many has 80 registers a
    // thread, so that three fit an SM, instead of two of up to 127 (15.5 instead of 17.0 us); what spills for it costs a few
    // tokens 0.1 to 0.3 us.
    p.tok_per_cta = p.team;
    while (2 * p.tok_per_cta <= std::min(p.block_size, p.team > 1 ? 128 : 16) &&
           (int64_t)p.tokens / (2 * p.tok_per_cta) * units * p.team >= 148 * 16)
        p.tok_per_cta *= 2;
    const dim3 grid((unsigned)((p.tokens + p.tok_per_cta - 1) / p.tok_per_cta), groups);
    p.row_magic = (65536 + p.row_vecs - 1) / p.row_vecs;     // exact for a team's 256 lanes and up to 512 vectors
    p.row_step = 32 / p.row_vecs, p.piece_step = 32 % p.row_vecs;
    p.team_row_step = 32 * p.team / p.row_vecs, p.team_piece_step = 32 * p.team % p.row_vecs;
    const bool even = p.piece_step == 0, few = p.tok_per_cta == p.team;
    auto launch = [&](auto kernel) { return ps::launch_dependent(kernel, grid, dim3(kThreads), 0, s, p); };
    if (p.team > 1) {
        if (w == 16 && even) return few ? launch(quant_append_kernel<T, C, 16, true, true, 2>) : launch(quant_append_kernel<T, C, 16, true, true, 3>);
        if (w == 16) return few ? launch(quant_append_kernel<T, C, 16, false, true, 2>) : launch(quant_append_kernel<T, C, 16, false, true, 3>);
        if (w == 8) return launch(quant_append_kernel<T, C, 8, false, true, 2>);
        return launch(quant_append_kernel<T, C, 1, false, true, 2>);
    }
    if (w == 16 && even) return few ? launch(quant_append_kernel<T, C, 16, true, false, 2>) : launch(quant_append_kernel<T, C, 16, true, false, 3>);
    if (w == 16) return few ? launch(quant_append_kernel<T, C, 16, false, false, 2>) : launch(quant_append_kernel<T, C, 16, false, false, 3>);
    if (w == 8) return launch(quant_append_kernel<T, C, 8, false, false, 2>);
    return launch(quant_append_kernel<T, C, 1, false, false, 2>);
}
template <typename T, typename C>
cudaError_t launch_read(QuantParams p, cudaStream_t s) {
    const int w = fits(p, 16) ? 16 : fits(p, 8) ? 8 : 1;
    const int at_once = kThreads / std::min(kThreads, p.sides * p.hkv * p.dim / w);
    // Eight tokens a CTA, fewer while that leaves SMs without two CTAs.  (71000 tokens of 8 heads of 128: 1 / 2 / 4 / 8 / 16 / 32
    // tokens a CTA 140 / 99 / 72 / 68.7 / 69.7 / 71.8 us, 3264 of 4 heads 6.0 / 3.9 / 3.2 / 3.3 / 4.3 / 4.2.)
    p.tok_per_cta = std::min(at_once, kMaxTokens);
    while (2 * p.tok_per_cta <= 8 && p.tokens / (2 * p.tok_per_cta) >= 148 * 2) p.tok_per_cta *= 2;
    const dim3 grid((unsigned)((p.tokens + p.tok_per_cta - 1) / p.tok_per_cta));
    return w == 16  ? ps::launch_dependent(quant_read_kernel<T, C, 16>, grid, dim3(kThreads), 0, s, p)
           : w == 8 ? ps::launch_dependent(quant_read_kernel<T, C, 8>, grid, dim3(kThreads), 0, s, p)
                    : ps::launch_dependent(quant_read_kernel<T, C, 1>, grid, dim3(kThreads), 0, s, p);
}

int32_t refuse(const char* name, const char* text, char* buf, int32_t cap) {
    if (buf && cap > 0) snprintf(buf, (size_t)cap, "%s: %s", name, text);
    return PS_ERR_INVALID;
}

}  // namespace

extern "C" int32_t ps_quant_append(const ps_quant_append_args* args, void* stream, char* err_buf, int32_t err_cap) {
    if (err_buf && err_cap > 0) err_buf[0] = 0;
    if (!args) return refuse("ps_quant_append", "null arguments", err_buf, err_cap);
    const ps_quant_append_args a = *args;
    const ps_quant_cache& c = a.cache;
    const Given given[2] = {{a.k, c.kpool, c.k_scale, a.k_stride, c.k_block_stride, c.k_scale_stride},
                            {a.v, c.vpool, c.v_scale, a.v_stride, c.v_block_stride, c.v_scale_stride}};
    QuantParams p{};
    if (const char* m = plan(c, given, a.slots, a.status_word, a.tokens, a.dtype, false, &p)) return refuse("ps_quant_append", m, err_buf, err_cap);
    if (a.tokens == 0) return PS_OK;
    cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e;
    if (a.dtype == PS_DTYPE_BF16) e = c.codes == PS_CODE_INT8 ? launch_append<__nv_bfloat16, Int8>(p, s) : launch_append<__nv_bfloat16, E4m3>(p, s);
    else e = c.codes == PS_CODE_INT8 ? launch_append<__half, Int8>(p, s) : launch_append<__half, E4m3>(p, s);
    if (e != cudaSuccess) return ps::launch_fail(err_buf, err_cap, "ps_quant_append", e);
    return PS_OK;
}

extern "C" int32_t ps_quant_read(const ps_quant_read_args* args, void* stream, char* err_buf, int32_t err_cap) {
    if (err_buf && err_cap > 0) err_buf[0] = 0;
    if (!args) return refuse("ps_quant_read", "null arguments", err_buf, err_cap);
    const ps_quant_read_args a = *args;
    ps_quant_cache c = a.cache;
    if (!a.k_out) c.kpool = nullptr, c.k_scale = nullptr;
    if (!a.v_out) c.vpool = nullptr, c.v_scale = nullptr;
    const Given given[2] = {{a.k_out, c.kpool, c.k_scale, a.k_out_stride, c.k_block_stride, c.k_scale_stride},
                            {a.v_out, c.vpool, c.v_scale, a.v_out_stride, c.v_block_stride, c.v_scale_stride}};
    QuantParams p{};
    if (const char* m = plan(c, given, a.slots, a.status_word, a.tokens, a.dtype, true, &p)) return refuse("ps_quant_read", m, err_buf, err_cap);
    if (a.tokens == 0) return PS_OK;
    cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e;
    if (a.dtype == PS_DTYPE_BF16) e = c.codes == PS_CODE_INT8 ? launch_read<__nv_bfloat16, Int8>(p, s) : launch_read<__nv_bfloat16, E4m3>(p, s);
    else e = c.codes == PS_CODE_INT8 ? launch_read<__half, Int8>(p, s) : launch_read<__half, E4m3>(p, s);
    if (e != cudaSuccess) return ps::launch_fail(err_buf, err_cap, "ps_quant_read", e);
    return PS_OK;
}

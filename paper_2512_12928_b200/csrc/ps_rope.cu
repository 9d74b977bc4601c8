// ps_rope_append: rotary positions with several axes on queries and keys, and the append of keys and values to the
// paged pools.
//
//   angle_i = positions[axis_i][t] * inv_freq_i,   i < R / 2
//   (x1, x2) -> (x1 cos - x2 sin, x2 cos + x1 sin)      PS_ROPE_INVERSE turns by -angle: the transpose, the gradient
//
// on the pairs (x_i, x_{i + R/2}), or (x_{2i}, x_{2i+1}) with PS_ROPE_NEIGHBOURS; dims from R on pass unchanged.
//
// Bound: memory (every element is read once and written once, 3 flops for 4 bytes).  So the rotation shares its pass
// with the append: the rotated key goes from registers into its slot of the pool instead of to memory and back.
//
// Angles: a position of 10^6 times a frequency of 1 in 32 bits is off by up to 0.03 radians, so the product and its
// reduction to a fraction of a turn are done in 64 bits, once per token and frequency, and sine and cosine (of the
// fraction, 32 bits) are kept in shared memory for all heads of the token.
//
// Inputs are rotated in 32 bits and rounded once, at the store.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ps_internal.h"
#include "ps_kvswap.h"

namespace {

constexpr int kThreads = 256;
constexpr int kMaxHeadDim = 512;
constexpr int kTokensPerCta = 8;      // most tokens of a CTA
constexpr int kStatusBadSlot = 1;

struct FreqAxes {
    uint8_t v[kMaxHeadDim / 2];
};

struct RopeParams {
    const void *q, *k, *v;
    void *q_out, *k_out, *kpool, *vpool;
    const int64_t* slots;
    const int32_t* positions;
    const float* inv_freq;
    int32_t* status;
    int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride, axis_stride, k_block_stride, v_block_stride;
    int64_t num_slots;
    int32_t tokens, hq, hkv, dim, rot, block_size, tok_per_cta;
    float sign;
};

struct TokenPlace {   // of one token of the CTA
    int64_t k_off, v_off;   // element offset of its row in the pools; -1: not appended
    int32_t live;           // 0: padding, nothing of it is written
    int32_t pad;
};

template <typename T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f(float x) { return __float2half_rn(x); }

// W elements that are loaded and stored at once: 16, 8 or 4 bytes.
template <typename T, int W>
struct alignas(2 * W) Vec {
    T e[W];
};
template <int W> struct Bits;
template <> struct Bits<8> { using type = uint4; };
template <> struct Bits<4> { using type = uint2; };
template <> struct Bits<2> { using type = uint32_t; };
template <int W, typename T>
__device__ __forceinline__ Vec<T, W> ld(const T* p) {
    using B = typename Bits<W>::type;
    Vec<T, W> r;
    *reinterpret_cast<B*>(&r) = *reinterpret_cast<const B*>(p);
    return r;
}
template <int W, typename T>
__device__ __forceinline__ void st(T* p, const Vec<T, W>& v) {
    using B = typename Bits<W>::type;
    *reinterpret_cast<B*>(p) = *reinterpret_cast<const B*>(&v);
}

// Places and sines of the CTA's tokens.
__device__ __forceinline__ void token_setup(const RopeParams& p, const FreqAxes& axes, int32_t t0, int n, float2* cs,
                                            TokenPlace* place) {
    const int half = p.rot >> 1;
    for (int i = threadIdx.x; i < n * half; i += kThreads) {
        const int k = i / half, f = i - k * half;
        const double turns = (double)p.positions[axes.v[f] * p.axis_stride + t0 + k] * (double)p.inv_freq[f] *
                             0.15915494309189533577;   // 1 / (2 pi)
        const float frac = (float)(turns - rint(turns));
        float s, c;
        sincospif(2.0f * frac, &s, &c);
        cs[k * half + f] = make_float2(c, p.sign * s);
    }
    for (int k = threadIdx.x; k < n; k += kThreads) {
        TokenPlace pl{-1, -1, 1, 0};
        if (p.slots != nullptr) {
            const int64_t slot = p.slots[t0 + k];
            if (slot < 0) {
                pl.live = 0;
            } else if (slot >= p.num_slots) {
                if (p.status) *(volatile int32_t*)p.status = kStatusBadSlot;
            } else if (p.kpool != nullptr) {
                const int64_t blk = slot / p.block_size;
                const int64_t in_block = (slot - blk * p.block_size) * (int64_t)p.hkv * p.dim;
                pl.k_off = blk * p.k_block_stride + in_block;
                pl.v_off = blk * p.v_block_stride + in_block;
            }
        }
        place[k] = pl;
    }
}

// Where head `head` of a token is read and written: heads 0 .. hq-1 are queries, then keys, then values.
template <typename T>
struct HeadAt {
    const T* src;
    T *dst, *dst2;   // dst2: a key that goes to k_out and into the pool; no dst: nothing of the head is written
    bool rotate;
};
template <typename T>
__device__ __forceinline__ HeadAt<T> head_source(const RopeParams& p, int64_t t, int head) {
    HeadAt<T> h{nullptr, nullptr, nullptr, true};
    if (head < p.hq) {
        h.src = (const T*)p.q + t * p.q_stride + (int64_t)head * p.dim;
    } else if (head < p.hq + p.hkv) {
        h.src = (const T*)p.k + t * p.k_stride + (int64_t)(head - p.hq) * p.dim;
    } else {
        h.rotate = false;
        h.src = (const T*)p.v + t * p.v_stride + (int64_t)(head - p.hq - p.hkv) * p.dim;
    }
    return h;
}
template <typename T>
__device__ __forceinline__ void head_target(const RopeParams& p, int64_t t, int head, const TokenPlace& pl, HeadAt<T>& h) {
    if (!pl.live) return;
    if (head < p.hq) {
        h.dst = (T*)p.q_out + t * p.q_out_stride + (int64_t)head * p.dim;
    } else if (head < p.hq + p.hkv) {
        const int64_t o = (int64_t)(head - p.hq) * p.dim;
        if (p.k_out) h.dst = (T*)p.k_out + t * p.k_out_stride + o;
        if (pl.k_off >= 0) (h.dst ? h.dst2 : h.dst) = (T*)p.kpool + pl.k_off + o;
    } else if (pl.v_off >= 0) {
        h.dst = (T*)p.vpool + pl.v_off + (int64_t)(head - p.hq - p.hkv) * p.dim;
    }
}

// W elements per access: every address and row is aligned to as many, and a pair's partners lie in whole vectors.  W is
// 8 for most heads; a part of a head whose half is no multiple of 8 (24 of 96 dims, 40 of 80) has 4 or 2 (4096 tokens of
// 48 heads, bf16: 40 of 80 dims 16.3 us, 24 of 96 20.8, 20 of 80 28.5; element by element 91, 104 and 98).
//
// A CTA's threads are dealt evenly to its tokens.  A head has `units` of two vectors: of partners half a rotation apart
// and of what passes, or, with neighbouring pairs, of dims half a head apart (one vector a unit: 4096 tokens of 48 heads
// of 128, 32 dims rotated, 27.0 instead of 18.9 us, 128 as neighbours 22.7 instead of 19.7).  A thread has one unit of
// every `slots`-th head of its token, so its sines stay in registers.  kAtOnce heads are loaded at a time, and the first
// of them before the sines are made, whose latency hides behind the loads' (three at a time spill: 21.6 instead of
// 20.2 us for 48 heads of 128).
template <typename T, bool kNeighbours, int W>
__global__ void __launch_bounds__(kThreads, 4)
rope_append_kernel(const __grid_constant__ RopeParams p, const __grid_constant__ FreqAxes axes, int32_t heads, int32_t units, int32_t slots) {
    extern __shared__ float2 cs[];
    __shared__ TokenPlace place[kTokensPerCta];
    constexpr int kAtOnce = W == 8 ? 2 : 4;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int32_t t0 = blockIdx.x * p.tok_per_cta;
    const int n = min(p.tok_per_cta, p.tokens - t0);
    const int threads = kThreads / p.tok_per_cta;          // of a token
    const int k = threadIdx.x / threads, me = threadIdx.x - k * threads;
    const int slot = me / units, lane = me - slot * units;
    const int64_t t = t0 + k;
    const int half = p.rot >> 1, turned = kNeighbours ? p.rot / W : half / W;
    // this thread's vectors of a query or key head, and of a value head; -1: none
    const bool pairs = lane < turned, pairs2 = kNeighbours && units + lane < turned;
    // (spelled out twice: shared between the two, they cost small calls 0.2 us)
    const int passing = (p.dim - p.rot) / W, pass = lane - turned, pass_units = units - turned;
    const int first = pairs || kNeighbours ? W * lane : p.rot + W * pass;
    const int second = kNeighbours ? (units + lane < p.dim / W ? W * (units + lane) : -1)
                       : pairs     ? half + W * lane
                                   : pass + pass_units < passing ? first + W * pass_units : -1;
    const int v_first = W * lane, v_second = units + lane < p.dim / W ? W * (units + lane) : -1;
    Vec<T, W> a[kAtOnce], b[kAtOnce];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    auto load = [&](int h0) {
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int h = h0 + i * slots;
            if (h >= heads) continue;
            const bool value = h >= p.hq + p.hkv;
            const T* src = h < p.hq ? (const T*)p.q + t * p.q_stride + (int64_t)h * p.dim
                           : !value ? (const T*)p.k + t * p.k_stride + (int64_t)(h - p.hq) * p.dim
                                    : (const T*)p.v + t * p.v_stride + (int64_t)(h - p.hq - p.hkv) * p.dim;
            a[i] = ld<W>(src + (value ? v_first : first));
            const int s = value ? v_second : second;
            if (s >= 0) b[i] = ld<W>(src + s);
        }
    };
    const bool busy = k < n && slot < slots;
    if (busy) load(slot);
    token_setup(p, axes, t0, n, cs, place);
    __syncthreads();
    if (!busy) return;
    const TokenPlace pl = place[k];
    if (!pl.live) return;
    float2 w[W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
        if (!kNeighbours && pairs) w[j] = cs[k * half + W * lane + j];
        if (kNeighbours && (j < W / 2 ? pairs : pairs2)) w[j] = cs[k * half + W / 2 * (j < W / 2 ? lane : units + lane - 1) + j];
    }
    for (int h0 = slot; h0 < heads;) {
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int h = h0 + i * slots;
            if (h >= heads) continue;
            const bool value = h >= p.hq + p.hkv;
            if (pairs && !value)
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    if (kNeighbours && j == W / 2 && !pairs2) break;
                    Vec<T, W>& at = kNeighbours && j >= W / 2 ? b[i] : a[i];
                    T& e1 = kNeighbours ? at.e[(2 * j) % W] : a[i].e[j];
                    T& e2 = kNeighbours ? at.e[(2 * j + 1) % W] : b[i].e[j];
                    const float x1 = to_f(e1), x2 = to_f(e2);
                    e1 = from_f<T>(fmaf(x1, w[j].x, -x2 * w[j].y));
                    e2 = from_f<T>(fmaf(x2, w[j].x, x1 * w[j].y));
                }
            const int f = value ? v_first : first, s = value ? v_second : second;
            T *dst = nullptr, *dst2 = nullptr;             // dst2: a key that goes to k_out and into the pool
            if (h < p.hq) {
                dst = (T*)p.q_out + t * p.q_out_stride + (int64_t)h * p.dim;
            } else if (!value) {
                if (p.k_out) dst = (T*)p.k_out + t * p.k_out_stride + (int64_t)(h - p.hq) * p.dim;
                if (pl.k_off >= 0) dst2 = (T*)p.kpool + pl.k_off + (int64_t)(h - p.hq) * p.dim;
            } else if (pl.v_off >= 0) {
                dst = (T*)p.vpool + pl.v_off + (int64_t)(h - p.hq - p.hkv) * p.dim;
            }
            if (dst) {
                st<W>(dst + f, a[i]);
                if (s >= 0) st<W>(dst + s, b[i]);
            }
            if (dst2) {
                st<W>(dst2 + f, a[i]);
                if (s >= 0) st<W>(dst2 + s, b[i]);
            }
        }
        h0 += kAtOnce * slots;
        if (h0 < heads) load(h0);
    }
}

// Element by element, for rows that are not even on 4-byte boundaries and halves of an odd number of pairs.
template <typename T>
__global__ void __launch_bounds__(kThreads)
rope_append_elements_kernel(const __grid_constant__ RopeParams p, const __grid_constant__ FreqAxes axes, int32_t heads,
                            bool neighbours) {
    extern __shared__ float2 cs[];
    __shared__ TokenPlace place[kTokensPerCta];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int32_t t0 = blockIdx.x * p.tok_per_cta;
    const int n = min(p.tok_per_cta, p.tokens - t0);
    token_setup(p, axes, t0, n, cs, place);
    __syncthreads();
    const int half = p.rot >> 1;
    const int units = p.dim - half;   // of a rotated head: its pairs, then the dims that pass
    for (int u = threadIdx.x >> 5; u < n * heads; u += kThreads >> 5) {
        const int k = u / heads, head = u - k * heads;
        HeadAt<T> h = head_source<T>(p, t0 + k, head);
        head_target(p, t0 + k, head, place[k], h);
        if (!h.dst) continue;
        for (int i = threadIdx.x & 31; i < (h.rotate ? units : p.dim); i += 32) {
            if (h.rotate && i < half) {
                const float2 w = cs[k * half + i];
                const int d1 = neighbours ? 2 * i : i, d2 = neighbours ? 2 * i + 1 : i + half;
                const float x1 = to_f(h.src[d1]), x2 = to_f(h.src[d2]);
                const T y1 = from_f<T>(fmaf(x1, w.x, -x2 * w.y)), y2 = from_f<T>(fmaf(x2, w.x, x1 * w.y));
                h.dst[d1] = y1;
                h.dst[d2] = y2;
                if (h.dst2) {
                    h.dst2[d1] = y1;
                    h.dst2[d2] = y2;
                }
            } else {
                const int d = h.rotate ? i + half : i;
                const T x = h.src[d];
                h.dst[d] = x;
                if (h.dst2) h.dst2[d] = x;
            }
        }
    }
}

// Whether rows that begin there are aligned to w elements.
bool aligned(const void* p, int64_t stride, int w) { return (reinterpret_cast<uintptr_t>(p) % (2 * w)) == 0 && stride % w == 0; }

template <typename T, bool kNeighbours, int W>
cudaError_t launch_vectors(RopeParams p, const FreqAxes& axes, int32_t heads, cudaStream_t s) {
    const int units = kNeighbours ? (p.dim / W + 1) / 2 : p.rot / 2 / W + ((p.dim - p.rot) / W + 1) / 2;
    // Few tokens: one per CTA, so that they spread over the chip.  Many: a round of four CTAs per SM costs about 2 us
    // that its sines take, so as many as make a sine per thread and leave the chip filled, but not a little more than
    // a round, whose rest then runs alone (only the first round's rest is avoided: 5003 tokens of 32 heads of 80 are two
    // full rounds and a third of 67 CTAs).  Times (80 heads of 128, 1 / 2 / 4 tokens a CTA: 512 tokens 5.6 / 7.0 / 7.8 us, 2048
    // 22.4 / 18.2 / 16.7, 8192 74.7 / 60.1 / 57.6; 32 heads of 80, 1 / 2 / 4 / 8: 2500 tokens 11.3 / 8.5 / 8.0 / 9.0, 5003
    // 22.8 / 16.5 / 14.7 / 14.8, 9000 39.2 / 26.9 / 22.6 / 19.6).
    constexpr int kRound = 4 * 148, kFilled = 350;
    p.tok_per_cta = 1;
    for (int n = 2; n <= kTokensPerCta && n * p.rot <= 2 * kThreads && n * units <= kThreads; n *= 2) {
        const int ctas = p.tokens / n;
        if (ctas >= kFilled && (ctas <= kRound || ctas > kRound * 3 / 2)) p.tok_per_cta = n;
    }
    const dim3 grid((unsigned)((p.tokens + p.tok_per_cta - 1) / p.tok_per_cta));
    return ps::launch_dependent(rope_append_kernel<T, kNeighbours, W>, grid, dim3(kThreads),
                                (size_t)p.tok_per_cta * (p.rot / 2) * sizeof(float2), s, p, axes, heads, units,
                                kThreads / p.tok_per_cta / units);
}

// width: elements per access, 1 = element by element.
template <typename T>
cudaError_t launch_rope(RopeParams p, const FreqAxes& axes, int32_t heads, bool neighbours, int width, cudaStream_t s) {
    switch (width) {
        case 8: return neighbours ? launch_vectors<T, true, 8>(p, axes, heads, s) : launch_vectors<T, false, 8>(p, axes, heads, s);
        case 4: return neighbours ? launch_vectors<T, true, 4>(p, axes, heads, s) : launch_vectors<T, false, 4>(p, axes, heads, s);
        case 2: return neighbours ? launch_vectors<T, true, 2>(p, axes, heads, s) : launch_vectors<T, false, 2>(p, axes, heads, s);
    }
    p.tok_per_cta = 1;
    return ps::launch_dependent(rope_append_elements_kernel<T>, dim3((unsigned)p.tokens), dim3(kThreads), (size_t)(p.rot / 2) * sizeof(float2), s,
                                p, axes, heads, neighbours);
}

}  // namespace

extern "C" int32_t ps_rope_append(const ps_rope_args* args, void* stream, char* err_buf, int32_t err_cap) {
    using ps::arg_fail;
    if (err_buf && err_cap > 0) err_buf[0] = 0;
    auto bad = [&](const char* m) { return arg_fail(err_buf, err_cap, PS_ERR_INVALID, m); };
    if (!args) return bad("ps_rope_append: null arguments");
    const ps_rope_args a = *args;
    if (a.tokens < 0 || a.num_q_heads < 0 || a.num_kv_heads < 0 || a.head_dim <= 0 || a.rot_dim < 0 || a.num_axes < 0)
        return bad("ps_rope_append: negative count or non-positive size");
    if (a.head_dim > kMaxHeadDim || a.rot_dim > a.head_dim || a.rot_dim % 2)
        return bad("ps_rope_append: head_dim is at most 512, rot_dim an even number up to head_dim");
    if (a.dtype != PS_DTYPE_BF16 && a.dtype != PS_DTYPE_FP16) return bad("ps_rope_append: dtype must be PS_DTYPE_BF16 or PS_DTYPE_FP16");
    if (a.flags & ~(PS_ROPE_NEIGHBOURS | PS_ROPE_INVERSE)) return bad("ps_rope_append: unknown flag");
    if (a.tokens == 0) return PS_OK;         // tensors without elements have no address
    const bool append = a.kpool || a.vpool;
    const bool do_q = a.q != nullptr && a.num_q_heads > 0, do_k = a.k != nullptr && a.num_kv_heads > 0;
    if (do_q && !a.q_out) return bad("ps_rope_append: q without q_out");
    if (append && (!a.kpool || !a.vpool || !a.k || !a.v || !a.slots || a.num_kv_heads == 0))
        return bad("ps_rope_append: an append needs k, v, both pools and slots");
    if (append && (a.block_size <= 0 || a.num_gpu_blocks <= 0)) return bad("ps_rope_append: non-positive block size or pool");
    const int64_t block_elems = append ? (int64_t)a.block_size * a.num_kv_heads * a.head_dim : 0;
    if (append && ((a.num_gpu_blocks > 1 && (a.k_block_stride < block_elems || a.v_block_stride < block_elems))))
        return bad("ps_rope_append: a pool's block stride is smaller than a block");
    if (do_k && !append && !a.k_out) return bad("ps_rope_append: k without k_out or pools");
    FreqAxes axes{};
    if (a.rot_dim > 0) {
        if (!a.inv_freq || a.num_axes < 1 || a.num_axes > 8) return bad("ps_rope_append: a rotation needs positions, inv_freq and 1 to 8 axes");
        for (int i = 0; i < a.rot_dim / 2; ++i) {
            if (a.freq_axis[i] >= a.num_axes) return bad("ps_rope_append: freq_axis names an axis that is not there");
            axes.v[i] = a.freq_axis[i];
        }
    }
    if (!do_q && !do_k) return PS_OK;
    // An output may be its own input, whose elements a thread has loaded before it stores theirs; anything else that an
    // output shares with an input or with the other output would be stored by one thread while another reads or stores it.
    const int64_t q_width = (int64_t)a.num_q_heads * a.head_dim, kv_width = (int64_t)a.num_kv_heads * a.head_dim;
    using ps::RowSet;
    const RowSet q{a.q, a.q_stride, q_width}, k{a.k, a.k_stride, kv_width}, v{a.v, a.v_stride, kv_width};
    const RowSet q_out{a.q_out, a.q_out_stride, q_width}, k_out{a.k_out, a.k_out_stride, kv_width};
    const bool to_k = do_k && a.k_out;
    auto apart = [&](const RowSet& out, const RowSet& in, bool may_be) {
        return (may_be && out.p == in.p && (out.stride == in.stride || a.tokens == 1)) || !ps::rows_meet(out, in, a.tokens);
    };
    auto rows_apart = [&](const RowSet& out) { return a.tokens == 1 || out.stride >= out.width || -out.stride >= out.width; };
    if ((do_q && !rows_apart(q_out)) || (to_k && !rows_apart(k_out))) return bad("ps_rope_append: rows of q_out or k_out overlap");
    if ((do_q && (!apart(q_out, q, true) || (do_k && !apart(q_out, k, false)) || (append && !apart(q_out, v, false)))) ||
        (to_k && (!apart(k_out, k, true) || (do_q && !apart(k_out, q, false)) || (append && !apart(k_out, v, false)))) ||
        (do_q && to_k && !apart(q_out, k_out, false)))
        return bad("ps_rope_append: q_out or k_out overlaps an input other than its own, or its own by another stride or in part");
    if (a.rot_dim > 0 && !a.positions) return bad("ps_rope_append: a rotation needs positions, inv_freq and 1 to 8 axes");
    RopeParams p{};
    p.q = a.q, p.k = a.k, p.v = a.v, p.q_out = a.q_out, p.k_out = a.k_out, p.kpool = a.kpool, p.vpool = a.vpool;
    p.slots = a.slots, p.positions = a.positions, p.inv_freq = a.inv_freq, p.status = a.status_word;
    p.q_stride = a.q_stride, p.k_stride = a.k_stride, p.v_stride = a.v_stride;
    p.q_out_stride = a.q_out_stride, p.k_out_stride = a.k_out_stride, p.axis_stride = a.axis_stride;
    p.k_block_stride = a.k_block_stride, p.v_block_stride = a.v_block_stride;
    p.tokens = a.tokens, p.dim = a.head_dim, p.rot = a.rot_dim, p.block_size = append ? a.block_size : 1;
    p.hq = do_q ? a.num_q_heads : 0;
    p.hkv = do_k ? a.num_kv_heads : 0;
    // slots without pools only mark the padding: none of them is out of range
    p.num_slots = append ? (int64_t)a.num_gpu_blocks * a.block_size : INT64_MAX;
    p.sign = a.flags & PS_ROPE_INVERSE ? -1.f : 1.f;
    const int32_t heads = p.hq + p.hkv + (append ? p.hkv : 0);
    const bool neighbours = a.flags & PS_ROPE_NEIGHBOURS;
    // the widest access that rows, heads and the parts of a head allow
    int width = 8;
    auto fits = [&](int w) {
        bool ok = a.head_dim % w == 0 && a.rot_dim % (neighbours ? w : 2 * w) == 0;
        if (do_q) ok = ok && aligned(a.q, a.q_stride, w) && aligned(a.q_out, a.q_out_stride, w);
        if (do_k) ok = ok && aligned(a.k, a.k_stride, w) && aligned(a.k_out, a.k_out ? a.k_out_stride : 0, w);
        if (append) ok = ok && aligned(a.v, a.v_stride, w) && aligned(a.kpool, a.k_block_stride, w) && aligned(a.vpool, a.v_block_stride, w);
        return ok;
    };
    while (width > 1 && !fits(width)) width /= 2;
    cudaError_t e = a.dtype == PS_DTYPE_BF16 ? launch_rope<__nv_bfloat16>(p, axes, heads, neighbours, width, (cudaStream_t)stream)
                                             : launch_rope<__half>(p, axes, heads, neighbours, width, (cudaStream_t)stream);
    if (e != cudaSuccess) return ps::launch_fail(err_buf, err_cap, "ps_rope_append", e);
    return PS_OK;
}

// ps_build_slots: block tables, slot map and positions of a batch from request lengths that live on the device.
//
//   need_b   = ceil((ctx_b + new_b) / S) - ceil(ctx_b / S)      blocks row b takes from the free stack
//   start_b  = sum of new over the rows before b
//   slot[t]  = table[b][p / S] * S + p % S,   p = ctx_b + (t - start_b),   start_b <= t < start_b + new_b
//
// Rows that end give their blocks back first (pushed in row order, table order), then the growing rows pop one id at
// a time in row order: the free stack and the tables come out as from ps_kv_free and ps_kv_alloc in those orders.
//
// The work is a few words per row and token; what bounds it is latency: the chain "load lengths, scan, load a free
// id, store".  Two ways, chosen by the room for tokens and the number of rows:
//   - slots_one_cta_kernel: one CTA scans, pushes, pops and maps; barriers order its steps and one launch does all.
//     For room for up to 512 tokens (2048 with over 512 rows, 4096 in place): 64 rows of a token each 3.1 us; 200 rows
//     4.6 us for 1000 tokens, 5.4 for 2000, 7.0 for 4000, 14.4 for 16000.  And for over 4096 rows, whose counts the other
//     way does not hold in shared memory, whatever the room: 4097 rows of a token each 20.9 us, 24.7 with room for 16000
//     more; 5000 rows 42 us with room for 100000 tokens and 89 with as many live ones (4096 rows the other way: 9.8).
//   - slots_wide_kernel: every CTA scans all rows for itself (cheaper than another launch) and takes its part of
//     pushes, pops and tokens.  A popped id is found without waiting for the pushes: an index above the old top
//     belongs to the table of a row that ended, which a search in the scanned counts names.  Where lengths or count are
//     updated in place, a second kernel of one CTA does that when nobody reads them any more, which takes 2.5 us more
//     (256 rows with prompt chunks 7.1 instead of 4.5), 3 to 4 with 1000 rows and over.
//     (200 rows: 4.1 us for 1000 to 16000 tokens; 1024 rows of a token each 6.5 us and 5.8 in one CTA.)
// Work on blocks and tokens is dealt to threads by the scanned counts (binary search in shared memory), so one long
// prompt costs the same as many short ones.
#include <algorithm>
#include <atomic>
#include <cstdio>

#include "ps_internal.h"
#include "ps_kvswap.h"

namespace {

constexpr int kStatusNoMem = 4;     // not enough free blocks
constexpr int kStatusLength = 5;    // a length, a total or the free count is out of range
constexpr int kStatusBadId = 2;     // a block id outside the pool

constexpr int kMaxThreads = 1024;
constexpr int kWideAtOnce = 148 * 1024;  // threads: each CTA scans all rows
constexpr int32_t kWideRows = 4096;      // the scanned counts of so many rows fit into shared memory

struct Row {
    int32_t ctx, add, old_blocks, need, back;
};

// Blocks of n >= 0 tokens; in 32 bits, where a division takes a tenth of one in 64.
__device__ __forceinline__ int32_t blocks_of(const ps_slots_args& a, int32_t n) {
    return (int32_t)(((uint32_t)n + (uint32_t)a.block_size - 1u) / (uint32_t)a.block_size);
}

// Row b's figures; *bad is raised when a length does not fit.
__device__ __forceinline__ Row load_row(const ps_slots_args& a, int b, bool* bad) {
    Row r{0, 0, 0, 0, 0};
    const int32_t ctx = a.ctx_lens[b], nw = a.new_lens[b];
    const int64_t room = (int64_t)a.table_stride * a.block_size;
    if (ctx < 0 || nw < PS_SLOTS_END || (int64_t)ctx + (nw > 0 ? nw : 0) > room || (int64_t)ctx + nw > INT32_MAX) {
        *bad = true;
        return r;
    }
    r.ctx = ctx;
    r.old_blocks = blocks_of(a, ctx);
    if (nw == PS_SLOTS_END) {
        r.back = r.old_blocks;
    } else {
        r.add = nw;
        r.need = blocks_of(a, ctx + nw) - r.old_blocks;
    }
    return r;
}

// What keeps a call with these totals from being carried out; 0: nothing.
__device__ __forceinline__ int refusal(const ps_slots_args& a, bool bad, int64_t add, int64_t need, int64_t back, int32_t count) {
    if (bad || add > a.max_tokens) return kStatusLength;
    if (!a.free_ids) return 0;
    if (count < 0 || count + back > a.num_gpu_blocks) return kStatusLength;
    return count + back - need < 0 ? kStatusNoMem : 0;
}

// Three counts; in 64 bits, so that no sum of valid or invalid lengths wraps.
struct Counts {
    long long v[3];
};
__device__ __forceinline__ void warp_scan3(Counts& c) {   // inclusive
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const long long n = __shfl_up_sync(0xffffffffu, c.v[k], o);
            if (lane >= o) c.v[k] += n;
        }
}
// Exclusive scan over the CTA; the totals come back in all.  Every thread calls it.
__device__ void cta_scan3(Counts& c, Counts& all, long long (*warp_sums)[32]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
    Counts inc = c;
    warp_scan3(inc);
    __syncthreads();   // the sums of an earlier call have been read
    if (lane == 31)
#pragma unroll
        for (int k = 0; k < 3; ++k) warp_sums[k][warp] = inc.v[k];
    __syncthreads();
    Counts w;
#pragma unroll
    for (int k = 0; k < 3; ++k) w.v[k] = lane < nwarps ? warp_sums[k][lane] : 0;
    warp_scan3(w);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        all.v[k] = __shfl_sync(0xffffffffu, w.v[k], 31);
        const long long before = __shfl_sync(0xffffffffu, w.v[k], warp > 0 ? warp - 1 : 0);
        c.v[k] = inc.v[k] - c.v[k] + (warp > 0 ? before : 0);
    }
}

// Largest r in [0, n) with pfx[r] <= e, pfx ascending and pfx[0] <= e: of equal entries the last, which is the
// row that is not empty.
template <typename P>
__device__ __forceinline__ int row_of(P pfx, int n, int e) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (pfx[mid] <= e) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(kMaxThreads)
slots_one_cta_kernel(const ps_slots_args a) {
    __shared__ long long warp_sums[3][32];
    __shared__ int pfx[kMaxThreads], pfx_need[kMaxThreads];
    __shared__ int32_t row_ctx[kMaxThreads], row_old[kMaxThreads];
    const int tid = threadIdx.x, nt = blockDim.x;
    const bool pool = a.free_ids != nullptr;

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // totals first: a call that does not fit changes nothing
    const int32_t count = pool ? *a.free_count : 0;
    bool bad = false;
    Row r{0, 0, 0, 0, 0};
    Counts c{{0, 0, 0}}, all;
    for (int b = tid; b < a.batch; b += nt) {
        r = load_row(a, b, &bad);
        c.v[0] += r.add;
        c.v[1] += r.need;
        c.v[2] += r.back;
    }
    cta_scan3(c, all, warp_sums);
    const int code = refusal(a, __syncthreads_or(bad), all.v[0], all.v[1], all.v[2], count);
    const int32_t total = code ? 0 : (int32_t)all.v[0];
    const int32_t top = count + (int32_t)all.v[2];      // of the stack after the pushes
    if (tid == 0) {
        if (code && a.status_word) *(volatile int32_t*)a.status_word = code;
        if (pool) *a.free_count_out = code ? count : (int32_t)(top - all.v[1]);
        a.token_start[a.batch] = total;
    }
    if (code) {
        for (int b = tid; b < a.batch; b += nt) {
            a.ctx_lens_out[b] = a.ctx_lens[b];
            a.token_start[b] = 0;
        }
    } else {
        const bool once = a.batch <= nt;                 // the scan above is the one that is needed
        // blocks of the rows that end go onto the stack
        if (pool && all.v[2] > 0) {
            int carry = 0;
            for (int c0 = 0; c0 < a.batch; c0 += nt) {
                Counts v = c, tot = all;
                if (!once) {
                    r = c0 + tid < a.batch ? load_row(a, c0 + tid, &bad) : Row{0, 0, 0, 0, 0};
                    v = Counts{{0, 0, r.back}};
                    cta_scan3(v, tot, warp_sums);
                }
                pfx[tid] = (int)v.v[2];
                __syncthreads();
                for (int e = tid; e < (int)tot.v[2]; e += nt) {
                    const int k = row_of(pfx, min(nt, a.batch - c0), e);
                    a.free_ids[count + carry + e] = a.block_tables[(int64_t)(c0 + k) * a.table_stride + (e - pfx[k])];
                }
                carry += (int)tot.v[2];
                __syncthreads();
            }
        }
        // growing rows take theirs from the top, and the tokens get their slots
        int carry_tok = 0, carry_need = 0;
        for (int c0 = 0; c0 < a.batch; c0 += nt) {
            const int b = c0 + tid, rows = min(nt, a.batch - c0);
            Counts v = c, tot = all;
            if (!once) {
                r = b < a.batch ? load_row(a, b, &bad) : Row{0, 0, 0, 0, 0};
                v = Counts{{r.add, r.need, 0}};
                cta_scan3(v, tot, warp_sums);
            }
            pfx[tid] = (int)v.v[0];
            pfx_need[tid] = (int)v.v[1];
            row_ctx[tid] = r.ctx;
            row_old[tid] = r.old_blocks;
            if (b < a.batch) {
                a.ctx_lens_out[b] = a.new_lens[b] == PS_SLOTS_END ? 0 : r.ctx + r.add;
                a.token_start[b] = carry_tok + (int)v.v[0];
            }
            __syncthreads();
            if (pool)
                for (int e = tid; e < (int)tot.v[1]; e += nt) {
                    const int k = row_of(pfx_need, rows, e);
                    a.block_tables[(int64_t)(c0 + k) * a.table_stride + row_old[k] + (e - pfx_need[k])] =
                        __ldcg(a.free_ids + (top - 1 - carry_need - e));
                }
            for (int e = tid; e < (int)tot.v[0]; e += nt) {
                const int k = row_of(pfx, rows, e);
                const int32_t p = row_ctx[k] + (e - pfx[k]);
                const int32_t blk = (int32_t)((uint32_t)p / (uint32_t)a.block_size);
                // a block taken in this call is read from the stack, so that no barrier has to order the table's
                // store before this load
                const int32_t id = pool && blk >= row_old[k]
                                       ? __ldcg(a.free_ids + (top - 1 - carry_need - pfx_need[k] - (blk - row_old[k])))
                                       : __ldcg(a.block_tables + (int64_t)(c0 + k) * a.table_stride + blk);
                const bool in_pool = (unsigned)id < (unsigned)a.num_gpu_blocks;
                if (!in_pool && a.status_word) *(volatile int32_t*)a.status_word = kStatusBadId;
                a.slots[carry_tok + e] = in_pool ? (int64_t)id * a.block_size + (p - blk * a.block_size) : -1;
                if (a.positions) a.positions[carry_tok + e] = p;
            }
            carry_tok += (int)tot.v[0];
            carry_need += (int)tot.v[1];
            __syncthreads();
        }
    }
    for (int t = total + tid; t < a.max_tokens; t += nt) {
        a.slots[t] = -1;
        if (a.positions) a.positions[t] = 0;
    }
}

__device__ __forceinline__ void update_row(const ps_slots_args& a, int b, int code) {
    const int32_t n = a.ctx_lens[b], m = a.new_lens[b];
    a.ctx_lens_out[b] = code ? n : m == PS_SLOTS_END ? 0 : n + m;
}
__device__ __forceinline__ void update_count(const ps_slots_args& a, int code, int32_t count, const Counts& all) {
    if (a.free_ids) *a.free_count_out = code ? count : (int32_t)(count + all.v[2] - all.v[1]);
    if (code && a.status_word) *(volatile int32_t*)a.status_word = code;
}

// Every CTA knows all rows; the CTAs share pushes, pops and tokens.  Reads what it does not write: table entries of
// blocks that rows have, and the stack below its top.  apart: lengths and count have places of their own to go to.
__global__ void __launch_bounds__(kMaxThreads)
slots_wide_kernel(const ps_slots_args a, bool apart) {
    extern __shared__ int32_t rows_smem[];     // [batch] each: tokens, needs, returns before the row; its length
    int32_t *tok = rows_smem, *need = tok + a.batch, *back = need + a.batch, *ctx = back + a.batch;
    __shared__ long long warp_sums[3][32];
    const int tid = threadIdx.x;
    const bool pool = a.free_ids != nullptr;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int32_t count = pool ? *a.free_count : 0;
    const int per = (a.batch + (int)blockDim.x - 1) / (int)blockDim.x;
    const int b_lo = min(a.batch, tid * per), b_hi = min(a.batch, b_lo + per);
    bool bad = false;
    Row r{0, 0, 0, 0, 0};
    Counts c{{0, 0, 0}}, all;
    for (int b = b_lo; b < b_hi; ++b) {
        r = load_row(a, b, &bad);
        c.v[0] += r.add;
        c.v[1] += r.need;
        c.v[2] += r.back;
    }
    cta_scan3(c, all, warp_sums);
    const int code = refusal(a, __syncthreads_or(bad), all.v[0], all.v[1], all.v[2], count);
    const bool failed = code != 0;
    if (apart && blockIdx.x == 0) {
        for (int b = tid; b < a.batch; b += blockDim.x) update_row(a, b, code);
        if (tid == 0) update_count(a, code, count, all);
    }
    const int32_t total = failed ? 0 : (int32_t)all.v[0];
    const int32_t top = count + (int32_t)(failed ? 0 : all.v[2]);    // of the stack after the pushes
    if (!failed) {                              // every total that is used fits 32 bits
        int at[3] = {(int)c.v[0], (int)c.v[1], (int)c.v[2]};
        for (int b = b_lo; b < b_hi; ++b) {
            if (per > 1) r = load_row(a, b, &bad);
            tok[b] = at[0];
            need[b] = at[1];
            back[b] = at[2];
            ctx[b] = r.ctx;
            at[0] += r.add;
            at[1] += r.need;
            at[2] += r.back;
        }
        __syncthreads();
    }
    const int64_t me = (int64_t)blockIdx.x * blockDim.x + tid, everyone = (int64_t)gridDim.x * blockDim.x;
    for (int64_t b = me; b <= a.batch; b += everyone) a.token_start[b] = failed ? 0 : b < a.batch ? tok[b] : total;
    auto returned = [&](int e) {                // the e-th id that goes back
        const int k = row_of(back, a.batch, e);
        return a.block_tables[(int64_t)k * a.table_stride + (e - back[k])];
    };
    auto popped = [&](int e) {                  // the e-th id that is taken
        const int at = top - 1 - e;
        return at < count ? a.free_ids[at] : returned(at - count);
    };
    if (!failed && pool) {
        // by the last CTAs first: the first ones take the blocks
        for (int64_t e = everyone - 1 - me; e < all.v[2]; e += everyone) a.free_ids[count + e] = returned((int)e);
        for (int64_t e = me; e < all.v[1]; e += everyone) {
            const int k = row_of(need, a.batch, (int)e);
            a.block_tables[(int64_t)k * a.table_stride + blocks_of(a, ctx[k]) + ((int)e - need[k])] = popped((int)e);
        }
    }
    for (int64_t t = me; t < a.max_tokens; t += everyone) {
        int64_t slot = -1;
        int32_t p = 0;
        if (t < total) {
            const int k = row_of(tok, a.batch, (int)t);
            p = ctx[k] + ((int)t - tok[k]);
            const int32_t blk = (int32_t)((uint32_t)p / (uint32_t)a.block_size), old_blocks = blocks_of(a, ctx[k]);
            const int32_t id = pool && blk >= old_blocks ? popped(need[k] + (blk - old_blocks))
                                                         : a.block_tables[(int64_t)k * a.table_stride + blk];
            if ((unsigned)id < (unsigned)a.num_gpu_blocks) slot = (int64_t)id * a.block_size + (p - blk * a.block_size);
            else if (a.status_word) *(volatile int32_t*)a.status_word = kStatusBadId;
        }
        a.slots[t] = slot;
        if (a.positions) a.positions[t] = p;
    }
}

// Behind slots_wide_kernel: what it read and may be updated in place.
__global__ void __launch_bounds__(kMaxThreads)
slots_update_kernel(const ps_slots_args a) {
    __shared__ long long warp_sums[3][32];
    const int tid = threadIdx.x;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int32_t count = a.free_ids ? *a.free_count : 0;
    bool bad = false;
    Counts c{{0, 0, 0}}, all;
    for (int b = tid; b < a.batch; b += kMaxThreads) {
        const Row r = load_row(a, b, &bad);
        c.v[0] += r.add;
        c.v[1] += r.need;
        c.v[2] += r.back;
    }
    cta_scan3(c, all, warp_sums);
    const int code = refusal(a, __syncthreads_or(bad), all.v[0], all.v[1], all.v[2], count);
    for (int b = tid; b < a.batch; b += kMaxThreads) update_row(a, b, code);
    if (tid == 0) update_count(a, code, count, all);
}

// Lets slots_wide_kernel have the shared memory of kWideRows rows on the current device: asked for once per device, and
// not by the size of a call, whose limit would then depend on the calls before it.
constexpr int kMaxDevices = 64;
cudaError_t allow_wide_rows() {
    static std::atomic<bool> allowed[kMaxDevices];
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    if (allowed[dev].load(std::memory_order_acquire)) return cudaSuccess;
    e = cudaFuncSetAttribute(slots_wide_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kWideRows * 4 * sizeof(int32_t)));
    if (e == cudaSuccess) allowed[dev].store(true, std::memory_order_release);
    return e;
}

}  // namespace

extern "C" int32_t ps_build_slots(const ps_slots_args* args, void* stream, char* err_buf, int32_t err_cap) {
    using ps::arg_fail;
    if (err_buf && err_cap > 0) err_buf[0] = 0;
    if (!args) return arg_fail(err_buf, err_cap, PS_ERR_INVALID, "ps_build_slots: null arguments");
    const ps_slots_args a = *args;
    if (a.batch < 0 || a.max_tokens < 0 || a.block_size <= 0 || a.num_gpu_blocks <= 0 || a.table_stride <= 0)
        return arg_fail(err_buf, err_cap, PS_ERR_INVALID, "ps_build_slots: negative count or non-positive size");
    if ((a.batch > 0 && (!a.ctx_lens || !a.new_lens || !a.block_tables || !a.ctx_lens_out)) || !a.token_start ||
        (a.max_tokens > 0 && !a.slots))
        return arg_fail(err_buf, err_cap, PS_ERR_INVALID, "ps_build_slots: null pointer");
    if (a.free_ids && (!a.free_count || !a.free_count_out))
        return arg_fail(err_buf, err_cap, PS_ERR_INVALID, "ps_build_slots: a free stack needs free_count and free_count_out");
    cudaStream_t s = (cudaStream_t)stream;
    const bool apart = a.ctx_lens_out != a.ctx_lens && (!a.free_ids || a.free_count_out != a.free_count);
    cudaError_t e;
    const int32_t one_cta = !apart ? 4096 : a.batch <= 512 ? 512 : 2048;    // room for so many tokens
    if (a.max_tokens <= one_cta || a.batch > kWideRows) {
        // few rows and tokens: fewer warps make the barriers of the scan cheaper
        const int threads = a.batch <= 256 && a.max_tokens <= 1024 ? 256 : kMaxThreads;
        e = ps::launch_dependent(slots_one_cta_kernel, dim3(1), dim3(threads), 0, s, a);
    } else {
        // a row a thread in the scan, and a token a thread
        const int threads = a.batch <= 256 ? 256 : a.batch <= 512 ? 512 : kMaxThreads;
        const int ctas = (int)std::min<int64_t>(((int64_t)a.max_tokens + threads - 1) / threads, kWideAtOnce / threads);
        const size_t smem = (size_t)a.batch * 4 * sizeof(int32_t);
        e = allow_wide_rows();
        if (e == cudaSuccess) e = ps::launch_dependent(slots_wide_kernel, dim3(ctas), dim3(threads), smem, s, a, apart);
        if (e == cudaSuccess && !apart) e = ps::launch_dependent(slots_update_kernel, dim3(1), dim3(kMaxThreads), 0, s, a);
    }
    if (e != cudaSuccess) return ps::launch_fail(err_buf, err_cap, "ps_build_slots", e);
    return PS_OK;
}

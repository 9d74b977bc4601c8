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
// id, store".  One CTA does all of it (slots_plan_kernel): a scan over the rows needs no second launch, and because
// one CTA both pushes and pops, a barrier orders them.  Work on blocks and tokens is dealt to threads by the scanned
// prefix (binary search in shared memory), so one long prompt costs the same as many short ones.  With room for
// many tokens the map itself is filled by a second kernel over the whole chip (slots_fill_kernel).
#include <cstdio>

#include "ps_internal.h"
#include "ps_kvswap.h"

namespace {

constexpr int kStatusNoMem = 4;     // not enough free blocks
constexpr int kStatusLength = 5;    // a length, a total or the free count is out of range
constexpr int kStatusBadId = 2;     // a block id outside the pool

constexpr int kMaxThreads = 1024;
constexpr int kFillThreads = 256;
constexpr int32_t kFillInPlan = 4096;  // room for at most so many tokens: the plan kernel writes the map itself

struct Plan {
    int64_t total, need, back;
    int ok;
};

struct Row {
    int32_t ctx, add, old_blocks, need, back;
};

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
    r.old_blocks = (int32_t)(((int64_t)ctx + a.block_size - 1) / a.block_size);
    if (nw == PS_SLOTS_END) {
        r.back = r.old_blocks;
    } else {
        r.add = nw;
        r.need = (int32_t)(((int64_t)ctx + nw + a.block_size - 1) / a.block_size) - r.old_blocks;
    }
    return r;
}

__device__ __forceinline__ int warp_scan(int v) {   // inclusive
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int n = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += n;
    }
    return v;
}

// Exclusive scans of three values over the CTA; the totals come back in tot.  Every thread calls it.
__device__ void block_scan3(int (&v)[3], int (&tot)[3], int (*warp_sums)[32]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
    int inc[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) inc[k] = warp_scan(v[k]);
    __syncthreads();   // the sums of an earlier call have been read
    if (lane == 31)
#pragma unroll
        for (int k = 0; k < 3; ++k) warp_sums[k][warp] = inc[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const int s = warp_scan(lane < nwarps ? warp_sums[k][lane] : 0);
        const int before = __shfl_sync(0xffffffffu, s, warp > 0 ? warp - 1 : 0);
        tot[k] = __shfl_sync(0xffffffffu, s, 31);
        v[k] = inc[k] - v[k] + (warp > 0 ? before : 0);
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
slots_plan_kernel(const ps_slots_args a, int32_t fill) {
    __shared__ int warp_sums[3][32];
    __shared__ int pfx[kMaxThreads + 1], pfx_need[kMaxThreads + 1];
    __shared__ int32_t row_ctx[kMaxThreads], row_old[kMaxThreads];
    __shared__ unsigned long long sum_add, sum_need, sum_back;
    __shared__ int sh_bad;
    const int tid = threadIdx.x, nt = blockDim.x;
    const bool pool = a.free_ids != nullptr;

    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (tid == 0) {
        sum_add = sum_need = sum_back = 0;
        sh_bad = 0;
    }
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // totals first: a call that does not fit changes nothing
    {
        const int32_t count = pool ? *a.free_count : 0;
        bool bad = false;
        long long add = 0, need = 0, back = 0;
        for (int b = tid; b < a.batch; b += nt) {
            const Row r = load_row(a, b, &bad);
            add += r.add;
            need += r.need;
            back += r.back;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            add += __shfl_xor_sync(0xffffffffu, add, o);
            need += __shfl_xor_sync(0xffffffffu, need, o);
            back += __shfl_xor_sync(0xffffffffu, back, o);
        }
        if ((tid & 31) == 0) {
            if (add) atomicAdd(&sum_add, (unsigned long long)add);
            if (need) atomicAdd(&sum_need, (unsigned long long)need);
            if (back) atomicAdd(&sum_back, (unsigned long long)back);
        }
        if (bad) sh_bad = kStatusLength;
        __syncthreads();
        if (tid == 0) {
            int code = sh_bad;
            if (!code && (int64_t)sum_add > a.max_tokens) code = kStatusLength;
            if (!code && pool) {
                if (count < 0 || count + (int64_t)sum_back > a.num_gpu_blocks) code = kStatusLength;
                else if (count + (int64_t)sum_back - (int64_t)sum_need < 0) code = kStatusNoMem;
            }
            sh_bad = code;
            if (code && a.status_word) *(volatile int32_t*)a.status_word = code;
            if (pool) *a.free_count_out = code ? count : (int32_t)(count + (int64_t)sum_back - (int64_t)sum_need);
            if (a.batch == 0) a.token_start[0] = 0;
            sum_need = (unsigned long long)(count + (int64_t)sum_back);   // top of the stack after the pushes
        }
        __syncthreads();
    }
    const bool failed = sh_bad != 0;
    const int32_t count_after = (int32_t)(int64_t)sum_need;                // valid unless failed
    const int32_t count = count_after - (int32_t)(int64_t)sum_back;
    const int32_t total = failed ? 0 : (int32_t)(int64_t)sum_add;
    if (failed) {
        for (int b = tid; b < a.batch; b += nt) {
            a.ctx_lens_out[b] = a.ctx_lens[b];
            a.token_start[b + 1] = 0;
        }
        if (tid == 0) a.token_start[0] = 0;
    } else {
        // blocks of the rows that end go onto the stack
        if (pool && sum_back > 0) {
            int carry = 0;
            for (int c0 = 0; c0 < a.batch; c0 += nt) {
                bool bad = false;
                Row r{0, 0, 0, 0, 0};
                if (c0 + tid < a.batch) r = load_row(a, c0 + tid, &bad);
                int v[3] = {r.back, 0, 0}, tot[3];
                block_scan3(v, tot, warp_sums);
                pfx[tid] = v[0];
                __syncthreads();
                for (int e = tid; e < tot[0]; e += nt) {
                    const int k = row_of(pfx, min(nt, a.batch - c0), e);
                    a.free_ids[count + carry + e] = a.block_tables[(int64_t)(c0 + k) * a.table_stride + (e - pfx[k])];
                }
                carry += tot[0];
                __syncthreads();
            }
        }
        // growing rows take theirs from the top, and the tokens get their slots
        int carry_tok = 0, carry_need = 0;
        for (int c0 = 0; c0 < a.batch; c0 += nt) {
            bool bad = false;
            Row r{0, 0, 0, 0, 0};
            const int b = c0 + tid;
            const int rows = min(nt, a.batch - c0);
            if (b < a.batch) r = load_row(a, b, &bad);
            int v[3] = {r.add, r.need, 0}, tot[3];
            block_scan3(v, tot, warp_sums);
            pfx[tid] = v[0];
            pfx_need[tid] = v[1];
            row_ctx[tid] = r.ctx;
            row_old[tid] = r.old_blocks;
            if (b < a.batch) {
                a.ctx_lens_out[b] = r.back > 0 || a.new_lens[b] == PS_SLOTS_END ? 0 : r.ctx + r.add;
                a.token_start[b] = carry_tok + v[0];
                if (b == a.batch - 1) a.token_start[a.batch] = carry_tok + v[0] + r.add;
            }
            __syncthreads();
            if (pool)
                for (int e = tid; e < tot[1]; e += nt) {
                    const int k = row_of(pfx_need, rows, e);
                    a.block_tables[(int64_t)(c0 + k) * a.table_stride + row_old[k] + (e - pfx_need[k])] =
                        __ldcg(a.free_ids + (count_after - 1 - carry_need - e));
                }
            if (fill)
                for (int e = tid; e < tot[0]; e += nt) {
                    const int k = row_of(pfx, rows, e);
                    const int32_t p = row_ctx[k] + (e - pfx[k]);
                    const int32_t blk = p / a.block_size;
                    // a block taken in this call is read from the stack, so that no barrier has to order the
                    // table's store before this load
                    const int32_t id = pool && blk >= row_old[k]
                                           ? __ldcg(a.free_ids + (count_after - 1 - carry_need - pfx_need[k] - (blk - row_old[k])))
                                           : __ldcg(a.block_tables + (int64_t)(c0 + k) * a.table_stride + blk);
                    const bool in_pool = (unsigned)id < (unsigned)a.num_gpu_blocks;
                    if (!in_pool && a.status_word) *(volatile int32_t*)a.status_word = kStatusBadId;
                    a.slots[carry_tok + e] = in_pool ? (int64_t)id * a.block_size + (p - blk * a.block_size) : -1;
                    if (a.positions) a.positions[carry_tok + e] = p;
                }
            carry_tok += tot[0];
            carry_need += tot[1];
            __syncthreads();
        }
    }
    if (fill)
        for (int t = total + tid; t < a.max_tokens; t += nt) {
            a.slots[t] = -1;
            if (a.positions) a.positions[t] = 0;
        }
}

// The slot map for many tokens: one thread per token.  The CTA's first and last token are located in the row starts
// first, so that the threads search a few rows instead of all.
__global__ void __launch_bounds__(kFillThreads)
slots_fill_kernel(const ps_slots_args a) {
    __shared__ int range[2];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int32_t total = __ldcg(a.token_start + a.batch);
    const int64_t t0 = (int64_t)blockIdx.x * kFillThreads;
    const int64_t t = t0 + threadIdx.x;
    if (t0 < total && threadIdx.x < 2)
        range[threadIdx.x] = row_of(a.token_start, a.batch, threadIdx.x ? (int)min((int64_t)total - 1, t0 + kFillThreads - 1) : (int)t0);
    __syncthreads();
    if (t >= a.max_tokens) return;
    int64_t slot = -1;
    int32_t p = 0;
    if (t < total) {
        const int first = range[0];
        const int b = first + row_of(a.token_start + first, range[1] - first + 1, (int)t);
        p = a.ctx_lens_out[b] - (a.token_start[b + 1] - (int32_t)t);
        const int32_t blk = p / a.block_size;
        const int32_t id = a.block_tables[(int64_t)b * a.table_stride + blk];
        if ((unsigned)id < (unsigned)a.num_gpu_blocks)
            slot = (int64_t)id * a.block_size + (p - blk * a.block_size);
        else if (a.status_word)
            *(volatile int32_t*)a.status_word = kStatusBadId;
    }
    a.slots[t] = slot;
    if (a.positions) a.positions[t] = p;
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
    const bool fill = a.max_tokens <= kFillInPlan;
    // few rows and tokens: fewer warps make the barriers of the scan cheaper
    const int threads = a.batch <= 256 && (!fill || a.max_tokens <= 1024) ? 256 : kMaxThreads;
    cudaError_t e = ps::launch_dependent(slots_plan_kernel, dim3(1), dim3(threads), 0, s, a, (int32_t)fill);
    if (e == cudaSuccess && !fill)
        e = ps::launch_dependent(slots_fill_kernel, dim3((unsigned)((a.max_tokens + (int64_t)kFillThreads - 1) / kFillThreads)),
                                 dim3(kFillThreads), 0, s, a);
    if (e != cudaSuccess) return ps::launch_fail(err_buf, err_cap, "ps_build_slots", e);
    return PS_OK;
}

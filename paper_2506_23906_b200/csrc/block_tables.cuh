// Block tables and slot maps of a packed batch, from the requests' lengths.
//
// Two exclusive sums over the requests (tokens added, blocks added), then one independent look-up per new token: its
// request is found by bisection in the token sums, its block is either held (read from the table) or new (read from
// the free list at the request's sum of new blocks), so that no token waits for another's table entry; the token that
// opens a block writes the entry.
//
// What bounds it: latency.  A decoding step of 256 requests moves a few KB, a million new tokens 8 MB.  So there is one
// launch: every CTA forms both sums for itself in shared memory (8 bytes per request, from the L2) and then
// serves its own tokens: one per thread as long as that fits the SMs (a thread's tokens wait for each other's table
// entries: 256 requests of one token 3.7 against 6.8 us, 8192 of 18 tokens 13.5 against 16.9; from 10^6 tokens on both take the same), then eight consecutive ones, of which only the first is searched for.  Beyond TABLES_FUSED_MAX requests the
// sums no longer fit shared memory and one CTA leaves them in global memory for a second kernel (for fewer the one launch is
// always the faster: 6.9 against 9.8 us for 256 requests of one token each).  Where the totals go over the past or the added lengths
// and several kernels or CTAs read those, one more kernel writes them at the end.
#pragma once
#include <cstdint>
#include "common.cuh"

namespace mmv {

constexpr int TABLES_THREADS = 1024;
constexpr int TABLES_FUSED_MAX = 8192;

struct TablesParams {
    const int32_t *past, *added, *free_blocks;
    int32_t *table, *offsets, *total, *used;                         // total null: left to block_tables_total_kernel
    int64_t* slots;
    long long nfree, table_stride, nslots;
    int nreq, block_size;
    long long max_blocks;
    int32_t* base;                 // per-request sums of new blocks (two-kernel form only)
    int shift;                     // log2 of block_size, or -1
    WorkspaceHeader* hdr;
};
// n / block_size
__device__ __forceinline__ unsigned tables_div(const TablesParams& p, unsigned n) {
    return p.shift >= 0 ? n >> p.shift : n / static_cast<unsigned>(p.block_size);
}

struct TablesLen {
    int past, added, total;
    unsigned had, need;
    bool bad;
};
__device__ __forceinline__ TablesLen tables_len(const TablesParams& p, int r) {
    TablesLen x;
    x.past = p.past[r];
    x.added = p.added[r];
    x.bad = x.past < 0 || x.added < 0;
    x.past = max(x.past, 0);
    x.added = max(x.added, 0);
    if (x.added > INT32_MAX - x.past) {
        x.added = INT32_MAX - x.past;
        x.bad = true;
    }
    x.total = x.past + x.added;
    const unsigned b = static_cast<unsigned>(p.block_size);
    // (ceil of an int32 by an int32, in unsigned arithmetic: no overflow)
    x.need = tables_div(p, static_cast<unsigned>(x.total) + b - 1u);
    x.had = tables_div(p, static_cast<unsigned>(x.past) + b - 1u);
    return x;
}

// Exclusive sums over all requests into off[0..nreq] and base[0..nreq) (shared or global memory) by one CTA; `keep`, if not
// null, gets the requests' past lengths, and p.total is written if `totals`.
// The token sum is carried in 64 bits and stored cut to int32; the block sum is at most the token sum.
// Returns the number of new blocks; sets `code` (thread-wise) to what is wrong with the lengths.
__device__ __forceinline__ long long tables_scan(const TablesParams& p, int32_t* off, int32_t* base, int32_t* keep, bool totals, long long& tokens, unsigned& code) {
    __shared__ long long s_a[TABLES_THREADS / 32], s_b[TABLES_THREADS / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    long long run_a = 0, run_b = 0;
    for (int r0 = 0; r0 < p.nreq; r0 += TABLES_THREADS) {
        const int r = r0 + tid;
        long long a = 0, b = 0;
        if (r < p.nreq) {
            const TablesLen x = tables_len(p, r);
            a = x.added;
            if (keep) keep[r] = x.past;
            if (totals) p.total[r] = x.total;
            b = x.need - x.had;
            if (x.bad) code = code ? code : 4u;                                       // MMV_ERR_BAD_SEGMENTS
            if (x.need > p.max_blocks && a > 0)                                       // (the last new token's block, new or held, is past the row)
                code = code ? code : 7u;                                              // MMV_ERR_OUT_OF_BLOCKS
        }
        long long ia = a, ib = b;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long ta = __shfl_up_sync(0xffffffffu, ia, o), tb = __shfl_up_sync(0xffffffffu, ib, o);
            if (lane >= o) { ia += ta; ib += tb; }
        }
        if (lane == 31) { s_a[warp] = ia; s_b[warp] = ib; }
        __syncthreads();
        if (warp == 0) {
            long long wa = s_a[lane], wb = s_b[lane];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long ta = __shfl_up_sync(0xffffffffu, wa, o), tb = __shfl_up_sync(0xffffffffu, wb, o);
                if (lane >= o) { wa += ta; wb += tb; }
            }
            s_a[lane] = wa;
            s_b[lane] = wb;
        }
        __syncthreads();
        const long long before_a = run_a + (warp ? s_a[warp - 1] : 0) + ia - a, before_b = run_b + (warp ? s_b[warp - 1] : 0) + ib - b;
        if (r < p.nreq) {
            off[r] = static_cast<int32_t>(min(before_a, static_cast<long long>(INT32_MAX)));
            base[r] = static_cast<int32_t>(min(before_b, static_cast<long long>(INT32_MAX)));
        }
        run_a += s_a[TABLES_THREADS / 32 - 1];
        run_b += s_b[TABLES_THREADS / 32 - 1];
        __syncthreads();
    }
    if (tid == 0) off[p.nreq] = static_cast<int32_t>(min(run_a, static_cast<long long>(INT32_MAX)));
    tokens = run_a;
    return run_b;
}

// The status word: what a thread of CTA 0 found in the lengths, or in the sums.
__device__ __forceinline__ void tables_status(const TablesParams& p, unsigned code, long long tokens, long long fresh) {
    __shared__ unsigned s_code[2];
    if (threadIdx.x < 2) s_code[threadIdx.x] = 0u;
    __syncthreads();
    if (code) s_code[code == 4u ? 0 : 1] = code;       // (one value per place: the order of the writes does not matter)
    __syncthreads();
    if (threadIdx.x == 0) {
        unsigned e = s_code[0] ? s_code[0] : s_code[1];
        if (!e && (fresh > p.nfree || tokens > p.nslots)) e = 7u;
        if (tokens > INT32_MAX) e = 4u;
        p.hdr->tile_counter = 0u;
        p.hdr->error = e;
        *p.used = static_cast<int32_t>(min(min(fresh, p.nfree), static_cast<long long>(INT32_MAX)));
    }
}

// slots[t0 .. t0 + TOKENS) and the table entries that open with these tokens.
template <int TOKENS>
__device__ __forceinline__ void tables_expand(const TablesParams& p, const int32_t* off, const int32_t* base, const int32_t* pasts, long long t0) {
    if (t0 >= p.nslots) return;
    const int tokens = off[p.nreq];
    int64_t out[TOKENS];
#pragma unroll
    for (int i = 0; i < TOKENS; ++i) out[i] = -1;
    if (t0 < tokens) {
        // last request with off[r] <= t0 (empty requests in front of it share its offset)
        int lo = 0, hi = p.nreq;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (off[mid] <= t0) lo = mid;
            else hi = mid;
        }
        int r = lo, begin = 0, end = 0, had = 0;
        unsigned q = 0, rem = 0;
        const unsigned bs = static_cast<unsigned>(p.block_size);
        long long first = 0;
        int id = -1;
        bool fresh_block = false;
        const auto enter = [&](int t) {             // request r, whose token t is next
            begin = off[r];
            end = off[r + 1];
            const int past = max(pasts[r], 0);
            had = static_cast<int>(tables_div(p, static_cast<unsigned>(past) + bs - 1u));
            first = base[r];
            const unsigned pos = static_cast<unsigned>(past + (t - begin));
            q = tables_div(p, pos);
            rem = pos - q * bs;
        };
        const auto block = [&] {                    // the id of request r's block q
            id = -1;
            fresh_block = false;
            if (q >= p.max_blocks) return;
            if (q < static_cast<unsigned>(had)) {
                id = p.table[r * p.table_stride + q];
            } else {
                const long long at = first + (q - static_cast<unsigned>(had));
                fresh_block = at < p.nfree;
                if (fresh_block) id = p.free_blocks[at];
            }
        };
        enter(static_cast<int>(t0));
        block();
#pragma unroll
        for (int i = 0; i < TOKENS; ++i) {
            const long long t = t0 + i;
            if (t < tokens && t < p.nslots) {
                if (t >= end) {
                    do ++r; while (off[r + 1] <= t);        // (off[nreq] = tokens > t ends it)
                    enter(static_cast<int>(t));
                    block();
                } else if (rem == bs) {
                    rem = 0;
                    ++q;
                    block();
                }
                if (rem == 0 && fresh_block) p.table[r * p.table_stride + q] = id;
                out[i] = id < 0 ? -1 : static_cast<int64_t>(id) * bs + rem;
                ++rem;
            }
        }
    }
    int64_t* dst = p.slots + t0;
    if (TOKENS % 2 == 0 && t0 + TOKENS <= p.nslots && (reinterpret_cast<uintptr_t>(dst) & 15u) == 0) {
#pragma unroll
        for (int i = 0; i + 1 < TOKENS; i += 2)
            *reinterpret_cast<longlong2*>(dst + i) = make_longlong2(out[i], out[i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < TOKENS; ++i)
            if (t0 + i < p.nslots) dst[i] = out[i];
    }
}

// A block that a dropped token (past nslots) would have opened stays out of the table; so does its request's tail.
template <int TOKENS>
__global__ void __launch_bounds__(TABLES_THREADS) block_tables_kernel(TablesParams p) {
    extern __shared__ int32_t tables_smem[];
    int32_t* off = tables_smem;
    int32_t* base = off + p.nreq + 1;
    int32_t* pasts = base + p.nreq;
    long long tokens;
    unsigned code = 0u;
    const long long fresh = tables_scan(p, off, base, pasts, blockIdx.x == 0 && p.total, tokens, code);
    __syncthreads();
    for (long long t0 = static_cast<long long>(blockIdx.x) * TABLES_THREADS * TOKENS; t0 < p.nslots; t0 += static_cast<long long>(gridDim.x) * TABLES_THREADS * TOKENS)
        tables_expand<TOKENS>(p, off, base, pasts, t0 + threadIdx.x * TOKENS);
    if (blockIdx.x == 0) {
        for (int r = threadIdx.x; r <= p.nreq; r += TABLES_THREADS) p.offsets[r] = off[r];
        tables_status(p, code, tokens, fresh);
    }
}

// Many requests: the sums by one CTA, in global memory ...
__global__ void __launch_bounds__(TABLES_THREADS) block_tables_scan_kernel(TablesParams p) {
    griddep_launch_dependents();
    long long tokens;
    unsigned code = 0u;
    const long long fresh = tables_scan(p, p.offsets, p.base, nullptr, p.total != nullptr, tokens, code);
    tables_status(p, code, tokens, fresh);
}
// ... and the look-ups by all.
template <int TOKENS>
__global__ void __launch_bounds__(TABLES_THREADS) block_tables_expand_kernel(TablesParams p) {
    griddep_wait();
    for (long long t0 = static_cast<long long>(blockIdx.x) * TABLES_THREADS * TOKENS; t0 < p.nslots; t0 += static_cast<long long>(gridDim.x) * TABLES_THREADS * TOKENS)
        tables_expand<TOKENS>(p, p.offsets, p.base, p.past, t0 + threadIdx.x * TOKENS);
}
// The totals, in place of the lengths that they are made of.
__global__ void __launch_bounds__(TABLES_THREADS) block_tables_total_kernel(TablesParams p, int32_t* total) {
    const int r = blockIdx.x * TABLES_THREADS + threadIdx.x;
    if (r < p.nreq) total[r] = tables_len(p, r).total;
}

}  // namespace mmv

// Attention of one new token per request over a paged key-value cache.
//
//     s_j = scale q . k_j for the tokens j in [max(0, len - window), len);  out = sum_j softmax(s)_j v_j;  lse = log sum_j exp s_j
//
// What bounds it: the cache is read once, 4 dim bytes per token and key head against 4 dim flops per token and QUERY
// head, so HBM, as long as the query heads of a group share one read.  The up to 16 query heads of a key head are the
// rows of an m16n8k16 product (one such product per token and pass: a few percent of its rate); more than 16 are served in
// parts that follow each other closely, the second read coming from the L2.
//
// Split: the work is the list of (request, key head, tile of PA_TILE tokens) in this order, cut into equal contiguous
// ranges, one per CTA, whatever the lengths: a long context is spread over many CTAs, short ones share one.  A
// (request, head) that lies inside one range is finished there; one that is cut leaves a partial (running maximum, sum,
// unnormalised result) per range, and a second small kernel joins them in order: results do not depend on timing.
//
// Inside a CTA each of the four warps owns 16 of a tile's 64 tokens and keeps its own running maximum, sum and result
// (one pass, softmax in the base-2 exponent), so that warps meet only where a (request, head) ends.  Every warp
// fetches its own tokens with 16-byte asynchronous copies, PA_STAGES tiles ahead and across the ends of requests: nothing but the
// warp waits for them.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "common.cuh"

namespace mmv {

constexpr int PA_WARPS = 4;
constexpr int PA_THREADS = PA_WARPS * 32;
constexpr int PA_TOKENS = 16;                            // tokens of a warp in one tile
constexpr int PA_TILE = PA_WARPS * PA_TOKENS;
constexpr int PA_STAGES = 2;
constexpr int PA_ROWS = 16;                              // query heads of one product

struct PagedParams {
    const uint16_t *q, *k, *v;
    long long q_req, q_head;
    long long c_block, c_tok, c_head;
    const int32_t *table, *lens;
    long long table_stride, capacity;                    // capacity = max_blocks * block_size tokens (cut to int32)
    long long num_blocks;
    long long window;                                    // 0: none
    int nreq, block_size, dim, heads, kv_heads, group;   // group = query heads per key head
    int parts, rows;                                     // groups of `rows` query heads per key head
    float scale_log2;                                    // scale * log2(e)
    uint16_t* out;                                       // [request, heads, dim]
    float* lse;                                          // [request, heads] or null
    // workspace
    WorkspaceHeader* hdr;
    int32_t* desc;                                       // [grid][4]: joined (request, head part) or -1, last CTA of it, error code
    float* part_ml;                                      // [grid][2][2][PA_ROWS]: maximum (less the kernel's LIFT), sum
    float* part_o;                                       // [grid][2][rows][dim]
};

// request r's tokens [begin, len) and its number of tiles; tiles start at a multiple of PA_TOKENS
struct PagedSpan {
    int begin, len, first, tiles;
    bool bad;
};
__device__ __forceinline__ PagedSpan paged_span(const PagedParams& p, int r) {
    PagedSpan s;
    const int len = p.lens[r];
    s.bad = len < 0 || len > p.capacity;
    s.len = static_cast<int>(min(static_cast<long long>(max(len, 0)), p.capacity));
    s.begin = (p.window > 0 && p.window < s.len) ? s.len - static_cast<int>(p.window) : 0;
    s.first = s.begin & ~(PA_TOKENS - 1);
    s.tiles = s.len > 0 ? static_cast<int>((static_cast<unsigned>(s.len - s.first) + PA_TILE - 1) / PA_TILE) : 0;
    return s;
}

// 2^x for x <= 0 in one instruction (2 units in the last place, as exp2f; results under 2^-126 are 0)
__device__ __forceinline__ float paged_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// first unit of CTA c's range, and the CTA whose range holds unit u (ranges [c W / G, (c + 1) W / G))
__device__ __forceinline__ long long paged_first(long long c, long long units, int ctas) { return c * units / ctas; }
__device__ __forceinline__ int paged_cta_of(long long u, long long units, int ctas) { return static_cast<int>(((u + 1) * ctas - 1) / units); }

__device__ __forceinline__ void cp_async_16_or_zero(uint32_t dst, const void* src, bool on) {
    const int bytes = on ? 16 : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldsm_x4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <bool BF16>
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// two fp32 values -> packed 16-bit pair (a in the low half), and what the rounding left of each
template <bool BF16>
__device__ __forceinline__ uint32_t pack_pair(float a, float b) {
    if constexpr (BF16) {
        const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&x);
    } else {
        const __half2 x = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&x);
    }
}
template <bool BF16>
__device__ __forceinline__ float2 unpack_pair(uint32_t w) {
    if constexpr (BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    else return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

template <int DP>
struct PagedCfg {
    static constexpr int kRow = DP * 2;                                        // bytes of a token's row
    static constexpr int kChunks = DP / 8;                                     // 16-byte words of it
    static constexpr int kStage = PA_TOKENS * kRow * 2;                        // keys and values of a warp's tokens
    static constexpr int kQ = PA_ROWS * kRow;
    static constexpr int kQSlots = PA_STAGES + 1;
    static constexpr int kPitch = DP + 8;                                      // floats of a row where warps meet
    static constexpr int kStages = PA_WARPS * PA_STAGES * kStage;
    static int smem_bytes(int rows) { return kStages + kQSlots * kQ + PA_WARPS * rows * kPitch * 4; }
};

// Where a walk over the units of a range stands.
struct PagedIter {
    int r, hp, tile, tiles;          // request; key head and part of it (hp = head * parts + part); tile of it
    int begin, len, first;
};
__device__ __forceinline__ void paged_enter(const PagedParams& p, PagedIter& it) {
    const PagedSpan s = paged_span(p, it.r);
    it.begin = s.begin;
    it.len = s.len;
    it.first = s.first;
    it.tiles = s.tiles;
}
// the next unit (the caller knows that there is one); true where a new (request, head part) begins
__device__ __forceinline__ bool paged_next(const PagedParams& p, PagedIter& it) {
    if (++it.tile < it.tiles) return false;
    it.tile = 0;
    if (++it.hp == p.kv_heads * p.parts) {
        it.hp = 0;
        do {
            ++it.r;
            paged_enter(p, it);
        } while (it.tiles == 0);
    }
    return true;
}

// SMALL: up to 8 query heads per key head.  Their rows fill half of the product; the other half takes what rounding the
// weights to 16 bits left of them, so that one product does for both (4 requests of 131072 tokens, 32/8 heads of 128: 386 -> 340 us; 64 requests
// of up to 4096: 119 -> 98 us; both sides on one GPU, others take up to a tenth more).
template <bool BF16, int DP, bool SMALL>
__global__ void __launch_bounds__(PA_THREADS) paged_attention_kernel(const PagedParams p) {
    using C = PagedCfg<DP>;
    constexpr int HALVES = SMALL ? 1 : 2;                             // of the 16 rows that hold query heads
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long s_sum[PA_WARPS];
    __shared__ int s_start[2];
    __shared__ long long s_skip;
    __shared__ float s_m[PA_WARPS][PA_ROWS], s_l[PA_WARPS][PA_ROWS];
    // The exponent that the largest weight gets.  fp16 holds nothing under 2^-24: a pair of values that starts at 2^15 reaches 2^-40 of the
    // largest weight, one that starts at 1 would lose all under 2^-25 of it.  bfloat16 has the range of fp32.
    constexpr float LIFT = BF16 ? 0.f : 15.f;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    griddep_launch_dependents();

    // ---- the range: units of all requests, and where this CTA's first one lies -------------------------------------
    const int per = (p.nreq + PA_THREADS - 1) / PA_THREADS, r_lo = min(p.nreq, tid * per), r_hi = min(p.nreq, r_lo + per);
    const long long heads = static_cast<long long>(p.kv_heads) * p.parts;
    long long mine = 0;
    bool bad = false;
    for (int r = r_lo; r < r_hi; ++r) {
        const PagedSpan s = paged_span(p, r);
        mine += s.tiles;
        bad |= s.bad;
    }
    long long inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
    }
    if (lane == 31) s_sum[warp] = inc;
    const bool any_bad = __syncthreads_or(bad);
    long long before = inc - mine, total = 0;
#pragma unroll
    for (int w = 0; w < PA_WARPS; ++w) {
        if (w < warp) before += s_sum[w];
        total += s_sum[w];
    }
    const long long units = total * heads;
    const int ctas = static_cast<int>(min(static_cast<long long>(gridDim.x), units));     // (no range is empty)
    const bool idle = static_cast<int>(blockIdx.x) >= ctas;
    const long long u0 = idle ? 0 : paged_first(blockIdx.x, units, ctas), u1 = idle ? 0 : paged_first(blockIdx.x + 1ll, units, ctas);
    int32_t* desc = p.desc + 4 * blockIdx.x;
    if (tid == 0) {
        desc[0] = -1;
        desc[2] = any_bad ? 1 : 0;                                    // MMV_ERR_INVALID_ARG
    }
    if (idle) return;
    if (u0 >= before * heads && u0 < (before + mine) * heads) {       // one thread's requests hold unit u0
        long long at = before * heads;
        int r = r_lo;
        long long n = paged_span(p, r).tiles * heads;
        while (u0 >= at + n) {
            at += n;
            n = paged_span(p, ++r).tiles * heads;
        }
        s_start[0] = r;
        s_skip = u0 - at;
    }
    __syncthreads();

    PagedIter ld;                                                     // the tile to fetch next
    ld.r = s_start[0];
    paged_enter(p, ld);
    ld.hp = static_cast<int>(s_skip / ld.tiles);
    ld.tile = static_cast<int>(s_skip - static_cast<long long>(ld.hp) * ld.tiles);
    PagedIter it = ld;                                                // the tile to work on next
    const bool cut_front = it.tile > 0;                               // the first (request, head) began in an earlier range

    const uint32_t sm = smem_u32(smem);
    const uint32_t sm_stage = sm + warp * PA_STAGES * C::kStage;
    const uint32_t sm_q = sm + C::kStages;
    float* sm_o = reinterpret_cast<float*>(smem + C::kStages + C::kQSlots * C::kQ);
    const int words = p.dim / 8;

    // ---- fetch of a tile: 16 tokens' keys and values per warp; with a new head the query rows too -----------------------
    int seg_ld = 0;
    const auto fetch_q = [&] {
        const int head = ld.hp / p.parts, part = ld.hp - head * p.parts;
        const int rows = min(p.rows, p.group - part * p.rows);
        const uint16_t* src = p.q + ld.r * p.q_req + (head * p.group + part * p.rows) * p.q_head;
        const uint32_t dst = sm_q + (seg_ld % C::kQSlots) * C::kQ;
        for (int i = tid; i < PA_ROWS * C::kChunks; i += PA_THREADS) {
            const int row = i / C::kChunks, c = i - row * C::kChunks;
            const bool on = row < rows && c < words;
            cp_async_16_or_zero(dst + row * C::kRow + ((c ^ (row & 7)) << 4), on ? src + row * p.q_head + c * 8 : p.q, on);
        }
        ++seg_ld;
    };
    const auto fetch = [&](int stage) {
        const int head = ld.hp / p.parts;
        const int tok = ld.first + ld.tile * PA_TILE + warp * PA_TOKENS + (lane & 15);
        long long at = -1;
        if (tok >= ld.begin && tok < ld.len) {
            const unsigned b = static_cast<unsigned>(tok) / static_cast<unsigned>(p.block_size);
            const int page = p.table[ld.r * p.table_stride + b];
            if (page >= 0 && page < p.num_blocks)
                at = page * p.c_block + static_cast<long long>(tok - b * p.block_size) * p.c_tok + head * p.c_head;
            else
                desc[2] = 1;                                          // (every writer stores the same value)
        }
        const uint32_t dst = sm_stage + stage * C::kStage;
        constexpr int kPerRow = C::kChunks < 32 ? C::kChunks : 32;    // lanes on one row
        constexpr int kRows = 32 / kPerRow;
#pragma unroll
        for (int i = 0; i < PA_TOKENS / kRows; ++i) {
            const int row = i * kRows + lane / kPerRow, c = lane % kPerRow;
            const long long a = __shfl_sync(0xffffffffu, at, row);
            const bool on = a >= 0 && c < words;
            const uint32_t d = dst + row * C::kRow + ((c ^ (row & 7)) << 4);
            cp_async_16_or_zero(d, on ? p.k + a + c * 8 : p.q, on);
            cp_async_16_or_zero(d + PA_TOKENS * C::kRow, on ? p.v + a + c * 8 : p.q, on);
        }
    };
    long long u_ld = u0;
    bool fresh = true;                                                // the next tile to fetch begins a head

    uint32_t qf[DP / 16][4];
    float o[DP / 8][4];
    float m[2], l[2];                                                 // maximum less LIFT; sum of weights 2^(s - m)
    int seg = 0, stage = 0;
    bool begins = true;
    // (The first PA_STAGES turns only fetch: with one place in the code that does, its loop fits the instruction cache.)
#pragma unroll 1
    for (long long u = u0 - PA_STAGES; u < u1; ++u) {
        cp_async_wait<PA_STAGES - 1>();
        __syncwarp();
        if (begins && u >= u0) {
            __syncthreads();                                          // every warp's share of the query rows has landed
            const uint32_t src = sm_q + (seg % C::kQSlots) * C::kQ;
            const int row = lane & 15;
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) ldsm_x4(qf[d], src + row * C::kRow + (((2 * d + (lane >> 4)) ^ (row & 7)) << 4));
#pragma unroll
            for (int n = 0; n < DP / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
            m[0] = m[1] = -INFINITY;
            l[0] = l[1] = 0.f;
            ++seg;
        }
        const int tok0 = it.first + it.tile * PA_TILE + warp * PA_TOKENS;
        if (u >= u0 && tok0 < it.len) {
            const uint32_t kb = sm_stage + stage * C::kStage, vb = kb + PA_TOKENS * C::kRow;
            float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
            {
                // lanes 0-7: tokens 0-7, first 8 columns; 8-15: the next 8 columns; 16-31: tokens 8-15
                const int row = (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
                for (int d = 0; d < DP / 16; ++d) {
                    uint32_t b[4];
                    ldsm_x4(b, kb + row * C::kRow + (((2 * d + ((lane >> 3) & 1)) ^ (row & 7)) << 4));
                    mma_16816<BF16>(s[0], qf[d], b[0], b[1]);
                    mma_16816<BF16>(s[1], qf[d], b[2], b[3]);
                }
            }
            const bool edge = tok0 < it.begin || tok0 + PA_TOKENS > it.len;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 2 * HALVES; ++i) {
                    s[n][i] *= p.scale_log2;
                    if (edge) {
                        const int tok = tok0 + n * 8 + (lane & 3) * 2 + (i & 1);
                        if (tok < it.begin || tok >= it.len) s[n][i] = -INFINITY;
                    }
                }
            uint32_t hi[4], lo[4];                                    // (SMALL: the low parts are hi[1] and hi[3], rows 8 to 15)
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {                        // rows lane / 4 and lane / 4 + 8
                float top = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                // (From 2^23 on fp32 does not hold every such difference: rounded up there, so that no weight passes 2^15.)
                const float low = !BF16 && fabsf(top) >= 8388608.f ? __fadd_ru(top, -LIFT) : top - LIFT;
                const float now = fmaxf(m[h], low);
                const float base = now == -INFINITY ? 0.f : now;      // (no token yet: every weight is 2^-inf = 0)
                const float fall = paged_exp2(m[h] - base);
                m[h] = now;
                float sum = 0.f;
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const float a = paged_exp2(s[n][2 * h] - base), b = paged_exp2(s[n][2 * h + 1] - base);
                    sum += a + b;
                    // The weights enter the product as the sum of two 16-bit values (2^-16 of themselves, in fp16 at least 2^-40 of the
                    // largest): rounded to one, their error would be as large as the result's own rounding.
                    hi[n * 2 + h] = pack_pair<BF16>(a, b);
                    const float2 back = unpack_pair<BF16>(hi[n * 2 + h]);
                    (SMALL ? hi[n * 2 + 1] : lo[n * 2 + h]) = pack_pair<BF16>(a - back.x, b - back.y);
                }
                l[h] = l[h] * fall + sum;
                if (__any_sync(0xffffffffu, fall != 1.f)) {           // (the maximum of a long context soon stands)
#pragma unroll
                    for (int n = 0; n < DP / 8; ++n) {
                        o[n][2 * h] *= fall;
                        o[n][2 * h + 1] *= fall;
                        if (SMALL) {
                            o[n][2] *= fall;
                            o[n][3] *= fall;
                        }
                    }
                }
            }
            {
                const int row = lane & 15;
#pragma unroll
                for (int d = 0; d < DP / 16; ++d) {
                    uint32_t b[4];
                    ldsm_x4_t(b, vb + row * C::kRow + (((2 * d + (lane >> 4)) ^ (row & 7)) << 4));
                    mma_16816<BF16>(o[2 * d], hi, b[0], b[1]);
                    mma_16816<BF16>(o[2 * d + 1], hi, b[2], b[3]);
                    if (!SMALL) {
                        mma_16816<BF16>(o[2 * d], lo, b[0], b[1]);
                        mma_16816<BF16>(o[2 * d + 1], lo, b[2], b[3]);
                    }
                }
            }
        }
        __syncwarp();                                                 // the stage has been read by all lanes
        if (u_ld < u1) {
            if (fresh) fetch_q();
            fetch(stage);
            if (++u_ld < u1) fresh = paged_next(p, ld);
        }
        cp_async_commit();
        stage = stage + 1 == PA_STAGES ? 0 : stage + 1;
        if (u < u0) continue;

        const PagedIter done = it;
        const bool ends = it.tile + 1 == it.tiles;                    // of this (request, head part)
        begins = ends;
        const bool last = u + 1 == u1;
        if (!last) paged_next(p, it);
        if (!ends && !last) continue;

        // ---- the warps meet --------------------------------------------------------------------------------------------
        const int head = done.hp / p.parts, part = done.hp - head * p.parts;
        const int rows = min(p.rows, p.group - part * p.rows);
        if (SMALL)
#pragma unroll
            for (int n = 0; n < DP / 8; ++n) {
                o[n][0] += o[n][2];
                o[n][1] += o[n][3];
            }
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
            const int row = (lane >> 2) + 8 * h;
            if ((lane & 3) == 0) {
                s_m[warp][row] = m[h];
                s_l[warp][row] = l[h];
            }
        }
        __syncthreads();
        float top[2];
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            const int row = (lane >> 2) + 8 * h;
            top[h] = s_m[0][row];
#pragma unroll
            for (int w = 1; w < PA_WARPS; ++w) top[h] = fmaxf(top[h], s_m[w][row]);
            // (a warp without tokens has maximum -infinity, sum 0 and result 0, and contributes 2^-inf = 0 times that; a NaN stays one)
            const float f = paged_exp2(m[h] - (top[h] == -INFINITY ? 0.f : top[h]));
            if (row < rows) {
#pragma unroll
                for (int n = 0; n < DP / 8; ++n)
                    *reinterpret_cast<float2*>(sm_o + (warp * p.rows + row) * C::kPitch + n * 8 + (lane & 3) * 2) =
                        make_float2(o[n][2 * h] * f, o[n][2 * h + 1] * f);
            }
        }
        __syncthreads();
        const bool began_here = !(cut_front && seg == 1);
        const bool whole = began_here && ends;
        const long long place = 2ll * blockIdx.x + (began_here ? 1 : 0);
        for (int i = tid; i < rows * (DP / 4); i += PA_THREADS) {
            const int row = i / (DP / 4), c = (i - row * (DP / 4)) * 4;
            float t = s_m[0][row];
#pragma unroll
            for (int w = 1; w < PA_WARPS; ++w) t = fmaxf(t, s_m[w][row]);
            float sum = 0.f;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < PA_WARPS; ++w) {
                sum += s_l[w][row] * paged_exp2(s_m[w][row] - (t == -INFINITY ? 0.f : t));
                const float4 y = *reinterpret_cast<const float4*>(sm_o + (w * p.rows + row) * C::kPitch + c);
                x.x += y.x;
                x.y += y.y;
                x.z += y.z;
                x.w += y.w;
            }
            const long long orow = done.r * static_cast<long long>(p.heads) + head * p.group + part * p.rows + row;
            if (whole) {
                const float inv = sum == 0.f ? 0.f : 1.f / sum;       // (every weight 0: the result is 0)
                if (c < p.dim)
                    *reinterpret_cast<uint2*>(p.out + orow * p.dim + c) =
                        make_uint2(pack_pair<BF16>(x.x * inv, x.y * inv), pack_pair<BF16>(x.z * inv, x.w * inv));
                if (c == 0 && p.lse) p.lse[orow] = sum == 0.f ? -INFINITY : (t + log2f(sum)) * 0.69314718055994531f;
            } else {
                if (c < p.dim) *reinterpret_cast<float4*>(p.part_o + (place * p.rows + row) * p.dim + c) = x;
                if (c == 0) {
                    p.part_ml[(place * 2) * PA_ROWS + row] = t;
                    p.part_ml[(place * 2 + 1) * PA_ROWS + row] = sum;
                }
            }
        }
        if (!whole && began_here && tid == 0) {                       // this range joins it; its last unit lies in a later one
            desc[0] = static_cast<int32_t>(done.r);
            desc[1] = static_cast<int32_t>(paged_cta_of(u + (done.tiles - 1 - done.tile), units, ctas));
            desc[3] = done.hp;
        }
        __syncthreads();
    }
}

// Joins the partials of the (request, head part) that begins in range blockIdx.x and is cut at its end: one row (query
// head) per CTA.  Also the requests without tokens and the status word.
constexpr int PA_JOIN_THREADS = 128;

template <bool BF16>
__global__ void __launch_bounds__(PA_JOIN_THREADS) paged_join_kernel(const PagedParams p, int ctas) {
    __shared__ float s_w[PA_JOIN_THREADS], s_red[4];
    __shared__ float4 s_x[PA_JOIN_THREADS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = blockIdx.y;
    griddep_wait();
    if (row == 0) {
        for (int r = blockIdx.x; r < p.nreq; r += gridDim.x) {        // nothing to attend to: 0, and the logarithm of an empty sum
            if (paged_span(p, r).tiles) continue;
            for (long long i = tid; i < static_cast<long long>(p.heads) * p.dim; i += PA_JOIN_THREADS) p.out[r * static_cast<long long>(p.heads) * p.dim + i] = 0;
            if (p.lse)
                for (int i = tid; i < p.heads; i += PA_JOIN_THREADS) p.lse[r * static_cast<long long>(p.heads) + i] = -INFINITY;
        }
        if (blockIdx.x == 0) {
            int e = 0;
            for (int i = tid; i < ctas; i += PA_JOIN_THREADS) e |= p.desc[4 * i + 2];
            e = __syncthreads_or(e);
            if (tid == 0) {
                p.hdr->tile_counter = 0u;
                p.hdr->error = e ? 1u : 0u;
            }
        }
    }
    const int32_t* desc = p.desc + 4 * blockIdx.x;
    const int r = desc[0];
    if (r < 0) return;
    const int last = desc[1], hp = desc[3], head = hp / p.parts, part = hp - head * p.parts;
    if (row >= min(p.rows, p.group - part * p.rows)) return;
    const int first = blockIdx.x, n = last - first + 1;
    const auto place = [&](int i) { return 2ll * (first + i) + (i == 0 ? 1 : 0); };
    // maximum, then the weights' sum
    float top = -INFINITY;
    for (int i = tid; i < n; i += PA_JOIN_THREADS) top = fmaxf(top, p.part_ml[place(i) * 2 * PA_ROWS + row]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) s_red[warp] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
    __syncthreads();
    const int cols = p.dim / 4, lanes = cols <= 32 ? 32 : 64, groups = PA_JOIN_THREADS / lanes;
    const int g = tid / lanes, c = tid - g * lanes;
    float sum = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0; i0 < n; i0 += PA_JOIN_THREADS) {                 // (in order: the same result every time)
        const int i = i0 + tid;
        float w = 0.f;
        if (i < n) {
            const float mi = p.part_ml[place(i) * 2 * PA_ROWS + row], li = p.part_ml[(place(i) * 2 + 1) * PA_ROWS + row];
            w = paged_exp2(mi - (top == -INFINITY ? 0.f : top));
            sum += w * li;
        }
        s_w[tid] = w;
        __syncthreads();
        if (c < cols)
            for (int j = g; j < min(PA_JOIN_THREADS, n - i0); j += groups) {
                const float f = s_w[j];
                const float4 y = *reinterpret_cast<const float4*>(p.part_o + (place(i0 + j) * p.rows + row) * p.dim + c * 4);
                x.x = fmaf(f, y.x, x.x);
                x.y = fmaf(f, y.y, x.y);
                x.z = fmaf(f, y.z, x.z);
                x.w = fmaf(f, y.w, x.w);
            }
        __syncthreads();
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) s_red[warp] = sum;
    s_x[tid] = x;
    __syncthreads();
    sum = s_red[0] + s_red[1] + s_red[2] + s_red[3];
    if (g == 0 && c < cols) {
        for (int j = 1; j < groups; ++j) {
            const float4 y = s_x[j * lanes + c];
            x.x += y.x;
            x.y += y.y;
            x.z += y.z;
            x.w += y.w;
        }
        const long long orow = r * static_cast<long long>(p.heads) + head * p.group + part * p.rows + row;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        *reinterpret_cast<uint2*>(p.out + orow * p.dim + c * 4) =
            make_uint2(pack_pair<BF16>(x.x * inv, x.y * inv), pack_pair<BF16>(x.z * inv, x.w * inv));
        if (c == 0 && p.lse) p.lse[orow] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
    }
}

}  // namespace mmv

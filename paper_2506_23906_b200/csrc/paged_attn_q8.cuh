// Attention of one new token per request over a paged key-value cache in 8 bits with a scale for each block of tokens and head.
//
//     s_j = scale (q . code^k_j) ks_j,   out = sum_j softmax(s)_j vs_j code^v_j,   lse = log sum_j exp s_j       (ks, vs: the scales of j's block)
//
// The split over CTAs and the join of cut parts are those of the attention over a 16-bit cache (paged_attn.cuh).  What differs:
//   The four warps of a CTA take two neighbouring key heads of the same tokens (where their number is even), not four times the tokens of one: a token's codes
//     of one head are 128 bytes or less, and memory answers at a lower rate where those of the next head are asked for at another time (4 requests of
//     131072 tokens, 8 heads of 128: 257 to 270 us, whatever the arithmetic, against 180).
//   Codes become fp16 in registers (every int8 and e4m3 value is one) and both products run in fp16.  A bfloat16 query is brought
//     into fp16's range by a power of two of its own row, exactly but for values 2^29 times smaller than the row's largest.
//   Both products are taken transposed: tokens (16), then columns of the result (16) are a product's rows, and up to 8 query heads its columns,
//     so that codes are the first operand as they come, and few heads cost half as many products and registers. The weights of up to
//     four heads fill the 8 columns with their high and low parts.
//   The columns of a query and of a key may be taken in any order that both share: a lane takes 16 neighbouring columns of a token's
//     key with one load, four of them for each of four products.  Values are read transposed in pairs of columns (8-bit
//     columns 2d and 2d + 1 are one 16-bit element) and taken apart by a byte permutation: the even columns are a product's first 8
//     rows, the odd ones the others.
//   Scales of values are part of the weights that meet the codes: 2^((s_j - m) + log2 vs_j - d), with a running maximum d of its own, so that no
//     scale leaves fp16's range; the weights of the sum are 2^(s_j - m).  d is counted from m: a logarithm added to the score itself would lose by
//     the score's size (of a score of 2^17 all but 7 binary places), while s_j - m is exact where the weight is large.
//
// What bounds it: HBM, 2 dim bytes per token and key head, and the instructions beside them (5 for four int8 codes).  8 key heads of 128, 32 query heads:
// 4 requests of 131072 tokens 188 us with e4m3 codes (5.7 of the 6.5 TB/s of a copy; with a cold L2 198 to 206, int8 198 to 202); 64 requests of up to 4096 70 us
// (3.9 TB/s: requests end inside tiles, warps meet there and a join follows); one of 777 12.3 us, two launches and the host's 9.6 us.  Blocks that are no
// multiple of 16 tokens (copies and scales token by token): 4 of 131072 with blocks of 24, 9, 8 204, 206, 213 us; 64 of 2048 72 us with blocks of 9, 71 with 16.
#pragma once
#include <cstdint>
#include "kv_cache_q8.cuh"
#include "paged_attn.cuh"

namespace mmv {

constexpr int Q8_TOKENS = 32;                                // of a warp in one tile: two groups of 16
constexpr float Q8_FLOOR = -1024.f;                          // the least maximum of the values' weights: 2^-1024 times anything is 0

struct PagedQ8Params : PagedParams {                         // (k and v of the base are not used)
    const uint8_t *k8, *v8;
    const float *ks, *vs;
    long long s_block, s_head;
    uint32_t by_block;                                       // floor(2^32 / block_size)
    int side;                                                // key heads side by side: 1 or 2
    int tile, groups;                                        // tokens of a unit: 128 / side; groups of key heads, times parts
    uint64_t budget_ns;                                      // bound of every wait
    long long debug_skip;                                    // test hook: the CTA that leaves out a load of each tile (-1: none)
    float* part_m2;                                          // [grid][2][side][PA_ROWS]: maximum of the values' weights, above that of the scores
};                                                           // (part_ml: [grid][2][side][2][PA_ROWS], part_o: [grid][2][side][rows][dim])

__device__ __forceinline__ PagedSpan q8_span(const PagedQ8Params& p, int r) {
    PagedSpan s = paged_span(p, r);
    s.tiles = s.len > 0 ? static_cast<int>((static_cast<unsigned>(s.len - s.first) + p.tile - 1) / static_cast<unsigned>(p.tile)) : 0;
    return s;
}
__device__ __forceinline__ void q8_enter(const PagedQ8Params& p, PagedIter& it) {
    const PagedSpan s = q8_span(p, it.r);
    it.begin = s.begin;
    it.len = s.len;
    it.first = s.first;
    it.tiles = s.tiles;
}
// the next unit (the caller knows that there is one); true where a new (request, heads) begins
__device__ __forceinline__ bool q8_next(const PagedQ8Params& p, PagedIter& it) {
    if (++it.tile < it.tiles) return false;
    it.tile = 0;
    if (++it.hp == p.groups) {
        it.hp = 0;
        do {
            ++it.r;
            q8_enter(p, it);
        } while (it.tiles == 0);
    }
    return true;
}

template <int DP, int ROWS>
struct PagedQ8Cfg {
    static constexpr int kStages = 2;
    static constexpr int kPerSm = ROWS == 16 && DP == 256 ? 2 : 3;             // CTAs that the registers allow (168 per thread)
    static constexpr int kChunks = DP / 16;                                    // 16-byte words of a token's codes
    static constexpr int kBox = DP < 128 ? DP : 128;                           // bytes of a row in shared memory: longer ones lie in two halves
    static constexpr int kGroup = 16 * DP, kKeys = 2 * kGroup;                 // of 16 tokens' keys; of a warp's, their values behind them
    static constexpr int kStage = 2 * kKeys;
    static constexpr int kScales = Q8_TOKENS * 8;
    static constexpr int kPitch = DP / 2 + 8;                                  // floats of half a row where warps meet
    static constexpr int kAll = PA_WARPS * kStages * kStage;
    static constexpr int kOOff = kAll + PA_WARPS * kStages * kScales;
    static int smem_bytes(int rows) { return kOOff + PA_WARPS * rows * kPitch * 4; }
    // Where word c of token `row` of 16 lies: eight rows' words of one column are in different banks (128-byte swizzle, 64-byte swizzle for short rows), and the
    // tokens of a product's columns n = 0 .. 7 are taken in an order in which two neighbouring ones' four words are, too.
    static __device__ __forceinline__ int place(int row, int c) {
        return DP < 128 ? row * 64 + ((c ^ ((row >> 1) & 3)) << 4) : (c >> 3) * 2048 + row * 128 + (((c & 7) ^ (row & 7)) << 4);
    }
    static __device__ __forceinline__ int token(int n) { return DP < 128 ? n : (n & 8) | ((n & 1) << 2) | ((n & 7) >> 1); }
};

// Bounded wait that sleeps in the barrier instruction (a turn of a loop that polls takes issue slots from the warps that work).
static __device__ __noinline__ bool q8_wait(uint64_t* bar, uint32_t parity, uint64_t budget_ns) {
    const uint64_t t0 = global_timer_ns();
    while (!mbar_try_wait_for(bar, parity, 20000u))
        if (global_timer_ns() - t0 > budget_ns) return false;
    return true;
}
// The loads of a stage, and of the one behind it if there are any, land before the warp gives up (1 ms each at most).
static __device__ __noinline__ void q8_land(uint64_t* bars, int stage, uint32_t turn, bool more) {
    q8_wait(&bars[stage], turn, 1000000u);
    if (more) q8_wait(&bars[stage ^ 1], stage ? turn ^ 1 : turn, 1000000u);
}
__device__ __forceinline__ void cp_async_4_or_zero(uint32_t dst, const void* src, bool on) {
    const int bytes = on ? 4 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint4 lds_128(uint32_t addr) {
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(addr) : "memory");
    return r;
}
__device__ __forceinline__ float lds_float(uint32_t addr) {
    float r;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(r) : "r"(addr) : "memory");
    return r;
}
__device__ __forceinline__ float paged_log2(float x) {
    float r;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// (a negative scale is none: NaN, as its logarithm is where it is one of values)
__device__ __forceinline__ float q8_key_scale(float x) { return x < 0.f ? __uint_as_float(0x7fc00000u) : x; }
// an 8 x 8 matrix of 16-bit values, as a product leaves its results, transposed
__device__ __forceinline__ uint32_t matrix_transpose(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
// Four codes as two fp16 pairs: (0, 1) and (2, 3), or with APART (0, 2) and (1, 3).
template <bool E4M3, bool APART>
__device__ __forceinline__ void q8_halves(uint32_t w, uint32_t& a, uint32_t& b) {
    if constexpr (E4M3) {
        if (APART) w = __byte_perm(w, 0u, 0x3120);
        asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}" : "=r"(a), "=r"(b) : "r"(w));
    } else {                                                 // 1024 + 128 + code, less that
        const uint32_t u = w ^ 0x80808080u;
        const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
        const uint32_t x = __byte_perm(u, 0x64646464u, APART ? 0x4240 : 0x4140), y = __byte_perm(u, 0x64646464u, APART ? 0x4341 : 0x4342);
        const __half2 p = __hsub2(*reinterpret_cast<const __half2*>(&x), off), q = __hsub2(*reinterpret_cast<const __half2*>(&y), off);
        a = *reinterpret_cast<const uint32_t*>(&p);
        b = *reinterpret_cast<const uint32_t*>(&q);
    }
}

__device__ __forceinline__ float q8_base(float top) { return top == -INFINITY ? 0.f : top; }

// ROWS: 4, 8 or 16, the query heads of a key head (or of a part of them) at most.
// BOX: blocks of a multiple of 16 tokens, so that a warp's 16 lie in one: they come as one box by TMA each for keys and values, and have one scale.
template <bool BF16, bool E4M3, int DP, int ROWS, bool BOX>
__global__ void __launch_bounds__(PA_THREADS, PagedQ8Cfg<DP, ROWS>::kPerSm)
paged_attention_q8_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const PagedQ8Params p) {
    using C = PagedQ8Cfg<DP, ROWS>;
    constexpr int HT = ROWS == 16 ? 2 : 1;                            // products' column tiles of 8 query heads
    constexpr bool PAIRED = ROWS == 4;                                // columns 4 to 7 are the same heads, for the weights' low parts
    constexpr float LIFT = 32768.f;                                   // the largest weight of a value (a pair of fp16 then reaches 2^-40 of it)
    extern __shared__ __align__(1024) uint8_t lin_smem[];             // (the loads' swizzle goes by the address)
    uint8_t* smem = lin_smem;
    __shared__ uint64_t s_full[PA_WARPS][C::kStages];
    __shared__ long long s_sum[PA_WARPS];
    __shared__ int s_start[2];
    __shared__ long long s_skip;
    __shared__ float s_m[PA_WARPS][PA_ROWS], s_l[PA_WARPS][PA_ROWS], s_m2[PA_WARPS][PA_ROWS];
    __shared__ float s_f[PA_WARPS][PA_ROWS];                          // what a warp's results are multiplied with where the warps meet
    __shared__ float2 s_top[2][PA_ROWS];                              // there: the maxima of a head
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    griddep_launch_dependents();
    if (BOX && tid == 0) {
        tma_prefetch_desc(&map_k);
        tma_prefetch_desc(&map_v);
    }

    // ---- the range: units of all requests, and where this CTA's first one lies -------------------------------------
    const int per = (p.nreq + PA_THREADS - 1) / PA_THREADS, r_lo = min(p.nreq, tid * per), r_hi = min(p.nreq, r_lo + per);
    const long long heads = p.groups;
    long long mine = 0;
    bool bad = false;
    for (int r = r_lo; r < r_hi; ++r) {
        const PagedSpan s = q8_span(p, r);
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
    if (BOX && tid < PA_WARPS * C::kStages) {
        mbar_init(&s_full[tid / C::kStages][tid % C::kStages], 2);
        mbar_fence_init();
    }
    if (u0 >= before * heads && u0 < (before + mine) * heads) {       // one thread's requests hold unit u0
        long long at = before * heads;
        int r = r_lo;
        long long n = q8_span(p, r).tiles * heads;
        while (u0 >= at + n) {
            at += n;
            n = q8_span(p, ++r).tiles * heads;
        }
        s_start[0] = r;
        s_skip = u0 - at;
    }
    __syncthreads();

    PagedIter ld;                                                     // the tile to fetch next
    ld.r = s_start[0];
    q8_enter(p, ld);
    ld.hp = static_cast<int>(s_skip / ld.tiles);
    ld.tile = static_cast<int>(s_skip - static_cast<long long>(ld.hp) * ld.tiles);
    PagedIter it = ld;                                                // the tile to work on next
    const bool cut_front = it.tile > 0;                               // the first (request, head) began in an earlier range

    const uint32_t sm = smem_u32(smem);
    const uint32_t sm_stage = sm + warp * C::kStages * C::kStage, sm_scale = sm + C::kAll + warp * C::kStages * C::kScales;
    float* sm_o = reinterpret_cast<float*>(smem + C::kOOff);
    if (BOX && (sm & 1023u)) {                                        // (never: the declaration asks for it)
        if (tid == 0) desc[2] = 1;
        return;
    }

    // this warp's key head among those side by side, and its tokens' place in a tile
    const int mine_head = warp & (p.side - 1), mine_tok = warp / p.side * Q8_TOKENS;
    const int words = p.dim / 16;

    // ---- fetch of a tile: 32 tokens' codes and scales per warp --------------------------------------------------------------------
    int head_ld = ld.hp / p.parts * p.side + mine_head;               // key head of the tile to fetch
    // BOX: the block of this lane's group of that tile (even lanes the first, odd ones the second), and the group's place in it; looked up one tile ahead
    int page_ld = -1, at_ld = 0;
    const auto look_up = [&] {
        const int tok = ld.first + ld.tile * p.tile + mine_tok + (lane & 1) * 16;
        page_ld = -1;
        if (tok < ld.len) {
            uint32_t b = __umulhi(static_cast<uint32_t>(tok), p.by_block);           // (at most one too small)
            at_ld = tok - static_cast<int>(b) * p.block_size;
            if (at_ld >= p.block_size) {
                ++b;
                at_ld -= p.block_size;
            }
            page_ld = p.table[ld.r * p.table_stride + b];
        }
    };
    if (BOX) look_up();
    const auto fetch = [&](int stage) {
        const uint32_t scales = sm_scale + stage * C::kScales;
        if constexpr (BOX) {
            if (lane < 4) {                                           // scales: the keys' of the first group, the second, the values'
                const bool there = ld.first + ld.tile * p.tile + mine_tok + (lane & 1) * 16 < ld.len, on = there && page_ld >= 0 && page_ld < p.num_blocks;
                if (there && !on) desc[2] = 1;                        // (every writer stores the same value)
                cp_async_4_or_zero(scales + lane * 4, on ? static_cast<const void*>((lane & 2 ? p.vs : p.ks) + page_ld * p.s_block + head_ld * p.s_head) : p.q, on);
                if (lane < 2 && !(lane == 0 && blockIdx.x == p.debug_skip)) {
                    uint64_t* bar = &s_full[warp][stage];
                    if (on) {
                        mbar_arrive_expect_tx(bar, 2 * C::kGroup);
                        uint8_t* dst = smem + (warp * C::kStages + stage) * C::kStage + lane * C::kGroup;
#pragma unroll
                        for (int x = 0; x < DP / C::kBox; ++x) {
                            tma_load_4d(dst + x * 2048, &map_k, bar, x * 128, head_ld, at_ld, page_ld);
                            tma_load_4d(dst + C::kKeys + x * 2048, &map_v, bar, x * 128, head_ld, at_ld, page_ld);
                        }
                    } else {
                        mbar_arrive(bar);
                    }
                }
            }
        } else {
            const int tok = ld.first + ld.tile * p.tile + mine_tok + lane;
            long long at = -1, sc = 0;
            if (tok >= ld.begin && tok < ld.len) {
                const unsigned b = static_cast<unsigned>(tok) / static_cast<unsigned>(p.block_size);
                const int page = p.table[ld.r * p.table_stride + b];
                if (page >= 0 && page < p.num_blocks) {
                    at = page * p.c_block + static_cast<long long>(tok - b * p.block_size) * p.c_tok + head_ld * p.c_head;
                    sc = page * p.s_block + head_ld * p.s_head;
                } else {
                    desc[2] = 1;                                      // (every writer stores the same value)
                }
            }
            const uint32_t dst = sm_stage + stage * C::kStage;
            constexpr int kRows = 32 / C::kChunks;                    // rows side by side
#pragma unroll
            for (int i = 0; i < Q8_TOKENS / kRows; ++i) {
                const int row = i * kRows + lane / C::kChunks, c = lane % C::kChunks;
                const long long a = __shfl_sync(0xffffffffu, at, row);
                const bool on = a >= 0 && c < words;
                const uint32_t d = dst + (row >> 4) * C::kGroup + C::place(row & 15, c);
                cp_async_16_or_zero(d, on ? static_cast<const void*>(p.k8 + a + c * 16) : p.q, on);
                cp_async_16_or_zero(d + C::kKeys, on ? static_cast<const void*>(p.v8 + a + c * 16) : p.q, on);
            }
            // scales, the keys' and the values' (zero for what is not a token)
            cp_async_4_or_zero(scales + lane * 4, at >= 0 ? static_cast<const void*>(p.ks + sc) : p.q, at >= 0);
            cp_async_4_or_zero(scales + (Q8_TOKENS + lane) * 4, at >= 0 ? static_cast<const void*>(p.vs + sc) : p.q, at >= 0);
        }
    };
    long long u_ld = u0;

    // Where this lane reads: word 4 g + c of its key's row is at (k_lane ^ 64 g) + 16 rows of 8, word 2 d + (lane / 16) of its value's at v_lane ^ 32 d (a row's
    // words lie within its 128 bytes, or 64).
    const uint32_t k_lane = sm_stage + C::place(C::token(lane >> 2), lane & 3), v_lane = sm_stage + C::kKeys + C::place(C::token(lane & 15), lane >> 4);
    const auto word = [](uint32_t base, int c) { return (base ^ ((c & 7) << 4)) + (c >> 3) * 2048; };
    // The query as the product's second operand: of columns 64 g + 16 c + 4 s to + 3 (c = lane modulo 4) in product 4 g + s; head lane / 4 of each tile.
    uint32_t qf[HT][DP / 16][2];
    // of heads 2 c and 2 c + 1 of each tile:
    float qs[HT][2];                                                  // scale * log2(e), times what the head's row was divided by
    float m[HT][2], l[HT][2], m2[HT][2];                              // maximum; sum of 2^(s - m); maximum of the values' weights, above m
    float o[HT][DP / 16][4];                                          // columns 16 d + 2 g (0, 1) and 16 d + 2 g + 1 (2, 3) of heads 2 c, 2 c + 1, g = lane / 4
    int seg = 0, stage = 0;
    bool begins = true, late = false;
    uint32_t turn = 0;                                                // of the stages' barriers
#pragma unroll 1
    for (long long u = u0 - C::kStages; u < u1; ++u) {
        if (begins && u >= u0) {
            const int part = it.hp % p.parts, head = it.hp / p.parts * p.side + mine_head, rows = min(p.rows, p.group - part * p.rows);
#pragma unroll
            for (int h = 0; h < HT; ++h) {
                const int row = PAIRED ? (lane >> 2) & 3 : (lane >> 2) + 8 * h;
                const uint16_t* src = p.q + it.r * p.q_req + (static_cast<long long>(head) * p.group + part * p.rows + row) * p.q_head + (lane & 3) * 16;
                uint32_t most = 0u;
#pragma unroll
                for (int g = 0; g < DP / 64; ++g) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        uint4 w = make_uint4(0u, 0u, 0u, 0u);
                        if (row < rows && 64 * g + (lane & 3) * 16 + half * 8 < p.dim) w = *reinterpret_cast<const uint4*>(src + 64 * g + half * 8);
                        const uint32_t in[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            qf[h][4 * g + 2 * half + (e >> 1)][e & 1] = in[e];
                            most = __vmaxu2(most, in[e] & 0x7fff7fffu);
                        }
                    }
                }
                float divided = 1.f;
                if constexpr (BF16) {
                    most = max(most & 0xffffu, most >> 16);
                    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
                    most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
                    // largest magnitude in [2^e, 2^(e + 1)): times 2^(14 - e)
                    const int e = static_cast<int>(most >> 7) - 127, up = most >= 0x7f80u ? 0 : max(-126, min(126, 14 - e));
                    const float f = __int_as_float((up + 127) << 23);
                    divided = __int_as_float((127 - up) << 23);
#pragma unroll
                    for (int d = 0; d < DP / 16; ++d)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float2 x = unpack_pair<true>(qf[h][d][i]);
                            qf[h][d][i] = pack_pair<false>(x.x * f, x.y * f);
                        }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    qs[h][i] = p.scale_log2 * __shfl_sync(0xffffffffu, divided, (2 * (lane & 3) + i) * 4);
                    m[h][i] = -INFINITY;
                    m2[h][i] = Q8_FLOOR;
                    l[h][i] = 0.f;
                }
#pragma unroll
                for (int d = 0; d < DP / 16; ++d) o[h][d][0] = o[h][d][1] = o[h][d][2] = o[h][d][3] = 0.f;
            }
            ++seg;
        }
        cp_async_wait<C::kStages - 1>();
        if (BOX && u >= u0 && !late) {
            const bool there = mbar_try_wait_for(&s_full[warp][stage], turn, 20000u) || q8_wait(&s_full[warp][stage], turn, p.budget_ns);
            if (__any_sync(0xffffffffu, !there)) {
                // This warp's part ends: it fetches and works on nothing more, and comes along to where the warps meet.  The loads on their way (this tile's and the next
                // one's) land before the CTA leaves.
                late = true;
                q8_land(s_full[warp], stage, turn, u + 1 < u1);
                u_ld = u1;
            }
            if (stage + 1 == C::kStages) turn ^= 1;
        }
        __syncwarp();
        const int tok0 = it.first + it.tile * p.tile + mine_tok;
        if (u >= u0 && tok0 < it.len && !late) {
            const uint32_t sb = sm_scale + stage * C::kScales;
            const bool edge = tok0 < it.begin || tok0 + Q8_TOKENS > it.len;
            if (BOX && E4M3 && edge) {                                // codes of no token of this request: a weight of zero does not hide a NaN
                for (int i = lane; i < Q8_TOKENS * C::kChunks; i += 32) {
                    const int row = i / C::kChunks;
                    if (tok0 + row < it.begin || tok0 + row >= it.len)
                        *reinterpret_cast<uint4*>(smem + (warp * C::kStages + stage) * C::kStage + C::kKeys + (row >> 4) * C::kGroup + C::place(row & 15, i % C::kChunks)) =
                            make_uint4(0u, 0u, 0u, 0u);
                }
                fence_proxy_async_smem();
                __syncwarp();
            }
            // scores of tokens g (0, 1) and g + 8 (2, 3) of each group of 16 for heads 2 c, 2 c + 1
            float s[HT][2][4], lift[2][2];                            // lift: log2 of the values' scale, of the two tokens
#pragma unroll
            for (int y = 0; y < 2; ++y) {
#pragma unroll
                for (int h = 0; h < HT; ++h) s[h][y][0] = s[h][y][1] = s[h][y][2] = s[h][y][3] = 0.f;
#pragma unroll
                for (int g = 0; g < DP / 64; ++g) {
                    const uint32_t at = word(k_lane + stage * C::kStage + y * C::kGroup, 4 * g);
                    const uint4 v0 = lds_128(at), v1 = lds_128(at + 8 * C::kBox);
                    const uint32_t lo8[4] = {v0.x, v0.y, v0.z, v0.w}, hi8[4] = {v1.x, v1.y, v1.z, v1.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t a[4];
                        q8_halves<E4M3, false>(lo8[e], a[0], a[2]);
                        q8_halves<E4M3, false>(hi8[e], a[1], a[3]);
#pragma unroll
                        for (int h = 0; h < HT; ++h) mma_16816<false>(s[h][y], a, qf[h][4 * g + e][0], qf[h][4 * g + e][1]);
                    }
                }
                float ks[2];
                if constexpr (BOX) {
                    ks[0] = ks[1] = q8_key_scale(lds_float(sb + y * 4));
                    lift[y][0] = paged_log2(lds_float(sb + 8 + y * 4));
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t at = sb + (y * 16 + C::token((lane >> 2) + 8 * i)) * 4;
                        ks[i] = q8_key_scale(lds_float(at));
                        lift[y][i] = paged_log2(lds_float(at + Q8_TOKENS * 4));
                    }
                }
#pragma unroll
                for (int h = 0; h < HT; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[h][y][i] *= qs[h][i & 1] * ks[i >> 1];
            }
            if (edge)
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int tok = tok0 + y * 16 + C::token((lane >> 2) + 8 * i);
                        if (tok < it.begin || tok >= it.len) {
#pragma unroll
                            for (int h = 0; h < HT; ++h) s[h][y][2 * i] = s[h][y][2 * i + 1] = -INFINITY;
                        }
                    }
            uint32_t hi[HT][2][2], lo[HT][2][2];                      // the weights as a product's second operand: tokens 0 to 7, 8 to 15 of each group
#pragma unroll
            for (int h = 0; h < HT; ++h) {
                float w[2][4], fall[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {                         // heads 2 c, 2 c + 1
                    float top[2];                                     // of each group of 16 tokens
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        top[y] = fmaxf(s[h][y][i], s[h][y][2 + i]);
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) top[y] = fmaxf(top[y], __shfl_xor_sync(0xffffffffu, top[y], x));
                    }
                    const float now = fmaxf(m[h][i], fmaxf(top[0], top[1]));
                    const float base = now == -INFINITY ? 0.f : now;  // (no token yet: every weight is 2^-inf = 0)
                    float t[2][2], top2;
#pragma unroll
                    for (int y = 0; y < 2; ++y)
#pragma unroll
                        for (int j = 0; j < 2; ++j) t[y][j] = s[h][y][2 * j + i] - base;
                    if constexpr (BOX) {                              // (one scale in each group: its largest score has the largest weight)
                        top2 = fmaxf((top[0] - base) + lift[0][0], (top[1] - base) + lift[1][0]);
                    } else {
                        top2 = -INFINITY;
#pragma unroll
                        for (int y = 0; y < 2; ++y)
#pragma unroll
                            for (int j = 0; j < 2; ++j) top2 = fmaxf(top2, t[y][j] + lift[y][j]);
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) top2 = fmaxf(top2, __shfl_xor_sync(0xffffffffu, top2, x));
                    }
                    const float sinks = m[h][i] - base, was2 = m2[h][i] + sinks, now2 = fmaxf(fmaxf(was2, top2), Q8_FLOOR);
                    fall[i] = paged_exp2(was2 - now2);
                    l[h][i] *= paged_exp2(sinks);
                    m[h][i] = now;
                    m2[h][i] = now2;
#pragma unroll
                    for (int y = 0; y < 2; ++y)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int x = BOX ? 0 : j;
                            l[h][i] += paged_exp2(t[y][j]);
                            w[y][2 * j + i] = LIFT * paged_exp2(t[y][j] + (lift[y][x] - now2));
                        }
                }
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        // The weights enter the product as the sum of two fp16 values (2^-22 of themselves, at least 2^-40 of the largest): rounded to
                        // one, their error would be as large as the result's own rounding.
                        uint32_t x = pack_pair<false>(w[y][2 * j], w[y][2 * j + 1]);
                        const float2 back = unpack_pair<false>(x);
                        const uint32_t rest = pack_pair<false>(w[y][2 * j] - back.x, w[y][2 * j + 1] - back.y);
                        if (PAIRED) {
                            if (lane & 2) x = rest;                   // (columns 4 to 7)
                        } else {
                            lo[h][y][j] = matrix_transpose(rest);
                        }
                        hi[h][y][j] = matrix_transpose(x);
                    }
                if (__any_sync(0xffffffffu, fall[0] != 1.f || fall[1] != 1.f)) {      // (the maximum of a long context soon stands)
#pragma unroll
                    for (int d = 0; d < DP / 16; ++d)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[h][d][i] *= fall[i & 1];
                }
            }
            // lanes 0-7: tokens 0-7, 16 columns; 8-15: tokens 8-15 of them; 16-31: the next 16 columns
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) {
                    uint32_t w[4];
                    ldsm_x4_t(w, word(v_lane + stage * C::kStage + y * C::kGroup, 2 * d));
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        uint32_t a[4];
                        q8_halves<E4M3, true>(w[2 * x], a[0], a[1]);
                        q8_halves<E4M3, true>(w[2 * x + 1], a[2], a[3]);
#pragma unroll
                        for (int h = 0; h < HT; ++h) {
                            mma_16816<false>(o[h][2 * d + x], a, hi[h][y][0], hi[h][y][1]);
                            if (!PAIRED) mma_16816<false>(o[h][2 * d + x], a, lo[h][y][0], lo[h][y][1]);
                        }
                    }
                }
        }
        __syncwarp();                                                 // the stage has been read by all lanes
        if (u_ld < u1) {
            fetch(stage);
            if (++u_ld < u1) {
                if (q8_next(p, ld)) head_ld = ld.hp / p.parts * p.side + mine_head;
                if (BOX) look_up();
            }
        }
        cp_async_commit();
        stage = stage + 1 == C::kStages ? 0 : stage + 1;
        if (u < u0) continue;

        const PagedIter done = it;
        const bool ends = it.tile + 1 == it.tiles;                    // of this (request, head part)
        begins = ends;
        const bool last = u + 1 == u1;
        if (!last) q8_next(p, it);
        if (!ends && !last) continue;

        // ---- the warps of a head meet ------------------------------------------------------------------------------------
        const int part = done.hp % p.parts, head0 = done.hp / p.parts * p.side;
        const int rows = min(p.rows, p.group - part * p.rows);
        if (PAIRED)
#pragma unroll
            for (int d = 0; d < DP / 16; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[0][d][i] += __shfl_xor_sync(0xffffffffu, o[0][d][i], 2);
#pragma unroll
        for (int h = 0; h < HT; ++h)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l[h][i] += __shfl_xor_sync(0xffffffffu, l[h][i], x);
                if (lane < 4) {
                    const int row = 8 * h + 2 * lane + i;
                    s_m[warp][row] = m[h][i];
                    s_l[warp][row] = l[h][i];
                    s_m2[warp][row] = m2[h][i];
                }
            }
        __syncthreads();
        if (tid < PA_WARPS * PA_ROWS) {
            const int w = tid / PA_ROWS, row = tid % PA_ROWS, hh = w & (p.side - 1);
            float a[PA_WARPS], b[PA_WARPS], t = -INFINITY, t2 = Q8_FLOOR;
#pragma unroll
            for (int x = 0; x < PA_WARPS; ++x) {
                a[x] = s_m[x][row];
                b[x] = s_m2[x][row];
                if ((x & (p.side - 1)) == hh) t = fmaxf(t, a[x]);
            }
#pragma unroll
            for (int x = 0; x < PA_WARPS; ++x)
                if ((x & (p.side - 1)) == hh) t2 = fmaxf(t2, b[x] + (a[x] - q8_base(t)));
            // (a warp without tokens has maximum -infinity, sum 0 and result 0, and contributes 2^-inf = 0 times that; a NaN stays one)
            const float sinks = s_m[w][row] - q8_base(t);
            s_f[w][row] = paged_exp2(s_m2[w][row] + sinks - t2) * (1.f / LIFT);
            s_l[w][row] *= paged_exp2(sinks);
            if (w < p.side) s_top[w][row] = make_float2(t, t2);
        }
        __syncthreads();
        const bool began_here = !(cut_front && seg == 1);
        const bool whole = began_here && ends;
        const long long slot = 2ll * blockIdx.x + (began_here ? 1 : 0);
        for (int half = 0; half < 2; ++half) {                        // half of the columns at a time
#pragma unroll
            for (int h = 0; h < HT; ++h)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int row = 8 * h + 2 * (lane & 3) + i;
                    if (row < rows) {
                        const float f = s_f[warp][row];
#pragma unroll
                        for (int d = 0; d < DP / 16; ++d)             // columns 16 d + 2 g, + 1
                            if (d / (DP / 32) == half)
                                *reinterpret_cast<float2*>(sm_o + (warp * p.rows + row) * C::kPitch + d % (DP / 32) * 16 + (lane >> 2) * 2) =
                                    make_float2(o[h][d][i] * f, o[h][d][2 + i] * f);
                    }
                }
            __syncthreads();
            for (int i = tid; i < p.side * rows * (DP / 8); i += PA_THREADS) {
                const int line = i / (DP / 8), at = (i - line * (DP / 8)) * 4, c = half * (DP / 2) + at, hh = line / rows, row = line - hh * rows;
                const float t = s_top[hh][row].x, t2 = s_top[hh][row].y;
                float sum = 0.f;
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int w = hh; w < PA_WARPS; w += p.side) {
                    sum += s_l[w][row];
                    const float4 y = *reinterpret_cast<const float4*>(sm_o + (w * p.rows + row) * C::kPitch + at);
                    x.x += y.x;
                    x.y += y.y;
                    x.z += y.z;
                    x.w += y.w;
                }
                const long long orow = done.r * static_cast<long long>(p.heads) + static_cast<long long>(head0 + hh) * p.group + part * p.rows + row;
                if (whole) {
                    // (every weight 0: the result is 0.  Every value's scale 0: x is, or NaN, and 2^Q8_FLOOR is)
                    const float inv = sum == 0.f ? 0.f : exp2f(t2) / sum;
                    if (c < p.dim)
                        *reinterpret_cast<uint2*>(p.out + orow * p.dim + c) =
                            make_uint2(pack_pair<BF16>(x.x * inv, x.y * inv), pack_pair<BF16>(x.z * inv, x.w * inv));
                    if (c == 0 && p.lse) p.lse[orow] = sum == 0.f ? -INFINITY : (t + log2f(sum)) * 0.69314718055994531f;
                } else {
                    const long long to = slot * p.side + hh;
                    if (c < p.dim) *reinterpret_cast<float4*>(p.part_o + (to * p.rows + row) * p.dim + c) = x;
                    if (c == 0) {
                        p.part_ml[(to * 2) * PA_ROWS + row] = t;
                        p.part_ml[(to * 2 + 1) * PA_ROWS + row] = sum;
                        p.part_m2[to * PA_ROWS + row] = t2;
                    }
                }
            }
            __syncthreads();
        }
        if (!whole && began_here && tid == 0) {                       // this range joins it; its last unit lies in a later one
            desc[0] = static_cast<int32_t>(done.r);
            desc[1] = static_cast<int32_t>(paged_cta_of(u + (done.tiles - 1 - done.tile), units, ctas));
            desc[3] = done.hp;
        }
    }
    if (BOX && late) desc[2] = 5;                                     // MMV_ERR_TIMEOUT
}

// Joins the partials of the (request, heads) that begins in range blockIdx.x and is cut at its end: one query head per CTA.  Also the requests without tokens and the status word.
template <bool BF16>
__global__ void __launch_bounds__(PA_JOIN_THREADS) paged_join_q8_kernel(const PagedQ8Params p, int ctas) {
    __shared__ float s_w[PA_JOIN_THREADS], s_red[4], s_red2[4];
    __shared__ float4 s_x[PA_JOIN_THREADS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, hh = blockIdx.y / p.rows, row = blockIdx.y - hh * p.rows;
    griddep_wait();
    if (blockIdx.y == 0) {
        for (int r = blockIdx.x; r < p.nreq; r += gridDim.x) {        // nothing to attend to: 0, and the logarithm of an empty sum
            if (q8_span(p, r).tiles) continue;
            for (long long i = tid; i < static_cast<long long>(p.heads) * p.dim; i += PA_JOIN_THREADS) p.out[r * static_cast<long long>(p.heads) * p.dim + i] = 0;
            if (p.lse)
                for (int i = tid; i < p.heads; i += PA_JOIN_THREADS) p.lse[r * static_cast<long long>(p.heads) + i] = -INFINITY;
        }
        if (blockIdx.x == 0) {
            int e = 0;
            for (int i = tid; i < ctas; i += PA_JOIN_THREADS) e |= p.desc[4 * i + 2];
            const bool late = __syncthreads_or(e & 4), bad = __syncthreads_or(e & 1);
            if (tid == 0) {
                p.hdr->tile_counter = 0u;
                p.hdr->error = late ? 5u : bad ? 1u : 0u;             // MMV_ERR_TIMEOUT, MMV_ERR_INVALID_ARG
            }
        }
    }
    const int32_t* desc = p.desc + 4 * blockIdx.x;
    const int r = desc[0];
    if (r < 0) return;
    const int last = desc[1], hp = desc[3], head = hp / p.parts * p.side + hh, part = hp % p.parts;
    if (row >= min(p.rows, p.group - part * p.rows)) return;
    const int first = blockIdx.x, n = last - first + 1;
    const auto place = [&](int i) { return (2ll * (first + i) + (i == 0 ? 1 : 0)) * p.side + hh; };
    // the maxima, of the scores and then of the values' weights above it, then the weights' sum
    const auto most = [&](float x, float (&red)[4]) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
        if (lane == 0) red[warp] = x;
        __syncthreads();
        return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    };
    const auto score = [&](int i) { return i < n ? p.part_ml[place(i) * 2 * PA_ROWS + row] : -INFINITY; };
    const auto weight = [&](int i) { return i < n ? p.part_m2[place(i) * PA_ROWS + row] : -INFINITY; };
    const float mine = score(tid), mine2 = weight(tid);               // (all there are, but for the longest contexts)
    float top = mine;
    for (int i = tid + PA_JOIN_THREADS; i < n; i += PA_JOIN_THREADS) top = fmaxf(top, score(i));
    top = most(top, s_red);
    const float base = q8_base(top);
    float top2 = mine2 + (mine - base);
    for (int i = tid + PA_JOIN_THREADS; i < n; i += PA_JOIN_THREADS) top2 = fmaxf(top2, weight(i) + (score(i) - base));
    top2 = most(top2, s_red2);
    const float base2 = q8_base(top2);
    const int cols = p.dim / 4, lanes = cols <= 32 ? 32 : 64, groups = PA_JOIN_THREADS / lanes;
    const int g = tid / lanes, c = tid - g * lanes;
    float sum = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0; i0 < n; i0 += PA_JOIN_THREADS) {                 // (in order: the same result every time)
        const int i = i0 + tid;
        float w = 0.f;
        if (i < n) {
            const float above = (i0 ? score(i) : mine) - base;
            sum += paged_exp2(above) * p.part_ml[(place(i) * 2 + 1) * PA_ROWS + row];
            w = paged_exp2((i0 ? weight(i) : mine2) + above - base2);
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
        const long long orow = r * static_cast<long long>(p.heads) + static_cast<long long>(head) * p.group + part * p.rows + row;
        const float inv = sum == 0.f ? 0.f : exp2f(top2) / sum;
        *reinterpret_cast<uint2*>(p.out + orow * p.dim + c * 4) =
            make_uint2(pack_pair<BF16>(x.x * inv, x.y * inv), pack_pair<BF16>(x.z * inv, x.w * inv));
        if (c == 0 && p.lse) p.lse[orow] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
    }
}

}  // namespace mmv

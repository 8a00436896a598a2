// Attention of one new token per request over a paged key-value cache in 8 bits with a scale for each block of tokens and head.
//
//     s_j = scale (q . code^k_j) ks_j,   out = sum_j softmax(s)_j vs_j code^v_j,   lse = log sum_j exp s_j       (ks, vs: the scales of j's block)
//
// The split over CTAs, the order of the units and the join of cut (request, head)s are those of the attention over a 16-bit cache
// (paged_attn.cuh).  What differs:
//   Codes become fp16 in registers (every int8 and e4m3 value is one) and both products run in fp16.  A bfloat16 query is brought
//     into fp16's range by a power of two of its own row, exactly but for values 2^29 times smaller than the row's largest.
//   The columns of a query and of a key may be taken in any order that both share: a lane takes 16 neighbouring columns of a token's
//     key with one load, four of them for each of four products.  Values are read transposed in pairs of columns (8-bit
//     columns 2d and 2d + 1 are one 16-bit element) and taken apart by a byte permutation: a product's result columns are the even, or
//     the odd ones.
//   Scales of values are part of the weights that meet the codes: 2^(s_j + log2 vs_j - m'), with a running maximum m' of its own, so that no
//     scale leaves fp16's range; the weights of the sum are 2^(s_j - m).
//
// What bounds it: HBM, 2 dim bytes per token and key head, with about 380 instructions per 16 tokens of a warp beside them (5 for four int8
// codes), half of what the issue slots allow at that rate: so more warps per SM than the 16-bit kernel has.
#pragma once
#include <cstdint>
#include "kv_cache_q8.cuh"
#include "paged_attn.cuh"

namespace mmv {

struct PagedQ8Params : PagedParams {                         // (k and v of the base are not used)
    const uint8_t *k8, *v8;
    const float *ks, *vs;
    long long s_block, s_head;
    float* part_m2;                                          // [grid][2][PA_ROWS]: maximum of the values' weights (less LIFT)
};

template <int DP>
struct PagedQ8Cfg {
    static constexpr int kStages = 2;
    static constexpr int kPerSm = DP == 256 ? 2 : 3;                           // CTAs that the registers allow
    static constexpr int kRow = DP;                                            // bytes of a token's codes
    static constexpr int kChunks = DP / 16;                                    // 16-byte words of it
    static constexpr int kCodes = PA_TOKENS * kRow * 2;                        // keys and values of a warp's tokens
    static constexpr int kStage = kCodes + PA_TOKENS * 8;                      // and their scales
    static constexpr int kQ = PA_ROWS * DP * 2;
    static constexpr int kQSlots = kStages + 1;
    static constexpr int kPitch = DP + 8;                                      // floats of a row where warps meet
    static constexpr int kAll = PA_WARPS * kStages * kStage;
    static int smem_bytes(int rows) { return kAll + kQSlots * kQ + PA_WARPS * rows * kPitch * 4; }
};

__device__ __forceinline__ void cp_async_4_or_zero(uint32_t dst, const void* src, bool on) {
    const int bytes = on ? 4 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint4 lds_128(uint32_t addr) {
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(addr) : "memory");
    return r;
}
__device__ __forceinline__ float2 lds_float2(uint32_t addr) {
    float2 r;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(r.x), "=f"(r.y) : "r"(addr) : "memory");
    return r;
}
__device__ __forceinline__ float paged_log2(float x) {
    float r;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
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

// SMALL: up to 8 query heads per key head, the product's other 8 rows take the low parts of the weights.
template <bool BF16, bool E4M3, int DP, bool SMALL>
__global__ void __launch_bounds__(PA_THREADS, PagedQ8Cfg<DP>::kPerSm) paged_attention_q8_kernel(const PagedQ8Params p) {
    using C = PagedQ8Cfg<DP>;
    constexpr int HALVES = SMALL ? 1 : 2;                             // of the 16 rows that hold query heads
    constexpr float LIFT = 15.f;                                      // the exponent of the largest weight of a value (a pair of fp16 then reaches 2^-40 of it)
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long s_sum[PA_WARPS];
    __shared__ int s_start[2];
    __shared__ long long s_skip;
    __shared__ float s_m[PA_WARPS][PA_ROWS], s_l[PA_WARPS][PA_ROWS], s_m2[PA_WARPS][PA_ROWS];
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
    const uint32_t sm_stage = sm + warp * C::kStages * C::kStage;
    const uint32_t sm_q = sm + C::kAll;
    float* sm_o = reinterpret_cast<float*>(smem + C::kAll + C::kQSlots * C::kQ);
    const int words = p.dim / 16;
    // Where word c of a row lies: eight rows' words of one column lie in different banks, and so do four words of two neighbouring rows.
    const auto place = [](int row, int c) { return c ^ (((row >> 1) & 3) | (C::kChunks >= 8 ? (row & 1) << 2 : 0)); };

    // ---- fetch of a tile: 16 tokens' codes and scales per warp; with a new head the query rows too ------------------------
    int seg_ld = 0;
    const auto fetch_q = [&] {
        const int head = ld.hp / p.parts, part = ld.hp - head * p.parts;
        const int rows = min(p.rows, p.group - part * p.rows);
        const uint16_t* src = p.q + ld.r * p.q_req + (head * p.group + part * p.rows) * p.q_head;
        const uint32_t dst = sm_q + (seg_ld % C::kQSlots) * C::kQ;
        for (int i = tid; i < PA_ROWS * (DP / 8); i += PA_THREADS) {
            const int row = i / (DP / 8), c = i - row * (DP / 8);
            const bool on = row < rows && c < p.dim / 8;
            cp_async_16_or_zero(dst + row * DP * 2 + c * 16, on ? src + row * p.q_head + c * 8 : p.q, on);
        }
        ++seg_ld;
    };
    const auto fetch = [&](int stage) {
        const int head = ld.hp / p.parts;
        const int tok = ld.first + ld.tile * PA_TILE + warp * PA_TOKENS + (lane & 15);
        long long at = -1, sc = 0;
        if (tok >= ld.begin && tok < ld.len) {
            const unsigned b = static_cast<unsigned>(tok) / static_cast<unsigned>(p.block_size);
            const int page = p.table[ld.r * p.table_stride + b];
            if (page >= 0 && page < p.num_blocks) {
                at = page * p.c_block + static_cast<long long>(tok - b * p.block_size) * p.c_tok + head * p.c_head;
                sc = page * p.s_block + head * p.s_head;
            } else {
                desc[2] = 1;                                          // (every writer stores the same value)
            }
        }
        const uint32_t dst = sm_stage + stage * C::kStage;
        constexpr int kPerRow = C::kChunks;                           // lanes on one row
        constexpr int kRows = 32 / kPerRow;
#pragma unroll
        for (int i = 0; i < PA_TOKENS / kRows; ++i) {
            const int row = i * kRows + lane / kPerRow, c = lane % kPerRow;
            const long long a = __shfl_sync(0xffffffffu, at, row);
            const bool on = a >= 0 && c < words;
            const uint32_t d = dst + row * C::kRow + (place(row, c) << 4);
            cp_async_16_or_zero(d, on ? static_cast<const void*>(p.k8 + a + c * 16) : p.q, on);
            cp_async_16_or_zero(d + PA_TOKENS * C::kRow, on ? static_cast<const void*>(p.v8 + a + c * 16) : p.q, on);
        }
        // scales: lanes 0 to 15 the keys', 16 to 31 the values' (zero for what is not a token)
        cp_async_4_or_zero(dst + C::kCodes + lane * 4, at >= 0 ? static_cast<const void*>((lane < 16 ? p.ks : p.vs) + sc) : p.q, at >= 0);
    };
    long long u_ld = u0;
    bool fresh = true;                                                // the next tile to fetch begins a head

    // The query as the product's first operand: of columns 64 g + 16 c + 4 s to + 3 (c = lane modulo 4) in product 4 g + s; rows lane / 4 and, if
    // not SMALL, lane / 4 + 8 (which are zero otherwise).
    uint32_t qf[DP / 16][2 * HALVES];
    float qs[HALVES];                                                 // scale * log2(e), times what the row was divided by
    float o[DP / 8][4];
    float m[HALVES], l[HALVES], m2[HALVES];                           // maximum; sum of 2^(s - m); maximum of the values' weights less LIFT
    int seg = 0, stage = 0;
    bool begins = true;
#pragma unroll 1
    for (long long u = u0 - C::kStages; u < u1; ++u) {
        cp_async_wait<C::kStages - 1>();
        __syncwarp();
        if (begins && u >= u0) {
            __syncthreads();                                          // every warp's share of the query rows has landed
            const uint32_t src = sm_q + (seg % C::kQSlots) * C::kQ + (lane & 3) * 32;
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                const uint32_t row = src + ((lane >> 2) + 8 * h) * DP * 2;
                uint32_t most = 0u;
#pragma unroll
                for (int g = 0; g < DP / 64; ++g) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint4 w = lds_128(row + g * 128 + half * 16);
                        const uint32_t in[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            qf[4 * g + 2 * half + (e >> 1)][(e & 1) * HALVES + h] = in[e];
                            most = __vmaxu2(most, in[e] & 0x7fff7fffu);
                        }
                    }
                }
                qs[h] = p.scale_log2;
                if constexpr (BF16) {
                    most = max(most & 0xffffu, most >> 16);
                    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
                    most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
                    // largest magnitude in [2^e, 2^(e + 1)): times 2^(14 - e)
                    const int e = static_cast<int>(most >> 7) - 127, up = most >= 0x7f80u ? 0 : max(-126, min(126, 14 - e));
                    const float f = __int_as_float((up + 127) << 23);
                    qs[h] *= __int_as_float((127 - up) << 23);
#pragma unroll
                    for (int d = 0; d < DP / 16; ++d)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float2 x = unpack_pair<true>(qf[d][i * HALVES + h]);
                            qf[d][i * HALVES + h] = pack_pair<false>(x.x * f, x.y * f);
                        }
                }
                m[h] = m2[h] = -INFINITY;
                l[h] = 0.f;
            }
#pragma unroll
            for (int n = 0; n < DP / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
            ++seg;
        }
        const int tok0 = it.first + it.tile * PA_TILE + warp * PA_TOKENS;
        if (u >= u0 && tok0 < it.len) {
            const uint32_t kb = sm_stage + stage * C::kStage, vb = kb + PA_TOKENS * C::kRow, sb = kb + C::kCodes;
            float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int g = 0; g < DP / 64; ++g)
#pragma unroll
                for (int n = 0; n < 2; ++n) {                         // tokens lane / 4 and lane / 4 + 8
                    const int row = (lane >> 2) + 8 * n;
                    const uint4 w = lds_128(kb + row * C::kRow + (place(row, 4 * g + (lane & 3)) << 4));
                    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t b0, b1;
                        q8_halves<E4M3, false>(in[e], b0, b1);
                        const uint32_t(&q)[2 * HALVES] = qf[4 * g + e];
                        const uint32_t a[4] = {q[0], SMALL ? 0u : q[1], q[HALVES], SMALL ? 0u : q[2 * HALVES - 1]};
                        mma_16816<false>(s[n], a, b0, b1);
                    }
                }
            const bool edge = tok0 < it.begin || tok0 + PA_TOKENS > it.len;
            float lift[2][2];                                         // log2 of the value scales of this lane's tokens
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const float2 ks = lds_float2(sb + (n * 8 + (lane & 3) * 2) * 4), vs = lds_float2(sb + (PA_TOKENS + n * 8 + (lane & 3) * 2) * 4);
                lift[n][0] = paged_log2(vs.x);
                lift[n][1] = paged_log2(vs.y);
#pragma unroll
                for (int i = 0; i < 2 * HALVES; ++i) {
                    s[n][i] *= qs[i >> 1] * ((i & 1) ? ks.y : ks.x);
                    if (edge) {
                        const int tok = tok0 + n * 8 + (lane & 3) * 2 + (i & 1);
                        if (tok < it.begin || tok >= it.len) {
                            s[n][i] = -INFINITY;
                            lift[n][i & 1] = 0.f;
                        }
                    }
                }
            }
            uint32_t hi[4], lo[4];                                    // (SMALL: the low parts are hi[1] and hi[3], rows 8 to 15)
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {                        // rows lane / 4 and lane / 4 + 8
                float t[2][2];
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) t[n][i] = s[n][2 * h + i] + lift[n][i];
                float top = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
                float top2 = fmaxf(fmaxf(t[0][0], t[0][1]), fmaxf(t[1][0], t[1][1]));
#pragma unroll
                for (int x = 1; x <= 2; x <<= 1) {
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                    top2 = fmaxf(top2, __shfl_xor_sync(0xffffffffu, top2, x));
                }
                const float now = fmaxf(m[h], top), now2 = fmaxf(m2[h], top2 - LIFT);
                const float base = now == -INFINITY ? 0.f : now;      // (no token yet: every weight is 2^-inf = 0)
                const float base2 = now2 == -INFINITY ? 0.f : now2;
                const float fall = paged_exp2(m2[h] - base2);
                l[h] *= paged_exp2(m[h] - base);
                m[h] = now;
                m2[h] = now2;
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    l[h] += paged_exp2(s[n][2 * h] - base) + paged_exp2(s[n][2 * h + 1] - base);
                    const float a = paged_exp2(t[n][0] - base2), b = paged_exp2(t[n][1] - base2);
                    // The weights enter the product as the sum of two fp16 values (2^-22 of themselves, at least 2^-40 of the largest): rounded to
                    // one, their error would be as large as the result's own rounding.
                    hi[n * 2 + h] = pack_pair<false>(a, b);
                    const float2 back = unpack_pair<false>(hi[n * 2 + h]);
                    (SMALL ? hi[n * 2 + 1] : lo[n * 2 + h]) = pack_pair<false>(a - back.x, b - back.y);
                }
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
                // lanes 0-7: tokens 0-7, 16 columns; 8-15: tokens 8-15 of them; 16-31: the next 16 columns
                const int row = lane & 15;
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) {
                    uint32_t w[4];
                    ldsm_x4_t(w, vb + row * C::kRow + (place(row, 2 * d + (lane >> 4)) << 4));
#pragma unroll
                    for (int x = 0; x < 2; ++x) {                     // 16 columns: the even ones' result in o[4 d + 2 x], the odd ones' in the next
                        uint32_t even0, odd0, even1, odd1;
                        q8_halves<E4M3, true>(w[2 * x], even0, odd0);
                        q8_halves<E4M3, true>(w[2 * x + 1], even1, odd1);
                        mma_16816<false>(o[4 * d + 2 * x], hi, even0, even1);
                        mma_16816<false>(o[4 * d + 2 * x + 1], hi, odd0, odd1);
                        if (!SMALL) {
                            mma_16816<false>(o[4 * d + 2 * x], lo, even0, even1);
                            mma_16816<false>(o[4 * d + 2 * x + 1], lo, odd0, odd1);
                        }
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
        stage = stage + 1 == C::kStages ? 0 : stage + 1;
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
                s_m2[warp][row] = m2[h];
            }
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            const int row = (lane >> 2) + 8 * h;
            float top = s_m2[0][row];
#pragma unroll
            for (int w = 1; w < PA_WARPS; ++w) top = fmaxf(top, s_m2[w][row]);
            // (a warp without tokens has maximum -infinity, sum 0 and result 0, and contributes 2^-inf = 0 times that; a NaN stays one)
            const float f = paged_exp2(m2[h] - (top == -INFINITY ? 0.f : top));
            if (row < rows) {
#pragma unroll
                for (int n = 0; n < DP / 8; n += 2)                   // 16 columns: this lane's four
                    *reinterpret_cast<float4*>(sm_o + (warp * p.rows + row) * C::kPitch + n * 8 + (lane & 3) * 4) =
                        make_float4(o[n][2 * h] * f, o[n + 1][2 * h] * f, o[n][2 * h + 1] * f, o[n + 1][2 * h + 1] * f);
            }
        }
        __syncthreads();
        const bool began_here = !(cut_front && seg == 1);
        const bool whole = began_here && ends;
        const long long slot = 2ll * blockIdx.x + (began_here ? 1 : 0);
        for (int i = tid; i < rows * (DP / 4); i += PA_THREADS) {
            const int row = i / (DP / 4), c = (i - row * (DP / 4)) * 4;
            float t = s_m[0][row], t2 = s_m2[0][row];
#pragma unroll
            for (int w = 1; w < PA_WARPS; ++w) {
                t = fmaxf(t, s_m[w][row]);
                t2 = fmaxf(t2, s_m2[w][row]);
            }
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
                // (every weight 0: the result is 0)
                const float inv = sum == 0.f ? 0.f : exp2f((t2 == -INFINITY ? 0.f : t2) - (t == -INFINITY ? 0.f : t)) / sum;
                if (c < p.dim)
                    *reinterpret_cast<uint2*>(p.out + orow * p.dim + c) =
                        make_uint2(pack_pair<BF16>(x.x * inv, x.y * inv), pack_pair<BF16>(x.z * inv, x.w * inv));
                if (c == 0 && p.lse) p.lse[orow] = sum == 0.f ? -INFINITY : (t + log2f(sum)) * 0.69314718055994531f;
            } else {
                if (c < p.dim) *reinterpret_cast<float4*>(p.part_o + (slot * p.rows + row) * p.dim + c) = x;
                if (c == 0) {
                    p.part_ml[(slot * 2) * PA_ROWS + row] = t;
                    p.part_ml[(slot * 2 + 1) * PA_ROWS + row] = sum;
                    p.part_m2[slot * PA_ROWS + row] = t2;
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
template <bool BF16>
__global__ void __launch_bounds__(PA_JOIN_THREADS) paged_join_q8_kernel(const PagedQ8Params p, int ctas) {
    __shared__ float s_w[PA_JOIN_THREADS], s_red[4], s_red2[4];
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
    // the maxima, then the weights' sum
    float top = -INFINITY, top2 = -INFINITY;
    for (int i = tid; i < n; i += PA_JOIN_THREADS) {
        top = fmaxf(top, p.part_ml[place(i) * 2 * PA_ROWS + row]);
        top2 = fmaxf(top2, p.part_m2[place(i) * PA_ROWS + row]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        top2 = fmaxf(top2, __shfl_xor_sync(0xffffffffu, top2, o));
    }
    if (lane == 0) {
        s_red[warp] = top;
        s_red2[warp] = top2;
    }
    __syncthreads();
    top = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
    top2 = fmaxf(fmaxf(s_red2[0], s_red2[1]), fmaxf(s_red2[2], s_red2[3]));
    const float base = top == -INFINITY ? 0.f : top, base2 = top2 == -INFINITY ? 0.f : top2;
    __syncthreads();
    const int cols = p.dim / 4, lanes = cols <= 32 ? 32 : 64, groups = PA_JOIN_THREADS / lanes;
    const int g = tid / lanes, c = tid - g * lanes;
    float sum = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0; i0 < n; i0 += PA_JOIN_THREADS) {                 // (in order: the same result every time)
        const int i = i0 + tid;
        float w = 0.f;
        if (i < n) {
            sum += paged_exp2(p.part_ml[place(i) * 2 * PA_ROWS + row] - base) * p.part_ml[(place(i) * 2 + 1) * PA_ROWS + row];
            w = paged_exp2(p.part_m2[place(i) * PA_ROWS + row] - base2);
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
        const float inv = sum == 0.f ? 0.f : exp2f(base2 - base) / sum;
        *reinterpret_cast<uint2*>(p.out + orow * p.dim + c * 4) =
            make_uint2(pack_pair<BF16>(x.x * inv, x.y * inv), pack_pair<BF16>(x.z * inv, x.w * inv));
        if (c == 0 && p.lse) p.lse[orow] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
    }
}

}  // namespace mmv

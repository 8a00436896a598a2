// Linear attention with a decay per head:  S_t = exp(g) S_{t-1} + k_t v_t^T,  o_t = scale q_t S_t.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "common.cuh"

namespace mmv {

struct LinParams {
    const uint16_t *q, *k, *v;
    long long q_tok, q_head, k_tok, k_head, v_tok, v_head;   // element strides
    int heads, group;                                        // query heads; query heads per key / value head
    int dk, dv;
    const float* log_decay;                                  // [heads]
    float scale;
    uint16_t* out;                                           // [token, heads, dv]
    // single tokens
    const float* state;                                      // [num_slots, heads, dk, dv]
    float* state_out;
    const int32_t* slots;                                    // request -> state; null: its own index
    long long nreq, num_slots;
    int parts;                                               // column parts of a state
    // packed prompts
    const int32_t* offsets;
    long long nseq, ntok;
    WorkspaceHeader* hdr;
    float* carry;                                            // [CTA][padded dk][128]: what a range adds to a state
    uint64_t budget_ns;                                      // bound of every wait
};

template <bool BF16>
__device__ __forceinline__ float lin_load(const uint16_t* p) {
    if constexpr (BF16) return __uint_as_float(static_cast<uint32_t>(*p) << 16);
    else return __half2float(*reinterpret_cast<const __half*>(p));
}
template <bool BF16>
__device__ __forceinline__ uint16_t lin_store(float x) {
    if constexpr (BF16) return __bfloat16_as_ushort(__float2bfloat16_rn(x));
    else return __half_as_ushort(__float2half_rn(x));
}

// exp(g) as the sum of two fp32 values.  Rounded to one, its error (up to 2^-24 of itself, the same for every token) would
// add up over all the tokens that a slow decay reaches; a state is multiplied as fma(S, hi, fma(S, lo, update)).
struct LinDecay {
    float hi, lo;
};
__device__ __forceinline__ LinDecay lin_decay(float log_decay, int tokens) {
    const double x = exp(static_cast<double>(log_decay) * tokens);
    LinDecay d;
    d.hi = static_cast<float>(x);
    d.lo = static_cast<float>(x - d.hi);
    return d;
}

// One token per request.  The state is the traffic (8 bytes per element against 5 flops): a CTA owns COLS columns of one
// (request, head) and streams their dk rows once, 16 bytes per thread, LIN_STEP_AHEAD rows in flight; columns do not
// depend on one another, so a state is cut by columns and nothing is joined across CTAs.  Row partial sums of
// q S stay in registers and meet in shared memory at the end.
constexpr int LIN_STEP_THREADS = 256;
constexpr int LIN_STEP_AHEAD = 8;

template <bool BF16, int COLS>
__global__ void __launch_bounds__(LIN_STEP_THREADS) linear_step_kernel(LinParams p) {
    constexpr int LANES = COLS / 4;                              // threads per row
    constexpr int ROWS = LIN_STEP_THREADS / LANES;               // rows per sweep
    __shared__ float s_q[128], s_k[128];
    __shared__ float4 s_o[ROWS][LANES];
    __shared__ LinDecay s_decay;
    long long w = blockIdx.x;
    const int part = static_cast<int>(w % p.parts);
    w /= p.parts;
    const int h = static_cast<int>(w % p.heads), hk = h / p.group;
    const long long r = w / p.heads;
    const int tid = threadIdx.x, lane = tid % LANES, row = tid / LANES;
    const int col = part * COLS + lane * 4;
    const long long slot = p.slots ? static_cast<long long>(p.slots[r]) : r;
    uint16_t* out = p.out + (r * p.heads + h) * p.dv;
    if (slot < 0 || slot >= p.num_slots) {                       // no state: nothing is kept, the result is zero
        for (int c = part * COLS + tid; c < min(p.dv, (part + 1) * COLS); c += LIN_STEP_THREADS) out[c] = 0;
        return;
    }
    const long long base = (slot * p.heads + h) * static_cast<long long>(p.dk) * p.dv;
    const float* src = p.state + base;
    float* dst = p.state_out + base;
    float4 s[LIN_STEP_AHEAD];
    const bool mine = col < p.dv;
#pragma unroll
    for (int i = 0; i < LIN_STEP_AHEAD; ++i) {
        const int d = row + i * ROWS;
        if (mine && d < p.dk) s[i] = *reinterpret_cast<const float4*>(src + static_cast<long long>(d) * p.dv + col);
    }
    for (int d = tid; d < p.dk; d += LIN_STEP_THREADS) {
        s_q[d] = lin_load<BF16>(p.q + r * p.q_tok + h * p.q_head + d);
        s_k[d] = lin_load<BF16>(p.k + r * p.k_tok + hk * p.k_head + d);
    }
    if (tid == 0) s_decay = lin_decay(p.log_decay[h], 1);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f), o = v;
    if (mine) {
        const uint16_t* pv = p.v + r * p.v_tok + hk * p.v_head + col;
        v = make_float4(lin_load<BF16>(pv), lin_load<BF16>(pv + 1), lin_load<BF16>(pv + 2), lin_load<BF16>(pv + 3));
    }
    __syncthreads();
    const LinDecay decay = s_decay;
    for (int d0 = row; d0 < p.dk; d0 += ROWS * LIN_STEP_AHEAD) {
#pragma unroll
        for (int i = 0; i < LIN_STEP_AHEAD; ++i) {
            const int d = d0 + i * ROWS;
            if (mine && d < p.dk) {
                float4 x = s[i];
                const float kd = s_k[d], qd = s_q[d];
                x.x = fmaf(x.x, decay.hi, fmaf(x.x, decay.lo, kd * v.x));
                x.y = fmaf(x.y, decay.hi, fmaf(x.y, decay.lo, kd * v.y));
                x.z = fmaf(x.z, decay.hi, fmaf(x.z, decay.lo, kd * v.z));
                x.w = fmaf(x.w, decay.hi, fmaf(x.w, decay.lo, kd * v.w));
                o.x = fmaf(qd, x.x, o.x);
                o.y = fmaf(qd, x.y, o.y);
                o.z = fmaf(qd, x.z, o.z);
                o.w = fmaf(qd, x.w, o.w);
                *reinterpret_cast<float4*>(dst + static_cast<long long>(d) * p.dv + col) = x;
                const int n = d + ROWS * LIN_STEP_AHEAD;
                if (n < p.dk) s[i] = *reinterpret_cast<const float4*>(src + static_cast<long long>(n) * p.dv + col);
            }
        }
    }
    s_o[row][lane] = o;
    __syncthreads();
    for (int c = tid; c < COLS; c += LIN_STEP_THREADS) {
        if (part * COLS + c < p.dv) {
            float x = 0.f;
#pragma unroll 4
            for (int i = 0; i < ROWS; ++i) x += reinterpret_cast<const float*>(s_o[i])[c];
            out[part * COLS + c] = lin_store<BF16>(p.scale * x);
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// Packed prompts, 64 tokens (a chunk) at a time on the tensor cores.  With S the state in front of a chunk of n tokens:
//     A_ij = exp(g (i - j)) q_i . k_j  for j <= i, else 0
//     o_i  = scale (exp(g (i + 1)) q_i S + sum_j A_ij v_j)
//     S'   = exp(g n) S + sum_j exp(g (n - 1 - j)) k_j v_j^T
// so a chunk is four products with a 128-row accumulator each (transposed: rows are columns of v, or keys):
//     AT = K Q^T,   KV = V^T K',   O1 = S^T Q^T,   O2 = V^T A^T
//
// The state lives in fp32 registers, one row (a column of v) per thread, half of its columns in either of two warpgroups.
// Operands that are formed here are sums of bfloat16 values: the copy of S that meets the queries and A two (2^-16 relative,
// well under the result's own rounding), the decayed keys K' three, so that the fp32 state stays exact to its own
// rounding (two would leave 2^-17 of every update).
//
// Roles of a CTA (one per SM): two warpgroups keep the state, one forms K', one forms A and stores results, one warp issues the loads
// and one the products; they meet at mbarriers only.  Two chunks' q, k, v are in shared memory, the next landing while one
// is worked on.
//
// Split: the list of (sequence, head, chunk) is cut into equal contiguous ranges, one per CTA.  A range that ends inside a
// (sequence, head) hands its state on; a first, short kernel (CARRY: the same code with keys and values only) computes what the
// part behind its last start adds to a state, and a range that starts inside one sums the decayed contributions of the
// ranges in front of it.  Batches of many sequences are hardly cut; one long prompt reads its keys and values twice.
// ---------------------------------------------------------------------------------------------------------------------
constexpr int LIN_C = 64;                                   // tokens of a chunk
constexpr int LIN_WORKERS = 16;                             // warps: state 0-7, keys 8-11, scores and results 12-15
constexpr int LIN_WARP_LOAD = 16, LIN_WARP_MMA = 17;
constexpr int LIN_THREADS = 18 * 32;
constexpr int LIN_BOX = LIN_C * 128;                        // bytes of 64 tokens x 64 columns, 128-byte rows, 128-byte swizzle
constexpr int LIN_MIN_UNITS = 4;                            // chunks that a range has at least

template <int DK, bool CARRY>
struct LinCfg {
    static constexpr int kBoxes = DK / 64;
    static constexpr int kStages = 2;
    static constexpr int kQ = 0;
    static constexpr int kK = CARRY ? 0 : kBoxes * LIN_BOX;
    static constexpr int kV = kK + kBoxes * LIN_BOX;        // (the product K Q^T reads 64 rows past K: they are V's)
    static constexpr int kStage = kV + 2 * LIN_BOX;
    static constexpr int kKp = kStages * kStage;            // three parts of K'
    static constexpr int kA = kKp + 3 * kBoxes * LIN_BOX;   // two parts of A
    static constexpr int kOPitch = 272;
    static constexpr int kO = kA + (CARRY ? 0 : 2 * LIN_BOX);
    static constexpr int kSmemBytes = kO + (CARRY ? 0 : LIN_C * kOPitch) + 1024;      // (+ alignment)
    static constexpr uint32_t kTmemCols = CARRY ? DK : 512;
    // columns of tensor memory
    static constexpr uint32_t kColKV = 0, kColS = 128, kColAT = 256, kColO1 = 384, kColO2 = 448;
};

struct LinBars {
    uint64_t full[2], empty[2], at_full[2], at_empty[2];
    uint64_t kp_full, kv_full, kv_empty, s_full, s_free, a_full, o_full, o_empty, drain;
};

// A place in the list of (sequence, head, chunk).
struct LinIter {
    int seq, head, chunk, chunks, tok, len;                 // tok: first token of the sequence
};
__device__ __forceinline__ bool lin_sequence(const LinParams& p, int s, int& tok, int& len) {
    const int lo = p.offsets[s], hi = p.offsets[s + 1];
    const bool ok = lo >= 0 && hi >= lo && hi <= p.ntok;
    tok = ok ? lo : 0;
    len = ok ? hi - lo : 0;
    return ok;
}
__device__ __forceinline__ int lin_chunks(int len) { return static_cast<int>((static_cast<unsigned>(len) + LIN_C - 1) / LIN_C); }
__device__ __forceinline__ void lin_enter(const LinParams& p, LinIter& it) {
    lin_sequence(p, it.seq, it.tok, it.len);
    it.chunks = lin_chunks(it.len);
}
__device__ __forceinline__ void lin_next(const LinParams& p, LinIter& it) {          // (the caller knows that there is a next one)
    if (++it.chunk < it.chunks) return;
    it.chunk = 0;
    if (++it.head < p.heads) return;
    it.head = 0;
    do {
        ++it.seq;
        lin_enter(p, it);
    } while (it.chunks == 0);
}
__device__ __forceinline__ int lin_tokens(const LinIter& it) { return min(LIN_C, it.len - it.chunk * LIN_C); }
__device__ __forceinline__ long long lin_first(long long c, long long units, int ctas) { return c * units / ctas; }
__device__ __forceinline__ float lin_power(float g, int n) { return n == 0 ? 1.f : expf(g * static_cast<float>(n)); }

// Descriptor of an operand whose rows (128 bytes, 128-byte swizzle) run along M or N: `lbo` bytes between blocks of 64 of
// them, 1024 between groups of 8 along K.  Along K (make_desc): 1024 between groups of 8 rows.
__device__ __forceinline__ uint64_t lin_desc_mn(uint32_t addr, uint32_t lbo) {
    return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(lbo >> 4) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) |
           (static_cast<uint64_t>(1) << 46) | (static_cast<uint64_t>(2) << 61);
}
// Both operands bfloat16, fp32 accumulator, M = 128; A / B with their rows along M / N.
__host__ __device__ constexpr uint32_t lin_idesc(uint32_t N, bool a_mn, bool b_mn) {
    return make_idesc_f16_f32(128, N) | (1u << 7) | (1u << 10) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u);
}

// Two fp32 values as a pair of bfloat16, and what that leaves of them.
__device__ __forceinline__ uint32_t lin_peel(float& a, float& b) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
    const uint32_t w = *reinterpret_cast<const uint32_t*>(&x);
    a -= __uint_as_float(w << 16);
    b -= __uint_as_float(w & 0xffff0000u);
    return w;
}
// A wait of a whole warp: all of its lanes get the same answer.
__device__ __forceinline__ bool lin_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, uint64_t budget_ns) {
    return __all_sync(0xffffffffu, wait_bar(bar, parity, abort_flag, budget_ns));
}
// The four warps of scores and results: whether all of them say yes (they leave together when a wait has given up).
__device__ __forceinline__ bool lin_group_all(bool ok) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"(static_cast<uint32_t>(ok)) : "memory");
    return r != 0;
}
__device__ __forceinline__ void lin_group_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

template <int DK, bool CARRY>
__global__ void __launch_bounds__(LIN_THREADS, 1)
linear_chunks_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v, const LinParams p) {
    using C = LinCfg<DK, CARRY>;
    constexpr int HALF = DK / 2;                            // state columns of a thread
    extern __shared__ uint8_t lin_smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(lin_smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    __shared__ LinBars bars;
    __shared__ long long s_sum[LIN_THREADS / 32];
    __shared__ long long s_skip;
    __shared__ int s_seq;
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    __shared__ float s_pw[LIN_C + 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    volatile int* abort_flag = &s_abort;
    griddep_launch_dependents();

    // ---- the list, this CTA's range of it ---------------------------------------------------------------------------------
    const int nseq = static_cast<int>(p.nseq);
    const int per = (nseq + LIN_THREADS - 1) / LIN_THREADS, q_lo = min(nseq, tid * per), q_hi = min(nseq, q_lo + per);
    long long mine = 0;
    bool bad = false;
    for (int s = q_lo; s < q_hi; ++s) {
        int tok, len;
        bad |= !lin_sequence(p, s, tok, len);
        mine += lin_chunks(len);
    }
    long long inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
    }
    if (lane == 31) s_sum[warp] = inc;
    if (tid == 0) {
        s_abort = 0;
        s_seq = -1;
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars.full[i], 1);
            mbar_init(&bars.empty[i], 1);
            mbar_init(&bars.at_full[i], 1);
            mbar_init(&bars.at_empty[i], 2);
        }
        mbar_init(&bars.kp_full, 4);
        mbar_init(&bars.kv_full, 1);
        mbar_init(&bars.kv_empty, 8);
        mbar_init(&bars.s_full, 8);
        mbar_init(&bars.s_free, 1);
        mbar_init(&bars.a_full, 2);
        mbar_init(&bars.o_full, 1);
        mbar_init(&bars.o_empty, 4);
        mbar_init(&bars.drain, 1);
        mbar_fence_init();
    }
    const bool any_bad = __syncthreads_or(bad);
    long long before = inc - mine, total = 0;
    for (int w = 0; w < LIN_THREADS / 32; ++w) {
        if (w < warp) before += s_sum[w];
        total += s_sum[w];
    }
    const long long units = total * p.heads;
    const int ctas = static_cast<int>(min(static_cast<long long>(gridDim.x), max(1ll, units / LIN_MIN_UNITS)));
    const int cta = blockIdx.x;
    if constexpr (CARRY) {
        if (cta == 0 && tid == 0) {
            p.hdr->tile_counter = 0u;
            p.hdr->error = any_bad ? 4u : 0u;               // MMV_ERR_BAD_SEGMENTS
        }
        // sequences without tokens: their state is handed through
        if (p.state_out)
            for (int s = cta; s < nseq; s += gridDim.x) {
                int tok, len;
                lin_sequence(p, s, tok, len);
                if (len) continue;
                const long long n = static_cast<long long>(p.heads) * p.dk * p.dv;
                for (long long i = tid; i < n; i += LIN_THREADS) p.state_out[s * n + i] = p.state ? p.state[s * n + i] : 0.f;
            }
    }
    if (cta >= ctas || units == 0) return;
    long long u0 = lin_first(cta, units, ctas);
    const long long u1 = lin_first(cta + 1ll, units, ctas);
    {
        const long long u = CARRY ? u1 - 1 : u0;            // find its (sequence, head, chunk)
        if (u >= before * p.heads && u < (before + mine) * p.heads) {
            long long at = before * p.heads;
            int s = q_lo, tok, len;
            lin_sequence(p, s, tok, len);
            while (u >= at + static_cast<long long>(lin_chunks(len)) * p.heads) {
                at += static_cast<long long>(lin_chunks(len)) * p.heads;
                lin_sequence(p, ++s, tok, len);
            }
            s_seq = s;
            s_skip = u - at;
        }
    }
    __syncthreads();
    LinIter start;
    start.seq = s_seq;
    lin_enter(p, start);
    start.head = static_cast<int>(s_skip / start.chunks);
    start.chunk = static_cast<int>(s_skip - static_cast<long long>(start.head) * start.chunks);
    if constexpr (CARRY) {
        if (start.chunk + 1 == start.chunks) return;        // the range ends where a (sequence, head) does: nothing to hand on
        const int back = static_cast<int>(min(static_cast<long long>(start.chunk), u1 - 1 - u0));
        start.chunk -= back;
        u0 = u1 - 1 - back;
    }
    const int count = static_cast<int>(u1 - u0);

    if (warp == LIN_WARP_MMA) {
        tmem_alloc(&s_tmem, C::kTmemCols);
        tmem_relinquish();
        tc_fence_before_sync();
    }
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = s_tmem;
    if constexpr (!CARRY) griddep_wait();                   // the carried states, and the status word, are there

    const uint64_t budget = p.budget_ns;
    LinIter it = start;
    bool ok = true;

    if (warp < 8) {
        // ---- the state: rows = columns of v (lanes of tensor memory), HALF columns of k per thread ------------------------
        const int half = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        const bool stored = row < p.dv;
        float s[HALF];
        LinDecay whole{};
        float g = 0.f;
        for (int c = 0; c < count; ++c) {
            const int n = lin_tokens(it);
            const long long base = ((static_cast<long long>(it.seq) * p.heads + it.head) * p.dk + half * HALF) * p.dv + row;
            if (c == 0 || it.chunk == 0) {
                g = p.log_decay[it.head];
                whole = lin_decay(g, LIN_C);
#pragma unroll
                for (int i = 0; i < HALF; ++i) s[i] = 0.f;
                if (!CARRY && p.state && stored) {
                    const float f = it.chunk == 0 ? 1.f : static_cast<float>(exp(static_cast<double>(g) * (static_cast<double>(it.chunk) * LIN_C)));
                    if (f != 0.f)
#pragma unroll
                        for (int i = 0; i < HALF; ++i) {
                            if (half * HALF + i < p.dk) s[i] = f * p.state[base + static_cast<long long>(i) * p.dv];
                            if (i % 16 == 15) asm volatile("" ::: "memory");        // (16 loads in flight: registers)
                        }
                }
                if (!CARRY && it.chunk > 0) {
                    const long long seg = u0 - it.chunk;    // first unit of this (sequence, head)
                    for (int j = cta - 1; j >= 0; --j) {
                        const long long end = lin_first(j + 1ll, units, ctas);
                        if (end <= seg) break;
                        const double lag = static_cast<double>(u0 - end) * LIN_C;
                        const float f = u0 == end ? 1.f : static_cast<float>(exp(static_cast<double>(g) * lag));
                        if (f == 0.f) break;                // (and those in front of it weigh less)
                        const float* src = p.carry + (static_cast<long long>(j) * DK + half * HALF) * 128 + row;
#pragma unroll
                        for (int i = 0; i < HALF; ++i) {
                            s[i] = fmaf(f, src[i * 128], s[i]);
                            if (i % 16 == 15) asm volatile("" ::: "memory");
                        }
                    }
                }
            }
            if constexpr (!CARRY) {
                if (c > 0) ok = lin_wait(&bars.s_free, (c - 1) & 1, abort_flag, budget);
                if (!ok) break;
                tc_fence_after_sync();
#pragma unroll
                for (int b = 0; b < HALF / 16; ++b) {
                    uint32_t hi[8], lo[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float x = s[b * 16 + 2 * i], y = s[b * 16 + 2 * i + 1];
                        hi[i] = lin_peel(x, y);
                        lo[i] = lin_peel(x, y);
                    }
                    const uint32_t at = lanes + C::kColS + half * (HALF / 2) + b * 8;
                    tmem_st_32x8(at, hi);
                    tmem_st_32x8(at + DK / 2, lo);
                }
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.s_full);
            }
            const LinDecay d = n == LIN_C ? whole : lin_decay(g, n);
            ok = lin_wait(&bars.kv_full, c & 1, abort_flag, budget);
            if (!ok) break;
            tc_fence_after_sync();
#pragma unroll
            for (int b = 0; b < HALF / 16; ++b) {
                uint32_t r[16];
                tmem_ld_32x16(lanes + C::kColKV + half * HALF + b * 16, r);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b * 16 + i] = fmaf(s[b * 16 + i], d.hi, fmaf(s[b * 16 + i], d.lo, __uint_as_float(r[i])));
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.kv_empty);
            if (!CARRY && it.chunk + 1 == it.chunks && p.state_out && stored) {
#pragma unroll
                for (int i = 0; i < HALF; ++i)
                    if (half * HALF + i < p.dk) p.state_out[base + static_cast<long long>(i) * p.dv] = s[i];
            }
            if (c + 1 < count) lin_next(p, it);
        }
        if (CARRY && ok) {
            float* dst = p.carry + (static_cast<long long>(cta) * DK + half * HALF) * 128 + row;
#pragma unroll
            for (int i = 0; i < HALF; ++i) dst[i * 128] = s[i];
        }
    } else if (warp < 12) {
        // ---- K': a thread scales half of a token's key ------------------------------------------------------------------------
        const int t = tid - 256, j = t >> 1, part = t & 1;
        for (int c = 0; c < count; ++c) {
            const int n = lin_tokens(it), stage = c % C::kStages;
            const float f = j < n ? lin_power(p.log_decay[it.head], n - 1 - j) : 0.f;
            ok = lin_wait(&bars.full[stage], (c / C::kStages) & 1, abort_flag, budget);
            if (ok && c > 0) ok = lin_wait(&bars.kv_full, (c - 1) & 1, abort_flag, budget);      // the product has read the last K'
            if (!ok) break;
            const uint8_t* src = smem + stage * C::kStage + C::kK;
            uint8_t* dst = smem + C::kKp;
#pragma unroll
            for (int i = 0; i < DK / 16; ++i) {
                // the two threads of a token read different banks
                const int box = DK == 128 ? part : 0, chunk = DK == 128 ? i ^ (part << 2) : i + (part << 2);
                const uint32_t at = box * LIN_BOX + swz_offset<128>(j, chunk * 16);
                const uint4 w = *reinterpret_cast<const uint4*>(src + at);
                const uint32_t in[4] = {w.x, w.y, w.z, w.w};
                uint32_t a[4], b[4], d[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = __uint_as_float(in[e] << 16) * f, y = __uint_as_float(in[e] & 0xffff0000u) * f;
                    if (j >= n) x = y = 0.f;                // (another sequence's token: whatever it holds)
                    a[e] = lin_peel(x, y);
                    b[e] = lin_peel(x, y);
                    d[e] = lin_peel(x, y);
                }
                *reinterpret_cast<uint4*>(dst + at) = make_uint4(a[0], a[1], a[2], a[3]);
                *reinterpret_cast<uint4*>(dst + C::kBoxes * LIN_BOX + at) = make_uint4(b[0], b[1], b[2], b[3]);
                *reinterpret_cast<uint4*>(dst + 2 * C::kBoxes * LIN_BOX + at) = make_uint4(d[0], d[1], d[2], d[3]);
            }
            if (j >= n) {                                   // a zero weight does not hide a value that is not finite
                uint8_t* v = smem + stage * C::kStage + C::kV + part * LIN_BOX + j * 128;
#pragma unroll
                for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4*>(v + i * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.kp_full);
            if (c + 1 < count) lin_next(p, it);
        }
    } else if (warp < LIN_WORKERS) {
        if constexpr (!CARRY) {
            // ---- A, then the chunk's results ------------------------------------------------------------------------------
            const int w = warp - 12, t = tid - 384;
            const uint32_t lanes = tmem + (static_cast<uint32_t>(w * 32) << 16);
            const int j = t;                                // A: key j of queries i = 0..63 (warps 12 and 13)
            for (int c = 0; c < count; ++c) {
                const int n = lin_tokens(it);
                if (c == 0 || it.chunk == 0) {
                    lin_group_sync();
                    if (t <= LIN_C) s_pw[t] = lin_power(p.log_decay[it.head], t);
                    lin_group_sync();
                }
                if (w < 2) {
                    // (o_full of chunk c - 1, waited for below, says that the product has read the last A)
                    ok = lin_wait(&bars.at_full[c & 1], (c >> 1) & 1, abort_flag, budget);
                }
                if (w < 2 && ok) {
                    tc_fence_after_sync();
                    uint8_t* dst = smem + C::kA;
#pragma unroll
                    for (int b = 0; b < LIN_C / 16; ++b) {
                        uint32_t r[16];
                        tmem_ld_32x16(lanes + C::kColAT + (c & 1) * 64 + b * 16, r);
                        tmem_ld_wait();
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            uint32_t hi[4], lo[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int i = b * 16 + q * 8 + e * 2;
                                float x = i >= j && j < n ? __uint_as_float(r[q * 8 + e * 2]) * s_pw[max(i - j, 0)] : 0.f;
                                float y = i + 1 >= j && j < n ? __uint_as_float(r[q * 8 + e * 2 + 1]) * s_pw[max(i + 1 - j, 0)] : 0.f;
                                hi[e] = lin_peel(x, y);
                                lo[e] = lin_peel(x, y);
                            }
                            const uint32_t at = swz_offset<128>(j, (b * 2 + q) * 16);
                            *reinterpret_cast<uint4*>(dst + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                            *reinterpret_cast<uint4*>(dst + LIN_BOX + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                        }
                    }
                    tc_fence_before_sync();
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(&bars.at_empty[c & 1]);
                        mbar_arrive(&bars.a_full);
                    }
                }
                if (ok) ok = lin_wait(&bars.o_full, c & 1, abort_flag, budget);
                ok = lin_group_all(ok);                     // (and the last chunk's results have left the staging rows)
                if (!ok) break;
                tc_fence_after_sync();
                uint8_t* stage = smem + C::kO;
#pragma unroll
                for (int b = 0; b < LIN_C / 16; ++b) {
                    uint32_t x[16], y[16];
                    tmem_ld_32x16(lanes + C::kColO1 + b * 16, x);
                    tmem_ld_32x16(lanes + C::kColO2 + b * 16, y);
                    tmem_ld_wait();
                    if (b == LIN_C / 16 - 1) {
                        tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&bars.o_empty);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float o = p.scale * fmaf(s_pw[b * 16 + i + 1], __uint_as_float(x[i]), __uint_as_float(y[i]));
                        *reinterpret_cast<uint16_t*>(stage + (b * 16 + i) * C::kOPitch + t * 2) = __bfloat16_as_ushort(__float2bfloat16_rn(o));
                    }
                }
                lin_group_sync();
                const int words = p.dv / 8;
                uint16_t* out = p.out + ((static_cast<long long>(it.tok) + it.chunk * LIN_C) * p.heads + it.head) * p.dv;
                for (int i = t; i < n * words; i += 128) {
                    const int r = i / words, q = i - r * words;
                    *reinterpret_cast<uint4*>(out + static_cast<long long>(r) * p.heads * p.dv + q * 8) =
                        *reinterpret_cast<const uint4*>(stage + r * C::kOPitch + q * 16);
                }
                if (c + 1 < count) lin_next(p, it);
            }
        }
    } else if (warp == LIN_WARP_LOAD) {
        if (lane == 0) {
            const int vboxes = p.dv > 64 ? 2 : 1;
            const uint32_t bytes = ((CARRY ? 1 : 2) * C::kBoxes + vboxes) * LIN_BOX;
            for (int c = 0; c < count; ++c) {
                const int stage = c % C::kStages;
                if (c >= C::kStages) ok = wait_bar(&bars.empty[stage], (c / C::kStages - 1) & 1, abort_flag, budget);
                if (!ok) break;
                uint8_t* dst = smem + stage * C::kStage;
                const int tok = it.tok + it.chunk * LIN_C, hk = it.head / p.group;
                mbar_arrive_expect_tx(&bars.full[stage], bytes);
#pragma unroll
                for (int b = 0; b < C::kBoxes; ++b) {
                    if (!CARRY) tma_load_3d(dst + C::kQ + b * LIN_BOX, &map_q, &bars.full[stage], b * 64, it.head, tok);
                    tma_load_3d(dst + C::kK + b * LIN_BOX, &map_k, &bars.full[stage], b * 64, hk, tok);
                }
                for (int b = 0; b < vboxes; ++b) tma_load_3d(dst + C::kV + b * LIN_BOX, &map_v, &bars.full[stage], b * 64, hk, tok);
                if (c + 1 < count) lin_next(p, it);
            }
        }
        __syncwarp();
    } else {
        if (lane == 0) {
            constexpr uint32_t kIdescAT = lin_idesc(LIN_C, false, false), kIdescKV = lin_idesc(DK, true, true);
            constexpr uint32_t kIdescO1 = lin_idesc(LIN_C, false, false), kIdescO2 = lin_idesc(LIN_C, true, true);
            const uint32_t sm = smem_u32(smem);
            const auto scores = [&](int c) {                // AT = K Q^T
                const uint32_t st = sm + (c % C::kStages) * C::kStage;
#pragma unroll
                for (int k = 0; k < DK / 16; ++k) {
                    const uint32_t at = (k >> 2) * LIN_BOX + (k & 3) * 32;
                    mma_f16_ss(tmem + C::kColAT + (c & 1) * 64, make_desc(st + C::kK + at, 1024, 2), make_desc(st + C::kQ + at, 1024, 2),
                               kIdescAT, k > 0);
                }
                tc_commit(&bars.at_full[c & 1]);
            };
            const auto scores_wait = [&](int c) {
                bool r = wait_bar(&bars.full[c % C::kStages], (c / C::kStages) & 1, abort_flag, budget);
                if (r && c >= 2) r = wait_bar(&bars.at_empty[c & 1], ((c >> 1) - 1) & 1, abort_flag, budget);
                tc_fence_after_sync();
                return r;
            };
            if (!CARRY) {
                ok = scores_wait(0);
                if (ok) scores(0);
            }
            for (int c = 0; ok && c < count; ++c) {
                const int stage = c % C::kStages;
                const uint32_t st = sm + stage * C::kStage;
                ok = wait_bar(&bars.full[stage], (c / C::kStages) & 1, abort_flag, budget) && wait_bar(&bars.kp_full, c & 1, abort_flag, budget);
                if (ok && c > 0) ok = wait_bar(&bars.kv_empty, (c - 1) & 1, abort_flag, budget);
                if (!ok) break;
                tc_fence_after_sync();
#pragma unroll
                for (int x = 0; x < 3; ++x)                 // KV = V^T K'
#pragma unroll
                    for (int k = 0; k < LIN_C / 16; ++k)
                        mma_f16_ss(tmem + C::kColKV, lin_desc_mn(st + C::kV + k * 2048, LIN_BOX),
                                   lin_desc_mn(sm + C::kKp + x * C::kBoxes * LIN_BOX + k * 2048, LIN_BOX), kIdescKV, x > 0 || k > 0);
                tc_commit(&bars.kv_full);
                if constexpr (CARRY) {
                    tc_commit(&bars.empty[stage]);
                } else {
                    ok = wait_bar(&bars.s_full, c & 1, abort_flag, budget);
                    if (ok && c > 0) ok = wait_bar(&bars.o_empty, (c - 1) & 1, abort_flag, budget);
                    if (!ok) break;
                    tc_fence_after_sync();
#pragma unroll
                    for (int x = 0; x < 2; ++x)             // O1 = S^T Q^T
#pragma unroll
                        for (int k = 0; k < DK / 16; ++k)
                            mma_f16_ts(tmem + C::kColO1, tmem + C::kColS + x * (DK / 2) + k * 8,
                                       make_desc(st + C::kQ + (k >> 2) * LIN_BOX + (k & 3) * 32, 1024, 2), kIdescO1, x > 0 || k > 0);
                    tc_commit(&bars.s_free);
                    // the next chunk's scores go in front of this chunk's last product if its tokens are there already
                    bool ahead = false;
                    if (c + 1 < count && mbar_try_wait(&bars.full[(c + 1) % C::kStages], ((c + 1) / C::kStages) & 1)) {
                        ok = scores_wait(c + 1);
                        if (!ok) break;
                        scores(c + 1);
                        ahead = true;
                    }
                    ok = wait_bar(&bars.a_full, c & 1, abort_flag, budget);
                    if (!ok) break;
                    tc_fence_after_sync();
#pragma unroll
                    for (int x = 0; x < 2; ++x)             // O2 = V^T A^T
#pragma unroll
                        for (int k = 0; k < LIN_C / 16; ++k)
                            mma_f16_ss(tmem + C::kColO2, lin_desc_mn(st + C::kV + k * 2048, LIN_BOX),
                                       lin_desc_mn(sm + C::kA + x * LIN_BOX + k * 2048, LIN_BOX), kIdescO2, x > 0 || k > 0);
                    tc_commit(&bars.o_full);
                    tc_commit(&bars.empty[stage]);
                    if (!ahead && c + 1 < count) {
                        ok = scores_wait(c + 1);
                        if (!ok) break;
                        scores(c + 1);
                    }
                }
            }
            // products in flight end before the tensor memory is given back (all of them have, unless a wait gave up)
            tc_commit(&bars.drain);
            mbar_wait(&bars.drain, 0, budget);
        }
        __syncwarp();
    }
    if (!ok) {
        *abort_flag = 1;
        report_error(p.hdr, 5u);                            // MMV_ERR_TIMEOUT
    }
    __syncthreads();
    if (*abort_flag && tid == 0) {                          // loads in flight land before the CTA leaves
        for (int i = 0; i < C::kStages; ++i) mbar_wait(&bars.full[i], 0, 1000000), mbar_wait(&bars.full[i], 1, 1000000);
    }
    tc_fence_after_sync();
    if (warp == LIN_WARP_MMA) tmem_dealloc(tmem, C::kTmemCols);
}

}  // namespace mmv

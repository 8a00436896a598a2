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
static __device__ __noinline__ LinDecay lin_decay(float log_decay, double tokens) {
    const double x = exp(static_cast<double>(log_decay) * tokens);
    LinDecay d;
    d.hi = static_cast<float>(x);
    d.lo = static_cast<float>(x - d.hi);
    return d;
}

// One token per request.  The state is the traffic (8 bytes per element against 5 flops): a CTA owns COLS columns of one
// (request, head) and takes their dk rows with all loads in flight before the first store, 16 bytes per thread each (256
// states of 16 heads, 128 x 128: 89.8 us, 93 % of the copy rate; with half of the rows in flight 106.6); columns do not
// depend on one another, so a state is cut by columns where there are few (32 columns instead of 128: 4.9 us for the 16 states
// of one request) and nothing is joined across CTAs.  Row partial sums of q S stay in registers and meet in shared memory.
constexpr int LIN_STEP_THREADS = 256;

template <bool BF16, int COLS>
__global__ void __launch_bounds__(LIN_STEP_THREADS) linear_step_kernel(LinParams p) {
    constexpr int LANES = COLS / 4;                              // threads per row
    constexpr int ROWS = LIN_STEP_THREADS / LANES;               // rows side by side
    constexpr int MINE = 128 / ROWS;                             // rows of a thread
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
    float4 s[MINE];
    const bool mine = col < p.dv;
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
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
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        const int d = row + i * ROWS;
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
// The state lives in fp32 registers, one row (a column of v) per thread, half of its columns in each of two warpgroups.
// Operands that are formed here are sums of bfloat16 values: the copy of S that meets the queries and A two (2^-16 relative,
// well under the result's own rounding), the decayed keys K' three, so that the fp32 state stays exact to its own
// rounding (two would leave 2^-17 of every update).
//
// The roles' loops are kept short (few of them unrolled): five different ones run at a time on each scheduler, and unrolled they
// waited for instructions more than for anything else.
//
// Measured: one prompt of 65536 tokens, 16 heads of 128: 565 to 588 us (1.9 TB/s; 166 us is what the copy rate would allow, 249 with keys and
// values read twice); 16 prompts of 32768 tokens in all: 307 to 327 us.  Neither memory (28 %) nor the tensor pipe (26 % busy) bounds it:
// without the splits of the keys the first kernel takes 120 instead of 170 us and the second 285 instead of 331; the rest is roles that
// wait for one another.
//
// Roles of a CTA (one per SM): two warpgroups keep the state, one forms K', one stores results, two warps form A, one issues the loads
// and one the products; they meet at mbarriers.  Three chunks' q, k, v are in shared memory, the next ones landing while one
// is worked on.
//
// Split: the list of (sequence, head, chunk) is cut into equal contiguous ranges, one per CTA.  A range that ends inside a
// (sequence, head) hands its state on; a first, short kernel (CARRY: the same code with keys and values only) computes what the
// part behind its last start adds to a state, and a range that starts inside one sums the decayed contributions of the
// ranges in front of it.  One long prompt reads its keys and values twice; of a batch, the part of a cut (sequence, head) that lies in front of
// a range's end is, and the first kernel lasts as long as the longest such part.  A range is no
// shorter than half the root of the longest sequence's number of chunks: a sequence of n chunks cut into m ranges takes n / m
// chunks' time and up to m contributions', and of these two a chunk takes about twice as long.
// ---------------------------------------------------------------------------------------------------------------------
constexpr int LIN_C = 64;                                   // tokens of a chunk
// warps (a warp reaches the 32 lanes of tensor memory that its number modulo 4 says)
constexpr int LIN_STATE = 8;                                // of them keep the state: 2 of columns x 4 of rows
constexpr int LIN_WARP_KEYS = LIN_STATE, LIN_WARP_OUT = LIN_WARP_KEYS + 4, LIN_WARP_SCORES = LIN_WARP_OUT + 4;
constexpr int LIN_WARP_LOAD = LIN_WARP_SCORES + 2, LIN_WARP_MMA = LIN_WARP_LOAD + 1;
constexpr int LIN_THREADS = (LIN_WARP_MMA + 1) * 32;
constexpr int LIN_BOX = LIN_C * 128;                        // bytes of 64 tokens x 64 columns, 128-byte rows, 128-byte swizzle

template <int DK, bool CARRY>
struct LinCfg {
    static constexpr int kBoxes = DK / 64;
    static constexpr int kStages = 3;
    static constexpr int kKeyWarps = CARRY ? 8 : 4;         // that form K' (without results to store there are four more)
    static constexpr int kQ = 0;
    static constexpr int kK = CARRY ? 0 : kBoxes * LIN_BOX;
    static constexpr int kV = kK + kBoxes * LIN_BOX;        // (the product K Q^T reads 64 rows past K: they are V's)
    static constexpr int kStage = kV + 2 * LIN_BOX;
    static constexpr int kKp = kStages * kStage;            // three parts of K' for 32 tokens, twice
    static constexpr int kKpPart = kBoxes * LIN_BOX / 2, kKpBytes = 3 * kKpPart;
    static constexpr int kA = kKp + 2 * kKpBytes;           // two parts of A
    static constexpr int kOPitch = 256;
    static constexpr int kO = kA + (CARRY ? 0 : 2 * LIN_BOX);
    static constexpr int kSmemBytes = kO + (CARRY ? 0 : LIN_C * kOPitch);
    static constexpr int kUpdates = CARRY ? 2 : 1;          // accumulators of KV (there is room for a second without results)
    static constexpr uint32_t kTmemCols = CARRY ? 2 * DK : 512;
    // columns of tensor memory
    static constexpr uint32_t kColKV = 0, kColS = 128, kColAT = 256, kColO1 = 384, kColO2 = 448;
};

struct LinBars {
    uint64_t full[3], empty[3], at_full[2], at_empty[2];
    uint64_t kp_full[2], kv_done[2], kv_full[2], kv_empty[2], s_full, s_free, a_full, a_free, o_full, o_empty, drain;
};

// A place in the list of (sequence, head, chunk).
struct LinIter {
    int seq, head, chunk, chunks, tok, len;                 // tok: first token of the sequence
};
__device__ __forceinline__ bool lin_sequence(const int32_t* offsets, long long ntok, int s, int& tok, int& len) {
    const int lo = offsets[s], hi = offsets[s + 1];
    const bool ok = lo >= 0 && hi >= lo && hi <= ntok;
    tok = ok ? lo : 0;
    len = ok ? hi - lo : 0;
    return ok;
}
__device__ __forceinline__ int lin_chunks(int len) { return static_cast<int>((static_cast<unsigned>(len) + LIN_C - 1) / LIN_C); }
__device__ __forceinline__ void lin_enter(const LinParams& p, LinIter& it) {
    lin_sequence(p.offsets, p.ntok, it.seq, it.tok, it.len);
    it.chunks = lin_chunks(it.len);
}
// the first sequence with tokens behind `seq` (there is one)
static __device__ __noinline__ int lin_seek(const int32_t* offsets, long long ntok, int seq) {
    int tok, len;
    do lin_sequence(offsets, ntok, ++seq, tok, len);
    while (len == 0);
    return seq;
}
__device__ __forceinline__ void lin_next(const LinParams& p, LinIter& it) {          // (the caller knows that there is a next one)
    if (++it.chunk < it.chunks) return;
    it.chunk = 0;
    if (++it.head < p.heads) return;
    it.head = 0;
    it.seq = lin_seek(p.offsets, p.ntok, it.seq);
    lin_enter(p, it);
}
__device__ __forceinline__ int lin_tokens(const LinIter& it) { return min(LIN_C, it.len - it.chunk * LIN_C); }
__device__ __forceinline__ long long lin_first(long long c, long long units, int ctas) { return c * units / ctas; }
static __device__ __noinline__ float lin_power(float g, int n) { return n == 0 ? 1.f : expf(g * static_cast<float>(n)); }

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

// Two fp32 values in one register pair: one instruction for both.
__device__ __forceinline__ uint64_t lin_pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void lin_unpair(uint64_t r, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r)); }
__device__ __forceinline__ uint64_t lin_mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t lin_fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t lin_add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// Splits two fp32 values: rounded to 8 bits as a pair of bfloat16, and what that leaves of them (exactly), by Veltkamp's method:
// four instructions of the fp32 pipe for two values, where masking takes the integer pipe, which has half its rate and is the
// busiest of this kernel.  Three such parts hold all 24 bits; two, the second rounded (lin_near), 2^-16 of the value.
// Values of 2^111 and more, and infinities, become NaN.
__device__ __forceinline__ uint32_t lin_cut(uint64_t& v) {
    const uint64_t wide = lin_mul2(v, lin_pair(65537.f, 65537.f)), minus = lin_pair(-1.f, -1.f);
    const uint64_t hi = lin_add2(wide, lin_fma2(wide, minus, v));
    v = lin_fma2(hi, minus, v);
    float a, b;
    lin_unpair(hi, a, b);
    return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
}
// The upper halves of two values that are bfloat16 already.
__device__ __forceinline__ uint32_t lin_upper(uint64_t v) {
    float a, b;
    lin_unpair(v, a, b);
    return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
}
__device__ __forceinline__ uint32_t lin_near(uint64_t v) {
    float a, b;
    lin_unpair(v, a, b);
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&x);
}
// Bounded wait that sleeps in the barrier instruction (out of line: there are many, and the roles' loops have to stay short).
static __device__ __noinline__ bool lin_wait_one(uint64_t* bar, uint32_t parity, volatile int* abort_flag, uint64_t budget_ns) {
    if (mbar_try_wait_for(bar, parity, 20000u)) return true;
    const uint64_t t0 = global_timer_ns();
    while (!mbar_try_wait_for(bar, parity, 20000u)) {
        if (*abort_flag) return false;
        if (global_timer_ns() - t0 > budget_ns) return false;
    }
    return true;
}
// sum_j scale exp(g (i - j)) (q_i . k_j) v_j over j <= i for one column of v, from the tiles in shared memory (of = scale exp(g (x + 1))).
static __device__ __noinline__ float lin_repair(const uint8_t* q, const uint8_t* k, const uint8_t* v, int dk, int i, int col, float scale, const float* of) {
    const auto at = [](const uint8_t* tile, int row, int c) {
        const uint16_t x = *reinterpret_cast<const uint16_t*>(tile + (c >> 6) * LIN_BOX + swz_offset<128>(row, (c & 63) * 2));
        return __uint_as_float(static_cast<uint32_t>(x) << 16);
    };
    float y = 0.f;
    for (int j = 0; j <= i; ++j) {
        float s = 0.f;
        for (int d = 0; d < dk; ++d) s = fmaf(at(q, i, d), at(k, j, d), s);
        y = fmaf(s * (i == j ? scale : of[i - j - 1]), at(v, j, col), y);
    }
    return y;
}
// A wait of a whole warp: all of its lanes get the same answer.
__device__ __forceinline__ bool lin_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, uint64_t budget_ns) {
    return __all_sync(0xffffffffu, lin_wait_one(bar, parity, abort_flag, budget_ns));
}
// The four warps that store results: whether all of them say yes (they leave together when a wait has given up).
__device__ __forceinline__ bool lin_out_all(bool ok) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"(static_cast<uint32_t>(ok)) : "memory");
    return r != 0;
}
__device__ __forceinline__ void lin_out_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

template <int DK, bool CARRY>
__global__ void __launch_bounds__(LIN_THREADS, 1)
linear_chunks_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v, const LinParams p) {
    using C = LinCfg<DK, CARRY>;
    constexpr int COLS = DK / (LIN_STATE / 4);              // state columns of a thread
    extern __shared__ __align__(1024) uint8_t lin_smem[];   // (the swizzle goes by the address: tiles start at multiples of 1024)
    uint8_t* smem = lin_smem;
    __shared__ LinBars bars;
    __shared__ long long s_sum[LIN_THREADS / 32];
    __shared__ int s_most;
    __shared__ long long s_skip;
    __shared__ int s_seq;
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    __shared__ __align__(16) float s_pw[2][96], s_of[LIN_C];       // scale exp(g i); scale exp(g (i + 1))
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    volatile int* abort_flag = &s_abort;
    griddep_launch_dependents();
    if (smem_u32(smem) & 1023u) {                           // (never: the declaration asks for it)
        if (tid == 0) report_error(p.hdr, 6u);              // MMV_ERR_CUDA
        return;
    }

    // ---- the list, this CTA's range of it ---------------------------------------------------------------------------------
    const int nseq = static_cast<int>(p.nseq);
    const int per = (nseq + LIN_THREADS - 1) / LIN_THREADS, q_lo = min(nseq, tid * per), q_hi = min(nseq, q_lo + per);
    long long mine = 0;
    int most = 0;
    bool bad = false;
    for (int s = q_lo; s < q_hi; ++s) {
        int tok, len;
        bad |= !lin_sequence(p.offsets, p.ntok, s, tok, len);
        mine += lin_chunks(len);
        most = max(most, lin_chunks(len));
    }
    if (tid == 0) s_most = 0;
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
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(&bars.full[i], 1);
            mbar_init(&bars.empty[i], CARRY ? 1 : 7);       // the products that read the tile last, and the results' warps
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars.at_full[i], 1);
            mbar_init(&bars.at_empty[i], 2);
            mbar_init(&bars.kp_full[i], C::kKeyWarps);
            mbar_init(&bars.kv_done[i], 1);
        }
        for (int i = 0; i < C::kUpdates; ++i) {
            mbar_init(&bars.kv_full[i], 1);
            mbar_init(&bars.kv_empty[i], LIN_STATE);
        }
        mbar_init(&bars.s_full, LIN_STATE);
        mbar_init(&bars.s_free, 1);
        mbar_init(&bars.a_full, 2);
        mbar_init(&bars.a_free, 1);
        mbar_init(&bars.o_full, 2);
        mbar_init(&bars.o_empty, 4);
        mbar_init(&bars.drain, 1);
        mbar_fence_init();
    }
    const bool any_bad = __syncthreads_or(bad);
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0 && most > 0) atomicMax(&s_most, most);
    __syncthreads();
    const int least = max(1, static_cast<int>(0.5f * sqrtf(static_cast<float>(s_most))));       // chunks of a range
    long long before = inc - mine, total = 0;
    for (int w = 0; w < LIN_THREADS / 32; ++w) {
        if (w < warp) before += s_sum[w];
        total += s_sum[w];
    }
    const long long units = total * p.heads;
    const int ctas = static_cast<int>(min(static_cast<long long>(gridDim.x), max(1ll, units / least)));
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
                lin_sequence(p.offsets, p.ntok, s, tok, len);
                if (len) continue;
                const long long n = static_cast<long long>(p.heads) * p.dk * p.dv;
                for (long long i = tid; i < n; i += LIN_THREADS) p.state_out[s * n + i] = p.state ? p.state[s * n + i] : 0.f;
            }
    }
    if (cta >= ctas || units == 0) {
        if constexpr (!CARRY) griddep_wait();               // (what follows in the stream waits for this kernel, and for the first one through it)
        return;
    }
    long long u0 = lin_first(cta, units, ctas);
    const long long u1 = lin_first(cta + 1ll, units, ctas);
    {
        const long long u = CARRY ? u1 - 1 : u0;            // find its (sequence, head, chunk)
        if (u >= before * p.heads && u < (before + mine) * p.heads) {
            long long at = before * p.heads;
            int s = q_lo, tok, len;
            lin_sequence(p.offsets, p.ntok, s, tok, len);
            while (u >= at + static_cast<long long>(lin_chunks(len)) * p.heads) {
                at += static_cast<long long>(lin_chunks(len)) * p.heads;
                lin_sequence(p.offsets, p.ntok, ++s, tok, len);
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

    if (warp < LIN_STATE) {
        // ---- the state: rows = columns of v (lanes of tensor memory), COLS columns (of k) per thread ------------------------
        const int part = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        const bool stored = row < p.dv;                     // (rows past dv: whatever the tiles hold there, kept nowhere)
        uint64_t s[COLS / 2];                               // pairs of columns
        LinDecay whole{};
        float g = 0.f;
        const uint32_t cols = lanes + C::kColKV + part * COLS;
        const int held = stored ? min(COLS, p.dk - part * COLS) : 0;
        for (int c = 0; c < count; ++c) {
            const int n = lin_tokens(it);
            if (c == 0 || it.chunk == 0) {
                g = p.log_decay[it.head];
                whole = lin_decay(g, LIN_C);
                const float f = it.chunk == 0 ? 1.f : lin_decay(g, it.chunk * static_cast<double>(LIN_C)).hi;
                if (!CARRY && p.state && f != 0.f) {
                    const float* src = p.state + ((static_cast<long long>(it.seq) * p.heads + it.head) * p.dk + part * COLS) * p.dv + row;
#pragma unroll
                    for (int i = 0; i < COLS / 2; ++i) {
                        const float x = 2 * i < held ? *src : 0.f, y = 2 * i + 1 < held ? src[p.dv] : 0.f;
                        s[i] = lin_pair(f * x, f * y);
                        src += 2 * p.dv;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < COLS / 2; ++i) s[i] = 0ull;
                }
                if (!CARRY && it.chunk > 0) {
                    const long long seg = u0 - it.chunk;    // first unit of this (sequence, head)
                    for (int j = cta - 1; j >= 0; --j) {
                        const long long end = lin_first(j + 1ll, units, ctas);
                        if (end <= seg) break;
                        const float w = u0 == end ? 1.f : lin_decay(g, static_cast<double>(u0 - end) * LIN_C).hi;
                        if (w == 0.f) break;                // (and those in front of it weigh less)
                        const float* src = p.carry + (static_cast<long long>(j) * DK + part * COLS) * 128 + row;
#pragma unroll
                        for (int i = 0; i < COLS / 2; ++i) {
                            s[i] = lin_fma2(lin_pair(w, w), lin_pair(src[2 * i * 128], src[(2 * i + 1) * 128]), s[i]);
                            if (i % 8 == 7) asm volatile("" ::: "memory");          // (16 loads in flight: registers)
                        }
                    }
                }
            }
            if constexpr (!CARRY) {
                if (c > 0) ok = lin_wait(&bars.s_free, (c - 1) & 1, abort_flag, budget);
                if (!ok) break;
                tc_fence_after_sync();
#pragma unroll
                for (int b = 0; b < COLS / 8; ++b) {
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint64_t x = s[b * 4 + i];
                        hi[i] = lin_cut(x);
                        lo[i] = lin_near(x);
                    }
                    const uint32_t at = lanes + C::kColS + part * (COLS / 2) + b * 4;
                    tmem_st_32x4(at, hi);
                    tmem_st_32x4(at + DK / 2, lo);
                }
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.s_full);
            }
            const LinDecay d = n == LIN_C ? whole : lin_decay(g, n);
            const uint64_t dhi = lin_pair(d.hi, d.hi), dlo = lin_pair(d.lo, d.lo);
            ok = lin_wait(&bars.kv_full[c % C::kUpdates], (c / C::kUpdates) & 1, abort_flag, budget);
            if (!ok) break;
            tc_fence_after_sync();
#pragma unroll
            for (int b = 0; b < COLS / 8; ++b) {
                uint32_t r[8];
                tmem_ld_32x8(cols + (c % C::kUpdates) * DK + b * 8, r);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint64_t x = lin_pair(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]));
                    s[b * 4 + i] = lin_fma2(s[b * 4 + i], dhi, lin_fma2(s[b * 4 + i], dlo, x));
                }
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.kv_empty[c % C::kUpdates]);
            if (!CARRY && it.chunk + 1 == it.chunks && p.state_out) {
                float* dst = p.state_out + ((static_cast<long long>(it.seq) * p.heads + it.head) * p.dk + part * COLS) * p.dv + row;
#pragma unroll
                for (int i = 0; i < COLS / 2; ++i) {
                    float x, y;
                    lin_unpair(s[i], x, y);
                    if (2 * i < held) *dst = x;
                    if (2 * i + 1 < held) dst[p.dv] = y;
                    dst += 2 * p.dv;
                }
            }
            if (c + 1 < count) lin_next(p, it);
        }
        if (CARRY && ok) {
            float* dst = p.carry + (static_cast<long long>(cta) * DK + part * COLS) * 128 + row;
#pragma unroll
            for (int i = 0; i < COLS / 2; ++i) {
                float x, y;
                lin_unpair(s[i], x, y);
                dst[2 * i * 128] = x;
                dst[(2 * i + 1) * 128] = y;
            }
        }
    } else if (warp < LIN_WARP_KEYS + C::kKeyWarps) {
        // ---- K', 32 tokens at a time: a thread scales a quarter (CARRY: an eighth) of a token's key ---------------------------------
        constexpr int TPT = C::kKeyWarps, WORDS = DK / 8 / TPT;                    // threads of a token, 16-byte words of each
        const int t = tid - LIN_WARP_KEYS * 32, row = t / TPT, part = t % TPT;
        // Word i of this thread: in an order in which eight neighbouring threads (of 2 tokens or 1) meet eight different
        // 16-byte columns of the swizzled rows.
        const int box = part * WORDS >> 3, word0 = part * WORDS & 7;
        const auto place = [&](int i) {
            const int word = word0 + (DK == 128 ? i ^ (box << (TPT == 4 ? 1 : 0)) : i);
            return swz_offset<128>(row, word * 16);
        };
        float whole[2] = {0.f, 0.f};                        // exp(g (63 - j)), this head's, of this thread's tokens j
        for (int c = 0; c < count; ++c) {
            const int n = lin_tokens(it), stage = c % C::kStages;
            if (c == 0 || it.chunk == 0) {
                const float g = p.log_decay[it.head];
                whole[0] = lin_power(g, LIN_C - 1 - row);
                whole[1] = lin_power(g, LIN_C / 2 - 1 - row);
            }
            ok = lin_wait(&bars.full[stage], (c / C::kStages) & 1, abort_flag, budget);
            if (!ok) break;
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const int j = h * 32 + row;
                float f = h ? whole[1] : whole[0];
                if (n < LIN_C) f = j < n ? lin_power(p.log_decay[it.head], n - 1 - j) : 0.f;
                if (c > 0) ok = lin_wait(&bars.kv_done[h], (c - 1) & 1, abort_flag, budget);      // the product has read this K'
                if (!ok) break;
                const uint64_t ff = lin_pair(f, f);
                const uint8_t* src = smem + stage * C::kStage + C::kK + box * LIN_BOX + h * (LIN_BOX / 2);
                uint8_t* dst = smem + C::kKp + h * C::kKpBytes + box * (LIN_BOX / 2);
                uint4 key[WORDS];
#pragma unroll
                for (int i = 0; i < WORDS; ++i) key[i] = *reinterpret_cast<const uint4*>(src + place(i));
#pragma unroll
                for (int i = 0; i < WORDS; ++i) {
                    const uint32_t at = place(i);
                    const uint32_t in[4] = {key[i].x, key[i].y, key[i].z, key[i].w};
                    uint32_t a[4], b[4], d[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint64_t x = lin_mul2(lin_pair(__uint_as_float(in[e] << 16), __uint_as_float(in[e] & 0xffff0000u)), ff);
                        a[e] = lin_cut(x);
                        b[e] = lin_cut(x);
                        d[e] = lin_upper(x);
                    }
                    if (j >= n)                             // another sequence's token counts as zero whatever it holds
#pragma unroll
                        for (int e = 0; e < 4; ++e) a[e] = b[e] = d[e] = 0u;
                    *reinterpret_cast<uint4*>(dst + at) = make_uint4(a[0], a[1], a[2], a[3]);
                    *reinterpret_cast<uint4*>(dst + C::kKpPart + at) = make_uint4(b[0], b[1], b[2], b[3]);
                    *reinterpret_cast<uint4*>(dst + 2 * C::kKpPart + at) = make_uint4(d[0], d[1], d[2], d[3]);
                }
                if (j >= n) {                               // (and a zero weight does not hide a value that is not finite)
                    uint8_t* v = smem + stage * C::kStage + C::kV + j * 128;
#pragma unroll 1
                    for (int i = part; i < 16; i += TPT) *reinterpret_cast<uint4*>(v + (i >> 3) * LIN_BOX + (i & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.kp_full[h]);
            }
            if (!ok) break;
            if (c + 1 < count) lin_next(p, it);
        }
    } else if (warp < LIN_WARP_SCORES) {
        if constexpr (!CARRY) {
            // ---- the chunk's results: from tensor memory (a column of v per thread) by way of shared memory into rows -------------
            const int t = tid - LIN_WARP_OUT * 32, words = p.dv / 8, q = t & 15, r0 = t >> 4;
            const uint32_t lanes = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
            uint8_t* stage = smem + C::kO;
            for (int c = 0; c < count; ++c) {
                const int n = lin_tokens(it);
                if ((c == 0 || it.chunk == 0) && t < LIN_C) s_of[t] = p.scale * lin_power(p.log_decay[it.head], t + 1);
                ok = lin_wait(&bars.o_full, c & 1, abort_flag, budget);
                ok = lin_out_all(ok);                       // (s_of is there, and the last chunk's results have left the staging rows)
                if (!ok) break;
                tc_fence_after_sync();
                bool wild = false;
#pragma unroll 1
                for (int i0 = 0; i0 < LIN_C; i0 += 8) {
                    uint32_t x[8], y[8];
                    tmem_ld_32x8(lanes + C::kColO1 + i0, x);
                    tmem_ld_32x8(lanes + C::kColO2 + i0, y);
                    float f[8];
#pragma unroll
                    for (int i = 0; i < 8; i += 4) *reinterpret_cast<float4*>(f + i) = *reinterpret_cast<const float4*>(s_of + i0 + i);
                    tmem_ld_wait();
                    if (i0 == 0) wild = t < p.dv && (y[0] & 0x7f800000u) == 0x7f800000u;
                    uint8_t* dst = stage + i0 * C::kOPitch + t * 2;
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const uint32_t o = lin_near(lin_fma2(lin_pair(f[i], f[i + 1]), lin_pair(__uint_as_float(x[i]), __uint_as_float(x[i + 1])),
                                                             lin_pair(__uint_as_float(y[i]), __uint_as_float(y[i + 1]))));
                        *reinterpret_cast<uint16_t*>(dst + i * C::kOPitch) = static_cast<uint16_t>(o);
                        *reinterpret_cast<uint16_t*>(dst + (i + 1) * C::kOPitch) = static_cast<uint16_t>(o >> 16);
                    }
                }
                // The first token's sum has a weight of 0 for every later one.  Where it is not finite, a value of v may be to blame (0 times
                // an infinity): the tokens in front of this column's first such value are summed up again, one by one.
                if (__any_sync(0xffffffffu, wild)) {
                    const uint8_t* tile = smem + (c % C::kStages) * C::kStage;
                    int stop = 0;                           // first token whose value in this column is not finite
                    if (wild) {
                        const uint8_t* v = tile + C::kV + (t >> 6) * LIN_BOX;
                        while (stop < n && (*reinterpret_cast<const uint16_t*>(v + swz_offset<128>(stop, (t & 63) * 2)) & 0x7f80u) != 0x7f80u) ++stop;
                        if (stop == n) stop = 0;            // (none: the sum's own scores are not finite)
                    }
#pragma unroll 1
                    for (int i0 = 0; i0 < LIN_C; i0 += 8) {
                        uint32_t x[8];
                        tmem_ld_32x8(lanes + C::kColO1 + i0, x);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (i0 + i < stop) {
                                const float y = lin_repair(tile + C::kQ, tile + C::kK, tile + C::kV, p.dk, i0 + i, t, p.scale, s_of);
                                *reinterpret_cast<uint16_t*>(stage + (i0 + i) * C::kOPitch + t * 2) =
                                    lin_store<true>(fmaf(s_of[i0 + i], __uint_as_float(x[i]), y));
                            }
                    }
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&bars.o_empty);
                    mbar_arrive(&bars.empty[c % C::kStages]);
                }
                lin_out_sync();
                if (q < words) {                            // 16 threads to a row, rows r0, r0 + 8, ...
                    uint16_t* out = p.out + ((static_cast<long long>(it.tok) + it.chunk * LIN_C + r0) * p.heads + it.head) * p.dv + q * 8;
                    const long long step = 8ll * p.heads * p.dv;
                    uint4 w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const uint4*>(stage + (r0 + i * 8) * C::kOPitch + q * 16);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (r0 + i * 8 < n) *reinterpret_cast<uint4*>(out + i * step) = w[i];
                }
                if (c + 1 < count) lin_next(p, it);
            }
        }
    } else if (warp < LIN_WARP_LOAD) {
        if constexpr (!CARRY) {
            // ---- A: the scores of key j = lane, queries i = 0..63 -----------------------------------------------------------------
            const int j = tid - LIN_WARP_SCORES * 32;
            const uint32_t lanes = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
            uint8_t* dst = smem + C::kA;
            // Keys 32 to 63 (the second warp) meet queries 32 to 63 only; the zeros in front of them are written once.
            const int first = (warp & 1) * 4;               // in blocks of 8 queries
            for (int q = 0; q < first; ++q) {
                const uint32_t at = swz_offset<128>(j, q * 16);
                *reinterpret_cast<uint4*>(dst + at) = make_uint4(0u, 0u, 0u, 0u);
                *reinterpret_cast<uint4*>(dst + LIN_BOX + at) = make_uint4(0u, 0u, 0u, 0u);
            }
            float* pw = s_pw[warp & 1];                     // scale exp(g (x - 32)) from x = 32 on
            const float* mine = pw + 32 - lane;             // of query i: mine[i - 8 first]
            for (int c = 0; c < count; ++c) {
                const int n = lin_tokens(it);
                const bool enter = c == 0 || it.chunk == 0;
                ok = lin_wait(&bars.at_full[c & 1], (c >> 1) & 1, abort_flag, budget);
                if (ok && c > 0) ok = lin_wait(&bars.a_free, (c - 1) & 1, abort_flag, budget);       // the product has read the last A
                if (!ok) break;
                if (enter) {
                    __syncwarp();
                    const float g = p.log_decay[it.head];
                    pw[lane] = 0.f;
                    pw[lane + 32] = p.scale * lin_power(g, lane);
                    pw[lane + 64] = p.scale * lin_power(g, lane + 32);
                    __syncwarp();
                }
                tc_fence_after_sync();
                const int from = j < n ? j : LIN_C;         // first query that this key has a score with
#pragma unroll 1
                for (int i0 = first * 8; i0 < LIN_C; i0 += 8) {
                    uint32_t r[8];
                    tmem_ld_32x8(lanes + C::kColAT + (c & 1) * 64 + i0, r);
                    float f[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] = mine[i0 - first * 8 + i];
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 8; ++i) r[i] = i0 + i >= from ? r[i] : 0u;       // (not a product with 0: a later token may hold a NaN)
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint64_t x = lin_mul2(lin_pair(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1])), lin_pair(f[2 * e], f[2 * e + 1]));
                        hi[e] = lin_cut(x);
                        lo[e] = lin_near(x);
                    }
                    const uint32_t at = swz_offset<128>(j, i0 * 2);
                    *reinterpret_cast<uint4*>(dst + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    *reinterpret_cast<uint4*>(dst + LIN_BOX + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
                tc_fence_before_sync();
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&bars.at_empty[c & 1]);
                    mbar_arrive(&bars.a_full);
                }
                if (c + 1 < count) lin_next(p, it);
            }
        }
    } else if (warp == LIN_WARP_LOAD) {
        if (elect_one()) {
            const int vboxes = p.dv > 64 ? 2 : 1;
            const uint32_t bytes = ((CARRY ? 1 : 2) * C::kBoxes + vboxes) * LIN_BOX;
            for (int c = 0; c < count; ++c) {
                const int stage = c % C::kStages;
                if (c >= C::kStages) ok = lin_wait_one(&bars.empty[stage], (c / C::kStages - 1) & 1, abort_flag, budget);
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
        if (elect_one()) {
            [[maybe_unused]] constexpr uint32_t kIdescAT = lin_idesc(LIN_C, false, false), kIdescKV = lin_idesc(DK, true, true);
            [[maybe_unused]] constexpr uint32_t kIdescO1 = lin_idesc(LIN_C, false, false), kIdescO2 = lin_idesc(LIN_C, true, true);
            const uint32_t sm = smem_u32(smem);
            // (a descriptor's low word is an address in units of 16 bytes: 2 per step of 16 values along a row, 128 per 16 rows)
            constexpr uint32_t kBox = LIN_BOX >> 4;
            const auto update = [&](int kv) {                // KV = V^T K', half a chunk
                tc_fence_after_sync();
                const int stage = (kv >> 1) % C::kStages, h = kv & 1;
                const uint64_t dv = lin_desc_mn(sm + stage * C::kStage + C::kV + h * (LIN_BOX / 2), LIN_BOX);
                uint64_t dk = lin_desc_mn(sm + C::kKp + h * C::kKpBytes, LIN_BOX / 2);
#pragma unroll 1
                for (int x = 0; x < 3; ++x, dk += C::kKpPart >> 4)
#pragma unroll
                    for (int k = 0; k < 2; ++k) mma_f16_ss(tmem + C::kColKV + ((kv >> 1) % C::kUpdates) * DK, dv + 128 * k, dk + 128 * k, kIdescKV, h > 0 || x > 0 || k > 0);
                tc_commit(&bars.kv_done[h]);
                if (h) {
                    tc_commit(&bars.kv_full[(kv >> 1) % C::kUpdates]);
                    tc_commit(&bars.empty[stage]);
                }
            };
            if constexpr (CARRY) {
                for (int kv = 0; ok && kv < 2 * count; ++kv) {
                    ok = lin_wait_one(&bars.kp_full[kv & 1], (kv >> 1) & 1, abort_flag, budget);
                    if (ok && kv >= 4 && !(kv & 1)) ok = lin_wait_one(&bars.kv_empty[(kv >> 1) & 1], ((kv >> 2) - 1) & 1, abort_flag, budget);
                    if (ok) update(kv);
                }
            }
            // Each of the four products goes out when its operands are there, whichever chunk it belongs to: the numbers of the next ones.
            int at = CARRY ? count : 0, kv = CARRY ? 2 * count : 0, o1 = CARRY ? count : 0, o2 = CARRY ? count : 0;
            uint64_t since = global_timer_ns();
            uint32_t polls = 0;
            while (at < count || kv < 2 * count || o1 < count || o2 < count) {
                const int before = at + kv + o1 + o2;
                if (at < count && mbar_try_wait(&bars.full[at % C::kStages], (at / C::kStages) & 1) &&
                    (at < 2 || mbar_try_wait(&bars.at_empty[at & 1], ((at >> 1) - 1) & 1))) {
                    tc_fence_after_sync();
                    const uint32_t st = sm + (at % C::kStages) * C::kStage;
                    uint64_t dk = make_desc(st + C::kK, 1024, 2), dq = make_desc(st + C::kQ, 1024, 2);
#pragma unroll 1
                    for (int b = 0; b < C::kBoxes; ++b, dk += kBox, dq += kBox)            // AT = K Q^T
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            mma_f16_ss(tmem + C::kColAT + (at & 1) * 64, dk + 2 * k, dq + 2 * k, kIdescAT, b > 0 || k > 0);
                    tc_commit(&bars.at_full[at & 1]);
                    ++at;
                }
                if (kv < 2 * count && mbar_try_wait(&bars.kp_full[kv & 1], (kv >> 1) & 1) && (kv == 0 || (kv & 1) || mbar_try_wait(&bars.kv_empty[0], ((kv >> 1) - 1) & 1)))
                    update(kv++);
                if (o1 < at && o1 < count && mbar_try_wait(&bars.s_full, o1 & 1) && (o1 == 0 || mbar_try_wait(&bars.o_empty, (o1 - 1) & 1))) {
                    tc_fence_after_sync();
                    const uint32_t st = sm + (o1 % C::kStages) * C::kStage;
#pragma unroll 1
                    for (int x = 0; x < 2 * C::kBoxes; ++x) {                              // O1 = S^T Q^T
                        const uint64_t dq = make_desc(st + C::kQ + (x & (C::kBoxes - 1)) * LIN_BOX, 1024, 2);
#pragma unroll
                        for (int k = 0; k < 4; ++k) mma_f16_ts(tmem + C::kColO1, tmem + C::kColS + x * 32 + k * 8, dq + 2 * k, kIdescO1, x > 0 || k > 0);
                    }
                    tc_commit(&bars.s_free);
                    tc_commit(&bars.o_full);
                    tc_commit(&bars.empty[o1 % C::kStages]);
                    ++o1;
                }
                // (behind the chunk's update: its keys' warps have zeroed the rows of V that are another sequence's, which A's zeros meet here too)
                if (2 * o2 + 1 < kv && mbar_try_wait(&bars.a_full, o2 & 1) && (o2 == 0 || mbar_try_wait(&bars.o_empty, (o2 - 1) & 1))) {
                    tc_fence_after_sync();
                    const uint64_t dv = lin_desc_mn(sm + (o2 % C::kStages) * C::kStage + C::kV, LIN_BOX);
                    uint64_t da = lin_desc_mn(sm + C::kA, LIN_BOX);
#pragma unroll 1
                    for (int x = 0; x < 2; ++x, da += kBox)                                // O2 = V^T A^T
#pragma unroll
                        for (int k = 0; k < LIN_C / 16; ++k) mma_f16_ss(tmem + C::kColO2, dv + 128 * k, da + 128 * k, kIdescO2, x > 0 || k > 0);
                    tc_commit(&bars.a_free);
                    tc_commit(&bars.o_full);
                    tc_commit(&bars.empty[o2 % C::kStages]);
                    ++o2;
                }
                if (at + kv + o1 + o2 != before) {
                    polls = 0;
                } else {
                    __nanosleep(20);                        // (a turn of this loop is some 40 instructions that others could issue)
                    if ((++polls & 63u) == 0u) {
                        if (polls == 64u) since = global_timer_ns();
                        if (*abort_flag || global_timer_ns() - since > budget) {
                            ok = false;
                            break;
                        }
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

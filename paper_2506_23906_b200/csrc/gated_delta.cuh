// Layers that keep a state under the gated delta rule:
//     S_t = a_t S_{t-1} + k_t u_t^T,   u_t = b_t (v_t - a_t S_{t-1}^T k_t),   o_t = scale S_t^T q_t,   a_t = exp(g_t)
// i.e. what the decayed state answers for the key k_t is moved towards v_t by the share b_t.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "common.cuh"
#include "linear_attn.cuh"
#include "paged_attn_q8.cuh"

namespace mmv {

struct DeltaParams {
    const uint16_t *q, *k, *v;
    long long q_tok, q_head, k_tok, k_head, v_tok, v_head;   // element strides
    const float *decay, *beta;                               // [token][heads]
    long long decay_tok, beta_tok;
    int heads, group;                                        // value heads; value heads per query / key head
    int dk, dv;
    float scale;
    uint16_t* out;                                           // [token, heads, dv]
    const float* state;                                      // [.., heads, dk, dv]
    float* state_out;
    // single tokens
    const int32_t* slots;                                    // request -> state; null: its own index
    long long num_slots;
    int parts;                                               // column parts of a state
    // packed prompts
    const int32_t* offsets;
    int nseq, ntok;
    long long first_slot, last_slot;                         // chunks that this launch takes, by their place in the workspace
    int slices;                                              // column parts of a (sequence, head)
    int present;                                             // sequences that a launch of the second kernel has CTAs for
    WorkspaceHeader* hdr;
    uint8_t* chunks;                                         // [last_slot - first_slot][heads] DeltaChunk
    uint64_t budget_ns;                                      // bound of every wait
    long long debug_skip;                                    // test hook: the first kernel's CTA that leaves its loads out, from 2^32 on the second one's (-1: none)
};

// ---------------------------------------------------------------------------------------------------------------------
// One token per request.  The state is the traffic (8 bytes per element against 7 flops).  A CTA owns COLS columns of one (request, head): all
// of its rows' loads are in flight before anything else, one sweep over them in registers gives k S and q S, which meet in shared
// memory, and a second one the new state; the result needs none of it: q S' = a q S + (q k) u.  HBM: 256 requests of 16 states of 128 x 128 98 us,
// 5.5 of the 6.5 TB/s of a copy; one request 5 us, the launch.
// ---------------------------------------------------------------------------------------------------------------------
template <bool BF16, int COLS>
__global__ void __launch_bounds__(LIN_STEP_THREADS) delta_step_kernel(const DeltaParams p) {
    constexpr int LANES = COLS / 4;                              // threads per row
    constexpr int ROWS = LIN_STEP_THREADS / LANES;               // rows side by side
    constexpr int MINE = 128 / ROWS;                             // rows of a thread
    __shared__ float s_q[128], s_k[128];
    __shared__ __align__(16) float4 s_ks[ROWS][LANES], s_qs[ROWS][LANES];
    __shared__ float4 s_u[LANES];
    __shared__ float s_qk[4];
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
    if (tid < 128) {
        float q = 0.f, k = 0.f;
        if (tid < p.dk) {
            q = lin_load<BF16>(p.q + r * p.q_tok + hk * p.q_head + tid);
            k = lin_load<BF16>(p.k + r * p.k_tok + hk * p.k_head + tid);
        }
        s_q[tid] = q;
        s_k[tid] = k;
        float qk = q * k;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) qk += __shfl_xor_sync(0xffffffffu, qk, o);
        if ((tid & 31) == 0) s_qk[tid >> 5] = qk;
    }
    if (tid == LIN_STEP_THREADS - 1) s_decay = lin_decay(p.decay[r * p.decay_tok + h], 1);
    const float beta = p.beta[r * p.beta_tok + h];
    __syncthreads();
    float4 ks = make_float4(0.f, 0.f, 0.f, 0.f), qs = ks;
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        const int d = row + i * ROWS;
        if (mine && d < p.dk) {
            const float kd = s_k[d], qd = s_q[d];
            ks.x = fmaf(kd, s[i].x, ks.x);
            ks.y = fmaf(kd, s[i].y, ks.y);
            ks.z = fmaf(kd, s[i].z, ks.z);
            ks.w = fmaf(kd, s[i].w, ks.w);
            qs.x = fmaf(qd, s[i].x, qs.x);
            qs.y = fmaf(qd, s[i].y, qs.y);
            qs.z = fmaf(qd, s[i].z, qs.z);
            qs.w = fmaf(qd, s[i].w, qs.w);
        }
    }
    s_ks[row][lane] = ks;
    s_qs[row][lane] = qs;
    __syncthreads();
    const LinDecay decay = s_decay;
    for (int c = tid; c < COLS; c += LIN_STEP_THREADS) {
        if (part * COLS + c < p.dv) {
            float x = 0.f, y = 0.f;
#pragma unroll 4
            for (int i = 0; i < ROWS; ++i) {
                x += reinterpret_cast<const float*>(s_ks[i])[c];
                y += reinterpret_cast<const float*>(s_qs[i])[c];
            }
            const float v = lin_load<BF16>(p.v + r * p.v_tok + h * p.v_head + part * COLS + c);
            const float u = beta * (v - fmaf(x, decay.hi, x * decay.lo));
            reinterpret_cast<float*>(s_u)[c] = u;
            const float qk = s_qk[0] + s_qk[1] + s_qk[2] + s_qk[3];
            out[part * COLS + c] = lin_store<BF16>(p.scale * fmaf(qk, u, fmaf(y, decay.hi, y * decay.lo)));
        }
    }
    __syncthreads();
    if (!mine) return;
    const float4 u = s_u[lane];
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        const int d = row + i * ROWS;
        if (d < p.dk) {
            const float kd = s_k[d];
            float4 x = s[i];
            x.x = fmaf(x.x, decay.hi, fmaf(x.x, decay.lo, kd * u.x));
            x.y = fmaf(x.y, decay.hi, fmaf(x.y, decay.lo, kd * u.y));
            x.z = fmaf(x.z, decay.hi, fmaf(x.z, decay.lo, kd * u.z));
            x.w = fmaf(x.w, decay.hi, fmaf(x.w, decay.lo, kd * u.w));
            *reinterpret_cast<float4*>(dst + static_cast<long long>(d) * p.dv + col) = x;
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// Packed prompts, chunks of 64 tokens on the tensor cores.  With G the running sum of g in a chunk of n tokens, S the state in front of it and
// D_ij = exp(G_i - G_j):
//     L_ij = b_i D_ij k_i . k_j  (j < i),  T = (1 + L)^-1,  A_ij = D_ij q_i . k_j  (j <= i)
//     R  = diag(b) (V - exp(G) K S),  U = T R            (row i is u_i)
//     O  = scale (exp(G) Q S + A U)
//     S' = exp(G_n) S + K^T diag(exp(G_n - G)) U
// T and A do not depend on the state: a first kernel forms them for all chunks side by side; the second one walks along a sequence's chunks, one
// CTA per (sequence, head, slice of columns), whose columns never meet others'.
//
// Operands that are formed here enter their products as sums of bfloat16 values, of two (2^-17 of the value) or, where the fp32 state would lose by
// it, of three: its own copy in K S, R and the update's exp(G_n - G) U.  U is R + (T - 1) R, the first term in fp32; what is added to a
// state or to R is summed up by itself, since the tensor core cuts a sum's last digits.  With two parts everywhere, T R as one product and the sums
// begun at S and R the state was off by 4.0e-6 of itself; it is by 0.9e-6 (fp32 throughout: 0.16e-6).
//
// What bounds it: latencies inside a chunk.  Its three products follow one another through shared memory, eight warps wait for one another three times, and an SM has
// room for nothing else meanwhile (166 KB of shared memory): 2.2 us with slices of 16 columns, 3.1 us with 32.
//   One prompt of 65536 tokens and 16 heads is a chain: 1024 chunks on 128 CTAs of 16 columns, 2.33 ms (the first kernels of later parts run beside it).
//   16 prompts of 32768 tokens in all and 16 heads are a queue: 1024 CTAs of 32 columns, about 228 chunks per SM one after the other, 0.70 ms (tensor pipe 46 %
//     busy) behind 0.14 ms of the first kernel, which ends before the second begins: 0.84 ms.
// tcgen05.mma takes about 44 clocks and half a clock per column of a slice for 16 rows of a product, as many as the warps' own instructions take for it, and its
// results come back through tensor memory: at these widths nothing is gained.  Whole states per CTA, whose products have its 64 and 128 rows, would fill the SMs
// from 148 (sequence, head) pairs on, and composing chunks (S -> M S + N) would shorten the chain of a few long prompts; neither has been built.
//
// A chunk that holds a value that is not finite (or whose products are not) is taken token by token: zeros of the triangles would carry it to
// tokens in front of it.
// ---------------------------------------------------------------------------------------------------------------------
constexpr int DELTA_C = 64;
constexpr int DELTA_TILES = 10;                              // 16 x 16 blocks on and under the diagonal, by rows
__host__ __device__ constexpr int delta_tile(int i, int j) { return i * (i + 1) / 2 + j; }

// What the first kernel leaves of a chunk and head.  A block's 32 x 16 bytes are the lanes' registers of a product's first operand.
struct DeltaScalars {
    float beta[DELTA_C], past[DELTA_C], left[DELTA_C];       // b, exp(G), exp(G_n - G)
    float whole_hi, whole_lo;                                // exp(G_n)
    int wild;                                                // to be taken token by token
    int pad;
};
struct DeltaChunk {
    uint4 t[2][DELTA_TILES][32];                             // T - 1: high parts, low parts
    uint4 a[2][DELTA_TILES][32];                             // A
    DeltaScalars x;
};
static_assert(sizeof(DeltaScalars) % 16 == 0 && sizeof(DeltaChunk) % 16 == 0, "copied in 16-byte words");

// Sequence s: its first token and length; its chunk c lies at place tok / 64 + s + c (no two at the same, in any offsets that grow).
__device__ __forceinline__ long long delta_slot(int tok, int seq) { return static_cast<long long>(tok / DELTA_C) + seq; }
// x -> the sequence whose chunks' places hold x: the last one that begins at or in front of it
__device__ __forceinline__ int delta_sequence_of(const int32_t* offsets, int n, long long x) {
    const int lane = threadIdx.x & 31;
    int lo = 0, len = n;                                     // how many of the sequences 1 .. n begin at or in front of x
    while (len > 0) {
        const int step = (len + 31) >> 5, i = (lane + 1) * step - 1;
        const int c = __popc(__ballot_sync(0xffffffffu, i < len && delta_slot(offsets[lo + i + 1], lo + i + 1) <= x));
        lo += c * step;
        len = min(step - 1, len - c * step);
    }
    return lo;
}

__device__ __forceinline__ void delta_split(float a, float b, uint32_t& hi, uint32_t& lo) {
    hi = pack_pair<true>(a, b);
    const float2 x = unpack_pair<true>(hi);
    lo = pack_pair<true>(a - x.x, b - x.y);
}
__device__ __forceinline__ void delta_split3(float a, float b, uint32_t (&r)[3]) {
    r[0] = pack_pair<true>(a, b);
    const float2 x = unpack_pair<true>(r[0]);
    delta_split(a - x.x, b - x.y, r[1], r[2]);
}
// d += (ahi + alo)(bhi + blo) less alo blo
__device__ __forceinline__ void delta_mma3(float (&d)[4], const uint32_t (&ahi)[4], const uint32_t (&alo)[4], uint32_t bh0, uint32_t bh1, uint32_t bl0, uint32_t bl1) {
    mma_16816<true>(d, ahi, bh0, bh1);
    mma_16816<true>(d, alo, bh0, bh1);
    mma_16816<true>(d, ahi, bl0, bl1);
}
__device__ __forceinline__ bool delta_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }
__device__ __forceinline__ bool delta_finite2(uint32_t pair) { return (pair & 0x7f80u) != 0x7f80u && (pair & 0x7f800000u) != 0x7f800000u; }
__device__ __forceinline__ void ldsm_x2_t(uint32_t& a, uint32_t& b, uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0, %1}, [%2];" : "=r"(a), "=r"(b) : "r"(addr) : "memory");
}
// 2^(a - b) for sums of two values each (2^-22 of it; small results are kept down to the smallest fp32)
__device__ __forceinline__ float delta_decay(float2 a, float2 b) {
    float r;
    asm("ex2.approx.f32 %0, %1;" : "=f"(r) : "f"((a.x - b.x) + (a.y - b.y)));
    return r;
}
constexpr int DELTA_BOX = DELTA_C * 128;                     // bytes of 64 tokens x 64 columns, as the loads leave them
// Word c of a token's row in a tile of 64 tokens x DK columns: boxes of 64 columns, 128-byte swizzle.
__device__ __forceinline__ uint32_t delta_word(int row, int c) { return (c >> 3) * DELTA_BOX + row * 128 + (((c & 7) ^ (row & 7)) << 4); }

// ---------------------------------------------------------------------------------------------------------------------
// T and A of one chunk, for the value heads of one key head, 16 x 16 blocks at a time.  Warps 0 to 3 form K K^T on the diagonal and from it T's
// diagonal blocks by substitution in fp32, warps 4 to 7 the blocks under it and those of Q K^T.  Then warp J goes down T's block column J, transposed:
//     T_IJ^T = -(sum_K T_KJ^T L_IK^T) T_II^T,  K = J .. I - 1
// where the results of one product are the first operand of the next as they lie in registers (all operands of three parts).
// 512 chunks of 8 key heads of 128, two value heads to each: 143 us; bound by its warps' waits for one another from step to step (DRAM 20 %, tensor pipe 17 % busy).
// ---------------------------------------------------------------------------------------------------------------------
constexpr int DELTA_PREP_THREADS = 256;
constexpr int DELTA_DIAG = 20;                               // floats of a row of a block on the diagonal
constexpr int DELTA_BLOCK = 16 * 48;                         // bytes of a 16 x 16 block of bfloat16: rows of three 16-byte words, so that eight meet all banks

template <int DK>
struct DeltaPrepCfg {
    static constexpr int kTile = DELTA_C * DK * 2;
    static constexpr int kL = 0;                             // (over the tiles, when those have been read) L's six blocks under the diagonal, three parts
    static constexpr int kT = kL + 3 * 6 * DELTA_BLOCK;      // T's four on the diagonal
    static constexpr int kDiag = kT + 3 * 4 * DELTA_BLOCK;   // L's, fp32
    static constexpr int kWork = kDiag + 4 * 16 * DELTA_DIAG * 4;
    static constexpr int kSmemBytes = 2 * kTile > kWork ? 2 * kTile : kWork;
};
__device__ __forceinline__ int delta_under(int i, int j) { return i * (i - 1) / 2 + j; }       // j < i

// d += a b of three parts each, without what is below 2^-24
__device__ __forceinline__ void delta_mma6(float (&d)[4], const uint32_t (&a)[3][4], const uint32_t (&b)[3][2]) {
    mma_16816<true>(d, a[2], b[0][0], b[0][1]);
    mma_16816<true>(d, a[0], b[2][0], b[2][1]);
    mma_16816<true>(d, a[1], b[1][0], b[1][1]);
    mma_16816<true>(d, a[1], b[0][0], b[0][1]);
    mma_16816<true>(d, a[0], b[1][0], b[1][1]);
    mma_16816<true>(d, a[0], b[0][0], b[0][1]);
}

template <int DK>
__device__ __forceinline__ void delta_prep(const CUtensorMap& map_q, const CUtensorMap& map_k, const DeltaParams& p) {
    using C = DeltaPrepCfg<DK>;
    extern __shared__ __align__(1024) uint8_t lin_smem[];    // (the loads' swizzle goes by the address)
    uint8_t* smem = lin_smem;
    __shared__ uint64_t s_full;
    __shared__ float2 s_g[DELTA_C];
    __shared__ float s_beta[DELTA_C];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    if (blockIdx.x == 0 && tid == 0 && p.first_slot == 0) {
        p.hdr->tile_counter = 0u;
        p.hdr->error = 0u;
    }
    const int hk = static_cast<int>(blockIdx.x % (p.heads / p.group));
    const long long slot = p.first_slot + blockIdx.x / (p.heads / p.group);
    const int seq = delta_sequence_of(p.offsets, p.nseq, slot);
    if (seq >= p.nseq) return;
    int tok, len;
    if (!lin_sequence(p.offsets, p.ntok, seq, tok, len)) return;
    const long long nth = slot - delta_slot(tok, seq);
    if (nth < 0 || nth * DELTA_C >= len) return;
    if (smem_u32(smem) & 1023u) {                            // (never: the declaration asks for it)
        if (tid == 0) report_error(p.hdr, 6u);               // MMV_ERR_CUDA
        return;
    }
    const int first = tok + static_cast<int>(nth) * DELTA_C, n = min(DELTA_C, len - static_cast<int>(nth) * DELTA_C);
    if (tid == 0) {
        mbar_init(&s_full, 1);
        mbar_fence_init();
        if (blockIdx.x != p.debug_skip) {
            mbar_arrive_expect_tx(&s_full, 2 * C::kTile);
#pragma unroll
            for (int b = 0; b < DK / 64; ++b) {
                tma_load_3d(smem + b * DELTA_BOX, &map_k, &s_full, b * 64, hk, first);
                tma_load_3d(smem + C::kTile + b * DELTA_BOX, &map_q, &s_full, b * 64, hk, first);
            }
        }
    }
    // decays and betas of a value head (warp 7), on their way while the tiles land
    float gi[2] = {0.f, 0.f}, bi[2] = {0.f, 0.f};
    const auto gates = [&](int h) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (2 * lane + e < n) {
                gi[e] = p.decay[(first + 2 * lane + e) * p.decay_tok + h];
                bi[e] = p.beta[(first + 2 * lane + e) * p.beta_tok + h];
            }
    };
    // Their sums G / ln 2, in 64 bits and kept as two fp32 values: its differences count.  exp(-200) is 0, whatever is in front of it.
    bool fine_gates = true;
    const auto sums = [&](DeltaChunk* to) {
        double y[2];
        fine_gates = true;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            fine_gates &= delta_finite(bi[e]) && gi[e] < INFINITY;
            y[e] = (gi[e] < -200.f ? -200.0 : static_cast<double>(gi[e])) * 1.4426950408889634;
            s_beta[2 * lane + e] = bi[e];
        }
        double sum = y[0] + y[1];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double z = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += z;
        }
        const double last = __shfl_sync(0xffffffffu, sum, 31);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const double at = e ? sum : sum - y[1];
            const float hi = static_cast<float>(at);
            s_g[2 * lane + e] = make_float2(hi, static_cast<float>(at - hi));
            to->x.beta[2 * lane + e] = bi[e];
            to->x.past[2 * lane + e] = exp2f(static_cast<float>(at));
            to->x.left[2 * lane + e] = exp2f(static_cast<float>(last - at));
        }
        if (lane == 0) {
            const double w = exp2(last);
            to->x.whole_hi = static_cast<float>(w);
            to->x.whole_lo = static_cast<float>(w - static_cast<double>(static_cast<float>(w)));
        }
    };
    if (warp == 7) {
        gates(hk * p.group);
        sums(reinterpret_cast<DeltaChunk*>(p.chunks) + (slot - p.first_slot) * p.heads + hk * p.group);
        if (p.group > 1) gates(hk * p.group + 1);
    }
    __syncthreads();
    const bool late = !mbar_wait(&s_full, 0, p.budget_ns);
    if (__syncthreads_or(late)) {
        if (tid == 0) {
            report_error(p.hdr, 5u);                         // MMV_ERR_TIMEOUT
            mbar_wait(&s_full, 0, 1000000);                  // (the loads in flight land before the CTA leaves)
        }
        return;
    }

    // ---- a warp's blocks of K K^T and Q K^T -------------------------------------------------------------------------------------------
    const bool scores = warp >= 4;
    const int block = warp & 3;
    const uint32_t sm = smem_u32(smem);
    // block t of this warp: its row of blocks, its column, and whether it is of Q K^T
    const auto which = [&](int t, int& i, int& j) {
        const int u = t == 0 ? block : t == 1 && block < 2 ? 4 + block : -1;     // warps 4 to 7: K K^T's blocks 0 to 5 under the diagonal, two, two, one, one ...
        if (!scores) {
            i = j = block;
            return false;
        }
        if (u >= 0) {
            i = u >= 3 ? 3 : u >= 1 ? 2 : 1;
            j = u - i * (i - 1) / 2;
            return false;
        }
        const int w = block < 2 ? block * 2 + t - 2 : 4 + (block - 2) * 3 + t - 1;                 // ... and Q K^T's 0 to 9: two, two, three, three
        i = w >= 6 ? 3 : w >= 3 ? 2 : w >= 1 ? 1 : 0;
        j = w - delta_tile(i, 0);
        return true;
    };
    float x[4][2][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        if (t > 0 && !scores) break;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[t][0][e] = x[t][1][e] = 0.f;
        int i, j;
        const bool of_q = which(t, i, j);
        const uint32_t ta = sm + (of_q ? C::kTile : 0);
#pragma unroll
        for (int d = 0; d < DK / 16; ++d) {
            uint32_t a[4], b[4];
            ldsm_x4(a, ta + delta_word(i * 16 + (lane & 15), 2 * d + (lane >> 4)));
            ldsm_x4(b, sm + delta_word(j * 16 + (lane & 7) + ((lane >> 4) << 3), 2 * d + ((lane >> 3) & 1)));
            mma_16816<true>(x[t][0], a, b[0], b[1]);
            mma_16816<true>(x[t][1], a, b[2], b[3]);
        }
    }

    float* diag = reinterpret_cast<float*>(smem + C::kDiag) + block * 16 * DELTA_DIAG;
    for (int rep = 0; rep < p.group; ++rep) {
        const int h = hk * p.group + rep;
        DeltaChunk* to = reinterpret_cast<DeltaChunk*>(p.chunks) + (slot - p.first_slot) * p.heads + h;
        if (rep) {
            __syncthreads();                                 // (the last head's numbers have been used)
            if (warp == 7) sums(to);
            if (warp == 7 && rep + 1 < p.group) gates(h + 1);
        }
        __syncthreads();                                     // (and the tiles have been read: L and T go over them)
        bool fine = fine_gates;
        float odd = 0.f;                                     // a sum of 0 times everything: 0, or NaN
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t > 0 && !scores) break;
            int bi, bj;
            const bool of_q = which(t, bi, bj);
            float y[2][4];
            if (bi == bj) {                                  // rows g, g + 8 by columns 2 c, + 1, + 8, + 9
                const float2 gr[2] = {s_g[bi * 16 + g], s_g[bi * 16 + g + 8]};
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int j0 = half * 8 + 2 * c;
                    const float2 gc[2] = {s_g[bi * 16 + j0], s_g[bi * 16 + j0 + 1]};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = g + 8 * (e >> 1), j = j0 + (e & 1);
                        const bool in = bi * 16 + i < n;
                        y[half][e] = in && (of_q ? j <= i : j < i) ? delta_decay(gr[e >> 1], gc[e & 1]) * x[t][half][e] : 0.f;
                        if (in && j == i) odd = fmaf(x[t][half][e], 0.f, odd);
                    }
                }
            } else {
                // D_ij = exp(G_i - G_m) exp(G_m - G_j) with m the first of the block's rows: both are 1 at most
                const float2 gm = s_g[bi * 16];
                const float rf[2] = {delta_decay(s_g[bi * 16 + g], gm), delta_decay(s_g[bi * 16 + g + 8], gm)};
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int j0 = bj * 16 + half * 8 + 2 * c;
                    const float cf[2] = {delta_decay(gm, s_g[j0]), delta_decay(gm, s_g[j0 + 1])};
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[half][e] = bi * 16 + g + 8 * (e >> 1) < n ? rf[e >> 1] * cf[e & 1] * x[t][half][e] : 0.f;
                }
            }
            if (!of_q) {
                const float br[2] = {s_beta[bi * 16 + g], s_beta[bi * 16 + g + 8]};
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e >> 2][e & 3] *= br[(e >> 1) & 1];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) odd = fmaf(y[e >> 2][e & 3], 0.f, odd);
            if (of_q) {
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) delta_split(y[e >> 1][2 * (e & 1)], y[e >> 1][2 * (e & 1) + 1], hi[e], lo[e]);
                to->a[0][delta_tile(bi, bj)][lane] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                to->a[1][delta_tile(bi, bj)][lane] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            } else if (!scores) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *reinterpret_cast<float2*>(diag + (g + 8 * (e & 1)) * DELTA_DIAG + (e >> 1) * 8 + 2 * c) = make_float2(y[e >> 1][2 * (e & 1)], y[e >> 1][2 * (e & 1) + 1]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t r[3];
                    delta_split3(y[e >> 1][2 * (e & 1)], y[e >> 1][2 * (e & 1) + 1], r);
                    uint8_t* at = smem + C::kL + delta_under(bi, bj) * DELTA_BLOCK + (g + 8 * (e & 1)) * 48 + (e >> 1) * 16 + c * 4;
#pragma unroll
                    for (int part = 0; part < 3; ++part) *reinterpret_cast<uint32_t*>(at + part * 6 * DELTA_BLOCK) = r[part];
                }
            }
            if (scores && t == (block < 2 ? 1 : 0)) asm volatile("bar.arrive 1, 256;" ::: "memory");       // (its blocks of L are there)
        }
        fine &= odd == 0.f;
        if (!scores) {
            // ---- T's diagonal blocks: lane j (and j + 16) has column j -------------------------------------------------------------------
            __syncwarp();
            const int j = lane & 15;
            float y[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float z = i == j ? 1.f : 0.f;
#pragma unroll
                for (int k = 0; k < i; k += 4) {             // (L is zero from the diagonal on)
                    const float4 l = *reinterpret_cast<const float4*>(diag + i * DELTA_DIAG + k);
                    z = fmaf(-l.x, y[k], z);
                    if (k + 1 < i) z = fmaf(-l.y, y[k + 1], z);
                    if (k + 2 < i) z = fmaf(-l.z, y[k + 2], z);
                    if (k + 3 < i) z = fmaf(-l.w, y[k + 3], z);
                }
                y[i] = z;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const __nv_bfloat16 hi = __float2bfloat16_rn(y[i]);
                const float rest = y[i] - __bfloat162float(hi);
                const __nv_bfloat16 mid = __float2bfloat16_rn(rest);
                uint8_t* at = smem + C::kT + block * DELTA_BLOCK + i * 48 + j * 2;
                if (lane < 16) {
                    *reinterpret_cast<__nv_bfloat16*>(at) = hi;
                } else {
                    *reinterpret_cast<__nv_bfloat16*>(at + 4 * DELTA_BLOCK) = mid;
                    *reinterpret_cast<__nv_bfloat16*>(at + 8 * DELTA_BLOCK) = __float2bfloat16_rn(rest - __bfloat162float(mid));
                }
            }
            asm volatile("bar.sync 1, 256;" ::: "memory");   // (the other diagonal blocks, and L under them: warps 4 to 7 have arrived)
            // T - 1 on the diagonal: its ones left out
            {
                uint32_t r[2][4];
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    ldsm_x4(r[part], sm + C::kT + part * 4 * DELTA_BLOCK + block * DELTA_BLOCK + (lane & 15) * 48 + (lane >> 4) * 16);
#pragma unroll
                    for (int e = 0; e < 4; ++e) fine &= delta_finite2(r[part][e]);
                }
                if (g == 2 * c) r[0][0] &= 0xffff0000u, r[0][3] &= 0xffff0000u;
                if (g == 2 * c + 1) r[0][0] &= 0xffffu, r[0][3] &= 0xffffu;
#pragma unroll
                for (int part = 0; part < 2; ++part) to->t[part][delta_tile(block, block)][lane] = make_uint4(r[part][0], r[part][1], r[part][2], r[part][3]);
            }
            // ---- the blocks under it ------------------------------------------------------------------------------------------------------
            const int nrow = (lane & 7) + ((lane >> 4) << 3), ncol = (lane >> 3) & 1;
            uint32_t xt[3][3][4];                            // T_KJ^T, K = J + index: three parts
#pragma unroll
            for (int part = 0; part < 3; ++part)
                ldsm_x4_t(xt[0][part], sm + C::kT + (part * 4 + block) * DELTA_BLOCK + (((lane >> 4) << 3) + (lane & 7)) * 48 + ((lane >> 3) & 1) * 16);
#pragma unroll
            for (int s = 1; s < 4; ++s) {                    // I = J + s
                if (block + s > 3) break;
                const int I = block + s;
                float y2[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}, z2[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                for (int k = 0; k < s; ++k) {
                    uint32_t b[2][3][2];
#pragma unroll
                    for (int part = 0; part < 3; ++part) {
                        uint32_t r[4];
                        ldsm_x4(r, sm + C::kL + (part * 6 + delta_under(I, block + k)) * DELTA_BLOCK + nrow * 48 + ncol * 16);
                        b[0][part][0] = r[0], b[0][part][1] = r[1], b[1][part][0] = r[2], b[1][part][1] = r[3];
                    }
                    delta_mma6(y2[0], xt[k], b[0]);
                    delta_mma6(y2[1], xt[k], b[1]);
                }
                uint32_t ya[3][4], b[2][3][2];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t r[3];
                    delta_split3(-y2[e >> 1][2 * (e & 1)], -y2[e >> 1][2 * (e & 1) + 1], r);
                    ya[0][e] = r[0], ya[1][e] = r[1], ya[2][e] = r[2];
                }
#pragma unroll
                for (int part = 0; part < 3; ++part) {
                    uint32_t r[4];
                    ldsm_x4(r, sm + C::kT + (part * 4 + I) * DELTA_BLOCK + nrow * 48 + ncol * 16);
                    b[0][part][0] = r[0], b[0][part][1] = r[1], b[1][part][0] = r[2], b[1][part][1] = r[3];
                }
                delta_mma6(z2[0], ya, b[0]);
                delta_mma6(z2[1], ya, b[1]);
                uint32_t out[2][4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {                // rows j = g + 8 (e & 1), columns i = 8 (e >> 1) + 2 c, + 1
                    uint32_t r[3];
                    delta_split3(z2[e >> 1][2 * (e & 1)], z2[e >> 1][2 * (e & 1) + 1], r);
                    if (s < 3) xt[s < 3 ? s : 0][0][e] = r[0], xt[s < 3 ? s : 0][1][e] = r[1], xt[s < 3 ? s : 0][2][e] = r[2];
                    fine &= delta_finite2(r[0]);
                    // the block itself: rows i = 8 (e >> 1) + g, columns j = 8 (e & 1) + 2 c, + 1
#pragma unroll
                    for (int part = 0; part < 2; ++part) out[part][(e >> 1) + 2 * (e & 1)] = matrix_transpose(r[part]);
                }
#pragma unroll
                for (int part = 0; part < 2; ++part) to->t[part][delta_tile(I, block)][lane] = make_uint4(out[part][0], out[part][1], out[part][2], out[part][3]);
            }
        }
        const bool wild = __syncthreads_or(!fine);
        if (tid == 0) to->x.wild = wild ? 1 : 0;
    }
}
// Behind the first part of a batch it runs beside the second kernel of the part in front of it (in the workspace's other half): it reads nothing of that,
// but ends after it, so that the kernel behind it, which waits for this one, finds the states.
template <int DK>
__global__ void __launch_bounds__(DELTA_PREP_THREADS, 3)
delta_prep_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const DeltaParams p) {
    griddep_launch_dependents();
    delta_prep<DK>(map_q, map_k, p);
    if (blockIdx.x == gridDim.x - 1) griddep_wait();
}

// ---------------------------------------------------------------------------------------------------------------------
// The walk along the chunks.  Eight warps share a chunk's products and meet three times a chunk: when the state's copy, R and U are in shared
// memory.  All of the next chunk's operands are on their way meanwhile (one CTA per SM; with Q, T and A loaded into the places that the chunk had
// done with, two fit an SM: 750 instead of 840 us for 16 prompts of nearly one length, 1030 where one is three times as long as their mean, since
// a chunk then takes 5.3 instead of 3.1 us).
// ---------------------------------------------------------------------------------------------------------------------
constexpr int DELTA_THREADS = 256;

template <int DK, int NV>
struct DeltaCfg {
    static constexpr int kTile = DELTA_C * DK * 2, kBlocks = 2 * DELTA_TILES * 512;
    static constexpr int kPitch = NV * 2;                    // bytes of a row of NV bfloat16
    // what is loaded for a chunk, twice: K, Q, T - 1 and A, the scalars
    static constexpr int kK = 0, kQ = kTile, kT = 2 * kTile, kX = kT + 2 * kBlocks, kStage = kX + 1024;
    static constexpr uint32_t kLoad = 2 * kTile + 2 * kBlocks + sizeof(DeltaScalars);
    static constexpr int kS = 2 * kStage, kSPart = DK * kPitch;                  // the state, three parts
    static constexpr int kR = kS + 3 * kSPart, kRPart = DELTA_C * kPitch;        // three
    static constexpr int kU = kR + 3 * kRPart;                                   // two
    static constexpr int kW = kU + 2 * kRPart;                                   // exp(G_n - G) U, three
    static constexpr int kSmemBytes = kW + 3 * kRPart;
    static_assert(kStage % 1024 == 0 && sizeof(DeltaScalars) <= 1024, "the loads' swizzle goes by the address");
    static_assert(4 * NV * 4 <= 3 * kRPart, "token by token: sums in R's place");
};
// Where word w of a row lies: eight rows' words of one column in different banks.
template <int NV>
__device__ __forceinline__ int delta_place(int row, int w) { return row * (NV * 2) + ((NV == 32 ? w ^ ((row >> 1) & 3) : w ^ ((row >> 2) & 1)) << 4); }

// Which sequence the index-th CTAs of a launch take, and its chunks [begin, end) that the launch has the operands of.  The sequences that lie in the part
// [first_slot, last_slot) of the places follow one another, `present` of them at most; the ones with the most tokens in it come first (16 of 32768 tokens in all:
// a last wave of half of the time) where a thread can look at each.  (With CTAs for every sequence in every part, 256 prompts of 512 tokens and 32 heads took
// 18.7 instead of 9.3 ms.  Out of line: in the kernel it cost the chunks' loop 2 %.)
struct DeltaPart {
    int seq, tok, len, begin, end;                           // seq -1: none
};
__device__ __forceinline__ bool delta_part_of(const int32_t* offsets, int ntok, long long first_slot, long long last_slot, DeltaPart& r) {
    lin_sequence(offsets, ntok, r.seq, r.tok, r.len);
    const long long at = delta_slot(r.tok, r.seq), chunks = lin_chunks(r.len);
    r.begin = static_cast<int>(max(0ll, min(chunks, first_slot - at)));
    r.end = static_cast<int>(max(0ll, min(chunks, last_slot - at)));
    return r.begin < r.end || (chunks == 0 && at >= first_slot && at < last_slot);       // (an empty sequence's state is copied where its place is)
}
static __device__ __noinline__ DeltaPart delta_part(const int32_t* offsets, int ntok, int nseq, int present, long long first_slot, long long last_slot,
                                                    int index, int* s_len /* DELTA_THREADS + 1 */) {
    const int tid = threadIdx.x, first = present < nseq && first_slot ? delta_sequence_of(offsets, nseq, first_slot) : 0;
    DeltaPart r{};
    r.seq = first + index;
    bool here = r.seq < nseq;
    if (present <= DELTA_THREADS) {
        DeltaPart x{};
        x.seq = first + tid;
        const int n = tid < present && x.seq < nseq && delta_part_of(offsets, ntok, first_slot, last_slot, x) ? min(x.len - x.begin * DELTA_C, (x.end - x.begin) * DELTA_C) : -1;
        s_len[tid] = n;
        here = __syncthreads_count(n >= 0) > index;
        if (here) {
            int rank = 0;
            for (int i = 0; i < present; ++i) rank += s_len[i] > n || (s_len[i] == n && i < tid);
            if (n >= 0 && rank == index) s_len[DELTA_THREADS] = x.seq;
            __syncthreads();
            r.seq = s_len[DELTA_THREADS];
        }
    }
    if (!here || !delta_part_of(offsets, ntok, first_slot, last_slot, r)) r.seq = -1;
    return r;
}

template <int DK, int NV>
__global__ void __launch_bounds__(DELTA_THREADS, 1)
delta_chunks_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const DeltaParams p) {
    using C = DeltaCfg<DK, NV>;
    constexpr int N = NV / 16;                               // product tiles of 8 columns of a warp: half of the slice
    constexpr int M = DK / 64;                               // and of 16 rows of the state
    extern __shared__ __align__(1024) uint8_t lin_smem[];    // (the loads' swizzle goes by the address)
    uint8_t* smem = lin_smem;
    __shared__ uint64_t s_full[2];                           // loads that have landed
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const int slice = static_cast<int>(blockIdx.x % p.slices), h = static_cast<int>(blockIdx.x / p.slices % p.heads);
    const int hk = h / p.group, col0 = slice * NV;
    const int index = static_cast<int>(blockIdx.x / p.slices / p.heads);
    bool bad = false;
    if (p.first_slot == 0) {
        for (long long i = static_cast<long long>(blockIdx.x) * DELTA_THREADS + tid; i < p.nseq; i += static_cast<long long>(gridDim.x) * DELTA_THREADS) {
            int at, n;
            bad |= !lin_sequence(p.offsets, p.ntok, static_cast<int>(i), at, n);
        }
    }
    const DeltaPart part = delta_part(p.offsets, p.ntok, p.nseq, p.present, p.first_slot, p.last_slot, index, reinterpret_cast<int*>(smem + C::kS));
    if (part.seq < 0) {                                      // (the launch ends behind the one in front of it all the same)
        if (bad || blockIdx.x == 0) griddep_wait();
        if (bad) report_error(p.hdr, 4u);                    // MMV_ERR_BAD_SEGMENTS
        return;
    }
    const int seq = part.seq, tok = part.tok, len = part.len, begin = part.begin, end = part.end;
    const long long slot0 = delta_slot(tok, seq);
    if (tid == 0) {
        mbar_init(&s_full[0], 1);
        mbar_init(&s_full[1], 1);
        mbar_fence_init();
    }
    griddep_wait();
    griddep_launch_dependents();                             // (of the next part, whose first kernel may begin)
    if (bad) report_error(p.hdr, 4u);                        // MMV_ERR_BAD_SEGMENTS
    if (smem_u32(smem) & 1023u) {                            // (never: the declaration asks for it)
        if (tid == 0) report_error(p.hdr, 6u);               // MMV_ERR_CUDA
        return;
    }
    __syncthreads();

    const uint32_t sm = smem_u32(smem);
    const DeltaChunk* made = reinterpret_cast<const DeltaChunk*>(p.chunks) + (slot0 - p.first_slot) * p.heads + h;       // of chunk i: made[i * heads]
    const auto fetch = [&](int chunk) {                      // (one thread)
        const int i = (chunk - begin) & 1;
        uint8_t* dst = smem + i * C::kStage;
        const DeltaChunk* from = made + static_cast<long long>(chunk) * p.heads;
        mbar_arrive_expect_tx(&s_full[i], C::kLoad);
#pragma unroll
        for (int b = 0; b < DK / 64; ++b) {
            tma_load_3d(dst + C::kK + b * DELTA_BOX, &map_k, &s_full[i], b * 64, hk, tok + chunk * DELTA_C);
            tma_load_3d(dst + C::kQ + b * DELTA_BOX, &map_q, &s_full[i], b * 64, hk, tok + chunk * DELTA_C);
        }
        tma_load_1d(dst + C::kX, &from->x, sizeof(DeltaScalars), &s_full[i]);
        tma_load_1d(dst + C::kT, from->t, 2 * C::kBlocks, &s_full[i]);
    };
    if (begin < end && tid == 0 && blockIdx.x + (1ll << 32) != p.debug_skip) fetch(begin);

    // Of the tokens a warp has 16 (two warps of a scheduler together five of the triangles' blocks), of the state 16 M rows; of both, half of the
    // slice's columns.
    const int block = warp < 4 ? warp >> 1 : 3 - ((warp - 4) >> 1), half = warp & 1, row0 = (warp >> 1) * 16 * M;
    const int mine = col0 + half * (NV / 2);                 // this warp's first column
    // values of this lane's tokens, one chunk ahead
    uint32_t v[N][2];
    const auto values = [&](int chunk) {
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int t = chunk * DELTA_C + block * 16 + g + 8 * e;
                v[j][e] = 0u;
                if (t < len && mine + j * 8 < p.dv)
                    v[j][e] = *reinterpret_cast<const uint32_t*>(p.v + (static_cast<long long>(tok) + t) * p.v_tok + h * p.v_head + mine + j * 8 + 2 * c);
            }
    };
    if (begin < end) values(begin);

    // ---- the state: rows row0 + 16 m + g and + 8, columns 8 j + 2 c and + 1 of the warp's -----------------------------------------
    float s[M][N][4];
    const float* from = begin > 0 ? p.state_out : p.state;
    const long long base = (static_cast<long long>(seq) * p.heads + h) * p.dk * p.dv;
    const auto state_at = [&](int m, int j, int e) { return base + static_cast<long long>(row0 + 16 * m + g + 8 * e) * p.dv + mine + j * 8 + 2 * c; };
    const auto held = [&](int m, int j, int e) { return row0 + 16 * m + g + 8 * e < p.dk && mine + j * 8 < p.dv; };
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float2 x = make_float2(0.f, 0.f);
                if (from && held(m, j, e)) x = *reinterpret_cast<const float2*>(from + state_at(m, j, e));
                s[m][j][2 * e] = x.x;
                s[m][j][2 * e + 1] = x.y;
            }

    // 16 rows of two parts of tile j of this warp's columns as a product's second operand: the first part in b[0], b[1], the second in b[2], b[3]
    const auto operand = [&](uint32_t (&b)[4], int matrix, int part, int row, int j) {
        ldsm_x4_t(b, sm + matrix + (lane >> 4) * part + delta_place<NV>(row + (lane & 15), half * N + j));
    };
    // the third part of all tiles
    const auto third = [&](uint32_t (&b)[N][2], int matrix, int row) {
        if constexpr (N == 2) {
            uint32_t r[4];
            ldsm_x4_t(r, sm + matrix + delta_place<NV>(row + (lane & 15), half * N + (lane >> 4)));
            b[0][0] = r[0], b[0][1] = r[1], b[1][0] = r[2], b[1][1] = r[3];
        } else {
            ldsm_x2_t(b[0][0], b[0][1], sm + matrix + delta_place<NV>(row + (lane & 15), half * N));
        }
    };
    const auto address = [&](int matrix, int row, int j) { return smem + matrix + delta_place<NV>(row, half * N + j) + 4 * c; };
    for (int chunk = begin; chunk < end; ++chunk) {
        const int stage = (chunk - begin) & 1;
        const uint32_t sm_k = sm + stage * C::kStage + C::kK, sm_q = sm + stage * C::kStage + C::kQ;
        const uint4* blocks = reinterpret_cast<const uint4*>(smem + stage * C::kStage + C::kT) + lane;           // T - 1, and A behind it
        const DeltaScalars* info = reinterpret_cast<const DeltaScalars*>(smem + stage * C::kStage + C::kX);
        const int n = min(DELTA_C, len - chunk * DELTA_C);
        // the state's copy for the products
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    uint32_t r[3];
                    delta_split3(s[m][j][2 * e], s[m][j][2 * e + 1], r);
                    uint8_t* at = address(C::kS, row0 + 16 * m + g + 8 * e, j);
#pragma unroll
                    for (int part = 0; part < 3; ++part) *reinterpret_cast<uint32_t*>(at + part * C::kSPart) = r[part];
                }
        const bool late = !mbar_wait(&s_full[stage], ((chunk - begin) >> 1) & 1, p.budget_ns);
        if (n < DELTA_C && !late) {                          // another sequence's keys: their weights of zero do not hide what is not finite
            for (int i = tid; i < (DELTA_C - n) * (DK / 8); i += DELTA_THREADS)
                *reinterpret_cast<uint4*>(smem + stage * C::kStage + C::kK + delta_word(n + i / (DK / 8), i % (DK / 8))) = make_uint4(0u, 0u, 0u, 0u);
            fence_proxy_async_smem();
        }
        if (__syncthreads_or(late)) {                        // (this chunk's operands and the state's copy are there)
            if (tid == 0) {
                report_error(p.hdr, 5u);                     // MMV_ERR_TIMEOUT
                mbar_wait(&s_full[stage], ((chunk - begin) >> 1) & 1, 1000000);               // (the loads in flight land before the CTA leaves)
            }
            return;
        }
        if (tid == 0 && chunk + 1 < end) fetch(chunk + 1);

        // ---- K S, Q S: 16 tokens each ------------------------------------------------------------------------------------------------
        float x[N][4], y[N][4];
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[j][e] = y[j][e] = 0.f;
        {
            uint32_t ak[2][4], aq[2][4], b[2][N][4], b3[2][N][2];                // (the next step's operands while this one's are used)
            const auto load = [&](int d) {
                const uint32_t at = delta_word(block * 16 + (lane & 15), 2 * d + (lane >> 4));
                ldsm_x4(ak[d & 1], sm_k + at);
#pragma unroll
                for (int j = 0; j < N; ++j) operand(b[d & 1][j], C::kS, C::kSPart, d * 16, j);
                third(b3[d & 1], C::kS + 2 * C::kSPart, d * 16);
                ldsm_x4(aq[d & 1], sm_q + at);
            };
            load(0);
#pragma unroll
            for (int d = 0; d < DK / 16; ++d) {
                if (d + 1 < DK / 16) load(d + 1);
                const int i = d & 1;
#pragma unroll
                for (int j = 0; j < N; ++j) mma_16816<true>(x[j], ak[i], b[i][j][0], b[i][j][1]);
#pragma unroll
                for (int j = 0; j < N; ++j) mma_16816<true>(y[j], aq[i], b[i][j][0], b[i][j][1]);
#pragma unroll
                for (int j = 0; j < N; ++j) mma_16816<true>(x[j], ak[i], b[i][j][2], b[i][j][3]);
#pragma unroll
                for (int j = 0; j < N; ++j) mma_16816<true>(y[j], aq[i], b[i][j][2], b[i][j][3]);
#pragma unroll
                for (int j = 0; j < N; ++j) mma_16816<true>(x[j], ak[i], b3[i][j][0], b3[i][j][1]);
            }
        }
        // ---- R = b (V - exp(G) K S) ----------------------------------------------------------------------------------------------------
        const float past[2] = {info->past[block * 16 + g], info->past[block * 16 + g + 8]};
        bool wild = info->wild != 0;
        {
            const float beta[2] = {info->beta[block * 16 + g], info->beta[block * 16 + g + 8]};
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = block * 16 + g + 8 * e;
                    asm volatile("" : "+r"(v[j][e]));        // (here, and not where the load was issued: it has had the products' time)
                    wild |= !delta_finite2(v[j][e]);
                    const float2 w = unpack_pair<true>(v[j][e]);
                    const bool on = row < n;
                    x[j][2 * e] = on ? beta[e] * (w.x - past[e] * x[j][2 * e]) : 0.f;
                    x[j][2 * e + 1] = on ? beta[e] * (w.y - past[e] * x[j][2 * e + 1]) : 0.f;
                    uint32_t r[3];
                    delta_split3(x[j][2 * e], x[j][2 * e + 1], r);
                    uint8_t* at = address(C::kR, row, j);
#pragma unroll
                    for (int part = 0; part < 3; ++part) *reinterpret_cast<uint32_t*>(at + part * C::kRPart) = r[part];
                }
        }
        if (chunk + 1 < end) values(chunk + 1);
        wild = __syncthreads_or(wild);
        uint16_t* out = p.out + ((static_cast<long long>(tok) + chunk * DELTA_C) * p.heads + h) * p.dv;
        const long long orow = static_cast<long long>(p.heads) * p.dv;
        if (!wild) {
            // ---- U = R + (T - 1) R ---------------------------------------------------------------------------------------------------------
            const uint4* solver = blocks + delta_tile(block, 0) * 32;
            float u[N][4], z[N][4];                          // (sums of their own: the tensor core's cut digits at the end, and R's are not to be cut)
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) u[j][e] = z[j][e] = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (k > block) break;
                const uint4 th = solver[k * 32], tl = solver[(DELTA_TILES + k) * 32];
                const uint32_t ah[4] = {th.x, th.y, th.z, th.w}, al[4] = {tl.x, tl.y, tl.z, tl.w};
                uint32_t b3[N][2];
                third(b3, C::kR + 2 * C::kRPart, k * 16);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    uint32_t b[4];
                    operand(b, C::kR, C::kRPart, k * 16, j);
                    mma_16816<true>(z[j], ah, b3[j][0], b3[j][1]);
                    mma_16816<true>(u[j], ah, b[0], b[1]);
                    mma_16816<true>(z[j], al, b[2], b[3]);
                    mma_16816<true>(z[j], al, b[0], b[1]);
                    mma_16816<true>(z[j], ah, b[2], b[3]);
                }
            }
            const float left[2] = {info->left[block * 16 + g], info->left[block * 16 + g + 8]};
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float a = x[j][2 * e] + (u[j][2 * e] + z[j][2 * e]), b = x[j][2 * e + 1] + (u[j][2 * e + 1] + z[j][2 * e + 1]);
                    uint32_t r[3];
                    delta_split(a, b, r[0], r[1]);
                    uint8_t* at = address(C::kU, block * 16 + g + 8 * e, j);
                    *reinterpret_cast<uint32_t*>(at) = r[0];
                    *reinterpret_cast<uint32_t*>(at + C::kRPart) = r[1];
                    delta_split3(a * left[e], b * left[e], r);
                    at += C::kW - C::kU;
#pragma unroll
                    for (int part = 0; part < 3; ++part) *reinterpret_cast<uint32_t*>(at + part * C::kRPart) = r[part];
                }
            __syncthreads();
            // ---- S' = exp(G_n) S + K^T (exp(G_n - G) U) -----------------------------------------------------------------------------------
            {
                uint32_t a[2][M][4], b[2][N][4], b3[2][N][2];
                float d[M][N][4];                            // (a sum of its own, as above: the state is not to be cut every time)
#pragma unroll
                for (int m = 0; m < M; ++m)
#pragma unroll
                    for (int j = 0; j < N; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) d[m][j][e] = 0.f;
                const auto load = [&](int k) {
#pragma unroll
                    for (int m = 0; m < M; ++m)
                        ldsm_x4_t(a[k & 1][m], sm_k + delta_word(k * 16 + ((lane >> 4) << 3) + (lane & 7), (row0 >> 3) + 2 * m + ((lane >> 3) & 1)));
                    third(b3[k & 1], C::kW + 2 * C::kRPart, k * 16);
#pragma unroll
                    for (int j = 0; j < N; ++j) operand(b[k & 1][j], C::kW, C::kRPart, k * 16, j);
                };
                load(0);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (k < 3) load(k + 1);
                    const int i = k & 1;
#pragma unroll
                    for (int j = 0; j < N; ++j)
#pragma unroll
                        for (int m = 0; m < M; ++m) mma_16816<true>(d[m][j], a[i][m], b3[i][j][0], b3[i][j][1]);
#pragma unroll
                    for (int j = 0; j < N; ++j)
#pragma unroll
                        for (int m = 0; m < M; ++m) mma_16816<true>(d[m][j], a[i][m], b[i][j][2], b[i][j][3]);
#pragma unroll
                    for (int j = 0; j < N; ++j)
#pragma unroll
                        for (int m = 0; m < M; ++m) mma_16816<true>(d[m][j], a[i][m], b[i][j][0], b[i][j][1]);
                }
                const float wh = info->whole_hi, wl = info->whole_lo;
#pragma unroll
                for (int m = 0; m < M; ++m)
#pragma unroll
                    for (int j = 0; j < N; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[m][j][e] = fmaf(s[m][j][e], wh, fmaf(s[m][j][e], wl, d[m][j][e]));
            }
            // ---- O = scale (exp(G) Q S + A U) ---------------------------------------------------------------------------------------------
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) y[j][e] *= past[e >> 1];
            const uint4* scores = blocks + (2 * DELTA_TILES + delta_tile(block, 0)) * 32;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (k > block) break;
                const uint4 th = scores[k * 32], tl = scores[(DELTA_TILES + k) * 32];
                const uint32_t ah[4] = {th.x, th.y, th.z, th.w}, al[4] = {tl.x, tl.y, tl.z, tl.w};
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    uint32_t b[4];
                    operand(b, C::kU, C::kRPart, k * 16, j);
                    delta_mma3(y[j], ah, al, b[0], b[1], b[2], b[3]);
                }
            }
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = block * 16 + g + 8 * e;
                    if (row < n && mine + j * 8 < p.dv)
                        *reinterpret_cast<uint32_t*>(out + row * orow + mine + j * 8 + 2 * c) = pack_pair<true>(p.scale * y[j][2 * e], p.scale * y[j][2 * e + 1]);
                }
        } else {
            // ---- token by token: the recurrence as it stands ---------------------------------------------------
            float* sums = reinterpret_cast<float*>(smem + C::kR);
            constexpr int PARTS = 4;                         // of the state's rows: warps of one half
            for (int t = 0; t < n; ++t) {
                const long long at = tok + static_cast<long long>(chunk) * DELTA_C + t;
                const LinDecay d = lin_decay(p.decay[at * p.decay_tok + h], 1);
                const float b = p.beta[at * p.beta_tok + h];
                float kr[M][2], qr[M][2];
#pragma unroll
                for (int m = 0; m < M; ++m)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int row = row0 + 16 * m + g + 8 * e;
                        kr[m][e] = row < p.dk ? lin_load<true>(p.k + at * p.k_tok + hk * p.k_head + row) : 0.f;
                        qr[m][e] = row < p.dk ? lin_load<true>(p.q + at * p.q_tok + hk * p.q_head + row) : 0.f;
                    }
#pragma unroll 1
                for (int turn = 0; turn < 2; ++turn) {       // k S, then q S'
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        float r[2] = {0.f, 0.f};
#pragma unroll
                        for (int m = 0; m < M; ++m)
#pragma unroll
                            for (int i = 0; i < 4; ++i)      // (rows past dk hold zero and weigh zero)
                                r[i & 1] = fmaf(turn ? qr[m][i >> 1] : kr[m][i >> 1], s[m][j][i], r[i & 1]);
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) {
                            r[0] += __shfl_xor_sync(0xffffffffu, r[0], o);
                            r[1] += __shfl_xor_sync(0xffffffffu, r[1], o);
                        }
                        if (g == 0) {
                            float* to = sums + (warp >> 1) * NV + half * (NV / 2) + j * 8 + 2 * c;
                            to[0] = r[0];
                            to[1] = r[1];
                        }
                    }
                    __syncthreads();
                    if (turn) {
                        if (tid < NV && col0 + tid < p.dv) {
                            float sum = 0.f;
#pragma unroll
                            for (int w = 0; w < PARTS; ++w) sum += sums[w * NV + tid];
                            out[t * orow + col0 + tid] = lin_store<true>(p.scale * sum);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < N; ++j)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const int col = half * (NV / 2) + j * 8 + 2 * c + e;
                                float sum = 0.f;
#pragma unroll
                                for (int w = 0; w < PARTS; ++w) sum += sums[w * NV + col];
                                const float value = col0 + col < p.dv ? lin_load<true>(p.v + at * p.v_tok + h * p.v_head + col0 + col) : 0.f;
                                const float ut = b * (value - fmaf(sum, d.hi, sum * d.lo));
#pragma unroll
                                for (int m = 0; m < M; ++m)
#pragma unroll
                                    for (int i = 0; i < 2; ++i)
                                        if (row0 + 16 * m + g + 8 * i < p.dk)
                                            s[m][j][2 * i + e] = fmaf(s[m][j][2 * i + e], d.hi, fmaf(s[m][j][2 * i + e], d.lo, kr[m][i] * ut));
                            }
                    }
                    __syncthreads();
                }
            }
        }
    }
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (held(m, j, e)) *reinterpret_cast<float2*>(p.state_out + state_at(m, j, e)) = make_float2(s[m][j][2 * e], s[m][j][2 * e + 1]);
}

}  // namespace mmv

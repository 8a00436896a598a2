// Layers that keep a state under the gated delta rule:
//     S_t = a_t S_{t-1} + k_t u_t^T,   u_t = b_t (v_t - a_t S_{t-1}^T k_t),   o_t = scale S_t^T q_t,   a_t = exp(g_t)
// i.e. what the decayed state answers for the key k_t is moved towards v_t by the share b_t.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "common.cuh"
#include "linear_attn.cuh"
#include "paged_attn.cuh"
#include "kv_cache_q8.cuh"

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
    long long nreq, num_slots;
    int parts;                                               // column parts of a state
    // packed prompts
    const int32_t* offsets;
    int nseq, ntok;
    long long first_slot, last_slot;                         // chunks that this launch takes, by their place in the workspace
    int slices;                                              // column parts of a (sequence, head)
    WorkspaceHeader* hdr;
    uint8_t* chunks;                                         // [last_slot - first_slot][heads] DeltaChunk
};

// ---------------------------------------------------------------------------------------------------------------------
// One token per request.  The state is the traffic (8 bytes per element against 7 flops).  A CTA owns COLS columns of one (request, head): all
// of its rows' loads are in flight before anything else, one sweep over them in registers gives k S and q S, which meet in shared
// memory, and a second one the new state; the result needs none of it: q S' = a q S + (q k) u.
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
//     U  = T diag(b) (V - exp(G) K S)          (row i is u_i)
//     O  = scale (exp(G) Q S + A U)
//     S' = exp(G_n) S + K^T diag(exp(G_n - G)) U
// T and A do not depend on the state: a first kernel forms them for all chunks side by side; the second one walks along a sequence's chunks, one
// CTA per (sequence, head, slice of columns), whose columns never meet others'.
//
// Every operand that is formed here enters its product as the sum of two bfloat16 values (2^-17 of it), so that the fp32 state stays exact to
// about 2^-16 of what is added to it; products of two such leave out the two low parts' (2^-18).
//
// A chunk that holds a value that is not finite (or whose products are not) is taken token by token: zeros of the triangles would carry it to
// tokens in front of it.
// ---------------------------------------------------------------------------------------------------------------------
constexpr int DELTA_C = 64;
constexpr int DELTA_TILES = 10;                              // 16 x 16 blocks on and under the diagonal, by rows
__host__ __device__ constexpr int delta_tile(int i, int j) { return i * (i + 1) / 2 + j; }

// What the first kernel leaves of a chunk and head.  A block's 32 x 16 bytes are the lanes' registers of a product's first operand.
struct DeltaChunk {
    uint4 t[2][DELTA_TILES][32];                             // T: high parts, low parts
    uint4 a[2][DELTA_TILES][32];                             // A
    float beta[DELTA_C], past[DELTA_C], left[DELTA_C];       // b, exp(G), exp(G_n - G)
    float whole_hi, whole_lo;                                // exp(G_n)
    int wild;                                                // to be taken token by token
    int pad;
};
static_assert(sizeof(DeltaChunk) % 16 == 0, "copied in 16-byte words");

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

// 128-byte columns of 64 values; word c of a row at c ^ (row modulo 8)
template <int DK>
__device__ __forceinline__ uint32_t delta_at(int row, int c) { return row * (DK * 2) + ((c ^ (row & 7)) << 4); }
__device__ __forceinline__ void delta_split(float a, float b, uint32_t& hi, uint32_t& lo) {
    hi = pack_pair<true>(a, b);
    const float2 x = unpack_pair<true>(hi);
    lo = pack_pair<true>(a - x.x, b - x.y);
}
// d += (ahi + alo)(bhi + blo) less alo blo
__device__ __forceinline__ void delta_mma3(float (&d)[4], const uint32_t (&ahi)[4], const uint32_t (&alo)[4], uint32_t bh0, uint32_t bh1, uint32_t bl0, uint32_t bl1) {
    mma_16816<true>(d, ahi, bh0, bh1);
    mma_16816<true>(d, alo, bh0, bh1);
    mma_16816<true>(d, ahi, bl0, bl1);
}
__device__ __forceinline__ bool delta_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// A tile of 64 tokens x DK columns into shared memory; what lies behind the chunk or the row reads as zero.
template <int DK, int THREADS>
__device__ __forceinline__ void delta_fetch(uint32_t dst, const uint16_t* src, long long tok, int n, int words, const void* any) {
    for (int i = threadIdx.x; i < DELTA_C * (DK / 8); i += THREADS) {
        const int row = i / (DK / 8), c = i - row * (DK / 8);
        const bool on = row < n && c < words;
        cp_async_16_or_zero(dst + delta_at<DK>(row, c), on ? static_cast<const void*>(src + row * tok + c * 8) : any, on);
    }
}

constexpr int DELTA_PREP_THREADS = 128;
constexpr int DELTA_PITCH = 144;                             // bytes of a row of 64 bfloat16: nine words of 16, so that 8 rows' meet all banks

template <int DK>
struct DeltaPrepCfg {
    static constexpr int kTile = DELTA_C * DK * 2;
    static constexpr int kMat = DELTA_C * DELTA_PITCH;
    static constexpr int kDiag = 4 * 16 * 17 * 4;
    static constexpr int kLoads = 2 * kTile, kWork = 4 * kMat + kDiag;
    static constexpr int kSmemBytes = kLoads + kWork;
};

// T and A of one chunk, for the value heads of one key head.
template <int DK>
__global__ void __launch_bounds__(DELTA_PREP_THREADS) delta_prep_kernel(const DeltaParams p) {
    using C = DeltaPrepCfg<DK>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ double s_g[DELTA_C];
    __shared__ float s_beta[DELTA_C];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    griddep_launch_dependents();
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
    const int first = tok + static_cast<int>(nth) * DELTA_C, n = min(DELTA_C, len - static_cast<int>(nth) * DELTA_C);

    const uint32_t sm = smem_u32(smem), sm_k = sm, sm_q = sm + C::kTile;
    delta_fetch<DK, DELTA_PREP_THREADS>(sm_k, p.k + first * p.k_tok + hk * p.k_head, p.k_tok, n, p.dk / 8, p.offsets);
    delta_fetch<DK, DELTA_PREP_THREADS>(sm_q, p.q + first * p.q_tok + hk * p.q_head, p.q_tok, n, p.dk / 8, p.offsets);
    cp_async_commit();
    cp_async_wait<0>();
    __syncthreads();

    // ---- K K^T and Q K^T: a warp's 16 rows, columns up to the diagonal's ---------------------------------------------------------
    float kk[8][4], qk[8][4];
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) kk[j][e] = qk[j][e] = 0.f;
#pragma unroll
    for (int d = 0; d < DK / 16; ++d) {
        uint32_t ak[4], aq[4];
        const int arow = warp * 16 + (lane & 15);
        ldsm_x4(ak, sm_k + delta_at<DK>(arow, 2 * d + (lane >> 4)));
        ldsm_x4(aq, sm_q + delta_at<DK>(arow, 2 * d + (lane >> 4)));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j > warp) break;
            uint32_t b[4];
            ldsm_x4(b, sm_k + delta_at<DK>(j * 16 + (lane & 7) + ((lane >> 4) << 3), 2 * d + ((lane >> 3) & 1)));
            mma_16816<true>(kk[2 * j], ak, b[0], b[1]);
            mma_16816<true>(kk[2 * j + 1], ak, b[2], b[3]);
            mma_16816<true>(qk[2 * j], aq, b[0], b[1]);
            mma_16816<true>(qk[2 * j + 1], aq, b[2], b[3]);
        }
    }

    uint8_t* l_mat = smem + C::kLoads;                       // L, then T: high parts, low parts, [i][j]
    uint8_t* t_mat = l_mat + 2 * C::kMat;
    float* diag = reinterpret_cast<float*>(t_mat + 2 * C::kMat);
    const uint32_t sm_l = smem_u32(l_mat), sm_t = smem_u32(t_mat);

    for (int rep = 0; rep < p.group; ++rep) {
        const int h = hk * p.group + rep;
        DeltaChunk* to = reinterpret_cast<DeltaChunk*>(p.chunks) + (slot - p.first_slot) * p.heads + h;
        bool fine = true;
        __syncthreads();                                     // (the last head's numbers have been used)
        if (warp == 0) {                                     // G, in 64 bits: its differences count.  exp(-200) is 0, whatever is in front of it
            double x[2];
            float b[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int i = 2 * lane + e;
                float gi = 0.f;
                b[e] = 0.f;
                if (i < n) {
                    gi = p.decay[(first + i) * p.decay_tok + h];
                    b[e] = p.beta[(first + i) * p.beta_tok + h];
                }
                fine &= delta_finite(b[e]) && gi < INFINITY;
                x[e] = gi < -200.f ? -200.0 : static_cast<double>(gi);
                s_beta[i] = b[e];
            }
            double sum = x[0] + x[1];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double y = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += y;
            }
            const double last = __shfl_sync(0xffffffffu, sum, 31);
            s_g[2 * lane] = sum - x[1];
            s_g[2 * lane + 1] = sum;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const double at = e ? sum : sum - x[1];
                to->beta[2 * lane + e] = b[e];
                to->past[2 * lane + e] = expf(static_cast<float>(at));
                to->left[2 * lane + e] = expf(static_cast<float>(last - at));
            }
            if (lane == 0) {
                const double w = exp(last);
                to->whole_hi = static_cast<float>(w);
                to->whole_lo = static_cast<float>(w - static_cast<double>(static_cast<float>(w)));
            }
        }
        __syncthreads();
        // ---- L into shared memory, A as the second kernel's operand -----------------------------------------------------------------
        const double gr[2] = {s_g[warp * 16 + g], s_g[warp * 16 + g + 8]};
        const float br[2] = {s_beta[warp * 16 + g], s_beta[warp * 16 + g + 8]};
#pragma unroll
        for (int t = 0; t < 4; ++t) {                        // blocks of 16 columns
            if (t > warp) break;
            uint32_t ahi[4], alo[4];
#pragma unroll
            for (int half = 0; half < 2; ++half) {           // 8 columns
                const int j0 = t * 16 + half * 8 + 2 * c;
                const double gc[2] = {s_g[j0], s_g[j0 + 1]};
                float l[4], a[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = warp * 16 + g + 8 * (e >> 1), j = j0 + (e & 1);
                    const float d = j <= i ? expf(static_cast<float>(gr[e >> 1] - gc[e & 1])) : 0.f;
                    a[e] = j <= i ? d * qk[2 * t + half][e] : 0.f;
                    l[e] = j < i ? br[e >> 1] * d * kk[2 * t + half][e] : 0.f;
                    fine &= delta_finite(a[e]) && delta_finite(l[e]) && (j != i || delta_finite(kk[2 * t + half][e]));
                    if (t == warp) diag[warp * 16 * 17 + (g + 8 * (e >> 1)) * 17 + half * 8 + 2 * c + (e & 1)] = l[e];
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {                // rows g, g + 8
                    uint32_t hi, lo;
                    delta_split(l[2 * e], l[2 * e + 1], hi, lo);
                    uint8_t* at = l_mat + (warp * 16 + g + 8 * e) * DELTA_PITCH + j0 * 2;
                    *reinterpret_cast<uint32_t*>(at) = hi;
                    *reinterpret_cast<uint32_t*>(at + C::kMat) = lo;
                    delta_split(a[2 * e], a[2 * e + 1], ahi[2 * half + e], alo[2 * half + e]);
                }
            }
            to->a[0][delta_tile(warp, t)][lane] = make_uint4(ahi[0], ahi[1], ahi[2], ahi[3]);
            to->a[1][delta_tile(warp, t)][lane] = make_uint4(alo[0], alo[1], alo[2], alo[3]);
        }
        __syncwarp();
        // ---- T's diagonal blocks, by substitution: lane j has column j ----------------------------------------------------------------
        {
            const float* l = diag + warp * 16 * 17;
            const int j = lane & 15;
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float y = i == j ? 1.f : 0.f;
#pragma unroll
                for (int k = 0; k < i; ++k) y = fmaf(-l[i * 17 + k], x[k], y);
                x[i] = y;
                const __nv_bfloat16 hi = __float2bfloat16_rn(y);
                uint8_t* at = t_mat + (warp * 16 + i) * DELTA_PITCH + (warp * 16 + j) * 2;
                if (lane < 16) *reinterpret_cast<__nv_bfloat16*>(at) = hi;
                else *reinterpret_cast<__nv_bfloat16*>(at + C::kMat) = __float2bfloat16_rn(y - __bfloat162float(hi));
            }
        }
        __syncthreads();
        // ---- the blocks under them: warp J has block column J, transposed:  T_IJ^T = -(sum_K T_KJ^T L_IK^T) T_II^T,  K = J .. I - 1 ----------
        {
            const int trow = ((lane >> 4) << 3) + (lane & 7), tcol = (lane >> 3) & 1;       // operand by rows of k (transposed load)
            const int nrow = (lane & 7) + ((lane >> 4) << 3), ncol = (lane >> 3) & 1;
            uint32_t xh[4][4], xl[4][4];                     // T_KJ^T, K = J + index
            {
                const uint32_t at = sm_t + (warp * 16 + trow) * DELTA_PITCH + warp * 32 + tcol * 16;
                ldsm_x4_t(xh[0], at);
                ldsm_x4_t(xl[0], at + C::kMat);
            }
#pragma unroll
            for (int s = 1; s < 4; ++s) {                    // I = J + s
                if (warp + s > 3) break;
                const int I = warp + s;
                float y[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}, z[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                for (int k = 0; k < s; ++k) {
                    uint32_t bh[4], bl[4];
                    const uint32_t at = sm_l + (I * 16 + nrow) * DELTA_PITCH + (warp + k) * 32 + ncol * 16;
                    ldsm_x4(bh, at);
                    ldsm_x4(bl, at + C::kMat);
                    delta_mma3(y[0], xh[k], xl[k], bh[0], bh[1], bl[0], bl[1]);
                    delta_mma3(y[1], xh[k], xl[k], bh[2], bh[3], bl[2], bl[3]);
                }
                uint32_t yh[4], yl[4], bh[4], bl[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) delta_split(-y[e >> 1][2 * (e & 1)], -y[e >> 1][2 * (e & 1) + 1], yh[e], yl[e]);
                const uint32_t at = sm_t + (I * 16 + nrow) * DELTA_PITCH + I * 32 + ncol * 16;
                ldsm_x4(bh, at);
                ldsm_x4(bl, at + C::kMat);
                delta_mma3(z[0], yh, yl, bh[0], bh[1], bl[0], bl[1]);
                delta_mma3(z[1], yh, yl, bh[2], bh[3], bl[2], bl[3]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {                // rows j = g + 8 (e & 1), columns i = 8 (e >> 1) + 2 c, + 1
                    delta_split(z[e >> 1][2 * (e & 1)], z[e >> 1][2 * (e & 1) + 1], xh[s][e], xl[s][e]);
                    uint8_t* to_t = t_mat + (I * 16 + 8 * (e >> 1) + 2 * c) * DELTA_PITCH + (warp * 16 + g + 8 * (e & 1)) * 2;
                    *reinterpret_cast<uint16_t*>(to_t) = static_cast<uint16_t>(xh[s][e]);
                    *reinterpret_cast<uint16_t*>(to_t + DELTA_PITCH) = static_cast<uint16_t>(xh[s][e] >> 16);
                    *reinterpret_cast<uint16_t*>(to_t + C::kMat) = static_cast<uint16_t>(xl[s][e]);
                    *reinterpret_cast<uint16_t*>(to_t + C::kMat + DELTA_PITCH) = static_cast<uint16_t>(xl[s][e] >> 16);
                }
            }
        }
        __syncthreads();
        for (int x = warp; x < 2 * DELTA_TILES; x += DELTA_PREP_THREADS / 32) {
            const int part = x / DELTA_TILES, tile = x - part * DELTA_TILES;
            const int i = tile >= 6 ? 3 : tile >= 3 ? 2 : tile >= 1 ? 1 : 0, j = tile - delta_tile(i, 0);
            uint32_t r[4];
            ldsm_x4(r, sm_t + part * C::kMat + (i * 16 + (lane & 15)) * DELTA_PITCH + j * 32 + (lane >> 4) * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) fine &= (r[e] & 0x7f80u) != 0x7f80u && (r[e] & 0x7f800000u) != 0x7f800000u;
            to->t[part][tile][lane] = make_uint4(r[0], r[1], r[2], r[3]);
        }
        const bool wild = __syncthreads_or(!fine);
        if (tid == 0) to->wild = wild ? 1 : 0;
    }
}

// ---------------------------------------------------------------------------------------------------------------------
constexpr int DELTA_THREADS = 256;

template <int DK, int NV>
struct DeltaCfg {
    static constexpr int kTile = DELTA_C * DK * 2;
    static constexpr int kPitch = NV * 2 + 16;               // bytes of a row of NV bfloat16: an odd number of 16-byte words
    static constexpr int kK = 0, kQ = kTile, kV = 2 * kTile, kChunk = kV + DELTA_C * kPitch;
    static constexpr int kStage = kChunk + static_cast<int>(sizeof(DeltaChunk));
    static constexpr int kStages = 2;
    static constexpr int kS = kStages * kStage, kSPart = DK * kPitch;            // the state, high parts and low parts
    static constexpr int kR = kS + 2 * kSPart, kRPart = DELTA_C * kPitch;
    static constexpr int kU = kR + 2 * kRPart;                                   // U, then exp(G_n - G) U
    static constexpr int kSum = kU + 4 * kRPart;                                 // token by token: a row of sums per warp
    static constexpr int kSmemBytes = kSum + 8 * NV * 4;
};

template <int DK, int NV>
__global__ void __launch_bounds__(DELTA_THREADS, 1) delta_chunks_kernel(const DeltaParams p) {
    using C = DeltaCfg<DK, NV>;
    constexpr int N = NV / 8;                                // products' column tiles
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const int slice = static_cast<int>(blockIdx.x % p.slices), h = static_cast<int>(blockIdx.x / p.slices % p.heads);
    const int seq = static_cast<int>(blockIdx.x / p.slices / p.heads), hk = h / p.group, col0 = slice * NV;
    int tok, len;
    const bool good = lin_sequence(p.offsets, p.ntok, seq, tok, len);
    const int chunks = (len + DELTA_C - 1) / DELTA_C;
    const long long slot0 = delta_slot(tok, seq);
    // the chunks that this launch has the operands of
    const int begin = static_cast<int>(max(0ll, min(static_cast<long long>(chunks), p.first_slot - slot0)));
    const int end = static_cast<int>(max(0ll, min(static_cast<long long>(chunks), p.last_slot - slot0)));
    griddep_wait();
    if (!good && slice == 0 && h == 0 && tid == 0) p.hdr->error = 4u;            // MMV_ERR_BAD_SEGMENTS
    if (begin >= end && !(chunks == 0 && p.first_slot == 0)) return;

    const uint32_t sm = smem_u32(smem);
    const auto fetch = [&](int chunk) {
        const uint32_t dst = sm + (chunk & 1) * C::kStage;
        const long long first = tok + static_cast<long long>(chunk) * DELTA_C;
        const int n = min(DELTA_C, len - chunk * DELTA_C);
        delta_fetch<DK, DELTA_THREADS>(dst + C::kK, p.k + first * p.k_tok + hk * p.k_head, p.k_tok, n, p.dk / 8, p.offsets);
        delta_fetch<DK, DELTA_THREADS>(dst + C::kQ, p.q + first * p.q_tok + hk * p.q_head, p.q_tok, n, p.dk / 8, p.offsets);
        const uint16_t* v = p.v + first * p.v_tok + h * p.v_head + col0;
        for (int i = tid; i < DELTA_C * N; i += DELTA_THREADS) {
            const int row = i / N, w = i - row * N;
            const bool on = row < n && col0 + w * 8 < p.dv;
            cp_async_16_or_zero(dst + C::kV + row * C::kPitch + w * 16, on ? static_cast<const void*>(v + row * p.v_tok + w * 8) : p.offsets, on);
        }
        const uint8_t* src = p.chunks + ((slot0 + chunk - p.first_slot) * p.heads + h) * sizeof(DeltaChunk);
        for (int i = tid; i < static_cast<int>(sizeof(DeltaChunk) / 16); i += DELTA_THREADS) cp_async_16_or_zero(dst + C::kChunk + i * 16, src + i * 16, true);
    };
    if (begin < end) fetch(begin);
    cp_async_commit();

    // ---- the state: rows 16 warp + g and + 8, columns 8 j + 2 c and + 1 of the slice ------------------------------------------------
    float s[N][4];
    const bool keeps = warp * 16 < DK;
    const float* from = begin > 0 ? p.state_out : p.state;
    const long long base = (static_cast<long long>(seq) * p.heads + h) * p.dk * p.dv;
    const auto state_at = [&](int j, int e) { return base + static_cast<long long>(warp * 16 + g + 8 * e) * p.dv + col0 + j * 8 + 2 * c; };
    const auto held = [&](int j, int e) { return keeps && warp * 16 + g + 8 * e < p.dk && col0 + j * 8 < p.dv; };
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float2 x = make_float2(0.f, 0.f);
            if (from && held(j, e)) x = *reinterpret_cast<const float2*>(from + state_at(j, e));
            s[j][2 * e] = x.x;
            s[j][2 * e + 1] = x.y;
        }

    const int block = warp & 3;                              // this warp's 16 tokens; warps 0 to 3 form K S, the others Q S and the results
    const bool queries = warp >= 4;
    const int brow = lane & 15, bcol = lane >> 4;            // second operands: 16 rows, 16 columns
    for (int chunk = begin; chunk < end; ++chunk) {
        const uint32_t st = sm + (chunk & 1) * C::kStage;
        const DeltaChunk* info = reinterpret_cast<const DeltaChunk*>(smem + (chunk & 1) * C::kStage + C::kChunk);
        const int n = min(DELTA_C, len - chunk * DELTA_C);
        // the state's copy for the products
        if (keeps) {
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    uint32_t hi, lo;
                    delta_split(s[j][2 * e], s[j][2 * e + 1], hi, lo);
                    const uint32_t at = C::kS + (warp * 16 + g + 8 * e) * C::kPitch + (j * 8 + 2 * c) * 2;
                    *reinterpret_cast<uint32_t*>(smem + at) = hi;
                    *reinterpret_cast<uint32_t*>(smem + at + C::kSPart) = lo;
                }
        }
        cp_async_wait<0>();
        __syncthreads();                                     // this chunk's operands and the state's copy are there
        if (chunk + 1 < end) fetch(chunk + 1);
        cp_async_commit();

        // ---- K S, Q S ----------------------------------------------------------------------------------------------------------------
        float x[N][4];
#pragma unroll
        for (int j = 0; j < N; ++j) x[j][0] = x[j][1] = x[j][2] = x[j][3] = 0.f;
#pragma unroll
        for (int d = 0; d < DK / 16; ++d) {
            uint32_t a[4];
            ldsm_x4(a, st + (queries ? C::kQ : C::kK) + delta_at<DK>(block * 16 + (lane & 15), 2 * d + (lane >> 4)));
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                uint32_t hi[4], lo[4];
                const uint32_t at = sm + C::kS + (d * 16 + brow) * C::kPitch + (j / 2) * 32 + bcol * 16;
                ldsm_x4_t(hi, at);
                ldsm_x4_t(lo, at + C::kSPart);
                mma_16816<true>(x[j], a, hi[0], hi[1]);
                mma_16816<true>(x[j + 1], a, hi[2], hi[3]);
                mma_16816<true>(x[j], a, lo[0], lo[1]);
                mma_16816<true>(x[j + 1], a, lo[2], lo[3]);
            }
        }
        const float past[2] = {info->past[block * 16 + g], info->past[block * 16 + g + 8]};
        bool wild = info->wild != 0;
        if (!queries) {                                      // R = b (V - exp(G) K S)
            const float beta[2] = {info->beta[block * 16 + g], info->beta[block * 16 + g + 8]};
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = block * 16 + g + 8 * e;
                    const uint32_t vv = *reinterpret_cast<const uint32_t*>(smem + (chunk & 1) * C::kStage + C::kV + row * C::kPitch + (j * 8 + 2 * c) * 2);
                    wild |= (vv & 0x7f80u) == 0x7f80u || (vv & 0x7f800000u) == 0x7f800000u;
                    const float2 v = unpack_pair<true>(vv);
                    uint32_t hi, lo;
                    delta_split(beta[e] * (v.x - past[e] * x[j][2 * e]), beta[e] * (v.y - past[e] * x[j][2 * e + 1]), hi, lo);
                    const uint32_t at = C::kR + row * C::kPitch + (j * 8 + 2 * c) * 2;
                    *reinterpret_cast<uint32_t*>(smem + at) = hi;
                    *reinterpret_cast<uint32_t*>(smem + at + C::kRPart) = lo;
                }
        }
        wild = __syncthreads_or(wild);
        uint16_t* out = p.out + ((static_cast<long long>(tok) + chunk * DELTA_C) * p.heads + h) * p.dv + col0;
        const long long orow = static_cast<long long>(p.heads) * p.dv;
        if (!wild) {
            // ---- U = T R: 16 tokens, half of the columns ------------------------------------------------------------------------------
            {
                constexpr int H = N / 2;
                const int j0 = queries ? H : 0;
                float u[H][4], y[H][4];
#pragma unroll
                for (int j = 0; j < H; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) u[j][e] = y[j][e] = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (k > block) break;
                    const uint4 th = info->t[0][delta_tile(block, 0) + k][lane], tl = info->t[1][delta_tile(block, 0) + k][lane];
                    const uint32_t ah[4] = {th.x, th.y, th.z, th.w}, al[4] = {tl.x, tl.y, tl.z, tl.w};
#pragma unroll
                    for (int j = 0; j < H; j += 2) {
                        uint32_t hi[4], lo[4];
                        // (an odd number of tiles, NV = 16: the loads' other 8 columns are not used)
                        const uint32_t at = sm + C::kR + (k * 16 + brow) * C::kPitch + (H == 1 ? j0 * 16 : (j0 + j) * 16 + bcol * 16);
                        ldsm_x4_t(hi, at);
                        ldsm_x4_t(lo, at + C::kRPart);
                        mma_16816<true>(u[j], ah, hi[0], hi[1]);
                        mma_16816<true>(y[j], al, hi[0], hi[1]);
                        if (H > 1) {
                            mma_16816<true>(u[j + 1 < H ? j + 1 : j], ah, hi[2], hi[3]);
                            mma_16816<true>(y[j + 1 < H ? j + 1 : j], al, hi[2], hi[3]);
                        }
                        mma_16816<true>(y[j], ah, lo[0], lo[1]);
                        if (H > 1) mma_16816<true>(y[j + 1 < H ? j + 1 : j], ah, lo[2], lo[3]);
                    }
                }
                const float left[2] = {info->left[block * 16 + g], info->left[block * 16 + g + 8]};
#pragma unroll
                for (int j = 0; j < H; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float a = u[j][2 * e] + y[j][2 * e], b = u[j][2 * e + 1] + y[j][2 * e + 1];
                        uint32_t hi, lo;
                        uint8_t* at = smem + C::kU + (block * 16 + g + 8 * e) * C::kPitch + ((j0 + j) * 8 + 2 * c) * 2;
                        delta_split(a, b, hi, lo);
                        *reinterpret_cast<uint32_t*>(at) = hi;
                        *reinterpret_cast<uint32_t*>(at + C::kRPart) = lo;
                        delta_split(a * left[e], b * left[e], hi, lo);
                        *reinterpret_cast<uint32_t*>(at + 2 * C::kRPart) = hi;
                        *reinterpret_cast<uint32_t*>(at + 3 * C::kRPart) = lo;
                    }
            }
            __syncthreads();
            // ---- S' = exp(G_n) S + K^T (exp(G_n - G) U) -----------------------------------------------------------------------------------
            if (keeps) {
                const float wh = info->whole_hi, wl = info->whole_lo;
#pragma unroll
                for (int j = 0; j < N; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[j][e] = fmaf(s[j][e], wh, s[j][e] * wl);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t a[4];
                    ldsm_x4_t(a, st + C::kK + delta_at<DK>(k * 16 + ((lane >> 4) << 3) + (lane & 7), warp * 2 + ((lane >> 3) & 1)));
#pragma unroll
                    for (int j = 0; j < N; j += 2) {
                        uint32_t hi[4], lo[4];
                        const uint32_t at = sm + C::kU + 2 * C::kRPart + (k * 16 + brow) * C::kPitch + (j / 2) * 32 + bcol * 16;
                        ldsm_x4_t(hi, at);
                        ldsm_x4_t(lo, at + C::kRPart);
                        mma_16816<true>(s[j], a, hi[0], hi[1]);
                        mma_16816<true>(s[j + 1], a, hi[2], hi[3]);
                        mma_16816<true>(s[j], a, lo[0], lo[1]);
                        mma_16816<true>(s[j + 1], a, lo[2], lo[3]);
                    }
                }
            }
            // ---- O = scale (exp(G) Q S + A U) ---------------------------------------------------------------------------------------------
            if (queries) {
#pragma unroll
                for (int j = 0; j < N; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[j][e] *= past[e >> 1];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (k > block) break;
                    const uint4 th = info->a[0][delta_tile(block, 0) + k][lane], tl = info->a[1][delta_tile(block, 0) + k][lane];
                    const uint32_t ah[4] = {th.x, th.y, th.z, th.w}, al[4] = {tl.x, tl.y, tl.z, tl.w};
#pragma unroll
                    for (int j = 0; j < N; j += 2) {
                        uint32_t hi[4], lo[4];
                        const uint32_t at = sm + C::kU + (k * 16 + brow) * C::kPitch + (j / 2) * 32 + bcol * 16;
                        ldsm_x4_t(hi, at);
                        ldsm_x4_t(lo, at + C::kRPart);
                        delta_mma3(x[j], ah, al, hi[0], hi[1], lo[0], lo[1]);
                        delta_mma3(x[j + 1], ah, al, hi[2], hi[3], lo[2], lo[3]);
                    }
                }
#pragma unroll
                for (int j = 0; j < N; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int row = block * 16 + g + 8 * e;
                        if (row < n && col0 + j * 8 < p.dv)
                            *reinterpret_cast<uint32_t*>(out + row * orow + j * 8 + 2 * c) = pack_pair<true>(p.scale * x[j][2 * e], p.scale * x[j][2 * e + 1]);
                    }
            }
        } else {
            // ---- token by token: the recurrence as it stands ------------------------------------------------------------------------------
            float* sums = reinterpret_cast<float*>(smem + C::kSum);
            const auto column_sums = [&](const float (&w)[2], int j, float (&r)[2]) {       // over this warp's rows
                r[0] = w[0] * s[j][0] + w[1] * s[j][2];
                r[1] = w[0] * s[j][1] + w[1] * s[j][3];
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) {
                    r[0] += __shfl_xor_sync(0xffffffffu, r[0], o);
                    r[1] += __shfl_xor_sync(0xffffffffu, r[1], o);
                }
            };
            for (int t = 0; t < n; ++t) {
                const long long at = tok + static_cast<long long>(chunk) * DELTA_C + t;
                const LinDecay d = lin_decay(p.decay[at * p.decay_tok + h], 1);
                const float beta = p.beta[at * p.beta_tok + h];
                float kr[2] = {0.f, 0.f}, qr[2] = {0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = warp * 16 + g + 8 * e;
                    if (keeps && row < p.dk) {
                        kr[e] = lin_load<true>(p.k + at * p.k_tok + hk * p.k_head + row);
                        qr[e] = lin_load<true>(p.q + at * p.q_tok + hk * p.q_head + row);
                    }
                }
#pragma unroll 1
                for (int turn = 0; turn < 2; ++turn) {       // k S, then q S'
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        float r[2];
                        column_sums(turn ? qr : kr, j, r);
                        if (g == 0) {
                            sums[warp * NV + j * 8 + 2 * c] = r[0];
                            sums[warp * NV + j * 8 + 2 * c + 1] = r[1];
                        }
                    }
                    __syncthreads();
                    if (turn) {
                        if (tid < NV && col0 + tid < p.dv) {
                            float y = 0.f;
                            for (int w = 0; w < DELTA_THREADS / 32 && w * 16 < p.dk; ++w) y += sums[w * NV + tid];
                            out[t * orow + tid] = lin_store<true>(p.scale * y);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < N; ++j)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const int col = j * 8 + 2 * c + e;
                                float y = 0.f;
                                for (int w = 0; w < DELTA_THREADS / 32 && w * 16 < p.dk; ++w) y += sums[w * NV + col];
                                const float v = col0 + col < p.dv ? lin_load<true>(p.v + at * p.v_tok + h * p.v_head + col0 + col) : 0.f;
                                const float u = beta * (v - fmaf(y, d.hi, y * d.lo));
#pragma unroll
                                for (int i = 0; i < 2; ++i)
                                    if (warp * 16 + g + 8 * i < p.dk) s[j][2 * i + e] = fmaf(s[j][2 * i + e], d.hi, fmaf(s[j][2 * i + e], d.lo, kr[i] * u));
                            }
                    }
                    __syncthreads();
                }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (held(j, e)) *reinterpret_cast<float2*>(p.state_out + state_at(j, e)) = make_float2(s[j][2 * e], s[j][2 * e + 1]);
}

}  // namespace mmv

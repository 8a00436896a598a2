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

// Packed prompts, token by token: a CTA keeps 32 columns of one (sequence, head)'s state in registers.
constexpr int LIN_TOKENS_THREADS = 128;

template <bool BF16>
__global__ void __launch_bounds__(LIN_TOKENS_THREADS) linear_tokens_kernel(LinParams p) {
    __shared__ float s_q[128], s_k[128], s_o[4][32];
    long long w = blockIdx.x;
    const int part = static_cast<int>(w % p.parts);
    w /= p.parts;
    const int h = static_cast<int>(w % p.heads), hk = h / p.group;
    const long long seq = w / p.heads;
    const int tid = threadIdx.x, lane = tid & 31, grp = tid >> 5;
    const int col = part * 32 + lane;
    const bool mine = col < p.dv;
    const int lo = p.offsets[seq], hi = p.offsets[seq + 1];
    const bool ok = lo >= 0 && hi >= lo && hi <= p.ntok;
    if (!ok && tid == 0) report_error(p.hdr, 4u);
    const LinDecay decay = lin_decay(p.log_decay[h], 1);
    const long long base = (seq * p.heads + h) * static_cast<long long>(p.dk) * p.dv + col;
    float s[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const int d = grp * 32 + i;
        s[i] = p.state && mine && d < p.dk ? p.state[base + static_cast<long long>(d) * p.dv] : 0.f;
    }
    if (ok)
        for (long long t = lo; t < hi; ++t) {
            for (int d = tid; d < 128; d += LIN_TOKENS_THREADS) {
                s_q[d] = d < p.dk ? lin_load<BF16>(p.q + t * p.q_tok + h * p.q_head + d) : 0.f;
                s_k[d] = d < p.dk ? lin_load<BF16>(p.k + t * p.k_tok + hk * p.k_head + d) : 0.f;
            }
            const float v = mine ? lin_load<BF16>(p.v + t * p.v_tok + hk * p.v_head + col) : 0.f;
            __syncthreads();
            float o = 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                s[i] = fmaf(s[i], decay.hi, fmaf(s[i], decay.lo, s_k[grp * 32 + i] * v));
                o = fmaf(s_q[grp * 32 + i], s[i], o);
            }
            s_o[grp][lane] = o;
            __syncthreads();
            if (grp == 0 && mine)
                p.out[(t * p.heads + h) * p.dv + col] = lin_store<BF16>(p.scale * (s_o[0][lane] + s_o[1][lane] + s_o[2][lane] + s_o[3][lane]));
        }
    if (p.state_out && mine)
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const int d = grp * 32 + i;
            if (d < p.dk) p.state_out[base + static_cast<long long>(d) * p.dv] = s[i];
        }
}

}  // namespace mmv

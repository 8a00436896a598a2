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
    const float decay = expf(p.log_decay[h]);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f), o = v;
    if (mine) {
        const uint16_t* pv = p.v + r * p.v_tok + hk * p.v_head + col;
        v = make_float4(lin_load<BF16>(pv), lin_load<BF16>(pv + 1), lin_load<BF16>(pv + 2), lin_load<BF16>(pv + 3));
    }
    __syncthreads();
    for (int d0 = row; d0 < p.dk; d0 += ROWS * LIN_STEP_AHEAD) {
#pragma unroll
        for (int i = 0; i < LIN_STEP_AHEAD; ++i) {
            const int d = d0 + i * ROWS;
            if (mine && d < p.dk) {
                float4 x = s[i];
                const float kd = s_k[d], qd = s_q[d];
                x.x = fmaf(x.x, decay, kd * v.x);
                x.y = fmaf(x.y, decay, kd * v.y);
                x.z = fmaf(x.z, decay, kd * v.z);
                x.w = fmaf(x.w, decay, kd * v.w);
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

}  // namespace mmv

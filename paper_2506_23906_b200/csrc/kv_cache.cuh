// The write of a packed batch's keys and values into a paged cache.
//
// A copy with a scattered target: 4 bytes of traffic per value, no arithmetic.  Bound by HBM for a long
// prompt and by the launch for a decoding step.  A thread moves 16-byte words, two of the keys and the two of the
// values at the same place, all four loads in flight before the first store
// (65536 tokens of 8 heads of 128: 92 us a call, 5.7 TB/s; 255 tokens: 4.1 us, the launch).
#pragma once
#include <cstdint>
#include "common.cuh"

namespace mmv {

constexpr int APPEND_THREADS = 256;
constexpr int APPEND_UNROLL = 2;

struct AppendParams {
    const uint16_t *k, *v;
    uint16_t *ck, *cv;
    const int64_t* slots;
    long long ntok;
    long long k_tok, k_head, v_tok, v_head;                  // element strides of the new rows
    long long c_block, c_tok, c_head;                        // and of the cache
    long long nslots;                                        // num_blocks * block_size
    int block_size, words_per_head, words_per_row;           // 16-byte words
};

__global__ void __launch_bounds__(APPEND_THREADS) kv_append_kernel(AppendParams p) {
    const long long words = p.ntok * p.words_per_row;
    const long long step = static_cast<long long>(gridDim.x) * APPEND_THREADS;
    for (long long i0 = static_cast<long long>(blockIdx.x) * APPEND_THREADS + threadIdx.x; i0 < words; i0 += step * APPEND_UNROLL) {
        uint4 kw[APPEND_UNROLL], vw[APPEND_UNROLL];
        long long dst[APPEND_UNROLL];
#pragma unroll
        for (int u = 0; u < APPEND_UNROLL; ++u) {
            const long long i = i0 + u * step;
            dst[u] = -1;
            if (i < words) {
                const long long t = words <= INT32_MAX ? static_cast<long long>(static_cast<uint32_t>(i) / static_cast<uint32_t>(p.words_per_row))
                                                       : i / p.words_per_row;
                const int x = static_cast<int>(i - t * p.words_per_row);
                const int h = x / p.words_per_head, c = (x - h * p.words_per_head) * 8;
                const long long slot = p.slots[t];
                if (slot >= 0 && slot < p.nslots) {
                    const long long b = p.nslots <= INT32_MAX
                                            ? static_cast<long long>(static_cast<uint32_t>(slot) / static_cast<uint32_t>(p.block_size))
                                            : slot / p.block_size;
                    dst[u] = b * p.c_block + (slot - b * p.block_size) * p.c_tok + h * p.c_head + c;
                    kw[u] = *reinterpret_cast<const uint4*>(p.k + t * p.k_tok + h * p.k_head + c);
                    vw[u] = *reinterpret_cast<const uint4*>(p.v + t * p.v_tok + h * p.v_head + c);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < APPEND_UNROLL; ++u) {
            if (dst[u] >= 0) {
                *reinterpret_cast<uint4*>(p.ck + dst[u]) = kw[u];
                *reinterpret_cast<uint4*>(p.cv + dst[u]) = vw[u];
            }
        }
    }
}

}  // namespace mmv

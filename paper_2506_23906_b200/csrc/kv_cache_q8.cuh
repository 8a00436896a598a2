// A paged key-value cache in 8 bits with a scale for each block of tokens and head: the quantising write and the read in 16 bits.
//
// A code stands for code * scale.  With top = 127 (int8) or 448 (e4m3) and amax the largest magnitude of a (block, head):
//     int8   scale = amax / top rounded up to 11 significant bits;  code = x / scale to the nearest whole number, halves away from zero
//     e4m3   scale = the smallest power of two >= amax / top;       code = x / scale to the nearest e4m3 value, halves to even
// Both are reproducible bit by bit from products alone.  e4m3: x / scale is exact.  int8: x and scale have at most 11 significant bits, so that
// x / scale = X / S (integers) differs from n + 1/2 = N / 2 by |2X - NS| / 2S, which is 0 or at least 2^-19 of it (2X < 2^12 or, for a
// held code being converted, 2 code S < 2^19).  x times the rounded reciprocal times 1 + 2^-21 is off by 2^-21 +- 2^-23: every half goes
// away from zero and nothing else changes its side.  The product is rounded once, by the fused sum that puts it in a float's low bits.
// A block that is continued may have any scale >= 0, of another program's making: there a quotient can lie 2^-32 of itself beside a half, and is
// rounded to odd first (q8_pack_any), which keeps it on its side.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include "common.cuh"

namespace mmv {

struct CacheQ8 {
    uint8_t* code[2];                                        // keys, values
    float* scale[2];
    long long block, tok, head;                              // strides of the codes
    long long s_block, s_head;                               // and of the scales
    long long num_blocks;
    int block_size, heads, dim;
};

constexpr float Q8_TINY = 7.888609052210118e-31f;            // 2^-100: magnitudes below it are held as zero (1 / scale stays finite)
constexpr float Q8_MAGIC = 12582912.f;                       // 1.5 * 2^23: a sum's low bits are the addend as an integer

template <bool E4M3>
__device__ __forceinline__ float q8_scale_of(float amax) {
    if (amax < Q8_TINY) return 0.f;
    if constexpr (E4M3) {                                    // amax / 448 = m 2^e with 1 <= m < 2: 2^e if m is 1, else 2^(e + 1)
        const uint32_t b = __float_as_uint(__fdiv_rn(amax, 448.f));
        return __uint_as_float((b + 0x7fffffu) & 0x7f800000u);
    } else {
        const uint32_t b = __float_as_uint(__fdiv_rn(amax, 127.f));
        return __uint_as_float((b + 0x1fffu) & ~0x1fffu);    // (up at the 13th bit from below: 11 bits are left)
    }
}
// what a value is multiplied with in front of q8_code
template <bool E4M3>
__device__ __forceinline__ float q8_inverse(float scale) {
    if (!(scale > 0.f)) return 0.f;
    const float r = __frcp_rn(scale);
    return E4M3 ? r : r * (1.f + 4.76837158203125e-7f);      // 1 + 2^-21
}
// four codes in a word
template <bool E4M3>
__device__ __forceinline__ uint32_t q8_pack(float a, float b, float c, float d, float inv) {
    if constexpr (E4M3) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a * inv, b * inv), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c * inv, d * inv), __NV_SATFINITE, __NV_E4M3);
        return lo | (hi << 16);
    } else {
        const uint32_t ab = __byte_perm(__float_as_uint(fmaf(a, inv, Q8_MAGIC)), __float_as_uint(fmaf(b, inv, Q8_MAGIC)), 0x0040);
        const uint32_t cd = __byte_perm(__float_as_uint(fmaf(c, inv, Q8_MAGIC)), __float_as_uint(fmaf(d, inv, Q8_MAGIC)), 0x0040);
        return __byte_perm(ab, cd, 0x5410);
    }
}
// Whether a scale is finite and > 0 but none that q8_scale_of gives, which the two functions above are for: those lie between 2^-109 and 2^122 (2^-100 / 448, the
// largest bfloat16 / 127) and have no more places than their masks leave.
template <bool E4M3>
__device__ __forceinline__ bool q8_other(float scale) {
    const uint32_t b = __float_as_uint(scale);
    const bool own = (b & (E4M3 ? 0x7fffffu : 0x1fffu)) == 0u && b - 0x09000000u <= 0x73800000u;
    return b - 1u < 0x7f7fffffu && !own;
}
// x, which has been rounded towards zero with the rest r left out, to odd: it stays on its side of every number of fewer bits
__device__ __forceinline__ float q8_odd(float x, float r) { return r != 0.f ? __uint_as_float(__float_as_uint(x) | 1u) : x; }
// Four codes of x * of for any scale > 0: the product to odd (values: of = 1), its quotient by the scale to odd, then to the nearest.
template <bool E4M3>
__device__ __forceinline__ uint32_t q8_pack_any(float4 x, float of, float scale) {
    const float up = scale < 9.313225746154785e-10f ? 7.922816251426434e28f : 1.f;      // below 2^-30 both times 2^96, so that fp32 holds what a rounding leaves
    of *= up;
    scale *= up;
    const float y[4] = {x.x, x.y, x.z, x.w};
    uint32_t out = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float p = __fmul_rz(y[i], of), v = q8_odd(p, fmaf(y[i], of, -p));
        const float d = __fdiv_rz(v, scale), q = q8_odd(d, fmaf(-d, scale, v));
        uint32_t code;
        if constexpr (E4M3) code = __nv_cvt_float_to_fp8(q, __NV_SATFINITE, __NV_E4M3);
        else code = static_cast<uint32_t>(static_cast<int>(copysignf(floorf(__fadd_rz(fabsf(q), 0.5f)), q))) & 0xffu;
        out |= code << (8 * i);
    }
    return out;
}
// the numbers that four codes are (without their scale)
template <bool E4M3>
__device__ __forceinline__ float4 q8_unpack(uint32_t w) {
    if constexpr (E4M3) {
        const float2 a = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w & 0xffffu), __NV_E4M3)));
        const float2 b = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w >> 16), __NV_E4M3)));
        return make_float4(a.x, a.y, b.x, b.y);
    } else {                                                 // 2^23 + 128 + code, less that
        const uint32_t u = w ^ 0x80808080u;
        constexpr float off = 8388608.f + 128.f;
        return make_float4(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440)) - off, __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7441)) - off,
                           __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7442)) - off, __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7443)) - off);
    }
}
template <bool BF16>
__device__ __forceinline__ float2 q8_widen(uint32_t w) {
    if constexpr (BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    else return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <bool BF16>
__device__ __forceinline__ uint32_t q8_narrow(float a, float b) {
    if constexpr (BF16) {
        const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&x);
    } else {
        const __half2 x = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&x);
    }
}

// n / d for n * d < 2^32, by = ceil(2^32 / d); 0 for a divisor of 1
__device__ __forceinline__ int q8_quotient(int n, uint32_t by) { return by ? static_cast<int>(__umulhi(static_cast<uint32_t>(n), by)) : n; }

// 32 bytes in one access where `wide` says that they are aligned so (a lane's two accesses of 16 each leave half of every 32-byte sector to the other)
__device__ __forceinline__ void q8_load(uint4 (&v)[2], const void* p, bool wide) {
    if (wide) {
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(v[0].x), "=r"(v[0].y), "=r"(v[0].z), "=r"(v[0].w), "=r"(v[1].x), "=r"(v[1].y), "=r"(v[1].z), "=r"(v[1].w)
                     : "l"(p));
    } else {
        v[0] = static_cast<const uint4*>(p)[0];
        v[1] = static_cast<const uint4*>(p)[1];
    }
}
__device__ __forceinline__ void q8_store(void* p, const uint32_t (&v)[8], bool wide) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
    } else {
        static_cast<uint4*>(p)[0] = make_uint4(v[0], v[1], v[2], v[3]);
        static_cast<uint4*>(p)[1] = make_uint4(v[4], v[5], v[6], v[7]);
    }
}

// How many of offsets[1 .. n] are <= t: the sequence that token t belongs to (n: none).  32 samples per trip to memory; any values in
// offsets give a result in [0, n].
__device__ __forceinline__ int q8_sequence_of(const int32_t* offsets, int n, int t) {
    const int lane = threadIdx.x & 31;
    int lo = 0, len = n;
    while (len > 0) {
        const int step = (len + 31) >> 5, i = (lane + 1) * step - 1;
        const int c = __popc(__ballot_sync(0xffffffffu, i < len && offsets[lo + i + 1] <= t));
        lo += c * step;
        len = min(step - 1, len - c * step);
    }
    return lo;
}

// ---------------------------------------------------------------------------------------------------------------------
// The write.  3 bytes of traffic per value: bound by HBM for prompts (53000 tokens of 8 heads of 128: 64 us, 5.1 of the 6.5 TB/s of a copy), by the launch and
// a chain of dependent trips (offsets, page, old scale and values, store) for a decoding step (255 tokens: 6.5 us).
//
// Split: a unit is (window of tokens, group of heads, keys or values), taken by a group of threads (a warp where a run is short, else the CTA); it
// takes the RUNS that begin in its window, head by head.  A run is a request's tokens that lie in one block: all that a scale depends on
// besides the old one, so that no unit meets another's and nothing has to be joined.  The run's values are loaded once and stay in
// registers (Q8_KEEP elements of 16 per thread; what is longer is read a second time, from the L2) between the maximum and the codes.
// ---------------------------------------------------------------------------------------------------------------------
constexpr int Q8_THREADS = 128;
constexpr int Q8_KEEP = 4;

struct AppendQ8Params {
    CacheQ8 c;
    const uint16_t* x[2];
    long long x_tok[2], x_head[2];
    const int32_t *offsets, *total, *table;
    long long table_stride, max_blocks;
    int nreq, ntok, window, side;                            // side: heads of a unit
    bool wide;                                               // rows on 32-byte words
    uint32_t by_row;                                         // reciprocal (q8_quotient) of dim / 16
    long long units;
};

// The runs that begin in a unit's window: f(first row, rows, place in the block, page) for each.
template <typename F>
__device__ __forceinline__ void q8_runs(const AppendQ8Params& p, int t0, int t1, F&& f) {
    // the request that token t belongs to: its rows [lo, hi), and what it holds with them (one token of every request: request t)
    int r = t0 < p.nreq ? t0 : 0, lo = p.offsets[r], hi = p.offsets[r + 1], total = p.total[r];
    for (int t = t0; t < t1;) {
        if (t < lo || t >= hi) {
            r = q8_sequence_of(p.offsets, p.nreq, t);
            if (r >= p.nreq) return;
            lo = p.offsets[r];
            hi = p.offsets[r + 1];
            total = p.total[r];
        }
        if (lo < 0 || hi > p.ntok || hi <= t) return;        // (not offsets: nothing is written)
        if (lo > t) {                                        // tokens in front of the first request
            t = lo;
            continue;
        }
        const long long past = static_cast<long long>(total) - (hi - lo), at = past + (t - lo);
        if (past < 0) {
            t = hi;
            continue;
        }
        const int b = static_cast<int>(static_cast<uint32_t>(at) / static_cast<uint32_t>(p.c.block_size)), place = static_cast<int>(at - static_cast<long long>(b) * p.c.block_size);
        const int len = min(p.c.block_size - place, hi - t);
        const int first = t;
        t += len;
        if (place > 0 && first > lo) continue;               // the run began in an earlier window
        if (b >= p.max_blocks) continue;
        const long long page = p.table[r * p.table_stride + b];
        if (page < 0 || page >= p.c.num_blocks) continue;
        f(first, len, place, page);
    }
}

// The runs of a unit that go on in blocks whose scale no write has made, which the kernel leaves out.  (It comes last and out of line: inside the kernel's loop it took
// from a twentieth to a quarter of the time that the others need.)
template <bool BF16, bool E4M3, bool WARP>
static __device__ __noinline__ void kv_append_q8_any(const AppendQ8Params& p, int kv, int head0, int head1, int t0, int t1, uint32_t* s_max) {
    constexpr int G = WARP ? 32 : Q8_THREADS;
    constexpr float top = E4M3 ? 448.f : 127.f;
    const int me = threadIdx.x % G, per = p.c.dim / 16;
    q8_runs(p, t0, t1, [&](int first, int len, int place, long long page) {
        if (place == 0) return;
        for (int head = head0; head < head1; ++head) {
            float* scale = p.c.scale[kv] + page * p.c.s_block + head * p.c.s_head;
            const float old = *scale;
            if (!q8_other<E4M3>(old)) continue;
            const uint16_t* x = p.x[kv] + first * p.x_tok[kv] + head * p.x_head[kv];
            uint8_t* dst = p.c.code[kv] + page * p.c.block + head * p.c.head;
            uint32_t most = 0u;
            for (int i = me; i < len * per; i += G) {
                const uint32_t* in = reinterpret_cast<const uint32_t*>(x + i / per * p.x_tok[kv] + i % per * 16);
                for (int j = 0; j < 8; ++j) most = __vmaxu2(most, in[j] & 0x7fff7fffu);
            }
            most = __reduce_max_sync(0xffffffffu, max(most & 0xffffu, most >> 16));
            if constexpr (WARP) {
                __syncwarp();                                // (every lane has read the old scale)
            } else {
                if ((threadIdx.x & 31) == 0) s_max[threadIdx.x / 32] = most;
                __syncthreads();
                for (int i = 0; i < Q8_THREADS / 32; ++i) most = max(most, s_max[i]);
                __syncthreads();
            }
            const bool wild = most >= (BF16 ? 0x7f80u : 0x7c00u);
            const float amax = q8_widen<BF16>(most).x;
            const float now = wild ? __uint_as_float(0x7fc00000u) : amax <= __fmul_rd(old, top) ? old : q8_scale_of<E4M3>(amax);
            if (now > old)
                for (int i = me; i < place * per; i += G) {
                    uint32_t* word = reinterpret_cast<uint32_t*>(dst + i / per * p.c.tok + i % per * 16);
                    for (int j = 0; j < 4; ++j) word[j] = q8_pack_any<E4M3>(q8_unpack<E4M3>(word[j]), old, now);
                }
            for (int i = me; i < len * per; i += G) {
                const uint32_t* in = reinterpret_cast<const uint32_t*>(x + i / per * p.x_tok[kv] + i % per * 16);
                uint32_t* word = reinterpret_cast<uint32_t*>(dst + (place + i / per) * p.c.tok + i % per * 16);
                for (int j = 0; j < 4; ++j) {
                    const float2 a = q8_widen<BF16>(in[2 * j]), b = q8_widen<BF16>(in[2 * j + 1]);
                    word[j] = now > 0.f ? q8_pack_any<E4M3>(make_float4(a.x, a.y, b.x, b.y), 1.f, now) : 0u;
                }
            }
            if (me == 0) *scale = now;
        }
    });
}

template <bool BF16, bool E4M3, bool WARP>
__global__ void __launch_bounds__(Q8_THREADS, 6) kv_append_q8_kernel(const __grid_constant__ AppendQ8Params p) {
    constexpr int G = WARP ? 32 : Q8_THREADS;
    constexpr float top = E4M3 ? 448.f : 127.f;
    __shared__ uint32_t s_max[2][Q8_THREADS / 32];
    const int me = threadIdx.x % G, per = p.c.dim / 16;      // elements of 16 values per row
    const long long unit = static_cast<long long>(blockIdx.x) * (Q8_THREADS / G) + threadIdx.x / G;
    if (unit >= p.units) return;
    const int groups = (p.c.heads + p.side - 1) / p.side;
    const int head0 = static_cast<int>(unit % groups) * p.side, head1 = min(p.c.heads, head0 + p.side), kv = static_cast<int>(unit / groups % 2);
    const int t0 = static_cast<int>(unit / (2 * groups)) * p.window, t1 = t0 + min(p.window, p.ntok - t0);  // (t0 + window may pass 2^31)
    int turn = 0;
    bool others = false;                                     // blocks of other scales were left out
    q8_runs(p, t0, t1, [&](int first, int len, int place, long long page) {
        const int n = len * per;
        uint4 w[Q8_KEEP][2];
        float old;                                           // the old scale
        // this thread's elements: offsets in the values and in the block
        long long src[Q8_KEEP], to[Q8_KEEP];
#pragma unroll
        for (int i = 0; i < Q8_KEEP; ++i) {
            const int row = q8_quotient(me + i * G, p.by_row), col = me + i * G - row * per;
            src[i] = (first + row) * p.x_tok[kv] + col * 16;
            to[i] = (place + row) * p.c.tok + col * 16;
        }
        const auto fetch = [&](int i, int head, uint4 (&v)[2]) {                 // (elements past those)
            const int row = i / per, col = i - row * per;
            q8_load(v, p.x[kv] + (first + row) * p.x_tok[kv] + head * p.x_head[kv] + col * 16, p.wide);
        };
        const auto load = [&](int head) {
            old = place > 0 ? p.c.scale[kv][page * p.c.s_block + head * p.c.s_head] : 0.f;
#pragma unroll
            for (int i = 0; i < Q8_KEEP; ++i)
                if (me + i * G < n) q8_load(w[i], p.x[kv] + head * p.x_head[kv] + src[i], p.wide);
        };
        const auto process = [&](int head) {
            // the run's largest magnitude (as bits: a NaN is above infinity)
            uint32_t most = 0u;
            const auto widest = [&](const uint4 (&v)[2]) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    most = __vmaxu2(most, v[j].x & 0x7fff7fffu);
                    most = __vmaxu2(most, v[j].y & 0x7fff7fffu);
                    most = __vmaxu2(most, v[j].z & 0x7fff7fffu);
                    most = __vmaxu2(most, v[j].w & 0x7fff7fffu);
                }
            };
#pragma unroll
            for (int i = 0; i < Q8_KEEP; ++i)
                if (me + i * G < n) widest(w[i]);
            for (int i = me + Q8_KEEP * G; i < n; i += G) {
                uint4 v[2];
                fetch(i, head, v);
                widest(v);
            }
            most = __reduce_max_sync(0xffffffffu, max(most & 0xffffu, most >> 16));
            if constexpr (!WARP) {
                if ((threadIdx.x & 31) == 0) s_max[turn][threadIdx.x / 32] = most;
                __syncthreads();
#pragma unroll
                for (int i = 0; i < Q8_THREADS / 32; ++i) most = max(most, s_max[turn][i]);
                turn ^= 1;                                   // (the next maxima go elsewhere: one barrier is enough)
            }
            const bool wild = most >= (BF16 ? 0x7f80u : 0x7c00u) || !(old >= 0.f && old < INFINITY);
            const float amax = q8_widen<BF16>(most).x;
            const float now = wild ? __uint_as_float(0x7fc00000u) : amax <= old * top ? old : q8_scale_of<E4M3>(amax);
            const float inv = q8_inverse<E4M3>(now);         // (0 for a scale that is 0 or NaN: the codes are 0)
            uint8_t* dst = p.c.code[kv] + page * p.c.block + head * p.c.head;
            if (place > 0 && now > old) {                    // the scale grows: the codes in front of the run are converted
                for (int i = me; i < place * per; i += G) {
                    const int row = i / per, col = i - row * per;
                    uint4* q = reinterpret_cast<uint4*>(dst + row * p.c.tok + col * 16);
                    uint4 v = *q;
                    uint32_t* word = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float4 y = q8_unpack<E4M3>(word[j]);
                        word[j] = q8_pack<E4M3>(y.x * old, y.y * old, y.z * old, y.w * old, inv);
                    }
                    *q = v;
                }
            }
            const auto store = [&](long long at, const uint4 (&v)[2]) {
                uint32_t out[4];
                const uint32_t in[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 a = q8_widen<BF16>(in[2 * j]), c = q8_widen<BF16>(in[2 * j + 1]);
                    out[j] = wild ? 0u : q8_pack<E4M3>(a.x, a.y, c.x, c.y, inv);
                }
                *reinterpret_cast<uint4*>(dst + at) = make_uint4(out[0], out[1], out[2], out[3]);
            };
#pragma unroll
            for (int i = 0; i < Q8_KEEP; ++i)
                if (me + i * G < n) store(to[i], w[i]);
            for (int i = me + Q8_KEEP * G; i < n; i += G) {
                uint4 v[2];
                fetch(i, head, v);
                store((place + i / per) * p.c.tok + i % per * 16, v);
            }
            if constexpr (WARP) __syncwarp();                // (every lane has read the old scale)
            if (me == 0 && !(now == old && place > 0)) p.c.scale[kv][page * p.c.s_block + head * p.c.s_head] = now;
        };
        for (int head = head0; head < head1; ++head) {
            load(head);
            if (q8_other<E4M3>(old)) others = true;
            else process(head);
        }
    });
    if (others) {
        if constexpr (!WARP) __syncthreads();
        kv_append_q8_any<BF16, E4M3, WARP>(p, kv, head0, head1, t0, t1, s_max[0]);
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// The read: 1 byte in, 2 out per value, HBM (131072 tokens of 8 heads of 128: 127 us, 6.3 of the 6.5 TB/s of a copy).  A warp takes `tile` (up to 32) tokens of the packed result; lane i finds where token i lies,
// then the warp moves the rows' words of 16 values, keys and values side by side.
// ---------------------------------------------------------------------------------------------------------------------
constexpr int READ_Q8_THREADS = 256;
constexpr int READ_Q8_UNROLL = 2;

struct ReadQ8Params {
    CacheQ8 c;
    uint16_t* out[2];                                        // [token, heads, dim]
    const int32_t *offsets, *table;
    long long table_stride, max_blocks;
    int nreq, ntok, tile;
    bool wide;                                               // results on 32-byte words
    int words;                                               // of a token: heads * dim / 16
    uint32_t by_words, by_head;                              // reciprocals (q8_quotient) of words and dim / 16
};

template <bool BF16, bool E4M3>
__global__ void __launch_bounds__(READ_Q8_THREADS) kv_read_q8_kernel(const ReadQ8Params p) {
    const int lane = threadIdx.x & 31;
    const long long warps = static_cast<long long>(gridDim.x) * (READ_Q8_THREADS / 32);
    const long long tiles = (static_cast<long long>(p.ntok) + p.tile - 1) / p.tile;
    for (long long i = static_cast<long long>(blockIdx.x) * (READ_Q8_THREADS / 32) + threadIdx.x / 32; i < tiles; i += warps) {
        const int t0 = static_cast<int>(i * p.tile), held = min(p.tile, p.ntok - t0), t = t0 + lane;
        int r = q8_sequence_of(p.offsets, p.nreq, t0);
        if (r >= p.nreq) return;                             // behind the last sequence
        // where token t lies: -2 behind the sequences or in front of them (not written), -1 without a page (zero)
        long long codes = -2, scales = 0;
        if (lane < held) {
            int hi = p.nreq;                                 // the first sequence from r on that ends behind t
            if (p.offsets[r + 1] > t) hi = r;
            while (r < hi) {
                const int mid = (r + hi) >> 1;
                if (p.offsets[mid + 1] > t) hi = mid;
                else r = mid + 1;
            }
            if (r < p.nreq && p.offsets[r] <= t && p.offsets[r] >= 0) {
                const uint32_t at = static_cast<uint32_t>(t - p.offsets[r]), b = at / static_cast<uint32_t>(p.c.block_size);
                const long long page = b < p.max_blocks ? p.table[r * p.table_stride + b] : -1;
                codes = -1;
                if (page >= 0 && page < p.c.num_blocks) {
                    codes = page * p.c.block + (at - b * static_cast<uint32_t>(p.c.block_size)) * p.c.tok;
                    scales = page * p.c.s_block;
                }
            }
        }
        const int n = held * p.words, per = p.c.dim / 16;
#pragma unroll 1
        for (int j0 = 0; j0 < n; j0 += 32 * READ_Q8_UNROLL) {
            uint4 w[READ_Q8_UNROLL][2];
            float s[READ_Q8_UNROLL][2];
            long long dst[READ_Q8_UNROLL];
#pragma unroll
            for (int u = 0; u < READ_Q8_UNROLL; ++u) {
                const int j = j0 + u * 32 + lane, row = q8_quotient(j, p.by_words);
                const long long at = __shfl_sync(0xffffffffu, codes, row & 31), sc = __shfl_sync(0xffffffffu, scales, row & 31);
                dst[u] = -1;
                if (j < n && at >= -1) {
                    const int c = j - row * p.words, head = q8_quotient(c, p.by_head), col = c - head * per;
                    dst[u] = (static_cast<long long>(t0) * p.words + j) * 16;
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv) {
                        w[u][kv] = make_uint4(0u, 0u, 0u, 0u);
                        s[u][kv] = 0.f;
                        if (at >= 0) {
                            w[u][kv] = *reinterpret_cast<const uint4*>(p.c.code[kv] + at + head * p.c.head + col * 16);
                            s[u][kv] = p.c.scale[kv][sc + head * p.c.s_head];
                        }
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < READ_Q8_UNROLL; ++u) {
                if (dst[u] < 0) continue;
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    const uint32_t in[4] = {w[u][kv].x, w[u][kv].y, w[u][kv].z, w[u][kv].w};
                    uint32_t out[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float4 y = q8_unpack<E4M3>(in[e]);
                        out[2 * e] = q8_narrow<BF16>(y.x * s[u][kv], y.y * s[u][kv]);
                        out[2 * e + 1] = q8_narrow<BF16>(y.z * s[u][kv], y.w * s[u][kv]);
                    }
                    q8_store(p.out[kv] + dst[u], out, p.wide);
                }
            }
        }
    }
}

}  // namespace mmv

// Host side of the operators on a key-value cache in 8 bits of include/mmv.h: argument checks, workspace carve-up and launches.
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/mmv.h"
#include "common.cuh"
#include "host_state.h"
#include "kv_cache_q8.cuh"
#include "paged_attn_q8.cuh"
#include "serve_host.h"

namespace mmv {
namespace {

ServeDevice g_devices[kMaxDevices];

template <bool BF16, bool E4M3, int DP, int ROWS>
bool allow_one() {
    return allow_smem(paged_attention_q8_kernel<BF16, E4M3, DP, ROWS, false>, PagedQ8Cfg<DP, ROWS>::smem_bytes(ROWS)) &&
           allow_smem(paged_attention_q8_kernel<BF16, E4M3, DP, ROWS, true>, PagedQ8Cfg<DP, ROWS>::smem_bytes(ROWS));
}
template <int DP, int ROWS>
bool allow_rows() {
    return allow_one<false, false, DP, ROWS>() && allow_one<false, true, DP, ROWS>() && allow_one<true, false, DP, ROWS>() && allow_one<true, true, DP, ROWS>();
}
template <int DP>
bool allow_paged() {
    return allow_rows<DP, 4>() && allow_rows<DP, 8>() && allow_rows<DP, 16>();
}
ServeDevice* device() {
    return device_once(g_devices, [] { return allow_paged<64>() && allow_paged<128>() && allow_paged<256>(); });
}

mmv_status check_cache(const mmv_kv_cache_q8* c) {
    if (!c || (c->code != MMV_CODE_INT8 && c->code != MMV_CODE_E4M3)) return MMV_ERR_INVALID_ARG;
    if (c->num_blocks < 0 || c->num_blocks > INT32_MAX || c->block_size < 1 || c->heads < 1 || c->heads > kMaxHeads) return MMV_ERR_INVALID_ARG;
    if (c->dim < 16 || c->dim > 256 || c->dim % 16) return MMV_ERR_INVALID_ARG;
    if (c->block_size > INT32_MAX / 16 - Q8_THREADS) return MMV_ERR_INVALID_ARG;             // (words of a block's rows are counted in 32 bits)
    if (!word_stride(c->stride_block, c->num_blocks, 16) || !word_stride(c->stride_token, c->block_size, 16) || !word_stride(c->stride_head, c->heads, 16))
        return MMV_ERR_INVALID_ARG;
    if (c->num_blocks && (!c->k || !c->v || !aligned(c->k, 16) || !aligned(c->v, 16))) return MMV_ERR_INVALID_ARG;
    if (c->num_blocks && (!c->k_scale || !c->v_scale || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))) return MMV_ERR_INVALID_ARG;
    return MMV_OK;
}
bool check_table(const int32_t* table, int64_t stride, int64_t max_blocks, int64_t nreq) {
    return max_blocks >= 0 && !(nreq && max_blocks && (!table || !aligned(table, 4) || (nreq > 1 && stride < max_blocks)));
}
CacheQ8 cache_params(const mmv_kv_cache_q8* c) {
    CacheQ8 p;
    p.code[0] = static_cast<uint8_t*>(c->k);
    p.code[1] = static_cast<uint8_t*>(c->v);
    p.scale[0] = c->k_scale;
    p.scale[1] = c->v_scale;
    p.block = c->stride_block;
    p.tok = c->stride_token;
    p.head = c->stride_head;
    p.s_block = c->scale_stride_block;
    p.s_head = c->scale_stride_head;
    p.num_blocks = c->num_blocks;
    p.block_size = c->block_size;
    p.heads = c->heads;
    p.dim = c->dim;
    return p;
}
uint32_t reciprocal(uint32_t d) { return d == 1 ? 0u : static_cast<uint32_t>(((1ull << 32) + d - 1) / d); }

// Resident CTAs per SM: what the shared memory allows (codes' stages, query rows, rows where the warps meet), and the registers.
template <int DP, int ROWS>
int fit(int rows) {
    using C = PagedQ8Cfg<DP, ROWS>;
    const int shared = 228 * 1024 / (C::smem_bytes(rows) + 3 * 1024);           // (the kernel's other arrays, and 1 KB of every CTA's that is not its own)
    return shared < C::kPerSm ? shared : C::kPerSm;
}
template <int DP>
int fit(int rows) {
    return rows <= 4 ? fit<DP, 4>(rows) : rows <= 8 ? fit<DP, 8>(rows) : fit<DP, 16>(rows);
}
int per_sm(int padded, int rows) { return padded == 64 ? fit<64>(rows) : padded == 128 ? fit<128>(rows) : fit<256>(rows); }

struct Plan {
    size_t desc_off, ml_off, m2_off, o_off, total;
};
// Key heads that a CTA's four warps take beside one another: a token's codes of both are neighbours in memory, and a request's end costs half as many short
// tiles.  1, 2 or 4 of 8 heads (4 queries each, dim 128), 4 requests of 131072: 270, 180, 185 us; 64 of 2048: 66, 62, 64; 4 heads of 16 queries, 64 of 4096:
// 120, 122, 132; dim 256: no difference.  An odd number takes one: 4 of 131072 with 7, 6, 5, 4, 3 heads 237, 158, 179, 118, 97 us, 64 of 4096 with 8, 7, 5, 4, 3 heads
// 119, 105, 106, 70, 67.
int heads_side_by_side(int kv_heads) { return kv_heads % 2 == 0 ? 2 : 1; }
Plan plan_of(const PagedHeads& h, int kv_heads, int dim) {
    const size_t parts = 2 * static_cast<size_t>(heads_side_by_side(kv_heads));       // of a CTA
    const size_t ctas = static_cast<size_t>(kPagedMaxSms) * per_sm(paged_padded(dim), h.rows);
    Plan w;
    w.desc_off = sizeof(WorkspaceHeader);
    w.ml_off = round_up(w.desc_off + ctas * 4 * sizeof(int32_t), 256);
    w.m2_off = round_up(w.ml_off + ctas * parts * 2 * PA_ROWS * sizeof(float), 256);
    w.o_off = round_up(w.m2_off + ctas * parts * PA_ROWS * sizeof(float), 256);
    w.total = round_up(w.o_off + ctas * parts * h.rows * dim * sizeof(float), 256);
    return w;
}

// The cache's codes as boxes of 16 tokens of one head of one block, 128-byte swizzle (64-byte for rows of 64); false where they cannot be described so.
bool code_map(CUtensorMap* map, const void* x, const mmv_kv_cache_q8* c, int padded) {
    EncodeTiledFn enc = get_encode();
    if (!enc) return false;
    const cuuint64_t row = static_cast<cuuint64_t>(c->dim);
    const cuuint64_t dims[4] = {row, static_cast<cuuint64_t>(c->heads), static_cast<cuuint64_t>(c->block_size), static_cast<cuuint64_t>(c->num_blocks)};
    const cuuint64_t strides[3] = {c->heads > 1 ? static_cast<cuuint64_t>(c->stride_head) : row, static_cast<cuuint64_t>(c->stride_token),
                                   c->num_blocks > 1 ? static_cast<cuuint64_t>(c->stride_block) : row};
    const cuuint32_t box[4] = {padded < 128 ? 64u : 128u, 1, 16, 1}, estr[4] = {1, 1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(x), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               padded < 128 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) ==
           CUDA_SUCCESS;
}

struct CodeMaps {
    CUtensorMap k, v;
    bool box;
};
template <bool BF16, bool E4M3, int DP, int ROWS>
mmv_status launch_rows(const CodeMaps& m, const PagedQ8Params& p, int ctas, cudaStream_t st) {
    const size_t smem = static_cast<size_t>(PagedQ8Cfg<DP, ROWS>::smem_bytes(p.rows));
    const dim3 grid(static_cast<unsigned>(ctas));
    const mmv_status rc = m.box ? launch(paged_attention_q8_kernel<BF16, E4M3, DP, ROWS, true>, grid, PA_THREADS, smem, st, false, m.k, m.v, p)
                                : launch(paged_attention_q8_kernel<BF16, E4M3, DP, ROWS, false>, grid, PA_THREADS, smem, st, false, m.k, m.v, p);
    if (rc != MMV_OK) return rc;
    return launch(paged_join_q8_kernel<BF16>, dim3(static_cast<unsigned>(ctas), static_cast<unsigned>(p.rows * p.side)), PA_JOIN_THREADS, 0, st, true, p, ctas);
}
template <bool BF16, bool E4M3, int DP>
mmv_status launch_dim(const CodeMaps& m, const PagedQ8Params& p, int ctas, cudaStream_t st) {
    return p.rows <= 4   ? launch_rows<BF16, E4M3, DP, 4>(m, p, ctas, st)
           : p.rows <= 8 ? launch_rows<BF16, E4M3, DP, 8>(m, p, ctas, st)
                         : launch_rows<BF16, E4M3, DP, 16>(m, p, ctas, st);
}
template <bool BF16, bool E4M3>
mmv_status launch_paged(const CodeMaps& m, const PagedQ8Params& p, int padded, int ctas, cudaStream_t st) {
    return padded == 64    ? launch_dim<BF16, E4M3, 64>(m, p, ctas, st)
           : padded == 128 ? launch_dim<BF16, E4M3, 128>(m, p, ctas, st)
                           : launch_dim<BF16, E4M3, 256>(m, p, ctas, st);
}

template <bool BF16, bool E4M3>
mmv_status launch_append(const AppendQ8Params& p, bool warp, cudaStream_t st) {
    const long long per = warp ? Q8_THREADS / 32 : 1;
    const dim3 grid(static_cast<unsigned>((p.units + per - 1) / per));
    return warp ? launch(kv_append_q8_kernel<BF16, E4M3, true>, grid, Q8_THREADS, 0, st, false, p)
                : launch(kv_append_q8_kernel<BF16, E4M3, false>, grid, Q8_THREADS, 0, st, false, p);
}

}  // namespace
}  // namespace mmv

using namespace mmv;

extern "C" {

mmv_status mmv_kv_append_q8(const void* k, int64_t k_stride_token, int64_t k_stride_head, const void* v, int64_t v_stride_token, int64_t v_stride_head,
                            mmv_dtype dtype, int64_t ntok, const int32_t* offsets, const int32_t* total, int64_t nreq, const int32_t* table,
                            int64_t table_stride, int64_t max_blocks, const mmv_kv_cache_q8* cache, void* cuda_stream) {
    if (ntok < 0 || ntok > INT32_MAX || nreq < 0 || nreq >= (1ll << 20) || !value_type(dtype) || check_cache(cache) != MMV_OK) return MMV_ERR_INVALID_ARG;
    if (!word_stride(k_stride_token, ntok) || !word_stride(k_stride_head, cache->heads) || !word_stride(v_stride_token, ntok) ||
        !word_stride(v_stride_head, cache->heads) || !check_table(table, table_stride, max_blocks, nreq))
        return MMV_ERR_INVALID_ARG;
    if (ntok == 0 || nreq == 0 || cache->num_blocks == 0 || max_blocks == 0) return MMV_OK;
    if (!k || !v || !aligned(k, 16) || !aligned(v, 16) || !offsets || !aligned(offsets, 4) || !total || !aligned(total, 4)) return MMV_ERR_INVALID_ARG;
    ServeDevice* dev = device();
    if (!dev) return MMV_ERR_CUDA;
    AppendQ8Params p;
    p.c = cache_params(cache);
    p.x[0] = static_cast<const uint16_t*>(k);
    p.x[1] = static_cast<const uint16_t*>(v);
    p.x_tok[0] = k_stride_token;
    p.x_head[0] = k_stride_head;
    p.x_tok[1] = v_stride_token;
    p.x_head[1] = v_stride_head;
    p.offsets = offsets;
    p.total = total;
    p.table = table;
    p.table_stride = table_stride;
    p.max_blocks = max_blocks;
    p.nreq = static_cast<int>(nreq);
    p.ntok = static_cast<int>(ntok);
    p.wide = aligned(k, 32) && aligned(v, 32) && word_stride(k_stride_token, ntok, 16) && word_stride(k_stride_head, cache->heads, 16) &&
             word_stride(v_stride_token, ntok, 16) && word_stride(v_stride_head, cache->heads, 16);
    p.by_row = reciprocal(static_cast<uint32_t>(cache->dim / 16));
    // A window of a run's mean length: what a request adds, cut at the blocks' ends.
    const int64_t runs = ntok / cache->block_size + nreq;
    int64_t window = (ntok + runs - 1) / runs;
    if (window < 1) window = 1;
    // Heads of a unit: as many as leave 32 units per SM (eight CTAs' worth are resident; 53000 tokens of 8 heads: 64 us, with 12 units 72, with 128 71).
    int64_t side = (ntok + window - 1) / window * 2 * cache->heads / (32ll * dev->sm_count);
    side = side < 1 ? 1 : side > cache->heads ? cache->heads : side;
    const int64_t per_window = 2 * ((cache->heads + side - 1) / side);
    const int64_t most = INT32_MAX / per_window;             // (a grid's first axis ends at 2^31 - 1)
    if ((ntok + window - 1) / window > most) window = (ntok + most - 1) / most;
    p.window = static_cast<int>(window);
    p.side = static_cast<int>(side);
    p.units = (ntok + window - 1) / window * per_window;
    // A warp where the mean run fits its registers, else the CTA (255 runs of one token: 6.5 us, by CTAs 12.6; runs of 64 tokens of 128: 98, by CTAs 65).
    const bool warp = window * (cache->dim / 16) <= 32 * Q8_KEEP;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool e4m3 = cache->code == MMV_CODE_E4M3;
    if (dtype == MMV_BF16_TO_F32) return e4m3 ? launch_append<true, true>(p, warp, st) : launch_append<true, false>(p, warp, st);
    return e4m3 ? launch_append<false, true>(p, warp, st) : launch_append<false, false>(p, warp, st);
}

mmv_status mmv_kv_read_q8(const mmv_kv_cache_q8* cache, const int32_t* table, int64_t table_stride, int64_t max_blocks, const int32_t* offsets,
                          int64_t nreq, int64_t ntok, mmv_dtype dtype, void* k_out, void* v_out, void* cuda_stream) {
    if (ntok < 0 || ntok > INT32_MAX || nreq < 0 || nreq >= (1ll << 20) || !value_type(dtype) || check_cache(cache) != MMV_OK ||
        !check_table(table, table_stride, max_blocks, nreq))
        return MMV_ERR_INVALID_ARG;
    if (ntok == 0 || nreq == 0) return MMV_OK;
    if (!offsets || !aligned(offsets, 4) || !k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16)) return MMV_ERR_INVALID_ARG;
    ServeDevice* dev = device();
    if (!dev) return MMV_ERR_CUDA;
    ReadQ8Params p;
    p.c = cache_params(cache);
    p.out[0] = static_cast<uint16_t*>(k_out);
    p.out[1] = static_cast<uint16_t*>(v_out);
    p.offsets = offsets;
    p.table = table;
    p.table_stride = table_stride;
    p.max_blocks = max_blocks;
    p.nreq = static_cast<int>(nreq);
    p.ntok = static_cast<int>(ntok);
    p.wide = aligned(k_out, 32) && aligned(v_out, 32);
    p.words = cache->heads * (cache->dim / 16);
    p.by_words = reciprocal(static_cast<uint32_t>(p.words));
    p.by_head = reciprocal(static_cast<uint32_t>(cache->dim / 16));
    // Tokens of a warp: as many as its loads take at once, fewer where all warps that are resident (2048 threads per SM) then get some, up to 32.
    // 131072 tokens of 64 words (8 heads of 128): 127 us with 1 or 2, 134 with 8, 162 with 32; 262144 of 8 words: 125 us with 1, 37 with 8 or 16, 39 with 32.
    const int64_t warps = static_cast<int64_t>(dev->sm_count) * 64;
    int64_t tile = (ntok + warps - 1) / warps;
    const int64_t most = p.words >= 32 * READ_Q8_UNROLL ? 1 : 32 * READ_Q8_UNROLL / p.words;
    if (tile > most) tile = most;
    if (tile > 32) tile = 32;
    p.tile = static_cast<int>(tile);
    int64_t blocks = ((ntok + tile - 1) / tile + READ_Q8_THREADS / 32 - 1) / (READ_Q8_THREADS / 32);
    if (blocks > dev->sm_count * 64) blocks = dev->sm_count * 64;
    const dim3 grid(static_cast<unsigned>(blocks));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const bool e4m3 = cache->code == MMV_CODE_E4M3;
    if (dtype == MMV_BF16_TO_F32)
        return e4m3 ? launch(kv_read_q8_kernel<true, true>, grid, READ_Q8_THREADS, 0, st, false, p)
                    : launch(kv_read_q8_kernel<true, false>, grid, READ_Q8_THREADS, 0, st, false, p);
    return e4m3 ? launch(kv_read_q8_kernel<false, true>, grid, READ_Q8_THREADS, 0, st, false, p)
                : launch(kv_read_q8_kernel<false, false>, grid, READ_Q8_THREADS, 0, st, false, p);
}

size_t mmv_paged_attention_q8_workspace_bytes(int32_t heads, const mmv_kv_cache_q8* cache) {
    if (check_cache(cache) != MMV_OK || heads < 1 || heads > kMaxHeads || heads % cache->heads) return 0;
    return plan_of(paged_heads(heads, cache->heads, PA_ROWS), cache->heads, cache->dim).total;
}

mmv_status mmv_paged_attention_q8(const void* q, int64_t q_stride_request, int64_t q_stride_head, int32_t heads, mmv_dtype dtype,
                                  const mmv_kv_cache_q8* cache, const int32_t* table, int64_t table_stride, int64_t max_blocks, const int32_t* lens,
                                  int64_t nreq, float scale, int64_t window, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                  void* cuda_stream) {
    if (nreq < 0 || nreq >= (1ll << 20) || window < 0 || !value_type(dtype) || check_cache(cache) != MMV_OK) return MMV_ERR_INVALID_ARG;
    if (heads < 1 || heads > kMaxHeads || heads % cache->heads) return MMV_ERR_INVALID_ARG;
    if (!word_stride(q_stride_request, nreq) || !word_stride(q_stride_head, heads)) return MMV_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256)) return MMV_ERR_INVALID_ARG;
    if (nreq && (!q || !aligned(q, 16) || !lens || !aligned(lens, 4) || !out || !aligned(out, 16) || (lse && !aligned(lse, 4)))) return MMV_ERR_INVALID_ARG;
    if (!check_table(table, table_stride, max_blocks, nreq)) return MMV_ERR_INVALID_ARG;
    const PagedHeads h = paged_heads(heads, cache->heads, PA_ROWS);
    const Plan plan = plan_of(h, cache->heads, cache->dim);
    if (workspace_bytes < plan.total) return MMV_ERR_WORKSPACE_TOO_SMALL;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (nreq == 0) return cudaMemsetAsync(workspace, 0, sizeof(WorkspaceHeader), st) == cudaSuccess ? MMV_OK : MMV_ERR_CUDA;
    ServeDevice* dev = device();
    if (!dev) return MMV_ERR_CUDA;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    PagedQ8Params p;
    p.q = static_cast<const uint16_t*>(q);
    p.k = p.v = nullptr;
    p.k8 = static_cast<const uint8_t*>(cache->k);
    p.v8 = static_cast<const uint8_t*>(cache->v);
    p.ks = cache->k_scale;
    p.vs = cache->v_scale;
    p.s_block = cache->scale_stride_block;
    p.s_head = cache->scale_stride_head;
    p.q_req = q_stride_request;
    p.q_head = q_stride_head;
    p.c_block = cache->stride_block;
    p.c_tok = cache->stride_token;
    p.c_head = cache->stride_head;
    p.table = table;
    p.lens = lens;
    p.table_stride = table_stride;
    p.num_blocks = cache->num_blocks;
    const int64_t longest = INT32_MAX - 16 * PA_TILE;                // (positions past a tile's end stay within 32 bits)
    p.capacity = max_blocks > longest / cache->block_size ? longest : max_blocks * cache->block_size;
    p.window = window;
    p.nreq = static_cast<int>(nreq);
    p.block_size = cache->block_size;
    p.dim = cache->dim;
    p.heads = heads;
    p.kv_heads = cache->heads;
    p.group = h.group;
    p.parts = h.parts;
    p.rows = h.rows;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.out = static_cast<uint16_t*>(out);
    p.lse = lse;
    p.hdr = reinterpret_cast<WorkspaceHeader*>(ws);
    p.desc = reinterpret_cast<int32_t*>(ws + plan.desc_off);
    p.part_ml = reinterpret_cast<float*>(ws + plan.ml_off);
    p.part_m2 = reinterpret_cast<float*>(ws + plan.m2_off);
    p.part_o = reinterpret_cast<float*>(ws + plan.o_off);
    const int padded = paged_padded(p.dim);
    p.budget_ns = g_budget_ns.load();
    p.debug_skip = g_debug_skip_span.load();
    p.by_block = 0;
    CodeMaps maps{};
    maps.box = cache->num_blocks > 0 && cache->block_size % 16 == 0 && code_map(&maps.k, cache->k, cache, padded) && code_map(&maps.v, cache->v, cache, padded);
    if (maps.box) p.by_block = static_cast<uint32_t>((1ull << 32) / static_cast<uint32_t>(cache->block_size));
    // one CTA per tile that the tables could hold, up to all that are resident at once
    const int sms = dev->sm_count < kPagedMaxSms ? dev->sm_count : kPagedMaxSms;
    p.side = heads_side_by_side(p.kv_heads);
    p.tile = 4 * Q8_TOKENS / p.side;
    p.groups = p.kv_heads / p.side * p.parts;
    const double most = static_cast<double>(nreq) * p.groups * (static_cast<double>(p.capacity) / p.tile + 2.0);
    int ctas = sms * per_sm(padded, p.rows);
    if (most < ctas) ctas = static_cast<int>(most);
    const bool e4m3 = cache->code == MMV_CODE_E4M3;
    if (dtype == MMV_BF16_TO_F32) return e4m3 ? launch_paged<true, true>(maps, p, padded, ctas, st) : launch_paged<true, false>(maps, p, padded, ctas, st);
    return e4m3 ? launch_paged<false, true>(maps, p, padded, ctas, st) : launch_paged<false, false>(maps, p, padded, ctas, st);
}

}  // extern "C"

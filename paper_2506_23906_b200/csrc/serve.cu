// Host side of the serving operators of include/mmv.h: argument checks, workspace carve-up and launches.
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/mmv.h"
#include "common.cuh"
#include "host_state.h"
#include "block_tables.cuh"
#include "kv_cache.cuh"
#include "linear_attn.cuh"
#include "paged_attn.cuh"
#include "serve_host.h"

namespace mmv {
namespace {

ServeDevice g_serve[kMaxDevices];

template <int DP>
bool allow_paged() {
    const int bytes = PagedCfg<DP>::smem_bytes(PA_ROWS);
    return allow_smem(paged_attention_kernel<false, DP, false>, bytes) && allow_smem(paged_attention_kernel<false, DP, true>, bytes) &&
           allow_smem(paged_attention_kernel<true, DP, false>, bytes) && allow_smem(paged_attention_kernel<true, DP, true>, bytes);
}

constexpr int kTablesSmemMax = (3 * TABLES_FUSED_MAX + 1) * static_cast<int>(sizeof(int32_t));

// One-time set-up of the current device.
ServeDevice* serve_device() {
    return device_once(g_serve, [] {
        bool ok = allow_smem(block_tables_kernel<1>, kTablesSmemMax) && allow_smem(block_tables_kernel<8>, kTablesSmemMax);
        ok &= allow_paged<64>() && allow_paged<128>() && allow_paged<256>();
        ok &= allow_smem(linear_chunks_kernel<64, true>, LinCfg<64, true>::kSmemBytes);
        ok &= allow_smem(linear_chunks_kernel<64, false>, LinCfg<64, false>::kSmemBytes);
        ok &= allow_smem(linear_chunks_kernel<128, true>, LinCfg<128, true>::kSmemBytes);
        ok &= allow_smem(linear_chunks_kernel<128, false>, LinCfg<128, false>::kSmemBytes);
        return ok;
    });
}

mmv_status check_cache(const mmv_kv_cache* c) {
    if (!c || !value_type(c->dtype)) return MMV_ERR_INVALID_ARG;
    if (c->num_blocks < 0 || c->num_blocks > INT32_MAX || c->block_size < 1 || c->heads < 1 || c->heads > kMaxHeads) return MMV_ERR_INVALID_ARG;
    if (c->dim < 8 || c->dim > 256 || c->dim % 8) return MMV_ERR_INVALID_ARG;
    if (!word_stride(c->stride_block, c->num_blocks) || !word_stride(c->stride_token, c->block_size) || !word_stride(c->stride_head, c->heads))
        return MMV_ERR_INVALID_ARG;
    if (c->num_blocks && (!c->k || !c->v || !aligned(c->k, 16) || !aligned(c->v, 16))) return MMV_ERR_INVALID_ARG;
    return MMV_OK;
}

mmv_status check_linear(const mmv_linear_inputs* in, int64_t tokens) {
    if (!in || !value_type(in->dtype)) return MMV_ERR_INVALID_ARG;
    if (in->heads < 1 || in->heads > kMaxHeads || in->kv_heads < 1 || in->heads % in->kv_heads) return MMV_ERR_INVALID_ARG;
    if (in->dim_k < 8 || in->dim_k > 128 || in->dim_k % 8 || in->dim_v < 8 || in->dim_v > 128 || in->dim_v % 8) return MMV_ERR_INVALID_ARG;
    if (!word_stride(in->q_stride_token, tokens) || !word_stride(in->q_stride_head, in->heads) || !word_stride(in->k_stride_token, tokens) ||
        !word_stride(in->k_stride_head, in->kv_heads) || !word_stride(in->v_stride_token, tokens) || !word_stride(in->v_stride_head, in->kv_heads))
        return MMV_ERR_INVALID_ARG;
    if (!aligned(in->q, 16) || !aligned(in->k, 16) || !aligned(in->v, 16)) return MMV_ERR_INVALID_ARG;
    return MMV_OK;
}

LinParams linear_params(const mmv_linear_inputs* in, const float* log_decay, float scale, void* out) {
    LinParams p{};
    p.q = static_cast<const uint16_t*>(in->q);
    p.k = static_cast<const uint16_t*>(in->k);
    p.v = static_cast<const uint16_t*>(in->v);
    p.q_tok = in->q_stride_token;
    p.q_head = in->q_stride_head;
    p.k_tok = in->k_stride_token;
    p.k_head = in->k_stride_head;
    p.v_tok = in->v_stride_token;
    p.v_head = in->v_stride_head;
    p.heads = in->heads;
    p.group = in->heads / in->kv_heads;
    p.dk = in->dim_k;
    p.dv = in->dim_v;
    p.log_decay = log_decay;
    p.scale = scale;
    p.out = static_cast<uint16_t*>(out);
    return p;
}

// Resident CTAs per SM: what the shared memory of PA_ROWS rows allows (111, 57 and 220 KB of 227).
int paged_per_sm(int padded) { return padded == 64 ? 3 : padded == 128 ? 2 : 1; }

struct PagedPlan {
    size_t desc_off, ml_off, o_off, total;
};
PagedPlan paged_plan(const PagedHeads& h, int dim) {
    const size_t ctas = static_cast<size_t>(kPagedMaxSms) * paged_per_sm(paged_padded(dim));
    PagedPlan w;
    w.desc_off = sizeof(WorkspaceHeader);
    w.ml_off = round_up(w.desc_off + ctas * 4 * sizeof(int32_t), 256);
    w.o_off = round_up(w.ml_off + ctas * 4 * PA_ROWS * sizeof(float), 256);
    w.total = round_up(w.o_off + ctas * 2 * h.rows * dim * sizeof(float), 256);
    return w;
}

template <bool BF16, int DP>
mmv_status launch_paged(const PagedParams& p, int ctas, cudaStream_t st) {
    const size_t smem = static_cast<size_t>(PagedCfg<DP>::smem_bytes(p.rows));
    const dim3 grid(static_cast<unsigned>(ctas));
    const mmv_status rc = p.rows <= 8 ? launch(paged_attention_kernel<BF16, DP, true>, grid, PA_THREADS, smem, st, false, p)
                                      : launch(paged_attention_kernel<BF16, DP, false>, grid, PA_THREADS, smem, st, false, p);
    if (rc != MMV_OK) return rc;
    return launch(paged_join_kernel<BF16>, dim3(static_cast<unsigned>(ctas), static_cast<unsigned>(p.rows)), PA_JOIN_THREADS, 0, st, true, p, ctas);
}

// One CTA per SM, fewer where there are fewer chunks (their upper bound: every sequence ends in a short one).
constexpr int kLinearMaxSms = 160;
int linear_ctas(const mmv_linear_inputs* in, int64_t nseq, int64_t ntok, int sms) {
    int64_t ctas = (ntok / LIN_C + nseq) * in->heads;
    if (ctas > sms) ctas = sms;
    if (ctas > kLinearMaxSms) ctas = kLinearMaxSms;
    return ctas < 1 ? 1 : static_cast<int>(ctas);
}

struct LinearMaps {
    CUtensorMap q, k, v;
};
template <int DK>
mmv_status launch_linear(const LinearMaps& m, const LinParams& p, int ctas, cudaStream_t st) {
    const mmv_status rc = launch(linear_chunks_kernel<DK, true>, dim3(static_cast<unsigned>(ctas)), LIN_THREADS, LinCfg<DK, true>::kSmemBytes,
                                 st, false, m.q, m.k, m.v, p);
    if (rc != MMV_OK) return rc;
    return launch(linear_chunks_kernel<DK, false>, dim3(static_cast<unsigned>(ctas)), LIN_THREADS, LinCfg<DK, false>::kSmemBytes, st, true,
                  m.q, m.k, m.v, p);
}

}  // namespace
}  // namespace mmv

using namespace mmv;

extern "C" {

size_t mmv_block_tables_workspace_bytes(int64_t nreq) {
    if (nreq < 0 || nreq >= (1ll << 20)) return 0;
    const size_t sums = nreq > TABLES_FUSED_MAX ? static_cast<size_t>(nreq) * sizeof(int32_t) : 0;
    return round_up(sizeof(WorkspaceHeader) + sums, 256);
}

mmv_status mmv_block_tables(const int32_t* past, const int32_t* added, int64_t nreq, int32_t block_size, const int32_t* free_blocks,
                            int64_t nfree, int32_t* table, int64_t table_stride, int64_t max_blocks, int32_t* offsets, int32_t* total,
                            int64_t* slots, int64_t nslots, int32_t* used, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (nreq < 0 || nreq >= (1ll << 20) || block_size < 1 || nfree < 0 || max_blocks < 0 || nslots < 0) return MMV_ERR_INVALID_ARG;
    if (!offsets || !used || !workspace || !aligned(offsets, 4) || !aligned(used, 4) || !aligned(workspace, 256)) return MMV_ERR_INVALID_ARG;
    if (nreq && (!past || !added || !total || !aligned(past, 4) || !aligned(added, 4) || !aligned(total, 4))) return MMV_ERR_INVALID_ARG;
    if (nreq && max_blocks && (!table || !aligned(table, 4) || (nreq > 1 && table_stride < max_blocks))) return MMV_ERR_INVALID_ARG;
    if ((nfree && (!free_blocks || !aligned(free_blocks, 4))) || (nslots && (!slots || !aligned(slots, 8)))) return MMV_ERR_INVALID_ARG;
    if (workspace_bytes < mmv_block_tables_workspace_bytes(nreq)) return MMV_ERR_WORKSPACE_TOO_SMALL;
    const size_t lens = static_cast<size_t>(nreq) * sizeof(int32_t);
    const bool in_place = nreq && (total == past || total == added);
    const auto meets = [&](const void* out, size_t bytes) {           // an input that other CTAs may still read
        return overlap(out, bytes, past, lens) || overlap(out, bytes, added, lens) ||
               overlap(out, bytes, free_blocks, static_cast<size_t>(nfree) * sizeof(int32_t));
    };
    if (meets(offsets, lens + sizeof(int32_t)) || meets(used, sizeof(int32_t)) || meets(slots, static_cast<size_t>(nslots) * sizeof(int64_t)))
        return MMV_ERR_INVALID_ARG;
    if ((total != past && overlap(total, lens, past, lens)) || (total != added && overlap(total, lens, added, lens)) ||
        overlap(total, lens, free_blocks, static_cast<size_t>(nfree) * sizeof(int32_t)))
        return MMV_ERR_INVALID_ARG;
    ServeDevice* dev = serve_device();
    if (!dev) return MMV_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    TablesParams p;
    p.past = past;
    p.added = added;
    p.free_blocks = free_blocks;
    p.table = table;
    p.offsets = offsets;
    p.total = total;
    p.used = used;
    p.slots = slots;
    p.nfree = nfree;
    p.table_stride = table_stride;
    p.nslots = nslots;
    p.nreq = static_cast<int>(nreq);
    p.block_size = block_size;
    p.max_blocks = max_blocks;
    p.shift = (block_size & (block_size - 1)) ? -1 : __builtin_ctz(static_cast<unsigned>(block_size));
    p.hdr = static_cast<WorkspaceHeader*>(workspace);
    p.base = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(workspace) + sizeof(WorkspaceHeader));
    const bool single = nslots <= static_cast<int64_t>(dev->sm_count) * TABLES_THREADS;       // one token per thread
    const long long per_cta = TABLES_THREADS * (single ? 1 : 8);
    long long ctas = (nslots + per_cta - 1) / per_cta;
    if (ctas > dev->sm_count) ctas = dev->sm_count;
    if (ctas < 1) ctas = 1;
    const dim3 grid(static_cast<unsigned>(ctas));
    const bool fused = nreq <= TABLES_FUSED_MAX, late = in_place && !(fused && ctas == 1);      // (one CTA has its own copy of the lengths)
    if (late) p.total = nullptr;
    mmv_status rc;
    if (fused) {
        const size_t smem = (3 * nreq + 1) * sizeof(int32_t);
        rc = single ? launch(block_tables_kernel<1>, grid, TABLES_THREADS, smem, st, false, p)
                    : launch(block_tables_kernel<8>, grid, TABLES_THREADS, smem, st, false, p);
    } else {
        rc = launch(block_tables_scan_kernel, dim3(1), TABLES_THREADS, 0, st, false, p);
        if (rc == MMV_OK && nslots)
            rc = single ? launch(block_tables_expand_kernel<1>, grid, TABLES_THREADS, 0, st, true, p)
                        : launch(block_tables_expand_kernel<8>, grid, TABLES_THREADS, 0, st, true, p);
    }
    if (rc != MMV_OK || !late) return rc;
    return launch(block_tables_total_kernel, dim3(static_cast<unsigned>((nreq + TABLES_THREADS - 1) / TABLES_THREADS)), TABLES_THREADS, 0, st, false, p, total);
}

mmv_status mmv_kv_append(const void* k, int64_t k_stride_token, int64_t k_stride_head, const void* v, int64_t v_stride_token,
                         int64_t v_stride_head, const int64_t* slots, int64_t ntok, const mmv_kv_cache* cache, void* cuda_stream) {
    if (ntok < 0 || check_cache(cache) != MMV_OK) return MMV_ERR_INVALID_ARG;
    if (!word_stride(k_stride_token, ntok) || !word_stride(k_stride_head, cache->heads) || !word_stride(v_stride_token, ntok) ||
        !word_stride(v_stride_head, cache->heads))
        return MMV_ERR_INVALID_ARG;
    if (ntok == 0 || cache->num_blocks == 0) return MMV_OK;
    if (!k || !v || !slots || !aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8)) return MMV_ERR_INVALID_ARG;
    ServeDevice* dev = serve_device();
    if (!dev) return MMV_ERR_CUDA;
    AppendParams p;
    p.k = static_cast<const uint16_t*>(k);
    p.v = static_cast<const uint16_t*>(v);
    p.ck = static_cast<uint16_t*>(cache->k);
    p.cv = static_cast<uint16_t*>(cache->v);
    p.slots = slots;
    p.ntok = ntok;
    p.k_tok = k_stride_token;
    p.k_head = k_stride_head;
    p.v_tok = v_stride_token;
    p.v_head = v_stride_head;
    p.c_block = cache->stride_block;
    p.c_tok = cache->stride_token;
    p.c_head = cache->stride_head;
    p.nslots = cache->num_blocks * cache->block_size;
    p.block_size = cache->block_size;
    p.words_per_head = cache->dim / 8;
    p.words_per_row = cache->heads * p.words_per_head;
    const long long words = ntok * p.words_per_row;
    long long blocks = (words + APPEND_THREADS - 1) / APPEND_THREADS;
    const long long cap = static_cast<long long>(dev->sm_count) * 8;        // 2048 threads per SM
    if (blocks > cap) blocks = cap;
    return launch(kv_append_kernel, dim3(static_cast<unsigned>(blocks)), APPEND_THREADS, 0, static_cast<cudaStream_t>(cuda_stream), false, p);
}

size_t mmv_paged_attention_workspace_bytes(int32_t heads, const mmv_kv_cache* cache) {
    if (check_cache(cache) != MMV_OK || heads < 1 || heads > kMaxHeads || heads % cache->heads) return 0;
    return paged_plan(paged_heads(heads, cache->heads, PA_ROWS), cache->dim).total;
}

mmv_status mmv_paged_attention(const void* q, int64_t q_stride_request, int64_t q_stride_head, int32_t heads, const mmv_kv_cache* cache,
                               const int32_t* table, int64_t table_stride, int64_t max_blocks, const int32_t* lens, int64_t nreq,
                               float scale, int64_t window, void* out, float* lse, void* workspace, size_t workspace_bytes,
                               void* cuda_stream) {
    if (nreq < 0 || nreq >= (1ll << 20) || max_blocks < 0 || window < 0 || check_cache(cache) != MMV_OK) return MMV_ERR_INVALID_ARG;
    if (heads < 1 || heads > kMaxHeads || heads % cache->heads) return MMV_ERR_INVALID_ARG;
    if (!word_stride(q_stride_request, nreq) || !word_stride(q_stride_head, heads)) return MMV_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256)) return MMV_ERR_INVALID_ARG;
    if (nreq && (!q || !aligned(q, 16) || !lens || !aligned(lens, 4) || !out || !aligned(out, 16) || (lse && !aligned(lse, 4))))
        return MMV_ERR_INVALID_ARG;
    if (nreq && max_blocks && (!table || !aligned(table, 4) || (nreq > 1 && table_stride < max_blocks))) return MMV_ERR_INVALID_ARG;
    const PagedHeads h = paged_heads(heads, cache->heads, PA_ROWS);
    const PagedPlan plan = paged_plan(h, cache->dim);
    if (workspace_bytes < plan.total) return MMV_ERR_WORKSPACE_TOO_SMALL;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (nreq == 0) return cudaMemsetAsync(workspace, 0, sizeof(WorkspaceHeader), st) == cudaSuccess ? MMV_OK : MMV_ERR_CUDA;
    ServeDevice* dev = serve_device();
    if (!dev) return MMV_ERR_CUDA;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    PagedParams p;
    p.q = static_cast<const uint16_t*>(q);
    p.k = static_cast<const uint16_t*>(cache->k);
    p.v = static_cast<const uint16_t*>(cache->v);
    p.q_req = q_stride_request;
    p.q_head = q_stride_head;
    p.c_block = cache->stride_block;
    p.c_tok = cache->stride_token;
    p.c_head = cache->stride_head;
    p.table = table;
    p.lens = lens;
    p.table_stride = table_stride;
    p.num_blocks = cache->num_blocks;
    const int64_t longest = INT32_MAX - 4 * PA_TILE;                 // (positions past a tile's end stay within 32 bits)
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
    p.part_o = reinterpret_cast<float*>(ws + plan.o_off);
    const int padded = paged_padded(p.dim);
    // one CTA per tile that the tables could hold, up to all that are resident at once
    const int sms = dev->sm_count < kPagedMaxSms ? dev->sm_count : kPagedMaxSms;
    const double most = static_cast<double>(nreq) * p.kv_heads * p.parts * (static_cast<double>(p.capacity) / PA_TILE + 2.0);
    int ctas = sms * paged_per_sm(padded);
    if (most < ctas) ctas = static_cast<int>(most);
    const bool bf16 = cache->dtype == MMV_BF16_TO_F32;
    if (padded == 64) return bf16 ? launch_paged<true, 64>(p, ctas, st) : launch_paged<false, 64>(p, ctas, st);
    if (padded == 128) return bf16 ? launch_paged<true, 128>(p, ctas, st) : launch_paged<false, 128>(p, ctas, st);
    return bf16 ? launch_paged<true, 256>(p, ctas, st) : launch_paged<false, 256>(p, ctas, st);
}

mmv_status mmv_linear_attention_step(const mmv_linear_inputs* in, int64_t nreq, const float* log_decay, float scale, const float* state,
                                     float* state_out, const int32_t* slots, int64_t num_slots, void* out, void* cuda_stream) {
    if (nreq < 0 || num_slots < 0 || check_linear(in, nreq) != MMV_OK) return MMV_ERR_INVALID_ARG;
    if (nreq == 0) return MMV_OK;
    if (!in->q || !in->k || !in->v || !log_decay || !out || !aligned(log_decay, 4) || !aligned(out, 16)) return MMV_ERR_INVALID_ARG;
    if (num_slots && (!state || !state_out || !aligned(state, 16) || !aligned(state_out, 16))) return MMV_ERR_INVALID_ARG;
    if (slots ? !aligned(slots, 4) : num_slots < nreq) return MMV_ERR_INVALID_ARG;
    if (nreq > INT32_MAX / (static_cast<int64_t>(in->heads) * 16)) return MMV_ERR_INVALID_ARG;       // one CTA per state and column part
    const size_t states = static_cast<size_t>(num_slots) * in->heads * in->dim_k * in->dim_v * sizeof(float);
    if (state != state_out && overlap(state, states, state_out, states)) return MMV_ERR_INVALID_ARG;      // (in place, or apart)
    ServeDevice* dev = serve_device();
    if (!dev) return MMV_ERR_CUDA;
    LinParams p = linear_params(in, log_decay, scale, out);
    p.state = state;
    p.state_out = state_out;
    p.slots = slots;
    p.nreq = nreq;
    p.num_slots = num_slots;
    // Whole rows, or parts of 32 columns: up to 64 columns parts are always faster (2048 states 128 x 64: 25.2 against 31.9 us), with 128 from
    // about one state per SM on whole rows are (64 states 3.4 against 3.9 us, 256 states 6.4 against 5.6 us, 4096 states 89.6 against 81.9 us).
    const bool wide = p.dv > 64 && nreq * p.heads >= dev->sm_count;
    p.parts = wide ? 1 : (p.dv + 31) / 32;
    const dim3 grid(static_cast<unsigned>(nreq * p.heads * p.parts));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (in->dtype == MMV_BF16_TO_F32)
        return wide ? launch(linear_step_kernel<true, 128>, grid, LIN_STEP_THREADS, 0, st, false, p)
                    : launch(linear_step_kernel<true, 32>, grid, LIN_STEP_THREADS, 0, st, false, p);
    return wide ? launch(linear_step_kernel<false, 128>, grid, LIN_STEP_THREADS, 0, st, false, p)
                : launch(linear_step_kernel<false, 32>, grid, LIN_STEP_THREADS, 0, st, false, p);
}

size_t mmv_linear_attention_workspace_bytes(const mmv_linear_inputs* in, int64_t nseq, int64_t ntok) {
    if (nseq < 0 || ntok < 0 || ntok > INT32_MAX || check_linear(in, ntok) != MMV_OK) return 0;
    return sizeof(WorkspaceHeader) + static_cast<size_t>(linear_ctas(in, nseq, ntok, kLinearMaxSms)) * (in->dim_k <= 64 ? 64 : 128) * 128 * sizeof(float);
}

mmv_status mmv_linear_attention(const mmv_linear_inputs* in, const int32_t* offsets, int64_t nseq, int64_t ntok, const float* log_decay,
                                float scale, const float* state, float* state_out, void* out, void* workspace, size_t workspace_bytes,
                                void* cuda_stream) {
    if (nseq < 0 || nseq >= (1ll << 20) || ntok < 0 || ntok > INT32_MAX || check_linear(in, ntok) != MMV_OK || in->dtype != MMV_BF16_TO_F32)
        return MMV_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256)) return MMV_ERR_INVALID_ARG;
    if (nseq && (!offsets || !aligned(offsets, 4) || !log_decay || !aligned(log_decay, 4))) return MMV_ERR_INVALID_ARG;
    if (ntok && (!in->q || !in->k || !in->v || !out || !aligned(out, 16))) return MMV_ERR_INVALID_ARG;
    if ((state && !aligned(state, 16)) || (state_out && !aligned(state_out, 16))) return MMV_ERR_INVALID_ARG;
    if (workspace_bytes < mmv_linear_attention_workspace_bytes(in, nseq, ntok)) return MMV_ERR_WORKSPACE_TOO_SMALL;
    const size_t states = static_cast<size_t>(nseq) * in->heads * in->dim_k * in->dim_v * sizeof(float);
    if (state && state_out && overlap(state, states, state_out, states)) return MMV_ERR_INVALID_ARG;      // (a cut sequence's state is read by several CTAs)
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (nseq == 0) return cudaMemsetAsync(workspace, 0, sizeof(WorkspaceHeader), st) == cudaSuccess ? MMV_OK : MMV_ERR_CUDA;
    ServeDevice* dev = serve_device();
    if (!dev) return MMV_ERR_CUDA;
    LinParams p = linear_params(in, log_decay, scale, out);
    p.state = state;
    p.state_out = state_out;
    p.offsets = offsets;
    p.nseq = nseq;
    p.ntok = ntok;
    p.hdr = static_cast<WorkspaceHeader*>(workspace);
    p.carry = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + sizeof(WorkspaceHeader));
    p.budget_ns = g_budget_ns.load();
    LinearMaps maps;
    if (!token_map(&maps.q, in->q, in->dim_k, in->heads, ntok, in->q_stride_head, in->q_stride_token) ||
        !token_map(&maps.k, in->k, in->dim_k, in->kv_heads, ntok, in->k_stride_head, in->k_stride_token) ||
        !token_map(&maps.v, in->v, in->dim_v, in->kv_heads, ntok, in->v_stride_head, in->v_stride_token))
        return MMV_ERR_INVALID_ARG;
    const int ctas = linear_ctas(in, nseq, ntok, dev->sm_count);
    return in->dim_k <= 64 ? launch_linear<64>(maps, p, ctas, st) : launch_linear<128>(maps, p, ctas, st);
}

}  // extern "C"

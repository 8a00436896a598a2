// Host side of the gated delta rule of include/mmv.h: argument checks, workspace carve-up and launches.
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/mmv.h"
#include "common.cuh"
#include "gated_delta.cuh"
#include "host_state.h"
#include "serve_host.h"

namespace mmv {
namespace {

ServeDevice g_devices[kMaxDevices];

template <int DK>
bool allow_dim() {
    return allow_smem(delta_prep_kernel<DK>, DeltaPrepCfg<DK>::kSmemBytes) && allow_smem(delta_chunks_kernel<DK, 16>, DeltaCfg<DK, 16>::kSmemBytes) &&
           allow_smem(delta_chunks_kernel<DK, 32>, DeltaCfg<DK, 32>::kSmemBytes);
}
ServeDevice* device() {
    return device_once(g_devices, [] { return allow_dim<64>() && allow_dim<128>(); });
}

mmv_status check_inputs(const mmv_delta_inputs* in, int64_t tokens) {
    if (!in || !value_type(in->dtype)) return MMV_ERR_INVALID_ARG;
    if (in->heads < 1 || in->heads > kMaxHeads || in->key_heads < 1 || in->heads % in->key_heads) return MMV_ERR_INVALID_ARG;
    if (in->dim_k < 8 || in->dim_k > 128 || in->dim_k % 8 || in->dim_v < 8 || in->dim_v > 128 || in->dim_v % 8) return MMV_ERR_INVALID_ARG;
    if (!word_stride(in->q_stride_token, tokens) || !word_stride(in->q_stride_head, in->key_heads) || !word_stride(in->k_stride_token, tokens) ||
        !word_stride(in->k_stride_head, in->key_heads) || !word_stride(in->v_stride_token, tokens) || !word_stride(in->v_stride_head, in->heads))
        return MMV_ERR_INVALID_ARG;
    if (!aligned(in->q, 16) || !aligned(in->k, 16) || !aligned(in->v, 16) || !aligned(in->log_decay, 4) || !aligned(in->beta, 4)) return MMV_ERR_INVALID_ARG;
    return MMV_OK;
}
bool missing(const mmv_delta_inputs* in) { return !in->q || !in->k || !in->v || !in->log_decay || !in->beta; }

DeltaParams params_of(const mmv_delta_inputs* in, float scale, void* out) {
    DeltaParams p{};
    p.q = static_cast<const uint16_t*>(in->q);
    p.k = static_cast<const uint16_t*>(in->k);
    p.v = static_cast<const uint16_t*>(in->v);
    p.q_tok = in->q_stride_token;
    p.q_head = in->q_stride_head;
    p.k_tok = in->k_stride_token;
    p.k_head = in->k_stride_head;
    p.v_tok = in->v_stride_token;
    p.v_head = in->v_stride_head;
    p.decay = in->log_decay;
    p.beta = in->beta;
    p.decay_tok = in->log_decay_stride_token;
    p.beta_tok = in->beta_stride_token;
    p.heads = in->heads;
    p.group = in->heads / in->key_heads;
    p.dk = in->dim_k;
    p.dv = in->dim_v;
    p.scale = scale;
    p.out = static_cast<uint16_t*>(out);
    return p;
}

// Places of chunks (delta_slot): all of them, and those of one part, a pair of launches, whose operands the workspace holds.  A batch that is longer is taken in parts,
// two of which the workspace holds then: the first kernel of a part runs beside the second one of the part in front of it.
struct DeltaParts {
    int64_t all, step;
    int halves;
};
constexpr int64_t kPlaces = 36864;                           // (chunk, head)s: 784 MB
constexpr int64_t kMostTokens = INT32_MAX - DELTA_C;         // (positions past a chunk's end stay within 32 bits)
DeltaParts parts_of(const mmv_delta_inputs* in, int64_t nseq, int64_t ntok) {
    const int64_t all = ntok / DELTA_C + nseq, most = kPlaces / in->heads;
    // One sequence whose heads leave half of the SMs idle: the chain of its chunks takes its time on few CTAs, and the first kernels of small parts all but the
    // first hide behind it (65536 tokens, 16 heads: 2.33 ms, as one part 2.55).  Several sequences would wait for one another (2 of 8192: 0.79 ms, as one
    // part 0.48), so their parts are as large as the workspace may be (2 of 32768: 1.87 ms, with a quarter of it 3.04; 256 of 512 and 32 heads: 8.3, 9.4).
    const bool alone = nseq == 1 && in->heads * ((in->dim_v + 31) / 32) <= 72;
    const int64_t small = most / 16 < 1 ? 1 : most / 16;
    if (all <= (alone ? small : most)) return {all, all, 1};
    const int64_t step = alone ? small : most / 2;
    return {all, step < 1 ? 1 : step, 2};
}

template <int DK>
mmv_status launch_delta(const CUtensorMap& q, const CUtensorMap& k, const DeltaParams& p, int64_t places, bool beside, int nv, cudaStream_t st) {
    const unsigned prep = static_cast<unsigned>(places * (p.heads / p.group)), ctas = static_cast<unsigned>(static_cast<int64_t>(p.present) * p.heads * p.slices);
    const mmv_status rc = launch(delta_prep_kernel<DK>, dim3(prep), DELTA_PREP_THREADS, DeltaPrepCfg<DK>::kSmemBytes, st, beside, q, k, p);
    if (rc != MMV_OK) return rc;
    return nv == 16 ? launch(delta_chunks_kernel<DK, 16>, dim3(ctas), DELTA_THREADS, DeltaCfg<DK, 16>::kSmemBytes, st, true, q, k, p)
                    : launch(delta_chunks_kernel<DK, 32>, dim3(ctas), DELTA_THREADS, DeltaCfg<DK, 32>::kSmemBytes, st, true, q, k, p);
}

}  // namespace
}  // namespace mmv

using namespace mmv;

extern "C" {

mmv_status mmv_gated_delta_step(const mmv_delta_inputs* in, int64_t nreq, float scale, const float* state, float* state_out, const int32_t* slots,
                                int64_t num_slots, void* out, void* cuda_stream) {
    if (nreq < 0 || num_slots < 0 || check_inputs(in, nreq) != MMV_OK) return MMV_ERR_INVALID_ARG;
    if (nreq == 0) return MMV_OK;
    if (missing(in) || !out || !aligned(out, 16)) return MMV_ERR_INVALID_ARG;
    if (num_slots && (!state || !state_out || !aligned(state, 16) || !aligned(state_out, 16))) return MMV_ERR_INVALID_ARG;
    if (slots ? !aligned(slots, 4) : num_slots < nreq) return MMV_ERR_INVALID_ARG;
    if (nreq > INT32_MAX / (static_cast<int64_t>(in->heads) * 16)) return MMV_ERR_INVALID_ARG;       // one CTA per state and column part
    const size_t states = static_cast<size_t>(num_slots) * in->heads * in->dim_k * in->dim_v * sizeof(float);
    if (state != state_out && overlap(state, states, state_out, states)) return MMV_ERR_INVALID_ARG;      // (in place, or apart)
    ServeDevice* dev = device();
    if (!dev) return MMV_ERR_CUDA;
    DeltaParams p = params_of(in, scale, out);
    p.state = state;
    p.state_out = state_out;
    p.slots = slots;
    p.num_slots = num_slots;
    // Whole rows of a state by one CTA, or 32 columns where that leaves SMs idle (16 heads: 4 requests 4.8 us, in whole rows 6.3; 128 48 us, by columns 55).
    const bool wide = p.dv > 64 && nreq * p.heads >= dev->sm_count;
    p.parts = wide ? 1 : (p.dv + 31) / 32;
    const dim3 grid(static_cast<unsigned>(nreq * p.heads * p.parts));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (in->dtype == MMV_BF16_TO_F32)
        return wide ? launch(delta_step_kernel<true, 128>, grid, LIN_STEP_THREADS, 0, st, false, p)
                    : launch(delta_step_kernel<true, 32>, grid, LIN_STEP_THREADS, 0, st, false, p);
    return wide ? launch(delta_step_kernel<false, 128>, grid, LIN_STEP_THREADS, 0, st, false, p)
                : launch(delta_step_kernel<false, 32>, grid, LIN_STEP_THREADS, 0, st, false, p);
}

size_t mmv_gated_delta_workspace_bytes(const mmv_delta_inputs* in, int64_t nseq, int64_t ntok) {
    if (nseq < 0 || nseq >= (1ll << 20) || ntok < 0 || ntok > kMostTokens || check_inputs(in, ntok) != MMV_OK) return 0;
    const DeltaParts parts = parts_of(in, nseq, ntok);
    return round_up(sizeof(WorkspaceHeader) + static_cast<size_t>(parts.step) * parts.halves * in->heads * sizeof(DeltaChunk), 256);
}

mmv_status mmv_gated_delta(const mmv_delta_inputs* in, const int32_t* offsets, int64_t nseq, int64_t ntok, float scale, const float* state,
                           float* state_out, void* out, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (nseq < 0 || nseq >= (1ll << 20) || ntok < 0 || ntok > kMostTokens || check_inputs(in, ntok) != MMV_OK || in->dtype != MMV_BF16_TO_F32)
        return MMV_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256)) return MMV_ERR_INVALID_ARG;
    if (nseq && (!offsets || !aligned(offsets, 4) || !state_out || !aligned(state_out, 16) || (state && !aligned(state, 16)))) return MMV_ERR_INVALID_ARG;
    if (ntok && (missing(in) || !out || !aligned(out, 16))) return MMV_ERR_INVALID_ARG;
    if (workspace_bytes < mmv_gated_delta_workspace_bytes(in, nseq, ntok)) return MMV_ERR_WORKSPACE_TOO_SMALL;
    const size_t states = static_cast<size_t>(nseq) * in->heads * in->dim_k * in->dim_v * sizeof(float);
    if (state && state != state_out && overlap(state, states, state_out, states)) return MMV_ERR_INVALID_ARG;      // (in place, or apart)
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (nseq == 0) return cudaMemsetAsync(workspace, 0, sizeof(WorkspaceHeader), st) == cudaSuccess ? MMV_OK : MMV_ERR_CUDA;
    ServeDevice* dev = device();
    if (!dev) return MMV_ERR_CUDA;
    DeltaParams p = params_of(in, scale, out);
    p.state = state;
    p.state_out = state_out;
    p.offsets = offsets;
    p.nseq = static_cast<int>(nseq);
    p.ntok = static_cast<int>(ntok);
    p.hdr = static_cast<WorkspaceHeader*>(workspace);
    p.budget_ns = g_budget_ns.load();
    p.debug_skip = g_debug_skip_span.load();
    CUtensorMap map_q, map_k;
    if (!token_map(&map_q, in->q, in->dim_k, in->key_heads, ntok, in->q_stride_head, in->q_stride_token) ||
        !token_map(&map_k, in->k, in->dim_k, in->key_heads, ntok, in->k_stride_head, in->k_stride_token))
        return MMV_ERR_INVALID_ARG;
    // Slices of 32 columns, of 16 where those leave half of the SMs idle (4096 tokens: 1 sequence of 18 heads 173 us, with 32 columns 224; of 20 heads
    // 228 us, with 16 columns 315).  This rule and parts_of's count sequences: how long each is only the device knows.  One long prompt beside short ones, or beside
    // empty entries of a padded batch, is taken as several are (16 heads: 32768 tokens 1.19 ms, beside 1 or 15 others of a token or none 1.71).
    const int nv = nseq * p.heads * ((p.dv + 31) / 32) <= dev->sm_count / 2 ? 16 : 32;
    p.slices = (p.dv + nv - 1) / nv;
    if (nseq * p.heads > INT32_MAX / p.slices) return MMV_ERR_INVALID_ARG;       // one CTA per (sequence, head) and slice
    const DeltaParts parts = parts_of(in, nseq, ntok);
    uint8_t* const chunks = static_cast<uint8_t*>(workspace) + sizeof(WorkspaceHeader);
    for (int64_t at = 0, part = 0; at < parts.all; at += parts.step, ++part) {
        p.first_slot = at;
        p.last_slot = at + parts.step < parts.all ? at + parts.step : parts.all;
        p.chunks = chunks + static_cast<size_t>(part & (parts.halves - 1)) * parts.step * p.heads * sizeof(DeltaChunk);
        const int64_t places = p.last_slot - at;
        // (a sequence has a place of its own at least, and one may reach in from the part in front)
        p.present = static_cast<int>(nseq < places + 1 ? nseq : places + 1);
        const mmv_status rc = in->dim_k <= 64 ? launch_delta<64>(map_q, map_k, p, places, at > 0, nv, st) : launch_delta<128>(map_q, map_k, p, places, at > 0, nv, st);
        if (rc != MMV_OK) return rc;
    }
    return MMV_OK;
}

}  // extern "C"

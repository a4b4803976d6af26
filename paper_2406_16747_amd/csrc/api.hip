// C-ABI entry points of libsparsek: argument validation, then the launch wrappers.
#include "common.hpp"
#include "block_parts.hpp"
#include "mask_ranges.hpp"

#include <initializer_list>
#include <utility>

using namespace spk;

namespace {

int check_common(const sparsek_cfg* c)
{
    if (!c) return SPARSEK_ERR_INVALID_ARG;
    if (c->B < 1 || c->H < 1 || c->n < 1 || c->k < 0 || c->w < 0 || (long long)c->k + c->w < 1)
        return SPARSEK_ERR_INVALID_ARG;
    if (c->Gu != 1 && c->Gu != c->H) return SPARSEK_ERR_INVALID_ARG;
    if ((long long)c->B * c->H > 65535) return SPARSEK_ERR_UNSUPPORTED;
    if ((long long)c->n > (1 << 28)) return SPARSEK_ERR_UNSUPPORTED;
    // k and w beyond n mean the same as n; larger values are refused rather than clamped so that sums such as
    // k + w and w - 1 + death[j] stay far from the int32 range everywhere
    if (c->k > (1 << 28) || c->w > (1 << 28)) return SPARSEK_ERR_UNSUPPORTED;
    return SPARSEK_OK;
}

int check_attn(const sparsek_cfg* c)
{
    int rc = check_common(c);
    if (rc) return rc;
    if (c->gate_mode < 0 || c->gate_mode > 3) return SPARSEK_ERR_INVALID_ARG;
    if (c->dtype != SPARSEK_F32 && c->dtype != SPARSEK_BF16) return SPARSEK_ERR_UNSUPPORTED;
    if (c->d < 4 || c->d > 128 || (c->d % 4) != 0) return SPARSEK_ERR_UNSUPPORTED;
    if (!(c->softmax_scale > 0.0f) || !(c->softmax_scale < INFINITY)) return SPARSEK_ERR_INVALID_ARG;
    return SPARSEK_OK;
}

}  // namespace

extern "C" {

const char* sparsek_strerror(int code)
{
    switch (code) {
        case SPARSEK_OK: return "ok";
        case SPARSEK_ERR_INVALID_ARG: return "invalid argument";
        case SPARSEK_ERR_UNSUPPORTED: return "unsupported shape or dtype";
        case SPARSEK_ERR_WORKSPACE: return "workspace or state buffer too small";
        case SPARSEK_ERR_LAUNCH: return "HIP launch failed";
        case SPARSEK_ERR_TOO_LARGE: return "problem larger than the built-in scratch array of sparsek_mask_static";
        default: return "unknown error";
    }
}

size_t sparsek_mask_workspace_bytes(const sparsek_cfg* cfg)
{
    if (check_common(cfg)) return 0;
    return mask_ws_bytes(*cfg);
}

int sparsek_mask(const sparsek_cfg* cfg, const float* u, float* tau, int32_t* death, void* ws,
                 size_t ws_bytes, void* stream)
{
    int rc = check_common(cfg);
    if (rc) return rc;
    if (!u || !tau || !death || !ws) return SPARSEK_ERR_INVALID_ARG;
    if (ws_bytes < mask_ws_bytes(*cfg)) return SPARSEK_ERR_WORKSPACE;
    return launch_mask(*cfg, u, tau, death, ws, (hipStream_t)stream);
}

int sparsek_mask_status(const sparsek_cfg* cfg, const void* ws, size_t ws_bytes, int32_t* host_flag, void* stream)
{
    int rc = check_common(cfg);
    if (rc) return rc;
    if (!ws || !host_flag) return SPARSEK_ERR_INVALID_ARG;
    if (ws_bytes < mask_ws_bytes(*cfg)) return SPARSEK_ERR_WORKSPACE;
    return mask_status(*cfg, ws, host_flag, (hipStream_t)stream);
}

int sparsek_materialize(const sparsek_cfg* cfg, const float* u, const float* tau, const int32_t* death,
                        int32_t t_begin, int32_t t_end, int32_t* idx, float* gate, void* stream)
{
    int rc = check_common(cfg);
    if (rc) return rc;
    if (!u || !tau || !death || !idx) return SPARSEK_ERR_INVALID_ARG;
    if (t_begin < 0 || t_end < t_begin || t_end > cfg->n) return SPARSEK_ERR_INVALID_ARG;
    if (t_end - t_begin > 65535 * 16) return SPARSEK_ERR_UNSUPPORTED;
    return launch_materialize(*cfg, u, tau, death, t_begin, t_end, idx, gate, (hipStream_t)stream);
}

size_t sparsek_attn_fwd_workspace_bytes(const sparsek_cfg* cfg)
{
    if (check_attn(cfg)) return 0;
    return attn_fwd_ws_bytes(*cfg);
}

int sparsek_attn_fwd(const sparsek_cfg* cfg, const void* q, const void* k, const void* v, const float* u,
                     const float* tau, const int32_t* death, void* o, float* lse, void* ws,
                     size_t ws_bytes, void* stream)
{
    int rc = check_attn(cfg);
    if (rc) return rc;
    if (!q || !k || !v || !u || !tau || !death || !o || !ws) return SPARSEK_ERR_INVALID_ARG;
    if (ws_bytes < attn_fwd_ws_bytes(*cfg)) return SPARSEK_ERR_WORKSPACE;
    sparsek_cfg c = *cfg;
    if (c.gate_mode == 3) c.gate_mode = 2;  // the straight-through forward is the hard-selection forward
    return launch_attn_fwd(c, q, k, v, u, tau, death, o, lse, ws, (hipStream_t)stream);
}

}  // extern "C"


extern "C" {

size_t sparsek_attn_bwd_workspace_bytes(const sparsek_cfg* cfg)
{
    if (check_attn(cfg)) return 0;
    return spk::attn_bwd_ws_bytes(*cfg);
}

int sparsek_attn_bwd(const sparsek_cfg* cfg, const void* q, const void* k, const void* v, const float* u,
                     const float* tau, const int32_t* death, const void* o, const float* lse, const void* dO, void* dq,
                     void* dk, void* dv, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_attn(cfg);
    if (rc) return rc;
    if (!q || !k || !v || !u || !tau || !death || !o || !lse || !dO || !dq || !dk || !dv || !ws)
        return SPARSEK_ERR_INVALID_ARG;
    if (ws_bytes < spk::attn_bwd_ws_bytes(*cfg)) return SPARSEK_ERR_WORKSPACE;
    sparsek_cfg c = *cfg;
    if (c.gate_mode == 3) c.gate_mode = 2;  // the straight-through forward has no gates on q, k, v
    return spk::launch_attn_bwd(c, q, k, v, u, tau, death, o, lse, dO, dq, dk, dv, ws, (hipStream_t)stream);
}

}  // extern "C"

// ---- importance scores (scores.hip) ----
namespace spk {
size_t scores_ws_bytes(int B, int n);
int launch_scores(int B, int n, int D, int dtype, int norm, double slope, double norm_eps, const void* x,
                  const float* w, float* u, void* ws, hipStream_t st);
}  // namespace spk

namespace {
int check_scores(const sparsek_scores_cfg* c)
{
    if (!c) return SPARSEK_ERR_INVALID_ARG;
    if (c->B < 1 || c->n < 1 || c->D < 1) return SPARSEK_ERR_INVALID_ARG;
    if (c->norm != 0 && c->norm != 1) return SPARSEK_ERR_INVALID_ARG;
    if (!(c->slope > -INFINITY) || !(c->slope < INFINITY)) return SPARSEK_ERR_INVALID_ARG;
    if (c->norm == 1 && (!(c->norm_eps > 0.0f) || !(c->norm_eps < INFINITY))) return SPARSEK_ERR_INVALID_ARG;
    if (c->dtype != SPARSEK_F32 && c->dtype != SPARSEK_BF16) return SPARSEK_ERR_UNSUPPORTED;
    if ((c->D % 8) != 0 || c->D > 8192) return SPARSEK_ERR_UNSUPPORTED;
    if ((long long)c->n > (1 << 28) || c->B > 65535) return SPARSEK_ERR_UNSUPPORTED;
    return SPARSEK_OK;
}
}  // namespace

extern "C" {

size_t sparsek_scores_workspace_bytes(const sparsek_scores_cfg* cfg)
{
    if (check_scores(cfg)) return 0;
    return spk::scores_ws_bytes(cfg->B, cfg->n);
}

int sparsek_scores(const sparsek_scores_cfg* cfg, const void* x, const float* w, float* u, void* ws,
                   size_t ws_bytes, void* stream)
{
    int rc = check_scores(cfg);
    if (rc) return rc;
    if (!x || !w || !u) return SPARSEK_ERR_INVALID_ARG;
    if (cfg->norm == 1 && (!ws || ws_bytes < spk::scores_ws_bytes(cfg->B, cfg->n))) return SPARSEK_ERR_WORKSPACE;
    return spk::launch_scores(cfg->B, cfg->n, cfg->D, cfg->dtype, cfg->norm, (double)cfg->slope,
                              (double)cfg->norm_eps, x, w, u, ws, (hipStream_t)stream);
}

}  // extern "C"

// ---- entry points whose kernels live in mask_bwd.hip and decode.hip ----
namespace spk {
size_t decode_state_bytes(const sparsek_decode_cfg& c);
int launch_decode_init(const sparsek_decode_cfg& c, void* state, hipStream_t st);
int launch_decode_load(const sparsek_decode_cfg& c, void* state, int n_ctx, const void* k, const void* v,
                       const float* u, const float* tau, const int32_t* death, hipStream_t st);
int launch_decode_step(const sparsek_decode_cfg& c, void* state, const void* q, const void* k, const void* v,
                       const float* u_new, void* o, hipStream_t st);
int decode_status(const sparsek_decode_cfg& c, const void* state, int32_t* host_flags, hipStream_t st);
}  // namespace spk

namespace {
int check_decode(const sparsek_decode_cfg* c)
{
    if (!c) return SPARSEK_ERR_INVALID_ARG;
    if (c->B < 1 || c->H < 1 || c->k < 0 || c->w < 0 || (long long)c->k + c->w < 1 || c->cand_cap < 0)
        return SPARSEK_ERR_INVALID_ARG;
    if (c->Gu != 1 && c->Gu != c->H) return SPARSEK_ERR_INVALID_ARG;
    if (c->gate_mode < 0 || c->gate_mode > 3) return SPARSEK_ERR_INVALID_ARG;
    if (c->dtype != SPARSEK_F32 && c->dtype != SPARSEK_BF16) return SPARSEK_ERR_UNSUPPORTED;
    // the state holds k + w slots per head and cand_cap (default 4k) scores per row: sizes are computed in int
    if (c->k > (1 << 24) || c->w > (1 << 24) || c->cand_cap > (1 << 26)) return SPARSEK_ERR_UNSUPPORTED;
    if (c->d < 8 || c->d > 128 || (c->d % 8) != 0) return SPARSEK_ERR_UNSUPPORTED;
    if ((long long)c->B * c->H > (1 << 24)) return SPARSEK_ERR_UNSUPPORTED;
    if (!(c->softmax_scale > 0.0f) || !(c->softmax_scale < INFINITY)) return SPARSEK_ERR_INVALID_ARG;
    return SPARSEK_OK;
}
}  // namespace

extern "C" {

size_t sparsek_mask_bwd_workspace_bytes(const sparsek_cfg* cfg)
{
    if (check_attn(cfg)) return 0;
    return mask_bwd_ws_bytes(*cfg);
}

int sparsek_mask_bwd(const sparsek_cfg* cfg, const void* q, const void* k, const void* v, const float* u,
                     const float* tau, const int32_t* death, const void* o, const float* lse, const void* dO,
                     float* du, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_attn(cfg);
    if (rc) return rc;
    if (!q || !k || !v || !u || !tau || !death || !o || !lse || !dO || !du || !ws)
        return SPARSEK_ERR_INVALID_ARG;
    if (ws_bytes < mask_bwd_ws_bytes(*cfg)) return SPARSEK_ERR_WORKSPACE;
    return launch_mask_bwd(*cfg, q, k, v, u, tau, death, o, lse, dO, du, ws, (hipStream_t)stream);
}

size_t sparsek_bwd_workspace_bytes(const sparsek_cfg* cfg)
{
    if (check_attn(cfg)) return 0;
    return align_up(spk::attn_bwd_ws_bytes(*cfg), 256) + mask_bwd_ws_bytes(*cfg);
}

int sparsek_bwd(const sparsek_cfg* cfg, const void* q, const void* k, const void* v, const float* u, const float* tau,
                const int32_t* death, const void* o, const float* lse, const void* dO, void* dq, void* dk, void* dv,
                float* du, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_attn(cfg);
    if (rc) return rc;
    if (!q || !k || !v || !u || !tau || !death || !o || !lse || !dO || !dq || !dk || !dv || !du || !ws)
        return SPARSEK_ERR_INVALID_ARG;
    if (ws_bytes < sparsek_bwd_workspace_bytes(cfg)) return SPARSEK_ERR_WORKSPACE;
    return spk::launch_bwd(*cfg, q, k, v, u, tau, death, o, lse, dO, dq, dk, dv, du, ws,
                           (char*)ws + align_up(spk::attn_bwd_ws_bytes(*cfg), 256), (hipStream_t)stream);
}

size_t sparsek_decode_state_bytes(const sparsek_decode_cfg* cfg)
{
    if (check_decode(cfg)) return 0;
    return decode_state_bytes(*cfg);
}

int sparsek_decode_init(const sparsek_decode_cfg* cfg, void* state, size_t state_bytes, void* stream)
{
    int rc = check_decode(cfg);
    if (rc) return rc;
    if (!state) return SPARSEK_ERR_INVALID_ARG;
    if (state_bytes < decode_state_bytes(*cfg)) return SPARSEK_ERR_WORKSPACE;
    return launch_decode_init(*cfg, state, (hipStream_t)stream);
}

int sparsek_decode_load(const sparsek_decode_cfg* cfg, void* state, size_t state_bytes, int32_t n_ctx,
                        const void* k, const void* v, const float* u, const float* tau, const int32_t* death,
                        void* stream)
{
    int rc = check_decode(cfg);
    if (rc) return rc;
    if (!state || n_ctx < 0) return SPARSEK_ERR_INVALID_ARG;
    if (n_ctx > 0 && (!k || !v || !u || !tau || !death)) return SPARSEK_ERR_INVALID_ARG;
    if (state_bytes < decode_state_bytes(*cfg)) return SPARSEK_ERR_WORKSPACE;
    if (n_ctx == 0) return launch_decode_init(*cfg, state, (hipStream_t)stream);
    return launch_decode_load(*cfg, state, n_ctx, k, v, u, tau, death, (hipStream_t)stream);
}

int sparsek_decode_step(const sparsek_decode_cfg* cfg, void* state, const void* q_new, const void* k_new,
                        const void* v_new, const float* u_new, void* o, void* stream)
{
    int rc = check_decode(cfg);
    if (rc) return rc;
    if (!state || !q_new || !k_new || !v_new || !u_new || !o) return SPARSEK_ERR_INVALID_ARG;
    sparsek_decode_cfg c = *cfg;
    if (c.gate_mode == 3) c.gate_mode = 2;  // straight-through: the forward skips the gates
    return launch_decode_step(c, state, q_new, k_new, v_new, u_new, o, (hipStream_t)stream);
}

int sparsek_decode_status(const sparsek_decode_cfg* cfg, const void* state, int32_t* host_flags, void* stream)
{
    int rc = check_decode(cfg);
    if (rc) return rc;
    if (!state || !host_flags) return SPARSEK_ERR_INVALID_ARG;
    return decode_status(*cfg, state, host_flags, (hipStream_t)stream);
}

}  // extern "C"

// ---- chunk-wise recurrent prefill (chunk.hip) ----
namespace spk {
size_t chunk_state_bytes(const sparsek_chunk_cfg& c);
size_t chunk_ws_bytes(const sparsek_chunk_cfg& c);
int launch_chunk_init(const sparsek_chunk_cfg& c, void* state, hipStream_t st);
int launch_chunk_prefill(const sparsek_chunk_cfg& c, void* state, int clen, const void* q, const void* k,
                         const void* v, const float* u, void* o, void* ws, hipStream_t st);
int chunk_status(const sparsek_chunk_cfg& c, const void* state, int32_t* host_counts, int32_t* host_flags,
                 hipStream_t st);
int launch_chunk_to_decode(const sparsek_chunk_cfg& c, void* state, void* ws, const sparsek_decode_cfg& dc,
                           void* dstate, hipStream_t st);
size_t chunk_bwd_ws_bytes(const sparsek_chunk_cfg& c);
int launch_chunk_bwd(const sparsek_chunk_cfg& c, int clen, const void* q, const void* o, const void* dO,
                     const void* fwd_ws, void* dq, void* dk, void* dv, float* du, void* ws, hipStream_t st);
}  // namespace spk

namespace {
int check_chunk(const sparsek_chunk_cfg* c)
{
    if (!c) return SPARSEK_ERR_INVALID_ARG;
    if (c->B < 1 || c->H < 1 || c->k < 0 || c->w < 0 || (long long)c->k + c->w < 1 || c->cand_cap < 0 || c->chunk_max < 1)
        return SPARSEK_ERR_INVALID_ARG;
    if (c->Gu != 1 && c->Gu != c->H) return SPARSEK_ERR_INVALID_ARG;
    if (c->gate_mode < 0 || c->gate_mode > 3) return SPARSEK_ERR_INVALID_ARG;
    if (!(c->softmax_scale > 0.0f) || !(c->softmax_scale < INFINITY)) return SPARSEK_ERR_INVALID_ARG;
    if (c->dtype != SPARSEK_F32 && c->dtype != SPARSEK_BF16) return SPARSEK_ERR_UNSUPPORTED;
    if (c->d < 4 || c->d > 128 || (c->d % 4) != 0) return SPARSEK_ERR_UNSUPPORTED;
    if ((c->d * (c->dtype == SPARSEK_BF16 ? 2 : 4)) % 16 != 0) return SPARSEK_ERR_UNSUPPORTED;
    if ((long long)c->B * c->H > 65535) return SPARSEK_ERR_UNSUPPORTED;
    if ((long long)c->k + c->w + c->cand_cap + c->chunk_max > (1 << 26)) return SPARSEK_ERR_UNSUPPORTED;
    return SPARSEK_OK;
}
}  // namespace

extern "C" {

size_t sparsek_chunk_state_bytes(const sparsek_chunk_cfg* cfg)
{
    if (check_chunk(cfg)) return 0;
    return spk::chunk_state_bytes(*cfg);
}

size_t sparsek_chunk_workspace_bytes(const sparsek_chunk_cfg* cfg)
{
    if (check_chunk(cfg)) return 0;
    return spk::chunk_ws_bytes(*cfg);
}

int sparsek_chunk_init(const sparsek_chunk_cfg* cfg, void* state, size_t state_bytes, void* stream)
{
    int rc = check_chunk(cfg);
    if (rc) return rc;
    if (!state) return SPARSEK_ERR_INVALID_ARG;
    if (state_bytes < spk::chunk_state_bytes(*cfg)) return SPARSEK_ERR_WORKSPACE;
    return spk::launch_chunk_init(*cfg, state, (hipStream_t)stream);
}

int sparsek_chunk_prefill(const sparsek_chunk_cfg* cfg, void* state, size_t state_bytes, int32_t c, const void* q,
                          const void* k, const void* v, const float* u, void* o, void* ws, size_t ws_bytes,
                          void* stream)
{
    int rc = check_chunk(cfg);
    if (rc) return rc;
    if (!state || !q || !k || !v || !u || !o || !ws) return SPARSEK_ERR_INVALID_ARG;
    if (c < 1 || c > cfg->chunk_max) return SPARSEK_ERR_INVALID_ARG;
    if (state_bytes < spk::chunk_state_bytes(*cfg) || ws_bytes < spk::chunk_ws_bytes(*cfg)) return SPARSEK_ERR_WORKSPACE;
    return spk::launch_chunk_prefill(*cfg, state, c, q, k, v, u, o, ws, (hipStream_t)stream);
}

size_t sparsek_chunk_bwd_workspace_bytes(const sparsek_chunk_cfg* cfg)
{
    if (check_chunk(cfg)) return 0;
    if (cfg->dtype != SPARSEK_BF16 || (cfg->d != 64 && cfg->d != 128)) return 0;
    return spk::chunk_bwd_ws_bytes(*cfg);
}

int sparsek_chunk_bwd(const sparsek_chunk_cfg* cfg, int32_t c, const void* q, const void* o, const void* dO,
                      const void* fwd_ws, size_t fwd_ws_bytes, void* dq, void* dk, void* dv, float* du, void* ws,
                      size_t ws_bytes, void* stream)
{
    int rc = check_chunk(cfg);
    if (rc) return rc;
    if (!q || !o || !dO || !fwd_ws || !dq || !dk || !dv || !du || !ws) return SPARSEK_ERR_INVALID_ARG;
    if (c < 1 || c > cfg->chunk_max) return SPARSEK_ERR_INVALID_ARG;
    if (cfg->dtype != SPARSEK_BF16 || (cfg->d != 64 && cfg->d != 128)) return SPARSEK_ERR_UNSUPPORTED;
    if (fwd_ws_bytes < spk::chunk_ws_bytes(*cfg) || ws_bytes < spk::chunk_bwd_ws_bytes(*cfg)) return SPARSEK_ERR_WORKSPACE;
    return spk::launch_chunk_bwd(*cfg, c, q, o, dO, fwd_ws, dq, dk, dv, du, ws, (hipStream_t)stream);
}

int sparsek_chunk_to_decode(const sparsek_chunk_cfg* cfg, void* state, size_t state_bytes, int64_t n_consumed,
                            void* ws, size_t ws_bytes, const sparsek_decode_cfg* dcfg, void* decode_state,
                            size_t decode_state_bytes, void* stream)
{
    int rc = check_chunk(cfg);
    if (rc) return rc;
    rc = check_decode(dcfg);
    if (rc) return rc;
    if (!state || !ws || !decode_state) return SPARSEK_ERR_INVALID_ARG;
    if (dcfg->B != cfg->B || dcfg->H != cfg->H || dcfg->Gu != cfg->Gu || dcfg->d != cfg->d || dcfg->k != cfg->k ||
        dcfg->w != cfg->w || dcfg->dtype != cfg->dtype)
        return SPARSEK_ERR_INVALID_ARG;
    if (n_consumed < (int64_t)cfg->k + cfg->w) return SPARSEK_ERR_UNSUPPORTED;
    if (state_bytes < spk::chunk_state_bytes(*cfg) || ws_bytes < spk::chunk_ws_bytes(*cfg) ||
        decode_state_bytes < spk::decode_state_bytes(*dcfg))
        return SPARSEK_ERR_WORKSPACE;
    return spk::launch_chunk_to_decode(*cfg, state, ws, *dcfg, decode_state, (hipStream_t)stream);
}

int sparsek_chunk_status(const sparsek_chunk_cfg* cfg, const void* state, int32_t* host_counts, int32_t* host_flags,
                         void* stream)
{
    int rc = check_chunk(cfg);
    if (rc) return rc;
    if (!state) return SPARSEK_ERR_INVALID_ARG;
    return spk::chunk_status(*cfg, state, host_counts, host_flags, (hipStream_t)stream);
}

}  // extern "C"

// ---- attention over blocks of tokens (block_select.hip, block_attn.hip, block_attn_bwd.hip) and the caches in 8 and in 4 bits (cache8.hip, cache4.hip) ----
namespace spk {
size_t block_select_ws_bytes(const sparsek_block_cfg& c);
int launch_block_select(const sparsek_block_cfg& c, const void* q, const void* k, int32_t* idx, void* ws, hipStream_t st);
size_t block_fwd_ws_bytes(const sparsek_block_cfg& c);
int launch_block_fwd(const sparsek_block_cfg& c, const void* q, const void* k, const void* v, const int32_t* idx, void* o, float* lse,
                     float* mass, void* ws, hipStream_t st);
size_t block_bwd_ws_bytes(const sparsek_block_cfg& c);
int launch_block_bwd(const sparsek_block_cfg& c, const void* q, const void* k, const void* v, const int32_t* idx, const void* o,
                     const float* lse, const void* dO, void* dq, void* dk, void* dv, void* ws, hipStream_t st);
int launch_cache8_append(const sparsek_cache8_cfg& c, const sparsek_cache8& t, const int32_t* lens, const int32_t* counts, int count,
                         const void* k, const void* v, hipStream_t st);
int launch_cache8_select(const sparsek_cache8_cfg& c, const sparsek_cache8& t, const int32_t* lens, const void* q, int top, int32_t* idx,
                         hipStream_t st);
size_t cache8_attn_ws_bytes(const sparsek_cache8_cfg& c, int top);
int launch_cache8_attn(const sparsek_cache8_cfg& c, const sparsek_cache8& t, const int32_t* lens, const void* q, const int32_t* idx,
                       int top, int accumulate, void* o, float* lse, void* ws, hipStream_t st);
int launch_cache8_evict(const sparsek_cache8_cfg& c, const sparsek_cache8& t, const int32_t* lens, int budget, int sink, int recent,
                        int32_t* table, float* mass, int32_t* lens_out, hipStream_t st);
int launch_cache4_append(const sparsek_cache8_cfg& c, const sparsek_cache4& t, const int32_t* lens, const int32_t* counts, int count,
                         const void* k, const void* v, hipStream_t st);
int launch_cache4_read(const sparsek_cache8_cfg& c, const sparsek_cache4& t, const int32_t* lens, int begin, int n, void* k, void* v, hipStream_t st);
int launch_cache4_select(const sparsek_cache8_cfg& c, const sparsek_cache4& t, const int32_t* lens, const void* q, int top, int32_t* idx,
                         hipStream_t st);
int launch_cache4_attn(const sparsek_cache8_cfg& c, const sparsek_cache4& t, const int32_t* lens, const void* q, const int32_t* idx,
                       int top, int accumulate, void* o, float* lse, void* ws, hipStream_t st);
int launch_cache4_evict(const sparsek_cache8_cfg& c, const sparsek_cache4& t, const int32_t* lens, int budget, int sink, int recent,
                        int32_t* table, float* mass, int32_t* lens_out, hipStream_t st);
}  // namespace spk

namespace {

constexpr int MAX_BLOCK_TOP = 64, MAX_CACHE_BLOCKS = 8192;

int check_heads(int B, int H, int Hkv, int d, int dtype, float scale)
{
    if (B < 1 || H < 1 || Hkv < 1 || H % Hkv != 0) return SPARSEK_ERR_INVALID_ARG;
    if (!(scale > 0.0f) || !(scale < INFINITY)) return SPARSEK_ERR_INVALID_ARG;
    if (dtype != SPARSEK_BF16 || (d != 64 && d != 128)) return SPARSEK_ERR_UNSUPPORTED;
    if ((long long)B * H > 65535) return SPARSEK_ERR_UNSUPPORTED;
    return SPARSEK_OK;
}

int check_block(const sparsek_block_cfg* c)
{
    if (!c || c->n < 1 || c->top < 0) return SPARSEK_ERR_INVALID_ARG;
    int rc = check_heads(c->B, c->H, c->Hkv, c->d, c->dtype, c->softmax_scale);
    if (rc) return rc;
    if (c->n > (1 << 20) || c->top > MAX_BLOCK_TOP) return SPARSEK_ERR_UNSUPPORTED;
    if ((long long)c->n * (c->H / c->Hkv) > (1 << 28)) return SPARSEK_ERR_UNSUPPORTED;   // rows of one block's list
    return SPARSEK_OK;
}

// What is read or written 16 bytes at a time.
bool aligned(std::initializer_list<const void*> ps)
{
    for (const void* p : ps)
        if ((uintptr_t)p & 15) return false;
    return true;
}

bool overlap(const void* a, size_t na, const void* b, size_t nb)
{
    return (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

struct Place {
    const void* p;
    size_t n;
    bool on(const Place& x) const { return p && x.p && n && x.n && overlap(p, n, x.p, x.n); }
};

// Whether an output lies over an input or over another output.
template <int IN, int OUT>
bool any_overlap(const Place (&in)[IN], const Place (&out)[OUT])
{
    for (int x = 0; x < OUT; x++) {
        for (const Place& y : in)
            if (out[x].on(y)) return true;
        for (int y = 0; y < x; y++)
            if (out[x].on(out[y])) return true;
    }
    return false;
}

// Both caches: the same checks, and the same launches.
struct Of8 {
    typedef sparsek_cache8 Cache;
    static bool format(int f) { return f == SPARSEK_I8 || f == SPARSEK_E4M3; }
    static bool whole(const Cache& t) { return t.k8 && t.v8 && t.ks && t.vs && t.km && t.kms && t.kt && t.vt && t.table && t.mass; }
    static bool wide(const Cache& t) { return aligned({t.k8, t.v8, t.km, t.kt, t.vt}); }
    static constexpr auto append = spk::launch_cache8_append;
    static constexpr auto select = spk::launch_cache8_select;
    static constexpr auto attn = spk::launch_cache8_attn;
    static constexpr auto evict = spk::launch_cache8_evict;
};
struct Of4 {
    typedef sparsek_cache4 Cache;
    static bool format(int f) { return f == SPARSEK_E2M1; }
    static bool whole(const Cache& t) { return t.k4 && t.v4 && t.ke && t.ve && t.ks && t.vs && t.km && t.kms && t.kt && t.vt && t.table && t.mass; }
    static bool wide(const Cache& t) { return aligned({t.k4, t.v4, t.ke, t.ve, t.km, t.kt, t.vt}); }
    static constexpr auto append = spk::launch_cache4_append;
    static constexpr auto select = spk::launch_cache4_select;
    static constexpr auto attn = spk::launch_cache4_attn;
    static constexpr auto evict = spk::launch_cache4_evict;
};

template <class Of>
int check_cache(const sparsek_cache8_cfg* c, const typename Of::Cache* t)
{
    if (!c || c->cap < 1 || c->pages < 1) return SPARSEK_ERR_INVALID_ARG;
    int rc = check_heads(c->B, c->H, c->Hkv, c->d, c->dtype, c->softmax_scale);
    if (rc) return rc;
    if (!Of::format(c->format)) return SPARSEK_ERR_UNSUPPORTED;
    if (c->cap > MAX_CACHE_BLOCKS || c->pages > (1 << 24)) return SPARSEK_ERR_UNSUPPORTED;
    if (t && !Of::whole(*t)) return SPARSEK_ERR_INVALID_ARG;
    return SPARSEK_OK;
}

template <class Of>
int cache_append(const sparsek_cache8_cfg* cfg, const typename Of::Cache* cache, const int32_t* lens, const int32_t* counts,
                 int32_t c, const void* k, const void* v, void* stream)
{
    if (!cache) return SPARSEK_ERR_INVALID_ARG;
    int rc = check_cache<Of>(cfg, cache);
    if (rc) return rc;
    if (!lens || !k || !v || c < 1 || !Of::wide(*cache) || !aligned({k, v})) return SPARSEK_ERR_INVALID_ARG;
    if (c > (1 << 24)) return SPARSEK_ERR_UNSUPPORTED;
    return Of::append(*cfg, *cache, lens, counts, c, k, v, (hipStream_t)stream);
}

template <class Of>
int cache_select(const sparsek_cache8_cfg* cfg, const typename Of::Cache* cache, const int32_t* lens, const void* q, int32_t top,
                 int32_t* idx, void* stream)
{
    if (!cache) return SPARSEK_ERR_INVALID_ARG;
    int rc = check_cache<Of>(cfg, cache);
    if (rc) return rc;
    if (!lens || !q || !idx || top < 1 || !Of::wide(*cache) || !aligned({q})) return SPARSEK_ERR_INVALID_ARG;
    if (top > MAX_CACHE_BLOCKS) return SPARSEK_ERR_UNSUPPORTED;
    return Of::select(*cfg, *cache, lens, q, top, idx, (hipStream_t)stream);
}

template <class Of>
size_t cache_attn_workspace_bytes(const sparsek_cache8_cfg* cfg, int32_t top)
{
    if (check_cache<Of>(cfg, nullptr) || top < 0 || top > MAX_CACHE_BLOCKS) return 0;
    return spk::cache8_attn_ws_bytes(*cfg, top);
}

template <class Of>
int cache_attn(const sparsek_cache8_cfg* cfg, const typename Of::Cache* cache, const int32_t* lens, const void* q,
               const int32_t* idx, int32_t top, int32_t accumulate, void* o, float* lse, void* ws, size_t ws_bytes,
               void* stream)
{
    if (!cache) return SPARSEK_ERR_INVALID_ARG;
    int rc = check_cache<Of>(cfg, cache);
    if (rc) return rc;
    if (!lens || !q || !o || !lse || (idx ? top < 1 : top != 0)) return SPARSEK_ERR_INVALID_ARG;
    if (!Of::wide(*cache) || !aligned({q, o, ws})) return SPARSEK_ERR_INVALID_ARG;
    if (top > MAX_CACHE_BLOCKS) return ws ? SPARSEK_ERR_UNSUPPORTED : SPARSEK_ERR_INVALID_ARG;
    const size_t need = spk::cache8_attn_ws_bytes(*cfg, top);
    const bool none = cfg->format == SPARSEK_E2M1 && need == spk::NO_WORKSPACE;
    if (!ws && !none) return SPARSEK_ERR_INVALID_ARG;
    if (ws && ws_bytes < need) return SPARSEK_ERR_WORKSPACE;
    return Of::attn(*cfg, *cache, lens, q, idx, top, accumulate != 0, o, lse, ws, (hipStream_t)stream);
}

template <class Of>
int cache_evict(const sparsek_cache8_cfg* cfg, const typename Of::Cache* cache, const int32_t* lens, int32_t budget, int32_t sink,
                int32_t recent, int32_t* table_out, float* mass_out, int32_t* lens_out, void* stream)
{
    if (!cache) return SPARSEK_ERR_INVALID_ARG;
    int rc = check_cache<Of>(cfg, cache);
    if (rc) return rc;
    if (!lens || !table_out || !mass_out || !lens_out) return SPARSEK_ERR_INVALID_ARG;
    if (budget < 0 || sink < 0 || recent < 0 || (long long)sink + recent > budget) return SPARSEK_ERR_INVALID_ARG;
    const size_t nt = (size_t)cfg->B * cfg->Hkv * cfg->cap * 4, nl = (size_t)cfg->B * 4;
    const void* in[] = {cache->table, cache->mass, lens};
    const size_t nin[] = {nt, nt, nl};
    void* out[] = {table_out, mass_out, lens_out};
    for (int x = 0; x < 3; x++)
        for (int y = 0; y < 3; y++) {
            if (overlap(in[x], nin[x], out[y], nin[y])) return SPARSEK_ERR_INVALID_ARG;
            if (x < y && overlap(out[x], nin[x], out[y], nin[y])) return SPARSEK_ERR_INVALID_ARG;
        }
    return Of::evict(*cfg, *cache, lens, budget, sink, recent, table_out, mass_out, lens_out, (hipStream_t)stream);
}

}  // namespace

extern "C" {

size_t sparsek_block_select_workspace_bytes(const sparsek_block_cfg* cfg)
{
    if (check_block(cfg)) return 0;
    return spk::block_select_ws_bytes(*cfg);
}

int sparsek_block_select(const sparsek_block_cfg* cfg, const void* q, const void* k, int32_t* idx, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_block(cfg);
    if (rc) return rc;
    if (!q || !k || (!idx && cfg->top) || !ws || !aligned({q, k, ws})) return SPARSEK_ERR_INVALID_ARG;
    if (ws_bytes < spk::block_select_ws_bytes(*cfg)) return SPARSEK_ERR_WORKSPACE;
    return spk::launch_block_select(*cfg, q, k, idx, ws, (hipStream_t)stream);
}

size_t sparsek_block_attn_fwd_workspace_bytes(const sparsek_block_cfg* cfg)
{
    if (check_block(cfg)) return 0;
    return spk::block_fwd_ws_bytes(*cfg);
}

int sparsek_block_attn_fwd(const sparsek_block_cfg* cfg, const void* q, const void* k, const void* v, const int32_t* idx, void* o,
                           float* lse, float* mass, void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_block(cfg);
    if (rc) return rc;
    if (!q || !k || !v || (!idx && cfg->top) || !o || !lse || !ws || !aligned({q, k, v, o, ws})) return SPARSEK_ERR_INVALID_ARG;
    if (ws_bytes < spk::block_fwd_ws_bytes(*cfg)) return SPARSEK_ERR_WORKSPACE;
    return spk::launch_block_fwd(*cfg, q, k, v, idx, o, lse, mass, ws, (hipStream_t)stream);
}

size_t sparsek_block_attn_bwd_workspace_bytes(const sparsek_block_cfg* cfg)
{
    if (check_block(cfg)) return 0;
    return spk::block_bwd_ws_bytes(*cfg);
}

int sparsek_block_attn_bwd(const sparsek_block_cfg* cfg, const void* q, const void* k, const void* v, const int32_t* idx,
                           const void* o, const float* lse, const void* dO, void* dq, void* dk, void* dv, void* ws, size_t ws_bytes,
                           void* stream)
{
    int rc = check_block(cfg);
    if (rc) return rc;
    if (!q || !k || !v || (!idx && cfg->top) || !o || !lse || !dO || !dq || !dk || !dv || !ws) return SPARSEK_ERR_INVALID_ARG;
    if (!aligned({q, k, v, o, dO, dq, dk, dv, ws})) return SPARSEK_ERR_INVALID_ARG;
    if (ws_bytes < spk::block_bwd_ws_bytes(*cfg)) return SPARSEK_ERR_WORKSPACE;
    return spk::launch_block_bwd(*cfg, q, k, v, idx, o, lse, dO, dq, dk, dv, ws, (hipStream_t)stream);
}

int sparsek_cache8_append(const sparsek_cache8_cfg* cfg, const sparsek_cache8* cache, const int32_t* lens, const int32_t* counts,
                          int32_t c, const void* k, const void* v, void* stream)
{
    return cache_append<Of8>(cfg, cache, lens, counts, c, k, v, stream);
}

int sparsek_cache8_select(const sparsek_cache8_cfg* cfg, const sparsek_cache8* cache, const int32_t* lens, const void* q, int32_t top,
                          int32_t* idx, void* stream)
{
    return cache_select<Of8>(cfg, cache, lens, q, top, idx, stream);
}

size_t sparsek_cache8_attn_workspace_bytes(const sparsek_cache8_cfg* cfg, int32_t top)
{
    return cache_attn_workspace_bytes<Of8>(cfg, top);
}

int sparsek_cache8_attn(const sparsek_cache8_cfg* cfg, const sparsek_cache8* cache, const int32_t* lens, const void* q,
                        const int32_t* idx, int32_t top, int32_t accumulate, void* o, float* lse, void* ws, size_t ws_bytes,
                        void* stream)
{
    return cache_attn<Of8>(cfg, cache, lens, q, idx, top, accumulate, o, lse, ws, ws_bytes, stream);
}

int sparsek_cache8_evict(const sparsek_cache8_cfg* cfg, const sparsek_cache8* cache, const int32_t* lens, int32_t budget, int32_t sink,
                         int32_t recent, int32_t* table_out, float* mass_out, int32_t* lens_out, void* stream)
{
    return cache_evict<Of8>(cfg, cache, lens, budget, sink, recent, table_out, mass_out, lens_out, stream);
}

int sparsek_cache4_append(const sparsek_cache8_cfg* cfg, const sparsek_cache4* cache, const int32_t* lens, const int32_t* counts,
                          int32_t c, const void* k, const void* v, void* stream)
{
    return cache_append<Of4>(cfg, cache, lens, counts, c, k, v, stream);
}

int sparsek_cache4_select(const sparsek_cache8_cfg* cfg, const sparsek_cache4* cache, const int32_t* lens, const void* q, int32_t top,
                          int32_t* idx, void* stream)
{
    return cache_select<Of4>(cfg, cache, lens, q, top, idx, stream);
}

size_t sparsek_cache4_attn_workspace_bytes(const sparsek_cache8_cfg* cfg, int32_t top)
{
    return cache_attn_workspace_bytes<Of4>(cfg, top);
}

int sparsek_cache4_attn(const sparsek_cache8_cfg* cfg, const sparsek_cache4* cache, const int32_t* lens, const void* q,
                        const int32_t* idx, int32_t top, int32_t accumulate, void* o, float* lse, void* ws, size_t ws_bytes,
                        void* stream)
{
    return cache_attn<Of4>(cfg, cache, lens, q, idx, top, accumulate, o, lse, ws, ws_bytes, stream);
}

int sparsek_cache4_evict(const sparsek_cache8_cfg* cfg, const sparsek_cache4* cache, const int32_t* lens, int32_t budget, int32_t sink,
                         int32_t recent, int32_t* table_out, float* mass_out, int32_t* lens_out, void* stream)
{
    return cache_evict<Of4>(cfg, cache, lens, budget, sink, recent, table_out, mass_out, lens_out, stream);
}

int sparsek_cache4_read(const sparsek_cache8_cfg* cfg, const sparsek_cache4* cache, const int32_t* lens, int32_t begin, int32_t n, void* k,
                        void* v, void* stream)
{
    if (!cache) return SPARSEK_ERR_INVALID_ARG;
    int rc = check_cache<Of4>(cfg, cache);
    if (rc) return rc;
    if (!lens || !k || !v || begin < 0 || n < 1 || !Of4::wide(*cache) || !aligned({k, v})) return SPARSEK_ERR_INVALID_ARG;
    if ((long long)begin + n > (1 << 28)) return SPARSEK_ERR_UNSUPPORTED;
    const size_t pages = cfg->pages, rows = (size_t)cfg->B * cfg->Hkv, d = cfg->d, tail = rows * 64 * d * 2;
    const Place in[] = {{cache->k4, pages * 32 * d}, {cache->v4, pages * 32 * d}, {cache->ke, pages * 2 * d}, {cache->ve, pages * 2 * d}, {cache->ks, pages * 4},
                        {cache->vs, pages * 4}, {cache->kt, tail}, {cache->vt, tail}, {cache->table, rows * cfg->cap * 4}, {lens, cfg->B * 4u}};
    const Place out[] = {{k, rows * n * d * 2}, {v, rows * n * d * 2}};
    if (any_overlap(in, out)) return SPARSEK_ERR_INVALID_ARG;
    return spk::launch_cache4_read(*cfg, *cache, lens, begin, n, k, v, (hipStream_t)stream);
}

}  // extern "C"

// ---- norms of queries and keys with rotary positions (rope.hip) ----
namespace spk {
int launch_rope_fwd(const sparsek_rope_cfg& c, const void* q, const void* k, const int32_t* pos, const float* freq, const int32_t* axis,
                    const float* qw, const float* kw, void* qo, void* ko, hipStream_t st);
size_t rope_bwd_ws_bytes(const sparsek_rope_cfg& c);
int launch_rope_bwd(const sparsek_rope_cfg& c, const void* q, const void* k, const int32_t* pos, const float* freq, const int32_t* axis,
                    const float* qw, const float* kw, const void* dqo, const void* dko, void* dq, void* dk, float* dqw, float* dkw, void* ws,
                    hipStream_t st);
}  // namespace spk

namespace {

// Strides that the kernels can take: rows begin at multiples of 4 elements, and the last one below 2^46 of them.
bool good(const sparsek_rope_cfg& c, const sparsek_rope_strides& s, int heads)
{
    for (int64_t x : {s.batch, s.token, s.head})
        if (x < 0 || x > (1ll << 45) || x % 4) return false;
    return (double)(c.B - 1) * s.batch + (double)(c.n - 1) * s.token + (double)(heads - 1) * s.head < 0x1p46;
}

// What a strided [B,n,heads,d] spans, in bytes.
size_t span(const sparsek_rope_cfg& c, const sparsek_rope_strides& s, int heads)
{
    const int64_t last = (c.B - 1) * s.batch + (c.n - 1) * s.token + (heads - 1) * s.head + c.d;
    return (size_t)last * (c.dtype == SPARSEK_BF16 ? 2 : 4);
}

size_t positions(const sparsek_rope_cfg& c) { return c.rot ? (size_t)c.axes * c.B * c.n * 4 : 0; }

// Whether every place of a strided output has an address of its own: each stride steps over all that the smaller ones reach.
bool apart(const sparsek_rope_cfg& c, const sparsek_rope_strides& s, int heads)
{
    std::pair<int64_t, int64_t> dims[3] = {{s.batch, c.B}, {s.token, c.n}, {s.head, heads}};
    std::sort(dims, dims + 3);
    int64_t reach = c.d;
    for (const auto& x : dims) {
        if (x.second == 1) continue;
        if (x.first < reach) return false;
        reach += (x.second - 1) * x.first;
    }
    return true;
}

// Places of a strided output: rows of `row` bytes, and the steps between them, the largest first.
struct Rows {
    int64_t row, step[3], count[3], reach[4];   // reach[i]: what the steps from i on span
    int n = 0;
    Rows(const sparsek_rope_cfg& c, const sparsek_rope_strides& s, int heads)
    {
        const int64_t size = c.dtype == SPARSEK_BF16 ? 2 : 4;
        std::pair<int64_t, int64_t> dims[3] = {{s.batch, c.B}, {s.token, c.n}, {s.head, heads}};
        std::sort(dims, dims + 3);
        for (int x = 2; x >= 0; x--)
            if (dims[x].second > 1) {
                step[n] = dims[x].first * size;
                count[n++] = dims[x].second;
            }
        reach[n] = row = c.d * size;
        for (int x = n - 1; x >= 0; x--) reach[x] = reach[x + 1] + (count[x] - 1) * step[x];
    }
};

// Whether a row of b, which begins `off` bytes behind a, lies over one of a; both are apart() in themselves, from steps i and j on.  Equal steps leave three
// pairs of neighbours at most to look at; others are gone through one by one, and what is not through after `left` pairs counts as meeting (a
// fused gradient has the same steps for both but for the heads, of which there are 65535).
bool meet(const Rows& a, int i, const Rows& b, int j, int64_t off, int& left)
{
    if (off >= a.reach[i] || -off >= b.reach[j]) return false;
    if ((i == a.n && j == b.n) || --left < 0) return true;
    const int64_t sa = i < a.n ? a.step[i] : 0, sb = j < b.n ? b.step[j] : 0;
    const bool in_a = sa >= sb, in_b = sb >= sa;
    const int64_t step = std::max(sa, sb), ra = a.reach[i + in_a], rb = b.reach[j + in_b];
    // parts x of a and y of b that are off + (y - x) step apart, more than -rb and less than ra
    const int64_t x1 = in_a ? a.count[i] - 1 : 0, y1 = in_b ? b.count[j] - 1 : 0;
    for (int64_t m = std::max(-x1, -((off + rb - 1) / step)); m <= y1 && off + m * step < ra; m++)
        if (meet(a, i + in_a, b, j + in_b, off + m * step, left)) return true;
    return false;
}

int check_rope(const sparsek_rope_cfg* c)
{
    if (!c || c->B < 1 || c->H < 1 || c->Hkv < 0 || c->n < 1 || c->d < 1 || c->rot < 0 || c->rot > c->d || c->axes < 1) return SPARSEK_ERR_INVALID_ARG;
    if (c->norm && (!(c->eps >= 0x1p-126f) || !(c->eps < INFINITY))) return SPARSEK_ERR_INVALID_ARG;
    if (c->dtype != SPARSEK_BF16 && c->dtype != SPARSEK_F32) return SPARSEK_ERR_UNSUPPORTED;
    if (c->d % 8 || c->d > 256 || c->rot % 8 || c->axes > 4) return SPARSEK_ERR_UNSUPPORTED;
    if ((long long)c->H + c->Hkv > 65535 || (long long)c->B * c->n > (1ll << 26)) return SPARSEK_ERR_UNSUPPORTED;
    if (!good(*c, c->q, c->H) || (c->Hkv && !good(*c, c->k, c->Hkv))) return SPARSEK_ERR_INVALID_ARG;
    return SPARSEK_OK;
}

// Arguments that both directions share.  (x_read: q and k are read.)
int check_rope_inputs(const sparsek_rope_cfg& c, bool x_read, const void* q, const void* k, const int32_t* pos, const float* freq)
{
    if (x_read && (!q || (c.Hkv && !k))) return SPARSEK_ERR_INVALID_ARG;
    if (c.rot && (!pos || !freq)) return SPARSEK_ERR_INVALID_ARG;
    return aligned({q, k}) ? SPARSEK_OK : SPARSEK_ERR_INVALID_ARG;
}

}  // namespace

extern "C" {

int sparsek_rope_fwd(const sparsek_rope_cfg* cfg, const void* q, const void* k, const int32_t* pos, const float* freq, const int32_t* axis,
                     const float* qw, const float* kw, void* qo, void* ko, void* stream)
{
    int rc = check_rope(cfg);
    if (rc) return rc;
    const sparsek_rope_cfg& c = *cfg;
    if ((rc = check_rope_inputs(c, true, q, k, pos, freq))) return rc;
    if (!qo || (c.Hkv && !ko) || !aligned({qo, ko})) return SPARSEK_ERR_INVALID_ARG;
    const size_t row = (size_t)c.B * c.n * c.d * (c.dtype == SPARSEK_BF16 ? 2 : 4), nw = (size_t)c.d * 4;
    const Place in[] = {{q, span(c, c.q, c.H)}, {k, c.Hkv ? span(c, c.k, c.Hkv) : 0}, {pos, positions(c)}, {freq, c.rot * 2u}, {axis, c.rot * 2u},
                        {qw, nw}, {kw, nw}};
    const Place out[] = {{qo, row * c.H}, {ko, row * c.Hkv}};
    if (any_overlap(in, out)) return SPARSEK_ERR_INVALID_ARG;
    return spk::launch_rope_fwd(c, q, k, pos, freq, axis, qw, kw, qo, ko, (hipStream_t)stream);
}

size_t sparsek_rope_bwd_workspace_bytes(const sparsek_rope_cfg* cfg)
{
    if (check_rope(cfg)) return 0;
    return spk::rope_bwd_ws_bytes(*cfg);
}

int sparsek_rope_bwd(const sparsek_rope_cfg* cfg, const void* q, const void* k, const int32_t* pos, const float* freq, const int32_t* axis,
                     const float* qw, const float* kw, const void* dqo, const void* dko, void* dq, void* dk, float* dqw, float* dkw,
                     void* ws, size_t ws_bytes, void* stream)
{
    int rc = check_rope(cfg);
    if (rc) return rc;
    const sparsek_rope_cfg& c = *cfg;
    if ((rc = check_rope_inputs(c, c.norm, q, k, pos, freq))) return rc;
    if (!dqo || !dq || (c.Hkv && (!dko || !dk)) || !aligned({dqo, dko, dq, dk, ws})) return SPARSEK_ERR_INVALID_ARG;
    if ((dqw && !c.norm) || (dkw && (!c.norm || !c.Hkv)) || ((dqw || dkw) && !ws)) return SPARSEK_ERR_INVALID_ARG;
    if (!good(c, c.dq, c.H) || !apart(c, c.dq, c.H) || (c.Hkv && (!good(c, c.dk, c.Hkv) || !apart(c, c.dk, c.Hkv)))) return SPARSEK_ERR_INVALID_ARG;
    int pairs = 1 << 18;
    if (c.Hkv && meet(Rows(c, c.dq, c.H), 0, Rows(c, c.dk, c.Hkv), 0, (const char*)dk - (const char*)dq, pairs)) return SPARSEK_ERR_INVALID_ARG;
    const size_t row = (size_t)c.B * c.n * c.d * (c.dtype == SPARSEK_BF16 ? 2 : 4), nw = (size_t)c.d * 4, need = spk::rope_bwd_ws_bytes(c);
    const bool sums = dqw || dkw;
    const Place in[] = {{q, c.norm ? span(c, c.q, c.H) : 0}, {k, c.norm && c.Hkv ? span(c, c.k, c.Hkv) : 0}, {dqo, row * c.H}, {dko, row * c.Hkv},
                        {pos, positions(c)}, {freq, c.rot * 2u}, {axis, c.rot * 2u}, {qw, c.norm ? nw : 0}, {kw, c.norm ? nw : 0}};
    const Place dx[] = {{dq, span(c, c.dq, c.H)}, {dk, c.Hkv ? span(c, c.dk, c.Hkv) : 0}}, other[] = {{dqw, nw}, {dkw, nw}, {ws, sums ? need : 0}};
    for (const Place& x : dx) {   // (which may be slices of one gradient, row beside row)
        const Place one[] = {x};
        if (any_overlap(in, one) || any_overlap(one, other)) return SPARSEK_ERR_INVALID_ARG;
    }
    if (any_overlap(in, other)) return SPARSEK_ERR_INVALID_ARG;
    if (sums && ws_bytes < need) return SPARSEK_ERR_WORKSPACE;
    return spk::launch_rope_bwd(c, q, k, pos, freq, axis, qw, kw, dqo, dko, dq, dk, dqw, dkw, ws, (hipStream_t)stream);
}

}  // extern "C"

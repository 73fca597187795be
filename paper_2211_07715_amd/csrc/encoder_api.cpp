// C-ABI layer of the operators between the linears: argument checks, then the
// launchers. No exception crosses the ABI.
#include <math.h>

#include <exception>

#include "encoder.h"

using namespace sl;

template <class F>
static sl_status guarded(F &&body)
{
    try {
        return body();
    } catch (const std::exception &ex) {
        set_error("internal error: %s", ex.what());
        return SL_ERR_HIP;
    } catch (...) {
        set_error("internal error");
        return SL_ERR_HIP;
    }
}

#define REFUSE_IF(cond, status, ...)  \
    do {                              \
        if (cond) {                   \
            set_error(__VA_ARGS__);   \
            return status;            \
        }                             \
    } while (0)

static bool good_scale(float s) { return isfinite(s) && s > 0.0f; }
static bool layout_known(int32_t l) { return l == SL_LAYOUT_ROWS || l == SL_LAYOUT_T16X32; }
static bool misaligned(const void *p, uintptr_t by) { return reinterpret_cast<uintptr_t>(p) % by != 0; }

static sl_status check_residual_norm(const sl_residual_norm_args &a)
{
    REFUSE_IF(a.rows < 0, SL_ERR_SHAPE, "rows must be >= 0");
    REFUSE_IF(a.cols < 1 || a.cols > 65535, SL_ERR_SHAPE, "cols must be 1 .. 65535");
    REFUSE_IF(a.y_type != SL_ACT_F32 && a.y_type != SL_ACT_I8, SL_ERR_INVALID_ARG, "unknown y_type %d", a.y_type);
    REFUSE_IF(a.r_type < SL_ACT_NONE || a.r_type > SL_ACT_I8, SL_ERR_INVALID_ARG, "unknown r_type %d", a.r_type);
    REFUSE_IF(a.y_type == SL_ACT_I8 && !layout_known(a.y_layout), SL_ERR_INVALID_ARG, "unknown y_layout %d", a.y_layout);
    REFUSE_IF(a.r_type == SL_ACT_I8 && !layout_known(a.r_layout), SL_ERR_INVALID_ARG, "unknown r_layout %d", a.r_layout);
    REFUSE_IF(a.q && !layout_known(a.q_layout), SL_ERR_INVALID_ARG, "unknown q_layout %d", a.q_layout);
    REFUSE_IF(a.y_type == SL_ACT_I8 && !good_scale(a.y_scale), SL_ERR_INVALID_ARG, "y_scale must be finite and > 0");
    REFUSE_IF(a.r_type == SL_ACT_I8 && !good_scale(a.r_scale), SL_ERR_INVALID_ARG, "r_scale must be finite and > 0");
    REFUSE_IF(a.q && !good_scale(a.out_scale), SL_ERR_INVALID_ARG, "out_scale must be finite and > 0");
    REFUSE_IF(!isfinite(a.residual_scale), SL_ERR_INVALID_ARG, "residual_scale must be finite");
    REFUSE_IF(!isfinite(a.eps) || a.eps < 0, SL_ERR_INVALID_ARG, "eps must be finite and >= 0");
    REFUSE_IF(a.gate_kind < SL_GATE_NONE || a.gate_kind > SL_GATE_ELEMENT, SL_ERR_INVALID_ARG, "unknown gate_kind %d",
              a.gate_kind);
    for (int32_t k : {a.post_kind, a.norm_kind})
        REFUSE_IF(k < SL_NORM_NONE || k > SL_NORM_RMS, SL_ERR_INVALID_ARG, "unknown norm kind %d", k);
    if (a.rows == 0) return SL_OK;
    REFUSE_IF(!a.h && !a.u && !a.q, SL_ERR_INVALID_ARG, "h, u and q must not all be NULL");
    REFUSE_IF(!a.y, SL_ERR_INVALID_ARG, "y must not be NULL");
    REFUSE_IF(a.r_type != SL_ACT_NONE && !a.r, SL_ERR_INVALID_ARG, "r must not be NULL");
    REFUSE_IF(a.gate_kind != SL_GATE_NONE && !a.gate, SL_ERR_INVALID_ARG, "gate must not be NULL");
    for (const void *p : {(const void *)a.gate, (const void *)a.post_gamma, (const void *)a.post_beta,
                          (const void *)a.gamma, (const void *)a.beta, (const void *)a.h, (const void *)a.u,
                          a.y_type == SL_ACT_F32 ? a.y : nullptr, a.r_type == SL_ACT_F32 ? a.r : nullptr})
        REFUSE_IF(misaligned(p, 4), SL_ERR_INVALID_ARG, "fp32 pointers must be 4-byte aligned");
    REFUSE_IF((a.y_type == SL_ACT_I8 && a.y_layout == SL_LAYOUT_T16X32 && misaligned(a.y, 16)) ||
                  (a.r_type == SL_ACT_I8 && a.r_layout == SL_LAYOUT_T16X32 && misaligned(a.r, 16)) ||
                  (a.q && a.q_layout == SL_LAYOUT_T16X32 && misaligned(a.q, 16)),
              SL_ERR_INVALID_ARG, "SL_LAYOUT_T16X32 tensors must be 16-byte aligned");
    return SL_OK;
}

// the arguments that attention_run and attention_select share
static sl_status check_attention(const sl_attention_args &a)
{
    REFUSE_IF(a.m_tokens < 0 || a.m_tokens > 0x7fffff00, SL_ERR_SHAPE, "m_tokens must be 0 .. 2^31 - 256");
    REFUSE_IF(a.n_kv_heads < 1 || a.n_heads < 1 || a.n_heads % a.n_kv_heads, SL_ERR_SHAPE,
              "n_heads must be a multiple of n_kv_heads, both >= 1");
    REFUSE_IF(a.head_dim < 16 || a.head_dim > 128 || a.head_dim % 16, SL_ERR_SHAPE,
              "head_dim must be a multiple of 16, 16 .. 128");
    REFUSE_IF(((int64_t)a.n_heads + 2 * (int64_t)a.n_kv_heads) * a.head_dim > 0x1000000, SL_ERR_SHAPE,
              "(n_heads + 2 n_kv_heads) * head_dim must be at most 2^24");
    REFUSE_IF(a.n_seq < 0 || a.max_len < 0 || a.max_len > 0x7fffff00, SL_ERR_SHAPE,
              "n_seq and max_len must be >= 0 (max_len at most 2^31 - 256)");
    REFUSE_IF(!layout_known(a.x_layout), SL_ERR_INVALID_ARG, "unknown x_layout %d", a.x_layout);
    if (a.m_tokens == 0 || a.n_seq == 0) return SL_OK;
    REFUSE_IF(!a.x || !a.seq_start, SL_ERR_INVALID_ARG, "x and seq_start must not be NULL");
    REFUSE_IF(misaligned(a.x, 16), SL_ERR_INVALID_ARG, "x must be 16-byte aligned");
    REFUSE_IF(misaligned(a.seq_start, 4) || misaligned(a.key_len, 4), SL_ERR_INVALID_ARG,
              "seq_start and key_len must be 4-byte aligned");
    return SL_OK;
}

static sl_status check_lists(const sl_attention_args &a)
{
    REFUSE_IF(a.query_block != 16 && a.query_block != 32 && a.query_block != 64 && a.query_block != 128, SL_ERR_SHAPE,
              "query_block must be 16, 32, 64 or 128");
    REFUSE_IF(a.top_k < 1, SL_ERR_SHAPE, "top_k must be >= 1");
    return SL_OK;
}

extern "C" {

sl_status residual_norm(const sl_residual_norm_args *args, void *hip_stream)
{
    clear_error();
    REFUSE_IF(!args, SL_ERR_INVALID_ARG, "args must not be NULL");
    const sl_residual_norm_args a = *args;
    const sl_status st = check_residual_norm(a);
    if (st != SL_OK || a.rows == 0) return st;
    return guarded([&] { return launch_residual_norm(a, hip_stream); });
}

sl_status attention_run(const sl_attention_args *args, void *hip_stream)
{
    clear_error();
    REFUSE_IF(!args, SL_ERR_INVALID_ARG, "args must not be NULL");
    const sl_attention_args a = *args;
    sl_status st = check_attention(a);
    if (st != SL_OK) return st;
    REFUSE_IF(a.kind != SL_EPI_F32 && a.kind != SL_EPI_I8, SL_ERR_INVALID_ARG, "kind must be SL_EPI_F32 or SL_EPI_I8");
    REFUSE_IF(!layout_known(a.y_layout), SL_ERR_INVALID_ARG, "unknown y_layout %d", a.y_layout);
    REFUSE_IF(a.y_layout == SL_LAYOUT_T16X32 && a.kind != SL_EPI_I8, SL_ERR_INVALID_ARG,
              "y_layout SL_LAYOUT_T16X32 is for SL_EPI_I8 only");
    REFUSE_IF(!good_scale(a.x_scale) || !good_scale(a.softmax_scale), SL_ERR_INVALID_ARG,
              "x_scale and softmax_scale must be finite and > 0");
    REFUSE_IF(!(a.x_scale * a.x_scale * a.softmax_scale < 1e30f), SL_ERR_INVALID_ARG,
              "x_scale^2 * softmax_scale must be below 1e30");
    REFUSE_IF(a.kind == SL_EPI_I8 && !good_scale(a.out_scale), SL_ERR_INVALID_ARG,
              "out_scale must be finite and > 0 for SL_EPI_I8");
    if (a.blocks) {
        st = check_lists(a);
        if (st != SL_OK) return st;
        REFUSE_IF(misaligned(a.blocks, 4), SL_ERR_INVALID_ARG, "blocks must be 4-byte aligned");
    }
    if (a.m_tokens == 0 || a.n_seq == 0 || a.max_len == 0) return SL_OK;
    REFUSE_IF(!a.y, SL_ERR_INVALID_ARG, "y must not be NULL");
    REFUSE_IF(misaligned(a.y, 16), SL_ERR_INVALID_ARG, "y must be 16-byte aligned");
    return guarded([&] { return launch_attention(a, hip_stream); });
}

int64_t attention_select_workspace(const sl_attention_args *args)
{
    clear_error();
    if (!args || check_attention(*args) != SL_OK) return 0;
    const int64_t bytes = pooled_slots(*args) * args->n_kv_heads * args->head_dim * 2;
    return (bytes + 15) / 16 * 16;
}

sl_status attention_select(const sl_attention_args *args, int32_t *blocks, void *workspace, int64_t workspace_bytes,
                           void *hip_stream)
{
    clear_error();
    REFUSE_IF(!args, SL_ERR_INVALID_ARG, "args must not be NULL");
    const sl_attention_args a = *args;
    sl_status st = check_attention(a);
    if (st == SL_OK) st = check_lists(a);
    if (st != SL_OK) return st;
    REFUSE_IF(a.max_len > 262144, SL_ERR_UNSUPPORTED, "max_len is over 262144");
    if (a.m_tokens == 0 || a.n_seq == 0 || a.max_len == 0) return SL_OK;
    REFUSE_IF(!blocks || misaligned(blocks, 4), SL_ERR_INVALID_ARG, "blocks must be given and 4-byte aligned");
    REFUSE_IF(workspace_bytes < pooled_slots(a) * a.n_kv_heads * a.head_dim * 2, SL_ERR_INVALID_ARG,
              "workspace_bytes is below attention_select_workspace()");
    REFUSE_IF(!workspace || misaligned(workspace, 16), SL_ERR_INVALID_ARG,
              "workspace must be given and 16-byte aligned");
    return guarded([&] { return launch_attention_select(a, blocks, workspace, hip_stream); });
}

}  // extern "C"

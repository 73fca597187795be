// Internal declarations of the operators between the linears: the residual sum
// with its norms and the attention core (gfx950). Not part of the public ABI.
#pragma once

#include "sl_internal.h"

namespace sl {

// args have been checked (encoder_api.cpp) and describe some work
sl_status launch_residual_norm(const sl_residual_norm_args &a, void *stream);
sl_status launch_attention(const sl_attention_args &a, void *stream);
sl_status launch_attention_select(const sl_attention_args &a, int32_t *blocks, void *workspace, void *stream);

// Pooled key blocks that attention_select keeps in its workspace: sequence s's
// block b has slot seq_start[s] / 64 + s + b (sequences never share one, and a
// seq_start within 0 .. m_tokens stays within this many).
inline int64_t pooled_slots(const sl_attention_args &a) { return a.m_tokens / SL_KEY_BLOCK + a.n_seq + 2; }

}  // namespace sl

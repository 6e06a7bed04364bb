// Shared by the calls that stream the LM head over tokens (entropy.hip, token_loss.hip).
#pragma once

#include "estp_common.h"

namespace estp {
namespace detail {

// Host-side checks of X [n_tok, d] and W [V, d]; `fn` names the caller in the error message.
int check_lm_head_args(const char* fn, const void* X, const void* W, int64_t n_tok, int32_t d, int32_t V, int dtype);

// The entropy kernels of one call on checked arguments; `workspace` holds
// estp_token_entropy_workspace_size() bytes, 256-byte aligned.  H, vocab_argmax
// and lse (each row's log-sum-exp in nats) may each be null.
int launch_token_entropy(const void* X, const void* W, int n, int d, int V, int dtype, float* H,
                         int32_t* vocab_argmax, float* lse, void* workspace, hipStream_t s);

}  // namespace detail
}  // namespace estp

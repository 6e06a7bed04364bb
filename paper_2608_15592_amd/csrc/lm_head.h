// Shared by the calls that stream the LM head over tokens (entropy.hip, token_loss.hip, logprobs.hip, distill.hip).
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

// What a temperature makes of a logit: its factor, and its factor in units of ln 2, each rounded once.
inline float inverse_temperature(float temperature) { return float(1.0 / double(temperature)); }
inline float base2_of_logit(float temperature) { return float(1.4426950408889634 / double(temperature)); }

// Partial (maximum, sum) states in base 2 of every token's scaled logits, state p of token i at i states + p.
struct LseStates {
  float *m, *s;
  int states;
};
// Bytes of such states (few: of a call that forms them for up to 2048 tokens of bf16 only), and the kernels that form
// them, on checked arguments, at the start of `workspace`: logits times c2 are in base 2.
size_t lse_states_bytes(int64_t n_tok, int V, int dtype, bool few);
int launch_lse_states(const char* fn, const void* X, const void* W, int n, int d, int V, int dtype, float c2,
                      void* workspace, hipStream_t s, LseStates* out);

// The teacher of a distillation: K tokens of each row with log-probabilities, and the student's of the same.
struct Distillation {
  const int32_t* ids;
  const float *logp, *logq, *grad;
  int K, renormalise;
  float temperature;
};
// Threads of a token's workgroup that forms the logits of its K entries (distill_pick_kernel): 16 waves or 4, d 2048, in us:
// 12 tokens of 16 entries 7.4 and 7.2, 200 of 16 12.5 and 14.2, 900 of 16 28 and 18, 202 of 100 27 and 68, 901 of 100 65 and
// 86; d 4096, 400 of 32 31 and 49.  A launch holds 2^22 - 1 tokens of 16 waves.
inline int pick_threads(size_t n_tok, int K) { return (n_tok <= 256 || K > 24) && fits_launch(n_tok, 1024) ? 1024 : 256; }

// Overwrites the entries of a piece of G (vocabulary rows v0 .. v0 + Vc, a row of pitch Vc for each live slot) that
// belong to tokens of the teacher's.
int launch_teacher_entries(const Distillation& t, int n, int V, int dtype, const int* slot, const int* n_live,
                           int64_t v0, int Vc, void* G, hipStream_t s);

// The gradient's kernels on checked arguments: G_iv = grad_i (exp(z_i[v] - lse_i) - [v = t_i]), or with a teacher
// grad_i exp(z_i[v] / temperature - lse_i) except where launch_teacher_entries has written.
size_t lm_head_backward_bytes(int64_t n_tok, int d, int V, int dtype, bool teacher);
int launch_lm_head_backward(const void* X, const void* W, const int32_t* targets, const float* lse, const float* grad,
                            int n, int d, int V, int dtype, const Distillation* teacher, void* dX, void* dW,
                            void* workspace, hipStream_t s);

}  // namespace detail
}  // namespace estp

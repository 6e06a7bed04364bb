// Distillation over the LM head: a student held to a teacher's top tokens, and its gradient, without the n_tok x V
// logits.
//
//   s_i = W x_i / temperature,  lse_i = log sum_v exp s_i[v],  logq_ik = s_i[id_ik] - lse_i
//   p_ik = exp(logp_ik), or the softmax of logp_i over the row's held entries
//   loss_i = sum_k p_ik (log p_ik - logq_ik)
//   G_iv = grad_i / temperature (P_i exp(s_i[v] - lse_i) - sum_{k: id_ik = v} p_ik),  P_i = sum_k p_ik
//   dX = G W,  dW = G^T X
//
// Forward: one pass over the vocabulary keeps a maximum and a sum per token (distill_lse_few_kernel of few tokens,
// distill_lse_split_kernel of fp32, else token_loss.hip's), and distill_pick_kernel forms the logits of the teacher's
// tokens from a row of W each.
//
// Backward: the gradient of the LM-head loss (token_loss.hip) with weight grad_i P_i / temperature gives G but for the
// teacher's entries.  distill_entries_kernel writes those over it, n_tok K of n_tok V, from logq, before the products
// read G: each is formed in fp32 from the whole of its terms, whatever entries of the row name the same token, and is
// rounded as the others are.
//
// A row without a held entry (an id outside [0, V), or a logp of -inf) is ignored: loss 0, no gradient, and its row
// of X is never multiplied into one.
#include <algorithm>

#include "estp_common.h"
#include "f32_split.h"
#include "few_tokens.h"
#include "lm_head.h"
#include "lse_states.h"
#include "mfma_gemm.h"

namespace estp {
namespace detail {

constexpr int kMaxTeacher = 128;  // entries of a row: two a lane

// The teacher's row of token tok, by one wave: entries lane and lane + 64.
struct TeacherRow {
  int id[2];      // -1: not held
  float p[2];     // 0 where not held
  float logp[2];  // -inf where not held
  float mass;     // sum of p
  bool live;      // some entry has weight
};
__device__ __forceinline__ TeacherRow teacher_row(const int32_t* __restrict__ ids, const float* __restrict__ logp,
                                                  int tok, int K, int V, int renormalise, int lane) {
  TeacherRow r;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int k = lane + 64 * u;
    const int id = k < K ? ids[size_t(tok) * K + k] : -1;
    const float lp = k < K ? logp[size_t(tok) * K + k] : 0.f;
    const bool held = id >= 0 && id < V;
    r.id[u] = held ? id : -1;
    r.logp[u] = held ? lp : -INFINITY;
  }
  r.live = __any(r.logp[0] != -INFINITY || r.logp[1] != -INFINITY);  // (a NaN is weight: it reaches the loss)
  if (renormalise) {
    const float most = wave_max(fmaxf(r.logp[0], r.logp[1])), ref = most == -INFINITY ? 0.f : most;
#pragma unroll
    for (int u = 0; u < 2; ++u) r.p[u] = fast_exp2((r.logp[u] - ref) * kLog2e);
    const float sum = r.live ? wave_sum(r.p[0] + r.p[1]) : 1.f, log_sum = kLn2 * fast_log2(sum);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      r.p[u] = r.p[u] / sum;
      r.logp[u] = r.logp[u] - ref - log_sum;
    }
  } else {
#pragma unroll
    for (int u = 0; u < 2; ++u) r.p[u] = fast_exp2(r.logp[u] * kLog2e);
  }
  r.mass = wave_sum(r.p[0] + r.p[1]);
  return r;
}

// Partial (maximum, sum) states in base 2 of few tokens' logits times c2, one of each workgroup.  Bound by the bytes of W:
// 12 tokens, d 2048, V 128256 (525 MB) 80 us, 6.6 TB/s; 40 tokens 91, as the products of 48 columns and their sums' way
// through LDS come between.
template <int kSteps, int kNB>
__global__ __launch_bounds__(64 * few::kWaves, 2) void distill_lse_few_kernel(const __bf16* __restrict__ X,
                                                                              const __bf16* __restrict__ W, int n,
                                                                              int d, int V, float c2,
                                                                              float* __restrict__ part_m,
                                                                              float* __restrict__ part_s) {
  __shared__ __attribute__((aligned(16))) char lds[few::Rows<kSteps, kNB>::kLds];
  float m = -INFINITY, s = 0.f;
  few::run<kSteps, kNB, 0>(X, W, n, d, V, few::tiles_of(V), lds, [&](int64_t row, f32x4_t z) {
    float mx = m, zc[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      zc[r] = row + r < V ? z[r] * c2 : -INFINITY;
      mx = fmaxf(mx, zc[r]);
    }
    const float ref = fmaxf(mx, -0x1p127f);  // finite for a thread with no live row yet
    s *= fast_exp2(fmaxf(m - ref, kExp2Floor));
#pragma unroll
    for (int r = 0; r < 4; ++r) s += row + r < V ? fast_exp2(fmaf(z[r], c2, -ref)) : 0.f;
    m = mx;
  });
  // lanes l, l ^ 16, l ^ 32, l ^ 48 hold the same tokens
#pragma unroll
  for (int o = 16; o <= 32; o <<= 1) {
    const float mo = __shfl_xor(m, o, 64), so = __shfl_xor(s, o, 64), M = fmaxf(m, mo), ref = fmaxf(M, -0x1p127f);
    s = s * fast_exp2(fmaxf(m - ref, kExp2Floor)) + so * fast_exp2(fmaxf(mo - ref, kExp2Floor));
    m = M;
  }
  const int lane = threadIdx.x & 63, tok = threadIdx.x / 64 * 16 + lane;
  if (lane < 16 && tok < min(n, 16 * kNB)) {
    part_m[size_t(tok) * gridDim.x + blockIdx.x] = m;
    part_s[size_t(tok) * gridDim.x + blockIdx.x] = s;
  }
}

// The same of fp32 logits by the bf16 matrix cores: workgroup (token tile, slice) takes the vocabulary tiles slice, slice +
// n_slices, ..., and has a state for each of its waves.  90 tokens, d 1536, V 151936: 297 us, 3.1 TB/s of W and 0.9 PFLOP/s
// of its parts' products, whose splitting the vector units do meanwhile; 504 with the fp32 instructions.
template <int kNB, bool kStream>
__global__ __launch_bounds__(64 * split::kWaves, 2) void distill_lse_split_kernel(
    const __bf16* __restrict__ parts, const float* __restrict__ W, int n, int d, int V,
    float c2, int n_tt, int n_slices, float* __restrict__ part_m, float* __restrict__ part_s) {
  using Run = split::Tile<kNB, kStream>;
  __shared__ __attribute__((aligned(16))) char lds[Run::kLds];
  const gemm::SliceAt wg = gemm::slice_of(gemm::first_tile(blockIdx.x, gridDim.x), n_tt, n_slices);
  if (wg.slice >= n_slices) return;
  const int n_vt = (V + split::kRows - 1) / split::kRows, n0 = wg.tile * Run::kTN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float m[kNB], s[kNB];
#pragma unroll
  for (int b = 0; b < kNB; ++b) {
    m[b] = -INFINITY;
    s[b] = 0.f;
  }
  Run::run(
      lds, W, V, parts, n, n, d, (n_vt - wg.slice + n_slices - 1) / n_slices,
      [&](int i) { return typename Run::Place{(wg.slice + i * n_slices) * split::kRows, n0}; },
      [&](const typename Run::Place& at, const typename Run::Acc& acc) {
        const int lim = V - (at.m0 + 32 * wave + 4 * (lane >> 4));  // live rows: 16 i + r < lim
#pragma unroll
        for (int b = 0; b < kNB; ++b) {
          float mx = m[b];
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) mx = fmaxf(mx, 16 * i + r < lim ? acc[i][b][r] * c2 : -INFINITY);
          const float ref = fmaxf(mx, -0x1p127f);  // finite for a lane with no live row yet
          float sum = s[b] * fast_exp2(fmaxf(m[b] - ref, kExp2Floor));
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += 16 * i + r < lim ? fast_exp2(fmaf(acc[i][b][r], c2, -ref)) : 0.f;
          m[b] = mx;
          s[b] = sum;
        }
      });
#pragma unroll
  for (int b = 0; b < kNB; ++b) {
    // lanes l, l ^ 16, l ^ 32, l ^ 48 hold the same tokens
#pragma unroll
    for (int o = 16; o <= 32; o <<= 1) {
      const float mo = __shfl_xor(m[b], o, 64), so = __shfl_xor(s[b], o, 64), M = fmaxf(m[b], mo);
      const float ref = fmaxf(M, -0x1p127f);
      s[b] = s[b] * fast_exp2(fmaxf(m[b] - ref, kExp2Floor)) + so * fast_exp2(fmaxf(mo - ref, kExp2Floor));
      m[b] = M;
    }
    const int tok = n0 + 16 * b + lane;
    if (lane < 16 && tok < n) {
      const size_t o = size_t(tok) * (split::kWaves * n_slices) + split::kWaves * wg.slice + wave;
      part_m[o] = m[b];
      part_s[o] = s[b];
    }
  }
}

// lse, logq and loss of a token, one workgroup each.  Its waves share the K products of a row of W with the token's row
// of X, four at a time, whose rows are far apart: the bytes of n K rows bound it where tokens are many (4096 tokens, 64
// entries, d 4096: 2.1 GB in 290 us, 7.4 TB/s), the latency of one wave's rows where they are few.
template <typename T, int kThreads>
__global__ __launch_bounds__(kThreads) void distill_pick_kernel(
    const T* __restrict__ X, const T* __restrict__ W, const int32_t* __restrict__ ids, const float* __restrict__ logp,
    int d, int V, int K, int renormalise, float inv_t, const float* __restrict__ part_m,
    const float* __restrict__ part_s, int states, float* __restrict__ lse, float* __restrict__ loss,
    float* __restrict__ logq) {
  constexpr int kWaves = kThreads / 64, kRows = 4;
  __shared__ float z[kMaxTeacher];
  const int tok = blockIdx.x, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const T* x = X + size_t(tok) * d;
  for (int k0 = wave; k0 < K; k0 += kWaves * kRows) {
    const T* w[kRows];
    float sum[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {  // (an entry that is not held takes row 0, and its product is not used)
      const int id = k0 + kWaves * u < K ? ids[size_t(tok) * K + k0 + kWaves * u] : -1;
      w[u] = W + size_t(id >= 0 && id < V ? id : 0) * d;
      sum[u] = 0.f;
    }
    for (int k = 8 * lane; k < d; k += 512)
#pragma unroll
      for (int u = 0; u < kRows; ++u) sum[u] = dot8(x + k, w[u] + k, sum[u]);
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      sum[u] = wave_sum(sum[u]);
      if (lane == 0 && k0 + kWaves * u < K) z[k0 + kWaves * u] = sum[u];
    }
  }
  __syncthreads();
  if (wave != 0) return;
  const float l = lse_of_states(part_m, part_s, tok, states, lane);
  const TeacherRow r = teacher_row(ids, logp, tok, K, V, renormalise, lane);
  float term = 0.f;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int k = lane + 64 * u;
    const float q = r.id[u] >= 0 ? fmaf(z[k & (kMaxTeacher - 1)], inv_t, -l) : 0.f;
    if (k < K) logq[size_t(tok) * K + k] = q;
    term += r.p[u] == 0.f ? 0.f : r.p[u] * (r.logp[u] - q);
  }
  term = wave_sum(term);
  if (lane == 0) {
    lse[tok] = l;
    loss[tok] = r.live ? term : 0.f;
  }
}

// What the gradient of the LM-head loss takes for a row: a target to leave out (some token of the teacher's, whose entry
// is written over anyway; -1 for an ignored row) and the weight of the softmax.  One wave per token.  Latency, 3 to 5 us.
__global__ __launch_bounds__(256) void distill_rows_kernel(const int32_t* __restrict__ ids,
                                                           const float* __restrict__ logp,
                                                           const float* __restrict__ grad, int n_tok, int V, int K,
                                                           int renormalise, float inv_t, int32_t* __restrict__ target,
                                                           float* __restrict__ weight) {
  const int tok = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (tok >= n_tok) return;
  const TeacherRow r = teacher_row(ids, logp, tok, K, V, renormalise, lane);
  int some = max(r.id[0], r.id[1]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) some = max(some, __shfl_xor(some, o, 64));
  if (lane == 0) {
    target[tok] = r.live ? some : -1;
    weight[tok] = (grad ? grad[tok] : 1.f) * inv_t * r.mass;
  }
}

// The entries of G that belong to the teacher's tokens, in vocabulary rows v0 .. v0 + Vc.  One wave per token; entries of
// a row that name the same token write the same number.  Where G has two parts, the second holds what rounding the
// first leaves.  Latency where tokens are few, 4 to 5 us; 4096 tokens of 64 entries 12 us for each of four pieces.
template <typename T>
__global__ __launch_bounds__(256) void distill_entries_kernel(
    const int32_t* __restrict__ ids, const float* __restrict__ logp, const float* __restrict__ logq,
    const float* __restrict__ grad, int n_tok, int V, int K, int renormalise, float inv_t,
    const int* __restrict__ slot, const int* __restrict__ n_live, int64_t v0, int Vc, T* __restrict__ G) {
  const int tok = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (tok >= n_tok) return;
  const int s = slot[tok];
  if (s < 0) return;
  const TeacherRow r = teacher_row(ids, logp, tok, K, V, renormalise, lane);
  float same[2] = {0.f, 0.f};  // weight of all entries that name this one's token
  for (int k = 0; k < K; ++k) {
    const int u = k >> 6;
    const int id = __builtin_amdgcn_readlane(u ? r.id[1] : r.id[0], k & 63);
    const float p = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(u ? r.p[1] : r.p[0]), k & 63));
#pragma unroll
    for (int e = 0; e < 2; ++e) same[e] += r.id[e] == id ? p : 0.f;
  }
  const float g = (grad ? grad[tok] : 1.f) * inv_t;
  const int n_tokens = n_live[0];
  const bool two = n_live[1] > n_tokens;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int64_t v = int64_t(r.id[e]) - v0;
    if (r.id[e] < 0 || v < 0 || v >= Vc) continue;
    const float q = fast_exp2(logq[size_t(tok) * K + lane + 64 * e] * kLog2e);
    const float value = g * fmaf(r.mass, q, -same[e]);
    const T first = T(value);
    G[size_t(s) * Vc + v] = first;
    if (two) G[size_t(s + n_tokens) * Vc + v] = T(value - float(first));
  }
}

int launch_teacher_entries(const Distillation& t, int n, int V, int dtype, const int* slot, const int* n_live,
                           int64_t v0, int Vc, void* G, hipStream_t s) {
  const dim3 grid(unsigned((n + 3) / 4)), block(256);
  const float inv_t = inverse_temperature(t.temperature);
  if (dtype == ESTP_F32)
    distill_entries_kernel<float><<<grid, block, 0, s>>>(t.ids, t.logp, t.logq, t.grad, n, V, t.K, t.renormalise, inv_t,
                                                         slot, n_live, v0, Vc, static_cast<float*>(G));
  else
    distill_entries_kernel<__bf16><<<grid, block, 0, s>>>(t.ids, t.logp, t.logq, t.grad, n, V, t.K, t.renormalise,
                                                          inv_t, slot, n_live, v0, Vc, static_cast<__bf16*>(G));
  ESTP_CHECK_LAUNCH("distill_entries_kernel");
  return ESTP_OK;
}

}  // namespace detail
}  // namespace estp

using namespace estp;
using namespace estp::detail;

namespace {

// Token tiles of a call by the bf16 matrix cores, and slices of the vocabulary's: up to two rounds of workgroups, as many
// as make the longest sum of a compute unit's tiles shortest, with half a tile for a workgroup's first transfers.
struct SplitStates {
  int tiles, slices;
};
SplitStates split_states(int64_t n, int V) {
  const int tile = 16 * split::blocks_of(n);
  const int64_t n_tt = (n + tile - 1) / tile, n_vt = (int64_t(V) + split::kRows - 1) / split::kRows;
  SplitStates r{int(n_tt), 1};
  int64_t least = INT64_MAX;
  for (int64_t c = std::min(n_vt, std::max<int64_t>(1, 256 / n_tt)); c <= std::min(n_vt, std::max<int64_t>(1, 512 / n_tt));
       ++c) {
    const int64_t cost = (n_tt * c + 255) / 256 * (2 * ((n_vt + c - 1) / c) + 1);
    if (cost < least) {
      least = cost;
      r.slices = int(c);
    }
  }
  return r;
}

int check_distill(const char* fn, const void* X, const void* W, const int32_t* ids, const float* logp, int64_t n_tok,
                  int32_t d, int32_t V, int32_t K, float temperature, int dtype) {
  ESTP_REQUIRE(ids && logp, ESTP_ERR_INVALID_ARG, "%s: ids and logp must be non-null", fn);
  ESTP_REQUIRE(aligned(ids, 4) && aligned(logp, 4), ESTP_ERR_INVALID_ARG, "%s: ids and logp must be 4-byte aligned", fn);
  ESTP_REQUIRE(K >= 1 && K <= kMaxTeacher, ESTP_ERR_INVALID_ARG, "%s: K must be in [1, %d], got %d", fn, kMaxTeacher, K);
  ESTP_REQUIRE(temperature >= 1e-3f && temperature <= 1e3f, ESTP_ERR_INVALID_ARG,
               "%s: temperature must be in [0.001, 1000], got %g", fn, double(temperature));
  ESTP_REQUIRE(V <= INT32_MAX - 65536, ESTP_ERR_UNSUPPORTED, "%s: V = %d, at most 2^31 - 65537", fn, V);
  const int st = check_lm_head_args(fn, X, W, n_tok, d, V, dtype);
  if (st != ESTP_OK) return st;
  ESTP_REQUIRE(n_tok <= (int64_t(1) << 22), ESTP_ERR_UNSUPPORTED, "%s: n_tok = %lld, at most 4194304", fn,
               (long long)n_tok);
  return ESTP_OK;
}

}  // namespace

extern "C" size_t estp_distill_loss_workspace_size(int64_t n_tok, int32_t d, int32_t V, int dtype) {
  if (n_tok < 1 || d < 1 || V < 1) return 0;
  Carver own(nullptr);
  if (dtype == ESTP_F32) {
    // slices n_tok is at most 512 tiles' worth, or n_tok
    for (int i = 0; i < 2; ++i)
      own.take<float>(split::kWaves * std::max<size_t>(size_t(n_tok), 512 * 96));
    own.take<__bf16>(split::parts_bytes(size_t(n_tok), d) / 2);
  } else {
    for (int i = 0; i < 2; ++i) own.take<float>(size_t(few::workgroups(few::tiles_of(V))) * size_t(std::min<int64_t>(n_tok, 64)));
  }
  return std::max(lse_states_bytes(n_tok, V, dtype, false), own.bytes());
}

extern "C" int estp_distill_loss(const void* X, const void* W, const int32_t* ids, const float* logp, int64_t n_tok,
                                 int32_t d, int32_t V, int32_t K, float temperature, int renormalise, int dtype,
                                 float* loss, float* lse, float* logq, void* workspace, size_t workspace_bytes,
                                 void* stream) {
  clear_error();
  const char* fn = "estp_distill_loss";
  ESTP_REQUIRE(loss && lse && logq, ESTP_ERR_INVALID_ARG, "%s: loss, lse and logq must be non-null", fn);
  ESTP_REQUIRE(aligned(loss, 4) && aligned(lse, 4) && aligned(logq, 4), ESTP_ERR_INVALID_ARG,
               "%s: loss, lse and logq must be 4-byte aligned", fn);
  const int st = check_distill(fn, X, W, ids, logp, n_tok, d, V, K, temperature, dtype);
  if (st != ESTP_OK) return st;
  const size_t need = estp_distill_loss_workspace_size(n_tok, d, V, dtype);
  ESTP_REQUIRE(workspace_bytes >= need, ESTP_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn,
               workspace_bytes, need);
  ESTP_REQUIRE(workspace && aligned(workspace, 256), ESTP_ERR_INVALID_ARG,
               "%s: workspace must be non-null and 256-byte aligned", fn);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int n = int(n_tok);
  LseStates p;
  if (few::takes(n, d, dtype)) {
    p.states = int(few::workgroups(few::tiles_of(V)));
    Carver c(workspace);
    p.m = c.take<float>(size_t(p.states) * size_t(n));
    p.s = c.take<float>(size_t(p.states) * size_t(n));
    few::choose(n, d, [&](auto steps, auto nb) {
      distill_lse_few_kernel<decltype(steps)::value, decltype(nb)::value>
          <<<dim3(unsigned(p.states)), dim3(64 * few::kWaves), 0, s>>>(static_cast<const __bf16*>(X),
                                                                       static_cast<const __bf16*>(W), n, d, V,
                                                                       base2_of_logit(temperature), p.m, p.s);
    });
    ESTP_CHECK_LAUNCH("distill_lse_few_kernel");
  } else if (dtype == ESTP_F32 && split::takes(n, d, V)) {
    const float *x = static_cast<const float*>(X), *w = static_cast<const float*>(W);
    const SplitStates r = split_states(n, V);
    p.states = split::kWaves * r.slices;
    Carver c(workspace);
    p.m = c.take<float>(size_t(p.states) * size_t(n));
    p.s = c.take<float>(size_t(p.states) * size_t(n));
    __bf16* parts = c.take<__bf16>(split::parts_bytes(size_t(n), d) / 2);
    split::split_rows_kernel<<<dim3(unsigned(n)), dim3(256), 0, s>>>(x, n, nullptr, d, parts);
    split::choose(n, [&](auto nb, auto stream) {
      distill_lse_split_kernel<decltype(nb)::value, decltype(stream)::value>
          <<<dim3(unsigned((r.tiles * r.slices + 7) / 8 * 8)), dim3(64 * split::kWaves), 0, s>>>(
              parts, w, n, d, V, base2_of_logit(temperature), r.tiles, r.slices, p.m, p.s);
    });
    ESTP_CHECK_LAUNCH("distill_lse_split_kernel");
  } else {
    const int rc = launch_lse_states(fn, X, W, n, d, V, dtype, base2_of_logit(temperature), workspace, s, &p);
    if (rc != ESTP_OK) return rc;
  }
  const float inv_t = inverse_temperature(temperature);
  auto go = [&](auto kernel, int threads, auto* x, auto* w) {
    kernel<<<dim3(unsigned(n)), dim3(unsigned(threads)), 0, s>>>(x, w, ids, logp, d, V, K, renormalise != 0, inv_t, p.m,
                                                                 p.s, p.states, lse, loss, logq);
  };
  const bool wide = pick_threads(size_t(n), K) == 1024;
  if (dtype == ESTP_F32) {
    const float *x = static_cast<const float*>(X), *w = static_cast<const float*>(W);
    wide ? go(distill_pick_kernel<float, 1024>, 1024, x, w) : go(distill_pick_kernel<float, 256>, 256, x, w);
  } else {
    const __bf16 *x = static_cast<const __bf16*>(X), *w = static_cast<const __bf16*>(W);
    wide ? go(distill_pick_kernel<__bf16, 1024>, 1024, x, w) : go(distill_pick_kernel<__bf16, 256>, 256, x, w);
  }
  ESTP_CHECK_LAUNCH("distill_pick_kernel");
  return ESTP_OK;
}

extern "C" size_t estp_distill_loss_backward_workspace_size(int64_t n_tok, int32_t d, int32_t V, int dtype) {
  if (n_tok < 1 || d < 1 || V < 1) return 0;
  Carver c(nullptr);
  c.take<int32_t>(size_t(n_tok));
  c.take<float>(size_t(n_tok));
  return c.bytes() + lm_head_backward_bytes(n_tok, d, V, dtype, true);
}

extern "C" int estp_distill_loss_backward(const void* X, const void* W, const int32_t* ids, const float* logp,
                                          const float* lse, const float* logq, const float* grad, int64_t n_tok,
                                          int32_t d, int32_t V, int32_t K, float temperature, int renormalise,
                                          int dtype, void* dX, void* dW, void* workspace, size_t workspace_bytes,
                                          void* stream) {
  clear_error();
  const char* fn = "estp_distill_loss_backward";
  ESTP_REQUIRE(lse && logq, ESTP_ERR_INVALID_ARG, "%s: lse and logq must be non-null", fn);
  ESTP_REQUIRE(dX || dW, ESTP_ERR_INVALID_ARG, "%s: dX and dW are both null", fn);
  ESTP_REQUIRE(aligned(lse, 4) && aligned(logq, 4) && aligned(grad, 4), ESTP_ERR_INVALID_ARG,
               "%s: lse, logq and grad must be 4-byte aligned", fn);
  ESTP_REQUIRE(aligned(dX, 16) && aligned(dW, 16), ESTP_ERR_INVALID_ARG, "%s: dX and dW must be 16-byte aligned", fn);
  const int st = check_distill(fn, X, W, ids, logp, n_tok, d, V, K, temperature, dtype);
  if (st != ESTP_OK) return st;
  ESTP_REQUIRE(d <= (1 << 20), ESTP_ERR_UNSUPPORTED, "%s: d = %d, at most 1048576", fn, d);
  ESTP_REQUIRE(n_tok * d <= (int64_t(1) << 36), ESTP_ERR_UNSUPPORTED, "%s: n_tok d = %lld, at most 2^36", fn,
               (long long)n_tok * d);
  const size_t need = estp_distill_loss_backward_workspace_size(n_tok, d, V, dtype);
  ESTP_REQUIRE(workspace_bytes >= need, ESTP_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn,
               workspace_bytes, need);
  ESTP_REQUIRE(workspace && aligned(workspace, 256), ESTP_ERR_INVALID_ARG,
               "%s: workspace must be non-null and 256-byte aligned", fn);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int n = int(n_tok);
  Carver c(workspace);
  int32_t* target = c.take<int32_t>(size_t(n));
  float* weight = c.take<float>(size_t(n));
  distill_rows_kernel<<<dim3(unsigned((n + 3) / 4)), dim3(256), 0, s>>>(
      ids, logp, grad, n, V, K, renormalise != 0, inverse_temperature(temperature), target, weight);
  ESTP_CHECK_LAUNCH("distill_rows_kernel");
  const Distillation t{ids, logp, logq, grad, K, renormalise != 0, temperature};
  return launch_lm_head_backward(X, W, target, lse, weight, n, d, V, dtype, &t, dX, dW,
                                 static_cast<char*>(workspace) + c.bytes(), s);
}

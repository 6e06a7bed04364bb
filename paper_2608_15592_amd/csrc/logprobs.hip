// Log-probabilities of given tokens under the LM head, with the entropy of their distributions and the most probable
// alternatives.
//
//   z_i = W x_i,  s_i = z_i / temperature,  lse_i = log sum_v exp s_i[v],  logprob_i = s_i[t_i] - lse_i
//   H_i = lse_i - sum_v exp(s_i[v] - lse_i) s_i[v]
//   top_i = the k largest z_i[v], descending, the lowest v first among equals
//
// The logits of a block of tokens over a piece of the vocabulary are formed by the matrix cores and kept in fp32
// (logits_mfma_kernel, logits_f32_kernel); logprob_select_kernel makes of each chunk of a row a partial state and its k
// largest logits; logprob_merge_kernel joins a row's chunks.
#include <algorithm>

#include "estp_common.h"
#include "f32_gemm.h"
#include "lm_head.h"
#include "lse_states.h"
#include "mfma_gemm.h"
#include "top_k.h"

namespace estp {
namespace detail {

// ------------------------------------------------------------------ logits

// Z[token][v] of vocabulary rows v0 .. v0 + Vc (columns past V: 0), pitch Vc.  M side: vocabulary rows.  A lane holds 8
// consecutive vocabulary rows of a token: two 16-byte stores.
template <int kNBN, bool kOdd>
__global__ __launch_bounds__(256, 1) void logits_mfma_kernel(const __bf16* __restrict__ X,
                                                             const __bf16* __restrict__ W, int n, int d, int V,
                                                             int64_t v0, int Vc, float* __restrict__ Z) {
  using Run = gemm::Tiles<true, true, true, kNBN, kOdd, 8 * kNBN < 48 ? 8 * kNBN : 48, kNBN == 4>;
  __shared__ __attribute__((aligned(16))) char lds[gemm::kSlots * gemm::kSlotBytes];
  const int rows = __builtin_amdgcn_readfirstlane(int(min(int64_t(V) - v0, int64_t(Vc))));
  const int n_m = (rows + 255) / 256, n_n = (n + Run::kBN - 1) / Run::kBN;
  const gemm::TileOrder order(n_m, n_n);
  const gemm::Operand A{reinterpret_cast<const char*>(W + size_t(v0) * d), uint32_t(d) * 2u, rows};
  const gemm::Operand B{reinterpret_cast<const char*>(X), uint32_t(d) * 2u, n};
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1;
  Run::run(
      lds, A, B, gemm::first_tile(blockIdx.x, gridDim.x), gridDim.x, n_m * n_n,
      [&](int id) {
        const gemm::TileAt t = order(id);
        return gemm::Place{256 * t.m, Run::kBN * t.n, 0, d, 0};
      },
      [&](const gemm::Place& at, const f32x4_t(&acc)[8][kNBN]) {
        const int lane = gemm::fresh_lane(), fr = lane & 15, fq = lane >> 4;
        const int live = min(Run::kBN, n - at.n0);
        const buf_rsrc_t out = make_rsrc(Z + size_t(at.n0) * Vc, uint32_t(live) * uint32_t(Vc) * 4u);
        const int c0 = at.m0 + 128 * wm + 8 * fq;
#pragma unroll
        for (int j = 0; j < kNBN; ++j) {
          const uint32_t row = uint32_t(16 * kNBN * wn + 16 * j + fr) * uint32_t(Vc);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            buf_store16(out, (row + uint32_t(c0 + 32 * (i / 2) + 4 * (i % 2))) * 4u,
                        __builtin_bit_cast(uint4, acc[i][j]));
        }
      });
}

template <int kTN>
__global__ __launch_bounds__(256, 2) void logits_f32_kernel(const float* __restrict__ X, const float* __restrict__ W,
                                                            int n, int d, int V, int64_t v0, int Vc,
                                                            float* __restrict__ Z) {
  using Run = F32Tile<true, true, kTN>;
  __shared__ __attribute__((aligned(16))) char lds[Run::kLds];
  const int n0 = blockIdx.y * kTN, m0 = blockIdx.x * kFT;
  const int rows = int(min(int64_t(V) - v0, int64_t(Vc)));
  if (m0 >= rows) return;
  const gemm::Operand A{reinterpret_cast<const char*>(W + size_t(v0) * d), uint32_t(d) * 4u, rows};
  const gemm::Operand B{reinterpret_cast<const char*>(X), uint32_t(d) * 4u, n};
  typename Run::Acc acc;
  Run::run(lds, A, B, m0, n0, 0, d, acc);
  const auto at = Run::place(m0, n0);
#pragma unroll
  for (int j = 0; j < Run::kNJ; ++j) {
    const int s = at.n + 32 * j;
    if (s >= n) continue;
#pragma unroll
    for (int i = 0; i < Run::kMI; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4_t*>(Z + size_t(s) * Vc + at.m + 32 * i + 8 * q) =
            f32x4_t{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
  }
}

// ------------------------------------------------------------------ selection

__device__ __forceinline__ float exp2_arg_floor(float x) { return x < kExp2Floor ? kExp2Floor : x; }  // (NaN stays)

// Partial state (base 2) and the k largest logits of 256 kE columns of Z's row, chunk `chunk0 + c` of the token's.
// One workgroup each.
template <int kE>
__global__ __launch_bounds__(256) void logprob_select_kernel(const float* __restrict__ Z, int Vc, int live, int64_t v0,
                                                             float c2, int k, int piece_chunks, int chunk0, int chunks,
                                                             float* __restrict__ part, uint64_t* __restrict__ top) {
  __shared__ TopK<kMaxTop * kE> pick;
  __shared__ float wave_m[4], wave_s[4], wave_t[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tok = blockIdx.x / piece_chunks, c = blockIdx.x % piece_chunks;
  const float* row = Z + size_t(tok) * Vc;
  const int first = 256 * kE * c + 4 * tid;  // columns first + 1024 u + e, ascending in 4 u + e
  f32x4_t z[kE / 4];
#pragma unroll
  for (int u = 0; u < kE / 4; ++u) z[u] = *reinterpret_cast<const f32x4_t*>(row + first + 1024 * u);
  float m = -INFINITY;
#pragma unroll
  for (int u = 0; u < kE / 4; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      z[u][e] = first + 1024 * u + e < live ? z[u][e] : -INFINITY;
      m = fmaxf(m, z[u][e]);
    }
  m = wave_max(m);
  if (lane == 0) wave_m[wave] = m;
  if (tid == 0) pick.count = 0;
  __syncthreads();
  m = fmaxf(fmaxf(wave_m[0], wave_m[1]), fmaxf(wave_m[2], wave_m[3])) * c2;
  const float ref = fmaxf(m, -0x1p127f);
  float s = 0.f, t = 0.f;
#pragma unroll
  for (int u = 0; u < kE / 4; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float dd = exp2_arg_floor(fmaf(z[u][e], c2, -ref)), p = fast_exp2(dd);
      s += p;
      t = fmaf(p, dd, t);
    }
  s = wave_sum(s);
  t = wave_sum(t);
  if (lane == 0) {
    wave_s[wave] = s;
    wave_t[wave] = t;
  }
  __syncthreads();
  const size_t at = size_t(tok) * chunks + chunk0 + c;
  if (tid == 0) {
    part[3 * at] = m;
    part[3 * at + 1] = wave_s[0] + wave_s[1] + wave_s[2] + wave_s[3];
    part[3 * at + 2] = wave_t[0] + wave_t[1] + wave_t[2] + wave_t[3];
  }
  if (k == 0) return;
  uint32_t up[kE], most = 0;
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    up[e] = first + 1024 * (e / 4) + e % 4 < live ? ascending(z[e / 4][e % 4]) : 0;
    most = max(most, up[e]);
  }
  int which = 0;
#pragma unroll
  for (int e = kE - 1; e >= 0; --e) which = up[e] == most ? e : which;  // the lowest
  auto id = [&](int e) { return int(v0) + first + 1024 * (e / 4) + e % 4; };
  const uint64_t from = pick.bound_of(most ? key_of(most, id(which)) : 0, k);
#pragma unroll
  for (int e = 0; e < kE; ++e)
    if (up[e] >= uint32_t(from >> 32) && key_of(up[e], id(e)) >= from && up[e])
      pick.list[atomicAdd(&pick.count, 1)] = key_of(up[e], id(e));
  __syncthreads();
  uint64_t* out = top + at * k;
  const int n = pick.count;
  if (tid >= n && tid < k) out[tid] = 0;  // (fewer columns than k)
  pick.rank(n, k, [&](int r, uint64_t v) { out[r] = v; });
}

// A token's outputs from its chunks.  One workgroup each.
template <typename T>
__global__ __launch_bounds__(256) void logprob_merge_kernel(const T* __restrict__ X, const T* __restrict__ W,
                                                            const int32_t* __restrict__ targets, int d, int V, int k,
                                                            float inv_t, int chunks, const float* __restrict__ part,
                                                            const uint64_t* __restrict__ top,
                                                            float* __restrict__ logprob, float* __restrict__ lse,
                                                            float* __restrict__ H, int32_t* __restrict__ top_id,
                                                            float* __restrict__ top_logprob) {
  __shared__ TopK<2048> pick;
  __shared__ uint64_t best[kMaxTop];
  __shared__ float wave_z[4];
  __shared__ Ent2 wave_state[4];
  __shared__ bool among;  // the given token is an alternative
  const int tok = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // the given token's logit
  const int t = targets ? targets[tok] : -1;
  const bool live = t >= 0 && t < V;
  float z = 0.f;
  if (live)
    for (int i = 8 * tid; i < d; i += 2048) z = dot8(X + size_t(tok) * d + i, W + size_t(t) * d + i, z);
  z = wave_sum(z);
  // the chunks' states
  Ent2 a{-INFINITY, 0.f, 0.f};
  for (int c = tid; c < chunks; c += 256) {
    const float* p = part + 3 * (size_t(tok) * chunks + c);
    a = ent2_merge(a, Ent2{p[0], p[1], p[2]});
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1)
    a = ent2_merge(a, Ent2{__shfl_xor(a.m, o, 64), __shfl_xor(a.s, o, 64), __shfl_xor(a.t, o, 64)});
  if (lane == 0) {
    wave_z[wave] = z;
    wave_state[wave] = a;
  }
  if (tid == 0) among = false;
  __syncthreads();
  z = wave_z[0] + wave_z[1] + wave_z[2] + wave_z[3];
  a = ent2_merge(ent2_merge(wave_state[0], wave_state[1]), ent2_merge(wave_state[2], wave_state[3]));
  const float l = natural_lse(a.m, a.s);
  // the k largest of the chunks' largest, as many at a time as the list takes with those so far
  if (tid < k) best[tid] = 0;
  const uint64_t* from = top + size_t(tok) * chunks * k;
  int have = 0;
  for (size_t at = 0, total = size_t(chunks) * k; at < total;) {
    const int now = int(min(total - at, size_t(2048 - have)));
    if (tid < have) pick.list[tid] = best[tid];
    for (int i = tid; i < now; i += 256) pick.list[have + i] = from[at + i];
    __syncthreads();
    pick.rank(have + now, k, [&](int r, uint64_t v) { best[r] = v; });
    __syncthreads();
    at += now;
    have = k;
  }
  if (tid < k) {
    const uint64_t key = best[tid];
    const float zk = logit_of(key);
    top_id[size_t(tok) * k + tid] = id_of(key);
    top_logprob[size_t(tok) * k + tid] = fmaf(zk, inv_t, -l);
    if (live && id_of(key) == t) {  // one value of the given token, whichever output it is read from
      wave_z[0] = zk;
      among = true;
    }
  }
  __syncthreads();
  if (tid == 0) {
    if (logprob) logprob[tok] = live ? fmaf(among ? wave_z[0] : z, inv_t, -l) : 0.f;
    if (lse) lse[tok] = l;
    if (H) H[tok] = kLn2 * (fast_log2(a.s) - a.t / a.s);
  }
}

// ------------------------------------------------------------------ plan and workspace

// A call takes its tokens in blocks of up to kBlockToks, and a block the vocabulary in pieces of Vc rows (a multiple of
// 8192), whose logits fit `room` floats.
constexpr int kBlockToks = 8192;
constexpr size_t kRoom = size_t(64) << 20;
constexpr int kChunk = 8192;  // columns of a selecting workgroup
constexpr int64_t kMaxPiece = int64_t(1) << 21;  // offsets of a tile's 256 tokens fit 32 bits

struct LogprobPlan {
  int Vc, chunks;
};
inline LogprobPlan plan_logprobs(int n, int V) {
  const int64_t v_pad = (int64_t(V) + kChunk - 1) / kChunk * kChunk;
  LogprobPlan p;
  p.Vc = int(std::min({v_pad, int64_t(kRoom / size_t(n)) / kChunk * kChunk, kMaxPiece}));
  p.chunks = int(v_pad / kChunk);
  return p;
}
struct LogprobBuffers {
  float *Z, *part;
  uint64_t* top;
  size_t bytes;
};
// At least what a call of n tokens or fewer, and of k alternatives or fewer, needs.
inline LogprobBuffers carve_logprobs(int64_t n_tok, int V, int k, void* ws) {
  const size_t n = size_t(std::min<int64_t>(n_tok, kBlockToks));
  const size_t chunks = (size_t(V) + kChunk - 1) / kChunk;
  Carver c(ws);
  LogprobBuffers b;
  b.Z = c.take<float>(std::min(n * chunks * kChunk, kRoom));
  b.part = c.take<float>(3 * n * chunks);
  b.top = c.take<uint64_t>(n * chunks * size_t(k));
  b.bytes = c.bytes();
  return b;
}

template <typename T>
int launch_logprobs(const T* X, const T* W, const int32_t* targets, int n, int d, int V, int k, float temperature,
                    const LogprobBuffers& b, float* logprob, float* lse, float* H, int32_t* top_id,
                    float* top_logprob, hipStream_t s) {
  const LogprobPlan p = plan_logprobs(n, V);
  const float c2 = base2_of_logit(temperature), inv_t = inverse_temperature(temperature);
  const dim3 block(256);
  for (int64_t v0 = 0; v0 < V; v0 += p.Vc) {
    const int rows = int(std::min<int64_t>(V - v0, p.Vc));
    if constexpr (sizeof(T) == 2) {
      const bool odd = d % 64 != 0, narrow = n <= 384;
      auto kernel = narrow ? (odd ? logits_mfma_kernel<4, true> : logits_mfma_kernel<4, false>)
                           : (odd ? logits_mfma_kernel<8, true> : logits_mfma_kernel<8, false>);
      kernel<<<dim3(256), block, 0, s>>>(X, W, n, d, V, v0, p.Vc, b.Z);
    } else {
      const int tile = n <= 32 ? 32 : n <= 64 ? 64 : kFT;
      auto kernel = tile == 32 ? logits_f32_kernel<32> : tile == 64 ? logits_f32_kernel<64> : logits_f32_kernel<kFT>;
      kernel<<<dim3(unsigned((rows + kFT - 1) / kFT), unsigned((n + tile - 1) / tile)), block, 0, s>>>(X, W, n, d, V, v0,
                                                                                                      p.Vc, b.Z);
    }
    ESTP_CHECK_LAUNCH("logits_kernel");
    const int in_piece = (rows + kChunk - 1) / kChunk;
    logprob_select_kernel<kChunk / 256><<<dim3(unsigned(n) * unsigned(in_piece)), block, 0, s>>>(
        b.Z, p.Vc, rows, v0, c2, k, in_piece, int(v0 / kChunk), p.chunks, b.part, b.top);
    ESTP_CHECK_LAUNCH("logprob_select_kernel");
  }
  logprob_merge_kernel<T><<<dim3(unsigned(n)), block, 0, s>>>(X, W, targets, d, V, k, inv_t, p.chunks, b.part, b.top,
                                                              logprob, lse, H, top_id, top_logprob);
  ESTP_CHECK_LAUNCH("logprob_merge_kernel");
  return ESTP_OK;
}

}  // namespace detail
}  // namespace estp

using namespace estp;
using namespace estp::detail;

extern "C" size_t estp_token_logprobs_workspace_size(int64_t n_tok, int32_t d, int32_t V, int32_t k, int dtype) {
  (void)dtype;
  if (n_tok < 1 || d < 1 || V < 1 || V > (1 << 24) || k < 0 || k > kMaxTop) return 0;
  return carve_logprobs(n_tok, V, k, nullptr).bytes;
}

extern "C" int estp_token_logprobs(const void* X, const void* W, const int32_t* targets, int64_t n_tok, int32_t d,
                                   int32_t V, int32_t k, float temperature, int dtype, float* logprob, float* lse,
                                   float* H, int32_t* top_id, float* top_logprob, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  clear_error();
  const char* fn = "estp_token_logprobs";
  ESTP_REQUIRE((targets != nullptr) == (logprob != nullptr), ESTP_ERR_INVALID_ARG,
               "%s: targets and logprob must be given together", fn);
  ESTP_REQUIRE(logprob || lse || H || k > 0, ESTP_ERR_INVALID_ARG, "%s: nothing to compute", fn);
  ESTP_REQUIRE(k >= 0 && k <= kMaxTop, ESTP_ERR_INVALID_ARG, "%s: k must be in [0, %d], got %d", fn, kMaxTop, k);
  ESTP_REQUIRE(k == 0 || (top_id && top_logprob), ESTP_ERR_INVALID_ARG, "%s: top_id and top_logprob must be non-null",
               fn);
  ESTP_REQUIRE(aligned(targets, 4) && aligned(logprob, 4) && aligned(lse, 4) && aligned(H, 4) && aligned(top_id, 4) &&
                   aligned(top_logprob, 4),
               ESTP_ERR_INVALID_ARG, "%s: targets and the outputs must be 4-byte aligned", fn);
  ESTP_REQUIRE(temperature >= 1e-3f && temperature <= 1e3f, ESTP_ERR_INVALID_ARG,
               "%s: temperature must be in [0.001, 1000], got %g", fn, double(temperature));
  ESTP_REQUIRE(V <= (1 << 24), ESTP_ERR_UNSUPPORTED, "%s: V = %d, at most 2^24", fn, V);
  const int st = check_lm_head_args(fn, X, W, n_tok, d, V, dtype);
  if (st != ESTP_OK) return st;
  ESTP_REQUIRE(k <= V, ESTP_ERR_INVALID_ARG, "%s: k = %d of a vocabulary of %d", fn, k, V);
  const size_t need = estp_token_logprobs_workspace_size(n_tok, d, V, k, dtype);
  ESTP_REQUIRE(workspace_bytes >= need, ESTP_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn,
               workspace_bytes, need);
  ESTP_REQUIRE(workspace && aligned(workspace, 256), ESTP_ERR_INVALID_ARG,
               "%s: workspace must be non-null and 256-byte aligned", fn);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const LogprobBuffers b = carve_logprobs(n_tok, V, k, workspace);
  for (int64_t at = 0; at < n_tok; at += kBlockToks) {
    const int n = int(std::min<int64_t>(kBlockToks, n_tok - at));
    auto go = [&](auto* x, auto* w) {
      return launch_logprobs(x + size_t(at) * d, w, targets ? targets + at : nullptr, n, d, V, k, temperature, b,
                             logprob ? logprob + at : nullptr, lse ? lse + at : nullptr, H ? H + at : nullptr,
                             top_id ? top_id + at * k : nullptr, top_logprob ? top_logprob + at * k : nullptr, s);
    };
    const int rc = dtype == ESTP_F32 ? go(static_cast<const float*>(X), static_cast<const float*>(W))
                                     : go(static_cast<const __bf16*>(X), static_cast<const __bf16*>(W));
    if (rc != ESTP_OK) return rc;
  }
  return ESTP_OK;
}

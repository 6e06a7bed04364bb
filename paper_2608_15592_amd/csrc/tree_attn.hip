// Attention of drafted tokens over a cache, and the weight each cached token
// receives from it.
//
// Sequence b holds lens[b] cached tokens in slots [0, lens[b]) of its KV heads
// and T = cu_q[b + 1] - cu_q[b] <= 64 drafted ones in the slots after them.
// Drafted row t sees every cached slot and the drafted slots whose bit its mask
// has.  Query head h reads KV head h / G, G = Hq / Hkv, so the T G rows of a KV
// head share its keys and are handled together: row r is token r / G, head
// r % G of the group.
//
//   s_rj = scale q_r . k_j,  lse_r = log sum_j exp s_rj,  O_r = sum_j exp(s_rj - lse_r) v_j
//   acc_j += sum_r w_r exp(s_rj - lse_r)
//
// A row that sees nothing has lse -inf and O 0, and adds nothing.
//
// The keys of a (sequence, KV head) are cut into n_split ranges, each the work
// of one workgroup per 16 rows, in one pass with the running maximum and sum of
// the softmax (base 2); tree_join_kernel joins the ranges' partial results.
// tree_weight_kernel then forms the scores again, per 64 keys over all rows,
// since the weights need the rows' normalisers.  No atomics: bitwise
// reproducible.
#include <algorithm>
#include <cmath>

#include "estp_common.h"

namespace estp {
namespace detail {

constexpr int kMaxTree = 64;  // drafted tokens of a sequence: the bits of a mask
constexpr int kTRows = 16;    // rows of a workgroup
constexpr int kTKeys = 64;    // keys of a tile

struct TreeShape {
  int B, n_q, Hq, Hkv, cap, max_kv, n_split;
};

// One sequence as the kernels see it: counts out of range (invalid input) never become an access out of range.
struct TreeSeq {
  int q0, T, len, keys;
};
__device__ __forceinline__ TreeSeq tree_seq(const TreeShape& sh, const int* lens, const int* cu_q, int b) {
  TreeSeq q;
  q.q0 = max(0, min(cu_q[b], sh.n_q));
  q.T = max(0, min(min(cu_q[b + 1], sh.n_q) - q.q0, kMaxTree));
  q.len = max(0, min(lens[b], sh.max_kv));
  q.keys = min(q.len + q.T, sh.max_kv);
  return q;
}
// The mask of drafted token t (row q0 + t); without masks a chain: every drafted token up to its own.
__device__ __forceinline__ uint64_t tree_bits(const int64_t* mask, int q0, int t) {
  return mask ? uint64_t(mask[q0 + t]) : (uint64_t(2) << t) - 1;
}
// Whether a row with mask `bits` sees the key `rel` places past the cached ones.
__device__ __forceinline__ bool tree_sees(uint64_t bits, int rel) {
  return rel < 0 || (rel < kMaxTree && ((bits >> (rel & 63)) & 1));
}

template <typename T>
__device__ __forceinline__ void load4(const T* p, float (&v)[4]);
template <>
__device__ __forceinline__ void load4<float>(const float* p, float (&v)[4]) {
  const f32x4_t x = *reinterpret_cast<const f32x4_t*>(p);
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = x[j];
}
template <>
__device__ __forceinline__ void load4<uint16_t>(const uint16_t* p, float (&v)[4]) {
  const uint2 x = *reinterpret_cast<const uint2*>(p);
  v[0] = __uint_as_float(x.x << 16);
  v[1] = __uint_as_float(x.x & 0xffff0000u);
  v[2] = __uint_as_float(x.y << 16);
  v[3] = __uint_as_float(x.y & 0xffff0000u);
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(uint16_t* p, float v) {
  *p = __builtin_bit_cast(uint16_t, __bf16(v));  // round to nearest even
}

// n rows of DH elements (contiguous) into LDS rows of pitch P, as floats; rows at or past `live` become 0.
template <typename T, int DH, int P>
__device__ __forceinline__ void stage_rows(const T* src, int n, int live, float* lds) {
  for (int i = threadIdx.x; i < n * (DH / 4); i += 256) {
    const int r = i / (DH / 4), c = 4 * (i % (DH / 4));
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (r < live) load4<T>(src + size_t(r) * DH + c, v);
    *reinterpret_cast<f32x4_t*>(lds + r * P + c) = f32x4_t{v[0], v[1], v[2], v[3]};
  }
}
// the 16 query rows from r0 of a KV head's T G rows
template <typename T, int DH, int P>
__device__ __forceinline__ void stage_queries(const T* Q, const TreeShape& sh, const TreeSeq& q, int g, int r0, int R,
                                              float* lds) {
  const int G = sh.Hq / sh.Hkv;
  for (int i = threadIdx.x; i < kTRows * (DH / 4); i += 256) {
    const int r = r0 + i / (DH / 4), c = 4 * (i % (DH / 4));
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (r < R) load4<T>(Q + (size_t(q.q0 + r / G) * sh.Hq + g * G + r % G) * DH + c, v);
    *reinterpret_cast<f32x4_t*>(lds + (i / (DH / 4)) * P + c) = f32x4_t{v[0], v[1], v[2], v[3]};
  }
}
// s[j] = q row rr . key 16 j + c
template <int DH, int P>
__device__ __forceinline__ void scores4(const float* qs, const float* ks, int rr, int c, float (&s)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) s[j] = 0.f;
  for (int d = 0; d < DH; d += 4) {
    const f32x4_t a = *reinterpret_cast<const f32x4_t*>(qs + rr * P + d);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4_t k = *reinterpret_cast<const f32x4_t*>(ks + (16 * j + c) * P + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[j] = fmaf(a[e], k[e], s[j]);
    }
  }
}

// Vector-unit kernel.  Thread (rr, c) = (tid / 16, tid % 16) forms row rr's scores of keys c, 16 + c, 32 + c,
// 48 + c of a tile and its output columns c DH / 16 ...
template <typename T, int DH>
__global__ __launch_bounds__(256) void tree_attn_kernel(const T* __restrict__ Q, const T* __restrict__ K,
                                                        const T* __restrict__ V, const int* __restrict__ lens,
                                                        const int* __restrict__ cu_q,
                                                        const int64_t* __restrict__ mask, TreeShape sh, float c2,
                                                        float* __restrict__ part_m, float* __restrict__ part_l,
                                                        float* __restrict__ part_o) {
  constexpr int P = DH + 4, PP = kTKeys + 4, NC = DH / 16;
  __shared__ __attribute__((aligned(16))) float qs[kTRows * P], ks[kTKeys * P], vs[kTKeys * P], ps[kTRows * PP];
  const int split = blockIdx.x % sh.n_split, bg = blockIdx.x / sh.n_split, b = bg / sh.Hkv, g = bg % sh.Hkv;
  const int G = sh.Hq / sh.Hkv, r0 = blockIdx.y * kTRows;
  const TreeSeq q = tree_seq(sh, lens, cu_q, b);
  const int R = q.T * G;
  if (r0 >= R) return;
  const int per = ((q.keys + sh.n_split - 1) / sh.n_split + kTKeys - 1) / kTKeys * kTKeys;
  const int k0 = min(q.keys, split * per), k1 = min(q.keys, k0 + per);
  const int tid = threadIdx.x, rr = tid >> 4, c = tid & 15, r = r0 + rr;
  const uint64_t bits = r < R ? tree_bits(mask, q.q0, r / G) : 0;
  const T* Kb = K + size_t(bg) * sh.cap * DH;
  const T* Vb = V + size_t(bg) * sh.cap * DH;
  stage_queries<T, DH, P>(Q, sh, q, g, r0, R, qs);
  float m = -INFINITY, l = 0.f, o[NC];
#pragma unroll
  for (int e = 0; e < NC; ++e) o[e] = 0.f;
  for (int k = k0; k < k1; k += kTKeys) {
    __syncthreads();
    stage_rows<T, DH, P>(Kb + size_t(k) * DH, kTKeys, k1 - k, ks);
    stage_rows<T, DH, P>(Vb + size_t(k) * DH, kTKeys, k1 - k, vs);
    __syncthreads();
    float s[4], mx = m;
    scores4<DH, P>(qs, ks, rr, c, s);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int key = k + 16 * j + c;
      s[j] = key < k1 && tree_sees(bits, key - q.len) ? s[j] * c2 : -INFINITY;
      mx = fmaxf(mx, s[j]);
    }
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) mx = fmaxf(mx, __shfl_xor(mx, x, 64));
    const float ref = mx == -INFINITY ? 0.f : mx;  // nothing seen yet: all weights are 0
    const float f = fast_exp2(m - ref);
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float p = fast_exp2(s[j] - ref);
      ps[rr * PP + 16 * j + c] = p;
      sum += p;
    }
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) sum += __shfl_xor(sum, x, 64);
    l = l * f + sum;
    m = mx;
#pragma unroll
    for (int e = 0; e < NC; ++e) o[e] *= f;
    __syncthreads();
    const int n = min(kTKeys, k1 - k), rel = k - q.len;
    for (int j = 0; j < n; ++j) {
      // a drafted token the row does not see adds nothing, whatever its values are
      if (rel + j >= 0 && !tree_sees(bits, rel + j)) continue;
      const float p = ps[rr * PP + j];
#pragma unroll
      for (int e = 0; e < NC; ++e) o[e] = fmaf(p, vs[j * P + c * NC + e], o[e]);
    }
  }
  if (r >= R) return;
  const size_t row = size_t(split) * sh.n_q * sh.Hq + size_t(q.q0 + r / G) * sh.Hq + g * G + r % G;
  if (c == 0) {
    part_m[row] = m;
    part_l[row] = l;
  }
#pragma unroll
  for (int e = 0; e < NC; ++e) part_o[row * DH + c * NC + e] = o[e];
}

// Joins the ranges' partial results of each row: one wave per row.  Rows past the last sequence's are left as
// they are.
template <typename T, int DH>
__global__ __launch_bounds__(256) void tree_join_kernel(const float* __restrict__ part_m,
                                                        const float* __restrict__ part_l,
                                                        const float* __restrict__ part_o,
                                                        const int* __restrict__ q_end, int n_split, int n_q, int Hq,
                                                        T* __restrict__ O, float* __restrict__ lse) {
  const int lane = threadIdx.x & 63;
  const int64_t rows = int64_t(n_q) * Hq, row = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (row >= rows || row / Hq >= q_end[0]) return;
  float M = -INFINITY;
  for (int p = lane; p < n_split; p += 64) M = fmaxf(M, part_m[p * rows + row]);
  M = wave_max(M);
  const float ref = M == -INFINITY ? 0.f : M;
  float l = 0.f, o[(DH + 63) / 64] = {};
  for (int p = 0; p < n_split; ++p) {
    const float f = fast_exp2(part_m[p * rows + row] - ref), lp = part_l[p * rows + row];
    if (lp == 0.f) continue;  // the range holds nothing the row sees
    l = fmaf(f, lp, l);
#pragma unroll
    for (int e = 0; e < (DH + 63) / 64; ++e)
      if (64 * e + lane < DH) o[e] = fmaf(f, part_o[(p * rows + row) * DH + 64 * e + lane], o[e]);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < (DH + 63) / 64; ++e)
    if (64 * e + lane < DH) store1(O + row * DH + 64 * e + lane, o[e] * inv);
  if (lane == 0) lse[(row % Hq) * n_q + row / Hq] = l == 0.f ? -INFINITY : kLn2 * (M + fast_log2(l));
}

// acc[b][g][key] += sum over the rows of w exp(s - lse): one workgroup per 64 keys of a (sequence, KV head).
template <typename T, int DH>
__global__ __launch_bounds__(256) void tree_weight_kernel(const T* __restrict__ Q, const T* __restrict__ K,
                                                          const float* __restrict__ lse, const int* __restrict__ lens,
                                                          const int* __restrict__ cu_q,
                                                          const int64_t* __restrict__ mask,
                                                          const float* __restrict__ row_weight, TreeShape sh, float c2,
                                                          float* __restrict__ acc) {
  constexpr int P = DH + 4, PP = kTKeys + 4;
  __shared__ __attribute__((aligned(16))) float qs[kTRows * P], ks[kTKeys * P], ps[kTRows * PP];
  const int bg = blockIdx.x % (sh.B * sh.Hkv), b = bg / sh.Hkv, g = bg % sh.Hkv;
  const int k = blockIdx.x / (sh.B * sh.Hkv) * kTKeys;
  const int G = sh.Hq / sh.Hkv;
  const TreeSeq q = tree_seq(sh, lens, cu_q, b);
  const int R = q.T * G, tid = threadIdx.x, rr = tid >> 4, c = tid & 15;
  if (k >= q.keys || R == 0) return;
  stage_rows<T, DH, P>(K + (size_t(bg) * sh.cap + k) * DH, kTKeys, q.keys - k, ks);
  float sum = 0.f;
  for (int r0 = 0; r0 < R; r0 += kTRows) {
    __syncthreads();
    stage_queries<T, DH, P>(Q, sh, q, g, r0, R, qs);
    __syncthreads();
    const int r = r0 + rr;
    const uint64_t bits = r < R ? tree_bits(mask, q.q0, r / G) : 0;
    const float l = r < R ? lse[size_t(g * G + r % G) * sh.n_q + q.q0 + r / G] : -INFINITY;
    const float w = r >= R ? 0.f : row_weight ? row_weight[q.q0 + r / G] : 1.f;
    float s[4];
    scores4<DH, P>(qs, ks, rr, c, s);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool sees = w != 0.f && l != -INFINITY && tree_sees(bits, k + 16 * j + c - q.len);
      ps[rr * PP + 16 * j + c] = sees ? w * fast_exp2(fmaf(s[j], c2, -l * kLog2e)) : 0.f;
    }
    __syncthreads();
    if (tid < kTKeys)
#pragma unroll
      for (int i = 0; i < kTRows; ++i) sum += ps[i * PP + tid];
  }
  if (tid < kTKeys && k + tid < q.keys) acc[size_t(bg) * sh.cap + k + tid] += sum;
}

// ------------------------------------------------------------------ plan and workspace

// Ranges of the keys of one (sequence, KV head): enough workgroups for the chip, ranges of at least 128 keys.
inline int plan_tree(int B, int max_q, int max_kv, int Hq, int Hkv) {
  const int64_t groups = int64_t(B) * Hkv * ((int64_t(max_q) * (Hq / Hkv) + kTRows - 1) / kTRows);
  const int64_t most = (int64_t(max_kv) + 127) / 128;
  return int(std::max<int64_t>(1, std::min<int64_t>(most, (1024 + groups - 1) / groups)));
}

struct TreeBuffers {
  float *m, *l, *o, *lse;
  size_t bytes;
};
inline TreeBuffers carve_tree(int n_split, int64_t n_q, int Hq, int dh, void* ws) {
  const size_t rows = size_t(n_q) * Hq;
  Carver c(ws);
  TreeBuffers t;
  t.m = c.take<float>(n_split * rows);
  t.l = c.take<float>(n_split * rows);
  t.o = c.take<float>(n_split * rows * dh);
  t.lse = c.take<float>(rows);
  t.bytes = c.bytes();
  return t;
}

int check_tree_args(const char* fn, const void* Q, const void* K, const int32_t* lens, const int32_t* cu_q, int B,
                    int max_q, int64_t n_q, int Hq, int Hkv, int64_t cap, int max_kv, int dh, float scale, int dtype) {
  ESTP_REQUIRE(Q && K && lens && cu_q, ESTP_ERR_INVALID_ARG, "%s: Q, K, lens and cu_q must be non-null", fn);
  ESTP_REQUIRE(B >= 1 && n_q >= 1 && n_q <= INT32_MAX && Hq >= 1 && Hkv >= 1, ESTP_ERR_INVALID_ARG,
               "%s: B, n_q, Hq and Hkv must be >= 1", fn);
  ESTP_REQUIRE(Hq % Hkv == 0, ESTP_ERR_INVALID_ARG, "%s: Hq = %d is not a multiple of Hkv = %d", fn, Hq, Hkv);
  ESTP_REQUIRE(max_q >= 1 && max_q <= n_q, ESTP_ERR_INVALID_ARG, "%s: max_q = %d must be in [1, n_q = %lld]", fn, max_q,
               (long long)n_q);
  ESTP_REQUIRE(cap >= 1 && cap <= INT32_MAX - 256 && max_kv >= 1 && max_kv <= cap, ESTP_ERR_INVALID_ARG,
               "%s: max_kv = %d must be in [1, cap = %lld]", fn, max_kv, (long long)cap);
  ESTP_REQUIRE(n_q <= int64_t(B) * max_q, ESTP_ERR_INVALID_ARG, "%s: n_q = %lld, more than B max_q = %lld", fn,
               (long long)n_q, (long long)B * max_q);
  ESTP_REQUIRE(std::isfinite(scale) && scale > 0.f, ESTP_ERR_INVALID_ARG, "%s: scale must be finite and > 0", fn);
  ESTP_REQUIRE(dtype == ESTP_BF16 || dtype == ESTP_F32, ESTP_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, dtype);
  ESTP_REQUIRE(aligned(Q, 16) && aligned(K, 16), ESTP_ERR_INVALID_ARG, "%s: Q and K must be 16-byte aligned", fn);
  ESTP_REQUIRE(aligned(lens, 4) && aligned(cu_q, 4), ESTP_ERR_INVALID_ARG, "%s: lens and cu_q must be 4-byte aligned",
               fn);
  ESTP_REQUIRE(dh == 32 || dh == 64 || dh == 128, ESTP_ERR_UNSUPPORTED, "%s: head_dim %d not in {32, 64, 128}", fn, dh);
  ESTP_REQUIRE(max_q <= kMaxTree, ESTP_ERR_UNSUPPORTED, "%s: max_q = %d, at most %d drafted tokens", fn, max_q, kMaxTree);
  ESTP_REQUIRE(int64_t(max_q) * (Hq / Hkv) <= 65535, ESTP_ERR_UNSUPPORTED, "%s: %d query heads share a KV head", fn,
               Hq / Hkv);
  ESTP_REQUIRE(int64_t(B) * Hkv <= INT32_MAX / 4096 && n_q * Hq <= INT32_MAX / 64, ESTP_ERR_UNSUPPORTED,
               "%s: B Hkv = %lld or n_q Hq = %lld too large", fn, (long long)B * Hkv, (long long)n_q * Hq);
  const size_t tiles = size_t(max_kv + kTKeys - 1) / kTKeys;
  ESTP_REQUIRE(fits_launch(tiles * size_t(B) * Hkv, 256), ESTP_ERR_UNSUPPORTED, "%s: B Hkv max_kv too large", fn);
  return ESTP_OK;
}

template <typename T, int DH>
int launch_tree(const T* Q, const T* K, const T* V, const int* lens, const int* cu_q, const int64_t* mask,
                const TreeShape& sh, int max_q, float scale, T* O, float* lse, const TreeBuffers& t, hipStream_t s) {
  const unsigned chunks = unsigned((max_q * (sh.Hq / sh.Hkv) + kTRows - 1) / kTRows);
  tree_attn_kernel<T, DH><<<dim3(unsigned(sh.n_split * sh.B * sh.Hkv), chunks), dim3(256), 0, s>>>(
      Q, K, V, lens, cu_q, mask, sh, scale * kLog2e, t.m, t.l, t.o);
  ESTP_CHECK_LAUNCH("tree_attn_kernel");
  tree_join_kernel<T, DH><<<dim3(unsigned((size_t(sh.n_q) * sh.Hq + 3) / 4)), dim3(256), 0, s>>>(
      t.m, t.l, t.o, cu_q + sh.B, sh.n_split, sh.n_q, sh.Hq, O, lse);
  ESTP_CHECK_LAUNCH("tree_join_kernel");
  return ESTP_OK;
}
template <typename T, int DH>
int launch_weight(const T* Q, const T* K, const float* lse, const int* lens, const int* cu_q, const int64_t* mask,
                  const float* row_weight, const TreeShape& sh, float scale, float* acc, hipStream_t s) {
  const unsigned tiles = unsigned((sh.max_kv + kTKeys - 1) / kTKeys);
  tree_weight_kernel<T, DH><<<dim3(tiles * unsigned(sh.B * sh.Hkv)), dim3(256), 0, s>>>(
      Q, K, lse, lens, cu_q, mask, row_weight, sh, scale * kLog2e, acc);
  ESTP_CHECK_LAUNCH("tree_weight_kernel");
  return ESTP_OK;
}

// f(element, head size) for the call's type and head size
template <typename F>
int tree_dispatch(int dtype, int dh, F&& f) {
  if (dtype == ESTP_F32) {
    if (dh == 32) return f(float{}, std::integral_constant<int, 32>{});
    if (dh == 64) return f(float{}, std::integral_constant<int, 64>{});
    return f(float{}, std::integral_constant<int, 128>{});
  }
  if (dh == 32) return f(uint16_t{}, std::integral_constant<int, 32>{});
  if (dh == 64) return f(uint16_t{}, std::integral_constant<int, 64>{});
  return f(uint16_t{}, std::integral_constant<int, 128>{});
}

}  // namespace detail
}  // namespace estp

using namespace estp;
using namespace estp::detail;

extern "C" size_t estp_tree_attention_workspace_size(int32_t B, int32_t max_q, int64_t n_q, int32_t Hq, int32_t Hkv,
                                                     int32_t max_kv, int32_t dh, int dtype) {
  (void)dtype;
  if (B < 1 || max_q < 1 || n_q < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || max_kv < 1 || dh < 1) return 0;
  return carve_tree(plan_tree(B, max_q, max_kv, Hq, Hkv), n_q, Hq, dh, nullptr).bytes;
}

extern "C" int estp_tree_attention(const void* Q, const void* K, const void* V, const int32_t* lens,
                                   const int32_t* cu_q, const int64_t* tree_mask, int32_t B, int32_t max_q,
                                   int64_t n_q, int32_t Hq, int32_t Hkv, int64_t cap, int32_t max_kv, int32_t dh,
                                   float scale, int dtype, void* O, float* lse, float* acc, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  clear_error();
  const char* fn = "estp_tree_attention";
  const int st = check_tree_args(fn, Q, K, lens, cu_q, B, max_q, n_q, Hq, Hkv, cap, max_kv, dh, scale, dtype);
  if (st != ESTP_OK) return st;
  ESTP_REQUIRE(V && O, ESTP_ERR_INVALID_ARG, "%s: V and O must be non-null", fn);
  ESTP_REQUIRE(aligned(V, 16) && aligned(O, 16) && aligned(tree_mask, 8) && aligned(lse, 4) && aligned(acc, 4),
               ESTP_ERR_INVALID_ARG, "%s: V and O must be 16-byte, tree_mask 8-byte, lse and acc 4-byte aligned", fn);
  const size_t need = estp_tree_attention_workspace_size(B, max_q, n_q, Hq, Hkv, max_kv, dh, dtype);
  ESTP_REQUIRE(workspace_bytes >= need, ESTP_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn,
               workspace_bytes, need);
  ESTP_REQUIRE(workspace && aligned(workspace, 256), ESTP_ERR_INVALID_ARG,
               "%s: workspace must be non-null and 256-byte aligned", fn);
  const TreeShape sh{B, int(n_q), Hq, Hkv, int(cap), max_kv, plan_tree(B, max_q, max_kv, Hq, Hkv)};
  const TreeBuffers t = carve_tree(sh.n_split, n_q, Hq, dh, workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  float* row_lse = lse ? lse : t.lse;
  return tree_dispatch(dtype, dh, [&](auto element, auto size) {
    using T = decltype(element);
    constexpr int DH = decltype(size)::value;
    const int rc = launch_tree<T, DH>(static_cast<const T*>(Q), static_cast<const T*>(K), static_cast<const T*>(V),
                                      lens, cu_q, tree_mask, sh, max_q, scale, static_cast<T*>(O), row_lse, t, s);
    if (rc != ESTP_OK || !acc) return rc;
    return launch_weight<T, DH>(static_cast<const T*>(Q), static_cast<const T*>(K), row_lse, lens, cu_q, tree_mask,
                                nullptr, sh, scale, acc, s);
  });
}

extern "C" int estp_tree_importance(const void* Q, const void* K, const float* lse, const int32_t* lens,
                                    const int32_t* cu_q, const int64_t* tree_mask, const float* row_weight, int32_t B,
                                    int32_t max_q, int64_t n_q, int32_t Hq, int32_t Hkv, int64_t cap, int32_t max_kv,
                                    int32_t dh, float scale, int dtype, float* acc, void* stream) {
  clear_error();
  const char* fn = "estp_tree_importance";
  const int st = check_tree_args(fn, Q, K, lens, cu_q, B, max_q, n_q, Hq, Hkv, cap, max_kv, dh, scale, dtype);
  if (st != ESTP_OK) return st;
  ESTP_REQUIRE(lse && acc, ESTP_ERR_INVALID_ARG, "%s: lse and acc must be non-null", fn);
  ESTP_REQUIRE(aligned(tree_mask, 8) && aligned(lse, 4) && aligned(acc, 4) && aligned(row_weight, 4),
               ESTP_ERR_INVALID_ARG, "%s: tree_mask must be 8-byte, lse, row_weight and acc 4-byte aligned", fn);
  const TreeShape sh{B, int(n_q), Hq, Hkv, int(cap), max_kv, 1};
  return tree_dispatch(dtype, dh, [&](auto element, auto size) {
    using T = decltype(element);
    return launch_weight<T, decltype(size)::value>(static_cast<const T*>(Q), static_cast<const T*>(K), lse, lens, cu_q,
                                                   tree_mask, row_weight, sh, scale, acc,
                                                   static_cast<hipStream_t>(stream));
  });
}

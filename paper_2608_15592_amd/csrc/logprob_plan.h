// How a call of estp_token_logprobs is cut, and its workspace (logprobs.hip).
#pragma once

#include <algorithm>

#include "estp_common.h"
#include "f32_split.h"

namespace estp {
namespace detail {

// Logits that reach a bound, of the vocabulary tiles outside of the sample: tile (token tile, place) is [256 tokens][256
// rows], of which the quads are written whose bits are set.
struct Quads {
  float* z;
  uint32_t* bits;  // [token][2 place + half of 128 rows]: bit 8 q + i is quad 4 i + q of the half
};
constexpr int kQuadTile = 256 * 256;

// Few tokens, and fp32: the logits of a block of up to kBlockToks tokens over pieces of Vc vocabulary rows (a multiple of
// kChunk) that fit kRoom floats.
constexpr int kBlockToks = 8192;
constexpr size_t kRoom = size_t(64) << 20;
constexpr int kChunk = 8192;  // columns of a selecting workgroup
constexpr int64_t kMaxPiece = int64_t(1) << 21;  // offsets of a tile's 256 tokens fit 32 bits
struct PiecePlan {
  int Vc, chunks;
};
inline PiecePlan plan_pieces(int n, int V) {
  const int64_t v_pad = (int64_t(V) + kChunk - 1) / kChunk * kChunk;
  PiecePlan p;
  p.Vc = int(std::min({v_pad, int64_t(kRoom / size_t(n)) / kChunk * kChunk, kMaxPiece}));
  p.chunks = int(v_pad / kChunk);
  return p;
}

// Many tokens of bf16: blocks of up to kQuadToks tokens, a sample of `sample` vocabulary tiles (every `step`-th) and
// `slices` slices of the others.
constexpr int kQuadToks = 2048;
constexpr int kSampleTiles = 40, kLeastSample = 24;  // a sample is one chunk of kSampleTiles tiles
struct QuadPlan {
  int sample, step, n_main, slices;
};
// Rounds of workgroups times tiles of a workgroup, of the sample and of the rest, with half a tile for a workgroup's
// first transfers: the least over the sizes of the sample and the slices.
inline QuadPlan plan_quads(int n, int V, int k) {
  const int n_vt = (V + 255) / 256, n_tt = (n + 255) / 256;
  QuadPlan best{};
  int64_t least = INT64_MAX;
  const int first = k > 0 ? (n_vt + kSampleTiles - 1) / kSampleTiles : 0, last = k > 0 ? n_vt / kLeastSample : 0;
  for (int step = first; step <= last; step += std::max(1, (last - first) / 16)) {
    QuadPlan p;
    p.step = step;
    p.sample = step ? (n_vt + step - 1) / step : 0;
    p.n_main = n_vt - p.sample;
    const int fewest = std::min(p.n_main, std::max(1, 256 / n_tt)), most = std::min(p.n_main, std::max(1, 512 / n_tt));
    for (p.slices = fewest; p.slices <= most; ++p.slices) {
      const int64_t cost = 2 * ((int64_t(n_tt) * p.sample + 255) / 256) +
                           (int64_t(n_tt) * p.slices + 255) / 256 * (2 * ((p.n_main + p.slices - 1) / p.slices) + 1);
      if (cost < least) {
        least = cost;
        best = p;
      }
    }
  }
  return best;
}
// By quads and by pieces, us, 20 alternatives: d 2048, V 128256, 256 tokens 247 and 236, 385 tokens 312 and 311, 500 tokens
// 321 and 367, with 128 alternatives 407 and 397, 1000 tokens of 128 604 and 894; d 1024, V 33000, 400 tokens 96 and 86, 800
// tokens 132 and 132, 2000 tokens 208 and 273.  (A smaller vocabulary has no sample of its own size to leave out; of a
// larger one the room for 2048 tokens' logits would pass 8.6 GB.)
inline bool use_quads(int64_t n_tok, int V, int dtype) {
  return dtype == ESTP_BF16 && n_tok > 384 && V >= 256 * 128 && V <= (1 << 20);
}

struct LogprobBuffers {
  float *Z, *part;
  uint64_t* top;
  __bf16* parts;  // of fp32 tokens
  Quads quads;
};
// Room of one form: logits, partial states, keys, words of bits and tiles of quads.
struct LogprobRoom {
  size_t Z, states, keys, words, tiles, parts;
};
inline size_t carve_logprobs(const LogprobRoom& r, void* ws, LogprobBuffers* b) {
  Carver c(ws);
  b->Z = c.take<float>(r.Z);
  b->part = c.take<float>(3 * r.states);
  b->top = c.take<uint64_t>(r.keys);
  b->parts = c.take<__bf16>(r.parts / 2);
  b->quads.bits = c.take<uint32_t>(r.words);
  b->quads.z = c.take<float>(r.tiles * kQuadTile);
  return c.bytes();
}
inline LogprobRoom piece_room(int64_t n, int d, int V, int k, int dtype) {
  const size_t toks = size_t(n), chunks = (size_t(V) + kChunk - 1) / kChunk;
  return {std::min(toks * chunks * kChunk, kRoom), toks * chunks, toks * chunks * size_t(k), 0, 0,
          dtype == ESTP_F32 ? split::parts_bytes(toks, d) : 0};
}
inline LogprobRoom quad_room(int n, const QuadPlan& p, int k) {
  const size_t toks = size_t(n), n_tt = (toks + 255) / 256, main = k > 0 ? size_t(p.n_main) : 0;
  return {k > 0 ? toks * 256 * kSampleTiles : 0, toks * size_t((k > 0) + 2 * p.slices), toks * size_t(k),
          n_tt * 256 * 2 * main, n_tt * main, 0};
}
// The most that a block of up to n tokens takes, in either form.
inline size_t logprob_bytes(int64_t n_tok, int d, int V, int k, int dtype) {
  LogprobBuffers b;
  const int64_t listed = std::min<int64_t>(use_quads(n_tok, V, dtype) ? 384 : n_tok, kBlockToks);
  size_t most = carve_logprobs(piece_room(listed, d, V, k, dtype), nullptr, &b);
  if (use_quads(n_tok, V, dtype)) {
    // slices: up to 512 tiles of workgroups
    const size_t toks = size_t(std::min<int64_t>(n_tok, kQuadToks)), n_tt = (toks + 255) / 256;
    const size_t main = k > 0 ? (size_t(V) + 255) / 256 : 0;
    most = std::max(most, carve_logprobs({toks * 256 * kSampleTiles, toks + 2 * 512 * 256, toks * size_t(k),
                                          n_tt * 256 * 2 * main, n_tt * main, 0}, nullptr, &b));
  }
  return most;
}

}  // namespace detail
}  // namespace estp

// Internal interface between the C-ABI layer (opd_api.cpp) and the kernels around
// the rows of logits: token embeddings, adapters, beams.  Not installed.
#pragma once

#include "opd_internal.h"

namespace opd {

// Token embeddings (opd_embed_tokens, opd_embed_grads).  Launches go over rows (tokens,
// entries, tiles) times chunks of columns.
constexpr int kEmbTile = 16;   // sorted tokens of a tile (a lane each: no more than 64)
constexpr int kEmbKeys = 512;  // entries that a workgroup sorts, at most
struct EmbedArgs {
  const void* table;      // [V, ld]
  int64_t V, H, ld;
  const int32_t* ids;     // [N]
  int64_t N;
  float scale;
  void* out;              // [N, ldo]
  int64_t ldo;
  int64_t row0;           // (the launch sets these)
  uint32_t units, chunks;
};
struct EmbedGradArgs {
  const void* dy;         // [N, ldy]
  int64_t V, H, ldy;
  const int32_t* ids;     // [N]
  int64_t N;
  float scale;
  int accumulate;
  void* out;              // [V, ldo]
  int64_t ldo;
  int keys;               // entries that a workgroup sorts
  int32_t* start;         // [V + 1]; NULL: tokens are not sorted (few)
  int32_t* perm;          // [N]
  float* partial;         // [ceil(N / kEmbTile), 2, hp]
  int64_t hp;
  int64_t tiles;          // of sorted tokens (the launch sets these)
  int64_t row0;
  uint32_t units, chunks;
};
hipError_t launch_embed(const EmbedArgs& a, int in_dt, int out_dt, hipStream_t stream);
hipError_t launch_embed_grad(const EmbedGradArgs& a, int in_dt, int out_dt, hipStream_t stream);

// Low-rank adapters (opd_add_adapters, opd_adapter_grads).
constexpr int kAdTile = 64;  // tokens of one adapter in a tile, at most
constexpr int kAdFew = 64;  // tokens that the first product groups itself
struct AdTile {
  int32_t key, pos, count, unused;  // adapter (G: none, G + 1: bad id), place of its first token
};
struct AdaptArgs {
  const int32_t* ids;     // [N]
  int64_t N;
  int G;
  int32_t* perm;          // [N] tokens by adapter
  int32_t* start;         // [G + 3] first places; nullable
  AdTile* tiles;          // [max_tiles]
  int64_t max_tiles;
};
// tokens times the rows of an adapter: out[n, 0 .. r)
struct LowArgs {
  AdTile* tiles;
  int32_t* perm;
  int64_t max_tiles;
  int G, r;
  const void* x;          // [N, ldx]
  const void* w;          // [G, r, ldw]
  int64_t ldx, ldw, D;
  int splits;             // parts of the long axis, of `span` columns, `stride` floats apart
  int64_t span, stride;
  float* out;             // [splits][N, ldo]
  int64_t ldo;
  const int32_t* ids;     // [N] nullable: the tiles are made here, from kAdFew tokens at most
  int N;
};
struct LowPair {
  LowArgs a[2];           // of one plan; the second with no splits: there is none
};
// what they are, to the kernels that read them
struct LowRef {
  const float* p;
  int64_t ld, stride;
  int splits, r;
};
// out = base + scale * low * w
struct ExpandArgs {
  const AdTile* tiles;
  const int32_t* perm;
  int64_t max_tiles;
  int G, r;
  LowRef low;
  const float* scales;    // [G] nullable
  const void* w;          // [G, r, ldw]
  int64_t ldw, D;
  const void* base;       // [N, ldb] nullable
  int64_t ldb;
  void* out;              // [N, ldo]
  int64_t ldo;
  float* low_out;         // [N, r] nullable
  uint32_t per;           // workgroups to a tile (the launch sets it)
};
// out[g] = scale * sum over the adapter's tokens of low^T x (low: one part)
struct OuterArgs {
  const int32_t* perm;
  const int32_t* start;
  int G, r;
  LowRef low;
  const float* scales;
  const void* x;          // [N, ldx]
  int64_t ldx, D;
  int splits;             // parts of the tokens, `stride` floats apart
  int64_t stride;
  float* out;             // [splits][G, r, ldo]
  int64_t ldo;
  float* sum;             // [G, r, lds] the result
  int64_t lds;
  uint32_t chunks;        // of columns (the launch sets it)
};
struct OuterPair {
  OuterArgs a[2];         // da, db
  uint32_t blocks;        // of the first (the launch sets it)
};
hipError_t launch_adapt_plan(const AdaptArgs& a, hipStream_t stream);
hipError_t launch_low(const LowPair& pair, int x_dt, int w_dt, hipStream_t stream);
// adds the parts up in the first one's place, for N tokens
hipError_t launch_low_sum(const LowPair& pair, int64_t N, hipStream_t stream);
hipError_t launch_expand(const ExpandArgs& a, int64_t N, int w_dt, int y_dt, hipStream_t stream);
hipError_t launch_outer(const OuterPair& pair, int x_dt, int y_dt, hipStream_t stream);

// Beam selection and reordering (opd_beam_select, opd_reorder_beams).
constexpr int kBeamMax = 64;
struct BeamRec {
  double s;               // sum of exp(z - m)
  float m;
  uint32_t n;             // candidates
};
struct BeamArgs {
  const void* logits;     // [B W, ld]
  int64_t B, V, ld;
  int W, k;
  const float* scores;    // [B, W]
  const uint8_t* finished;  // [B, W] nullable
  int slots;              // vectors of 16 bytes per lane: a part is 256 times that
  uint32_t parts;         // of a row
  void* recs;             // [B W, parts] BeamRec
  uint64_t* cands;        // [B W, parts, kBeamMax] (order key of the logit, ~token)
  float* out_scores;      // [B, k]
  int32_t* parents;
  int32_t* ids;
  int64_t row0;           // (the launch sets it)
};
struct ReorderArgs {
  const void* states;     // [B W] states of `outer` slices of `inner` bytes
  int64_t B;
  int W, k;
  int64_t outer, inner, stride, outer_stride;  // bytes
  const int32_t* parents; // [B, k]
  void* out;              // [B k]
  int64_t out_stride, out_outer_stride;
  int in_place;
  int64_t item0, span0;   // (the launch sets these)
  uint32_t spans;
};
hipError_t launch_beam(const BeamArgs& a, int in_dt, hipStream_t stream);
// states lie at any address and stride: 16 bytes at a time, or 4 where there are many beams
hipError_t launch_reorder(const ReorderArgs& a, hipStream_t stream);

}  // namespace opd

// Host-side planning of the gradient operators: workspace regions, the tables that the launches take, and how work is shared
// out.  Plain C++ (no HIP), so that it is compiled by itself in the sanitized build and in the CPU tests.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "iso.h"
#include "iso_workspace.h"

namespace iso {

// ---- embedding lookup ----------------------------------------------------------------------------------------------

// Whether one workgroup looks at all ids, under the copies of the others; where its walk (0.65 us for 1024 ids) outlasts them, a
// launch before clears the status word and every workgroup looks at its own.  Microseconds on the GPU, alone against that
// launch, bf16 rows of a table of about 152000 (fp32 rows of the same bytes take about the same; a table of 32000 too):
//   columns      4096 tokens      6000      8192        16384       32768
//        64      4.2  4.6           -     6.7  4.6   11.8  4.7   22.2  5.2
//      1024      5.2  6.0    6.9  7.2    10.3  8.0   23.3 12.3   42.3 17.7
//      2048      6.4  8.0    8.8 10.1    12.9 12.3   20.6 18.8   45.4 33.2
//      2560      7.9  9.4   10.4 11.7    10.5 11.8   22.9 22.8   49.0 41.0
//      3584      9.9 11.4   10.8 12.3    15.6 17.1   29.0 30.6   54.4 55.8
inline bool lookup_checks_alone(int64_t tokens, int64_t row_bytes) { return tokens <= (row_bytes > 4096 ? 16384 : 6144); }

// ---- embedding gradient --------------------------------------------------------------------------------------------

// The tokens of an id are added in runs of kRun, whose sums are then added in order.
constexpr int kRun = 32;

// Tokens of the gradient's single launch: as many as its workgroups hold (eight ids a thread, two bytes of LDS a token).
// Microseconds on the GPU, the single launch against the sorted ones, bf16 rows added to fp32:
//   table, ids                          256 tokens       1024          2048          4096
//   1031 x 256, by frequency             6.9  17.5     9.8  24.4    11.3  25.7    16.4  27.2
//   151936 x 1536, by frequency          9.5  18.2    12.7  26.5    16.2  29.4    20.6  32.9
//   151936 x 1536, evenly                9.9  17.4    13.7  21.6    18.0  27.2    24.5  30.5
//   152064 x 3584, by frequency         16.2  17.9    23.3  29.2    30.6  33.9    41.1  40.3
//   152064 x 3584, evenly               17.2  18.5    25.8  26.9    33.3  31.9    43.9  43.2
//   151936 x 1536, all the same         10.3  20.2    26.3  24.3    47.6  30.5    98.5  41.2
// It is ahead over its whole range but for the widest rows (level from 2048 on) and for batches of one id from 1024 on, whose
// tokens one workgroup a column block adds: which ids there are is not known on the host.
constexpr int kFewTokens = 4096;

constexpr int kMaxTiles = 64;
constexpr int kMinTile = 1024;
constexpr int kMaxBuckets = 512;

// Counters of the lists of distinct ids: groups of buckets, and words between their counters.
constexpr int kGroups = 16;
constexpr int kLine = 32;

// Workspace regions of the embedding's gradient (many tokens; few take the status block alone).
struct EmbedPlan {
  int64_t tiles = 0, tile = 0;     // tokens are counted and scattered by tiles of `tile`
  int64_t most_runs = 0;           // partial sums of ids with many tokens
  size_t bad = 0, hist = 0, bucket0 = 0, pairs = 0, perm = 0, listed = 0, ids = 0, runs = 0, many = 0, part = 0, total = 0;
};

int log2_up(int64_t n);
EmbedPlan embed_plan(int64_t tokens, int64_t vocab, int64_t dim);

// ---- checkpoints ---------------------------------------------------------------------------------------------------

inline int64_t ckpt_ld(int64_t cols) { return (cols + ISO_CKPT_GROUP - 1) / ISO_CKPT_GROUP * ISO_CKPT_GROUP; }

constexpr int kTable = 16;     // tensors a launch

// Cuts n entries, in the form that the kernel takes (`arg`), into tables of up to 16 tensors and 2^22 workgroups (a larger
// tensor goes alone), and hands each to `launch`, with its workgroups and the bytes that they write.  `items`: groups of eight
// columns a thread, 256 threads a workgroup; `size`: bytes written for such a group.
template <class Table, class Entry, class Arg, class Launch>
void for_tables(const Entry* c, int n, int items, int size, Arg arg, Launch launch) {
  Table T;
  int64_t bytes = 0;
  T.n = 0;
  T.block0[0] = 0;
  auto flush = [&] {
    if (T.n > 0) launch(T, T.block0[T.n], bytes);
    T.n = 0;
    bytes = 0;
  };
  for (int j = 0; j < n; ++j) {
    const auto a = arg(c[j]);
    if (a.rows == 0 || a.cols == 0) continue;
    const int64_t blocks = (a.rows * a.per_row + 256 * items - 1) / (256 * items);
    if (T.n == kTable || (T.n > 0 && T.block0[T.n] + blocks > (1 << 22))) flush();
    T.t[T.n] = a;
    T.block0[T.n + 1] = T.block0[T.n] + (uint32_t)blocks;
    bytes += a.rows * a.per_row * size;
    ++T.n;
  }
  flush();
}

// ---- weight gradients ----------------------------------------------------------------------------------------------

constexpr int kLayers = 16;               // layers a launch
constexpr int kStep = 32;                 // tokens of a step
constexpr int64_t kMaxStride = 1 << 25;   // 32 rows of it stay within 32-bit offsets

struct Prep {
  const void* src;        // q, or dY
  const uint8_t* e;       // exponents of q; null for dY
  uint16_t* dst;
  int64_t rows, ld;       // rows and row stride of the source
  int64_t part;           // rows of a part of the destination (rows rounded up to whole steps); 0 for X
  uint32_t cols, per_row; // columns of the source; groups of eight in a destination row
  uint32_t block0;
};

struct PrepTable {
  Prep p[2 * kLayers];
  int n;
  uint32_t blocks;
  uint32_t* status;
};

struct Layer {
  const uint8_t* y;            // bf16 dY and X, token rows
  const uint8_t* x;
  void* g;
  int64_t y_ld, x_ld;          // row strides, bytes
  int64_t y_bytes, x_bytes;    // bytes from the first element to past the last (dY: of all its parts)
  int32_t rows, cols;          // of G
  int32_t across, down;        // tiles of a tile row, and tile rows
  int32_t steps, parts;        // steps of a part of dY
  uint32_t tile0;
};

struct LayerTable {
  Layer l[kLayers];
  int n;
  uint32_t tiles;     // of all layers
  uint32_t whole;     // tiles one workgroup does alone; the others' tokens are split `split` ways
  uint32_t split;
  float* part;        // their partial sums, a tile's size a piece, (tile, piece) in order
};

// What up to 16 layers take: the tables of their launches, with workspace offsets in place of pointers until bound.
struct WeightGradPlan {
  PrepTable prep{};
  LayerTable layers{};
  int tile = 256;
  size_t total = 0;
};

// How many of the first n layers (at most kLayers) go into one launch: those before the first whose gradient shares memory with
// an earlier one's.  Tiles of one launch run in any order, two that add to the same element would lose one of the sums.
int weight_grad_group(const iso_weight_grad* g, int n, int dt_grad);

// `ws` may be null where only sizes matter.
WeightGradPlan plan_weight_grad(const iso_weight_grad* g, int n, int dt, bool accumulate, uint8_t* ws);
size_t weight_grad_workspace_bytes(const iso_weight_grad* g, int n, int dt);

// ---- attention -----------------------------------------------------------------------------------------------------

// Whether the rows of a call and its launches stay within 32 bits.
bool attend_fits(const iso_attn& a);

constexpr int kAttnTileRows = 128;     // rows (queries times the group) or keys of a tile
constexpr int kPartLd = 132;           // floats of a row's piece: its sums, maximum and sum of weights

// How the keys (or rows) that a tile walks over are shared out: `most` pieces, each of at least `keys`.
struct Pieces {
  int32_t most = 1, keys = 1;
};

// Pieces of tiles of `rows` rows in `sequences` sequences that walk over `list` keys (or the other way round) at most, a head.
uint32_t attend_items(int64_t rows, int64_t list, int64_t sequences, const Pieces& p);

struct AttendPlan {
  Pieces rows, keys;   // of tiles of rows (O, dQ) and of keys (dK and dV)
  size_t part = 0, key_part = 0, total = 0;
};
AttendPlan plan_attend(const iso_attn& a, bool grad);
size_t attend_workspace_bytes(const iso_attn& a, int dt, bool grad);

// ---- distillation --------------------------------------------------------------------------------------------------

constexpr int64_t kMostPieces = 4096;   // of all rows of a call whose rows are shared out
inline size_t distill_workspace_bytes() { return kStatusBytes + kMostPieces * 2 * sizeof(float); }

}  // namespace iso

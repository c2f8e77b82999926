// Host-side planning of the gradient operators (iso_grad_plan.h).
#include "iso_grad_plan.h"

#include <algorithm>
#include <cmath>

namespace iso {

int log2_up(int64_t n) {
  int b = 0;
  while ((1ll << b) < n) ++b;
  return b;
}

EmbedPlan embed_plan(int64_t tokens, int64_t vocab, int64_t dim) {
  EmbedPlan P;
  P.total = kStatusBytes;
  if (tokens <= kFewTokens) return P;
  const size_t buckets = (size_t)1 << std::min(9, log2_up(vocab));
  P.tile = std::max<int64_t>(kMinTile, (tokens + kMaxTiles - 1) / kMaxTiles);
  P.tiles = (tokens + P.tile - 1) / P.tile;
  P.most_runs = tokens / (kRun / 2) + 1;   // an id with m > kRun tokens has ceil(m / kRun) <= m / (kRun / 2)
  auto region = [&](size_t bytes) {
    const size_t o = P.total;
    P.total = align_up(P.total + bytes, 256);
    return o;
  };
  P.bad = region(sizeof(uint32_t) * P.tiles);
  P.hist = region(sizeof(uint32_t) * P.tiles * buckets);
  P.bucket0 = region(sizeof(uint32_t) * (buckets + 1));
  P.pairs = region(2 * sizeof(uint32_t) * tokens);
  P.perm = region(sizeof(uint32_t) * tokens);
  P.listed = region(sizeof(uint32_t) * kLine * (kGroups + 1));
  P.ids = region(4 * sizeof(uint32_t) * tokens);
  P.runs = region(2 * sizeof(uint32_t) * P.most_runs);
  P.many = region(4 * sizeof(uint32_t) * (tokens / kRun + 1));
  P.part = region(sizeof(float) * P.most_runs * dim);
  return P;
}

namespace {

bool direct(const iso_weight_grad& x, int dt) { return dt == ISO_BF16 && x.ld_dy % 8 == 0 && x.ld_dy <= kMaxStride; }

int64_t whole_steps(int64_t tokens) { return (tokens + kStep - 1) / kStep * kStep; }

// How the tiles of a table, of `side` x `side`, are shared out: full rounds of workgroups take whole tiles, those past the
// last full round are split into the pieces that take the fewest microseconds, by an estimate from measured parts: a step,
// which takes longer the more workgroups are at work (memory, clock); a workgroup's start and end; for split tiles the second
// launch, the pieces' writes and reads, and each piece that a thread adds.  The table takes the side whose estimate is less.
// bf16 in microseconds, 256 x 256 tiles against 128 x 128: 2048 x 2048 of 203 tokens 18.6 and 15.4, of 1024 34 and 22, of 8192 95
// and 108; four such matrices of 2048 tokens 72 and 88; 512 x 1024 of 512 tokens 19.3 and 15.8.  In one to sixteen pieces
// (256 x 256) 512 x 1024 of 2048 tokens took 51, 33, 26, 24 and 26, 2048 x 2048 of 203 tokens 19, 25 and 32.
struct Schedule {
  uint32_t tiles = 0, whole = 0, split = 1;
  double us = 0.0;
};

uint32_t units_of(int side) { return side == 256 ? 256 : 512; }   // workgroups at once: one or two a CU

uint32_t tiles_of(const Layer& l, int side) {
  return (uint32_t)((l.rows + side - 1) / side) * (uint32_t)((l.cols + side - 1) / side);
}

Schedule schedule(const Layer* layers, int n_layers, int side) {
  const bool big = side == 256;
  const double few = big ? 0.59 : 0.35, full = big ? 0.89 : 0.60, ends = big ? 8.0 : 5.0, piece = big ? 0.05 : 0.0125;
  const uint32_t units = units_of(side), alone = big ? 0 : 256;
  auto step = [&](uint32_t n) { return few + (full - few) * (double)(n - std::min(n, alone)) / (units - alone); };
  Schedule S;
  for (int j = 0; j < n_layers; ++j) S.tiles += tiles_of(layers[j], side);
  S.whole = S.tiles / units * units;
  uint32_t at = 0;
  int steps = 0;   // of the longest tile past the full rounds
  for (int j = 0; j < n_layers; ++j) {
    const uint32_t n = tiles_of(layers[j], side), in = std::min(n, S.whole > at ? S.whole - at : 0u);
    const int all = layers[j].steps * layers[j].parts;
    S.us += (double)in / units * (full * all + ends);
    if (in < n) steps = std::max(steps, all);
    at += n;
  }
  const uint32_t rest = S.tiles - S.whole;
  if (rest == 0) return S;
  double least = step(rest) * steps + ends;
  for (uint32_t s = 2; s <= units / rest && s <= (uint32_t)steps; ++s) {
    const double us = step(rest * s) * ((steps + s - 1) / s) + ends + 3.0 + piece * rest * s + 0.15 * s;
    if (us < least) least = us, S.split = s;
  }
  S.us += least;
  if (S.split == 1) S.whole = S.tiles;
  return S;
}

// Bytes that hold the pieces of split tiles by either side: as many as workgroups run at once (64 MiB), fewer only where the
// tiles have no more steps in all.  The pieces that a schedule makes fall here and there as tokens grow; this does not, so that a
// workspace for the longest batch holds the shorter ones.
size_t most_pieces(const Layer* layers, int n_layers) {
  size_t most = 0;
  for (int side : {128, 256}) {
    uint64_t tiles = 0;
    int steps = 0;
    for (int j = 0; j < n_layers; ++j) {
      tiles += tiles_of(layers[j], side);
      steps = std::max(steps, layers[j].steps * layers[j].parts);
    }
    if (steps > 1) most = std::max(most, sizeof(float) * side * side * (size_t)std::min<uint64_t>(units_of(side), tiles * steps));
  }
  return most;
}

}  // namespace

int weight_grad_group(const iso_weight_grad* g, int n, int dt_grad) {
  const uint64_t size = dt_grad == ISO_BF16 ? 2 : 4;
  uint64_t from[kLayers], to[kLayers];
  n = std::min(n, kLayers);
  for (int j = 0; j < n; ++j) {
    from[j] = (uintptr_t)g[j].grad;
    to[j] = from[j] + size * (uint64_t)(g[j].rows * g[j].in.cols);   // an empty matrix shares nothing
    for (int k = 0; k < j; ++k)
      if (std::max(from[j], from[k]) < std::min(to[j], to[k])) return j;
  }
  return n;
}

WeightGradPlan plan_weight_grad(const iso_weight_grad* g, int n, int dt, bool accumulate, uint8_t* ws) {
  WeightGradPlan P;
  size_t at = kStatusBytes;
  auto region = [&](size_t bytes) {
    const uintptr_t o = (uintptr_t)ws + at;   // ws is null where only the size is asked for
    at = align_up(at + bytes, 256);
    return (uint8_t*)o;
  };
  const int parts = dt == ISO_F32 ? 3 : 1;
  struct Kept {
    const iso_ckpt* c;
    const uint8_t* x;
  };
  Kept kept[kLayers];
  Layer layers[kLayers];
  int n_kept = 0, n_layers = 0;
  auto add_prep = [&](Prep p, int64_t rows) {
    p.block0 = P.prep.blocks;
    P.prep.blocks += (uint32_t)((rows * p.per_row + 255) / 256);
    P.prep.p[P.prep.n++] = p;
  };
  for (int j = 0; j < n; ++j) {
    const iso_weight_grad& x = g[j];
    const int64_t t = x.in.rows;
    if (x.rows == 0 || x.in.cols == 0 || (t == 0 && accumulate)) continue;
    Layer l{};
    l.g = x.grad;
    l.rows = (int32_t)x.rows, l.cols = (int32_t)x.in.cols;
    l.steps = (int32_t)(whole_steps(t) / kStep);
    l.parts = parts;
    const int64_t ld = ckpt_ld(x.in.cols);
    l.x_ld = 2 * ld, l.x_bytes = 2 * t * ld;
    if (t > 0) {
      for (int k = 0; k < n_kept; ++k) {
        const iso_ckpt& c = *kept[k].c;
        if (x.in.q != nullptr && c.q == x.in.q && c.e == x.in.e && c.rows == t && c.cols == x.in.cols) l.x = kept[k].x;
      }
      if (l.x == nullptr) {
        uint8_t* const to = region(2 * (size_t)(t * ld));
        add_prep(Prep{x.in.q, x.in.e, (uint16_t*)to, t, ld, 0, (uint32_t)ld, (uint32_t)(ld / 8), 0}, t);
        kept[n_kept++] = Kept{&x.in, to};
        l.x = to;
      }
      if (direct(x, dt)) {
        l.y = (const uint8_t*)x.dy;
        l.y_ld = 2 * x.ld_dy;
        l.y_bytes = (int64_t)align_up(2 * (size_t)((t - 1) * x.ld_dy + x.rows), 16);
      } else {
        const int64_t per = (x.rows + 7) / 8, part = whole_steps(t);
        uint8_t* const to = region(2 * (size_t)(parts * part * per * 8));
        add_prep(Prep{x.dy, nullptr, (uint16_t*)to, t, x.ld_dy, part, (uint32_t)x.rows, (uint32_t)per, 0}, part);
        l.y = to;
        l.y_ld = 16 * per;
        l.y_bytes = 16 * parts * part * per;
      }
    }
    // long sums first: the tiles past the last full round, which may be split, are then the shortest
    int to = n_layers++;
    for (; to > 0 && layers[to - 1].steps < l.steps; --to) layers[to] = layers[to - 1];
    layers[to] = l;
  }
  LayerTable& L = P.layers;
  const Schedule big = schedule(layers, n_layers, 256), small = schedule(layers, n_layers, 128);
  P.tile = small.us < big.us ? 128 : 256;
  const Schedule& S = P.tile == 128 ? small : big;
  L.whole = S.whole, L.split = S.split;
  for (int j = 0; j < n_layers; ++j) {
    Layer& l = layers[j];
    l.across = (l.cols + P.tile - 1) / P.tile, l.down = (l.rows + P.tile - 1) / P.tile;
    l.tile0 = L.tiles;
    L.tiles += (uint32_t)l.across * (uint32_t)l.down;
    L.l[L.n++] = l;
  }
  L.part = (float*)region(most_pieces(layers, n_layers));
  P.prep.status = (uint32_t*)ws;
  P.total = at;
  return P;
}

size_t weight_grad_workspace_bytes(const iso_weight_grad* g, int n, int dt) {
  size_t most = kStatusBytes;
  for (int j = 0; j < n; j += kLayers)
    for (bool accumulate : {false, true})   // a layer without tokens takes part in the one and not in the other
      most = std::max(most, plan_weight_grad(g + j, std::min(kLayers, n - j), dt, accumulate, nullptr).total);
  return most;
}

// ---- attention -----------------------------------------------------------------------------------------------------

bool attend_fits(const iso_attn& a) {
  // launches hold fewer than 2^32 threads: a workgroup of 256 for up to 128 rows or keys of a sequence and kv head, and for eight
  // rows that are joined
  const int64_t most = ISO_ATTN_MAX_ROWS;
  if (a.heads / a.heads_kv > ISO_ATTN_MAX_GROUP || a.tokens_q > most || a.tokens_k > most) return false;
  return a.tokens_q * a.heads <= most && a.tokens_k * a.heads_kv <= most && a.sequences * a.heads_kv <= most / 8;
}

namespace {

constexpr int kPieceKeys = 256;         // fewest keys of a piece
constexpr int kMostTilePieces = 64;         // of a tile
constexpr double kSparse = 2.0;
constexpr int64_t kRound = 512;         // workgroups at once, counted as two a CU (forward with bf16 heads up to 64 runs three)
constexpr int64_t kFullTiles = 1536;    // three rounds of them: heavy tiles first, these balance by themselves

// Tiles of `owners` rows walk over `length` keys on average.  In p pieces a tile's time falls by p, and every row writes and
// reads p partial sums: the sum of both is least at p = f sqrt(length / owners).  f was measured, 6.5 for rows and 9.1 for keys
// (which have dK and dV).  Microseconds with f at 11, 9, 6.5 and 5.5, forward: 2048 tokens, 12 heads, 40, 43, 42, 42; 4096 tokens
// 92, 94, 83, 82; 512 tokens 19, 18.6, 17.1, 17.1; 64 new tokens after 4032 for four sequences, 28 heads, 37.5, 38.2, 36.4, 36.9; with f at
// 4.5 39.8.  Backward with keys' f at 9.1 and 6: 2048 tokens, 12 heads, 94 and 90; 16 samples of 1 to 2048 tokens 294 and 308.  Tiles that are mostly
// empty (one new token a sequence) write little and are bound by what a workgroup waits for at its start and each panel: twice as
// many pieces, but all of them at once (16 tokens over 77 to 8192 keys, 28 heads: pieces of 256 keys 37.5 us, 512 30.0, 640 30.1).
Pieces share_out(int64_t owners, int64_t list, int64_t sequences, int64_t heads, double f) {
  Pieces P;
  if (owners <= 0 || list <= 0 || sequences <= 0) return P;
  const int64_t tiles = std::max(owners / kAttnTileRows, sequences * heads), length = (list + sequences - 1) / sequences;
  const bool sparse = owners < sequences * heads * (kAttnTileRows / 2);
  if (sparse) f *= kSparse;
  int64_t p = (int64_t)(f * std::sqrt((double)length / (double)owners));
  p = std::min({p, kFullTiles / std::max<int64_t>(1, tiles), (list + kPieceKeys - 1) / kPieceKeys, (int64_t)kMostTilePieces});
  if (p <= 1) return P;
  P.most = (int32_t)p;
  P.keys = (int32_t)std::max<int64_t>(kPieceKeys, length / (2 * p));   // sequences differ in length
  if (sparse) {   // in one round, a sequence's last piece half full
    const int64_t full = std::max<int64_t>(kRound / 4, kRound - tiles / 2), keys = (list * heads + full - 1) / full;
    P.keys = std::max(P.keys, (int32_t)std::min<int64_t>((keys + 63) / 64 * 64, 1 << 30));
  }
  return P;
}
// Partial sums that a call of up to so many owners and keys may take, whatever its sequences.  t whole tiles are up to
// (t + 1) kAttnTileRows owners with at most kFullTiles / t pieces, and kMostTilePieces.
size_t most_parts(int64_t owners, int64_t list, double f) {
  if (owners <= 0 || list <= 0) return 0;
  const double each = (double)std::min<int64_t>(kMostTilePieces, (list + kPieceKeys - 1) / kPieceKeys);
  return (size_t)std::min({kSparse * f * std::sqrt((double)list * (double)owners), (double)owners * each, (double)(kFullTiles + kMostTilePieces) * kAttnTileRows});
}

}  // namespace

uint32_t attend_items(int64_t rows, int64_t list, int64_t sequences, const Pieces& p) {
  // a sequence of n tiles and length m has n min(most, m / keys + 1) items at most
  const int64_t tiles = rows / kAttnTileRows + sequences, longest = rows / kAttnTileRows + 1;
  if (p.most == 1) return (uint32_t)tiles;
  return (uint32_t)std::min(tiles * p.most, longest * (list / p.keys + sequences));
}

AttendPlan plan_attend(const iso_attn& a, bool grad) {
  const int64_t rows = a.tokens_q * a.heads, keys = a.tokens_k * a.heads_kv, list = a.tokens_q * (a.heads / a.heads_kv);
  constexpr double kRows = 6.5, kKeys = 9.1;
  AttendPlan P;
  auto parts = [](size_t n) { return align_up(sizeof(float) * kPartLd * n, 256); };
  P.rows = share_out(rows, a.tokens_k, a.sequences, a.heads_kv, kRows);
  // a panel's rows are read whole, and one panel too many: up to 64 behind the last one
  P.part = grad ? align_up(kStatusBytes + sizeof(float) * (2 * (size_t)rows + 64), 256) : kStatusBytes;
  P.key_part = P.total = P.part + parts(most_parts(rows, a.tokens_k, kRows));
  if (!grad) return P;
  P.keys = share_out(keys, list, a.sequences, a.heads_kv, kKeys);
  P.total = P.key_part + parts(2 * most_parts(keys, list, kKeys));
  return P;
}

size_t attend_workspace_bytes(const iso_attn& a, int, bool grad) { return plan_attend(a, grad).total; }

}  // namespace iso

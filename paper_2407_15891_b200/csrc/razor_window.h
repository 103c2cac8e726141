// Attention of prompt tokens with a window and sink tokens per KV head: which tiles of keys a tile of queries needs, and how
// the work is laid out over the CTAs.  Plain arithmetic, the same on the host (tests) and in the kernels.
//
// A tile is 128 rows = up to 128 / G query tokens x the G query heads of a KV head; a unit is a pair of tiles of one
// (sequence, KV head).  Keys come in tiles of 128 tokens.  The key tiles that some query of a unit sees are numbered
// 0 .. n_steps - 1: first those that hold sink tokens, then the window's run up to the diagonal.
#ifndef RAZOR_WINDOW_H_
#define RAZOR_WINDOW_H_

#include <stdint.h>

#include "razor_internal.h"

namespace razor {

constexpr int kWinTile = 128;          // rows of a tile of queries, tokens of a tile of keys
constexpr int kWinMaxSpans = 160;      // most CTAs that share the steps of a launch between them
constexpr int kWinSpanUnits = 1024;    // launches of up to so many units are cut into spans, larger ones hand out whole units
constexpr int kWinMinSpan = 4;         // steps that a span has at least
constexpr int kWinUnitCost = 3;        // what a unit costs beside its steps (its queries' way in, its results' way out), in steps

// One tile of a unit: its live tokens [tok, tok + n_tok) and the steps that it takes part in, [0, sink_end) and
// [win_begin, win_end); with parity 0 or 1 only the even or the odd ones of them.
struct WinTileSteps {
  int32_t tok, n_tok, pos;             // pos: position of token `tok`
  int32_t sink_end, win_begin, win_end;
  int32_t parity;                      // -1: every step
  RAZOR_HD bool active(int j) const {
    return (j < sink_end || (j >= win_begin && j < win_end)) && (parity < 0 || (j & 1) == parity);
  }
  RAZOR_HD int count(int a, int b) const {   // its steps among a .. b - 1, 0 <= a
    if (b <= a) return 0;
    return parity < 0 ? b - a : (b + 1 - parity) / 2 - (a + 1 - parity) / 2;
  }
  RAZOR_HD int steps_in(int a, int b) const {
    return count(a, b < sink_end ? b : sink_end) + count(a > win_begin ? a : win_begin, b < win_end ? b : win_end);
  }
};
struct WinUnit {
  int32_t live;                        // query tokens of the unit (0: nothing to do)
  int32_t n_steps;                     // key tiles of the union of both tiles
  int32_t n_sink_steps, win_first;     // step j is key tile j below n_sink_steps, win_first + j - n_sink_steps above
  WinTileSteps tile[2];
  RAZOR_HD int key_tile(int j) const { return j < n_sink_steps ? j : win_first + (j - n_sink_steps); }
  // what the unit counts for when the work is shared out (one with nothing to see still has its zeros to write)
  RAZOR_HD int weight() const { return live == 0 ? 0 : n_steps + kWinUnitCost; }
  // The steps [j0, j1) that the stretch [a, z) of its weight stands for.  A cut within the unit's fixed cost moves to its
  // start.  False: none.
  RAZOR_HD bool part(long long a, long long z, int& j0, int& j1) const {
    j0 = a > kWinUnitCost ? (int)(a - kWinUnitCost) : 0;
    j1 = z > kWinUnitCost ? (int)(z - kWinUnitCost) : 0;
    return n_steps == 0 ? a == 0 && z > 0 : j1 > j0;
  }
  // A unit whose queries fit one tile leaves the other idle.  Where it is cut up anyway (its records are folded later), both
  // tiles take its queries, one the even and one the odd steps.
  RAZOR_HD void share_steps() {
    tile[1] = tile[0];
    tile[0].parity = 0;
    tile[1].parity = 1;
  }
};

// q_len queries at positions ctx - q_len .. ctx - 1; window < 0: a head that sees everything.  tok0: the unit's first query
// token, tpt: query tokens of a tile.
RAZOR_HD inline WinUnit win_unit(int tok0, int tpt, int q_len, int ctx, int window, int n_sink) {
  WinUnit u;
  u.live = q_len > tok0 ? (q_len - tok0 < 2 * tpt ? q_len - tok0 : 2 * tpt) : 0;
  const int pos0 = ctx - q_len + tok0, last = pos0 + u.live - 1;   // positions of the unit's first and last query
  u.n_sink_steps = u.win_first = u.n_steps = 0;
  const bool any = u.live > 0 && last >= 0;
  if (any) {
    const int hi = last / kWinTile;
    if (window < 0) {
      u.n_steps = hi + 1;
    } else {
      const int sink_tiles = (int)(((long long)n_sink + kWinTile - 1) / kWinTile);
      u.n_sink_steps = sink_tiles < hi + 1 ? sink_tiles : hi + 1;
      const long long lo_tok = (long long)pos0 - window + 1;
      int lo = window == 0 ? hi + 1 : (lo_tok > 0 ? (int)(lo_tok / kWinTile) : 0);
      if (lo > hi + 1) lo = hi + 1;
      u.win_first = lo > u.n_sink_steps ? lo : u.n_sink_steps;
      u.n_steps = u.n_sink_steps + (hi + 1 - u.win_first);
    }
  }
  for (int i = 0; i < 2; ++i) {
    WinTileSteps& t = u.tile[i];
    t.tok = tok0 + i * tpt;
    const int left = u.live - i * tpt;
    t.n_tok = left < 0 ? 0 : (left < tpt ? left : tpt);
    t.pos = pos0 + i * tpt;
    t.sink_end = t.win_begin = t.win_end = 0;
    t.parity = -1;
    const int t_last = t.pos + t.n_tok - 1;
    if (!any || t.n_tok == 0 || t_last < 0) continue;
    const int hi = t_last / kWinTile;
    t.sink_end = u.n_sink_steps < hi + 1 ? u.n_sink_steps : hi + 1;
    int lo = u.win_first;
    if (window > 0) {
      const long long lo_tok = (long long)t.pos - window + 1;
      if (lo_tok > 0 && lo_tok / kWinTile > lo) lo = (int)(lo_tok / kWinTile);
    } else if (window == 0) {
      lo = hi + 1;
    }
    if (lo <= hi) {
      t.win_begin = u.n_sink_steps + (lo - u.win_first);
      t.win_end = u.n_sink_steps + (hi + 1 - u.win_first);
    }
  }
  return u;
}

// Does key tile kt need masking for the queries at positions [first, last]?
RAZOR_HD inline bool win_masked(int kt, int first, int last, int window, int n_sink) {
  const int a = kt * kWinTile, b = a + kWinTile - 1;
  return !(b <= first && (window < 0 || b < n_sink || (long long)a > (long long)last - window));
}

// Is key n in sight of some query at the positions first .. last (some position, first <= last)?
RAZOR_HD inline bool win_seen(long long n, int first, int last, int window, int n_sink) {
  return n <= last && (n < n_sink || window < 0 || (first > n ? first : n) - n < window);
}

// Spans: the units' weights end to end, cut into n_spans pieces of equal length.
RAZOR_HD inline int win_n_spans(long long total, int ctas) {
  const long long most = total / kWinMinSpan;
  return (int)(most < 1 ? 1 : (most < ctas ? most : ctas));
}
RAZOR_HD inline long long win_span_begin(long long total, int n_spans, int c) {   // total * c / n_spans
  if (total < (1LL << 31)) {   // (in 32 bits where they do: a division of 64 takes ten times as long)
    const uint32_t each = (uint32_t)total / (uint32_t)n_spans, rest = (uint32_t)total % (uint32_t)n_spans;
    return (long long)each * c + rest * (uint32_t)c / (uint32_t)n_spans;
  }
  return total * c / n_spans;
}
// The span that place s lies in.
RAZOR_HD inline int win_span_of(long long total, int n_spans, long long s) {
  int c = (int)((double)s / (double)total * n_spans);   // (a guess)
  if (c >= n_spans) c = n_spans - 1;
  while (c + 1 < n_spans && win_span_begin(total, n_spans, c + 1) <= s) ++c;
  while (c > 0 && win_span_begin(total, n_spans, c) > s) --c;
  return c;
}

// The spans that hold parts of a unit of weight w > 0 that begins at place s: the first and their number.
RAZOR_HD inline void win_unit_spans(long long total, int n_spans, long long s, long long w, int& first, int& parts) {
  first = win_span_of(total, n_spans, w > kWinUnitCost ? s + kWinUnitCost : s);
  parts = w > kWinUnitCost ? win_span_of(total, n_spans, s + w - 1) - first + 1 : 1;
}

}  // namespace razor
#endif

// razor_window.h against what it stands for: the key tiles that hold a key some query of a tile sees, found one by one.
#include <cstdio>
#include <cstdlib>

#include "razor_window.h"

using namespace razor;

static unsigned long long rng_state = 1;
static int rnd(int lo, int hi) {   // lo .. hi
  rng_state = rng_state * 6364136223846793005ull + 1442695040888963407ull;
  return lo + (int)((rng_state >> 33) % (unsigned long long)(hi - lo + 1));
}
static bool sees(int m, int n, int window, int n_sink) { return n <= m && (n < n_sink || window < 0 || m - n < window); }
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s (case %d)\n", __LINE__, #x, at); return 1; } } while (0)

int main() {
  for (int at = 0; at < 4000; ++at) {
    const int G = rnd(1, 8), tpt = kWinTile / G;
    const int ctx = rnd(0, 3) ? rnd(0, 1500) : rnd(0, 40), q_len = rnd(0, 5) ? rnd(0, ctx) : rnd(0, ctx + 300);
    const int window = rnd(0, 4) == 0 ? -1 : rnd(0, 3) ? rnd(0, 700) : rnd(0, 3);
    const int n_sink = rnd(0, 2) ? rnd(0, 5) : rnd(0, 600);
    for (int tok0 = 0; tok0 < q_len + 2 * tpt; tok0 += 2 * tpt) {
      const WinUnit u = win_unit(tok0, tpt, q_len, ctx, window, n_sink);
      int live = q_len - tok0;
      live = live < 0 ? 0 : live > 2 * tpt ? 2 * tpt : live;
      CHECK(u.live == live);
      CHECK((u.weight() == 0) == (live == 0) && u.n_steps >= 0);
      CHECK(u.tile[0].n_tok + u.tile[1].n_tok == live);
      for (int j = 1; j < u.n_steps; ++j) CHECK(u.key_tile(j) > u.key_tile(j - 1));
      if (u.n_steps) CHECK(u.key_tile(0) >= 0 && u.key_tile(u.n_steps - 1) * kWinTile < ctx);
      for (int i = 0; i < 2; ++i) {
        const WinTileSteps& t = u.tile[i];
        if (t.n_tok == 0) { CHECK(t.steps_in(0, u.n_steps) == 0); continue; }
        CHECK(t.tok == tok0 + i * tpt && t.pos == ctx - q_len + t.tok);
        const int first = t.pos, last = t.pos + t.n_tok - 1;
        int n_active = 0, j_of[16];
        for (int k = 0; k < 16; ++k) j_of[k] = -1;
        for (int j = 0; j < u.n_steps; ++j) {
          j_of[u.key_tile(j)] = j;
          n_active += t.active(j);
        }
        CHECK(t.steps_in(0, u.n_steps) == n_active);
        const int cut = rnd(0, u.n_steps);
        CHECK(t.steps_in(0, cut) + t.steps_in(cut, u.n_steps) == n_active);
        for (int kt = 0; kt * kWinTile < ctx; ++kt) {
          bool any = false, all = true;
          for (int m = first; m <= last; ++m)
            for (int n = kt * kWinTile; n < (kt + 1) * kWinTile; ++n) {
              const bool s = sees(m, n, window, n_sink);
              any |= s;
              all &= s;
            }
          // a tile that some query sees is a step the tile takes part in; one whose mask is left out is seen by all
          if (any) CHECK(j_of[kt] >= 0 && t.active(j_of[kt]));
          if (!win_masked(kt, first, last, window, n_sink)) CHECK(all);
          if (all) CHECK(!win_masked(kt, first, last, window, n_sink) || last - first + 1 < 1 || n_sink > 0);
        }
      }
    }
  }
  // a unit of one tile shared by both: every step goes to exactly one of them
  for (int at = 0; at < 3000; ++at) {
    WinUnit u = win_unit(0, 128, rnd(1, 128), rnd(1, 1500), rnd(0, 2) ? rnd(0, 700) : -1, rnd(0, 300));
    const WinTileSteps whole = u.tile[0];
    u.share_steps();
    for (int j = 0; j < u.n_steps; ++j) CHECK((int)u.tile[0].active(j) + (int)u.tile[1].active(j) == (int)whole.active(j));
    const int a = rnd(0, u.n_steps), b = rnd(a, u.n_steps);
    for (int i = 0; i < 2; ++i) {
      int n = 0;
      for (int j = a; j < b; ++j) n += u.tile[i].active(j);
      CHECK(u.tile[i].steps_in(a, b) == n);
    }
  }
  for (int at = 0; at < 20000; ++at) {
    const long long total = rnd(1, 5) == 1 ? rnd(1, 30) : (long long)rnd(1, 2000000) * rnd(1, 3000);
    const int ctas = rnd(1, kWinMaxSpans), n = win_n_spans(total, ctas);
    CHECK(n >= 1 && n <= ctas && n <= total);
    CHECK(win_span_begin(total, n, 0) == 0 && win_span_begin(total, n, n) == total);
    for (int k = 0; k < 20; ++k) {
      const int c = rnd(0, n - 1);
      const long long b = win_span_begin(total, n, c), e = win_span_begin(total, n, c + 1);
      CHECK(b < e);
      CHECK(win_span_of(total, n, b) == c && win_span_of(total, n, e - 1) == c);
    }
  }
  // units end to end, cut into spans: every step of every unit in one part, in order; the parts where the combining side looks
  for (int at = 0; at < 3000; ++at) {
    const int n = rnd(1, 12), ctas = rnd(1, 20);
    WinUnit us[12];
    long long begin[13] = {0};
    for (int i = 0; i < n; ++i) {
      us[i] = WinUnit();
      us[i].live = rnd(0, 4) ? 5 : 0;
      us[i].n_steps = rnd(0, 3) ? rnd(0, 40) : 0;
      begin[i + 1] = begin[i] + us[i].weight();
    }
    const long long total = begin[n];
    if (total == 0) continue;
    const int ns = win_n_spans(total, ctas);
    for (int i = 0; i < n; ++i) {
      const int w = us[i].weight();
      if (w == 0) continue;
      int first, parts, next = 0, seen = 0;
      win_unit_spans(total, ns, begin[i], w, first, parts);
      for (int c = 0; c < ns; ++c) {
        long long a = win_span_begin(total, ns, c) - begin[i], z = win_span_begin(total, ns, c + 1) - begin[i];
        if (a < 0) a = 0;
        if (z > w) z = w;
        int j0 = 0, j1 = 0;
        if (a >= z || !us[i].part(a, z, j0, j1)) continue;
        CHECK(c == first + seen);
        CHECK(j0 == next);
        next = j1;
        ++seen;
      }
      CHECK(seen == parts && next == us[i].n_steps);
    }
  }
  std::printf("ok\n");
  return 0;
}

// How many columns the attention of drafted trees takes, and how many of its CTAs share an SM: rules on the sizes of a call, for host code alone.
#pragma once

#include <stdint.h>

namespace pq_tree {

constexpr int KEYS = 128;  // of a key tile
constexpr int SHORT = 8;   // an item of so many key tiles or fewer is not shared between workers

// The longest prefix beside which two CTAs of 32 or 64 columns share an SM (its scores are in shared memory); a CTA of 128 columns has its SM to itself.
constexpr int two_ctas_prefix(int columns, bool own_steps) { return columns == 32 ? (own_steps ? 24 : 56) : columns == 64 ? (own_steps ? 12 : 24) : -1; }
constexpr int ctas_of_sm(int columns, bool own_steps, int n_prefix) { return n_prefix <= two_ctas_prefix(columns, own_steps) ? 2 : 1; }

// Key tiles that an estimate counts for a bound on the cached keys: about what a window leaves of them.
inline int64_t tiles_seen(int64_t max_len, int32_t window, int32_t n_sink) {
  const int64_t most = static_cast<int64_t>(window) + n_sink + 3 * KEYS;
  if (window > 0 && max_len > most) max_len = most;
  return max_len < KEYS ? 1 : (max_len + KEYS - 1) / KEYS;
}

// By an estimate for B sequences of max_new rows, fitted to 176 ragged batches of 1 to 48 sequences (on their average 1 % above the best of the three, 35 % at most). An item
// costs its key tiles and 4 to 6 more of 1.5 us with 32 columns, 2.2 with 64 (two CTAs share the SM) and 1.9 with 128; short items are not cut, so that CTAs walk whole rounds
// of them; and with long ones a stretch is no shorter than a short item. us with 32 / 64 / 128 columns, 32 heads on 8: 1 x 26 rows at 1021 keys 18 / 22 / 24, at 4000
// 23 / 30 / 33; 1 x 128 at 20000 106 / 82 / 74; 16 x 16 at 4000 55 / 52 / 56, 64 x 8 at 6000 139 / 170 / 250, 32 x 30 at 4000 185 / 136 / 123.
// Beside a longer prefix, with the CTAs that then share an SM: 28 prefixed keys, 16 x 16 at 4000 56 / 74 / 77 us (own steps 80 / 77 / 81), 1 x 26 at 4000, own steps
// 28 / 43 / 44; counted as two CTAs everywhere, these calls took 84 to 91 and 40. With 64 prefixed keys, whose scores an item waits for, the choice is up to 13 % from the best.
inline int columns_of(bool own_steps, int n_prefix, int sms, int B, int Hkv, int G, int max_new, int64_t max_len, int32_t window, int32_t n_sink) {
  const double tiles = static_cast<double>(tiles_seen(max_len, window, n_sink));
  auto estimate = [&](int columns, double fixed, double more, double tile) {
    const int per_item = columns / G, ctas = ctas_of_sm(columns, own_steps, n_prefix);
    const int64_t items = static_cast<int64_t>(B) * Hkv * ((max_new + per_item - 1) / per_item), workers = static_cast<int64_t>(ctas) * sms;
    const double least = SHORT + more, share = static_cast<double>(items) / workers * (tiles + more);
    const double units = tiles <= SHORT ? static_cast<double>((items + workers - 1) / workers) * (tiles + more) : share > least ? share : least;
    return fixed + units * tile;
  };
  const double t32 = estimate(32, 3.0, 5.0, 1.5), t64 = estimate(64, 2.0, 4.0, 2.2), t128 = estimate(128, 0.0, 6.0, 1.9);
  if (t32 <= t64 && t32 <= t128) return 32;
  return t64 <= t128 ? 64 : 128;
}

}  // namespace pq_tree

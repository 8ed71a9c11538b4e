// lh_paged_lds.h -- where the waves of rows_tile (lh_paged_rows.h) keep their memory when it is the ring of the tile
// kernel (k_paged_tile.hip). Host and device, of nothing but integers, so that a test can go through all of it.
#pragma once

namespace lh {

// Four arrays of 32 D floats each (a ring slot of K or V: 64 rows of D bf16). In them
//   part(w), 16 D floats of wave w, PER waves at a time, two to an array: written when the wave's keys are done;
//   words(w), 8 D floats of a wave alone (4 KB at D = 128), used while its keys last.
// A wave may write its part while another still uses its words. So either words(w) lies in part(w), or a barrier
// stands between the last words and the first part (kOwnWords says which).
template <int D, int NW>
struct TileLdsMap {
  static constexpr int ARRAYS = 4, SIZE = 32 * D, PART = 16 * D, WORDS = 8 * D;
  static constexpr int PER = NW < 8 ? NW : 8;
  static constexpr bool kOwnWords = PER == NW;
  static constexpr int part_array(int w) { return w & 3; }
  static constexpr int part_off(int w) { return (w >> 2) * PART; }
  static constexpr int words_array(int w) { return kOwnWords ? part_array(w) : w >> 2; }
  static constexpr int words_off(int w) { return kOwnWords ? part_off(w) : (w & 3) * WORDS; }

  // Inside the arrays, no two waves' words or parts in the same place, and no wave's words in another's part unless a
  // barrier parts them.
  static constexpr bool sound() {
    for (int w = 0; w < NW; ++w) {
      const int a = words_array(w) * SIZE + words_off(w);
      if (words_array(w) >= ARRAYS || words_off(w) + WORDS > SIZE) return false;
      if (w < PER && (part_array(w) >= ARRAYS || part_off(w) + PART > SIZE)) return false;
      for (int y = 0; y < NW; ++y) {
        if (y == w) continue;
        const int b = words_array(y) * SIZE + words_off(y);
        if (a < b + WORDS && b < a + WORDS) return false;
        if (y >= PER) continue;
        const int p = part_array(y) * SIZE + part_off(y);
        if (kOwnWords && a < p + PART && p < a + WORDS) return false;
        if (w < PER && part_array(w) == part_array(y) && part_off(w) == part_off(y)) return false;
      }
    }
    return true;
  }
};

}  // namespace lh

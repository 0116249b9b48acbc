// Places of the attention tiles that go from memory straight to LDS, for every
// thread and pass, evaluated at compile time on the host: every 16-byte piece
// that is loaded lies within its row of D components, and every piece of the
// row is loaded, to the place where the tile's layout has it.
#include "wbmm_attn.h"

namespace wbmm {

template <class Tag, int DP, int ROWS, bool PLAIN>
constexpr bool places_hold(int D) {
  using P = DirectTile<Tag, DP, ROWS, PLAIN>;
  using M = Mover<Tag, DP, ROWS, 256>;
  using T = Tile<Tag, DP>;
  int loaded = 0;
  for (int tid = 0; tid < 256; ++tid)
    for (int p = 0; p < M::NP; ++p) {
      const int row = M::row(tid, p);
      if (row >= ROWS || !P::has(tid, p, D)) continue;
      const int at = T::chunk_at(M::chunk(tid), row) * T::CE;
      if (at < 0 || at + T::CE > D) return false;
      const int to = p * 4096 + tid * 16;  // where the load leaves it in the tile
      if (to / T::PITCH != row || T::chunk_at(to % T::PITCH / 16, row) * T::CE != at) return false;
      ++loaded;
    }
  return loaded == ROWS * (D / T::CE);
}

// Whole rows (PLAIN) have DP components; others any number that is padded to DP.
template <class Tag, int DP, int ROWS>
constexpr bool all_hold() {
  if (!places_hold<Tag, DP, ROWS, true>(DP)) return false;
  for (int D = DP - 32 + 16 / Tag::ES; D <= DP; D += 16 / Tag::ES)
    if (!places_hold<Tag, DP, ROWS, false>(D)) return false;
  return true;
}

#define WBMM_HOLDS(Tag, DP) \
  static_assert(all_hold<Tag, DP, 32>() && all_hold<Tag, DP, 64>(), #Tag " " #DP)
WBMM_HOLDS(TagBF16, 32);
WBMM_HOLDS(TagBF16, 64);
WBMM_HOLDS(TagBF16, 96);
WBMM_HOLDS(TagBF16, 128);
WBMM_HOLDS(TagF16, 96);
WBMM_HOLDS(TagF32, 32);
WBMM_HOLDS(TagF32, 64);
WBMM_HOLDS(TagF32, 96);
WBMM_HOLDS(TagF32, 128);

}  // namespace wbmm

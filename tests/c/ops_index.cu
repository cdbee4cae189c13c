// The index functions of the model operators' kernels, called on the host: no GPU, no kernel is launched.
#include <cstdio>
#include <set>
#include <utility>

#include "kb_matmul.cuh"
#include "kb_quant.cuh"

#define CHECK(cond, ...)                                  \
  do {                                                    \
    if (!(cond)) {                                        \
      std::printf("%s:%d: %s: ", __FILE__, __LINE__, #cond); \
      std::printf(__VA_ARGS__);                           \
      std::printf("\n");                                  \
      return 1;                                           \
    }                                                     \
  } while (0)

// every tile of a product is visited once, and neighbours share rows of tiles
static int tiles() {
  for (uint32_t m : {1u, 2u, 7u, 8u, 9u, 16u, 33u})
    for (uint32_t n : {1u, 3u, 32u, 41u}) {
      std::set<std::pair<uint32_t, uint32_t>> seen;
      for (uint32_t t = 0; t < m * n; ++t) {
        uint32_t tm = 0, tn = 0;
        kb::pair_tile(t, m, n, tm, tn);
        CHECK(tm < m && tn < n, "%u x %u, item %u: %u %u", m, n, t, tm, tn);
        CHECK(tm / kb::PairTile::kGroupM == t / (kb::PairTile::kGroupM * n), "item %u in row %u", t, tm);
        seen.insert({tm, tn});
      }
      CHECK(seen.size() == m * n, "%u x %u: %zu tiles", m, n, seen.size());
    }
  return 0;
}

// a cluster's CTAs share the columns without gap or overlap, and their parts fit the buffer
template <int BN>
static int clusters() {
  using T = kb::LaneTile<BN>;
  CHECK(T::kGroups * 4 == BN, "%u", T::kGroups);
  CHECK(T::kSmem <= 227 * 1024, "%u", T::kSmem);
  for (uint32_t splits = 1; splits <= 8; ++splits) {
    const uint32_t share = kb::cluster_share(T::kGroups, splits);
    CHECK(splits == 1 || splits * share * 128 * 16 <= T::kSumBytes, "%d columns, %u CTAs", BN, splits);
    CHECK(kb::cluster_first(T::kGroups, splits, 0) == 0 && kb::cluster_first(T::kGroups, splits, splits) == T::kGroups, "%u", splits);
    for (uint32_t o = 0; o < splits; ++o) {
      const uint32_t first = kb::cluster_first(T::kGroups, splits, o), last = kb::cluster_first(T::kGroups, splits, o + 1);
      CHECK(first <= last && last - first <= share, "%d columns, CTA %u of %u: %u to %u", BN, o, splits, first, last);
      for (uint32_t g = first; g < last; ++g)
        CHECK(kb::cluster_owner(T::kGroups, splits, g) == o, "%d columns, group %u of CTA %u", BN, g, o);
    }
  }
  return 0;
}

// the swizzled transposition: one place per piece, and a warp's writes and reads spread over the banks
static int transposition() {
  std::set<int> places;
  for (int r = 0; r < 128; ++r)
    for (int k = 0; k < 16; ++k) {
      const int at = kb::transposed_at(r, k);
      CHECK(at % 8 == 0 && at / 128 == r, "row %d, piece %d at %d", r, k, at);
      places.insert(at);
    }
  CHECK(places.size() == 128 * 16, "%zu places", places.size());
  for (int j = 0; j < 8; ++j)
    for (int ry = 0; ry < 16; ry += 2) {   // a warp writes one 8-byte piece per thread: two passes of 32 words
      int words[32] = {};
      for (int cx = 0; cx < 16; ++cx)
        for (int h = 0; h < 2; ++h) ++words[kb::transposed_at(cx * 8 + j, ry + h) / 4 % 32];
      for (int w : words) CHECK(w == 0 || w == 2, "column %d, piece %d: %d writes to a bank", j, ry, w);
    }
  return 0;
}

// a group of 256 columns goes to 32 lanes of 8, whole blocks of 128 to half of a lane set each
static int groups() {
  std::set<uint32_t> vec, plain;
  for (int lane = 0; lane < 32; ++lane)
    for (int j = 0; j < 8; ++j) {
      const uint32_t a = kb::group_col<true>(3, lane, j), b = kb::group_col<false>(3, lane, j);
      vec.insert(a);
      plain.insert(b);
      CHECK(a / 128 == 6u + (lane >> 4), "lane %d", lane);      // lanes 0..15 hold the first block
      CHECK(b / 128 == 6u + (j >> 2), "element %d", j);         // elements 0..3 of every lane hold it
    }
  CHECK(vec.size() == 256 && plain.size() == 256 && *vec.begin() == 768 && *plain.begin() == 768, "%zu", vec.size());
  return 0;
}

int main() {
  static_assert(kb::PairTile::kSmem + sizeof(float) * kb::PairTile::kScaleSlots * kb::kScaleStep * (128 + 256) < 227 * 1024, "");
  if (tiles() || clusters<16>() || clusters<32>() || clusters<64>() || clusters<128>() || transposition() || groups()) return 1;
  std::puts("ok");
  return 0;
}

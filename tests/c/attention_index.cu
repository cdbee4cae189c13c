// The index functions of the attention kernels, called on the host: no GPU, no kernel is launched.
#include <cstdio>
#include <set>
#include <vector>

#include "kb_paged.cuh"
#include "kb_prompt.cuh"
#include "kb_rope.cuh"

#define CHECK(cond, ...)                                  \
  do {                                                    \
    if (!(cond)) {                                        \
      std::printf("%s:%d: %s: ", __FILE__, __LINE__, #cond); \
      std::printf(__VA_ARGS__);                           \
      std::printf("\n");                                  \
      return 1;                                           \
    }                                                     \
  } while (0)

// a row of units is divided without gap or overlap, no piece is empty, and each unit knows its piece
static int pieces() {
  for (uint32_t n : {1u, 2u, 7u, 36u, 37u, 148u, 149u, 1000u, 32768u, 2147483647u})
    for (uint32_t most : {1u, 2u, 18u, 37u, 148u, 296u, 444u}) {
      const kb::PagedPieces p(n, most);
      CHECK(p.count >= 1 && p.count <= most && p.count <= n, "%u in %u: %u", n, most, p.count);
      CHECK(p.first(0) == 0 && p.first(p.count) == n, "%u in %u", n, most);
      const uint32_t longest = (uint32_t)(((uint64_t)n + most - 1) / most);
      for (uint32_t c = 0; c < p.count; ++c) {
        const uint32_t a = p.first(c), b = p.first(c + 1);
        CHECK(b > a && b - a <= longest, "%u in %u, piece %u: %u to %u", n, most, c, a, b);
        CHECK(p.of(a) == c && p.of(b - 1) == c, "%u in %u, piece %u", n, most, c);
      }
    }
  CHECK(kb::paged_length(-5, 4, 16) == 0 && kb::paged_length(0, 4, 16) == 0 && kb::paged_length(65, 4, 16) == 64, "lengths");
  CHECK(kb::paged_length(0x7FFFFFFF, 0xFFFFFFFFu, 0xFFFFFFFFu) == 0x7FFFFFFFu, "lengths past 32 bits");
  CHECK(kb::paged_units(0, 128) == 1 && kb::paged_units(128, 128) == 1 && kb::paged_units(129, 128) == 2 && kb::paged_units(65, 64) == 2, "units");
  return 0;
}

// kappa is a permutation of 8 keys, and the 8 lanes of each phase of a warp's 16-byte reads from swizzled rows (lane
// (g, t) = (lane / 4, lane % 4)) touch 8 different groups of banks
static int banks() {
  std::set<uint32_t> keys;
  for (uint32_t g = 0; g < 8; ++g) keys.insert(kb::paged_kappa(g));
  CHECK(keys.size() == 8 && *keys.rbegin() == 7, "%zu keys", keys.size());
  for (uint32_t phase = 0; phase < 4; ++phase)
    for (uint32_t half = 0; half < 2; ++half) {
      std::set<uint32_t> k;
      for (uint32_t lane = 8 * phase; lane < 8 * phase + 8; ++lane) k.insert((half * 4 + lane % 4) ^ (kb::paged_kappa(lane / 4) & 7));
      CHECK(k.size() == 8, "keys, phase %u, half %u: %zu", phase, half, k.size());
    }
  for (uint32_t odd = 0; odd < 2; ++odd)   // values of the keys kappa(2 t) and kappa(2 t + 1)
    for (uint32_t phase = 0; phase < 4; ++phase) {
      std::set<uint32_t> v;
      for (uint32_t lane = 8 * phase; lane < 8 * phase + 8; ++lane) v.insert((lane / 4) ^ (kb::paged_kappa(2 * (lane % 4) + odd) & 7));
      CHECK(v.size() == 8, "values, phase %u: %zu", phase, v.size());
    }
  return 0;
}

// steps and seen keys against a count of the pairs themselves
static int prompts() {
  for (uint32_t nq : {1u, 5u, 128u, 130u, 300u})
    for (uint32_t nk : {0u, 1u, 63u, 64u, 129u, 300u, 700u})
      for (int causal = 0; causal < 2; ++causal)
        for (uint32_t row = 0; row < nq; row += 128) {
          uint32_t most = 0;
          for (uint32_t i = row; i < nq && i < row + 128; ++i) {
            uint32_t seen = 0;
            for (uint32_t j = 0; j < nk; ++j) seen += !causal || (long long)j - i <= (long long)nk - nq;
            CHECK(kb::prompt_seen(i, nq, nk, causal) == seen, "query %u of %u, %u keys", i, nq, nk);
            if (seen > most) most = seen;
          }
          CHECK(kb::prompt_steps(row, 128, nq, nk, causal) == (most + kb::kPromptKeys - 1) / kb::kPromptKeys, "piece at %u of %u, %u keys", row, nq, nk);
        }
  CHECK(kb::prompt_steps(128, 128, 128, 500, true) == 0, "a piece past the end");
  return 0;
}

// a frequency's part of a turn, in units of 2^-64
static int turns() {
  const double two_pi = 6.283185307179586;
  CHECK(kb::rope_turn(0.0) == 0, "0");
  CHECK(kb::rope_turn(two_pi / 2) >> 40 == 1ull << 23 || (kb::rope_turn(two_pi / 2) >> 40) + 1 == 1ull << 23, "half a turn");
  for (double f : {1.0, 0.25, -0.25, 1e-4, 7.5, -100.0, 1e-30}) {
    const double t = f / two_pi, part = t - std::floor(t), got = (double)kb::rope_turn(f) / 18446744073709551616.0;
    CHECK(std::fabs(got - part) < 1e-14 || std::fabs(got - part) > 1 - 1e-14, "%g: %g, not %g", f, got, part);
  }
  return 0;
}

int main() {
  if (pieces() || banks() || prompts() || turns()) return 1;
  std::puts("ok");
  return 0;
}

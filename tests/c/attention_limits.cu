// Steps and seen keys at the largest sizes that the call accepts, on the host, against 64-bit arithmetic.
#include <cstdio>

#include "kb_prompt.cuh"

int main() {
  const uint32_t most_q = 1u << 30, most_k = kb::kPromptMostKeys;
  for (uint32_t nq : {1u, 130u, most_k, most_q - 1, most_q})
    for (uint32_t nk : {0u, 1u, 64u, most_k - 1, most_k})
      for (uint32_t row : {0u, nq / 2, nq > 200 ? nq - 200 : 0u, nq - 1}) {
        const long long seen = (long long)row + 1 + nk - nq, last = (long long)(row + 128 < nq ? row + 128 : nq) + nk - nq;
        const uint32_t want = seen <= 0 ? 0u : seen < nk ? (uint32_t)seen : nk;
        const uint32_t steps = last <= 0 ? 0u : (uint32_t)(((last < nk ? last : (long long)nk) + kb::kPromptKeys - 1) / kb::kPromptKeys);
        if (kb::prompt_seen(row, nq, nk, true) != want || kb::prompt_steps(row, 128, nq, nk, true) != steps) {
          std::printf("query %u of %u, %u keys: %u and %u, not %u and %u\n", row, nq, nk, kb::prompt_seen(row, nq, nk, true),
                      kb::prompt_steps(row, 128, nq, nk, true), want, steps);
          return 1;
        }
      }
  std::puts("ok");
  return 0;
}

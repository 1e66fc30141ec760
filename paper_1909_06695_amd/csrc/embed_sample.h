// Where a sample of 64 of N ids is taken: one of each 64th, in each at another place (multiples of the golden ratio).  At equal distances a batch whose
// streams divide them would show its first tokens alone, or none of its padding.
#pragma once
#include <cstdint>

namespace ouro {

constexpr int es_sample_at(int lane, int N) {
  return (int)((int64_t)lane * N / 64) + (int)((uint64_t)((uint32_t)lane * 0x9e3779b1u) * (uint32_t)(N / 64) >> 32);
}

}  // namespace ouro

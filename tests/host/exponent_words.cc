// The words that a cache's exponent bytes are copied by (csrc/wk_internal.cuh), for every byte of arrays of n.
#include "wk_internal.cuh"

// 0: every word holds its byte and lies in the array; otherwise the first byte + 1 whose word does not
extern "C" uint32_t exponent_words(uint32_t n, uint32_t from, uint32_t count) {
  for (uint32_t k = 0; k < count; ++k) {
    const uint32_t i = from + k;
    const wk::ByteWord w = wk::word_of_byte(i, n);
    if (w.at % 4 || w.bytes < 1 || w.bytes > 4 || w.at > i || i >= static_cast<uint64_t>(w.at) + w.bytes ||
        static_cast<uint64_t>(w.at) + w.bytes > n)
      return i + 1;
  }
  return 0;
}

// Which page of a table a chunk of 32 tokens lies in: chunk / (chunks of a page), without a division.
#pragma once
#include <cstdint>

namespace dfp4 {

// With L the least number for which chunks <= 2^L, per = 2^(31 + L) / chunks, rounded up, is at least 2^31 and less than 2^32, and
// chunk * per >> (31 + L) is chunk / chunks rounded down: per is too large by e < 1, and chunk * chunks * e < 2^31 * 2^L.
struct PageDivision {
    uint32_t per, shift;
};
constexpr PageDivision page_division(uint32_t chunks) {
    uint32_t shift = 0;
    while (((uint32_t)1 << shift) < chunks) ++shift;
    return PageDivision{(uint32_t)((((uint64_t)1 << (31 + shift)) + chunks - 1) / chunks), shift};
}
// 0 <= chunk < 2^31
constexpr int page_of(const PageDivision& by, int chunk) {
    return (int)((uint32_t)((uint64_t)(2u * (uint32_t)chunk) * by.per >> 32) >> by.shift);
}

}  // namespace dfp4

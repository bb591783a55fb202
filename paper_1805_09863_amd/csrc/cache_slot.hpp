// The slot of a new token in the attention cache.
#pragma once

#include <stdint.h>

namespace kb {

// Of a token whose length, its own slot included, is `len` in a table of `cap` slots; -1: it is not stored.
// Both bounds come before the subtraction: the lowest int32 less one is past every table.
constexpr int32_t new_slot(int32_t len, int32_t cap) { return len < 1 || len > cap ? -1 : len - 1; }

}  // namespace kb

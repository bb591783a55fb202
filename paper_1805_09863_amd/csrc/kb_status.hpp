// What every entry point returns through: the status and the calling thread's
// error text (kb_last_error).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "kbest.h"

namespace kb {

kb_status fail(kb_status status, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
kb_status ok();  // clears the text
const char* last_error();

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

}  // namespace kb

// What the files that implement include/pblock.h share.
#pragma once

#include "pblock.h"

namespace pb {

// Sets pblock_last_error() of this thread and returns st.
pb_status fail(pb_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
void clear_error();
// PB_OK and no error text, or what hipGetLastError() says.
pb_status finish_launches();

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

}  // namespace pb

// Token ids of the types programs hold them in (mb_token_type).
#pragma once

#include <stdint.h>

#include "../../include/mbscan.h"

namespace mbscan {

// Token i, or -1 for one outside [0, vocab).
__device__ __forceinline__ int load_token(const void *tokens, int type, int64_t i, int vocab) {
    int64_t t;
    if (type == MB_TOKEN_U8) t = static_cast<const uint8_t *>(tokens)[i];
    else if (type == MB_TOKEN_I32) t = static_cast<const int32_t *>(tokens)[i];
    else t = static_cast<const int64_t *>(tokens)[i];
    return t >= 0 && t < vocab ? (int)t : -1;
}

}  // namespace mbscan
